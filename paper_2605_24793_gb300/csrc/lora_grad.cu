// Gradients of the adapters' factors (cospec_lora_backward): sums over the rows m of one adapter,
//   dA_a[j][k] = sum_m t[m][j] drop(x)[m][k]        dB_a[n][j] = sum_m u[m][j] dy[m][n]
// Both are P^T Q with P fp32 [rows, rank] and Q bf16 [rows, width], and both are one launch: the column blocks of x
// come first, then those of dy.  Bound by reading x and dy once each.
//
// mma.sync with the rank as M, columns of Q as N and the rows as the contraction.  P enters as three
// bf16 parts, which hold all 24 bits of it, so the sums are those of fp32 products (a gradient that is
// summed over micro-batches starts from fp32).
//
// A CTA takes 256 columns of one adapter, 32 a warp; the adapter's rows, listed in shared memory first, so that rows
// of other adapters and what they hold are not read, come 32 at a time: Q by cp.async into a ring, P through
// registers, where it is split once for all warps.  A thread masks the 16-byte chunks of x that it copied itself, each one
// draw of the generator.  The rows are split over the CTAs of a cluster and joined in a fixed order.
#include "lora.cuh"

namespace cospec {

namespace {

constexpr int GRAD_THREADS = 256;
constexpr int CB = 256;              // columns of a CTA
constexpr int BR = 32;               // rows of a batch
constexpr int GDEPTH = 4;            // batches in the ring
constexpr int WIN = 2048;            // rows listed at a time
constexpr uint32_t Q_BYTES = BR * CB * 2;

struct GradArgs {
  const __nv_bfloat16 *x, *dy;
  const float *t, *u;
  long long ldx, ldy;
  int K, N;                          // widths; 0 where the gradient is not wanted
  float *da, *db;                    // [n][r][K], [n][N][r]
  int blocks0;                       // column blocks of x
  const int32_t* adapter;
  int M, r;
  int accumulate;
  LoraDrop drop;
};

struct GradSmem {
  int list[WIN];
  int warp_count[8];
};
// the ring of Q, two buffers of P's parts [3][BR rows][R], the list; then the sums, [R][CB + 8] or [CB][R + 4]
__host__ __device__ constexpr uint32_t grad_p_bytes(int R) { return (uint32_t)(3 * BR * R * 2); }
__host__ __device__ constexpr uint32_t grad_bytes(int R) {
  return GDEPTH * Q_BYTES + 2 * grad_p_bytes(R) + (uint32_t)sizeof(GradSmem);
}

template <int RT>
__global__ void __launch_bounds__(GRAD_THREADS) lora_grad_kernel(const GradArgs p) {
  extern __shared__ __align__(128) uint8_t raw[];
  constexpr int R = 16 * RT;
  constexpr int PV = BR * R / GRAD_THREADS;            // values of P a thread splits per batch
  constexpr uint32_t P_PART = (uint32_t)(BR * R * 2);
  GradSmem& sm = *reinterpret_cast<GradSmem*>(raw + GDEPTH * Q_BYTES + 2 * grad_p_bytes(R));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int S = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
  const int block = (int)blockIdx.x / S, which = block >= p.blocks0;
  const int c0 = (which ? block - p.blocks0 : block) * CB;
  const int a = (int)blockIdx.y;
  const __nv_bfloat16* Q = which ? p.dy : p.x;
  const float* P = which ? p.u : p.t;
  const long long ld = which ? p.ldy : p.ldx;
  const int width = which ? p.N : p.K;
  const bool drop = which == 0 && p.drop.thr != 0u;
  const uint32_t q0 = smem_u32(raw), p0 = q0 + GDEPTH * Q_BYTES;
  griddep_wait();
  griddep_launch_dependents();
  LoraKey key{0, 0};
  if (drop) key = lora_key(p.drop);

  float acc[RT][4][4];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][c][e] = 0.f;

  // 512-byte rows of Q, 2 R byte rows of P; the 16-byte chunks exchanged by the row, so that eight neighbouring rows lie
  // on different banks
  auto p_at = [&](int row, int c) {
    const int sw = RT >= 4 ? row & 7 : RT == 2 ? (row >> 1) & 3 : (row >> 2) & 1;
    return (uint32_t)(row * (R * 2) + ((c ^ sw) << 4));
  };
  const int m_lo = (int)((long long)p.M * rank / S), m_hi = (int)((long long)p.M * (rank + 1) / S);
  for (int w0 = m_lo; w0 < m_hi; w0 += WIN) {
    // the adapter's rows of the window, in order
    const int w1 = min(w0 + WIN, m_hi);
    int have = 0;
    for (int b = w0; b < w1; b += GRAD_THREADS) {
      const int m = b + tid;
      const bool in = m < w1 && p.adapter[m] == a;
      const unsigned mask = __ballot_sync(0xffffffffu, in);
      if (lane == 0) sm.warp_count[warp] = __popc(mask);
      __syncthreads();
      int at = have + __popc(mask & ((1u << lane) - 1u));
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const int c = sm.warp_count[w];
        if (w < warp) at += c;
        have += c;
      }
      if (in) sm.list[at] = m;
      __syncthreads();
    }
    const int batches = (have + BR - 1) / BR;
    // chunk i of a batch's Q: row (tid + 256 i) / 32, columns 8 (tid mod 32) ..
    const int qc = tid & 31, col = c0 + 8 * qc;
    auto load_q = [&](int b) {
      if (b < batches) {
        const uint32_t dst = q0 + (uint32_t)(b & (GDEPTH - 1)) * Q_BYTES;
#pragma unroll
        for (int i = 0; i < BR / 8; ++i) {
          const int row = (tid >> 5) + 8 * i;
          const bool on = b * BR + row < have && col < width;
          cp_async16(dst + (uint32_t)(row * 512 + ((qc ^ (row & 7)) << 4)), on ? Q + (long long)sm.list[b * BR + row] * ld + col : Q, on);
        }
      }
      cp_async_commit();
    };
    // value i of a batch's P: pairs along the rank, (tid + 256 i) counts pairs
    float2 pv[PV / 2];
    auto load_p = [&](int b) {
#pragma unroll
      for (int i = 0; i < PV / 2; ++i) {
        const int e = tid + GRAD_THREADS * i, row = e / (R / 2), j = 2 * (e % (R / 2));
        pv[i] = make_float2(0.f, 0.f);
        if (b * BR + row < have && j < p.r) pv[i] = __ldg(reinterpret_cast<const float2*>(P + (size_t)sm.list[b * BR + row] * p.r + j));
      }
    };
    auto store_p = [&](int b) {
      const uint32_t dst = (uint32_t)(b & 1) * grad_p_bytes(R);
#pragma unroll
      for (int i = 0; i < PV / 2; ++i) {
        const int e = tid + GRAD_THREADS * i, row = e / (R / 2), j = 2 * (e % (R / 2));
        float x = pv[i].x, y = pv[i].y;
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          float hx, lx, hy, ly;
          lora_split2(x, hx, lx);
          lora_split2(y, hy, ly);
          *reinterpret_cast<uint32_t*>(raw + GDEPTH * Q_BYTES + dst + k * P_PART + p_at(row, j >> 3) + (j & 7) * 2) = pack_bf16(hx, hy);
          x = lx;
          y = ly;
        }
      }
    };
#pragma unroll
    for (int i = 0; i < GDEPTH - 1; ++i) load_q(i);
    load_p(0);
    for (int b = 0; b < batches; ++b) {
      store_p(b);
      cp_async_wait<GDEPTH - 2>();
      const uint32_t qb = q0 + (uint32_t)(b & (GDEPTH - 1)) * Q_BYTES;
      if (drop) {
#pragma unroll 2
        for (int i = 0; i < BR / 8; ++i) {
          const int row = (tid >> 5) + 8 * i;
          if (b * BR + row >= have) break;
          uint4* q = reinterpret_cast<uint4*>(raw + (qb - q0) + row * 512 + ((qc ^ (row & 7)) << 4));
          *q = lora_dropped8(*q, (uint32_t)(col >> 3), (uint32_t)sm.list[b * BR + row], p.drop, key);
        }
      }
      __syncthreads();
      load_q(b + GDEPTH - 1);
      if (b + 1 < batches) load_p(b + 1);
      const uint32_t pb = p0 + (uint32_t)(b & 1) * grad_p_bytes(R);
      const int steps = min(BR / 16, (have - b * BR + 15) / 16);
      for (int ks = 0; ks < steps; ++ks) {
        const int row = ks * 16 + (lane & 15);
        uint32_t bq[4][2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {      // 16 columns: (k 0-7, 8-15) of the first eight, then of the others
          const int cc = warp * 4 + 2 * c + (lane >> 4);
          ldsm_x4_t(qb + (uint32_t)(row * 512 + ((cc ^ (row & 7)) << 4)), bq[2 * c][0], bq[2 * c][1], bq[2 * c + 1][0], bq[2 * c + 1][1]);
        }
        // the rank's blocks: (ranks 0-7, k 0-7), (8-15, 0-7), (0-7, 8-15), (8-15, 8-15), stored with k along the rows
        const int pr = ks * 16 + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            uint32_t pa[4];
            ldsm_x4_t(pb + (uint32_t)k * P_PART + p_at(pr, 2 * i + ((lane >> 3) & 1)), pa[0], pa[1], pa[2], pa[3]);
#pragma unroll
            for (int c = 0; c < 4; ++c) mma_16816(acc[i][c], pa, bq[c][0], bq[c][1]);
          }
      }
    }
    cp_async_wait<0>();
    __syncthreads();                       // the list and the ring are read
  }

  float* red = reinterpret_cast<float*>(raw);
  constexpr int LA = CB + 8, LB = R + 4;
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = warp * 32 + c * 8 + 2 * t + (e & 1), j = 16 * i + g + 8 * (e >> 1);
        red[which ? n * LB + j : j * LA + n] = acc[i][c][e];
      }
  __syncthreads();
  __syncwarp();
  cluster_arrive();
  cluster_wait();
  const uint32_t base = smem_u32(red);
  const int e0 = CB * R * rank / S, e1 = CB * R * (rank + 1) / S;
  float* out = which ? p.db : p.da;
  for (int e = e0 + tid; e < e1; e += GRAD_THREADS) {
    const int n = which ? e / R : e % CB, j = which ? e % R : e / CB;
    if (c0 + n >= width || j >= p.r) continue;
    const uint32_t at = base + 4u * (uint32_t)(which ? n * LB + j : j * LA + n);
    const float s = dsmem_sum(at, S);
    float* o = which ? out + ((size_t)a * width + c0 + n) * p.r + j : out + ((size_t)a * p.r + j) * width + c0 + n;
    *o = p.accumulate ? *o + s : s;
  }
  __syncwarp();
  cluster_arrive();
  cluster_wait();
}

template <int RT>
cudaError_t launch_grad(const GradArgs& p, int blocks, int n, int splits, cudaStream_t stream) {
  static KernelLimits lim;
  constexpr int R = 16 * RT;
  size_t smem = grad_bytes(R);
  const size_t red = (size_t)(R * (CB + 8) > CB * (R + 4) ? R * (CB + 8) : CB * (R + 4)) * sizeof(float);
  if (smem < red) smem = red;
  const cudaError_t e = ensure_kernel_limits((const void*)lora_grad_kernel<RT>, lim, smem, false);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(blocks * splits), (unsigned)n);
  cfg.blockDim = dim3(GRAD_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, lora_grad_kernel<RT>, p);
}

}  // namespace

cudaError_t launch_lora_grad(const LoraArgs& a, int num_sms, cudaStream_t stream) {
  GradArgs p{};
  p.x = a.x, p.dy = a.dy;
  p.t = a.t, p.u = a.u;
  p.ldx = a.ldx, p.ldy = a.ldy;
  p.K = a.da ? a.K : 0, p.N = a.db ? a.N : 0;
  p.da = a.da, p.db = a.db;
  p.blocks0 = (p.K + CB - 1) / CB;
  p.adapter = a.adapter;
  p.M = a.M;
  p.r = a.r;
  p.accumulate = a.accumulate;
  p.drop = LoraDrop{a.seed, a.site, a.thr};
  const int blocks = p.blocks0 + (p.N + CB - 1) / CB;
  if (blocks == 0) return cudaSuccess;
  // a split has at least four batches
  int splits = 1;
  while (splits < 8 && (long long)blocks * a.n * splits < num_sms && a.M >= 8 * BR * splits) splits *= 2;
  if (a.r <= 16) return launch_grad<1>(p, blocks, a.n, splits, stream);
  if (a.r <= 32) return launch_grad<2>(p, blocks, a.n, splits, stream);
  if (a.r <= 64) return launch_grad<4>(p, blocks, a.n, splits, stream);
  return launch_grad<8>(p, blocks, a.n, splits, stream);
}

}  // namespace cospec
