// Gradients of the adapters' factors (cospec_lora_backward): sums over the rows m of one adapter,
//   dA_a[j][k] = sum_m t[m][j] drop(x)[m][k]        dB_a[n][j] = sum_m u[m][j] dy[m][n]
// Both are P^T Q with P fp32 [rows, rank] and Q bf16 [rows, width], and both are one launch: the column blocks of x
// come first, then those of dy.  Bound by reading x and dy once each.
//
// mma.sync with the rank as M, columns of Q as N and the rows as the contraction.  P enters as three
// bf16 parts, which hold all 24 bits of it, so the sums are those of fp32 products (a gradient that is
// summed over micro-batches starts from fp32).  A lane loads 16 bytes of a row of Q, and movmatrix turns the 8 x 8
// blocks into fragments; the order of the columns inside a block of 32 that comes of it is undone when
// the sums are written.  A lane's 16 bytes are one draw of the dropout mask.
//
// A CTA takes 128 columns of one adapter (and 64 of its ranks); the rows are split over the CTAs of a cluster
// and four row groups of warps and joined in a fixed order.  The rows of the adapter are listed in shared memory
// first, so rows of other adapters, and what they hold, are not read.
#include "lora.cuh"

namespace cospec {

namespace {

constexpr int GRAD_THREADS = 256;
constexpr int CB = 128;              // columns of a CTA
constexpr int WIN = 2048;            // rows listed at a time

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
  int count;
};

template <int RT>
__global__ void __launch_bounds__(GRAD_THREADS) lora_grad_kernel(const GradArgs p) {
  extern __shared__ __align__(16) uint8_t raw[];
  GradSmem& sm = *reinterpret_cast<GradSmem*>(raw);
  float* red = reinterpret_cast<float*>(raw + (sizeof(GradSmem) + 15) / 16 * 16);   // [4 warps][64 columns][16 RT]
  constexpr int R = 16 * RT;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int S = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
  const int block = (int)blockIdx.x / S, which = block >= p.blocks0;
  const int c0 = (which ? block - p.blocks0 : block) * CB;
  const int a = (int)blockIdx.y, j0 = (int)blockIdx.z * 64;
  const int cw = c0 + (warp & 1) * 64, rg = warp >> 1;       // the warp's columns and row group
  const __nv_bfloat16* Q = which ? p.dy : p.x;
  const float* P = which ? p.u : p.t;
  const long long ld = which ? p.ldy : p.ldx;
  const int width = which ? p.N : p.K;
  const bool drop = which == 0 && p.drop.thr != 0u;
  griddep_wait();
  griddep_launch_dependents();
  LoraKey key{0, 0};
  if (drop) key = lora_key(p.drop);

  float acc[RT][8][4];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][c][e] = 0.f;

  const int m_lo = (int)((long long)p.M * rank / S), m_hi = (int)((long long)p.M * (rank + 1) / S);
  for (int w0 = m_lo; w0 < m_hi; w0 += WIN) {
    // the adapter's rows of the window, in order
    const int w1 = min(w0 + WIN, m_hi);
    int have = 0;
    __syncthreads();                     // the list before is read
    for (int b = w0; b < w1; b += GRAD_THREADS) {
      const int m = b + (int)threadIdx.x;
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
    for (int b = rg * 16; b < have; b += 64) {
      // rows of the fragments: loads by the lane's row g (and g + 8), products by 2 t, 2 t + 1 (and + 8)
      uint4 v[2][2];
      int row[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        row[h] = b + g + 8 * h < have ? sm.list[b + g + 8 * h] : -1;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int col = cw + 32 * c + 8 * t;
          v[h][c] = make_uint4(0, 0, 0, 0);
          if (row[h] >= 0 && col < width) v[h][c] = ldg16(Q + (long long)row[h] * ld + col);
        }
      }
      uint32_t pa[RT][3][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {       // rows 8 h + 2 t, + 1
        const int i0 = b + 8 * h + 2 * t;
        const int m0 = i0 < have ? sm.list[i0] : -1, m1 = i0 + 1 < have ? sm.list[i0 + 1] : -1;
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int j = j0 + 16 * i + 8 * e + g;
            float x = m0 >= 0 && j < p.r ? __ldg(P + (size_t)m0 * p.r + j) : 0.f;
            float y = m1 >= 0 && j < p.r ? __ldg(P + (size_t)m1 * p.r + j) : 0.f;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
              float hx, lx, hy, ly;
              lora_split2(x, hx, lx);
              lora_split2(y, hy, ly);
              pa[i][k][2 * h + e] = pack_bf16(hx, hy);
              x = lx;
              y = ly;
            }
          }
      }
      if (drop) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int c = 0; c < 2; ++c)
            v[h][c] = and4(v[h][c], lora_keep8((uint32_t)((cw + 32 * c) / 8 + t), (uint32_t)row[h], p.drop, key));
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t lo[4] = {v[0][c].x, v[0][c].y, v[0][c].z, v[0][c].w}, hi[4] = {v[1][c].x, v[1][c].y, v[1][c].z, v[1][c].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t b0 = movmatrix_t(lo[q]), b1 = movmatrix_t(hi[q]);
#pragma unroll
          for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int k = 0; k < 3; ++k) mma_16816(acc[i][4 * c + q], pa[i][k], b0, b1);
        }
      }
    }
  }

  // Row groups 2, 3 into 0, 1, then 1 into 0.  A buffer holds a warp's sums as [column][rank]; its column of
  // block c of 32, group q, fragment column 2 t + e is 32 c + 8 t + 2 q + e.
  auto each = [&](auto&& f) {
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int col = 32 * (c >> 2) + 8 * t + 2 * (c & 3) + (e & 1), j = 16 * i + g + 8 * (e >> 1);
          f(col * R + j, acc[i][c][e]);
        }
  };
#pragma unroll
  for (int half = 2; half >= 1; half >>= 1) {
    __syncthreads();
    if (rg >= half && rg < 2 * half) each([&](int at, float& x) { red[((rg - half) * 2 + (warp & 1)) * 64 * R + at] = x; });
    __syncthreads();
    if (rg < half) each([&](int at, float& x) { x += red[(rg * 2 + (warp & 1)) * 64 * R + at]; });
  }
  __syncthreads();
  if (rg == 0) each([&](int at, float& x) { red[(warp & 1) * 64 * R + at] = x; });       // [CB columns][R]
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  const uint32_t base = smem_u32(red);
  const int e0 = CB * R * rank / S, e1 = CB * R * (rank + 1) / S;
  float* out = which ? p.db : p.da;
  for (int e = e0 + (int)threadIdx.x; e < e1; e += GRAD_THREADS) {
    // dB: [column][rank] as it stands; dA: neighbouring threads take neighbouring columns
    int col, j;
    if (which) {
      col = e / R, j = e % R;
    } else {
      col = e % CB, j = e / CB;
    }
    if (c0 + col >= width || j0 + j >= p.r) continue;
    float s = 0.f;
    for (int i = 0; i < S; ++i) {
      float w;
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(w) : "r"(dsmem_map(base + 4u * (uint32_t)(col * R + j), (uint32_t)i)) : "memory");
      s += w;
    }
    float* o = which ? out + ((size_t)a * width + c0 + col) * p.r + j0 + j : out + ((size_t)a * p.r + j0 + j) * width + c0 + col;
    *o = p.accumulate ? *o + s : s;
  }
  __syncwarp();
  cluster_arrive();
  cluster_wait();
}

template <int RT>
cudaError_t launch_grad(const GradArgs& p, int blocks, int n, int chunks, int splits, cudaStream_t stream) {
  static KernelLimits lim;
  const size_t smem = (sizeof(GradSmem) + 15) / 16 * 16 + (size_t)4 * 64 * 16 * RT * sizeof(float);
  const cudaError_t e = ensure_kernel_limits((const void*)lora_grad_kernel<RT>, lim, smem, false);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(blocks * splits), (unsigned)n, (unsigned)chunks);
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
  // a split has at least 64 rows: a block of 16 for each row group
  const int chunks = (a.r + 63) / 64;
  int splits = 1;
  while (splits < 8 && (long long)blocks * a.n * chunks * splits < 2 * num_sms && a.M >= 128 * splits) splits *= 2;
  if (a.r <= 16) return launch_grad<1>(p, blocks, a.n, chunks, splits, stream);
  if (a.r <= 32) return launch_grad<2>(p, blocks, a.n, chunks, splits, stream);
  return launch_grad<4>(p, blocks, a.n, chunks, splits, stream);
}

}  // namespace cospec
