// The low-rank sides of the adapters (cospec_lora_forward, cospec_lora_backward):
//   forward   u[m][j] = c_a sum_k drop(x)[m][k] A_a[j][k]      A_a [rank, in]: the factor's rows run along k
//   backward  t[m][j] = c_a sum_n dy[m][n] B_a[n][j]           B_a [out, rank]: its rows run along j
// with a the row's adapter and c_a = scaling[a] / (1 - p); rows without one get zeros.  Both are fp32,
// and both are bound by reading x or dy once (and, for a few rows, by the latency of one read of the factor).
//
// Two kernels.  low_mma_kernel: warps of 16 rows on mma.sync; every operand goes from global memory to the
// fragments by 16-byte loads, without shared memory, because the order of the contraction inside a
// product of 32 is free: lane t of a quad takes elements 8t .. 8t + 7 of both operands.  A factor whose rows run
// along the rank is turned by movmatrix.  Rows of several adapters in one warp: the warp goes over
// the adapters and zeroes the other rows' elements, so that all of them add into one accumulator.  The contraction
// is split over the warps of a CTA and the CTAs of a cluster, joined in shared memory in a fixed order.
// low_row_kernel, for a few rows (rows x rank <= LOW_ROW_MAX): a CTA per row, which reads its adapter's factor
// in one wave of loads; 16 rows of as many adapters would keep one warp of the other kernel busy for 16
// round trips to memory.
//
// Dropout: a lane's eight elements of a row are one draw of the generator.
#include "lora.cuh"

namespace cospec {

namespace {

constexpr int LOW_THREADS = 256;
constexpr int LOW_ROW_MAX = 2048;
constexpr int ROW_THREADS = 512;

struct LowArgs {
  const __nv_bfloat16* x;
  long long ldx;
  const __nv_bfloat16* f;
  const float* scaling;
  const int32_t* adapter;
  float* u;
  int M, C, r, n;       // C: the contraction's length
  float keep_inv;       // 1 / (1 - p)
  LoraDrop drop;
  int rw_log2;          // log2 of the row groups of a CTA
  int* err;
};

// NT: rank in groups of 8, rounded up to 2, 4, 8 or 16.  The rank that column 2 t + e of group nt stands for
// follows from how the factor is loaded.
template <int NT, bool RM>
CS_DEV int low_rank_of(int nt, int col) {
  const int t = col >> 1, e = col & 1;
  if (!RM) return nt * 8 + col;
  if (NT == 2) return 4 * t + 2 * nt + e;
  return 32 * (nt >> 2) + 8 * t + 2 * (nt & 3) + e;
}

template <int NT, bool RM>
__global__ void __launch_bounds__(LOW_THREADS) low_mma_kernel(const LowArgs p) {
  extern __shared__ float red[];        // [8 warps][16][NT * 8]
  constexpr int R = NT * 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int S = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
  const int tile = (int)blockIdx.x / S;
  const int RW = 1 << p.rw_log2, KW = 8 >> p.rw_log2;
  const int rw = warp & (RW - 1), kw = warp >> p.rw_log2;
  const long long m0 = ((long long)tile * RW + rw) * 16;
  griddep_wait();
  griddep_launch_dependents();

  const int steps = (p.C + 31) / 32, parts = S * KW, part = rank * KW + kw;
  const int s0 = (int)((long long)steps * part / parts), s1 = (int)((long long)steps * (part + 1) / parts);
  int mine = -1;
  if (lane < 16 && m0 + lane < p.M) mine = lora_adapter(p.adapter, (int)m0 + lane, p.n, p.err);
  unsigned todo = __ballot_sync(0xffffffffu, mine >= 0);
  const bool drop = p.drop.thr != 0u;
  LoraKey key{0, 0};
  if (drop) key = lora_key(p.drop);

  float acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;

  while (todo) {
    const int a = __shfl_sync(0xffffffffu, mine, __ffs(todo) - 1);
    const unsigned who = __ballot_sync(0xffffffffu, mine == a) & 0xffffu;
    todo &= ~who;
    const bool on0 = (who >> g) & 1u, on1 = (who >> (g + 8)) & 1u;
    const __nv_bfloat16* x0 = p.x + (m0 + g) * p.ldx;
    const __nv_bfloat16* x1 = p.x + (m0 + g + 8) * p.ldx;
    const __nv_bfloat16* f = p.f + (size_t)a * p.r * p.C;
#pragma unroll 2
    for (int s = s0; s < s1; ++s) {
      const int k = s * 32 + 8 * t;
      const bool in = k < p.C;
      uint4 a0 = make_uint4(0, 0, 0, 0), a1 = a0;
      if (on0 && in) a0 = ldg16(x0 + k);
      if (on1 && in) a1 = ldg16(x1 + k);
      uint32_t b[NT][4];
      if (!RM) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const int j = i * 8 + g;
          uint4 v = make_uint4(0, 0, 0, 0);
          if (j < p.r && in) v = ldg16(f + (size_t)j * p.C + k);
          b[i][0] = v.x, b[i][1] = v.y, b[i][2] = v.z, b[i][3] = v.w;
        }
      } else {
        // matrix q: its rows 2 t + e are the contraction's elements 8 t + 2 q + e
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int kk = s * 32 + 8 * (g >> 1) + 2 * q + (g & 1);
          const bool kin = kk < p.C;
          const __nv_bfloat16* row = f + (size_t)kk * p.r;
          if constexpr (NT == 2) {
            uint2 v = make_uint2(0, 0);
            if (kin && 4 * t < p.r) v = __ldg(reinterpret_cast<const uint2*>(row + 4 * t));
            b[0][q] = v.x, b[1][q] = v.y;
          } else {
#pragma unroll
            for (int i = 0; i < NT; i += 4) {
              uint4 v = make_uint4(0, 0, 0, 0);
              if (kin && 8 * i + 8 * t < p.r) v = ldg16(row + 8 * i + 8 * t);
              b[i][q] = v.x, b[i + 1][q] = v.y, b[i + 2][q] = v.z, b[i + 3][q] = v.w;
            }
          }
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) b[i][q] = movmatrix_t(b[i][q]);
      }
      if (drop) {
        a0 = and4(a0, lora_keep8((uint32_t)(k >> 3), (uint32_t)(m0 + g), p.drop, key));
        a1 = and4(a1, lora_keep8((uint32_t)(k >> 3), (uint32_t)(m0 + g + 8), p.drop, key));
      }
      const uint32_t q0[4] = {a0.x, a1.x, a0.y, a1.y}, q1[4] = {a0.z, a1.z, a0.w, a1.w};
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        mma_16816(acc[i], q0, b[i][0], b[i][1]);
        mma_16816(acc[i], q1, b[i][2], b[i][3]);
      }
    }
  }

  float* mine_red = red + (size_t)warp * 16 * R;
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    mine_red[g * R + low_rank_of<NT, RM>(i, 2 * t)] = acc[i][0];
    mine_red[g * R + low_rank_of<NT, RM>(i, 2 * t + 1)] = acc[i][1];
    mine_red[(g + 8) * R + low_rank_of<NT, RM>(i, 2 * t)] = acc[i][2];
    mine_red[(g + 8) * R + low_rank_of<NT, RM>(i, 2 * t + 1)] = acc[i][3];
  }
  __syncthreads();
  const int total = RW * 16 * R;
  for (int e = threadIdx.x; e < total; e += LOW_THREADS) {
    float v = red[e];
    for (int i = 1; i < KW; ++i) v += red[i * total + e];
    red[e] = v;
  }
  __syncwarp();                          // (the cluster's barriers are a warp's together)
  cluster_arrive();
  cluster_wait();
  const int e0 = (int)((long long)total * rank / S), e1 = (int)((long long)total * (rank + 1) / S);
  const uint32_t base = smem_u32(red);
  for (int e = e0 + threadIdx.x; e < e1; e += LOW_THREADS) {
    const int j = e % R;
    const long long m = (long long)tile * RW * 16 + e / R;
    if (j >= p.r || m >= p.M) continue;
    float v = 0.f;
    for (int i = 0; i < S; ++i) {
      float w;
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(w) : "r"(dsmem_map(base + 4u * e, (uint32_t)i)) : "memory");
      v += w;
    }
    const int a = p.adapter[m];
    const float c = a >= 0 && a < p.n ? p.scaling[a] * p.keep_inv : 0.f;
    p.u[(size_t)m * p.r + j] = a >= 0 && a < p.n ? v * c : 0.f;
  }
  __syncwarp();
  cluster_arrive();                      // nobody leaves while its sums are read
  cluster_wait();
}

CS_DEV float dot2(uint32_t a, uint32_t b, float c) {
  c = fmaf(__uint_as_float(a << 16), __uint_as_float(b << 16), c);
  return fmaf(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u), c);
}
CS_DEV float dot8(uint4 a, uint4 b, float c) { return dot2(a.w, b.w, dot2(a.z, b.z, dot2(a.y, b.y, dot2(a.x, b.x, c)))); }

// A CTA per row.  Rows of the factor along the contraction: a warp takes two ranks and half of the
// contraction; along the rank: a thread takes eight ranks and every few rows of the factor.
template <bool RM>
__global__ void __launch_bounds__(ROW_THREADS) low_row_kernel(const LowArgs p) {
  __shared__ float part[16][128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int m = (int)blockIdx.x;
  griddep_wait();
  griddep_launch_dependents();
  const int a = lora_adapter(p.adapter, m, p.n, p.err);
  if (a < 0) {
    for (int j = threadIdx.x; j < p.r; j += ROW_THREADS) p.u[(size_t)m * p.r + j] = 0.f;
    return;
  }
  const __nv_bfloat16* x = p.x + (long long)m * p.ldx;
  const __nv_bfloat16* f = p.f + (size_t)a * p.r * p.C;
  const float c = p.scaling[a] * p.keep_inv;
  if (!RM) {
    const bool drop = p.drop.thr != 0u;
    LoraKey key{0, 0};
    if (drop) key = lora_key(p.drop);
    const int octets = p.C / 8, half = warp >> 3;
    const int o0 = half ? (octets + 1) / 2 : 0, o1 = half ? octets : (octets + 1) / 2;
    for (int j = 2 * (warp & 7); j < p.r; j += 16) {
      const __nv_bfloat16* f0 = f + (size_t)j * p.C;
      float v0 = 0.f, v1 = 0.f;
#pragma unroll 8
      for (int o = o0 + lane; o < o1; o += 32) {
        uint4 xv = ldg16(x + 8 * o);
        const uint4 a0 = ldg16(f0 + 8 * o), a1 = ldg16(f0 + p.C + 8 * o);
        if (drop) xv = and4(xv, lora_keep8((uint32_t)o, (uint32_t)m, p.drop, key));
        v0 = dot8(xv, a0, v0);
        v1 = dot8(xv, a1, v1);
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        v0 += __shfl_xor_sync(0xffffffffu, v0, d);
        v1 += __shfl_xor_sync(0xffffffffu, v1, d);
      }
      if (lane == 0) part[half][j] = v0, part[half][j + 1] = v1;
    }
    __syncthreads();
    for (int j = threadIdx.x; j < p.r; j += ROW_THREADS) p.u[(size_t)m * p.r + j] = (part[0][j] + part[1][j]) * c;
  } else {
    int og = 1;                          // octets of the rank, rounded up to a power of two
    while (og * 8 < p.r) og <<= 1;
    const int j = threadIdx.x & (og - 1), step = ROW_THREADS / og;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (8 * j < p.r) {
#pragma unroll 8
      for (int k = threadIdx.x / og; k < p.C; k += step) {
        const float xv = __bfloat162float(x[k]);
        const uint4 b = ldg16(f + (size_t)k * p.r + 8 * j);
        const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[2 * i] = fmaf(xv, __uint_as_float(w[i] << 16), v[2 * i]);
          v[2 * i + 1] = fmaf(xv, __uint_as_float(w[i] & 0xffff0000u), v[2 * i + 1]);
        }
      }
    }
    for (int d = 16; d >= og; d >>= 1)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
    if (lane < og) {
#pragma unroll
      for (int i = 0; i < 8; ++i) part[warp][lane * 8 + i] = v[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.r; i += ROW_THREADS) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < 16; ++w) s += part[w][i];
      p.u[(size_t)m * p.r + i] = s * c;
    }
  }
}

template <int NT, bool RM>
cudaError_t launch_low_mma(const LowArgs& p, int tiles, int splits, cudaStream_t stream) {
  static KernelLimits lim;
  const size_t smem = (size_t)8 * 16 * NT * 8 * sizeof(float);
  const cudaError_t e = ensure_kernel_limits((const void*)low_mma_kernel<NT, RM>, lim, smem, false);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * splits));
  cfg.blockDim = dim3(LOW_THREADS);
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
  return cudaLaunchKernelEx(&cfg, low_mma_kernel<NT, RM>, p);
}

template <bool RM>
cudaError_t launch_low(LowArgs p, int num_sms, cudaStream_t stream) {
  if ((long long)p.M * p.r <= LOW_ROW_MAX)
    return launch_pdl(low_row_kernel<RM>, dim3((unsigned)p.M), dim3(ROW_THREADS), 0, stream, p);
  // Four row groups a CTA share the factor's lines in L1; fewer where that leaves SMs without work.
  p.rw_log2 = 2;
  while (p.rw_log2 > 0 && (p.M + (16 << p.rw_log2) - 1) / (16 << p.rw_log2) * 8 < num_sms) --p.rw_log2;
  const int tiles = (p.M + (16 << p.rw_log2) - 1) / (16 << p.rw_log2);
  const int steps = (p.C + 31) / 32, kw = 8 >> p.rw_log2;
  int splits = 1;
  while (splits < 8 && tiles * splits < 2 * num_sms && steps >= 4 * splits * kw) splits *= 2;
  const int nt = (p.r + 7) / 8;
  if (nt <= 2) return launch_low_mma<2, RM>(p, tiles, splits, stream);
  if (nt <= 4) return launch_low_mma<4, RM>(p, tiles, splits, stream);
  if (nt <= 8) return launch_low_mma<8, RM>(p, tiles, splits, stream);
  return launch_low_mma<16, RM>(p, tiles, splits, stream);
}

}  // namespace

cudaError_t launch_lora_low(const LoraArgs& a, bool backward, int num_sms, int* err, cudaStream_t stream) {
  LowArgs p{};
  p.x = backward ? a.dy : a.x;
  p.ldx = backward ? a.ldy : a.ldx;
  p.f = backward ? a.b : a.a;
  p.scaling = a.scaling;
  p.adapter = a.adapter;
  p.u = backward ? a.t : a.u;
  p.M = a.M;
  p.C = backward ? a.N : a.K;
  p.r = a.r;
  p.n = a.n;
  p.keep_inv = 65536.f / (65536.f - (float)a.thr);
  p.drop = LoraDrop{a.seed, a.site, backward ? 0u : a.thr};
  p.err = err;
  return backward ? launch_low<true>(p, num_sms, stream) : launch_low<false>(p, num_sms, stream);
}

}  // namespace cospec
