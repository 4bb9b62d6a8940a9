// Attention of a block of rows over the 8-bit paged cache and the block's own bf16 rows.
//
// One CTA per (sequence, block row, query head); a warp takes every fourth key, its lanes the
// dimensions, with a running maximum and sum; the warps' parts meet in shared memory.
#include "cospec_internal.h"
#include "kv8.cuh"

namespace cospec {

namespace {

constexpr int WARPS = 4;

template <int D>
__global__ void __launch_bounds__(WARPS * 32) kv8_attn_kernel(const Kv8AttnArgs a, int* err) {
  constexpr int E = D / 32;
  __shared__ float part[WARPS][D + 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int hq = blockIdx.x % a.Hq, j = blockIdx.x / a.Hq % a.R, b = blockIdx.x / a.Hq / a.R;
  const int G = a.Hq / a.Hkv, h = hq / G;
  griddep_wait();
  griddep_launch_dependents();
  const int C = a.ctx_len[b];
  const bool bad = C < 0 || C > a.max_pages * KV8_PAGE;
  if (bad && threadIdx.x == 0 && hq == 0 && j == 0) set_err(err, ERR_CTX);
  const int32_t* table = a.page_table + (size_t)b * a.max_pages;
  const int32_t* sel = a.sel ? a.sel + (((size_t)b * a.R + j) * a.Hkv + h) * a.pages : nullptr;
  const int num = bad ? 0 : (C + KV8_PAGE - 1) / KV8_PAGE;
  const int entries = sel ? (bad ? 0 : a.pages) : num;
  float q[E], o[E], m = -INFINITY, sum = 0.f;
  const __nv_bfloat16* qp = a.q.p + b * a.q.batch + j * a.q.row + (size_t)hq * D;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = __bfloat162float(qp[e * 32 + lane]);
    o[e] = 0.f;
  }
  auto key = [&](const float (&k)[E], const float (&v)[E], float ks, float vs) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += q[e] * k[e];
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= ks * a.scale;
    const float n = fmaxf(m, s);
    const float w = expf(s - n), c = m == -INFINITY ? 0.f : expf(m - n);
    sum = sum * c + w;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * c + w * vs * v[e];
    m = n;
  };
  for (int i = 0; i < entries; ++i) {
    const int p = sel ? sel[i] : i;
    if (p < 0) break;
    const int phys = p < num ? table[p] : -1;
    if ((unsigned)phys >= (unsigned)a.num_pages) {
      if (lane == 0) set_err(err, ERR_PAGE);
      continue;
    }
    const size_t cell = (size_t)phys * a.Hkv + h;
    const float ks = a.pool.scale[cell * 2], vs = a.pool.scale[cell * 2 + 1];
    for (int t = warp; t < KV8_PAGE && p * KV8_PAGE + t < C; t += WARPS) {
      float k[E], v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = e * 32 + lane;
        k[e] = kv8_floats(a.pool.k[(cell * KV8_PAGE + t) * D + d]).x;
        v[e] = kv8_floats(a.pool.v[(cell * D + d) * KV8_PAGE + t]).x;
      }
      key(k, v, ks, vs);
    }
  }
  for (int t = warp; t < (a.block_full ? a.R : j + 1); t += WARPS) {
    float k[E], v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int d = e * 32 + lane;
      k[e] = __bfloat162float(a.k_blk.p[b * a.k_blk.batch + t * a.k_blk.row + (size_t)h * D + d]);
      v[e] = __bfloat162float(a.v_blk.p[b * a.v_blk.batch + t * a.v_blk.row + (size_t)h * D + d]);
    }
    key(k, v, 1.f, 1.f);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) part[warp][e * 32 + lane] = o[e];
  if (lane == 0) {
    part[warp][D] = m;
    part[warp][D + 1] = sum;
  }
  __syncthreads();
  for (int d = threadIdx.x; d < D; d += WARPS * 32) {
    float top = -INFINITY, l = 0.f, x = 0.f;
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, part[w][D]);
    for (int w = 0; w < WARPS; ++w) {
      const float c = part[w][D] == -INFINITY ? 0.f : expf(part[w][D] - top);
      l += part[w][D + 1] * c;
      x += part[w][d] * c;
    }
    a.out[(((size_t)b * a.R + j) * a.Hq + hq) * D + d] = __float2bfloat16_rn(x / l);
  }
}

}  // namespace

cudaError_t launch_kv8_attn(const Kv8AttnArgs& a, int* err, cudaStream_t stream) {
  const unsigned grid = (unsigned)a.B * a.R * a.Hq;
  return a.D == 128 ? launch_pdl(kv8_attn_kernel<128>, dim3(grid), dim3(WARPS * 32), 0, stream, a, err)
                    : launch_pdl(kv8_attn_kernel<64>, dim3(grid), dim3(WARPS * 32), 0, stream, a, err);
}

}  // namespace cospec
