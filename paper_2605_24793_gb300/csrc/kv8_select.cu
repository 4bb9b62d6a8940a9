// The pages of a long context that each block row reads, chosen by the integer products of the row's
// queries, rounded to 8 bits, with the pages' summaries.
//
// One CTA per (sequence, block row, KV head): the scores of all pages into shared memory as
// ordered 32-bit keys, the m-th largest by a radix selection of eight bits a pass, then one
// pass in page order that writes what lies above it and, of the pages equal to it, the first ones.
#include "cospec_internal.h"
#include "kv8.cuh"

namespace cospec {

namespace {

constexpr int CT = 256;
constexpr int GMAX = 64;                  // query rows of a KV head held at once

// A float's bits in an order that unsigned comparison follows.
CS_DEV uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum of v over the threads before this one, and over all of them.
CS_DEV int block_scan(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < CT / 32; ++w) {
    const int s = warp_sums[w];
    before += w < warp ? s : 0;
    all += s;
  }
  total = all;
  return before + inc - v;
}

template <int D>
__global__ void __launch_bounds__(CT) kv8_select_kernel(const Kv8SelectArgs a, int* err) {
  extern __shared__ uint32_t key[];        // [pages of the context]
  __shared__ int qi[GMAX][D / 4];          // 8-bit queries
  __shared__ int hist[256];
  __shared__ int sums[CT / 32];
  __shared__ float red[CT / 32];
  __shared__ int s_digit, s_left;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = blockIdx.x % a.Hkv, j = blockIdx.x / a.Hkv % a.R, b = blockIdx.x / a.Hkv / a.R;
  griddep_wait();
  griddep_launch_dependents();
  int32_t* sel = a.sel + (((size_t)b * a.R + j) * a.Hkv + h) * a.pages;
  const int C = a.ctx_len[b];
  const bool bad = C < 0 || C > a.max_pages * KV8_PAGE;
  if (bad && tid == 0 && h == 0 && j == 0) set_err(err, ERR_CTX);
  const int num = bad ? 0 : (C + KV8_PAGE - 1) / KV8_PAGE;
  if (num <= a.pages) {                    // every page
    for (int p = tid; p < a.pages; p += CT) sel[p] = p < num ? p : -1;
    return;
  }
  const int32_t* table = a.page_table + (size_t)b * a.max_pages;
  const int G = a.Hq / a.Hkv;
  const __nv_bfloat16* q = a.q.p + b * a.q.batch + j * a.q.row + (size_t)h * G * D;
  float amax = 0.f;
  for (int e = tid; e < G * D; e += CT) amax = fmaxf(amax, kv8_finite_abs(__bfloat162float(q[e])));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if (lane == 0) red[warp] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < CT / 32; ++w) amax = fmaxf(amax, red[w]);
  const float inv = kv8_inverse(kv8_scale127(amax));
  for (int p = tid; p < num; p += CT) key[p] = 0u;
  for (int g0 = 0; g0 < G; g0 += GMAX) {
    const int gn = min(GMAX, G - g0);
    __syncthreads();
    for (int e = tid; e < gn * (D / 4); e += CT) {
      float x[4];
      kv8_load4(q + (size_t)g0 * D + e * 4, x);
      uint32_t w = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y = fabsf(x[i]) <= 3.4028235e38f ? x[i] * inv : 0.f;
        w |= ((uint32_t)__float2int_rn(y) & 0xffu) << (8 * i);
      }
      qi[e / (D / 4)][e % (D / 4)] = (int)w;
    }
    __syncthreads();
    for (int p = tid; p < num; p += CT) {
      if (p < a.sink || p >= num - a.recent) continue;
      const int phys = table[p];
      if ((unsigned)phys >= (unsigned)a.num_pages) {
        set_err(err, ERR_PAGE);
        continue;                          // (key 0: below every score)
      }
      const size_t cell = (size_t)phys * a.Hkv + h;
      const int4* s = reinterpret_cast<const int4*>(a.pool.summary + cell * D);
      int4 sv[D / 16];
#pragma unroll
      for (int i = 0; i < D / 16; ++i) sv[i] = __ldg(s + i);
      int best = -0x7fffffff;
      for (int g = 0; g < gn; ++g) {
        int dot = 0;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          dot = __dp4a(sv[i].x, qi[g][4 * i], dot);
          dot = __dp4a(sv[i].y, qi[g][4 * i + 1], dot);
          dot = __dp4a(sv[i].z, qi[g][4 * i + 2], dot);
          dot = __dp4a(sv[i].w, qi[g][4 * i + 3], dot);
        }
        best = max(best, dot);
      }
      key[p] = max(key[p], ordered((float)best * a.pool.summary_scale[cell]));
    }
  }
  __syncthreads();
  // The m-th largest key among the pages that are not chosen anyway.
  const int lo = min(a.sink, num), hi = max(lo, num - a.recent);
  int m = a.pages - lo - (num - hi);       // num > pages >= sink + recent: 0 <= m < hi - lo
  uint32_t prefix = 0u, mask = 0u;
  for (int shift = 24; shift >= 0 && m > 0; shift -= 8) {
    for (int i = tid; i < 256; i += CT) hist[i] = 0;
    __syncthreads();
    for (int p = lo + tid; p < hi; p += CT)
      if ((key[p] & mask) == prefix) atomicAdd(&hist[key[p] >> shift & 255u], 1);
    __syncthreads();
    int total;
    const int mine = hist[255 - tid];      // thread t: the t-th digit from the top
    const int above = block_scan(mine, sums, total);
    if (above < m && m <= above + mine) {
      s_digit = 255 - tid;
      s_left = m - above;
    }
    __syncthreads();
    prefix |= (uint32_t)s_digit << shift;
    mask |= 255u << shift;
    m = s_left;
    __syncthreads();
  }
  // In page order: pages above the threshold and the first m equal to it.
  const bool none = a.pages == lo + (num - hi);
  int at = 0, equal = 0;
  for (int p0 = 0; p0 < num; p0 += CT) {
    const int p = p0 + tid;
    const bool in = p < num, always = in && (p < lo || p >= hi);
    const bool eq = in && !always && !none && key[p] == prefix;
    const bool gt = in && !always && !none && key[p] > prefix;
    int n_eq, n_take;
    const int e = equal + block_scan(eq ? 1 : 0, sums, n_eq);
    const bool take = always || gt || (eq && e < m);
    const int o = at + block_scan(take ? 1 : 0, sums, n_take);
    if (take) sel[o] = p;
    at += n_take;
    equal += n_eq;
  }
}

}  // namespace

cudaError_t launch_kv8_select(const Kv8SelectArgs& a, int* err, cudaStream_t stream) {
  const size_t smem = (size_t)a.max_pages * 4;
  const unsigned grid = (unsigned)a.B * a.R * a.Hkv;
  static KernelLimits lim128, lim64;
  const cudaError_t e = a.D == 128 ? ensure_kernel_limits((const void*)kv8_select_kernel<128>, lim128, smem, false)
                                   : ensure_kernel_limits((const void*)kv8_select_kernel<64>, lim64, smem, false);
  if (e != cudaSuccess) return e;
  return a.D == 128 ? launch_pdl(kv8_select_kernel<128>, dim3(grid), dim3(CT), smem, stream, a, err)
                    : launch_pdl(kv8_select_kernel<64>, dim3(grid), dim3(CT), smem, stream, a, err);
}

}  // namespace cospec
