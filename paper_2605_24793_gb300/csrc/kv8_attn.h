// What the two attention kernels over the 8-bit cache share on the host and as their argument.
#pragma once

#include "cospec_internal.h"

namespace cospec {

// Weights are held times 2^P_BITS and may grow by 2^P_ROOM before the output is rescaled: below f16's 2^16.
constexpr float P_BITS = 6.f, P_ROOM = 8.f;
// Values' scales up to 2^V_ROOM above the least are met with f16 weights, and the unit that outputs count in is at most 2^V_FAR
// below the largest scale, so that outputs stay within fp32.
constexpr int V_ROOM = 8, V_FAR = 64;
constexpr int ZERO_EXP = 27;              // biased exponent of 2^-100, the scale of a page of zeros

struct Kv8Params {
  Kv8Pool pool;
  Kv8Src q, k_blk, v_blk;
  const int32_t* page_table;
  const int32_t* ctx_len;
  const int32_t* sel;
  int pages;
  __nv_bfloat16* out;
  int B, R, Hq, Hkv, G, num_pages, max_pages;
  int rows;          // query rows of a unit before it is cut into groups: G * R, or G with selected pages
  int groups;        // row groups of a unit
  float scale_log2;
  int kv_stable, block_full;
  int* err;
};

// The matrix products run over all rows of the block, those that the mask hides with the weight 0: infinities and NaN among
// its values, which 0 would turn into NaN, enter the products as 0 and join the written outputs of the rows that see them
// here.  `rows` query rows of a unit from row0 on, by all the block's threads after a barrier.
__device__ inline void kv8_add_nonfinite(const Kv8Params& p, int D, bool sel, int jj, int b, int h, int row0, int rows) {
#pragma unroll 1
  for (int e = threadIdx.x; e < rows * D; e += blockDim.x) {
    const int row = row0 + e / D, x = e % D;
    const int j = sel ? jj : row / p.G, head = h * p.G + (sel ? row : row % p.G), last = p.block_full ? p.R - 1 : j;
    const __nv_bfloat16* v = p.v_blk.p + b * p.v_blk.batch + (size_t)h * D + x;
    float sum = 0.f;
#pragma unroll 1
    for (int k = 0; k <= last; ++k) {
      const float y = __bfloat162float(v[k * p.v_blk.row]);
      if (!(fabsf(y) <= 3.4028235e38f)) sum += y;
    }
    if (sum == 0.f) continue;
    __nv_bfloat16* o = p.out + (((size_t)b * p.R + j) * p.Hq + head) * D + x;
    *o = __float2bfloat16_rn(__bfloat162float(*o) + sum);
  }
}

// tcgen05 (kv8_attn_tc.cu): groups of 128 / G whole block rows, clusters of S CTAs.
int kv8_attn_tc_resident(int D, int S);     // such clusters resident at once
cudaError_t launch_kv8_attn_tc(const Kv8Params& p, int D, int S, cudaStream_t stream);

}  // namespace cospec
