// What the two attention kernels over the 8-bit cache share on the host and as their argument.
#pragma once

#include "cospec_internal.h"

namespace cospec {

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

// tcgen05 (kv8_attn_tc.cu): groups of 128 / G whole block rows, clusters of S CTAs.
int kv8_attn_tc_resident(int D, int S);     // such clusters resident at once
cudaError_t launch_kv8_attn_tc(const Kv8Params& p, int D, int S, cudaStream_t stream);

}  // namespace cospec
