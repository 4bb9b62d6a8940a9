// Rows of keys and values appended to the 8-bit paged cache, the keys (and the queries that come
// with them) rotated to their positions on the way.
//
// A warp owns one page of one layer for 128 dimensions' worth of KV heads (one head of 128, two of
// 64), keys or values: it takes every new row of the page into registers, four dimensions a lane,
// rotates keys, reduces the page's largest magnitude, moves older codes to the new scale where
// that grew, and writes the page's codes.  All 16 tokens of a dimension meet in one lane, which is
// what the values' layout (a dimension's tokens side by side) and the page's summary need.  No two
// warps write the same page, so nothing depends on an order between them.
//
// Every step before a rounding is a product or sum rounded by itself or exact (powers of two,
// sums of at most 16 codes), so the codes, scales and summaries are the same on every run and in any
// other program that follows the definition in 32 bits.
#include "cospec_internal.h"
#include "kv8.cuh"

namespace cospec {

namespace {

constexpr int WARPS = 4;

struct Geometry {
  int T;                  // pages that a sequence's rows can touch
  int HG;                 // head groups: warps of a page and tensor
  long long page_tasks;   // L * B * T * HG * 2
  int page_blocks;
  int q_chunks;           // groups of four dimensions of a row's query heads
};

// x (four dimensions from d on of the row `row`) turned by its position's angles.
CS_DEV void rotate4(const Kv8AppendArgs& a, const __nv_bfloat16* row, int d, int pos, float (&x)[4]) {
  if (a.cos == nullptr || d >= a.rot) return;
  const int h = a.rot >> 1;
  const size_t t = (size_t)pos * h;
  if (a.inter) {
    const float2 c = *reinterpret_cast<const float2*>(a.cos + t + (d >> 1));
    const float2 s = *reinterpret_cast<const float2*>(a.sin + t + (d >> 1));
    const float y0 = __fsub_rn(__fmul_rn(x[0], c.x), __fmul_rn(x[1], s.x));
    const float y1 = __fadd_rn(__fmul_rn(x[1], c.x), __fmul_rn(x[0], s.x));
    const float y2 = __fsub_rn(__fmul_rn(x[2], c.y), __fmul_rn(x[3], s.y));
    const float y3 = __fadd_rn(__fmul_rn(x[3], c.y), __fmul_rn(x[2], s.y));
    x[0] = y0;
    x[1] = y1;
    x[2] = y2;
    x[3] = y3;
    return;
  }
  const bool low = d < h;
  const int i = low ? d : d - h;
  const float4 c = *reinterpret_cast<const float4*>(a.cos + t + i);
  const float4 s = *reinterpret_cast<const float4*>(a.sin + t + i);
  float o[4];
  kv8_load4(row + (low ? d + h : d - h), o);
  const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float p = __fmul_rn(x[e], cc[e]), r = __fmul_rn(o[e], ss[e]);
    x[e] = low ? __fsub_rn(p, r) : __fadd_rn(p, r);
  }
}

// The largest over the lanes that share a head (32 of them, or 16).
template <int LPH>
CS_DEV float head_max(float v) {
#pragma unroll
  for (int o = LPH / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

template <int D>
__global__ void __launch_bounds__(WARPS * 32)
    kv8_append_kernel(const Kv8AppendArgs a, const Geometry g, int* err) {
  constexpr int LPH = D / 4;               // lanes of a head
  constexpr int HPW = 32 / LPH;            // heads of a warp
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  griddep_wait();
  griddep_launch_dependents();

  if ((int)blockIdx.x >= g.page_blocks) {
    // ------------------------------------------------------------ query rows
    const long long e = (long long)(blockIdx.x - g.page_blocks) * (WARPS * 32) + threadIdx.x;
    const long long row = e / g.q_chunks;
    const int c = (int)(e % g.q_chunks);
    if (row >= (long long)a.L * a.B * a.R) return;
    const int j = (int)(row % a.R), b = (int)(row / a.R % a.B), l = (int)(row / a.R / a.B);
    const int st = a.start[b];
    if (a.cos != nullptr && (st < 0 || st > a.positions - a.R)) {
      if (c == 0) set_err(err, ERR_POSITION);
      return;
    }
    const int h = c / LPH, d = c % LPH * 4;
    const __nv_bfloat16* src = a.q.p + l * a.q.layer + b * a.q.batch + j * a.q.row + (size_t)h * D;
    float x[4];
    kv8_load4(src + d, x);
    rotate4(a, src, d, st + j, x);
    kv8_store4(a.q_out + ((size_t)row * a.Hq + h) * D + d, x);
    return;
  }

  // -------------------------------------------------------------- pages
  const long long task = (long long)blockIdx.x * WARPS + warp;
  if (task >= g.page_tasks) return;
  const int hg = (int)(task % g.HG);
  const int which = (int)(task / g.HG % 2);                 // 0: keys, 1: values
  const int t = (int)(task / g.HG / 2 % g.T);
  const int b = (int)(task / g.HG / 2 / g.T % a.B);
  const int l = (int)(task / g.HG / 2 / g.T / a.B);
  const bool store = a.pool.k != nullptr;
  if (which == 1 && !store) return;
  const int h = hg * HPW + lane / LPH, d = lane % LPH * 4;
  const bool live = h < a.Hkv;              // (an odd head count leaves half a warp idle)
  const int st = a.start[b];
  const int n = !store ? 0 : a.num_rows ? a.num_rows[b] : a.R;
  const bool spoken = lane == 0 && hg == 0 && t == 0;
  if (store && (n < 0 || n > a.R || st < 0 || st > a.max_pages * KV8_PAGE - n)) {
    if (spoken) set_err(err, ERR_CTX);
    return;
  }
  if (st < 0 || (a.cos != nullptr && which == 0 && st > a.positions - (a.k_out ? a.R : n))) {
    if (spoken) set_err(err, a.cos != nullptr ? ERR_POSITION : ERR_CTX);
    return;
  }
  // (values of a sequence whose keys are skipped are skipped with them)
  if (a.cos != nullptr && which == 1 && st > a.positions - (a.k_out ? a.R : n)) return;
  const int page = st / KV8_PAGE + t;
  const int j0 = page * KV8_PAGE - st;      // row of the page's first token (negative: older tokens)
  const int first = max(0, -j0), last = min(KV8_PAGE, n - j0);       // new tokens [first, last)
  const int shown = which == 0 && a.k_out ? min(KV8_PAGE, a.R - j0) : last;
  if (first >= shown) return;

  const Kv8Src& src = which ? a.v : a.k;
  float x[KV8_PAGE][4];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < KV8_PAGE; ++i) {
    x[i][0] = x[i][1] = x[i][2] = x[i][3] = 0.f;
    if (i < first || i >= shown || !live) continue;
    const int j = j0 + i;
    const __nv_bfloat16* row = src.p + l * src.layer + b * src.batch + j * src.row + (size_t)h * D;
    kv8_load4(row + d, x[i]);
    if (which == 0) {
      rotate4(a, row, d, st + j, x[i]);
      if (a.k_out) kv8_store4(a.k_out + ((((size_t)l * a.B + b) * a.R + j) * a.Hkv + h) * D + d, x[i]);
    }
    if (i < last)
#pragma unroll
      for (int e = 0; e < 4; ++e) amax = fmaxf(amax, kv8_finite_abs(x[i][e]));
  }
  if (first >= last) return;                // rows shown in k_out only
  const int phys = a.page_table[(size_t)b * a.max_pages + page];
  if ((unsigned)phys >= (unsigned)a.num_pages) {
    if (lane == 0) set_err(err, ERR_PAGE);
    return;
  }
  amax = head_max<LPH>(amax);
  const size_t cell = ((size_t)l * a.num_pages + phys) * a.Hkv + h;   // this layer's page and head
  float scale = kv8_scale_of(amax), moved = 1.f;
  const bool old = first > 0;
  if (old && live) {
    const float was = a.pool.scale[cell * 2 + which];
    scale = fmaxf(scale, was);
    moved = was * kv8_inverse(scale);
  }
  const float inv = kv8_inverse(scale);

  if (which == 0) {
    uint32_t code[KV8_PAGE];
    uint8_t* dst = a.pool.k + cell * (KV8_PAGE * D) + d;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KV8_PAGE; ++i) {
      code[i] = 0u;
      if (i < first && live) {
        float f[4];
        kv8_floats4(*reinterpret_cast<const uint32_t*>(dst + i * D), f);
        code[i] = kv8_pack2(f[0] * moved, f[1] * moved) | kv8_pack2(f[2] * moved, f[3] * moved) << 16;
      } else if (i < last) {
        code[i] = kv8_pack2(x[i][0] * inv, x[i][1] * inv) | kv8_pack2(x[i][2] * inv, x[i][3] * inv) << 16;
      }
      float f[4];
      kv8_floats4(code[i], f);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += f[e] == f[e] ? f[e] : 0.f;
    }
    if (live)
#pragma unroll
      for (int i = 0; i < KV8_PAGE; ++i)
        if (i < last && (i >= first || moved != 1.f)) *reinterpret_cast<uint32_t*>(dst + i * D) = code[i];
    if (a.pool.summary) {
      const float u = kv8_scale127(head_max<LPH>(fmaxf(fmaxf(fabsf(sum[0]), fabsf(sum[1])), fmaxf(fabsf(sum[2]), fabsf(sum[3])))));
      const float ui = kv8_inverse(u);
      uint32_t w = 0u;
#pragma unroll
      for (int e = 0; e < 4; ++e) w |= ((uint32_t)__float2int_rn(sum[e] * ui) & 0xffu) << (8 * e);
      if (live) {
        *reinterpret_cast<uint32_t*>(a.pool.summary + cell * D + d) = w;
        if (d == 0) a.pool.summary_scale[cell] = u * scale;
      }
    }
  } else if (live) {
    uint8_t* dst = a.pool.v + (cell * D + d) * KV8_PAGE;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t w[4];
      uint4 was = make_uint4(0u, 0u, 0u, 0u);
      if (old || last < KV8_PAGE) was = *reinterpret_cast<const uint4*>(dst + e * KV8_PAGE);
      const uint32_t ow[4] = {was.x, was.y, was.z, was.w};
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        float f[4];
        kv8_floats4(ow[m], f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = m * 4 + i;                                // (from `last` on: left as they are)
          f[i] = tok < first ? f[i] * moved : tok < last ? x[tok][e] * inv : f[i];
        }
        w[m] = kv8_pack2(f[0], f[1]) | kv8_pack2(f[2], f[3]) << 16;
      }
      *reinterpret_cast<uint4*>(dst + e * KV8_PAGE) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  if (live && d == 0) a.pool.scale[cell * 2 + which] = scale;
}

template <int D>
cudaError_t launch(const Kv8AppendArgs& a, int* err, cudaStream_t stream) {
  Geometry g{};
  g.T = (a.R + KV8_PAGE - 2) / KV8_PAGE + 1;
  g.HG = (a.Hkv + 128 / D - 1) / (128 / D);
  const bool pages = a.pool.k || a.k_out;
  g.page_tasks = pages ? (long long)a.L * a.B * g.T * g.HG * 2 : 0;
  g.q_chunks = a.Hq * (D / 4);
  const long long pb = (g.page_tasks + WARPS - 1) / WARPS;
  const long long qb = ((long long)a.L * a.B * a.R * g.q_chunks + WARPS * 32 - 1) / (WARPS * 32);
  if (pb + qb > 0x7fffffffLL) return cudaErrorInvalidValue;
  if (pb + qb == 0) return cudaSuccess;
  g.page_blocks = (int)pb;
  return launch_pdl(kv8_append_kernel<D>, dim3((unsigned)(pb + qb)), dim3(WARPS * 32), 0, stream, a, g, err);
}

}  // namespace

cudaError_t launch_kv8_append(const Kv8AppendArgs& a, int* err, cudaStream_t stream) {
  return a.D == 128 ? launch<128>(a, err, stream) : launch<64>(a, err, stream);
}

}  // namespace cospec
