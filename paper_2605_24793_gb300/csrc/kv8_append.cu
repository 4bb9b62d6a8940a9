// Rows of keys and values appended to the 8-bit paged cache, the keys (and the queries that come
// with them) rotated to their positions on the way.
//
// A warp owns one page of one layer for 128 dimensions' worth of KV heads (one head of 128, two of
// 64), keys or values.  A lane has four dimensions: it takes the page's new rows, four in flight, rotates
// keys (a dimension's partner comes by shuffle), keeps them in shared memory (its own part: nothing is
// exchanged, but rows can be looked up by number in a short loop; unrolled over the 16 tokens in registers the
// instruction cache missed and 36 layers x 16 sequences x 8 rows took 51 us for 25), reduces the page's largest
// magnitude, moves older codes to the new scale where that grew, and writes the codes.  All 16 tokens
// of a dimension meet in one lane, which is what the values' layout (a dimension's tokens side by side)
// and the page's summary need.  No two warps write the same page, so nothing depends on an order between
// them.  Query rows are rotated by blocks of their own: a lane keeps its angles for several heads of a row.
//
// Every step before a rounding is a product or sum rounded by itself or exact (powers of two,
// sums of at most 16 codes), so the codes, scales and summaries are the same on every run and in any
// other program that follows the definition in 32 bits.
//
// Bound by instructions and their latencies at 17 warps an SM: 36 layers x 16 sequences x 8 rows 22.3 us (issue slots
// 46 % busy; more blocks an SM need fewer registers: 23.4 to 30 us), 4096 rows x 2 layers with queries 42.9 us, 0.69
// of the copy rate; one row of a small layer 3 us.
#include "cospec_internal.h"
#include "kv8.cuh"

namespace cospec {

namespace {

constexpr int WARPS = 4;

struct Geometry {
  int T;                  // pages that a sequence's rows can touch
  int HG;                 // head groups: warps of a page and tensor
  unsigned page_tasks;    // L * B * T * 2 * HG
  int page_blocks;
  int q_groups;           // warps of a query row
};

constexpr int QU = 8;     // heads in flight per lane (4096 rows of 32 heads: 2 59.7, 4 47.6, 8 42.9, 16 44.6 us)
constexpr int UR = 4;     // rows in flight per lane,
constexpr int UO = 8;     // and older codes' rows
constexpr float FINITE = 3.4028235e38f;

// Four products and sums, each rounded by itself: y = x c - o s in the low half, x c + o s in the high one.
CS_DEV void turn4(float (&x)[4], const float (&o)[4], float4 c, float4 s, bool low) {
  const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float p = __fmul_rn(x[e], cc[e]), r = __fmul_rn(o[e], ss[e]);
    x[e] = low ? __fsub_rn(p, r) : __fadd_rn(p, r);
  }
}
// Two adjacent pairs.
CS_DEV void turn_pairs(float (&x)[4], float c0, float s0, float c1, float s1) {
  const float y0 = __fsub_rn(__fmul_rn(x[0], c0), __fmul_rn(x[1], s0));
  const float y1 = __fadd_rn(__fmul_rn(x[1], c0), __fmul_rn(x[0], s0));
  const float y2 = __fsub_rn(__fmul_rn(x[2], c1), __fmul_rn(x[3], s1));
  const float y3 = __fadd_rn(__fmul_rn(x[3], c1), __fmul_rn(x[2], s1));
  x[0] = y0;
  x[1] = y1;
  x[2] = y2;
  x[3] = y3;
}

// The largest over the lanes that share a head (32 of them, or 16).
template <int LPH>
CS_DEV float head_max(float v) {
#pragma unroll
  for (int o = LPH / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

template <int D>
__global__ void __launch_bounds__(WARPS * 32, 5)
    kv8_append_kernel(const Kv8AppendArgs a, const Geometry g, int* err) {
  constexpr int LPH = D / 4;               // lanes of a head
  constexpr int HPW = 32 / LPH;            // heads of a warp
  __shared__ float4 held[WARPS][KV8_PAGE][32];             // a page's new rows, each lane's own dimensions
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  griddep_wait();
  griddep_launch_dependents();

  if ((int)blockIdx.x >= g.page_blocks) {
    // ------------------------------------------------------------ query rows
    // A lane has four dimensions and the four that they are turned with, of every (256 / D)-th head.
    constexpr int LPP = D / 8, HP = 32 / LPP;
    const long long e = (long long)(blockIdx.x - g.page_blocks) * WARPS + warp;
    const long long row = e / g.q_groups;
    if (row >= (long long)a.L * a.B * a.R) return;
    const int h0 = (int)(e % g.q_groups) * (QU * HP) + lane / LPP, i = lane % LPP;
    const int j = (int)(row % a.R), b = (int)(row / a.R % a.B), l = (int)(row / a.R / a.B);
    const __nv_bfloat16* src = a.q.p + l * a.q.layer + b * a.q.batch + j * a.q.row;
    const bool turned = i < a.rot / 8, half = turned && !a.inter;
    const int lo = half ? 4 * i : 8 * i, hi = lo + (half ? a.rot / 2 : 4);
    uint2 u[QU], w[QU];
#pragma unroll
    for (int x = 0; x < QU; ++x) {
      const int h = h0 + x * HP;
      u[x] = w[x] = make_uint2(0u, 0u);
      if (h < a.Hq) {
        u[x] = *reinterpret_cast<const uint2*>(src + (size_t)h * D + lo);
        w[x] = *reinterpret_cast<const uint2*>(src + (size_t)h * D + hi);
      }
    }
    float4 c = make_float4(1.f, 1.f, 1.f, 1.f), s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.cos != nullptr) {
      const int st = a.start[b];
      if (st < 0 || st > a.positions - a.R) {
        if (lane == 0) set_err(err, ERR_POSITION);
        return;
      }
      if (turned) {
        const size_t at = (size_t)(st + j) * (a.rot / 2) + 4 * i;
        c = *reinterpret_cast<const float4*>(a.cos + at);
        s = *reinterpret_cast<const float4*>(a.sin + at);
      }
    }
    __nv_bfloat16* dst = a.q_out + (size_t)row * a.Hq * D;
#pragma unroll
    for (int x = 0; x < QU; ++x) {
      const int h = h0 + x * HP;
      if (h >= a.Hq) break;
      float y[4], z[4];
      kv8_floats_of(u[x], y);
      kv8_floats_of(w[x], z);
      if (half) {
        float o[4] = {y[0], y[1], y[2], y[3]};
        turn4(y, z, c, s, true);
        turn4(z, o, c, s, false);
      } else if (turned) {
        turn_pairs(y, c.x, s.x, c.y, s.y);
        turn_pairs(z, c.z, s.z, c.w, s.w);
      }
      kv8_store4(dst + (size_t)h * D + lo, y);
      kv8_store4(dst + (size_t)h * D + hi, z);
    }
    return;
  }

  // -------------------------------------------------------------- pages
  const unsigned task = blockIdx.x * WARPS + warp;
  if (task >= g.page_tasks) return;
  const unsigned x0 = task / (2u * g.HG), x1 = x0 / g.T;
  const int hw = (int)(task - x0 * (2u * g.HG)), which = hw >= g.HG ? 1 : 0, hg = hw - which * g.HG;   // 0: keys, 1: values
  const int t = (int)(x0 - x1 * g.T);
  const int l = (int)(x1 / (unsigned)a.B), b = (int)(x1 - (unsigned)l * a.B);
  const bool store = a.pool.k != nullptr;
  if (which == 1 && !store) return;
  const int h = hg * HPW + lane / LPH, d = lane % LPH * 4;
  const bool live = h < a.Hkv;              // (an odd head count leaves half a warp idle)
  const int st = a.start[b];
  const int n = !store ? 0 : a.num_rows ? a.num_rows[b] : a.R;
  const int page = st / KV8_PAGE + t;
  const int j0 = page * KV8_PAGE - st;      // row of the page's first token (negative: older tokens)
  const int first = max(0, -j0), last = min(KV8_PAGE, n - j0);       // new tokens [first, last)
  const int shown = which == 0 && a.k_out ? min(KV8_PAGE, a.R - j0) : last;
  const bool spoken = lane == 0 && hg == 0 && t == 0;
  if (store && (n < 0 || n > a.R || st < 0 || st > a.max_pages * KV8_PAGE - n)) {
    if (spoken) set_err(err, ERR_CTX);
    return;
  }
  // (values of a sequence whose keys are skipped are skipped with them)
  if (st < 0 || (a.cos != nullptr && st > a.positions - (a.k_out ? a.R : n))) {
    if (spoken) set_err(err, a.cos != nullptr ? ERR_POSITION : ERR_CTX);
    return;
  }
  if (first >= shown) return;
  const bool fresh = first < last;          // the page receives rows (else k_out alone does)
  const Kv8Src& src = which ? a.v : a.k;
  const __nv_bfloat16* row0 = src.p + l * src.layer + b * src.batch + (long long)j0 * src.row + (size_t)(live ? h : 0) * D + d;
  // Rows and older codes are asked for as soon as their addresses are known: a lane half a row of 128 dimensions, and
  // 64 bytes of the page.
  if (first <= lane >> 1 && lane >> 1 < shown)
    prefetch_l2(src.p + l * src.layer + b * src.batch + (long long)(j0 + (lane >> 1)) * src.row + (size_t)min(hg * 128 + (lane & 1) * 64, a.Hkv * D - 1));
  const int phys = fresh ? a.page_table[(size_t)b * a.max_pages + page] : -1;

  const bool bad = fresh && (unsigned)phys >= (unsigned)a.num_pages;
  if (bad && lane == 0) set_err(err, ERR_PAGE);
  const bool put = fresh && !bad;
  const size_t cell = ((size_t)l * a.num_pages + (put ? phys : 0)) * a.Hkv + (live ? h : 0);   // this layer's page and head
  const bool old = put && first > 0;
  if (old && live) prefetch_l2((which ? a.pool.v : a.pool.k) + cell * (KV8_PAGE * D) + lane % LPH * 64);
  const float was_scale = old ? a.pool.scale[cell * 2 + which] : 0.f;
  float4* mine = &held[warp][0][lane];                     // this lane's row i: mine[32 * i]
  float amax = 0.f;

  if (which == 1) {
    // ------------------------------------------------------------ values
    if (!put) return;
    for (int i0 = first; i0 < last; i0 += UR) {
      uint2 u[UR];
#pragma unroll
      for (int i = 0; i < UR; ++i)
        if (i0 + i < last) u[i] = *reinterpret_cast<const uint2*>(row0 + (i0 + i) * src.row);
#pragma unroll
      for (int i = 0; i < UR; ++i) {
        if (i0 + i >= last) break;
        float x[4];
        kv8_floats_of(u[i], x);
        amax = fmaxf(fmaxf(amax, fmaxf(fabsf(x[0]), fabsf(x[1]))), fmaxf(fabsf(x[2]), fabsf(x[3])));
        mine[32 * (i0 + i)] = make_float4(x[0], x[1], x[2], x[3]);
      }
    }
  } else {
    // ------------------------------------------------------------ keys
    const int half = a.rot >> 1;
    const bool turned = d < a.rot, low = d < half;
    const int at = a.inter ? d >> 1 : low ? d : d - half;
    const int partner = turned && !a.inter ? (low ? lane + (half >> 2) : lane - (half >> 2)) : lane;
    const size_t t0 = (size_t)(st + j0) * half + at;       // (the page's first token)
    __nv_bfloat16* show = a.k_out && live ? a.k_out + ((((long long)l * a.B + b) * a.R + j0) * a.Hkv + h) * D + d : nullptr;
    for (int i0 = first; i0 < shown; i0 += UR) {           // (the same in every lane)
      uint2 u[UR];
      float4 c[UR], s[UR];
#pragma unroll
      for (int i = 0; i < UR; ++i) {
        u[i] = make_uint2(0u, 0u);
        c[i] = s[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i0 + i >= shown) continue;
        u[i] = *reinterpret_cast<const uint2*>(row0 + (i0 + i) * src.row);
        if (a.cos == nullptr || !turned) continue;
        const size_t o = t0 + (size_t)(i0 + i) * half;
        if (a.inter) {
          const float2 c2 = *reinterpret_cast<const float2*>(a.cos + o), s2 = *reinterpret_cast<const float2*>(a.sin + o);
          c[i] = make_float4(c2.x, c2.y, 0.f, 0.f);
          s[i] = make_float4(s2.x, s2.y, 0.f, 0.f);
        } else {
          c[i] = *reinterpret_cast<const float4*>(a.cos + o);
          s[i] = *reinterpret_cast<const float4*>(a.sin + o);
        }
      }
#pragma unroll
      for (int i = 0; i < UR; ++i) {
        float x[4];
        kv8_floats_of(u[i], x);
        if (a.cos != nullptr) {
          if (a.inter) {
            if (turned) turn_pairs(x, c[i].x, s[i].x, c[i].y, s[i].y);
          } else {
            const uint2 pr = make_uint2(__shfl_sync(0xffffffffu, u[i].x, partner), __shfl_sync(0xffffffffu, u[i].y, partner));
            float o[4];
            kv8_floats_of(pr, o);
            if (turned) turn4(x, o, c[i], s[i], low);
          }
        }
        if (i0 + i >= shown) continue;
        if (show) kv8_store4(show + (long long)(i0 + i) * a.Hkv * D, x);
        if (i0 + i >= last) continue;
        amax = fmaxf(fmaxf(amax, fmaxf(fabsf(x[0]), fabsf(x[1]))), fmaxf(fabsf(x[2]), fabsf(x[3])));
        mine[32 * (i0 + i)] = make_float4(x[0], x[1], x[2], x[3]);
      }
    }
    if (!put) return;
  }

  // ---------------------------------------------------------------- the page's scale
  amax = head_max<LPH>(amax);
  if (__any_sync(0xffffffffu, amax > FINITE)) {            // an infinity: again without it
    amax = 0.f;
    for (int i = first; i < last; ++i) {
      const float4 x = mine[32 * i];
      amax = fmaxf(fmaxf(amax, fmaxf(kv8_finite_abs(x.x), kv8_finite_abs(x.y))), fmaxf(kv8_finite_abs(x.z), kv8_finite_abs(x.w)));
    }
    amax = head_max<LPH>(amax);
  }
  const float scale = fmaxf(kv8_scale_of(amax), was_scale), inv = kv8_inverse(scale);
  const float moved = old ? was_scale * inv : 1.f;         // (a power of two, 1 where the scale stays)
  if (live && d == 0) a.pool.scale[cell * 2 + which] = scale;
  auto code = [&](int i) {                                 // of the lane's new row i
    const float4 x = mine[32 * i];
    const float y[4] = {kv8_scaled(x.x, inv), kv8_scaled(x.y, inv), kv8_scaled(x.z, inv), kv8_scaled(x.w, inv)};
    return kv8_pack4(y);
  };
  auto move = [&](uint32_t w) {                            // four older codes to the new scale
    float y[4];
    kv8_floats4(w, y);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] *= moved;
    return kv8_pack4(y);
  };

  if (which == 1) {
    if (!live) return;
    uint8_t* dst = a.pool.v + (cell * D + d) * KV8_PAGE;
    for (int m = moved == 1.f ? first >> 2 : 0; 4 * m < last; ++m) {
      // tokens 4 m .. 4 m + 3: bytes before `f` are older, from `u` on nobody's
      const int f = min(max(first - 4 * m, 0), 4), u = min(last - 4 * m, 4);
      uint32_t r[4], w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = i >= f && i < u ? code(4 * m + i) : 0u;
      // four rows of four dimensions turned into four dimensions of four tokens
      const uint32_t p0 = __byte_perm(r[0], r[1], 0x5140), p1 = __byte_perm(r[2], r[3], 0x5140);
      const uint32_t p2 = __byte_perm(r[0], r[1], 0x7362), p3 = __byte_perm(r[2], r[3], 0x7362);
      w[0] = __byte_perm(p0, p1, 0x5410);
      w[1] = __byte_perm(p0, p1, 0x7632);
      w[2] = __byte_perm(p2, p3, 0x5410);
      w[3] = __byte_perm(p2, p3, 0x7632);
      if (u - f < 4) {
        const uint32_t upto_u = u == 4 ? 0xffffffffu : (1u << (8 * u)) - 1u, upto_f = f == 4 ? 0xffffffffu : (1u << (8 * f)) - 1u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t was = *reinterpret_cast<const uint32_t*>(dst + e * KV8_PAGE + 4 * m);
          w[e] = (w[e] & upto_u & ~upto_f) | (was & ~upto_u) | ((moved == 1.f ? was : move(was)) & upto_f);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(dst + e * KV8_PAGE + 4 * m) = w[e];
    }
    return;
  }
  uint8_t* dst = a.pool.k + cell * (KV8_PAGE * D) + d;
  const bool sums = a.pool.summary != nullptr;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](uint32_t w, bool checked) {
    float y[4];
    kv8_floats4(w, y);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += checked && y[e] != y[e] ? 0.f : y[e];
  };
  if (sums || moved != 1.f) {
    for (int i0 = 0; i0 < first; i0 += UO) {
      uint32_t w[UO];
#pragma unroll
      for (int i = 0; i < UO; ++i)
        if (i0 + i < first) w[i] = *reinterpret_cast<const uint32_t*>(dst + (i0 + i) * D);
#pragma unroll
      for (int i = 0; i < UO; ++i) {
        if (i0 + i >= first) break;
        if (moved != 1.f) {
          w[i] = move(w[i]);
          if (live) *reinterpret_cast<uint32_t*>(dst + (i0 + i) * D) = w[i];
        }
        add(w[i], false);
      }
    }
  }
#pragma unroll 2
  for (int i = first; i < last; ++i) {
    const uint32_t w = code(i);
    if (live) *reinterpret_cast<uint32_t*>(dst + i * D) = w;
    if (sums) add(w, false);
  }
  if (!sums) return;
  const float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
  if (__any_sync(0xffffffffu, all != all)) {               // NaN codes: without them (each lane reads what it wrote)
    sum[0] = sum[1] = sum[2] = sum[3] = 0.f;
    if (live)
      for (int i = 0; i < last; ++i) add(*reinterpret_cast<const volatile uint32_t*>(dst + i * D), true);
  }
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

template <int D>
cudaError_t launch(const Kv8AppendArgs& a, int* err, cudaStream_t stream) {
  Geometry g{};
  g.T = (a.R + KV8_PAGE - 2) / KV8_PAGE + 1;
  g.HG = (a.Hkv + 128 / D - 1) / (128 / D);
  const bool pages = a.pool.k || a.k_out;
  const long long tasks = pages ? (long long)a.L * a.B * g.T * g.HG * 2 : 0;
  g.q_groups = (a.Hq + QU * (256 / D) - 1) / (QU * (256 / D));
  const long long pb = (tasks + WARPS - 1) / WARPS;
  const long long qb = ((long long)a.L * a.B * a.R * g.q_groups + WARPS - 1) / WARPS;
  if (tasks > 0x7fffffffLL || pb + qb > 0x7fffffffLL) return cudaErrorInvalidValue;
  g.page_tasks = (unsigned)tasks;
  if (pb + qb == 0) return cudaSuccess;
  g.page_blocks = (int)pb;
  return launch_pdl(kv8_append_kernel<D>, dim3((unsigned)(pb + qb)), dim3(WARPS * 32), 0, stream, a, g, err);
}

}  // namespace

cudaError_t launch_kv8_append(const Kv8AppendArgs& a, int* err, cudaStream_t stream) {
  return a.D == 128 ? launch<128>(a, err, stream) : launch<64>(a, err, stream);
}

}  // namespace cospec
