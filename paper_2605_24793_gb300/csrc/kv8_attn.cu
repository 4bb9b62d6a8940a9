// Attention of a block of rows over the 8-bit paged cache and the block's own bf16 rows.
//
// A unit is (sequence, KV head, up to 32 query rows that read it), or with selected pages (sequence, block
// row, KV head, up to 32 of its query heads).  Its pages go in pairs (32 keys: a tile) to the rings of a
// thread-block cluster, tile t of the unit to ring t mod (rings S).  A ring belongs to one warp or to two,
// and no ring waits for another until the end.  A ring's warps bring its tiles in together, asynchronously, and each puts
// its own rows to them.  Variants, chosen by the estimates below:
//   columns: the query rows are the products' columns, eight at a time, keys and values their rows, so that up to 8 and 17
//   to 24 rows are padded less than by 16.  A warp a ring and two CTAs an SM: six warps with rings of two tiles up to 8
//   rows, four with rings of three at 24 (as registers allow).  Up to 8 rows, with six warps, four, eight (one CTA an SM)
//   and padded: one user at 4096 tokens 7.1, 7.1, 8.4, 7.9 us, at 32768 20.1, 22.8, 23.8, 25.5; 128 selected pages for
//   each of 128 rows 84, 92, 107, 104.  At 24 rows: batch 16 at 2048 to 8192 tokens 49.5 us, padded 53.7; batch 64 at 8192
//   to 32768 481, padded 547;
//   rows: the query rows are the products' rows, by 16, which is as good where they fill them and has fewer shuffles: batch
//   64 at 32 rows 552 us for 613, at 12 rows one user 8.4 for 9.1.  Up to 16 a warp a ring, four warps and two CTAs an SM
//   or eight and one (long contexts of few users: one user at 32768 tokens 26.0 us and 21.7, at 4096 8.4 and 9.8); up to
//   32 a warp of 32 rows a ring (each code converted once), or two of 16 (half the registers, shorter steps) with four
//   warps and three CTAs an SM or with eight.  A warp of 32, two of four, two of eight at 32 rows: one user at 4096 tokens
//   11.3, 12.4, 10.3 us; batch 32 at 2048 to 16384 138, 161, 166; batch 64 at 8192 to 32768 552, 643, 710.
// More rows go to the tcgen05 kernel (kv8_attn_tc.cu): at 64 rows two groups of 32 here take 89 us where that takes 68
// (batch 16, 2048 to 8192 tokens), at 40 86 and 67, at 32 55 and 65; batch 64 552 and 666 at 32 rows, 1039 and 681 at 40.
// One user's 64 rows: 9.1 and 13.2 us at 256 tokens, 10.8 and 12.8 at 1024, 15.3 and 14.1 at 4096, 49 and 35 at 32768.
//
// q . k^T and p . v run on mma.m16n8k16 with f16 operands.  An e4m3 code is exact in f16; q is brought
// to f16 by a power of two per row (bf16's 8 bits fit f16's 11, values 2^-14 below the row's largest
// lose bits only below 2^-25 of it).  p is held as 2^6 p relative to a reference that follows the running
// maximum only when that has grown by 2^8, so that the output is seldom rescaled; weights down to 2^-30
// of the largest count.  The pages' scales are powers of two: the keys' joins the score's factor, the
// values' the weight's exponent, relative to a unit, the largest scale met that is within 2^8 of the least (the output is
// rescaled, exactly, when it moves).  Pages that are further above or below would take weights out of f16, theirs or,
// through the unit, all others', whatever the softmax makes of them: a tile with such a page takes bf16 weights
// and codes (f16's range is the reason, not its precision: 2^-8 of each product can be lost for 2^-11; such tiles take a third
// longer: batch 64 at 32 rows 552 us, with every other page apart 722).
//
// The contraction's order is free, so every lane converts what it can load wide: of a key it takes 32
// (16) dimensions side by side, the query rows laid out alike, and of a dimension's values four tokens of
// each page; accumulator columns 2c and 2c + 1 are then token 4c + i of the two pages, which is what
// the lane's value codes want (with the query rows as columns the weights are turned by movmatrix first).  A pad between
// the two pages' keys makes the loads conflict-free.
//
// The block's keys and values (bf16, up to 64) go 16 at a time to the warps of the cluster's last CTA, on
// bf16 operands, the weights in two parts.  The warps' partial (max, sum, output) meet in shared memory, the CTAs' in
// distributed shared memory, each CTA finishing a slice of the rows.
//
// One row at batch 64, 8192 to 32768 tokens (dimension 128, 8 KV heads): 400 us, 6.7 TB/s, the memory's rate.  32 rows
// there: 552 us, 4.9 TB/s: a tile takes an SM 500 cycles, its 128 products 260 of them, the rest latencies that two warps
// a scheduler leave.  One user is latency: at 4096 tokens 2 us to the first tile, 0.8 to 1.3 a tile, 2 to 3 for the parts.
#include <math.h>

#include <type_traits>

#include "cospec_internal.h"
#include "kv8.cuh"
#include "kv8_attn.h"

namespace cospec {

namespace {

// Larger clusters do not all find an SM for each CTA and start later: one user at 4096 tokens took 8.3 us with clusters of
// 12, 9.6 with 14 and 9.2 with 16; with 6 rows of 24 queries 11.7, 13.2 and 12.5.
constexpr int MAX_SPLIT = 12;

// MT > 0: 16 MT rows a warp, padded to the products' rows; MT < 0: 8 NT = -8 MT rows, the products' columns.
template <int D, int MT, int RW, int NW>
struct Lay {
  static constexpr int NT = -MT;
  static constexpr int KW = NW / RW;                      // rings of a CTA, of RW warps
  static constexpr int PB = KV8_PAGE * D;                 // bytes of a page-head
  static constexpr int PADK = D == 128 ? 16 : 64;
  static constexpr int KREG = 2 * PB + PADK;
  static constexpr int STAGE = KREG + 2 * PB;
  static constexpr int CTAS = NW == 8 ? 1 : RW == 2 ? 3 : 2;            // of an SM
  static constexpr int NST = D == 64 || RW == 2 ? 4 : NW == 6 ? 2 : 3;  // tiles of a ring
  static constexpr int RING = NST * STAGE;
  static constexpr int NR = RW * (MT > 0 ? 16 * MT : 8 * NT);
  static constexpr int PD = D + (MT > 0 ? 8 : 4);            // fp32 row of a partial: O, max, sum, unit, flag
  static constexpr int ROWB = PD * 4;
  static constexpr int PART = 0;                          // [KW][NR] rows; the CTA's own result in the first NR
  static constexpr int RECV = KW * NR * ROWB;             // [S][rows per owner], at most NR + 15 rows
  static constexpr int MERGE = RECV + (NR + MAX_SPLIT - 1) * ROWB;
  static constexpr int BODY = KW * RING > MERGE ? KW * RING : MERGE;
  // With many rows a warp the query fragments, the same for all warps, live in shared memory: [MT][D / 16][32 lanes][16 B],
  // [NT][D / 16][32 lanes][8 B]
  static constexpr bool QS = MT > 1 || NT > 2;
  static constexpr int TOTAL = BODY + (QS ? (MT > 0 ? MT * 512 : NT * 256) * (D / 16) : 0);
  static_assert(MT == 1 || RW == 1, "the warps share their query rows, or a ring");
  static_assert(STAGE % 16 == 0 && RING % 16 == 0 && ROWB % 16 == 0, "copies land on 16 bytes");
  static_assert(STAGE >= KV8_PAGE * D * 4, "16 bf16 rows of the block fit a stage");
};

using Params = Kv8Params;

CS_DEV uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
CS_DEV uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
CS_DEV uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}

// The values' scale in whose units outputs and weights count.  Exponents of scales are biased as fp32 holds them; 0: none.
struct Unit {
  int e = 0;                    // of the unit
  int span = 0;                 // exponents in (e - span, e] are met with f16 weights
  int ends = 0;                 // the least exponent so far (0: none yet), 8 bits of the largest
  CS_DEV bool covers(int x) const { return (unsigned)(e - x) < (unsigned)span; }
  CS_DEV float scale() const { return __uint_as_float((uint32_t)e << 23); }
};

// The unit for a tile whose pages have the exponents e0 and e1 (0: no such page; a page of zeros moves none); outputs so far
// are to be multiplied by 2^by.  Returns whether the tile needs bf16 weights.
CS_DEV bool take_scales(Unit& u, int e0, int e1, int& by) {
  const int a0 = e0 > ZERO_EXP ? e0 : 0, a1 = e1 > ZERO_EXP ? e1 : 0;
  const int hi = max(a0, a1), lo = a0 && a1 ? min(a0, a1) : hi, was = u.e;
  if (hi) {
    const int met = u.ends >> 8, least = met ? min(met, lo) : lo, most = max(u.ends & 255, hi), cap = least + V_ROOM;
    u.e = met && was <= cap ? (hi <= cap ? max(was, hi) : was) : (hi <= cap ? hi : least);
    u.span = max(u.e - least + 1, 0);
    if (u.e < most - V_FAR) {
      u.e = most - V_FAR;
      u.span = 0;
    }
    u.ends = least << 8 | most;
  } else if (was == 0 && max(e0, e1) > 0) {
    u.e = ZERO_EXP;
    u.span = 1;
  }
  by = was ? was - u.e : 0;
  return (e0 && !u.covers(e0)) || (e1 && !u.covers(e1));
}
// The same for block rows of exponents from lo to hi (0: zeros alone), whose weights are bf16 in any case: the largest may not
// take the outputs out of fp32, and what the least ones contribute counts beside the pages.
CS_DEV void take_block_scales(Unit& u, int lo, int hi, int& by) {
  const int was = u.e, met = u.ends >> 8, most = max(u.ends & 255, hi);
  u.ends = (met && lo ? min(met, lo) : max(met, lo)) << 8 | most;
  u.e = max(max(was, ZERO_EXP), most - V_FAR);
  u.span = 0;                              // (the next tile finds it)
  by = was ? was - u.e : 0;
}

// What a warp carries from tile to tile: 16 MT rows, this lane's two of each 16 (g and g + 8).
template <int D, int MT>
struct State {
  uint32_t q[MT == 1 ? D / 16 : 1][4];   // f16 queries: the lane's D / 4 dimensions, four a fragment
  uint32_t qs;                  // or where they are in shared memory
  float f[MT][2];               // score factor of a row: its power of two, the softmax scale, log2 e
  float o[MT][D / 8][4];
  float m[MT][2], l[MT][2];     // reference of the weights (base 2), their sum
  Unit v;
  CS_DEV void clear() {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      m[t][0] = m[t][1] = -INFINITY;
      l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) o[t][i][0] = o[t][i][1] = o[t][i][2] = o[t][i][3] = 0.f;
    }
  }
};

// The reference of a row's weights after scores whose largest is mx: it stays while that is less than
// 2^P_ROOM above it.  Where it moves for some row of the warp, sums and outputs follow.
template <int D, int MT>
CS_DEV void follow_max(State<D, MT>& st, int t, float mx0, float mx1, float (&base)[2]) {
  float mx[2] = {mx0, mx1}, a[2];
  bool moved = false;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 1));
    mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 2));
    const float was = st.m[t][r], now = mx[r] > was + P_ROOM ? mx[r] : was;
    moved |= now != was;
    st.m[t][r] = now;
    base[r] = (now == -INFINITY ? 0.f : now) - P_BITS;
    a[r] = exp2_approx(was - P_BITS - base[r]);
  }
  if (__any_sync(0xffffffffu, moved)) {
    st.l[t][0] *= a[0];
    st.l[t][1] *= a[1];
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      st.o[t][i][0] *= a[0];
      st.o[t][i][1] *= a[0];
      st.o[t][i][2] *= a[1];
      st.o[t][i][3] *= a[1];
    }
  }
}

// The same with 8 NT rows, the columns of products whose rows are keys or dimensions; this lane's are 8 t + 2 c and
// 8 t + 2 c + 1.
template <int D, int NT>
struct Cols {
  uint32_t q[NT > 2 ? 1 : NT][D / 16][2];                  // f16 queries of row 8 t + g: the lane's D / 4 dimensions, four a fragment
  uint32_t qs;                  // or where they are in shared memory
  float f[NT][2];               // score factor of a row: its power of two, the softmax scale, log2 e
  float o[NT][D / 16][4];       // dimensions 16 i + g of the two columns, then 16 i + 8 + g
  float m[NT][2], l[NT][2];     // reference of the weights (base 2), their sum
  Unit v;
  CS_DEV void clear() {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      m[t][0] = m[t][1] = -INFINITY;
      l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[t][i][0] = o[t][i][1] = o[t][i][2] = o[t][i][3] = 0.f;
    }
  }
};

template <int D, int NT>
CS_DEV void follow_max(Cols<D, NT>& st, int t, float mx0, float mx1, float (&base)[2]) {
  float mx[2] = {mx0, mx1}, a[2];
  bool moved = false;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
#pragma unroll
    for (int x = 4; x < 32; x *= 2) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], x));
    const float was = st.m[t][e], now = mx[e] > was + P_ROOM ? mx[e] : was;
    moved |= now != was;
    st.m[t][e] = now;
    base[e] = (now == -INFINITY ? 0.f : now) - P_BITS;
    a[e] = exp2_approx(was - P_BITS - base[e]);
  }
  if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      st.l[t][e] *= a[e];
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        st.o[t][i][e] *= a[e];
        st.o[t][i][2 + e] *= a[e];
      }
    }
  }
}
template <int D, int NT>
CS_DEV void rescale(Cols<D, NT>& st, int by) {
  const float a = kv8_two_to(by / 2), b = kv8_two_to(by - by / 2);               // (the whole may lie outside fp32)
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) st.o[t][i][e] = st.o[t][i][e] * a * b;
}
// An 8 x 8 matrix of 16-bit numbers, a row in four lanes, turned.
CS_DEV uint32_t turn8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

template <int D, int MT>
CS_DEV void rescale(State<D, MT>& st, int by) {
  const float a = kv8_two_to(by / 2), b = kv8_two_to(by - by / 2);               // (the whole may lie outside fp32)
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) st.o[t][i][e] = st.o[t][i][e] * a * b;
}

// A page's values' scale joins its weights as an exponent and leaves their sum again.  It joins them no further down than
// 2^-60, where nothing is left of it in f16 but the sum needs the weights; `rest` brings bf16 ones the rest of the way.
struct PageScale {
  float to, back, rest;
  CS_DEV PageScale(float scale, const Unit& u) {
    const int k = (int)(__float_as_uint(scale) >> 23) - u.e, kx = max(k, -60);
    to = (float)kx;
    back = kv8_two_to(-kx);
    rest = exp2f((float)(k - kx));
  }
};
// Two numbers in bf16, and what that leaves of them.
CS_DEV uint32_t two_parts(float a, float b, uint32_t& rest) {
  const uint32_t u = pack_bf16(a, b);
  rest = pack_bf16(a - __uint_as_float(u << 16), b - __uint_as_float(u & 0xffff0000u));
  return u;
}
// One tile: two pages' keys at sk and values at sv, ks / vs their scales, n their tokens (16 both
// unless MASK); wide, with MASK only: with bf16 weights.
template <int D, int MT, bool MASK>
CS_DEV void tile(State<D, MT>& st, uint32_t sk, uint32_t sv, const float (&ks)[2], const float (&vs)[2], int n0, int n1, bool wide, int lane) {
  using L = Lay<D, MT, 1, 4>;
  const int g = lane >> 2, c = lane & 3;
  float s[MT][4][4];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[t][i][0] = s[t][i][1] = s[t][i][2] = s[t][i][3] = 0.f;
  const uint32_t ka = sk + (uint32_t)((g & 1) * (L::PB + L::PADK) + (g >> 1) * 4 * D + c * (D / 4));
#pragma unroll
  for (int x = 0; x < D / 64; ++x) {
    uint32_t w[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 v = lds128(ka + (uint32_t)(i * D + x * 16));
      w[i][0] = v.x;
      w[i][1] = v.y;
      w[i][2] = v.z;
      w[i][3] = v.w;
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      uint32_t a[MT][4];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        if (L::QS) {
          const uint4 v = lds128(st.qs + (uint32_t)((t * (D / 16) + x * 4 + y) * 512));
          a[t][0] = v.x;
          a[t][1] = v.y;
          a[t][2] = v.z;
          a[t][3] = v.w;
        } else {
#pragma unroll
          for (int z = 0; z < 4; ++z) a[t][z] = st.q[L::QS ? 0 : x * 4 + y][z];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t b0 = kv8_f16x2(w[i][y]), b1 = kv8_f16x2_hi(w[i][y]);
#pragma unroll
        for (int t = 0; t < MT; ++t) mma_f16(s[t][i], a[t], b0, b1);
      }
    }
  }
  const PageScale pv[2] = {PageScale(vs[0], st.v), PageScale(vs[1], st.v)};
  uint32_t p[MT][2][4];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    if (MASK) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (4 * c + i >= n0) s[t][i][0] = s[t][i][2] = -INFINITY;
        if (4 * c + i >= n1) s[t][i][1] = s[t][i][3] = -INFINITY;
      }
    }
    float base[2], mx[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float m0 = fmaxf(fmaxf(s[t][0][2 * r], s[t][1][2 * r]), fmaxf(s[t][2][2 * r], s[t][3][2 * r]));
      const float m1 = fmaxf(fmaxf(s[t][0][2 * r + 1], s[t][1][2 * r + 1]), fmaxf(s[t][2][2 * r + 1], s[t][3][2 * r + 1]));
      mx[r] = fmaxf(m0 * (st.f[t][r] * ks[0]), m1 * (st.f[t][r] * ks[1]));     // (NaN, as of -inf and 0, does not count)
    }
    follow_max(st, t, mx[0], mx[1], base);
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float f = st.f[t][r] * ks[e], to = pv[e].to - base[r];
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = exp2_approx(fmaf(s[t][i][2 * r + e], f, to));
          if (MASK && 4 * c + i >= (e ? n1 : n0)) x[i] = 0.f;
        }
        st.l[t][r] = fmaf((x[0] + x[1]) + (x[2] + x[3]), pv[e].back, st.l[t][r]);
        const float w = pv[e].rest;
        p[t][e][r] = MASK && wide ? pack_bf16(x[0] * w, x[1] * w) : pack_f16(x[0], x[1]);
        p[t][e][2 + r] = MASK && wide ? pack_bf16(x[2] * w, x[3] * w) : pack_f16(x[2], x[3]);
      }
  }
  // cells behind a page's last token may hold anything, NaN too: they read as 0
  uint32_t keep[2] = {0xffffffffu, 0xffffffffu};
  if (MASK) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int have = (e ? n1 : n0) - 4 * c;
      keep[e] = have >= 4 ? 0xffffffffu : have <= 0 ? 0u : (1u << (8 * have)) - 1u;
    }
  }
  const uint32_t va = sv + (uint32_t)(g * KV8_PAGE + c * 4);
  auto load = [&](int e, int d) {
    const uint32_t w = lds32(va + (uint32_t)(e * L::PB + d * 8 * KV8_PAGE));
    return MASK ? w & keep[e] : w;
  };
  if (MASK && wide) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int d = 0; d < D / 8; ++d) {
        uint32_t b0, b1;
        kv8_codes_bf16(load(e, d), b0, b1);
#pragma unroll
        for (int t = 0; t < MT; ++t) mma_16816(st.o[t][d], p[t][e], b0, b1);
      }
    return;
  }
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int d = 0; d < D / 8; ++d) {
      const uint32_t w = load(e, d), b0 = kv8_f16x2(w), b1 = kv8_f16x2_hi(w);
#pragma unroll
      for (int t = 0; t < MT; ++t) mma_f16(st.o[t][d], p[t][e], b0, b1);
    }
}

// The same with the rows as columns: keys times rows, then dimensions times rows.  The same loads: here tokens
// 4 (g / 2) + i of page g mod 2 are rows g (i even) and g + 8 (i odd) of the score product i / 2.
template <int D, int NT, bool MASK>
CS_DEV void tile(Cols<D, NT>& st, uint32_t sk, uint32_t sv, const float (&ks)[2], const float (&vs)[2], int n0, int n1, bool wide, int lane) {
  using L = Lay<D, -NT, 1, 4>;
  const int g = lane >> 2, c = lane & 3;
  float s[NT][2][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int j = 0; j < 2; ++j) s[t][j][0] = s[t][j][1] = s[t][j][2] = s[t][j][3] = 0.f;
  const uint32_t ka = sk + (uint32_t)((g & 1) * (L::PB + L::PADK) + (g >> 1) * 4 * D + c * (D / 4));
#pragma unroll
  for (int x = 0; x < D / 64; ++x) {
    uint32_t w[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 v = lds128(ka + (uint32_t)(i * D + x * 16));
      w[i][0] = v.x;
      w[i][1] = v.y;
      w[i][2] = v.z;
      w[i][3] = v.w;
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      uint2 q[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) q[t] = L::QS ? lds64(st.qs + (uint32_t)((t * (D / 16) + x * 4 + y) * 256)) : make_uint2(st.q[L::QS ? 0 : t][x * 4 + y][0], st.q[L::QS ? 0 : t][x * 4 + y][1]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t a[4] = {kv8_f16x2(w[2 * j][y]), kv8_f16x2(w[2 * j + 1][y]), kv8_f16x2_hi(w[2 * j][y]), kv8_f16x2_hi(w[2 * j + 1][y])};
#pragma unroll
        for (int t = 0; t < NT; ++t) mma_f16(s[t][j], a, q[t].x, q[t].y);
      }
    }
  }
  const float kscale = g & 1 ? ks[1] : ks[0];
  const PageScale pv(g & 1 ? vs[1] : vs[0], st.v);
  const int have = (g & 1 ? n1 : n0) - 4 * (g >> 1);       // of this lane's four tokens
  uint32_t p[NT][2][2];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float base[2], mx[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (MASK) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i >= have) s[t][i >> 1][2 * (i & 1) + e] = -INFINITY;
      }
      // (NaN, as of -inf and 0, does not count)
      mx[e] = fmaxf(fmaxf(s[t][0][e], s[t][0][2 + e]), fmaxf(s[t][1][e], s[t][1][2 + e])) * (st.f[t][e] * kscale);
    }
    follow_max(st, t, mx[0], mx[1], base);
    float x[4][2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float f = st.f[t][e] * kscale, to = pv.to - base[e];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i][e] = exp2_approx(fmaf(s[t][i >> 1][2 * (i & 1) + e], f, to));
        if (MASK && i >= have) x[i][e] = 0.f;
      }
      st.l[t][e] = fmaf((x[0][e] + x[1][e]) + (x[2][e] + x[3][e]), pv.back, st.l[t][e]);
    }
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = turn8(MASK && wide ? pack_bf16(x[i][0] * pv.rest, x[i][1] * pv.rest) : pack_f16(x[i][0], x[i][1]));  // row g's weights of token 4 c + i of the two pages
    p[t][0][0] = __byte_perm(w[0], w[1], 0x5410);
    p[t][0][1] = __byte_perm(w[2], w[3], 0x5410);
    p[t][1][0] = __byte_perm(w[0], w[1], 0x7632);
    p[t][1][1] = __byte_perm(w[2], w[3], 0x7632);
  }
  uint32_t keep[2] = {0xffffffffu, 0xffffffffu};           // cells behind a page's last token read as 0
  if (MASK) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int left = (e ? n1 : n0) - 4 * c;
      keep[e] = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
    }
  }
  const uint32_t va = sv + (uint32_t)(g * KV8_PAGE + c * 4);
  auto load = [&](int e, int d) {
    const uint32_t w = lds32(va + (uint32_t)(e * L::PB + d * 8 * KV8_PAGE));
    return MASK ? w & keep[e] : w;
  };
  if (MASK && wide) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint32_t a[4];
        kv8_codes_bf16(load(e, 2 * i), a[0], a[2]);
        kv8_codes_bf16(load(e, 2 * i + 1), a[1], a[3]);
#pragma unroll
        for (int t = 0; t < NT; ++t) mma_16816(st.o[t][i], a, p[t][e][0], p[t][e][1]);
      }
    return;
  }
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const uint32_t w0 = load(e, 2 * i), w1 = load(e, 2 * i + 1);
      const uint32_t a[4] = {kv8_f16x2(w0), kv8_f16x2(w1), kv8_f16x2_hi(w0), kv8_f16x2_hi(w1)};
#pragma unroll
      for (int t = 0; t < NT; ++t) mma_f16(st.o[t][i], a, p[t][e][0], p[t][e][1]);
    }
}

template <int D, int MT, int RW, int NW, bool SEL>
__global__ void __launch_bounds__(NW * 32, Lay<D, MT, RW, NW>::CTAS) kv8_attn_kernel(const Params p) {
  using L = Lay<D, MT, RW, NW>;
  constexpr int NST = L::NST, KW = L::KW;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t recv_bar;
  __shared__ int seq_slot;
  __shared__ int list_end;
  __shared__ float factor[L::QS ? L::NR : 1];
  __shared__ float weight[L::NR + MAX_SPLIT];              // [S][rows per owner]
  const int S = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const int kw = warp / RW, rw = warp % RW;                // ring and group of rows of this warp
  if (tid == 0) {
    mbar_init(&recv_bar, 1);
    fence_barrier_init();
  }
  __syncthreads();
  // Without the stable-cache promise everything waits for the previous kernel; with it only what that
  // kernel may have written (q, the block, sel) does.  Dependents may start only then: one under the
  // promise reads the cache at once.
  if (!p.kv_stable) griddep_wait();
  griddep_launch_dependents();

  // ---------------------------------------------------------------- the unit
  int u = blockIdx.y;
  const int rg = u % p.groups;
  u /= p.groups;
  const int h = u % p.Hkv;
  const int jj = SEL ? u / p.Hkv : 0;                      // block row of the unit
  const int b = p.B > 1 && p.B <= RANK_MAX_B ? sequence_by_rank(p.ctx_len, p.B, (int)blockIdx.z, &seq_slot) : (int)blockIdx.z;
  const int row0 = rg * L::NR, nr = min(L::NR, p.rows - row0);
  const int C = p.ctx_len[b];
  const bool bad = C < 0 || C > p.max_pages * KV8_PAGE;
  if (bad && rank == 0 && blockIdx.y == 0 && tid == 0) set_err(p.err, ERR_CTX);
  const int num = bad ? 0 : (C + KV8_PAGE - 1) / KV8_PAGE;           // pages of the context
  if (SEL && p.kv_stable) griddep_wait();                            // the list comes from the kernel before
  const int32_t* list = SEL ? p.sel + (((size_t)b * p.R + jj) * p.Hkv + h) * p.pages : nullptr;
  int entries = num;
  if (SEL) {                                                         // up to the list's first -1
    if (tid == 0) list_end = bad ? 0 : p.pages;
    __syncthreads();
    for (int i = tid; !bad && i < p.pages; i += NW * 32)
      if (list[i] < 0) {
        atomicMin(&list_end, i);
        break;
      }
    __syncthreads();
    entries = list_end;
  }
  const int tiles = (entries + 1) >> 1, stride = S * KW, mine = rank * KW + kw;
  const int n = mine < tiles ? (tiles - mine + stride - 1) / stride : 0;      // tiles of this ring
  const int32_t* table = p.page_table + (size_t)b * p.max_pages;
  const int block_groups = bad || rank != S - 1 ? 0 : ((SEL && !p.block_full ? jj + 1 : p.R) + 15) / 16;

  // ---------------------------------------------------------------- the stream of tiles
  // Lane 2 i + e holds page e of the ring's i-th next tile: where it is, its tokens, its scales.
  const uint64_t pol = p.groups > 1 || (SEL && p.R > 1) ? l2_policy_evict_normal() : l2_policy_evict_first();
  uint8_t* ring = smem + kw * L::RING;
  int phys = 0, count = 0;                                 // of the 16 tiles being issued
  float2 scale_i = make_float2(0.f, 0.f), scale_c = scale_i;
  int count_c = 0;
  unsigned whole = 0u;                                     // of the 16 being consumed: pages of 16 tokens
  auto look_up = [&](int t0) {                             // tiles t0 .. t0 + 15 of the ring
    const int e = 2 * (mine + (t0 + (lane >> 1)) * stride) + (lane & 1);
    int page = -1;
    if (t0 + (lane >> 1) < n && e < entries) page = SEL ? list[e] : e;
    count = 0;
    scale_i = make_float2(0.f, 0.f);
    if (page >= 0) {
      phys = page < num ? table[page] : -1;
      if ((unsigned)phys < (unsigned)p.num_pages) {
        count = min(KV8_PAGE, C - page * KV8_PAGE);
        scale_i = *reinterpret_cast<const float2*>(p.pool.scale + ((size_t)phys * p.Hkv + h) * 2);
      } else {
        set_err(p.err, ERR_PAGE);
      }
    }
  };
  auto together = [&]() {                                  // the ring's warps
    if (RW == 1) __syncwarp();
    else named_bar_sync(1 + kw, RW * 32);
  };
  auto issue = [&](int t) {                                // this warp's part of the ring's tile t: all of it, or a page
    if ((t & 15) == 0) look_up(t);
    const int at = 2 * (t & 15);
    const unsigned have = __ballot_sync(0xffffffffu, count > 0) >> at;
    const uint32_t dst = smem_u32(ring + (t % NST) * L::STAGE) + lane * 16;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (RW > 1 && e != rw) continue;
      const int ph = __shfl_sync(0xffffffffu, phys, at + e);
      if (have >> e & 1u) {
        const size_t off = ((size_t)ph * p.Hkv + h) * L::PB + lane * 16;
#pragma unroll
        for (int i = 0; i < L::PB; i += 512) kv8_copy16(dst + e * (L::PB + L::PADK) + i, p.pool.k + off + i, pol);
#pragma unroll
        for (int i = 0; i < L::PB; i += 512) kv8_copy16(dst + L::KREG + e * L::PB + i, p.pool.v + off + i, pol);
      }
    }
    kv8_copy_group();
  };
  for (int t = 0; t < NST - 1; ++t) issue(t);
  if (!SEL && p.kv_stable) griddep_wait();
  // Sixteen of the block's rows, into the ring's last stage, which its tiles reach later: keys and then values, 2 D bytes
  // a row, the 16-byte chunks turned by the row against bank conflicts.
  uint8_t* kbuf = ring + (NST - 1) * L::STAGE;
  uint8_t* vbuf = kbuf + KV8_PAGE * D * 2;
  const uint64_t blk_pol = l2_policy_evict_normal();
  auto issue_block = [&](int k0) {
    for (int e = rw * 32 + lane; e < 16 * (D / 8); e += RW * 32) {
      const int r = e / (D / 8), ch = e % (D / 8), at = r * (2 * D) + ((ch ^ (r & 7)) * 16);
      if (k0 + r < p.R) {
        kv8_copy16(smem_u32(kbuf + at), p.k_blk.p + b * p.k_blk.batch + (k0 + r) * p.k_blk.row + (size_t)h * D + ch * 8, blk_pol);
        kv8_copy16(smem_u32(vbuf + at), p.v_blk.p + b * p.v_blk.batch + (k0 + r) * p.v_blk.row + (size_t)h * D + ch * 8, blk_pol);
      } else {
        *reinterpret_cast<uint4*>(kbuf + at) = *reinterpret_cast<uint4*>(vbuf + at) = make_uint4(0u, 0u, 0u, 0u);
      }
    }
    kv8_copy_group();
  };
  if (KW - 1 - kw < block_groups) issue_block((KW - 1 - kw) * 16);

  // ---------------------------------------------------------------- queries
  std::conditional_t<(MT > 0), State<D, (MT > 0 ? MT : 1)>, Cols<D, (MT > 0 ? 1 : L::NT)>> st;
  st.clear();
  st.qs = smem_u32(smem + L::BODY) + lane * (MT > 0 ? 16 : 8);
  auto row_of = [&](int x) { return row0 + min(x, nr - 1); };
  auto q_row = [&](int t) {                                // row 8 t + g, this lane's dimensions
    const int x = 8 * t + g, row = row_of(x);
    const int j = SEL ? jj : row / p.G, head = h * p.G + (SEL ? row : row % p.G);
    return x < nr ? p.q.p + b * p.q.batch + j * p.q.row + (size_t)head * D + c * (D / 4) : nullptr;
  };
  // A row's values of this lane as f16 pairs, dimensions 2 y and 2 y + 1 in v[y], times the inverse of the power of two
  // returned: |q / sc| <= 127.
  auto take = [&](const __nv_bfloat16* src, uint32_t (&v)[D / 8]) {
    uint4 w[D / 32];
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) w[i] = src ? *reinterpret_cast<const uint4*>(src + i * 8) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint32_t ww[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int y = 0; y < 4; ++y)
        amax = fmaxf(amax, fmaxf(kv8_finite_abs(__uint_as_float(ww[y] << 16)), kv8_finite_abs(__uint_as_float(ww[y] & 0xffff0000u))));
    }
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const float sc = kv8_scale127(amax), inv = kv8_inverse(sc);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint32_t ww[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int y = 0; y < 4; ++y) v[4 * i + y] = pack_f16(__uint_as_float(ww[y] << 16) * inv, __uint_as_float(ww[y] & 0xffff0000u) * inv);
    }
    return sc;
  };
  constexpr int MR = MT > 0 ? MT : 1;
  const __nv_bfloat16* qrow[MR][2];
  int lim[MR][2];                                          // last block row that the query row sees
  if constexpr (MT > 0) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int x = (rw * MT + t) * 16 + g + 8 * r, row = row_of(x);
        const int j = SEL ? jj : row / p.G, head = h * p.G + (SEL ? row : row % p.G);
        qrow[t][r] = x < nr ? p.q.p + b * p.q.batch + j * p.q.row + (size_t)head * D + c * (D / 4) : nullptr;
        lim[t][r] = p.block_full ? p.R - 1 : j;
      }
  }
  if constexpr (L::QS) {                                   // eight rows a warp, to all
    constexpr int UNITS = MT > 0 ? 2 * MT : L::NT;
    static_assert(UNITS <= NW, "a warp each");
    if (warp < UNITS) {
      uint32_t v[D / 8];
      const float sc = take(q_row(warp), v);
      if (c == 0) factor[warp * 8 + g] = sc * p.scale_log2;
#pragma unroll
      for (int fr = 0; fr < D / 16; ++fr) {
        if constexpr (MT > 0) {
#pragma unroll
          for (int y = 0; y < 2; ++y)
            *reinterpret_cast<uint32_t*>(smem + L::BODY + ((warp >> 1) * (D / 16) + fr) * 512 + lane * 16 + ((warp & 1) + 2 * y) * 4) = v[2 * fr + y];
        } else {
          *reinterpret_cast<uint2*>(smem + L::BODY + (warp * (D / 16) + fr) * 256 + lane * 8) = make_uint2(v[2 * fr], v[2 * fr + 1]);
        }
      }
    }
    __syncthreads();
    if constexpr (MT > 0) {
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int r = 0; r < 2; ++r) st.f[t][r] = factor[t * 16 + g + 8 * r];
    } else {
#pragma unroll
      for (int t = 0; t < L::NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) st.f[t][e] = factor[8 * t + 2 * c + e];
    }
  } else if constexpr (MT > 0) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      uint32_t v[D / 8];
      st.f[0][r] = take(qrow[0][r], v) * p.scale_log2;
#pragma unroll
      for (int fr = 0; fr < D / 16; ++fr) {
        st.q[fr][r] = v[2 * fr];
        st.q[fr][r + 2] = v[2 * fr + 1];
      }
    }
  } else {
#pragma unroll
    for (int t = 0; t < L::NT; ++t) {
      uint32_t v[D / 8];
      const float sc = take(q_row(t), v);
#pragma unroll
      for (int e = 0; e < 2; ++e) st.f[t][e] = __shfl_sync(0xffffffffu, sc, 8 * c + 4 * e) * p.scale_log2;
#pragma unroll
      for (int fr = 0; fr < D / 16; ++fr) {
        st.q[t][fr][0] = v[2 * fr];
        st.q[t][fr][1] = v[2 * fr + 1];
      }
    }
  }

  // ---------------------------------------------------------------- the block's own rows
  // 16 at a time to the rings, from the last one back.  Their values come as they are, so the weights hold the unit's inverse,
  // in bf16, whose range that takes; what bf16 drops (2^-8, where f16 drops 2^-11) is left over for a second product.
  float odd_values = 0.f;
  for (int kg = KW - 1 - kw; kg < block_groups; kg += KW) {
    const int k0 = kg * 16;
    if (kg >= KW) {
      together();
      issue_block(k0);
    }
    kv8_copy_wait<0>();
    together();
    // The exponents of its values; a lane has half of key lane / 2 (and every warp all of them).
    uint32_t top2 = 0u;                    // largest magnitudes as bits
    auto half_row = [&](bool mend) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const int r = lane >> 1, ch = (lane & 1) * (D / 16) + i;
        uint4* at = reinterpret_cast<uint4*>(vbuf + r * (2 * D) + ((ch ^ (r & 7)) * 16));
        uint4 v = *at;
        if (mend) *at = v = make_uint4(kv8_finite_bf16x2(v.x), kv8_finite_bf16x2(v.y), kv8_finite_bf16x2(v.z), kv8_finite_bf16x2(v.w));
        top2 = __vmaxu2(__vmaxu2(__vmaxu2(top2, v.x & 0x7fff7fffu), v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
      }
      return max(top2 & 0xffffu, top2 >> 16);
    };
    uint32_t vtop = half_row(false);
    if (__any_sync(0xffffffffu, vtop >= 0x7f80u)) {        // not finite: see kv8_add_nonfinite
      top2 = 0u;
      vtop = half_row(true);
      odd_values = 1.f;
      __syncwarp();
    }
    vtop = max(vtop, __shfl_xor_sync(0xffffffffu, vtop, 1));
    const int ve = (int)(__float_as_uint(kv8_scale_of(__uint_as_float(vtop << 16))) >> 23),
              vlo = (int)__reduce_min_sync(0xffffffffu, ve > ZERO_EXP ? (unsigned)ve : 255u), vhi = (int)__reduce_max_sync(0xffffffffu, (unsigned)ve);
    int by;
    take_block_scales(st.v, vhi > ZERO_EXP ? vlo : 0, vhi > ZERO_EXP ? vhi : 0, by);
    if (by != 0) rescale(st, by);
    const float iv = kv8_inverse(st.v.scale());
    if constexpr (MT < 0) {
      float s[L::NT][4];
      const __nv_bfloat16* src[L::NT];
#pragma unroll
      for (int t = 0; t < L::NT; ++t) {
        s[t][0] = s[t][1] = s[t][2] = s[t][3] = 0.f;
        src[t] = q_row(t);
      }
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const uint8_t* kr = kbuf + g * (2 * D) + ((c * (D / 32) + x) ^ g) * 16;
        const uint4 w = *reinterpret_cast<const uint4*>(kr), w8 = *reinterpret_cast<const uint4*>(kr + 8 * 2 * D);
        const uint32_t a0[4] = {w.x, w8.x, w.y, w8.y}, a1[4] = {w.z, w8.z, w.w, w8.w};
#pragma unroll
        for (int t = 0; t < L::NT; ++t) {
          const uint4 qv = src[t] ? *reinterpret_cast<const uint4*>(src[t] + x * 8) : make_uint4(0u, 0u, 0u, 0u);
          mma_16816(s[t], a0, qv.x, qv.y);
          mma_16816(s[t], a1, qv.z, qv.w);
        }
      }
      uint32_t pf[L::NT][2], pr[L::NT][2];
#pragma unroll
      for (int t = 0; t < L::NT; ++t) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // row g + 8 (e / 2) of the keys, this lane's column e mod 2: the last block row that its query row sees
          const int last = p.block_full ? p.R - 1 : SEL ? jj : row_of(8 * t + 2 * c + (e & 1)) / p.G;
          s[t][e] = k0 + g + 8 * (e >> 1) <= last ? s[t][e] * p.scale_log2 : -INFINITY;
        }
        float base[2];
        follow_max(st, t, fmaxf(s[t][0], s[t][2]), fmaxf(s[t][1], s[t][3]), base);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[t][e] = exp2_approx(s[t][e] - base[e & 1]);
          st.l[t][e & 1] += s[t][e];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t rest;
          pf[t][i] = turn8(two_parts(s[t][2 * i] * iv, s[t][2 * i + 1] * iv, rest));
          pr[t][i] = turn8(rest);
        }
      }
      const int key = (lane & 7) + (lane >> 4) * 8;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const int ch = 2 * i + ((lane >> 3) & 1);
        uint32_t a[4];
        ldsm_x4_t(smem_u32(vbuf) + (uint32_t)(key * (2 * D) + ((ch ^ (key & 7)) * 16)), a[0], a[1], a[2], a[3]);
#pragma unroll
        for (int t = 0; t < L::NT; ++t) {
          mma_16816(st.o[t][i], a, pf[t][0], pf[t][1]);
          mma_16816(st.o[t][i], a, pr[t][0], pr[t][1]);
        }
      }
    } else {
      float s[MT][2][4];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) s[t][i][0] = s[t][i][1] = s[t][i][2] = s[t][i][3] = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint8_t* kr = kbuf + (i * 8 + g) * (2 * D);
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
          const uint4 w = *reinterpret_cast<const uint4*>(kr + ((c * (D / 32) + x) ^ g) * 16);
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            uint4 qa = make_uint4(0u, 0u, 0u, 0u), qb = qa;
            if (qrow[t][0]) qa = *reinterpret_cast<const uint4*>(qrow[t][0] + x * 8);
            if (qrow[t][1]) qb = *reinterpret_cast<const uint4*>(qrow[t][1] + x * 8);
            const uint32_t a0[4] = {qa.x, qb.x, qa.y, qb.y}, a1[4] = {qa.z, qb.z, qa.w, qb.w};
            mma_16816(s[t][i], a0, w.x, w.y);
            mma_16816(s[t][i], a1, w.z, w.w);
          }
        }
      }
      uint32_t pf[MT][4], pr[MT][4];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int key = k0 + i * 8 + 2 * c + e;
            s[t][i][e] = key <= lim[t][0] ? s[t][i][e] * p.scale_log2 : -INFINITY;
            s[t][i][2 + e] = key <= lim[t][1] ? s[t][i][2 + e] * p.scale_log2 : -INFINITY;
          }
        float base[2];
        follow_max(st, t, fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][1][0], s[t][1][1])),
                   fmaxf(fmaxf(s[t][0][2], s[t][0][3]), fmaxf(s[t][1][2], s[t][1][3])), base);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[t][i][e] = exp2_approx(s[t][i][e] - base[e >> 1]);
            st.l[t][e >> 1] += s[t][i][e];
          }
#pragma unroll
        for (int i = 0; i < 4; ++i) pf[t][i] = two_parts(s[t][i >> 1][2 * (i & 1)] * iv, s[t][i >> 1][2 * (i & 1) + 1] * iv, pr[t][i]);
      }
      const int key = (lane & 7) + ((lane >> 3) & 1) * 8;
#pragma unroll
      for (int d = 0; d < D / 8; d += 2) {
        const int ch = d + (lane >> 4);
        uint32_t b0, b1, b2, b3;
        ldsm_x4_t(smem_u32(vbuf) + (uint32_t)(key * (2 * D) + ((ch ^ (key & 7)) * 16)), b0, b1, b2, b3);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          mma_16816(st.o[t][d], pf[t], b0, b1);
          mma_16816(st.o[t][d], pr[t], b0, b1);
          mma_16816(st.o[t][d + 1], pf[t], b2, b3);
          mma_16816(st.o[t][d + 1], pr[t], b2, b3);
        }
      }
    }
  }

  // ---------------------------------------------------------------- the cache
  for (int t = 0; t < n; ++t) {
    if ((t & 15) == 0) {
      scale_c = scale_i;                   // (copies run less than NST tiles ahead: still these 16)
      count_c = count;
      whole = __ballot_sync(0xffffffffu, count == KV8_PAGE);
    }
    const int sg = t % NST, at = 2 * (t & 15);
    kv8_copy_wait<NST - 2>();
    together();                            // tile t is there, and every warp is through with tile t - 1
    issue(t + NST - 1);                    // (past the last tile an empty group)
    const float ks[2] = {__shfl_sync(0xffffffffu, scale_c.x, at), __shfl_sync(0xffffffffu, scale_c.x, at + 1)};
    const float vs[2] = {__shfl_sync(0xffffffffu, scale_c.y, at), __shfl_sync(0xffffffffu, scale_c.y, at + 1)};
    const uint32_t sk = smem_u32(ring + sg * L::STAGE);
    constexpr int X = MT < 0 ? L::NT : MT;
    const int e0 = (int)(__float_as_uint(vs[0]) >> 23), e1 = (int)(__float_as_uint(vs[1]) >> 23);
    bool wide = false;
    if (!st.v.covers(e0) || !st.v.covers(e1)) {
      int by;
      wide = take_scales(st.v, e0, e1, by);
      if (by != 0) rescale(st, by);
    }
    if ((whole >> at & 3u) == 3u && !wide) {
      tile<D, X, false>(st, sk, sk + L::KREG, ks, vs, KV8_PAGE, KV8_PAGE, false, lane);
    } else {
      const int n0 = __shfl_sync(0xffffffffu, count_c, at), n1 = __shfl_sync(0xffffffffu, count_c, at + 1);
      if (n0 + n1 > 0) tile<D, X, true>(st, sk, sk + L::KREG, ks, vs, n0, n1, wide, lane);
    }
  }
  kv8_copy_wait<0>();

  // ---------------------------------------------------------------- the warps' parts
  __syncthreads();                         // every ring is idle
  const int rpo = (nr + S - 1) / S;        // rows finished by each CTA of the cluster
  if (S > 1) {
    if (tid == 0) mbar_arrive_expect_tx(&recv_bar, (uint32_t)(S * rpo * L::ROWB));
    cluster_arrive_relaxed();
  }
  float* part = reinterpret_cast<float*>(smem + L::PART);
  {
    // A row: outputs as they are, in the values' unit (a product with it could leave fp32), reference, sum, the unit's exponent.
    const float unit = (float)(st.v.e - 127);
    float* mypart = part + (kw * L::NR + rw * 16) * L::PD;
    if constexpr (MT < 0) {
#pragma unroll
      for (int t = 0; t < L::NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float* row = mypart + (8 * t + 2 * c + e) * L::PD;
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            row[16 * i + g] = st.o[t][i][e];
            row[16 * i + 8 + g] = st.o[t][i][2 + e];
          }
          float l = st.l[t][e];
#pragma unroll
          for (int x = 4; x < 32; x *= 2) l += __shfl_xor_sync(0xffffffffu, l, x);
          if (g == 0) *reinterpret_cast<float4*>(row + D) = make_float4(st.m[t][e], l, unit, odd_values);
        }
    } else {
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float* row = mypart + (t * 16 + g + 8 * r) * L::PD;
#pragma unroll
          for (int d = 0; d < D / 8; ++d)
            *reinterpret_cast<float2*>(row + d * 8 + 2 * c) = make_float2(st.o[t][d][2 * r], st.o[t][d][2 * r + 1]);
          float l = st.l[t][r];
          l += __shfl_xor_sync(0xffffffffu, l, 1);
          l += __shfl_xor_sync(0xffffffffu, l, 2);
          if (c == 0) *reinterpret_cast<float4*>(row + D) = make_float4(st.m[t][r], l, unit, odd_values);
        }
    }
  }
  __syncthreads();
  // A row's KW parts into the first, by a group of D / 4 lanes.
  constexpr int LPR = D / 4;
  static_assert(L::NR % (32 / LPR) == 0, "a warp's rows are all there, or none");
  for (int r0 = 0; r0 < nr; r0 += NW * 32 / LPR) {         // (a last pass may touch rows past nr)
    const int r = r0 + tid / LPR, x = tid % LPR * 4;
    if (r >= L::NR) continue;
    float4 ml[KW];
    float top = -INFINITY, most = -INFINITY;               // of the weights, and of outputs with their units
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      ml[w] = *reinterpret_cast<const float4*>(part + (w * L::NR + r) * L::PD + D);
      top = fmaxf(top, ml[w].x);
      most = fmaxf(most, ml[w].x + ml[w].z);
    }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f, odd = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const bool some = ml[w].x != -INFINITY;
      const float a = some ? exp2_approx(ml[w].x - top) : 0.f, b = some ? exp2_approx(ml[w].x + ml[w].z - most) : 0.f;
      const float4 v = *reinterpret_cast<const float4*>(part + (w * L::NR + r) * L::PD + x);
      acc.x += v.x * b;
      acc.y += v.y * b;
      acc.z += v.z * b;
      acc.w += v.w * b;
      l += ml[w].y * a;
      odd = fmaxf(odd, ml[w].w);
    }
    __syncwarp();                          // every lane of the row has read its maxima and sums
    *reinterpret_cast<float4*>(part + r * L::PD + x) = acc;
    if (x == 0) *reinterpret_cast<float4*>(part + r * L::PD + D) = make_float4(top, l, most - top, odd);
  }
  fence_proxy_async_smem();
  __syncthreads();

  // ---------------------------------------------------------------- the CTAs' parts
  const float* src = part;
  if (S > 1) {
    cluster_wait();                        // every CTA's receiving rows are free, its barrier armed
    float* recv = reinterpret_cast<float*>(smem + L::RECV);
    if (lane == 0) {
      for (int o = warp; o < S; o += NW)
        bulk_copy_s2s(dsmem_map(smem_u32(recv) + (uint32_t)(rank * rpo * L::ROWB), (uint32_t)o), smem_u32(part + o * rpo * L::PD),
                      (uint32_t)(rpo * L::ROWB), dsmem_map(smem_u32(&recv_bar), (uint32_t)o));
    }
    if (!mbar_wait(&recv_bar, 0)) set_err(p.err, ERR_TIMEOUT);
    src = recv;
    cluster_arrive_relaxed();
  }
  const int own0 = rank * rpo;
  for (int r = warp; r < rpo && own0 + r < nr; r += NW) {
    const float4 ml = lane < S ? *reinterpret_cast<const float4*>(src + (lane * rpo + r) * L::PD + D) : make_float4(-INFINITY, 0.f, 0.f, 0.f);
    float top = ml.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const bool some = ml.x != -INFINITY;
    float sum = some ? ml.y * exp2_approx(ml.x - top) : 0.f * ml.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane < S) weight[lane * rpo + r] = sum == 0.f ? 0.f : (some ? exp2f(ml.x - top + ml.z) : 0.f) / sum;    // (0: a skipped sequence)
  }
  __syncthreads();
  for (int e = tid; e < rpo * (D / 4); e += NW * 32) {
    const int r = e / (D / 4), x = e % (D / 4) * 4;
    if (own0 + r >= nr) break;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s = 0; s < S; ++s) {
      const float a = weight[s * rpo + r];
      const float4 v = *reinterpret_cast<const float4*>(src + (s * rpo + r) * L::PD + x);
      acc.x += v.x * a;
      acc.y += v.y * a;
      acc.z += v.z * a;
      acc.w += v.w * a;
    }
    const int row = row0 + own0 + r;
    const int j = SEL ? jj : row / p.G, head = h * p.G + (SEL ? row : row % p.G);
    *reinterpret_cast<uint2*>(p.out + (((size_t)b * p.R + j) * p.Hq + head) * D + x) = make_uint2(pack_bf16(acc.x, acc.y), pack_bf16(acc.z, acc.w));
  }
  // (the block is the last CTA's; its flag came with its rows)
  if (own0 < nr && src[(S - 1) * rpo * L::PD + D + 3] != 0.f) {
    __syncthreads();
    kv8_add_nonfinite(p, D, SEL, jj, b, h, row0 + own0, min(rpo, nr - own0));
  }
  if (S > 1) cluster_wait();               // every copy out of this CTA has landed
}

// What a CTA takes (us): to start and end, and for a tile of each of its lanes (rings, or itself) when few CTAs
// share the device and when all that fit do.  As measured at head dimension 128; the figures of 64 are within a fifth.
struct Cost {
  double start, alone, full;
};
struct Split {
  int S;                                  // CTAs of a unit's cluster
  double us;
};

// The split of the smallest estimate, put together for equal contexts (whole waves) and for contexts that average
// 0.65 of the longest, weighted 0.25 to 0.75 since only the longest is known.
template <typename Resident>
Split split_of(long long units, int tiles, int lanes, Cost c, Resident resident) {
  const double slots = resident(1) > 0 ? resident(1) : device_num_sms();
  Split best = {1, -1.0};
  for (int s = 1; s <= MAX_SPLIT; ++s) {
    if (s > 1 && (s - 1) * lanes >= tiles) break;          // a CTA without a tile
    const int fit = resident(s);
    if (fit < 1) continue;
    const double filled = (double)units * s / slots < 1.0 ? (double)units * s / slots : 1.0;
    const double per = c.full * filled > c.alone ? c.full * filled : c.alone;
    const double longest = c.start + per * ((tiles + s * lanes - 1) / (s * lanes));
    const double waves = (double)((units + fit - 1) / fit);
    const double spread = (double)units / fit * (c.start + per * 0.65 * tiles / (s * lanes));
    const double t = 0.25 * waves * longest + 0.75 * (longest > spread ? longest : spread);
    if (best.us < 0.0 || t < 0.98 * best.us) best = {s, t};           // (a larger split has to be worth it)
  }
  return best;
}

template <int D, int MT, int RW, int NW, bool SEL>
struct Variant {
  using L = Lay<D, MT, RW, NW>;
  static KernelLimits& limits() {
    static KernelLimits lim;
    return lim;
  }
  static void config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute* attr, dim3 grid, int S) {
    cfg.gridDim = grid;
    cfg.blockDim = dim3(NW * 32);
    cfg.dynamicSmemBytes = L::TOTAL;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = S;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
  }
  // Clusters of S CTAs resident at once (cached; the device's answer does not depend on the grid).
  static int resident(int S) {
    static std::atomic<int> cache[KL_MAX_DEV][MAX_SPLIT + 1];
    int dev = 0;
    cudaGetDevice(&dev);
    std::atomic<int>& slot = cache[dev < KL_MAX_DEV ? dev : KL_MAX_DEV - 1][S];
    int c = slot.load(std::memory_order_relaxed);
    if (c == 0) {
      cudaLaunchConfig_t cfg = {};
      cudaLaunchAttribute attr[2];
      config(cfg, attr, dim3(S, 1024, 1), S);
      cfg.numAttrs = 1;
      int n = 0;
      if (ensure_kernel_limits((const void*)kv8_attn_kernel<D, MT, RW, NW, SEL>, limits(), L::TOTAL, true) != cudaSuccess ||
          cudaOccupancyMaxActiveClusters(&n, kv8_attn_kernel<D, MT, RW, NW, SEL>, &cfg) != cudaSuccess) {
        cudaGetLastError();
        n = 0;
      }
      c = n + 1;
      slot.store(c, std::memory_order_relaxed);
    }
    return c - 1;
  }
  static long long units(const Params& p) { return (long long)groups(p) * p.Hkv * (SEL ? p.R : 1) * p.B; }
  static int groups(const Params& p) { return (p.rows + L::NR - 1) / L::NR; }
  static Split split(const Params& p, int tiles) {
    return split_of(units(p), tiles, L::KW,
                    MT == 2   ? Cost{10.0, 1.32, 1.96}
                    : MT == -1 ? Cost{5.5, 0.95, 2.2}
                    : MT == -3 ? Cost{8.3, 1.2, 1.75}
                    : RW == 2 ? (NW == 8 ? Cost{7.3, 1.15, 1.15} : Cost{6.8, 0.88, 2.2})
                              : (NW == 8 ? Cost{7.3, 1.27, 1.27} : Cost{6.0, 0.95, 1.45}),
                    resident);
  }
  static cudaError_t launch(Params& p, int S, cudaStream_t stream) {
    const cudaError_t e = ensure_kernel_limits((const void*)kv8_attn_kernel<D, MT, RW, NW, SEL>, limits(), L::TOTAL, true);
    if (e != cudaSuccess) return e;
    p.groups = groups(p);
    const long long uy = units(p) / p.B;
    if (uy > 65535) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    config(cfg, attr, dim3(S, (unsigned)uy, p.B), S);
    cfg.stream = stream;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kv8_attn_kernel<D, MT, RW, NW, SEL>, p);
  }
};

int resident_tc(int D, int S) {
  static std::atomic<int> cache[KL_MAX_DEV][2][MAX_SPLIT + 1];
  int dev = 0;
  cudaGetDevice(&dev);
  std::atomic<int>& slot = cache[dev < KL_MAX_DEV ? dev : KL_MAX_DEV - 1][D == 128][S];
  int c = slot.load(std::memory_order_relaxed);
  if (c == 0) {
    c = kv8_attn_tc_resident(D, S) + 1;
    slot.store(c, std::memory_order_relaxed);
  }
  return c - 1;
}

template <int D, bool SEL>
cudaError_t pick(Params& p, int pages, cudaStream_t stream) {
  if (!SEL && p.rows > 32 && p.G <= 128) {
    const int jb = 128 / p.G;
    p.groups = (p.R + jb - 1) / jb;
    if ((long long)p.groups * p.Hkv > 65535) return cudaErrorInvalidValue;
    const Split s = split_of((long long)p.groups * p.Hkv * p.B, (pages + 7) / 8, 1, Cost{12.0, 1.03, 1.2}, [](int n) { return resident_tc(D, n); });
    return launch_kv8_attn_tc(p, D, s.S, stream);
  }
  const int tiles = (pages + 1) / 2;
  if (p.rows <= 8) return Variant<D, -1, 1, 6, SEL>::launch(p, Variant<D, -1, 1, 6, SEL>::split(p, tiles).S, stream);
  if (p.rows <= 16) {
    const Split four = Variant<D, 1, 1, 4, SEL>::split(p, tiles), eight = Variant<D, 1, 1, 8, SEL>::split(p, tiles);
    return four.us < eight.us ? Variant<D, 1, 1, 4, SEL>::launch(p, four.S, stream) : Variant<D, 1, 1, 8, SEL>::launch(p, eight.S, stream);
  }
  const Split wide = p.rows <= 24 ? Variant<D, -3, 1, 4, SEL>::split(p, tiles) : Variant<D, 2, 1, 4, SEL>::split(p, tiles);
  const Split four = Variant<D, 1, 2, 4, SEL>::split(p, tiles);
  const Split eight = Variant<D, 1, 2, 8, SEL>::split(p, tiles);
  if (wide.us < four.us && wide.us < eight.us)
    return p.rows <= 24 ? Variant<D, -3, 1, 4, SEL>::launch(p, wide.S, stream) : Variant<D, 2, 1, 4, SEL>::launch(p, wide.S, stream);
  return four.us < eight.us ? Variant<D, 1, 2, 4, SEL>::launch(p, four.S, stream) : Variant<D, 1, 2, 8, SEL>::launch(p, eight.S, stream);
}

}  // namespace

cudaError_t launch_kv8_attn(const Kv8AttnArgs& a, int* err, cudaStream_t stream) {
  Params p{};
  p.pool = a.pool;
  p.q = a.q;
  p.k_blk = a.k_blk;
  p.v_blk = a.v_blk;
  p.page_table = a.page_table;
  p.ctx_len = a.ctx_len;
  p.sel = a.sel;
  p.pages = a.pages;
  p.out = a.out;
  p.B = a.B;
  p.R = a.R;
  p.Hq = a.Hq;
  p.Hkv = a.Hkv;
  p.G = a.Hq / a.Hkv;
  p.num_pages = a.num_pages;
  p.max_pages = a.max_pages;
  p.rows = a.sel ? p.G : p.G * a.R;
  p.scale_log2 = a.scale * 1.4426950408889634f;
  p.kv_stable = a.kv_stable;
  p.block_full = a.block_full;
  p.err = err;
  const int pages = a.sel ? a.pages : (a.max_ctx + KV8_PAGE - 1) / KV8_PAGE;
  if (a.D == 128) return a.sel ? pick<128, true>(p, pages, stream) : pick<128, false>(p, pages, stream);
  return a.sel ? pick<64, true>(p, pages, stream) : pick<64, false>(p, pages, stream);
}

}  // namespace cospec
