// The pages of a long context that each block row reads, chosen by the integer products of the row's
// queries, rounded to 8 bits, with the pages' summaries.
//
// A thread-block cluster owns (sequence, KV head, up to eight block rows): each of its CTAs scores a share of
// the pages for all the rows, so that a summary is read once for them, and then CTA i selects for row i.
// Scores: mma.m16n8k16, 16 pages by 8 query rows.  A summary's byte x becomes the f16 whose bits are x + 128,
// the subnormal (x + 128) 2^-24, a query the integer itself; the accumulator starts at -128 sum(q) 2^-24, and
// all partial sums are multiples of 2^-24 below 1, so exact in fp32.  A lane takes D / 4 dimensions of a page
// straight from memory, the query rows lie alike in shared memory.  The heads of a block row fill 1, 2, 4
// or 8 columns of a tile (the last head repeated), their maximum is taken in the lane and by shuffles, and
// the score goes as an ordered 32-bit key into the shared memory of the row's CTA.
// There the m-th largest key is found among 256 equal steps between the least and the largest score (a
// histogram of leading bits has nearly all of them in a bin or two, whose atomics wait for one another), then by
// eight bits a pass, until 64 keys or fewer are left, which are ranked by comparison; one pass in page order
// writes what lies above it and, of the pages equal to it, the first ones.
//
// One user at 32768 tokens takes 9 us: 1.8 to the queries, 1.2 for the scores, the rest for the m-th key and the list.  64
// sequences at 8192 to 32768 take 29 us: a CTA's step of 256 pages (32 KB of scattered rows) 1.8 us with three CTAs an SM,
// the longest has 8.  16 sequences of 8 rows 32 us: 1024 rows' lists on 456 resident CTAs.
#include "cospec_internal.h"
#include "kv8.cuh"

namespace cospec {

namespace {

constexpr int NW = 8;
constexpr int CT = NW * 32;
constexpr int ROWS = 8;                   // block rows of a cluster
constexpr int MAX_CLUSTER = 16;           // where it fits, else 8 (>= ROWS)
constexpr int STEP = 32;                  // pages that a warp scores at once
constexpr int FEW = 64;                   // keys ranked by comparison

struct Plan {
  int rows;                               // block rows of a cluster: min(R, ROWS)
  int groups;                             // clusters of a (sequence, KV head)
  int log_heads;                          // columns of a tile that a block row's heads fill: 1 to 8 (8 when there are more)
  int tiles_per_row;                      // tiles of a block row where it has more than 8 heads, else 0
  int tiles;
  int S;
  size_t smem;
};

// A float's bits in an order that unsigned comparison follows.
CS_DEV uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
CS_DEV float score_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// The sequence of the launch's z-th slot and its context, longest first (ties in order), so that long ones start early:
// as sequence_by_rank, by all the block's threads over a copy in shared memory (16 sequences of 8 rows 36.3 -> 35.5 us).
CS_DEV int sequence_of(const int32_t* ctx_len, int B, int z, int* room, int& ctx) {
  if (B == 1 || B > RANK_MAX_B) {
    ctx = ctx_len[z];
    return z;
  }
  const int tid = threadIdx.x;
  int mine = 0;
  if (tid < RANK_MAX_B) room[tid] = mine = tid < B ? ctx_len[tid] : (int)0x80000000;
  __syncthreads();
  if (tid < B) {
    int r = 0;
    for (int j = 0; j < B; j += 4) {
      const int4 v = *reinterpret_cast<const int4*>(room + j);
      r += (v.x > mine) | ((v.x == mine) & (j < tid));
      r += (v.y > mine) | ((v.y == mine) & (j + 1 < tid));
      r += (v.z > mine) | ((v.z == mine) & (j + 2 < tid));
      r += (v.w > mine) | ((v.w == mine) & (j + 3 < tid));
    }
    if (r == z) room[RANK_MAX_B] = tid;
  }
  __syncthreads();
  const int b = room[RANK_MAX_B];
  ctx = room[b];
  return b;
}

// KIND: ONE tile for all the rows (a token of up to 8 heads), SOME rows a tile, or a ROW of more than 8 heads over several.
// (Registers decide: in one form, with spills at three CTAs an SM, a token of 64 sequences took 36.4 us for 28.8.)
// CTAS of an SM: with several tiles of dimension 128 three still spill some words, which is worth it where many CTAs wait
// for their turn (16 sequences of 16 rows: 48.8 us, with two 57.6) and not where few do (one user's 6 rows 11.3 and
// 10.2 us, 16 sequences of 4 rows of 64 heads 18.7 and 16.8).
enum { ONE, SOME, ROW };
template <int D, int KIND, int CTAS>
__global__ void __launch_bounds__(CT, CTAS) kv8_select_kernel(const Kv8SelectArgs a, const Plan pl, int* err) {
  const int tiles = KIND == ONE ? 1 : pl.tiles, tiles_per_row = KIND == ROW ? pl.tiles_per_row : 0;
  extern __shared__ __align__(16) uint8_t smem[];
  uint2* qf = reinterpret_cast<uint2*>(smem);              // query fragments [tiles][D / 16][32 lanes]
  float* qsum = reinterpret_cast<float*>(smem + (size_t)tiles * (D / 16) * 256);        // [tiles][8]: where the sums start
  uint32_t* key = reinterpret_cast<uint32_t*>(qsum + tiles * 8);                        // this CTA's row: [pages from lo on]
  __shared__ __align__(16) int slot[RANK_MAX_B + 1];
  __shared__ int amax_bits[ROWS];
  __shared__ int hist[256];
  __shared__ int sums[NW], sums2[NW];
  __shared__ int s_digit, s_left, s_same, s_few;
  __shared__ uint32_t few[FEW], s_key;
  __shared__ float2 range[NW];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const int S = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
  const int h = blockIdx.y % a.Hkv, j0 = (int)(blockIdx.y / a.Hkv) * pl.rows;
  const int nrow = min(pl.rows, a.R - j0), heads = 1 << pl.log_heads;
  griddep_wait();
  griddep_launch_dependents();
  int C;
  const int b = sequence_of(a.ctx_len, a.B, (int)blockIdx.z, slot, C);
  const bool bad = C < 0 || C > a.max_pages * KV8_PAGE;
  if (bad && tid == 0 && rank == 0 && blockIdx.y == 0) set_err(err, ERR_CTX);
  const int num = bad ? 0 : (C + KV8_PAGE - 1) / KV8_PAGE;
  auto list = [&]() { return a.sel + (((size_t)b * a.R + j0 + rank) * a.Hkv + h) * a.pages; };   // of this CTA's row
  if (num <= a.pages) {                    // every page (the same in all CTAs of the cluster)
    int32_t* sel = list();
    if (rank < nrow)
      for (int p = tid; p < a.pages; p += CT) sel[p] = p < num ? p : -1;
    return;
  }
  if (S > 1) cluster_arrive_relaxed();     // this CTA runs: its shared memory may be written
  const int G = a.Hq / a.Hkv;
  const __nv_bfloat16* q = a.q.p + b * a.q.batch + (long long)j0 * a.q.row + (size_t)h * G * D;
  const int lo = min(a.sink, num), hi = max(lo, num - a.recent);   // pages chosen anyway lie outside [lo, hi)
  const int32_t* table = a.page_table + (size_t)b * a.max_pages;
  const int stride = S * NW * STEP;
  int p0 = lo + (rank * NW + warp) * STEP, t0 = 0, t1 = tiles;
  // Where 32 pages a warp leave warps without work (16 sequences of 8 rows: 12 to 32 steps for 64 warps), a warp takes a
  // part of the tiles, of whole rows where a row has several; that is then all it does (35.5 -> 32.5 us).
  const int steps = (hi - lo + STEP - 1) / STEP;
  if (KIND != ONE && 2 * steps <= S * NW) {
    const int row_tiles = max(tiles_per_row, 1), each = tiles / row_tiles, most = min(each, S * NW / steps);
    const int per = (each + most - 1) / most, parts = (each + per - 1) / per, u = rank * NW + warp;
    p0 = u < steps * parts ? lo + u / parts * STEP : hi;
    t0 = u % parts * per * row_tiles;
    t1 = min(tiles, t0 + per * row_tiles);
  }
  // Two steps ahead a lane reads its page's place, one step ahead the warp's summaries and their scales
  // are on their way: nothing waits for a load before the loads that do not need it are out.
  auto look_up = [&](int p) { return p + lane < hi ? table[p + lane] : -1; };
  auto fetch = [&](int ph, int p, uint4 (&w)[4][D / 64], float& scale) {
    const bool ok = (unsigned)ph < (unsigned)a.num_pages;
    if (!ok && p + lane < hi) set_err(err, ERR_PAGE);
#pragma unroll
    for (int i = 0; i < 4; ++i) {          // page i * 8 + g, this lane's dimensions
      const int at = __shfl_sync(0xffffffffu, ok ? ph : 0, i * 8 + g);
      const uint4* s = reinterpret_cast<const uint4*>(a.pool.summary + ((size_t)at * a.Hkv + h) * D + c * (D / 4));
#pragma unroll
      for (int x = 0; x < D / 64; ++x) w[i][x] = s[x];
    }
    scale = ok ? a.pool.summary_scale[(size_t)ph * a.Hkv + h] : __uint_as_float(0x7fffffffu);   // (NaN: no such page)
  };
  // ---------------------------------------------------------------- queries
  // A thread has a column's lane: D / 4 dimensions of a head, four of them a fragment.  (With more than CTA / 32
  // tiles the later columns are read twice.)
  const int cols = tiles * 32;
  auto column = [&](int e, int& j, uint2 (&v)[D / 16]) {
    const int t = e >> 5, col = (e & 31) >> 2;
    j = tiles_per_row ? t / tiles_per_row : (t << (3 - pl.log_heads)) + (col >> pl.log_heads);
    const int head = min(tiles_per_row ? t % tiles_per_row * 8 + col : col & (heads - 1), G - 1);
    const __nv_bfloat16* row = q + j * a.q.row + (size_t)head * D + (e & 3) * (D / 4);
#pragma unroll
    for (int f = 0; f < D / 16; f += 2) {
      uint4 u = make_uint4(0u, 0u, 0u, 0u);
      if (e < cols && j < nrow) u = *reinterpret_cast<const uint4*>(row + f * 4);
      v[f] = make_uint2(u.x, u.y);
      v[f + 1] = make_uint2(u.z, u.w);
    }
  };
  uint2 qv[D / 16];
  int qj;
  column(tid, qj, qv);
  if (tid < ROWS) amax_bits[tid] = 0;
  uint4 w0[4][D / 64];
  float s0;
  int after = look_up(p0), next = look_up(p0 + stride);
  fetch(after, p0, w0, s0);
  __syncthreads();
  for (int e = tid; e < cols; e += CT) {
    if (e != tid) column(e, qj, qv);
    float amax = 0.f;
#pragma unroll
    for (int f = 0; f < D / 16; ++f) {
      float x[4];
      kv8_floats_of(qv[f], x);
#pragma unroll
      for (int i = 0; i < 4; ++i) amax = fmaxf(amax, kv8_finite_abs(x[i]));
    }
    if (qj < nrow) atomicMax(&amax_bits[qj], __float_as_int(amax));
  }
  __syncthreads();
  for (int e = tid; e < cols; e += CT) {   // (a warp: one tile)
    if (cols > CT) column(e, qj, qv);
    const float by = qj < nrow ? kv8_inverse(kv8_scale127(__int_as_float(amax_bits[qj]))) : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int f = 0; f < D / 16; ++f) {
      float v[4];
      kv8_floats_of(qv[f], v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = fabsf(v[i]) <= 3.4028235e38f ? rintf(v[i] * by) : 0.f;
        sum += v[i];
      }
      qf[((e >> 5) * (D / 16) + f) * 32 + lane] = make_uint2(pack_f16(v[0], v[1]), pack_f16(v[2], v[3]));
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    if (c == 0) qsum[(e >> 5) * 8 + g] = sum * -0x1p-17f;           // -128 sum 2^-24
  }
  __syncthreads();
  if (S > 1) cluster_wait();               // every CTA of the cluster runs
  // ---------------------------------------------------------------- scores
  const uint32_t key_addr = smem_u32(key);
  auto place = [&](int j, int p0) {        // where block row j's key of page p0 + g goes (pages past hi: keys that nobody reads)
    const uint32_t at = key_addr + (uint32_t)(p0 - lo + g) * 4u;
    return S > 1 ? dsmem_map(at, (uint32_t)j) : at;
  };
  auto put = [&](uint32_t to, uint32_t k) {
    if (S > 1) dsmem_store_u32(to, k);
    else asm volatile("st.shared.u32 [%0], %1;" ::"r"(to), "r"(k) : "memory");
  };
  // Scores are compared times 2^-24, as the products come: below 2^123 even at the largest scales, exact down to the least that
  // a page with a summary has (2^-115), where the score itself would pass fp32's end and 0 times infinity would be NaN, above
  // every score.  (no -0; key 0, below every score: no such page, or a scale that is not finite)
  auto key_of = [](float dot, float s) { return fabsf(s) <= 3.4028235e38f ? ordered(fmaf(dot, s, 0.f)) : 0u; };
  auto score = [&](int p0, const uint4 (&w)[4][D / 64], float scale) {
    float keep[4] = {0.f, 0.f, 0.f, 0.f};  // of a block row over several tiles
    float sc[4];                           // the scales of this lane's pages g, g + 8, g + 16, g + 24
#pragma unroll
    for (int i = 0; i < 4; ++i) sc[i] = __shfl_sync(0xffffffffu, scale, i * 8 + g);
    for (int t = KIND == ONE ? 0 : t0; t < (KIND == ONE ? 1 : t1); ++t) {
      float acc[2][4];
      const float2 z = *reinterpret_cast<const float2*>(qsum + t * 8 + 2 * c);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        acc[i][0] = acc[i][2] = z.x;
        acc[i][1] = acc[i][3] = z.y;
      }
#pragma unroll
      for (int f = 0; f < D / 16; ++f) {
        const uint2 v = qf[(t * (D / 16) + f) * 32 + lane];
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4& ww = w[i][f / 4];
          y[i] = (f % 4 == 0 ? ww.x : f % 4 == 1 ? ww.y : f % 4 == 2 ? ww.z : ww.w) ^ 0x80808080u;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
          mma_f16(acc[i], __byte_perm(y[2 * i], 0u, 0x4140), __byte_perm(y[2 * i + 1], 0u, 0x4140), __byte_perm(y[2 * i], 0u, 0x4342),
                  __byte_perm(y[2 * i + 1], 0u, 0x4342), v.x, v.y);
      }
      // page g + 8 i: its two columns are parts 2 (i & 1) and 2 (i & 1) + 1 of tile i >> 1
      const int jt = tiles_per_row ? t / tiles_per_row : t << (3 - pl.log_heads);
      if (pl.log_heads == 0) {             // a column is a block row
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int j = jt + 2 * c + e;
          if (j < nrow) {
            const uint32_t to = place(j, p0);
#pragma unroll
            for (int i = 0; i < 4; ++i) put(to + i * 32, key_of(acc[i >> 1][2 * (i & 1) + e], sc[i]));
          }
        }
        continue;
      }
      float best[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        best[i] = fmaxf(acc[i >> 1][2 * (i & 1)], acc[i >> 1][2 * (i & 1) + 1]);
        if (pl.log_heads >= 2) best[i] = fmaxf(best[i], __shfl_xor_sync(0xffffffffu, best[i], 1));
        if (pl.log_heads >= 3) best[i] = fmaxf(best[i], __shfl_xor_sync(0xffffffffu, best[i], 2));
      }
      if (tiles_per_row) {
        const int part = t % tiles_per_row;
#pragma unroll
        for (int i = 0; i < 4; ++i) best[i] = keep[i] = part ? fmaxf(keep[i], best[i]) : best[i];
        if (part + 1 < tiles_per_row) continue;
      }
      // the lanes of a block row (1, 2 or 4) all have its maxima: they share its pages' keys
      const int lanes = heads >> 1, j = jt + (c >> (pl.log_heads - 1));
      if (j < nrow) {
        const uint32_t to = place(j, p0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if ((i & (lanes - 1)) == (c & (lanes - 1))) put(to + i * 32, key_of(best[i], sc[i]));
      }
    }
  };
  for (; p0 < hi; p0 += stride) {
    after = look_up(p0 + 2 * stride);
    score(p0, w0, s0);
    fetch(next, p0 + stride, w0, s0);
    next = after;
  }
  if (S > 1) {
    cluster_arrive();
    cluster_wait();                        // this CTA's row is complete; nothing is written from outside any more
  } else {
    __syncthreads();
  }
  if (rank >= nrow) return;
  // ---------------------------------------------------------------- the m-th largest key
  // 256 equal steps between the smallest and the largest score, then, among the keys of the step that holds the
  // m-th, eight bits a pass: until the few keys left can be ranked against each other.
  int m = a.pages - lo - (num - hi);       // num > pages >= sink + recent: 0 <= m < hi - lo
  const bool none = m == 0;
  const int cnt = hi - lo;
  // Keys are read by fours: one load would wait for the one before it, behind the atomics or the votes.
  auto each_key = [&](auto&& f) {
    for (int p = tid; p < cnt; p += 4 * CT) {
      uint32_t k[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) k[i] = p + i * CT < cnt ? key[p + i * CT] : 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p + i * CT < cnt) f(k[i]);
    }
  };
  float least = INFINITY, most = -INFINITY;
  each_key([&](uint32_t k) {
    if (k == 0u) return;
    least = fminf(least, score_of(k));
    most = fmaxf(most, score_of(k));
  });
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  }
  if (lane == 0) range[warp] = make_float2(least, most);
  __syncthreads();
#pragma unroll
  for (int w2 = 0; w2 < NW; ++w2) {
    least = fminf(least, range[w2].x);
    most = fmaxf(most, range[w2].y);
  }
  const float step = 255.f / (most - least);               // (rounded products keep the order of the scores)
  const bool even = step > 0.f && step <= 3.4028235e38f;   // else one step for all
  auto step_of = [&](uint32_t k) { return even && k != 0u ? min((int)((score_of(k) - least) * step), 255) : 0; };
  uint32_t prefix = 0u, mask = 0u;
  int in_step = 0;
  for (int shift = 32; shift >= 0 && !none; shift -= 8) {  // (32: the steps)
    auto counts = [&](uint32_t k) { return shift == 32 || ((k & mask) == prefix && step_of(k) == in_step); };
    hist[tid] = 0;
    if (tid == 0) s_few = 0;
    __syncthreads();
    each_key([&](uint32_t k) {
      if (counts(k)) atomicAdd(&hist[shift == 32 ? step_of(k) : (int)(k >> shift & 255u)], 1);
    });
    __syncthreads();
    const int n = hist[255 - tid];         // thread t: the t-th digit from the top
    int inc = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    if (lane == 31) sums[warp] = inc;
    __syncthreads();
    int above = inc - n;
#pragma unroll
    for (int w2 = 0; w2 < NW; ++w2) above += w2 < warp ? sums[w2] : 0;
    if (above < m && m <= above + n) {
      s_digit = 255 - tid;
      s_left = m - above;
      s_same = n;
    }
    __syncthreads();
    if (shift == 32) {
      in_step = s_digit;
    } else {
      prefix |= (uint32_t)s_digit << shift;
      mask |= 255u << shift;
    }
    m = s_left;
    const int same = s_same;
    if (same > FEW || shift == 0) continue;
    each_key([&](uint32_t k) {
      if ((k & mask) == prefix && step_of(k) == in_step) few[atomicAdd(&s_few, 1)] = k;
    });
    __syncthreads();
    if (tid < same) {                      // (equal keys find the same answer)
      const uint32_t k = few[tid];
      int more = 0, as_much = 0;
      for (int x = 0; x < same; ++x) {
        more += few[x] > k;
        as_much += few[x] == k;
      }
      if (more < m && m <= more + as_much) {
        s_key = k;
        s_left = m - more;
      }
    }
    __syncthreads();
    prefix = s_key;
    m = s_left;
    break;
  }
  __syncthreads();
  // ---------------------------------------------------------------- the list, in page order
  // A warp has a run of pages: counts first, then their places.
  const int run = (num + CT - 1) / CT * 32, r0 = warp * run, r1 = min(num, r0 + run);
  auto kinds = [&](int p, unsigned (&sure)[4], unsigned (&eq)[4]) {        // of pages p .. p + 127: chosen, equal to the m-th
    uint32_t k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = p + 32 * i + lane;
      k[i] = x >= lo && x < min(hi, r1) ? key[x - lo] : 0u;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = p + 32 * i + lane;
      const bool in = x < r1, own = in && x >= lo && x < hi;
      sure[i] = __ballot_sync(0xffffffffu, own ? !none && k[i] > prefix : in);
      eq[i] = __ballot_sync(0xffffffffu, own && !none && k[i] == prefix);
    }
  };
  int n_sure = 0, n_eq = 0;
  unsigned ms[4], me[4];
  for (int p = r0; p < r1; p += 128) {
    kinds(p, ms, me);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      n_sure += __popc(ms[i]);
      n_eq += __popc(me[i]);
    }
  }
  if (lane == 0) {
    sums[warp] = n_sure;
    sums2[warp] = n_eq;
  }
  __syncthreads();
  int sure = 0, eq = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    sure += w < warp ? sums[w] : 0;
    eq += w < warp ? sums2[w] : 0;
  }
  const unsigned below = (1u << lane) - 1u;
  int32_t* sel = list();
  const int end = a.pages;
  for (int p = r0; p < r1; p += 128) {
    if (r1 - r0 > 128) kinds(p, ms, me);   // (else the first pass left them)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = eq + __popc(me[i] & below);            // equal pages before this one
      const int at = sure + __popc(ms[i] & below) + min(e, m);
      const unsigned in = ms[i] | (e < m ? me[i] : 0u);
      if (in >> lane & 1u && at < end) sel[at] = p + 32 * i + lane;
      sure += __popc(ms[i]);
      eq += __popc(me[i]);
    }
  }
}

void config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute* attr, dim3 grid, size_t smem) {
  cfg.gridDim = grid;
  cfg.blockDim = dim3(CT);
  cfg.dynamicSmemBytes = smem;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = grid.x;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
}

using Kernel = void (*)(const Kv8SelectArgs, const Plan, int*);
constexpr size_t ROOM = 8192;             // shared memory is asked for in these steps (at most 25 of them: 32768 pages)
// Whether a cluster of MAX_CLUSTER CTAs finds room (up to 8 always do, the portable size): the device is asked once for each
// kernel and step of shared memory.
bool largest_fits(Kernel kernel, int which, size_t room) {
  static std::atomic<signed char> cache[KL_MAX_DEV][10][32];         // 0: not asked, 1: it does, -1: it does not
  int dev = 0;
  cudaGetDevice(&dev);
  std::atomic<signed char>& slot = cache[dev < KL_MAX_DEV ? dev : KL_MAX_DEV - 1][which][room / ROOM < 32 ? room / ROOM : 31];
  signed char c = slot.load(std::memory_order_relaxed);
  if (c == 0) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    config(cfg, attr, dim3(MAX_CLUSTER, 1, 1), room);
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
      cudaGetLastError();
      n = 0;
    }
    c = n >= 1 ? 1 : -1;
    slot.store(c, std::memory_order_relaxed);
  }
  return c > 0;
}

template <int D>
cudaError_t launch(const Kv8SelectArgs& a, int* err, cudaStream_t stream) {
  const int G = a.Hq / a.Hkv;
  Plan pl{};
  pl.rows = a.R < ROWS ? a.R : ROWS;
  while ((1 << pl.log_heads) < G && pl.log_heads < 3) ++pl.log_heads;
  pl.tiles_per_row = G > 8 ? (G + 7) / 8 : 0;
  auto tiles = [&]() { return pl.tiles_per_row ? pl.rows * pl.tiles_per_row : ((pl.rows << pl.log_heads) + 7) / 8; };
  // the query fragments take at most 64 KB beside a row's keys
  while (pl.rows > 1 && tiles() * (D / 16) * 256 > 65536) pl.rows = (pl.rows + 1) / 2;
  pl.tiles = tiles();
  pl.groups = (a.R + pl.rows - 1) / pl.rows;
  pl.smem = (size_t)pl.tiles * ((D / 16) * 256 + 32) + ((size_t)a.max_pages + STEP) * 4;
  // A CTA for every row; more where those would not fill the device, with work for every warp.
  const long long clusters = (long long)a.B * a.Hkv * pl.groups;
  pl.S = 1;
  while (pl.S < pl.rows) pl.S *= 2;
  while (pl.S < MAX_CLUSTER && clusters * pl.S < 2 * device_num_sms() && pl.S * NW * STEP < a.max_pages) pl.S *= 2;
  if (a.B > 65535 || (long long)pl.groups * a.Hkv > 65535) return cudaErrorInvalidValue;
  static KernelLimits lim[5];
  const int kind = pl.tiles_per_row ? ROW : pl.tiles == 1 ? ONE : SOME;
  const bool few = D == 128 && kind != ONE && clusters * pl.S <= 4 * device_num_sms();
  constexpr int C2 = D == 128 ? 2 : 3;
  const Kernel kernel = kind == ROW   ? (few ? kv8_select_kernel<D, ROW, C2> : kv8_select_kernel<D, ROW, 3>)
                      : kind == ONE ? kv8_select_kernel<D, ONE, 3>
                                    : (few ? kv8_select_kernel<D, SOME, C2> : kv8_select_kernel<D, SOME, 3>);
  const int variant = kind + (few ? 2 : 0);
  const size_t room = (pl.smem + ROOM - 1) / ROOM * ROOM;
  const cudaError_t e = ensure_kernel_limits((const void*)kernel, lim[variant], room, true);
  if (e != cudaSuccess) return e;
  if (pl.S == MAX_CLUSTER && !largest_fits(kernel, variant + (D == 128 ? 5 : 0), room)) pl.S = MAX_CLUSTER / 2;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  config(cfg, attr, dim3(pl.S, (unsigned)(pl.groups * a.Hkv), a.B), pl.smem);
  cfg.stream = stream;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a, pl, err);
}

}  // namespace

cudaError_t launch_kv8_select(const Kv8SelectArgs& a, int* err, cudaStream_t stream) {
  return a.D == 128 ? launch<128>(a, err, stream) : launch<64>(a, err, stream);
}

}  // namespace cospec
