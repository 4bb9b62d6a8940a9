// Attention over the 8-bit paged cache on the tcgen05 tensor cores, for KV heads that more than 32 query
// rows read.
//
// One CTA owns (sequence, KV head, up to 128 query rows: MMA M, split); the splits of a unit are a
// thread-block cluster and merge in distributed shared memory.  Tile t of 128 keys (8 pages) belongs to
// split t mod S.  Roles by warp:
//   warps 0-6   bring the cache in and convert it, two pages' keys or values at a time, through a ring each: e4m3 to
//               f16 (exact) into the 128-byte-swizzled K-major operand tiles, the keys of a tile ahead of the
//               values of the one before; of the block they make a last tile;
//   warps 8-15  softmax, two groups of four warps (a TMEM lane quarter each): group h has keys 64 h .. 64 h + 63
//               of a tile and its own reference maximum, sum and output accumulator; a thread has a row.  They
//               first bring the query rows to f16 in shared memory;
//   warp 7      issues S = Q K^T (M 128, N 128, K = D) into one of two TMEM score buffers and O_h += P_h V
//               (N = D, K = 64) with P_h in TMEM over its scores.
// The values' pages hold a dimension's tokens side by side, so V too is a K-major operand as it comes.
// The pages' scales are powers of two: the keys' joins the score's factor in the softmax, the values' the
// weight's exponent, relative to a unit; weights are held times 2^6 in f16 and the reference moves when a
// score exceeds it by 2^8, as on mma.sync.  The softmax warps look at the scales of all the CTA's pages first, while
// they convert the queries: the unit is the largest, and where that is more than 2^8 above the least the CTA takes bf16 weights
// and values for all of them (kv8_attn.cu says why; batch 16's 104 rows then take 142 us for 75, batch 64's 64 rows 1783 for
// 680: scales apart are not expected of a model's values, so that loop is kept short, not fast).  The block's keys come to f16 by a power of two per key, its values stay
// bf16 and its weights are two bf16 numbers each, the second what the first leaves over.
//
// 104 rows, batch 16 at 2048 to 8192 tokens: 75 us; 64 rows, batch 64 at 8192 to 32768: 684.  A softmax warp works four fifths
// of a tile's time (a quarter of it on the maxima of 64 keys, two fifths on their weights) beside the converting warps on its
// scheduler, which wait a quarter of theirs for free stages: instructions bound it, and fetching them (the roles' loops share
// an instruction cache: masks and bf16 weights inside them cost a third, the order of the roles in this file up to 4 %); the
// tensor pipe is busy for 20 %, shared memory for 26.  Codes loaded to registers past the ring, behind
// prefetches to L2, cost 10 us, the next tile's scores loaded behind this one's weights 5.
#include <math.h>

#include "cospec_internal.h"
#include "kv8.cuh"
#include "kv8_attn.h"

namespace cospec {

namespace {

constexpr int TK = 128;                   // keys of a tile: MMA N of S
constexpr int TP = TK / KV8_PAGE;         // pages of a tile
constexpr int TM = 128;                   // query rows of a CTA: MMA M
constexpr int CONV = 7;                   // converting warps (16 warps leave each 128 registers)
constexpr int MMA_WARP = 7;
constexpr int SOFT0 = 8;                  // first softmax warp
constexpr int THREADS = 16 * 32;
constexpr int NS = 2;                     // operand stages
constexpr int QB = 2;                     // query rows that a lane group loads at once (1: 73.6 us at 104 rows and batch 16, 2 72.1, 4 75.3, 8 76)
constexpr int SLOTS = 2;                  // pieces (two pages' keys or values) on their way per converting warp
constexpr float TINY = 1.2e-38f;          // a score factor is never 0: -inf stays -inf
constexpr uint64_t WAIT_NS = 2000000000ull;

template <int D>
struct TL {
  static constexpr int H = D / 64;
  static constexpr int PB = KV8_PAGE * D;
  static constexpr int QH = TM * 128;                   // 64 dimensions of the query rows
  static constexpr int KH = TK * 128;                   // 64 dimensions of a tile's keys
  static constexpr int VH = D * 128;                    // 64 keys of a tile's values
  static constexpr int KB = H * KH, VB = 2 * VH;
  static constexpr int TILES = H * QH;                  // [NS]: K then V
  static constexpr int STG = TILES + NS * (KB + VB);    // [CONV][SLOTS]: two pages' keys, or their values
  static constexpr int FAC = STG + CONV * SLOTS * 2 * PB;   // [TM]: the rows' score factors
  static constexpr int MISC = FAC + TM * 4;
  // k_full, v_full, k_empty, v_empty [NS], q_full, s_full [2], p_full [2][2], pv_done [2],
  // mma_done, recv, the values' scales, the block's operands [2]
  static constexpr int NBAR = 4 * NS + 14;
  static constexpr int HOLDER = MISC + NBAR * 8;        // TMEM base, abort, sequence, the exponents' ends [2], the
  static constexpr int BLK = HOLDER + 32;               // block's largest, whether a page is odd, the block keys' scales [64]
  static constexpr int NEED = BLK + 64 * 4;
  static constexpr int PD = D + 4;                      // fp32 row of a partial: O, max, sum, unit, flag
  static constexpr int ROWB = PD * 4;
  static constexpr int PART = 0, RECV = TM * ROWB;      // after the last tile, over everything before MISC
  static constexpr int SCL = RECV + (TM + 15) * ROWB;   // [S][rows per owner]
  static_assert(SCL + (TM + 16) * 4 <= MISC, "the partials fit");
  static constexpr uint32_t OCOL = 2 * TK;
  // one CTA per SM: each wants all of TMEM
  static constexpr int BYTES = (NEED > 118 * 1024 ? NEED : 118 * 1024) + 1024;
  static_assert(BYTES <= 232448, "shared memory of an SM");
};

// (both operands f16, or with `wide` both bf16)
constexpr uint32_t BF16_BOTH = (1u << 7) | (1u << 10);
constexpr uint32_t idesc_f16(int M, int N) { return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24); }

CS_DEV uint4 codes_f16(uint32_t a, uint32_t b) {        // eight codes
  return make_uint4(kv8_f16x2(a), kv8_f16x2_hi(a), kv8_f16x2(b), kv8_f16x2_hi(b));
}
CS_DEV uint4 codes_bf16(uint32_t a, uint32_t b) {       // the same in bf16 (exact)
  uint4 r;
  kv8_codes_bf16(a, r.x, r.y);
  kv8_codes_bf16(b, r.z, r.w);
  return r;
}
CS_DEV float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
CS_DEV float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
CS_DEV float amax8(float m, uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(kv8_finite_abs(bf_lo(w[i])), kv8_finite_abs(bf_hi(w[i]))));
  return m;
}
CS_DEV uint4 scaled8(uint4 v, float inv) {              // eight bf16 to f16, times inv
  return make_uint4(pack_f16(bf_lo(v.x) * inv, bf_hi(v.x) * inv), pack_f16(bf_lo(v.y) * inv, bf_hi(v.y) * inv),
                    pack_f16(bf_lo(v.z) * inv, bf_hi(v.z) * inv), pack_f16(bf_lo(v.w) * inv, bf_hi(v.w) * inv));
}

// Four MMAs of 16 along K in one statement, issued by a converged warp of which one thread (`on`) acts: both operands
// in 128-byte rows (32 bytes on per MMA), or A in TMEM (8 columns on).  Beside fifteen busy warps every instruction
// between two MMAs costs: in a loop an MMA took over 100 cycles to issue.
CS_DEV void umma_k64_on(uint32_t on, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, q, t;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
      " setp.eq.b32 t, %4, %4;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n add.s64 a, %1, 2;\n add.s64 b, %2, 2;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n add.s64 a, %1, 4;\n add.s64 b, %2, 4;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n add.s64 a, %1, 6;\n add.s64 b, %2, 6;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n}\n" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
CS_DEV void umma_tmem_a_k64_on(uint32_t on, uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, q, t;\n .reg .b64 b;\n .reg .b32 a;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
      " setp.eq.b32 t, %4, %4;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n add.s32 a, %1, 8;\n add.s64 b, %2, 2;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n add.s32 a, %1, 16;\n add.s64 b, %2, 4;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n add.s32 a, %1, 24;\n add.s64 b, %2, 6;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}

// What only some tiles need has loops of its own: those of all roles have to stay in the instruction cache together.
//
// Two pages' values, piece e of a tile, `have` tokens of each; cells behind a page's last token may hold anything: they enter
// as 0.  In f16, or `wide` in bf16.
template <int D>
CS_DEV void convert_values(const uint8_t* src, uint8_t* vt, int e, int have0, int have1, bool wide) {
  const int lane = threadIdx.x & 31;
  uint8_t* dst = vt + (e >> 1) * TL<D>::VH + lane * 128;
#pragma unroll 1
  for (int i = 0; i < 2 * (D / 32); ++i) {
    const int x = i & 1, y = i >> 1, have = x ? have1 : have0, at = ((e & 1) * 4 + 2 * x) ^ (lane & 7);
    const uint4 v = *reinterpret_cast<const uint4*>(src + x * TL<D>::PB + (y * 32 + lane) * KV8_PAGE);
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int m = have - 4 * k;
      w[k] &= m >= 4 ? 0xffffffffu : m <= 0 ? 0u : (1u << (8 * m)) - 1u;
    }
    *reinterpret_cast<uint4*>(dst + y * 32 * 128 + at * 16) = wide ? codes_bf16(w[0], w[1]) : codes_f16(w[0], w[1]);
    *reinterpret_cast<uint4*>(dst + y * 32 * 128 + (at ^ 1) * 16) = wide ? codes_bf16(w[2], w[3]) : codes_f16(w[2], w[3]);
  }
}

CS_DEV void tq_ld8(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])::"memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
CS_DEV void tq_st4(uint32_t taddr, const uint32_t (&v)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
// A softmax thread's row and reference, sum and unit.
struct RowState {
  float m, l;
  int unit, ok;
};
// Half a tile that is not all of pages in the ordinary way, in parts of 8 keys: of a context's end or with a page that is not
// of the pool (weights in f16), of pages whose scales lie apart (`wide`: bf16), or of the block (`key_scale`), whose values
// come as they are, so that the unit's inverse is with the weights, in bf16, and what that drops is left over for a second
// product; they are at most 448 times the scale of exponent `most`.  Page c's scales are in lane 4 (t mod 8) + c, the keys'
// below 0 for one that is not of the pool.  Keys 0 .. lim are seen.  The output so far is at `orow`, complete with phase t - 1 of
// pv_bar.
template <int D>
CS_DEV RowState soft_parts(uint32_t srow, uint32_t orow, int parts, int lim, float f, float2 scales, bool wide,
                           const float* key_scale, int most, uint64_t* pv_bar, int t, RowState st) {
  const bool blk = key_scale != nullptr;
  auto scores = [&](int c, float (&x)[8]) {
    tq_ld8(srow + c * 8, x);
    const float ks = __shfl_sync(0xffffffffu, scales.x, (t & 7) * 4 + (c >> 1)), fk = blk ? f : fmaxf(f * ks, TINY);
    const int last = blk || ks >= 0.f ? lim - 8 * c : -1;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float y = x[k] * (blk ? fk * key_scale[8 * c + k] : fk);
      x[k] = k <= last ? y : -INFINITY;
    }
  };
  float x[8], mx = -INFINITY, alpha = 1.f;
#pragma unroll 1
  for (int c = 0; c < parts; ++c) {
    scores(c, x);
#pragma unroll
    for (int k = 0; k < 8; ++k) mx = fmaxf(mx, x[k]);
  }
  if (mx > st.m + P_ROOM) {
    alpha = st.m == -INFINITY ? 0.f : exp2_approx(st.m - mx);
    st.m = mx;
    st.l *= alpha;
  }
  if (blk) {                                              // its values may not take the outputs out of fp32
    const int was = st.unit, far = most - V_FAR;
    st.unit = max(max(was, ZERO_EXP), was ? min(far, was + 126) : far);
    if (was) alpha *= kv8_two_to(was - st.unit);
  }
  st.ok = 1;
  if (__any_sync(0xffffffffu, alpha != 1.f && t > 0)) {
    st.ok = __all_sync(0xffffffffu, mbar_wait(pv_bar, (uint32_t)(t - 1) & 1u, WAIT_NS));
    tc_fence_after();
    if (st.ok) {
#pragma unroll 1
      for (int c = 0; c < D / 8; ++c) {
        tq_ld8(orow + c * 8, x);
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(x[k] * alpha);
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(orow + c * 8), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                     "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
      }
    }
  }
  const float nb = P_BITS - (st.m == -INFINITY ? 0.f : st.m);
#pragma unroll 1
  for (int c = 0; c < parts; ++c) {
    scores(c, x);
    // (no further down than 2^-60, which the sum needs; the rest of the way by a factor)
    const float vs = __shfl_sync(0xffffffffu, scales.y, (t & 7) * 4 + (c >> 1));
    const int k0 = blk ? 127 - st.unit : (int)(__float_as_uint(vs) >> 23) - st.unit, kx = blk ? 0 : max(k0, -60);
    const float to = nb + (float)kx, w = kv8_two_to(max(k0 - kx, -127));
    float sum = 0.f;
    uint32_t pk[4], rest[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float a = exp2_approx(x[2 * k] + to), b = exp2_approx(x[2 * k + 1] + to);
      sum += a + b;
      pk[k] = blk || wide ? pack_bf16(a * w, b * w) : pack_f16(a, b);
      rest[k] = pack_bf16(fmaf(a, w, -bf_lo(pk[k])), fmaf(b, w, -bf_hi(pk[k])));
    }
    st.l = fmaf(sum, kv8_two_to(-kx), st.l);
    tq_st4(srow + c * 4, pk);                             // over scores that have been read
    if (blk) tq_st4(srow + 64 + c * 4, rest);             // the other half's, which the block does not use
  }
  return st;
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1) kv8_attn_tc_kernel(const Kv8Params p) {
  using L = TL<D>;
  constexpr int H = L::H, PD = L::PD;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + L::MISC);
  uint64_t* v_full = k_full + NS;
  uint64_t* k_empty = v_full + NS;
  uint64_t* v_empty = k_empty + NS;
  uint64_t* q_full = v_empty + NS;
  uint64_t* s_full = q_full + 1;            // [2]
  uint64_t* p_full = s_full + 2;            // [2 buffers][2 halves]
  uint64_t* pv_done = p_full + 4;           // [2]
  uint64_t* mma_done = pv_done + 2;
  uint64_t* recv_bar = mma_done + 1;
  uint64_t* ends_bar = recv_bar + 1;        // the least and the largest exponent of the pages' values are there
  uint64_t* blk_done = ends_bar + 1;        // [2]: the block's keys and their scales, its values have been written
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem + L::HOLDER);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  volatile int* seq_slot = abort_flag + 1;
  volatile int* odd_values = seq_slot + 1;                         // the block has values that are not finite
  int* ends = reinterpret_cast<int*>(smem + L::HOLDER + 16);       // least (255: no page), largest (0)
  int* blk_most = ends + 2;                                        // the same of the block's values
  int* odd = ends + 3;                                             // a page is not of the pool, or has no scale
  float* blk_scale = reinterpret_cast<float*>(smem + L::BLK);

  const int S = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
  const int h = blockIdx.y / p.groups, rg = blockIdx.y % p.groups;
  const int jb = TM / p.G, j0 = rg * jb;                 // block rows of a group
  const int NR = min(jb, p.R - j0) * p.G;                // query rows
  const int nsw = (NR + 31) >> 5;                        // softmax warps of a group that own rows
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(&k_full[s], TP / 2);        // two pages each
      mbar_init(&v_full[s], TP / 2);
      mbar_init(&k_empty[s], 1);
      mbar_init(&v_empty[s], 1);
    }
    mbar_init(q_full, 8);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[2 * i], (uint32_t)nsw);
      mbar_init(&p_full[2 * i + 1], (uint32_t)nsw);
      mbar_init(&pv_done[i], 1);
    }
    mbar_init(mma_done, 1);
    mbar_init(recv_bar, 1);
    mbar_init(ends_bar, 8);
    mbar_init(&blk_done[0], CONV);
    mbar_init(&blk_done[1], CONV);
    *abort_flag = 0;
    ends[0] = 255;
    ends[1] = *blk_most = *odd = *odd_values = 0;
    fence_barrier_init();
  }
  if (warp == MMA_WARP) {
    tmem_alloc(tmem_holder, 512u);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  // (the stable-cache promise: as in kv8_attn_kernel)
  if (!p.kv_stable) griddep_wait();
  griddep_launch_dependents();
  const int b = p.B > RANK_MAX_B ? sequence_in_order(p.ctx_len, p.B, (int)blockIdx.z)
                : p.B > 1        ? sequence_by_rank(p.ctx_len, p.B, (int)blockIdx.z, seq_slot)
                                 : (int)blockIdx.z;
  const int C = p.ctx_len[b];
  const bool bad = C < 0 || C > p.max_pages * KV8_PAGE;
  if (bad && rank == 0 && blockIdx.y == 0 && tid == 0) set_err(p.err, ERR_CTX);
  const int num = bad ? 0 : (C + KV8_PAGE - 1) / KV8_PAGE;
  const int tiles = (num + TP - 1) / TP;
  const int n = rank < tiles ? (tiles - rank + S - 1) / S : 0;       // cache tiles of this CTA
  const bool do_blk = !bad && rank == S - 1;
  const int T = n + (do_blk ? 1 : 0);
  const int KBR = (p.R + 15) & ~15;
  const int32_t* table = p.page_table + (size_t)b * p.max_pages;
  float mref = -INFINITY, l = 0.f, vref = 0.f;            // softmax threads: of this row and half
  // (once they are there)
  auto is_wide = [&]() { return *(volatile int*)(ends + 1) - *(volatile int*)ends > V_ROOM; };
  auto is_odd = [&]() { return is_wide() || *(volatile int*)odd != 0; };
  const bool cut = (rank + (n - 1) * S) * TK + TK > C;    // the last cache tile is not all of the context's keys

  if (warp == MMA_WARP) {
    // ---------------------------------------------------------------- MMA
    if (T > 0) {
      const uint32_t on = elect_one();
      const uint32_t sbase = smem_u32(smem);
      const uint64_t q_desc = smem_desc_sw128(sbase), k_desc = smem_desc_sw128(sbase + L::TILES);
      constexpr uint64_t STAGE16 = (uint64_t)((L::KB + L::VB) >> 4);
      bool ok = __all_sync(0xffffffffu, mbar_wait(q_full, 0, WAIT_NS) && mbar_wait(ends_bar, 0, WAIT_NS));
      const bool wide = is_wide();
      tc_fence_after();
      auto issue_s = [&](int t) {
        const int nk = do_blk && t == n ? KBR : TK;
        const uint64_t kd = k_desc + (uint64_t)(t % NS) * STAGE16;
        const uint32_t dst = tmem + (uint32_t)((t & 1) * TK), id = idesc_f16(TM, nk);
#pragma unroll
        for (int x = 0; x < H; ++x)
          umma_k64_on(on, dst, q_desc + (uint64_t)(x * (L::QH >> 4)), kd + (uint64_t)(x * (L::KH >> 4)), id, x ? 1u : 0u);
        umma_commit_on(on, &k_empty[t % NS]);
        umma_commit_on(on, &s_full[t & 1]);
      };
      auto issue_pv = [&](int u, int x) {
        const uint64_t vd = k_desc + (uint64_t)(u % NS) * STAGE16 + (uint64_t)((L::KB + x * L::VH) >> 4);
        const uint32_t src = tmem + (uint32_t)((u & 1) * TK + x * 64), dst = tmem + L::OCOL + (uint32_t)(x * D);
        if (do_blk && u == n) {
#pragma unroll 1
          for (int ks = 0; ks < KBR / 16; ++ks) {         // the weights' first parts, then the second
            umma_bf16_tmem_a_on(on, dst, src + (uint32_t)(ks * 8), vd + (uint64_t)(ks * 2), idesc_f16(TM, D) | BF16_BOTH, (u | ks) != 0 ? 1u : 0u);
            umma_bf16_tmem_a_on(on, dst, src + (uint32_t)(64 + ks * 8), vd + (uint64_t)(ks * 2), idesc_f16(TM, D) | BF16_BOTH, 1u);
          }
        } else {
          if (wide) umma_tmem_a_k64_on(on, dst, src, vd, idesc_f16(TM, D) | BF16_BOTH, u ? 1u : 0u);
          else umma_tmem_a_k64_on(on, dst, src, vd, idesc_f16(TM, D), u ? 1u : 0u);
        }
        umma_commit_on(on, &pv_done[x]);
      };
      // A fixed order with waits that sleep: S of tile t + 2 takes the buffer that the products of tile t read (as P), and
      // goes behind them.  (A loop that polled for whatever was ready took 250 to 500 cycles a turn beside the busy
      // converting and softmax warps: 118 -> 92 us at batch 16, K = 25.)
      auto wait = [&](uint64_t* bar, int phase) { ok = ok && mbar_wait(bar, (uint32_t)phase & 1u, WAIT_NS); };
      for (int t = 0; t < min(T, 2); ++t) {
        wait(&k_full[t % NS], t / NS);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        tc_fence_after();
        issue_s(t);
      }
      for (int t = 0; t < T && ok; ++t) {
        wait(&v_full[t % NS], t / NS);
        wait(&p_full[2 * (t & 1)], t >> 1);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        tc_fence_after();
        issue_pv(t, 0);
        if (t < n) {                                      // (the block's keys are all in half 0)
          wait(&p_full[2 * (t & 1) + 1], t >> 1);
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
          tc_fence_after();
          issue_pv(t, 1);
        }
        umma_commit_on(on, &v_empty[t % NS]);
        if (t + 2 < T) {
          wait(&k_full[t % NS], t / NS + 1);
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
          tc_fence_after();
          issue_s(t + 2);
        }
      }
      if (!ok && on) {
        set_err(p.err, ERR_TIMEOUT);
        *abort_flag = 1;
      }
      umma_commit_on(on, mma_done);
      mbar_wait(mma_done, 0, WAIT_NS);
    }
  } else if (warp < CONV) {
    // ---------------------------------------------------------------- cache in, to f16
    // The work is pieces of two pages' keys or values, four to a group: the keys of tile 0, then for every tile t the
    // keys of t + 1 and the values of t, so that scores run ahead.  Piece u is warp u mod CONV's.  (Its fixed part,
    // waits, fences and addresses, is as long as the conversion of a page: pages one by one took 2500 cycles a tile.)
    constexpr int GP = TP / 2;                            // pieces of a group
    constexpr int NX = D / 32;                            // 16-byte parts of a lane per page
    constexpr uint32_t NONE = 0xffffffffu;
    uint8_t* ring = smem + L::STG + warp * (SLOTS * 2 * L::PB);
    const uint64_t pol = p.groups > 1 ? l2_policy_evict_normal() : l2_policy_evict_first();
    const int total = n > 0 ? (GP * (2 * n + 1) - warp + CONV - 1) / CONV : 0;     // pieces of this warp
    auto piece = [&](int k, bool& values, int& t, int& e) {
      const int u = warp + k * CONV, grp = u / GP;
      values = grp > 0 && !(grp & 1);
      t = values ? grp / 2 - 1 : (grp + 1) / 2;
      e = u % GP;
    };
    // Lane 2 i + x: page x of piece k0 + i, as its place among the pool's page-heads, and its tokens.
    uint32_t cell = NONE;
    int count = 0, count_c = 0;
    auto look_up = [&](int k0) {
      bool values;
      int t, e;
      piece(k0 + (lane >> 1), values, t, e);
      const int page = (rank + t * S) * TP + 2 * e + (lane & 1);
      count = 0;
      cell = NONE;
      if (k0 + (lane >> 1) < total && t < n && page < num) {
        const int phys = table[page];
        if ((unsigned)phys < (unsigned)p.num_pages) {
          count = min(KV8_PAGE, C - page * KV8_PAGE);
          cell = (uint32_t)phys * (uint32_t)p.Hkv + (uint32_t)h;
        } else {
          set_err(p.err, ERR_PAGE);
        }
      }
    };
    auto issue = [&](int k) {                             // one group, empty where there are no such pages
      if ((k & 15) == 0) look_up(k);
      bool values;
      int t, e;
      piece(k, values, t, e);
      const uint8_t* pool = (values ? p.pool.v : p.pool.k) + lane * 16;
      const uint32_t dst = smem_u32(ring + (k % SLOTS) * 2 * L::PB) + lane * 16;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const uint32_t at = __shfl_sync(0xffffffffu, cell, 2 * (k & 15) + x);
        if (at != NONE)
#pragma unroll
          for (int i = 0; i < L::PB; i += 512) kv8_copy16(dst + x * L::PB + i, pool + (size_t)at * L::PB + i, pol);
      }
      kv8_copy_group();
    };
    bool ok = true, wide = false;
    auto wait = [&](uint64_t* bar, int phase) { ok = ok && mbar_wait(bar, (uint32_t)phase & 1u, WAIT_NS); };
    // (`plain`: full pages of values, to f16)
    auto convert = [&](int k, bool plain) {
      if ((k & 15) == 0) count_c = count;                 // (copies run at most SLOTS ahead: still these 16)
      bool values;
      int t, e;
      piece(k, values, t, e);
      if (t >= n) return;                                 // (the keys after the last tile's: nothing)
      const int st = t % NS;
      uint8_t* kt = smem + L::TILES + st * (L::KB + L::VB);
      uint8_t* vt = kt + L::KB;
      const uint8_t* src = ring + (k % SLOTS) * 2 * L::PB;
      kv8_copy_wait<SLOTS - 1>();
      __syncwarp();
      uint4 v[2][NX];                                     // (all loads before the first store)
      if (t >= NS) wait(values ? &v_empty[st] : &k_empty[st], t / NS - 1);
      if (!values) {
        // a lane: 16 dimensions (chunk ch of the key's row) of every (512 / D)-th key; the two 16-byte halves in an order
        // that spreads a quarter-warp over all banks
        constexpr int CH = D / 16, KPI = 32 / CH;
        static_assert(NX == KV8_PAGE / KPI, "a page is as many loads either way");
        const int ch = lane % CH;
        const bool flip = H == 2 && ch >= 4;
#pragma unroll
        for (int x = 0; x < 2 * NX; ++x) v[x / NX][x % NX] = *reinterpret_cast<const uint4*>(src + (x * KPI + lane / CH) * D + ch * 16);
        uint8_t* dst = kt + (ch >> 2) * L::KH + (e * 2 * KV8_PAGE + lane / CH) * 128;
#pragma unroll
        for (int x = 0; x < 2 * NX; ++x) {
          const int at = ((ch & 3) * 2 + (flip ? 1 : 0)) ^ ((x * KPI + lane / CH) & 7);
          const uint4& w = v[x / NX][x % NX];
          *reinterpret_cast<uint4*>(dst + x * KPI * 128 + at * 16) = codes_f16(flip ? w.z : w.x, flip ? w.w : w.y);
          *reinterpret_cast<uint4*>(dst + x * KPI * 128 + (at ^ 1) * 16) = codes_f16(flip ? w.x : w.z, flip ? w.y : w.w);
        }
      } else if (!plain) {
        convert_values<D>(src, vt, e, __shfl_sync(0xffffffffu, count_c, 2 * (k & 15)), __shfl_sync(0xffffffffu, count_c, 2 * (k & 15) + 1), wide);
      } else {
        // a lane: 16 tokens of every 32nd dimension
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
          for (int y = 0; y < NX; ++y) v[x][y] = *reinterpret_cast<const uint4*>(src + x * L::PB + (y * 32 + lane) * KV8_PAGE);
        }
        uint8_t* dst = vt + (e >> 1) * L::VH + lane * 128;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int at = ((e & 1) * 4 + 2 * x) ^ (lane & 7);
#pragma unroll
          for (int y = 0; y < NX; ++y) {
            *reinterpret_cast<uint4*>(dst + y * 32 * 128 + at * 16) = codes_f16(v[x][y].x, v[x][y].y);
            *reinterpret_cast<uint4*>(dst + y * 32 * 128 + (at ^ 1) * 16) = codes_f16(v[x][y].z, v[x][y].w);
          }
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(values ? &v_full[st] : &k_full[st]);
    };
    for (int k = 0; k < SLOTS; ++k) issue(k);
    int k = 0, few = total - (cut && total > 0 && (warp + (total - 1) * CONV) / GP == 2 * n ? 1 : 0);   // pieces of whole pages
    bool go = true;
#pragma unroll 1
    for (; go && k < few; ++k) {
      convert(k, true);
      issue(k + SLOTS);                                   // (the slot has been read)
      if (k == 0) {                                       // (a warp's first piece is of keys)
        wait(ends_bar, 0);
        wide = is_wide();
        if (is_odd()) few = 1;
      }
      if ((k & 7) == 7) go = __all_sync(0xffffffffu, ok && !*abort_flag);     // (a wait that ran out makes the rest useless)
    }
#pragma unroll 1
    for (; go && k < total; ++k) {
      convert(k, false);
      issue(k + SLOTS);
      if ((k & 7) == 7) go = __all_sync(0xffffffffu, ok && !*abort_flag);
    }
    ok = go && ok;
    kv8_copy_wait<0>();                                   // no copy may be in flight when the ring is reused
    auto wait_all = [&](uint64_t* bar, int phase) {
      ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, (uint32_t)phase & 1u, WAIT_NS)) && !*abort_flag;
      return ok;
    };
    // ---------------------------------------------------------------- the block
    if (p.kv_stable) griddep_wait();
    if (ok && do_blk) {
      const int st = n % NS;
      uint8_t* kt = smem + L::TILES + st * (L::KB + L::VB);
      uint8_t* vt = kt + L::KB;
      const __nv_bfloat16* kb = p.k_blk.p + b * p.k_blk.batch + (size_t)h * D;
      const __nv_bfloat16* vb = p.v_blk.p + b * p.v_blk.batch + (size_t)h * D;
      if (ok && (n < NS || wait_all(&k_empty[st], n / NS - 1))) {
        // a group of D / 8 lanes takes a row
        float vm = 0.f;
#pragma unroll 1
        for (int e0 = warp * 32; e0 < p.R * (D / 8); e0 += CONV * 32) {
          const int row = (e0 + lane) / (D / 8), ch = lane % (D / 8);
          const bool live = row < p.R;
          uint4 k = make_uint4(0u, 0u, 0u, 0u), v = k;
          if (live) {
            k = *reinterpret_cast<const uint4*>(kb + row * p.k_blk.row + ch * 8);
            v = *reinterpret_cast<const uint4*>(vb + row * p.v_blk.row + ch * 8);
          }
          float km = amax8(0.f, k);
          vm = amax8(vm, v);
#pragma unroll
          for (int o = D / 16; o > 0; o >>= 1) km = fmaxf(km, __shfl_xor_sync(0xffffffffu, km, o));
          const float ks = kv8_scale_of(km);
          if (live) *reinterpret_cast<uint4*>(kt + (ch >> 3) * L::KH + row * 128 + (((ch & 7) ^ (row & 7)) * 16)) = scaled8(k, kv8_inverse(ks));
          if (live && ch == 0) blk_scale[row] = ks;
        }
        const unsigned most = __reduce_max_sync(0xffffffffu, __float_as_uint(kv8_scale_of(vm)) >> 23);
        if (lane == 0) atomicMax(blk_most, (int)most);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&blk_done[0]);
        if (warp < TP / 2) {                                // (a quarter of a tile each, once all have written)
          wait_all(&blk_done[0], 0);
          if (lane == 0 && ok) mbar_arrive(&k_full[st]);
        }
      }
      if (ok && (n < NS || wait_all(&v_empty[st], n / NS - 1))) {
        // two rows' eight dimensions turned into eight dimensions' two keys; rows from R on are zeros
#pragma unroll 1
        for (int e = tid; e < KBR / 2 * (D / 8); e += CONV * 32) {
          const int j = e / (D / 8) * 2, d = e % (D / 8) * 8;
          uint4 a = make_uint4(0u, 0u, 0u, 0u), c = a;
          if (j < p.R) a = *reinterpret_cast<const uint4*>(vb + j * p.v_blk.row + d);
          if (j + 1 < p.R) c = *reinterpret_cast<const uint4*>(vb + (j + 1) * p.v_blk.row + d);
          uint32_t aw[4] = {a.x, a.y, a.z, a.w}, cw[4] = {c.x, c.y, c.z, c.w};
          uint32_t odd_bits = 0u;
#pragma unroll
          for (int x = 0; x < 4; ++x) {                     // (see kv8_add_nonfinite)
            const uint32_t fa = kv8_finite_bf16x2(aw[x]), fc = kv8_finite_bf16x2(cw[x]);
            odd_bits |= (fa ^ aw[x]) | (fc ^ cw[x]);
            aw[x] = fa;
            cw[x] = fc;
          }
          if (odd_bits) *odd_values = 1;
#pragma unroll
          for (int x = 0; x < 8; ++x)
            *reinterpret_cast<uint32_t*>(vt + (d + x) * 128 + (((j >> 3) ^ x) * 16) + (j & 7) * 2) =
                __byte_perm(aw[x >> 1], cw[x >> 1], x & 1 ? 0x7632 : 0x5410);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&blk_done[1]);
        if (warp < TP / 2) {
          wait_all(&blk_done[1], 0);
          if (lane == 0 && ok) mbar_arrive(&v_full[st]);
        }
      }
    }
    if (!ok && lane == 0) {
      set_err(p.err, ERR_TIMEOUT);
      *abort_flag = 1;
    }
  } else {
    // ---------------------------------------------------------------- softmax
    const int sw = warp - SOFT0, grp = sw >> 2, quarter = sw & 3, r = quarter * 32 + lane;
    const bool valid = r < NR;
    const int jr = j0 + (valid ? r / p.G : 0);
    const int blim = p.block_full ? p.R - 1 : jr;         // last block key that this row sees
    // The values' exponents of the CTA's pages, 256 at a time; the first 256 on the way while queries are converted.
    auto place = [&](int i) {
      const int page = (rank + i / TP * S) * TP + i % TP;
      return i < n * TP && page < num ? table[page] : -2;
    };
    auto exponent = [&](int ph) {
      return (unsigned)ph < (unsigned)p.num_pages ? __float_as_uint(p.pool.scale[((size_t)ph * p.Hkv + h) * 2 + 1]) >> 23 : 0u;
    };
    unsigned lo = 255u, hi = 0u, first = 0u;
    bool none = false;
    auto join = [&](int ph, unsigned e) {
      none |= ph != -2 && e == 0u;
      lo = min(lo, e ? e : 255u);
      hi = max(hi, e);
    };
    const int first_ph = place(sw * 32 + lane);
    for (int i = sw * 32 + lane + 256; i < n * TP; i += 256) {
      const int ph = place(i);
      join(ph, exponent(ph));
    }
    if (p.kv_stable) griddep_wait();
    // The query rows in f16: a group of D / 8 lanes takes a row at a time, 16 rows a warp, QB loads ahead.  (All eight at
    // once are so much code, run once, that fetching it took most of 5000 cycles.)
    float* fac = reinterpret_cast<float*>(smem + L::FAC);
    {
      constexpr int LPR = D / 8, RPI = 32 / LPR, NI = 16 / RPI;
#pragma unroll 1
      for (int i0 = 0; i0 < NI; i0 += QB) {
        if (i0 == QB) first = exponent(first_ph);
        uint4 v[QB];
#pragma unroll
        for (int i = 0; i < QB; ++i) {
          const int row = sw * 16 + (i0 + i) * RPI + lane / LPR;
          v[i] = make_uint4(0u, 0u, 0u, 0u);
          if (row < NR)
            v[i] = *reinterpret_cast<const uint4*>(p.q.p + b * p.q.batch + (j0 + row / p.G) * p.q.row + ((size_t)h * p.G + row % p.G) * D +
                                                   lane % LPR * 8);
        }
#pragma unroll
        for (int i = 0; i < QB; ++i) {
          const int row = sw * 16 + (i0 + i) * RPI + lane / LPR, ch = lane % LPR;
          float amax = amax8(0.f, v[i]);
#pragma unroll
          for (int o = LPR / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
          const float sc = kv8_scale127(amax);
          *reinterpret_cast<uint4*>(smem + (ch >> 3) * L::QH + row * 128 + (((ch & 7) ^ (row & 7)) * 16)) = scaled8(v[i], kv8_inverse(sc));
          if (ch == 0) fac[row] = sc * p.scale_log2;
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
      join(first_ph, first);
      lo = __reduce_min_sync(0xffffffffu, lo);
      hi = __reduce_max_sync(0xffffffffu, hi);
      none = __any_sync(0xffffffffu, none);
      if (lane == 0) {
        atomicMin(ends, (int)lo);
        atomicMax(ends + 1, (int)hi);
        if (none) *(volatile int*)odd = 1;
        mbar_arrive(ends_bar);
      }
      named_bar_sync(1, 256);               // the rows' factors and the exponents' ends, from all eight warps
    }
    const bool wide = is_wide();
    int unit = wide ? max(ends[0], ends[1] - V_FAR) : ends[1];     // biased, as fp32 holds it; 0: no pages
    const float f = fac[r];
    const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t ocol = L::OCOL + (uint32_t)(grp * D);
    // (below 0: not of the pool; 0 of the values then, or where there is no page.)
    // Lane 4 i + e: the scales of page e of this half of the (8 c + i)-th tile; the next eight tiles' are on their way.
    auto scales = [&](int t0) {
      const int t = t0 + (lane >> 2), page = (rank + t * S) * TP + grp * 4 + (lane & 3);
      float2 s = make_float2(1.f, 0.f);
      if (t < n && page < num) {
        const int ph = table[page];
        s.x = -1.f;
        if ((unsigned)ph < (unsigned)p.num_pages) s = *reinterpret_cast<const float2*>(p.pool.scale + ((size_t)ph * p.Hkv + h) * 2);
      }
      return s;
    };
    const int mine = grp ? n : T;                         // the block's keys are all in half 0
    if (quarter < nsw) {
      float2 now = scales(0), next = scales(8);
      bool go = true;
      auto begin = [&](int t) {
        if ((t & 7) == 0 && t > 0) {
          now = next;
          next = scales(t + 8);
        }
        if (!__all_sync(0xffffffffu, mbar_wait(&s_full[t & 1], (uint32_t)(t >> 1) & 1u, WAIT_NS)) || *abort_flag) {
          if (lane == 0) {
            set_err(p.err, ERR_TIMEOUT);
            *abort_flag = 1;
          }
          go = false;
        }
        tc_fence_after();
        return go;
      };
      auto end = [&](int t) {
        tq_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[2 * (t & 1) + grp]);
      };
      // Tiles of whole pages in the pool, with weights in f16; then the rest, the context's end and the block, or all of them.
      const int plain = is_odd() ? 0 : n - (cut ? 1 : 0);
      int t = 0;
      for (; t < plain && begin(t); ++t) {
        const uint32_t srow = lane_base + (uint32_t)((t & 1) * TK + grp * 64);
        float x0[32], x1[32];
        tq_ld32(srow, x0);
        tq_ld32(srow + 32, x1);
        float ks[4], vs[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          ks[e] = __shfl_sync(0xffffffffu, now.x, (t & 7) * 4 + e);
          vs[e] = __shfl_sync(0xffffffffu, now.y, (t & 7) * 4 + e);
        }
        tq_wait_ld32(x0);
        tq_wait_ld32(x1);
        float fk[4], mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float* x = (e < 2 ? x0 : x1) + (e & 1) * 16;
          float m = fmaxf(x[0], x[1]);
#pragma unroll
          for (int k = 2; k < 16; ++k) m = fmaxf(m, x[k]);
          fk[e] = fmaxf(f * ks[e], TINY);
          mx = fmaxf(mx, m * fk[e]);
        }
        float alpha = 1.f;
        const bool up = valid && mx > mref + P_ROOM;
        if (up) {
          alpha = mref == -INFINITY ? 0.f : exp2_approx(mref - mx);
          mref = mx;
          l *= alpha;
        }
        if (__any_sync(0xffffffffu, up && t > 0)) {
          // O_h holds tiles 0 .. t - 1: wait for the last of them, then scale the row
          const bool okp = __all_sync(0xffffffffu, mbar_wait(&pv_done[grp], (uint32_t)(t - 1) & 1u, WAIT_NS));
          tc_fence_after();
          if (okp) {
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              float o[16];
              tq_ld16(lane_base + ocol + c * 16, o);
              tq_wait_ld();
              uint32_t w[16];
#pragma unroll
              for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(o[k] * alpha);
              tq_st16(lane_base + ocol + c * 16, w);
            }
          } else if (lane == 0) {
            set_err(p.err, ERR_TIMEOUT);
          }
        }
        // P in f16, two keys per TMEM column, over this half's scores
        const float nb = P_BITS - (mref == -INFINITY ? 0.f : mref);
        auto weights = [&](float (&x)[32], int e0) {
          uint32_t pk[16];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int kx = max((int)(__float_as_uint(vs[e0 + e]) >> 23) - unit, -60);
            const float to = nb + (float)kx;
            const float2 f2 = make_float2(fk[e0 + e], fk[e0 + e]), to2 = make_float2(to, to);
            float2 s2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              float2 a = fma2(make_float2(x[e * 16 + 2 * k], x[e * 16 + 2 * k + 1]), f2, to2);
              a.x = exp2_approx(a.x);
              a.y = exp2_approx(a.y);
              s2[k & 1] = add2(s2[k & 1], a);
              pk[e * 8 + k] = pack_f16(a.x, a.y);
            }
            s2[0] = add2(s2[0], s2[1]);
            l = fmaf(s2[0].x + s2[0].y, kv8_two_to(-kx), l);
          }
          tq_st16(srow + e0 * 8, pk);
        };
        weights(x0, 0);
        weights(x1, 2);
        end(t);
      }
      for (; go && t < mine && begin(t); ++t) {
        const bool blk = do_blk && t == n;
        if (blk) mbar_wait(&blk_done[0], 0, WAIT_NS);
        // keys 0..lim of this half are seen by this row
        const int lim = blk ? blim : min(64, C - (rank + t * S) * TK - grp * 64) - 1;
        const RowState r = soft_parts<D>(lane_base + (uint32_t)((t & 1) * TK + grp * 64), lane_base + ocol, blk ? KBR / 8 : 8, lim, f, now, wide,
                                         blk ? blk_scale : nullptr, *(volatile int*)blk_most, &pv_done[grp], t, RowState{mref, l, unit, 1});
        mref = r.m;
        l = r.l;
        unit = r.unit;
        if (!r.ok && lane == 0) set_err(p.err, ERR_TIMEOUT);
        end(t);
      }
      if (mine > 0 && !*abort_flag) {
        if (!__all_sync(0xffffffffu, mbar_wait(&pv_done[grp], (uint32_t)(mine - 1) & 1u, WAIT_NS)) && lane == 0) {
          set_err(p.err, ERR_TIMEOUT);
          *abort_flag = 1;
        }
      }
      vref = __uint_as_float((uint32_t)unit << 23);
      // this half's (reference, sum, unit) for the row's other half, through score columns that are free
      tq_st2(lane_base + (uint32_t)(grp * 64 + 32), mref, l);
      tq_st2(lane_base + (uint32_t)(grp * 64 + 34), vref, 0.f);
      tq_wait_st();
      tc_fence_before();
    }
  }
  __syncthreads();
  tc_fence_after();
  // ------------------------------------------------------------------ output
  const int rpo = (NR + S - 1) / S;
  if (S > 1) {                              // the operands and rings are idle from here on
    if (tid == 0) mbar_arrive_expect_tx(recv_bar, (uint32_t)(S * rpo * L::ROWB));
    cluster_arrive_relaxed();
  }
  const bool have = T > 0 && !*abort_flag;
  float* part = reinterpret_cast<float*>(smem + L::PART);
  if (warp >= SOFT0 && ((warp - SOFT0) & 3) < nsw) {
    // The row's halves together: common maximum, weighted sums; each group half of the row's columns.
    const int sw = warp - SOFT0, grp = sw >> 2, quarter = sw & 3, r = quarter * 32 + lane;
    const bool valid = r < NR;
    const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t orow = lane_base + L::OCOL;
    float mo, lo, vo, pad;
    tq_ld2(lane_base + (uint32_t)((grp ^ 1) * 64 + 32), mo, lo);
    tq_ld2(lane_base + (uint32_t)((grp ^ 1) * 64 + 34), vo, pad);
    const float mm = fmaxf(mref, mo);
    const float wm = mref == -INFINITY ? 0.f : exp2_approx(mref - mm), wo = mo == -INFINITY ? 0.f : exp2_approx(mo - mm);
    // (in one order in both groups: the sum is the same number)
    const float sum = grp ? lo * wo + l * wm : l * wm + lo * wo;
    // Outputs stay in units of the values' until a weight takes the exponent in: a product with the unit could leave fp32.
    const float tm = mref + kv8_exponent(vref), to = mo + kv8_exponent(vo), most = fmaxf(tm, to);
    const float pm = mref == -INFINITY ? 0.f : exp2_approx(tm - most), po = mo == -INFINITY ? 0.f : exp2_approx(to - most);
    const float w0 = grp ? po : pm, w1 = grp ? pm : po;
    const bool have1 = have && n > 0;       // half 1 holds cache tiles only
    const int j = j0 + (valid ? r / p.G : 0), g = valid ? r % p.G : 0;
    __nv_bfloat16* dst = p.out + (((size_t)b * p.R + j) * p.Hq + (size_t)h * p.G + g) * D;
    const float inv = have && sum != 0.f ? exp2f(most - mm) / sum : 0.f;         // (NaN stays)
    float* prow = part + r * PD;
#pragma unroll 1
    for (int c = grp * (D / 32); c < (grp + 1) * (D / 32); ++c) {
      float o[16], o1[16];
      if (have) {
        tq_ld16(orow + c * 16, o);
        if (have1) tq_ld16(orow + D + c * 16, o1);
        tq_wait_ld();
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) o[i] = !have ? 0.f : have1 ? o[i] * w0 + o1[i] * w1 : o[i] * w0;
      if (!valid) continue;
      if (S == 1) {
#pragma unroll
        for (int i = 0; i < 16; i += 8)
          *reinterpret_cast<uint4*>(dst + c * 16 + i) =
              make_uint4(pack_bf16(o[i] * inv, o[i + 1] * inv), pack_bf16(o[i + 2] * inv, o[i + 3] * inv),
                         pack_bf16(o[i + 4] * inv, o[i + 5] * inv), pack_bf16(o[i + 6] * inv, o[i + 7] * inv));
      } else {
#pragma unroll
        for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(prow + c * 16 + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
      }
    }
    if (S > 1 && valid && grp == 0) {
      prow[D] = have ? mm : -INFINITY;
      prow[D + 1] = have ? sum : 0.f;
      prow[D + 2] = most - mm;
      prow[D + 3] = do_blk && *odd_values ? 1.f : 0.f;
    }
  }
  if (S > 1) {
    fence_proxy_async_smem();
    __syncthreads();
    cluster_wait();                         // every CTA's receiving rows are free, its barrier armed
    float* recv = reinterpret_cast<float*>(smem + L::RECV);
    if (lane == 0 && warp < 4) {
      for (int o = warp; o < S; o += 4)
        bulk_copy_s2s(dsmem_map(smem_u32(recv) + (uint32_t)(rank * rpo * L::ROWB), (uint32_t)o), smem_u32(part + o * rpo * PD),
                      (uint32_t)(rpo * L::ROWB), dsmem_map(smem_u32(recv_bar), (uint32_t)o));
    }
    if (!mbar_wait(recv_bar, 0)) set_err(p.err, ERR_TIMEOUT);
    cluster_arrive_relaxed();
    const int row0 = rank * rpo;
    float* scl = reinterpret_cast<float*>(smem + L::SCL);          // [S][rpo]
    for (int rr = warp; rr < rpo && row0 + rr < NR; rr += THREADS / 32) {
      const float4 ml = lane < S ? *reinterpret_cast<const float4*>(recv + (lane * rpo + rr) * PD + D) : make_float4(-INFINITY, 0.f, 0.f, 0.f);
      float M = ml.x;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      const bool some = ml.x != -INFINITY;
      float sum = some ? ml.y * exp2_approx(ml.x - M) : 0.f * ml.y;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane < S) scl[lane * rpo + rr] = sum == 0.f ? 0.f : (some ? exp2f(ml.x - M + ml.z) : 0.f) / sum;
    }
    __syncthreads();
    for (int e = tid; e < rpo * (D / 4); e += THREADS) {
      const int rr = e / (D / 4), c = e % (D / 4) * 4, r = row0 + rr;
      if (r >= NR) break;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int s = 0; s < S; ++s) {
        const float w = scl[s * rpo + rr];
        const float4 v = *reinterpret_cast<const float4*>(recv + (s * rpo + rr) * PD + c);
        acc.x += v.x * w;
        acc.y += v.y * w;
        acc.z += v.z * w;
        acc.w += v.w * w;
      }
      const int j = j0 + r / p.G, g = r % p.G;
      *reinterpret_cast<uint2*>(p.out + (((size_t)b * p.R + j) * p.Hq + (size_t)h * p.G + g) * D + c) =
          make_uint2(pack_bf16(acc.x, acc.y), pack_bf16(acc.z, acc.w));
    }
    // (the block is the last CTA's; its flag came with its rows)
    if (row0 < NR && recv[(S - 1) * rpo * PD + D + 3] != 0.f) {
      __syncthreads();
      kv8_add_nonfinite(p, D, false, 0, b, h, j0 * p.G + row0, min(rpo, NR - row0));
    }
    cluster_wait();                         // every copy out of this CTA has landed
  } else if (*odd_values) {
    __syncthreads();
    kv8_add_nonfinite(p, D, false, 0, b, h, j0 * p.G, NR);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == MMA_WARP) {
    __syncwarp();
    tmem_dealloc(tmem, 512u);
  }
}

template <int D>
KernelLimits& limits() {
  static KernelLimits lim;
  return lim;
}

template <int D>
void config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute* attr, dim3 grid, int S) {
  cfg.gridDim = grid;
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = TL<D>::BYTES;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
}

template <int D>
int resident_t(int S) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  config<D>(cfg, attr, dim3(S, 1024, 1), S);
  cfg.numAttrs = 1;
  int n = 0;
  if (ensure_kernel_limits((const void*)kv8_attn_tc_kernel<D>, limits<D>(), TL<D>::BYTES, true) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, kv8_attn_tc_kernel<D>, &cfg) != cudaSuccess) {
    cudaGetLastError();
    n = 0;
  }
  return n;
}

template <int D>
cudaError_t launch_t(const Kv8Params& p, int S, cudaStream_t stream) {
  const cudaError_t e = ensure_kernel_limits((const void*)kv8_attn_tc_kernel<D>, limits<D>(), TL<D>::BYTES, true);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  config<D>(cfg, attr, dim3(S, (unsigned)(p.groups * p.Hkv), p.B), S);
  cfg.stream = stream;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kv8_attn_tc_kernel<D>, p);
}

}  // namespace

int kv8_attn_tc_resident(int D, int S) { return D == 128 ? resident_t<128>(S) : resident_t<64>(S); }

cudaError_t launch_kv8_attn_tc(const Kv8Params& p, int D, int S, cudaStream_t stream) {
  return D == 128 ? launch_t<128>(p, S, stream) : launch_t<64>(p, S, stream);
}

}  // namespace cospec
