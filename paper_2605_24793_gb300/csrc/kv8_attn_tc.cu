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
// weight's exponent, relative to the largest seen by the group; weights are held times 2^6 in f16 and the
// reference moves when a score exceeds it by 2^8, as on mma.sync.  The block's bf16 keys and values come
// to f16 by one power of two each: 2^-25 of the block's largest value is what can be lost.
//
// 104 rows, batch 16 at 2048 to 8192 tokens: 71.5 us.  A softmax warp works four fifths of a tile's time (a quarter of it on
// the maxima of 64 keys, two fifths on their weights) beside the converting warps on its scheduler, which wait a quarter of
// theirs for free stages: instructions bound it, and fetching them (75.6 us before the start and the block were in rolled
// loops); the tensor pipe is busy for 25 %, shared memory for 23.  Codes loaded to registers past the ring, behind
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
constexpr float P_BITS = 6.f, P_ROOM = 8.f;
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
  // mma_done, recv, the block's maxima, its scales, its operands [2]
  static constexpr int NBAR = 4 * NS + 15;
  static constexpr int HOLDER = MISC + NBAR * 8;        // TMEM base, abort, sequence, block's maxima [2][CONV]
  static constexpr int NEED = HOLDER + 16 + 2 * CONV * 4 + 16;
  static constexpr int PD = D + 4;                      // fp32 row of a partial: O, max, sum, pad
  static constexpr int ROWB = PD * 4;
  static constexpr int PART = 0, RECV = TM * ROWB;      // after the last tile, over everything before MISC
  static constexpr int SCL = RECV + (TM + 15) * ROWB;   // [S][rows per owner]
  static_assert(SCL + (TM + 16) * 4 <= MISC, "the partials fit");
  static constexpr uint32_t OCOL = 2 * TK;
  // one CTA per SM: each wants all of TMEM
  static constexpr int BYTES = (NEED > 118 * 1024 ? NEED : 118 * 1024) + 1024;
  static_assert(BYTES <= 232448, "shared memory of an SM");
};

constexpr uint32_t idesc_f16(int M, int N) { return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24); }

CS_DEV uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
CS_DEV uint4 codes_f16(uint32_t a, uint32_t b) {        // eight codes
  return make_uint4(kv8_f16x2(a), kv8_f16x2_hi(a), kv8_f16x2(b), kv8_f16x2_hi(b));
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
  uint64_t* max_bar = recv_bar + 1;         // the converting warps' maxima over the block are there
  uint64_t* blk_bar = max_bar + 1;          // its scales are
  uint64_t* blk_done = blk_bar + 1;         // [2]: its keys, its values have been written
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem + L::HOLDER);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  volatile int* seq_slot = abort_flag + 1;
  volatile float* blk_max = reinterpret_cast<volatile float*>(smem + L::HOLDER + 16);   // [2][CONV]
  volatile float* blk_scale = blk_max + 2 * CONV;                                       // [2]

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
    mbar_init(max_bar, CONV);
    mbar_init(blk_bar, 1);
    mbar_init(&blk_done[0], CONV);
    mbar_init(&blk_done[1], CONV);
    *abort_flag = 0;
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

  if (warp < CONV) {
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
    bool ok = true;
    auto wait = [&](uint64_t* bar, int phase) { ok = ok && mbar_wait(bar, (uint32_t)phase & 1u, WAIT_NS); };
    auto convert = [&](int k) {
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
      } else {
        // a lane: 16 tokens of every 32nd dimension; cells behind a page's last token may hold anything: they enter as 0
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
          for (int y = 0; y < NX; ++y) v[x][y] = *reinterpret_cast<const uint4*>(src + x * L::PB + (y * 32 + lane) * KV8_PAGE);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int have = __shfl_sync(0xffffffffu, count_c, 2 * (k & 15) + x);
          if (have < KV8_PAGE) {
            uint32_t keep[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int m = have - 4 * y;
              keep[y] = m >= 4 ? 0xffffffffu : m <= 0 ? 0u : (1u << (8 * m)) - 1u;
            }
#pragma unroll
            for (int y = 0; y < NX; ++y) {
              v[x][y].x &= keep[0];
              v[x][y].y &= keep[1];
              v[x][y].z &= keep[2];
              v[x][y].w &= keep[3];
            }
          }
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
#pragma unroll 1
    for (int k = 0; k < total; ++k) {
      convert(k);
      issue(k + SLOTS);                                   // (the slot has been read)
      if ((k & 7) == 7) {                                 // (a wait that ran out makes the rest useless)
        ok = __all_sync(0xffffffffu, ok && !*abort_flag);
        if (!ok) break;
      }
    }
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
      float km = 0.f, vm = 0.f;
#pragma unroll 1
      for (int e = tid; e < p.R * (D / 8); e += CONV * 32) {
        km = amax8(km, *reinterpret_cast<const uint4*>(kb + (e / (D / 8)) * p.k_blk.row + e % (D / 8) * 8));
        vm = amax8(vm, *reinterpret_cast<const uint4*>(vb + (e / (D / 8)) * p.v_blk.row + e % (D / 8) * 8));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        km = fmaxf(km, __shfl_xor_sync(0xffffffffu, km, o));
        vm = fmaxf(vm, __shfl_xor_sync(0xffffffffu, vm, o));
      }
      if (lane == 0) {
        blk_max[warp] = km;
        blk_max[CONV + warp] = vm;
        mbar_arrive(max_bar);
      }
      wait_all(max_bar, 0);                     // (bounded: a warp that gave up does not come)
#pragma unroll
      for (int w = 0; w < CONV; ++w) {
        km = fmaxf(km, blk_max[w]);
        vm = fmaxf(vm, blk_max[CONV + w]);
      }
      const float ks = kv8_scale_of(km), vs = kv8_scale_of(vm), ki = kv8_inverse(ks), vi = kv8_inverse(vs);
      if (tid == 0) {
        blk_scale[0] = ks;
        blk_scale[1] = vs;
        mbar_arrive(blk_bar);
      }
      if (ok && (n < NS || wait_all(&k_empty[st], n / NS - 1))) {
#pragma unroll 1
        for (int e = tid; e < p.R * (D / 8); e += CONV * 32) {
          const int row = e / (D / 8), ch = e % (D / 8);
          *reinterpret_cast<uint4*>(kt + (ch >> 3) * L::KH + row * 128 + (((ch & 7) ^ (row & 7)) * 16)) =
              scaled8(*reinterpret_cast<const uint4*>(kb + row * p.k_blk.row + ch * 8), ki);
        }
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
          const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, cw[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            const float lo = x & 1 ? bf_hi(aw[x >> 1]) : bf_lo(aw[x >> 1]), hi = x & 1 ? bf_hi(cw[x >> 1]) : bf_lo(cw[x >> 1]);
            *reinterpret_cast<uint32_t*>(vt + (d + x) * 128 + (((j >> 3) ^ x) * 16) + (j & 7) * 2) = pack_f16(lo * vi, hi * vi);
          }
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
  } else if (warp == MMA_WARP) {
    // ---------------------------------------------------------------- MMA
    if (T > 0) {
      const uint32_t on = elect_one();
      const uint32_t sbase = smem_u32(smem);
      const uint64_t q_desc = smem_desc_sw128(sbase), k_desc = smem_desc_sw128(sbase + L::TILES);
      constexpr uint64_t STAGE16 = (uint64_t)((L::KB + L::VB) >> 4);
      bool ok = __all_sync(0xffffffffu, mbar_wait(q_full, 0, WAIT_NS));
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
        if (do_blk && u == n && KBR < 64) {
          for (int ks = 0; ks < KBR / 16; ++ks)
            umma_bf16_tmem_a_on(on, dst, src + (uint32_t)(ks * 8), vd + (uint64_t)(ks * 2), idesc_f16(TM, D), (u | ks) != 0 ? 1u : 0u);
        } else {
          umma_tmem_a_k64_on(on, dst, src, vd, idesc_f16(TM, D), u ? 1u : 0u);
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
  } else {
    // ---------------------------------------------------------------- softmax
    const int sw = warp - SOFT0, grp = sw >> 2, quarter = sw & 3, r = quarter * 32 + lane;
    const bool valid = r < NR;
    const int jr = j0 + (valid ? r / p.G : 0);
    const int blim = p.block_full ? p.R - 1 : jr;         // last block key that this row sees
    if (p.kv_stable) griddep_wait();
    // The query rows in f16: a group of D / 8 lanes takes a row at a time, 16 rows a warp, QB loads ahead.  (All eight at
    // once are so much code, run once, that fetching it took most of 5000 cycles.)
    float* fac = reinterpret_cast<float*>(smem + L::FAC);
    {
      constexpr int LPR = D / 8, RPI = 32 / LPR, NI = 16 / RPI;
#pragma unroll 1
      for (int i0 = 0; i0 < NI; i0 += QB) {
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
      named_bar_sync(1, 256);               // the rows' factors, from all eight warps
    }
    const float f = fac[r];
    const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t ocol = L::OCOL + (uint32_t)(grp * D);
    // Lane 4 i + e: the scales of page e of this half of the (8 c + i)-th tile; the next eight tiles' are on their way.
    auto scales = [&](int t0) {
      const int t = t0 + (lane >> 2), page = (rank + t * S) * TP + grp * 4 + (lane & 3);
      float2 s = make_float2(1.f, 0.f);
      if (t < n && page < num) {
        const int ph = table[page];
        if ((unsigned)ph < (unsigned)p.num_pages) s = *reinterpret_cast<const float2*>(p.pool.scale + ((size_t)ph * p.Hkv + h) * 2);
      }
      return s;
    };
    auto there = [&](int t, int e) {                      // the page is in the pool (a bad one's scores are masked)
      const int page = (rank + t * S) * TP + grp * 4 + e;
      return page >= num || (unsigned)table[page] < (unsigned)p.num_pages;
    };
    const int mine = grp ? n : T;                         // the block's keys are all in half 0
    if (quarter < nsw) {
      float2 now = scales(0), next = scales(8);
      for (int t = 0; t < mine; ++t) {
        const bool blk = do_blk && t == n;
        if ((t & 7) == 0 && t > 0) {
          now = next;
          next = scales(t + 8);
        }
        if (!__all_sync(0xffffffffu, mbar_wait(&s_full[t & 1], (uint32_t)(t >> 1) & 1u, WAIT_NS)) || *abort_flag) {
          if (lane == 0) {
            set_err(p.err, ERR_TIMEOUT);
            *abort_flag = 1;
          }
          break;
        }
        tc_fence_after();
        const uint32_t srow = lane_base + (uint32_t)((t & 1) * TK + grp * 64);
        float x0[32], x1[32];
        tq_ld32(srow, x0);
        tq_ld32(srow + 32, x1);
        float ks[4], vs[4];
        if (blk) {
          mbar_wait(blk_bar, 0, WAIT_NS);
          ks[0] = ks[1] = ks[2] = ks[3] = blk_scale[0];
          vs[0] = vs[1] = vs[2] = vs[3] = blk_scale[1];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            ks[e] = __shfl_sync(0xffffffffu, now.x, (t & 7) * 4 + e);
            vs[e] = __shfl_sync(0xffffffffu, now.y, (t & 7) * 4 + e);
          }
        }
        tq_wait_ld32(x0);
        tq_wait_ld32(x1);
        // keys 0..lim of this half are seen by this row
        const int left = C - (rank + t * S) * TK - grp * 64;
        const int lim = blk ? blim : min(64, left) - 1;
        if (blk || lim < 63) {
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            x0[k] = k <= lim ? x0[k] : -INFINITY;
            x1[k] = 32 + k <= lim ? x1[k] : -INFINITY;
          }
        }
        if (!blk && vs[0] * vs[1] * vs[2] * vs[3] == 0.f) {         // (a page without a scale: none, or not of the pool)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!there(t, e))
#pragma unroll
              for (int k = 0; k < 16; ++k) (e < 2 ? x0 : x1)[(e & 1) * 16 + k] = -INFINITY;
        }
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
        const float top = fmaxf(fmaxf(vs[0], vs[1]), fmaxf(vs[2], vs[3]));
        const bool raise = top > vref;                    // (the same in the whole group)
        if (raise) {
          alpha *= vref * kv8_inverse(top);
          vref = top;
        }
        if (__any_sync(0xffffffffu, (up || raise) && t > 0)) {
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
            const int kx = max((int)(__float_as_uint(vs[e0 + e]) >> 23) - (int)(__float_as_uint(vref) >> 23), -60);
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
            l = fmaf(s2[0].x + s2[0].y, __uint_as_float((uint32_t)(127 - kx) << 23), l);
          }
          tq_st16(srow + e0 * 8, pk);
        };
        weights(x0, 0);
        weights(x1, 2);
        tq_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[2 * (t & 1) + grp]);
      }
      if (mine > 0 && !*abort_flag) {
        if (!__all_sync(0xffffffffu, mbar_wait(&pv_done[grp], (uint32_t)(mine - 1) & 1u, WAIT_NS)) && lane == 0) {
          set_err(p.err, ERR_TIMEOUT);
          *abort_flag = 1;
        }
      }
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
    const float w0 = grp ? wo * vo : wm * vref, w1 = grp ? wm * vref : wo * vo;
    const bool have1 = have && n > 0;       // half 1 holds cache tiles only
    const int j = j0 + (valid ? r / p.G : 0), g = valid ? r % p.G : 0;
    __nv_bfloat16* dst = p.out + (((size_t)b * p.R + j) * p.Hq + (size_t)h * p.G + g) * D;
    const float inv = have && sum != 0.f ? 1.f / sum : 0.f;         // (NaN stays)
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
      const float2 ml = lane < S ? *reinterpret_cast<const float2*>(recv + (lane * rpo + rr) * PD + D) : make_float2(-INFINITY, 0.f);
      float M = ml.x;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      const float a = ml.x == -INFINITY ? 0.f : exp2_approx(ml.x - M);
      float sum = ml.y * a;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane < S) scl[lane * rpo + rr] = sum == 0.f ? 0.f : a / sum;
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
    cluster_wait();                         // every copy out of this CTA has landed
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
