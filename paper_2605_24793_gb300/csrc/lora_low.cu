// The low-rank sides of the adapters (cospec_lora_forward, cospec_lora_backward):
//   forward   u[m][j] = c_a sum_k drop(x)[m][k] A_a[j][k]      A_a [rank, in]: the factor's rows run along k
//   backward  t[m][j] = c_a sum_n dy[m][n] B_a[n][j]           B_a [out, rank]: its rows run along j
// with a the row's adapter and c_a = scaling[a] / (1 - p); rows without one get zeros.  Both are fp32,
// and both are bound by reading x or dy once (and, for a few rows, by the latency of one read of the factor).
//
// low_tile_kernel: a CTA takes 32 to 128 rows, in chunks of 64 of the contraction that come by cp.async into a ring
// ahead of the products (mma.sync).  Rows of several adapters: a chunk of x stays while the factors of the
// tile's adapters pass, and a warp whose rows differ adds each product to the sums of that adapter's rows alone (what another
// adapter's factor holds, infinities or NaN, reaches no other row).  The contraction is split over the CTAs of a cluster (and, for few rows, the
// warps of a CTA) and joined in shared memory in a fixed order.
// Dropout: a thread masks the 16-byte chunks that it copied itself, each one draw of the generator, before the
// barrier that hands them on.
// Rows of many adapters in turn (requests of a batch in the order they came): above three changes a tile, the tiles take their
// rows in the order of the adapters, 2048 at a time, so that a tile's factors stay two or three (64 adapters of rank 32, 4096 rows of
// 4096: 251 -> 41 us).
// low_row_kernel, for a few rows: CTAs per row, which read its adapter's factor in one wave of loads; a tile's rows of as many
// adapters would pass one after another.  What it costs is the factors read, one a row; what the tiles cost is their chain of chunks.
// Taken up to LOW_ROW_MANY elements (128 MB) for at most 64 rows, or 256 of at least four adapters, else up to LOW_ROW_MAX (20 MB).
// (Whole forward passes 4096 -> 4096 in us, row / tile kernel: 64 rows of 1 adapter at rank 64 16.9 / 19.8, of 16 18.7 / 64; 28 rows of
// 6584 at rank 128 13.3 / 34.5; 256 rows of 4 adapters side by side 18.8 / 25 at rank 16, 23.1 / 26.1 at rank 32; 160 of 8 at rank 64 30 / 51;
// 256 of one adapter at rank 16 22.7 / 20.2; 848 of 2560 of four 33.6 / 30.9.)
// Bounds: low_tile_kernel 8192 x 5120 at rank 64 with dropout 64 us (84 MB, 12 us of memory: the products' and the draw's
// instructions), 4096 x 2560 at rank 16 16 us; low_row_kernel 4 to 9 us, latency.
#include "lora.cuh"

namespace cospec {

namespace {

constexpr int LOW_THREADS = 256;         // 8 warps
constexpr long long LOW_ROW_MAX = 10000000, LOW_ROW_MANY = 64000000;
constexpr int ROW_THREADS = 512;
constexpr int SORT_WIN = 2048;           // rows ordered by their adapters at a time

struct LowArgs {
  const __nv_bfloat16* x;
  long long ldx;
  const __nv_bfloat16* f;
  const float* scaling;
  const int32_t* adapter;
  float* u;
  int M, C, r, n;       // C: the contraction's length
  float keep_inv;       // 1 / (1 - p)
  LoraDrop drop;
  int rw_log2;          // log2 of the row groups of a CTA
  int sort;             // tiles may take their rows in the order of the adapters
  int ranks;            // (row kernel) ranks of a CTA, a multiple of 16
  int* err;
};

constexpr int CK = 64;                   // contraction of a chunk
constexpr int DEPTH = 4;                 // items in flight: a chunk and an adapter's factor for it
constexpr int LOW_MAX_ROWS = 128;

struct LowSmem {
  int ids[LOW_MAX_ROWS];
  int adapters[LOW_MAX_ROWS];
  int row[LOW_MAX_ROWS];       // of x
  int warp_count[8];
};
__host__ __device__ constexpr uint32_t low_bytes(int rows, int R) {
  return (uint32_t)DEPTH * (uint32_t)(rows * 128 + R * 128) + (uint32_t)sizeof(LowSmem);
}

// A window is SORT_WIN rows from w0 on, or what is left.  Whether its tiles take its rows in the order of the adapters: above three
// changes of the adapter a tile, by 256 pairs of neighbours.  (The same in all CTAs of the window.)
CS_DEV bool rows_in_turn(const LowArgs& p, int w0, int rows) {
  const int wn = min(SORT_WIN, p.M - w0), i = w0 + (((int)threadIdx.x * (wn - 1)) >> 8);
  const bool change = wn > 1 && p.adapter[i] != p.adapter[i + 1];
  static_assert(LOW_THREADS == 256, "a pair a thread");
  return __syncthreads_count(change) * rows > 3 * LOW_THREADS;
}
// The tile's share of the window's rows in that order, rows without an adapter behind: a counting sort by 8 bits of the adapter at
// a time, which keeps the order of equal ones.  A warp ranks 256 rows, 32 at a time.  (A sort by exchanges of 2048 keys took some
// 15 us, longer than many a tile's products.)
struct OrderSmem {
  uint16_t count[LOW_THREADS / 32][256];
  uint16_t row[SORT_WIN];
};
CS_DEV void order_rows(const LowArgs& p, OrderSmem& o, LowSmem& sm, int w0, int m0, int rows) {
  constexpr int PER = SORT_WIN / LOW_THREADS;
  static_assert(LOW_THREADS == 256 && PER * 32 * (LOW_THREADS / 32) == SORT_WIN, "a thread a digit");
  const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31, wn = min(SORT_WIN, p.M - w0);
  const int passes = p.n < 256 ? 1 : 2;
  for (int pass = 0; pass < passes; ++pass) {
    int row[PER], digit[PER], before[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = warp * (32 * PER) + k * 32 + lane;
      row[k] = i >= wn ? -1 : pass == 0 ? i : o.row[i];
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int id = row[k] >= 0 ? p.adapter[w0 + row[k]] : 0;
      digit[k] = row[k] < 0 ? -1 : ((id < 0 || id >= p.n ? p.n : id) >> (8 * pass)) & 255;
    }
    for (int e = tid; e < (int)sizeof(o.count) / 4; e += LOW_THREADS) reinterpret_cast<uint32_t*>(o.count)[e] = 0u;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const unsigned same = __match_any_sync(0xffffffffu, digit[k]);
      const int have = digit[k] >= 0 ? o.count[warp][digit[k]] : 0;
      before[k] = have + __popc(same & ((1u << lane) - 1u));
      __syncwarp();
      if (digit[k] >= 0 && (same >> lane) == 1u) o.count[warp][digit[k]] = (uint16_t)(before[k] + 1);      // the last of its kind
      __syncwarp();
    }
    __syncthreads();
    int total = 0;                         // of digit tid
#pragma unroll
    for (int w = 0; w < LOW_THREADS / 32; ++w) total += o.count[w][tid];
    int upto = total;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += v;
    }
    if (lane == 31) sm.warp_count[warp] = upto;
    __syncthreads();
    int at = upto - total;
#pragma unroll
    for (int w = 0; w < LOW_THREADS / 32; ++w) at += w < warp ? sm.warp_count[w] : 0;
#pragma unroll
    for (int w = 0; w < LOW_THREADS / 32; ++w) {
      const int c = o.count[w][tid];
      o.count[w][tid] = (uint16_t)at;
      at += c;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (digit[k] >= 0) o.row[o.count[warp][digit[k]] + before[k]] = (uint16_t)row[k];
    __syncthreads();
  }
  for (int i = tid; i < rows; i += LOW_THREADS) sm.row[i] = m0 + i < p.M ? w0 + o.row[m0 - w0 + i] : 0;
  __syncthreads();
}

// NT: rank in groups of 8 (2, 4, 8 or 16).  RM: the factor's rows run along the rank.
template <int NT, bool RM>
__global__ void __launch_bounds__(LOW_THREADS, NT <= 2 ? 3 : NT <= 8 ? 2 : 1) low_tile_kernel(const LowArgs p) {
  extern __shared__ __align__(128) uint8_t sraw[];
  constexpr int R = NT * 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2;
  const int S = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
  const int RW = 1 << p.rw_log2, KW = 8 >> p.rw_log2, rows = 16 * RW;
  const int rw = warp & (RW - 1), kw = warp >> p.rw_log2;
  const int m0 = ((int)blockIdx.x / S) * rows;
  const uint32_t x_off = smem_u32(sraw), f_off = x_off + (uint32_t)(DEPTH * rows * 128);
  LowSmem& sm = *reinterpret_cast<LowSmem*>(sraw + DEPTH * (rows * 128 + R * 128));
  griddep_wait();
  griddep_launch_dependents();

  const int chunks = (p.C + CK - 1) / CK;
  const int c0 = (int)((long long)chunks * rank / S), c1 = (int)((long long)chunks * (rank + 1) / S);
  const bool drop = p.drop.thr != 0u;
  LoraKey key{0, 0};
  if (drop) key = lora_key(p.drop);

  // The thread's 16-byte chunk i of an x chunk: row tid / 8 + 32 i, columns 8 (tid mod 8) ..; its swizzled place in the
  // 128-byte rows is the same for all i.  Items are walked with counters, without divisions.
  const int xc = (int)threadIdx.x & 7, xr = (int)threadIdx.x >> 3;
  const uint32_t xs = (uint32_t)(xr * 128 + ((xc ^ (xr & 7)) << 4));
  int m_of[LOW_MAX_ROWS / 32];             // the rows of x that it copies
#pragma unroll
  for (int i = 0; i < LOW_MAX_ROWS / 32; ++i) m_of[i] = m0 + xr + 32 * i;
  const __nv_bfloat16* xp = p.x + (long long)c0 * CK + 8 * xc;
  const int x_rows = min(rows, p.M - m0);                // rows of the tile that exist
  auto load_x = [&](int ci) {
    const uint32_t dst = x_off + (uint32_t)((ci & (DEPTH - 1)) * rows * 128) + xs;
    const bool kin = (c0 + ci) * CK + 8 * xc < p.C;
    const __nv_bfloat16* src = xp + ci * CK;
#pragma unroll
    for (int i = 0; i < LOW_MAX_ROWS / 32; ++i) {
      if (32 * i + xr >= rows) break;
      const bool on = kin && 32 * i + xr < x_rows;
      cp_async16(dst + (uint32_t)(i * 4096), on ? src + (long long)m_of[i] * p.ldx : p.x, on);
    }
  };
  // the first chunks set out before the tile's adapters are known
  const int early = min(DEPTH - 1, c1 - c0);
  for (int i = 0; i < early; ++i) load_x(i);
  static_assert(sizeof(OrderSmem) <= DEPTH * R * 128, "the order is made in the factors' place");
  const int w0 = m0 & ~(SORT_WIN - 1);
  const bool sorted = p.sort && rows_in_turn(p, w0, rows);
  if (sorted) {                            // other rows than those that are under way
    order_rows(p, *reinterpret_cast<OrderSmem*>(sraw + (f_off - x_off)), sm, w0, m0, rows);
    cp_async_commit();
    cp_async_wait<0>();
#pragma unroll
    for (int i = 0; i < LOW_MAX_ROWS / 32; ++i)
      if (xr + 32 * i < rows) m_of[i] = sm.row[xr + 32 * i];
    for (int i = 0; i < early; ++i) load_x(i);
  }

  // the adapters of the tile, in the order of their first rows
  if (threadIdx.x < LOW_MAX_ROWS) {
    const bool in = (int)threadIdx.x < x_rows;
    const int m = sorted && in ? sm.row[threadIdx.x] : m0 + (int)threadIdx.x;
    sm.row[threadIdx.x] = m;
    sm.ids[threadIdx.x] = in ? lora_adapter(p.adapter, m, p.n, p.err) : -1;
  }
  __syncthreads();
  bool first = false;
  unsigned mask = 0;
  if (threadIdx.x < LOW_MAX_ROWS) {
    const int id = sm.ids[threadIdx.x];
    first = id >= 0 && (threadIdx.x == 0 || sm.ids[threadIdx.x - 1] != id);       // (most rows follow one of their own)
    if (first) {
      for (int j = 0; j < (int)threadIdx.x; j += 4) {
        const int4 v = *reinterpret_cast<const int4*>(&sm.ids[j]);
        first = first && v.x != id && (j + 1 >= (int)threadIdx.x || v.y != id) && (j + 2 >= (int)threadIdx.x || v.z != id) &&
                (j + 3 >= (int)threadIdx.x || v.w != id);
      }
    }
    __syncwarp();
    mask = __ballot_sync(0xffffffffu, first);
    if (lane == 0) sm.warp_count[warp] = __popc(mask);
  }
  __syncthreads();
  if (threadIdx.x < LOW_MAX_ROWS) {
    int at = __popc(mask & ((1u << lane) - 1u));
    for (int w = 0; w < warp; ++w) at += sm.warp_count[w];
    if (first) sm.adapters[at] = sm.ids[threadIdx.x];
  }
  const int count = sm.warp_count[0] + sm.warp_count[1] + sm.warp_count[2] + sm.warp_count[3];
  __syncthreads();

  const int items = (c1 - c0) * count;
  int l_ci = 0, l_ai = 0, l_item = 0;                    // the next item to load
  auto load = [&]() {
    if (l_item < items) {
      const int k0 = (c0 + l_ci) * CK;
      const bool kin = k0 + 8 * xc < p.C;
      if (l_ai == 0 && l_ci >= early) load_x(l_ci);
      const __nv_bfloat16* f = p.f + (size_t)sm.adapters[l_ai] * p.r * p.C;
      const uint32_t dst = f_off + (uint32_t)((l_item & (DEPTH - 1)) * R * 128);
      if (!RM) {                           // [rank][64]
#pragma unroll
        for (int i = 0; 32 * i < R; ++i) {
          const int row = xr + 32 * i;
          if (row >= R) break;
          const bool on = row < p.r && kin;
          cp_async16(dst + (uint32_t)(i * 4096) + xs, on ? f + (size_t)row * p.C + k0 + 8 * xc : f, on);
        }
      } else {                             // [64][rank]: rows of 2 R bytes; 8 neighbouring rows on different banks
        for (int i = (int)threadIdx.x; i < 64 * NT; i += LOW_THREADS) {
          const int row = i / NT, c = i % NT, k = k0 + row;
          const bool on = k < p.C && 8 * c < p.r;
          const int sw = NT >= 8 ? row & 7 : NT == 4 ? (row >> 1) & 3 : (row >> 2) & 1;
          cp_async16(dst + (uint32_t)(row * (R * 2) + ((c ^ sw) << 4)), on ? f + (size_t)k * p.r + 8 * c : f, on);
        }
      }
      ++l_item;
      if (++l_ai == count) l_ai = 0, ++l_ci;
    }
    cp_async_commit();
  };

  // An mma truncates its running sum: after every four chunks (16 products of 16) the sums move to `sum` by rounded
  // additions, so that they do not drift with the contraction's length (5120: relative error 2e-6 -> 3e-7).
  float acc[NT][4], sum[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = sum[i][j] = 0.f;
  auto settle = [&](bool on0, bool on1) {
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[i][j] += (j < 2 ? on0 : on1) ? acc[i][j] : 0.f, acc[i][j] = 0.f;
  };
  const int id0 = sm.ids[rw * 16 + g], id1 = sm.ids[rw * 16 + g + 8];
  // whether the warp's rows are of one adapter (those of none end as zeros): one of them, the largest, is then every row's
  const int top = (int)__reduce_max_sync(0xffffffffu, (unsigned)(max(id0, id1) + 1)) - 1;
  const bool one = __all_sync(0xffffffffu, (id0 < 0 || id0 == top) && (id1 < 0 || id1 == top));
  int turns = 0;
  // ldmatrix: the lane's row and 16-byte column of a 16 x 16 block; the swizzled places are the first block's, others differ by an
  // exclusive or
  const int lr = lane & 15, lc = lane >> 4;
  const uint32_t xa = (uint32_t)((rw * 16 + lr) * 128 + ((lc ^ (lr & 7)) << 4));
  uint32_t fa;
  if (!RM) {
    const int fr = (lane & 7) + ((lane >> 4) << 3);
    fa = (uint32_t)(fr * 128 + ((((lane >> 3) & 1) ^ (fr & 7)) << 4));
  } else {
    const int sw = NT >= 8 ? lr & 7 : NT == 4 ? (lr >> 1) & 3 : (lr >> 2) & 1;
    fa = (uint32_t)(lr * (R * 2) + ((lc ^ sw) << 4));
  }

#pragma unroll
  for (int i = 0; i < DEPTH - 1; ++i) load();
  int ci = 0, ai = -1;
  for (int item = 0; item < items; ++item) {
    if (++ai == count) ai = 0, ++ci;
    cp_async_wait<DEPTH - 2>();
    const uint32_t xb = x_off + (uint32_t)((ci & (DEPTH - 1)) * rows * 128), fb = f_off + (uint32_t)((item & (DEPTH - 1)) * R * 128);
    if (drop && ai == 0) {
      const uint32_t c = (uint32_t)((c0 + ci) * (CK / 8) + xc);
#pragma unroll 2
      for (int row = xr; row < x_rows; row += 32) {
        uint4* q = reinterpret_cast<uint4*>(sraw + (xb - x_off) + (row - xr) * 128 + xs);
        *q = lora_dropped8(*q, c, (uint32_t)sm.row[row], p.drop, key);
      }
    }
    __syncthreads();
    load();
    const int a = sm.adapters[ai];
    const bool on0 = id0 == a, on1 = id1 == a;
    if (!__any_sync(0xffffffffu, on0 || on1)) continue;
#pragma unroll
    for (int ks = 0; ks < CK / 16; ++ks) {
      if ((ks & (KW - 1)) != kw) continue;
      uint32_t q[4];
      ldsm_x4(xb + (xa ^ (uint32_t)(ks << 5)), q[0], q[1], q[2], q[3]);
#pragma unroll
      for (int i = 0; i < NT; i += 2) {
        uint32_t b[4];
        if (!RM) {                         // (ranks 8 i .. + 7, k 0-7), (same, k 8-15), (the next 8 ranks, ..)
          ldsm_x4(fb + (uint32_t)(i * 1024) + (fa ^ (uint32_t)(ks << 5)), b[0], b[1], b[2], b[3]);
        } else {
          ldsm_x4_t(fb + (uint32_t)(ks * 16 * R * 2) + (fa ^ (uint32_t)(i << 4)), b[0], b[1], b[2], b[3]);
        }
        mma_16816(acc[i], q, b[0], b[1]);
        mma_16816(acc[i + 1], q, b[2], b[3]);
      }
    }
    if (!one || (++turns & 3) == 0) settle(on0 || one, on1 || one);
  }
  settle(true, true);
  cp_async_wait<0>();
  __syncthreads();

  // [warps][16][R + 4]: neighbouring rows on different banks
  constexpr int RP = R + 4;
  float* red = reinterpret_cast<float*>(sraw);
  float* mine = red + (size_t)warp * 16 * RP;
  const int t = lane & 3;
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    *reinterpret_cast<float2*>(&mine[g * RP + i * 8 + 2 * t]) = make_float2(sum[i][0], sum[i][1]);
    *reinterpret_cast<float2*>(&mine[(g + 8) * RP + i * 8 + 2 * t]) = make_float2(sum[i][2], sum[i][3]);
  }
  __syncthreads();
  __syncwarp();
  cluster_arrive();                        // (the cluster's barriers are a warp's together)
  cluster_wait();
  const int total = rows * R, e0 = (int)((long long)total * rank / S), e1 = (int)((long long)total * (rank + 1) / S);
  const uint32_t base = smem_u32(red);
  for (int e = e0 + (int)threadIdx.x; e < e1; e += LOW_THREADS) {
    const int j = e % R, row = e / R;
    if (j >= p.r || row >= x_rows) continue;
    const int m = sm.row[row];
    float v = 0.f;
    for (int w = 0; w < KW; ++w) v += dsmem_sum(base + 4u * (uint32_t)((w * rows + row) * RP + j), S);
    const int a = p.adapter[m];
    p.u[(size_t)m * p.r + j] = a >= 0 && a < p.n ? v * (p.scaling[a] * p.keep_inv) : 0.f;
  }
  __syncwarp();
  cluster_arrive();                        // nobody leaves while its sums are read
  cluster_wait();
}

CS_DEV float dot2(uint32_t a, uint32_t b, float c) {
  c = fmaf(__uint_as_float(a << 16), __uint_as_float(b << 16), c);
  return fmaf(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u), c);
}
CS_DEV float dot8(uint4 a, uint4 b, float c) { return dot2(a.w, b.w, dot2(a.z, b.z, dot2(a.y, b.y, dot2(a.x, b.x, c)))); }

// A CTA per row and p.ranks of its ranks (one row at rank 64, 5576 columns: 13 us by one CTA, 5 by four).  Rows of the factor along
// the contraction: a warp takes two ranks and half of the contraction; along the rank: a thread takes eight ranks and every
// few rows of the factor.
template <bool RM>
__global__ void __launch_bounds__(ROW_THREADS) low_row_kernel(const LowArgs p) {
  __shared__ float part[16][128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int m = (int)blockIdx.x, j0 = (int)blockIdx.y * p.ranks, j1 = min(p.r, j0 + p.ranks);
  griddep_wait();
  griddep_launch_dependents();
  const int a = lora_adapter(p.adapter, m, p.n, p.err);
  if (a < 0) {
    for (int j = j0 + threadIdx.x; j < j1; j += ROW_THREADS) p.u[(size_t)m * p.r + j] = 0.f;
    return;
  }
  const __nv_bfloat16* x = p.x + (long long)m * p.ldx;
  const __nv_bfloat16* f = p.f + (size_t)a * p.r * p.C;
  const float c = p.scaling[a] * p.keep_inv;
  if (!RM) {
    const bool drop = p.drop.thr != 0u;
    LoraKey key{0, 0};
    if (drop) key = lora_key(p.drop);
    const int octets = p.C / 8, half = warp >> 3;
    const int o0 = half ? (octets + 1) / 2 : 0, o1 = half ? octets : (octets + 1) / 2;
    for (int j = j0 + 2 * (warp & 7); j < j1; j += 16) {
      const __nv_bfloat16* f0 = f + (size_t)j * p.C;
      float v0 = 0.f, v1 = 0.f;
#pragma unroll 8
      for (int o = o0 + lane; o < o1; o += 32) {
        uint4 xv = ldg16(x + 8 * o);
        const uint4 a0 = ldg16(f0 + 8 * o), a1 = ldg16(f0 + p.C + 8 * o);
        if (drop) xv = lora_dropped8(xv, (uint32_t)o, (uint32_t)m, p.drop, key);
        v0 = dot8(xv, a0, v0);
        v1 = dot8(xv, a1, v1);
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        v0 += __shfl_xor_sync(0xffffffffu, v0, d);
        v1 += __shfl_xor_sync(0xffffffffu, v1, d);
      }
      if (lane == 0) part[half][j] = v0, part[half][j + 1] = v1;
    }
    __syncthreads();
    for (int j = j0 + threadIdx.x; j < j1; j += ROW_THREADS) p.u[(size_t)m * p.r + j] = (part[0][j] + part[1][j]) * c;
  } else {
    int og = 1;                          // octets of the ranks, rounded up to a power of two
    while (og * 8 < j1 - j0) og <<= 1;
    const int j = threadIdx.x & (og - 1), step = ROW_THREADS / og;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (j0 + 8 * j < j1) {
#pragma unroll 8
      for (int k = threadIdx.x / og; k < p.C; k += step) {
        const float xv = __bfloat162float(x[k]);
        const uint4 b = ldg16(f + (size_t)k * p.r + j0 + 8 * j);
        const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[2 * i] = fmaf(xv, __uint_as_float(w[i] << 16), v[2 * i]);
          v[2 * i + 1] = fmaf(xv, __uint_as_float(w[i] & 0xffff0000u), v[2 * i + 1]);
        }
      }
    }
    for (int d = 16; d >= og; d >>= 1)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
    if (lane < og) {
#pragma unroll
      for (int i = 0; i < 8; ++i) part[warp][lane * 8 + i] = v[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < j1 - j0; i += ROW_THREADS) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < 16; ++w) s += part[w][i];
      p.u[(size_t)m * p.r + j0 + i] = s * c;
    }
  }
}

template <int NT, bool RM>
cudaError_t launch_low_tile(const LowArgs& p, int tiles, int num_sms, cudaStream_t stream) {
  static KernelLimits lim;
  const int rows = 16 << p.rw_log2;
  const size_t smem = low_bytes(rows, NT * 8);
  static_assert(8 * 16 * (NT * 8 + 4) * sizeof(float) <= low_bytes(32, NT * 8) - sizeof(LowSmem), "the sums take the ring's place");
  const void* kern = (const void*)low_tile_kernel<NT, RM>;
  const cudaError_t e = ensure_kernel_limits(kern, lim, smem, false);
  if (e != cudaSuccess) return e;
  // (a CTA costs about ten chunks' time besides its chunks)
  const int dev = current_device();
  const int splits = pick_splits(tiles, (p.C + CK - 1) / CK, 10, [&](int s) {
    return resident_clusters(kern, lim, dev, 4 * p.rw_log2 - 4 + (s == 8 ? 3 : s / 2), LOW_THREADS, smem, s, num_sms);
  });
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * splits));
  cfg.blockDim = dim3(LOW_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, low_tile_kernel<NT, RM>, p);
}

template <bool RM>
cudaError_t launch_low(LowArgs p, int num_sms, cudaStream_t stream) {
  if ((long long)p.M * p.r * p.C <= (p.M <= 64 || (p.M <= 256 && p.n >= 4) ? LOW_ROW_MANY : LOW_ROW_MAX)) {
    // as many CTAs as the SMs hold at once
    p.ranks = 16;
    while (p.ranks < p.r && (long long)p.M * ((p.r + p.ranks - 1) / p.ranks) > 4 * num_sms) p.ranks += 16;
    return launch_pdl(low_row_kernel<RM>, dim3((unsigned)p.M, (unsigned)((p.r + p.ranks - 1) / p.ranks)), dim3(ROW_THREADS), 0, stream, p);
  }
  // 128 rows a CTA share an adapter's factor; fewer where that leaves SMs without work
  p.rw_log2 = 3;
  while (p.rw_log2 > 1 && (p.M + (16 << p.rw_log2) - 1) / (16 << p.rw_log2) * 8 < num_sms) --p.rw_log2;
  const int tiles = (p.M + (16 << p.rw_log2) - 1) / (16 << p.rw_log2);
  p.sort = p.n >= 4 && tiles > 1;
  const int nt = (p.r + 7) / 8;
  if (nt <= 2) return launch_low_tile<2, RM>(p, tiles, num_sms, stream);
  if (nt <= 4) return launch_low_tile<4, RM>(p, tiles, num_sms, stream);
  if (nt <= 8) return launch_low_tile<8, RM>(p, tiles, num_sms, stream);
  return launch_low_tile<16, RM>(p, tiles, num_sms, stream);
}

}  // namespace

cudaError_t launch_lora_low(const LoraArgs& a, bool backward, int num_sms, int* err, cudaStream_t stream) {
  LowArgs p{};
  p.x = backward ? a.dy : a.x;
  p.ldx = backward ? a.ldy : a.ldx;
  p.f = backward ? a.b : a.a;
  p.scaling = a.scaling;
  p.adapter = a.adapter;
  p.u = backward ? a.t : a.u;
  p.M = a.M;
  p.C = backward ? a.N : a.K;
  p.r = a.r;
  p.n = a.n;
  p.keep_inv = 65536.f / (65536.f - (float)a.thr);
  p.drop = LoraDrop{a.seed, a.site, backward ? 0u : a.thr};
  p.err = err;
  return backward ? launch_low<true>(p, num_sms, stream) : launch_low<false>(p, num_sms, stream);
}

}  // namespace cospec
