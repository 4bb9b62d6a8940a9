// The RL stage's objective and its gradient through the decision MLP (Sec. 3.4; the forward pass is
// arbitrate.cu's).  For every effective decision (a mismatch at or before the first rejection)
//   z = w2 . relu(W1 f + b1) + b2,  p = sigma(z),  pi = p or 1 - p by the action taken,  ratio = pi / pi_old
//   loss = -sum min(ratio A, clip(ratio) A) - beta_h sum H(p) + beta_kl sum KL(p || p_ref)
//   dz   = -A ratio (a - p) [the unclipped side counts] + p (1 - p) (beta_h z + beta_kl (z - logit p_ref))
// and, with S_h = sum dz 1[unit h is on] (f, 1) in nine numbers, all gradients follow from S alone:
//   dW1_h = w2_h S_h,  db1_h = w2_h S_h8,  dw2_h = W1_h . S_h + b1_h S_h8   (relu(x) = 1[x > 0] x),  db2 = sum dz.
//
// About a tenth of the positions are effective, so a CTA takes 512 positions at a time, compacts the
// effective ones and gathers what they need into shared memory.  Their products with the MLP run with the hidden
// units on the lanes: a thread keeps one or two pairs of units' weights and their sums S in registers (pairs, so
// that each instruction does two units), and every decision's features come by broadcast.  Each sum over the
// decisions then needs no exchange between threads; z does, one butterfly for four decisions.  Which units are on
// is kept as bits between the two walks.  H up to 64 units fits one warp, and the eight warps take
// decisions in turn; 256 units take two.  All sums have a fixed order.
// The terms of the loss are summed in 64 bits.  KL is p g(-d/p) + q g(d/q), d = p - p_ref, g(x) = x -
// log(1 + x), whose first-order terms are gone before they could cancel.
#include <math.h>

#include "cospec_device.cuh"
#include "cospec_internal.h"

namespace cospec {

namespace {

constexpr int THREADS = 256;
constexpr int STEP = 512;                 // positions of a step
constexpr int PER = STEP / THREADS;
constexpr int MAX_CTAS = 512;
constexpr int FIN_THREADS = 1024;

struct LossSmem {
  float feat[STEP][8];
  float adv[STEP], old[STEP], ref[STEP], g[STEP];
  int at[STEP];                           // position | action taken << 31
  uint32_t match[STEP / 32 + 2], act[STEP / 32];
};

// g(x) = x - log(1 + x), x >= -1
CS_DEV float log_rest(float x) {
  if (fabsf(x) < 0.25f) {
    // sum over k of (-x)^k / (k + 2), k to 11: the next term is below 2^-27 of the first
    float s = 1.f / 13.f;
    s = fmaf(-x, s, 1.f / 12.f);
    s = fmaf(-x, s, 1.f / 11.f);
    s = fmaf(-x, s, 1.f / 10.f);
    s = fmaf(-x, s, 1.f / 9.f);
    s = fmaf(-x, s, 1.f / 8.f);
    s = fmaf(-x, s, 1.f / 7.f);
    s = fmaf(-x, s, 1.f / 6.f);
    s = fmaf(-x, s, 1.f / 5.f);
    s = fmaf(-x, s, 1.f / 4.f);
    s = fmaf(-x, s, 1.f / 3.f);
    s = fmaf(-x, s, 0.5f);
    return x * x * s;
  }
  return x - log1pf(x);
}

struct Decision {
  float p, dz, surr, ent, kl;
};

CS_DEV Decision decide(float z, float adv, float old, float ref, bool took, const ArbLossArgs& a) {
  Decision d;
  const float e = expf(-fabsf(z)), big = 1.f / (1.f + e), small = e * big;
  const float p = z >= 0.f ? big : small, q = z >= 0.f ? small : z < 0.f ? big : z;
  d.p = z >= 0.f ? big : z < 0.f ? small : z;          // NaN stays
  const float ratio = (took ? p : q) / (took ? old : 1.f - old);
  const float plain = ratio * adv, cut = fminf(fmaxf(ratio, 1.f - a.clip_eps), 1.f + a.clip_eps) * adv;
  const bool inside = !(plain > cut);
  d.surr = inside ? plain : cut;
  d.ent = log1pf(e) + (small > 0.f ? fabsf(z) * small : 0.f);
  // p - p_ref from the sides that are not near 1
  const float diff = z >= 0.f ? (1.f - ref) - q : p - ref;
  d.kl = (p > 0.f ? p * log_rest(-diff / p) : -diff) + (q > 0.f ? q * log_rest(diff / q) : diff);
  const float pq = p * q;
  const float pull = pq > 0.f ? pq * (a.beta_h * z + a.beta_kl * (z - logf(ref / (1.f - ref)))) : pq;
  d.dz = (inside ? -plain * (took ? q : -p) : 0.f) + pull;
  return d;
}

// PP: pairs of units of a thread; TW: warps that hold all units.
template <int PP, int TW>
__global__ void __launch_bounds__(THREADS) arb_loss_kernel(const ArbLossArgs a, float* ws_s, double* ws_l) {
  extern __shared__ __align__(16) uint8_t raw[];
  LossSmem& sm = *reinterpret_cast<LossSmem*>(raw);
  constexpr int TEAMS = 8 / TW;
  constexpr int HP = 64 * PP * TW;                     // units that the threads hold
  float* zpart = reinterpret_cast<float*>(raw + sizeof(LossSmem));               // [TW][STEP]
  uint16_t* on = reinterpret_cast<uint16_t*>(zpart + TW * STEP);                 // [STEP / 4][TW * 32]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int team = warp / TW, tw = warp % TW;
  griddep_wait();
  griddep_launch_dependents();

  // units 2 j, 2 j + 1 of pair j = (i TW + tw) 32 + lane
  float2 w1[PP][8], b1[PP], w2[PP], S[PP][9];
#pragma unroll
  for (int i = 0; i < PP; ++i) {
    const int h = 2 * ((i * TW + tw) * 32 + lane);
    const bool x = h < a.H, y = h + 1 < a.H;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      w1[i][k] = make_float2(x ? a.w1[(size_t)h * 8 + k] : 0.f, y ? a.w1[(size_t)(h + 1) * 8 + k] : 0.f);
    b1[i] = make_float2(x ? a.b1[h] : 0.f, y ? a.b1[h + 1] : 0.f);
    w2[i] = make_float2(x ? a.w2[h] : 0.f, y ? a.w2[h + 1] : 0.f);
#pragma unroll
    for (int k = 0; k < 9; ++k) S[i][k] = make_float2(0.f, 0.f);
  }
  const float b2 = *a.b2, inv_k = 1.f / (float)a.K;
  const int total = a.n * a.K;
  double sums[4] = {0., 0., 0., 0.};

  for (long long base = (long long)blockIdx.x * STEP; base < total; base += (long long)gridDim.x * STEP) {
    int pos[PER];
    bool act[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const long long e = base + j * THREADS + tid;
      bool match = false;
      act[j] = false;
      pos[j] = (int)e;
      if (e < total) {
        const int r = (int)e / a.K, i = (int)e - r * a.K;
        match = a.draft[e] == a.argmax[(size_t)r * (a.K + 1) + i];
        act[j] = !match && a.eff[e] != 0;
        if (!act[j]) {
          a.p_new[e] = 0.f;
          a.dz[e] = 0.f;
        }
      }
      const unsigned mm = __ballot_sync(0xffffffffu, match), aa = __ballot_sync(0xffffffffu, act[j]);
      if (lane == 0) {
        sm.match[2 + j * 8 + warp] = mm;
        sm.act[j * 8 + warp] = aa;
      }
    }
    if (warp < 2) {                          // the positions before the step that may be of its first round
      const long long e = base - 64 + warp * 32 + lane;
      bool match = false;
      if (e >= 0) {
        const int r = (int)e / a.K, i = (int)e - r * a.K;
        match = a.draft[e] == a.argmax[(size_t)r * (a.K + 1) + i];
      }
      const unsigned mm = __ballot_sync(0xffffffffu, match);
      if (lane == 0) sm.match[warp] = mm;
    }
    __syncthreads();
    int count = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      int at = 0;
      count = 0;
#pragma unroll
      for (int w = 0; w < STEP / 32; ++w) {
        const int c = __popc(sm.act[w]);
        if (w < j * 8 + warp) at += c;
        count += c;
      }
      if (act[j]) {
        at += __popc(sm.act[j * 8 + warp] & ((1u << lane) - 1u));
        const int e = pos[j], r = e / a.K, i = e - r * a.K;
        const float* s0 = a.stats + ((size_t)r * (a.K + 1) + i) * 5;
        const float* s1 = s0 + 5;
        const float x0 = s0[0], x1 = s0[1], x2 = s0[2], x3 = s0[3], x4 = s0[4], y0 = s1[0], y2 = s1[2], y4 = s1[4];
        const float adv = a.adv[e], old = a.p_old[e], ref = a.p_ref[e];
        const bool took = a.accept[e] != 0;
        int before = 0;                      // matches of the round before position i: bits [lo, hi) of match
        const int hi = 64 + j * THREADS + tid, lo = hi - i;
#pragma unroll
        for (int w = 0; w < 3; ++w) {
          const int word = (hi >> 5) - w;
          if (word < 0 || word * 32 + 32 <= lo) continue;
          uint32_t m = sm.match[word];
          if (word * 32 + 32 > hi) m &= (1u << (hi & 31)) - 1u;
          if (word * 32 < lo) m &= 0xffffffffu << (lo & 31);
          before += __popc(m);
        }
        float4* f = reinterpret_cast<float4*>(sm.feat[at]);
        f[0] = make_float4(x4 - x2, x0 - x2, x0 - x1, x3);
        f[1] = make_float4(y0 - y2, i + 1 < a.K ? y4 - y2 : 0.f, (float)(i + 1) * inv_k, (float)before * inv_k);
        sm.adv[at] = adv;
        sm.old[at] = old;
        sm.ref[at] = ref;
        sm.at[at] = took ? (int)((unsigned)e | 0x80000000u) : e;
      }
    }
    __syncthreads();
    const int groups = (count + 3) / 4;
    for (int q = team; q < groups; q += TEAMS) {
      float z[4];
      unsigned bits = 0;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const float4 fa = *reinterpret_cast<const float4*>(&sm.feat[4 * q + d][0]);
        const float4 fb = *reinterpret_cast<const float4*>(&sm.feat[4 * q + d][4]);
        const float f[8] = {fa.x, fa.y, fa.z, fa.w, fb.x, fb.y, fb.z, fb.w};
        float2 zz = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < PP; ++i) {
          float2 v = b1[i];
#pragma unroll
          for (int k = 0; k < 8; ++k) v = fma2(w1[i][k], make_float2(f[k], f[k]), v);
          bits |= ((v.x > 0.f ? 1u : 0u) | (v.y > 0.f ? 2u : 0u)) << (4 * d + 2 * i);
          zz = fma2(w2[i], make_float2(fmaxf(v.x, 0.f), fmaxf(v.y, 0.f)), zz);
        }
        z[d] = zz.x + zz.y;
      }
      on[q * (TW * 32) + tw * 32 + lane] = (uint16_t)bits;
      // four sums over the warp; lanes 0, 8, 16, 24 end with decisions 0, 1, 2, 3
      const bool up = lane & 16, up2 = lane & 8;
      const float s0 = __shfl_xor_sync(0xffffffffu, up ? z[0] : z[2], 16), s1 = __shfl_xor_sync(0xffffffffu, up ? z[1] : z[3], 16);
      const float t0 = (up ? z[2] : z[0]) + s0, t1 = (up ? z[3] : z[1]) + s1;
      float v = (up2 ? t1 : t0) + __shfl_xor_sync(0xffffffffu, up2 ? t0 : t1, 8);
      v += __shfl_xor_sync(0xffffffffu, v, 4);
      v += __shfl_xor_sync(0xffffffffu, v, 2);
      v += __shfl_xor_sync(0xffffffffu, v, 1);
      if ((lane & 7) == 0) zpart[tw * STEP + 4 * q + (lane >> 3)] = v;
    }
    __syncthreads();
    for (int d = tid; d < 4 * groups; d += THREADS) {
      float g = 0.f;
      if (d < count) {
        float z = zpart[d];
#pragma unroll
        for (int w = 1; w < TW; ++w) z += zpart[w * STEP + d];
        const int at = sm.at[d];
        const Decision x = decide(z + b2, sm.adv[d], sm.old[d], sm.ref[d], at < 0, a);
        const int e = at & 0x7fffffff;
        g = x.dz * a.grad_scale;
        a.p_new[e] = x.p;
        a.dz[e] = g;
        sums[0] += (double)x.surr;
        sums[1] += (double)x.ent;
        sums[2] += (double)x.kl;
        sums[3] += (double)g;
      }
      sm.g[d] = g;
    }
    __syncthreads();
    for (int q = team; q < groups; q += TEAMS) {
      const unsigned bits = on[q * (TW * 32) + tw * 32 + lane];
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        if (4 * q + d >= count) break;       // what stands there is of another step
        const float4 fa = *reinterpret_cast<const float4*>(&sm.feat[4 * q + d][0]);
        const float4 fb = *reinterpret_cast<const float4*>(&sm.feat[4 * q + d][4]);
        const float f[8] = {fa.x, fa.y, fa.z, fa.w, fb.x, fb.y, fb.z, fb.w};
        const float g = sm.g[4 * q + d];
#pragma unroll
        for (int i = 0; i < PP; ++i) {
          const float2 m = make_float2((bits >> (4 * d + 2 * i)) & 1u ? g : 0.f, (bits >> (4 * d + 2 * i)) & 2u ? g : 0.f);
#pragma unroll
          for (int k = 0; k < 8; ++k) S[i][k] = fma2(m, make_float2(f[k], f[k]), S[i][k]);
          S[i][8] = add2(S[i][8], m);
        }
      }
    }
    __syncthreads();
  }

  // the teams' sums, then the CTA's to the workspace: [9][HP]
  float* red = reinterpret_cast<float*>(raw);          // [TEAMS][9][HP]
#pragma unroll
  for (int i = 0; i < PP; ++i)
#pragma unroll
    for (int k = 0; k < 9; ++k)
      *reinterpret_cast<float2*>(&red[(team * 9 + k) * HP + 2 * ((i * TW + tw) * 32 + lane)]) = S[i][k];
  __syncthreads();
  for (int e = tid; e < 9 * HP; e += THREADS) {
    float s = red[e];
#pragma unroll
    for (int m = 1; m < TEAMS; ++m) s += red[m * 9 * HP + e];
    ws_s[(size_t)blockIdx.x * 9 * HP + e] = s;
  }
  __syncthreads();
  double* wsum = reinterpret_cast<double*>(raw);       // [8][4]
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    double v = sums[k];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) wsum[warp * 4 + k] = v;
  }
  __syncthreads();
  if (tid < 4) {
    double v = 0.;
    for (int w = 0; w < 8; ++w) v += wsum[w * 4 + tid];
    ws_l[(size_t)blockIdx.x * 4 + tid] = v;
  }
}

// The CTAs' sums of 32 units (a lane each; 32 warps take CTAs in turn), then the gradients; block 0 the loss.
__global__ void __launch_bounds__(FIN_THREADS) arb_loss_finish_kernel(const ArbLossArgs a, const float* ws_s, const double* ws_l, int ctas, int hp) {
  __shared__ double part[32][33];
  __shared__ double tot[9][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = blockIdx.x * 32 + lane;
  griddep_wait();
  griddep_launch_dependents();
  float s[9];
  double sd[9];
#pragma unroll
  for (int k = 0; k < 9; ++k) sd[k] = 0.;
  for (int c = warp; c < ctas; c += 32) {
#pragma unroll
    for (int k = 0; k < 9; ++k) s[k] = ws_s[((size_t)c * 9 + k) * hp + h];
#pragma unroll
    for (int k = 0; k < 9; ++k) sd[k] += (double)s[k];
  }
  for (int k = 0; k < 9; ++k) {
    part[warp][lane] = sd[k];
    __syncthreads();
    double v = part[lane][warp];           // warp: unit, lane: part
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) tot[k][warp] = v;
    __syncthreads();
  }
  if (warp == 0 && h < a.H) {
    const double w2 = (double)a.w2[h];
    double dw2 = (double)a.b1[h] * tot[8][lane];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      a.dw1[(size_t)h * 8 + k] = (float)(w2 * tot[k][lane]);
      dw2 += (double)a.w1[(size_t)h * 8 + k] * tot[k][lane];
    }
    a.db1[h] = (float)(w2 * tot[8][lane]);
    a.dw2[h] = (float)dw2;
  }
  if (blockIdx.x == 0 && warp == 1) {
    double v[4] = {0., 0., 0., 0.};
    for (int c = lane; c < ctas; c += 32)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += ws_l[(size_t)c * 4 + k];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    if (lane == 0) {
      a.loss[0] = (float)v[0];
      a.loss[1] = (float)v[1];
      a.loss[2] = (float)v[2];
      a.loss[3] = (float)(-v[0] - (double)a.beta_h * v[1] + (double)a.beta_kl * v[2]);
      *a.db2 = (float)v[3];
    }
  }
}

int padded_units(int H) { return H <= 64 ? 64 : H <= 128 ? 128 : H <= 256 ? 256 : H <= 512 ? 512 : 1024; }

template <int PP, int TW>
cudaError_t launch_loss(const ArbLossArgs& a, int num_sms, cudaStream_t stream) {
  static KernelLimits lim;
  constexpr int HP = 64 * PP * TW;
  size_t smem = sizeof(LossSmem) + (size_t)TW * STEP * 4 + (size_t)(STEP / 4) * TW * 32 * 2;
  const size_t red = (size_t)(8 / TW) * 9 * HP * 4;
  if (smem < red) smem = red;
  cudaError_t e = ensure_kernel_limits((const void*)arb_loss_kernel<PP, TW>, lim, smem, false);
  if (e != cudaSuccess) return e;
  const long long steps = ((long long)a.n * a.K + STEP - 1) / STEP;
  int ctas = 2 * num_sms;
  if (ctas > MAX_CTAS) ctas = MAX_CTAS;
  if (ctas > steps) ctas = (int)steps;
  if (ctas < 1) ctas = 1;
  double* ws_l = static_cast<double*>(a.ws);
  float* ws_s = reinterpret_cast<float*>(ws_l + (size_t)MAX_CTAS * 4);
  e = launch_pdl(arb_loss_kernel<PP, TW>, dim3(ctas), dim3(THREADS), smem, stream, a, ws_s, ws_l);
  if (e != cudaSuccess) return e;
  return launch_pdl(arb_loss_finish_kernel, dim3((a.H + 31) / 32), dim3(FIN_THREADS), 0, stream, a, (const float*)ws_s, (const double*)ws_l, ctas, HP);
}

}  // namespace

size_t arb_loss_ws_bytes(int H) { return (size_t)MAX_CTAS * (32 + (size_t)9 * padded_units(H) * 4); }

cudaError_t launch_arb_loss(const ArbLossArgs& a, int num_sms, cudaStream_t stream) {
  if (a.H <= 64) return launch_loss<1, 1>(a, num_sms, stream);
  if (a.H <= 128) return launch_loss<2, 1>(a, num_sms, stream);
  if (a.H <= 256) return launch_loss<2, 2>(a, num_sms, stream);
  if (a.H <= 512) return launch_loss<2, 4>(a, num_sms, stream);
  return launch_loss<2, 8>(a, num_sms, stream);
}

}  // namespace cospec
