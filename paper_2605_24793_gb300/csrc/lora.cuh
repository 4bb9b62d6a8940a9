// Shared by the low-rank adapters' kernels: a row's adapter, the dropout mask, values in several bf16 parts.
#pragma once

#include "cospec_device.cuh"
#include "cospec_internal.h"

namespace cospec {

// The row's adapter: -1 for none, and (flagged) for an id outside the adapters.
CS_DEV int lora_adapter(const int32_t* adapter, int m, int n, int* err) {
  const int a = adapter[m];
  if (a >= n || a < -1) {
    set_err(err, ERR_ADAPTER);
    return -1;
  }
  return a;
}

// Dropout of eight neighbouring columns of a row.  Columns 8 c .. 8 c + 7 of row m take the eight 16-bit halves, low before high, of Philox4x32-10
// at counter (c, m, site, 2); an element stays where its half is at least the threshold.  The mask is a
// function of the element's place, so the passes that need it draw it again instead of storing it.
struct LoraDrop {
  const unsigned long long* seed;
  uint32_t site, thr;      // thr 0: nothing is dropped
};
struct LoraKey {
  uint32_t lo, hi;
};
CS_DEV LoraKey lora_key(const LoraDrop& d) {
  const unsigned long long s = *d.seed;
  return LoraKey{(uint32_t)s, (uint32_t)(s >> 32)};
}
// (the draw is half of the passes' instructions at rank 16: products of 64 bits in one instruction each)
CS_DEV uint4 lora_draw(uint32_t c, uint32_t m, const LoraDrop& d, LoraKey key) {
  uint4 v = make_uint4(c, m, d.site, 2u);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * v.x, b = (uint64_t)0xCD9E8D57u * v.z;
    v = make_uint4((uint32_t)(b >> 32) ^ v.y ^ (key.lo + (uint32_t)r * 0x9E3779B9u), (uint32_t)b,
                   (uint32_t)(a >> 32) ^ v.w ^ (key.hi + (uint32_t)r * 0xBB67AE85u), (uint32_t)a);
  }
  return v;
}
// x with its dropped elements zero.
CS_DEV uint4 lora_dropped8(uint4 x, uint32_t c, uint32_t m, const LoraDrop& d, LoraKey key) {
  const uint4 r = lora_draw(c, m, d, key);
  const uint32_t t = d.thr << 16;
  auto two = [&](uint32_t v, uint32_t w) {
    if ((w << 16) < t) v &= 0xffff0000u;
    if (w < t) v &= 0x0000ffffu;
    return v;
  };
  return make_uint4(two(x.x, r.x), two(x.y, r.y), two(x.z, r.z), two(x.w, r.w));
}
// The mask of the eight as bits, column 8 c in the lowest.
CS_DEV uint32_t lora_keep8_bits(uint32_t c, uint32_t m, const LoraDrop& d, LoraKey key) {
  const uint4 r = lora_draw(c, m, d, key);
  const uint32_t t = d.thr << 16;
  auto two = [&](uint32_t w) { return ((w << 16) >= t ? 1u : 0u) | (w >= t ? 2u : 0u); };
  return two(r.x) | two(r.y) << 2 | two(r.z) << 4 | two(r.w) << 6;
}

CS_DEV uint4 ldg16(const void* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

// x as hi + lo, each rounded to bf16: 16 bits of its mantissa.  What is not finite stays in hi.
CS_DEV void lora_split2(float x, float& hi, float& lo) {
  hi = __bfloat162float(__float2bfloat16_rn(x));
  const float d = x - hi;
  lo = fabsf(hi) <= 3.4028235e38f ? d : 0.f;
}

}  // namespace cospec
