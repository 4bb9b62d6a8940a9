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

// Dropout of eight neighbouring columns of a row: masks of two bf16 each, all ones where the element
// stays.  Columns 8 c .. 8 c + 7 of row m take the eight 16-bit halves, low before high, of Philox4x32-10
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
CS_DEV uint4 lora_keep8(uint32_t c, uint32_t m, const LoraDrop& d, LoraKey key) {
  const uint4 r = philox4x32_10(make_uint4(c, m, d.site, 2u), key.lo, key.hi);
  auto two = [&](uint32_t w) {
    return ((w & 0xffffu) >= d.thr ? 0xffffu : 0u) | ((w >> 16) >= d.thr ? 0xffff0000u : 0u);
  };
  return make_uint4(two(r.x), two(r.y), two(r.z), two(r.w));
}
// The same as eight bits, column 8 c in the lowest.
CS_DEV uint32_t lora_keep8_bits(uint32_t c, uint32_t m, const LoraDrop& d, LoraKey key) {
  const uint4 r = philox4x32_10(make_uint4(c, m, d.site, 2u), key.lo, key.hi);
  auto two = [&](uint32_t w) { return ((w & 0xffffu) >= d.thr ? 1u : 0u) | ((w >> 16) >= d.thr ? 2u : 0u); };
  return two(r.x) | two(r.y) << 2 | two(r.z) << 4 | two(r.w) << 6;
}

CS_DEV uint4 and4(uint4 a, uint4 b) { return make_uint4(a.x & b.x, a.y & b.y, a.z & b.z, a.w & b.w); }
CS_DEV uint4 ldg16(const void* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

// Transposes an 8 x 8 matrix of 16-bit values held as the mma fragments are.
CS_DEV uint32_t movmatrix_t(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// x as hi + lo, each rounded to bf16: 16 bits of its mantissa.  What is not finite stays in hi.
CS_DEV void lora_split2(float x, float& hi, float& lo) {
  hi = __bfloat162float(__float2bfloat16_rn(x));
  const float d = x - hi;
  lo = fabsf(hi) <= 3.4028235e38f ? d : 0.f;
}

}  // namespace cospec
