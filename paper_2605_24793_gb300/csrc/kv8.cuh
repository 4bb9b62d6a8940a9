// Shared by the kernels of the 8-bit KV cache: e4m3 codes and their power-of-two scales.
#pragma once

#include "cospec_device.cuh"

namespace cospec {

constexpr int KV8_PAGE = 16;     // tokens of a page

// pow2(a, c) for c = (1 + frac / 2^23) 2^e: the smallest power of two s with a <= c s, its exponent
// kept in [-100, 120].  a is not negative; below 2^-126 the lower bound holds anyway.
CS_DEV float kv8_pow2(float a, uint32_t frac, int e) {
  const uint32_t u = __float_as_uint(a);
  const int k = (int)(u >> 23) - 127 - e + ((u & 0x7fffffu) > frac ? 1 : 0);
  return __uint_as_float((uint32_t)(min(max(k, -100), 120) + 127) << 23);
}
CS_DEV float kv8_scale_of(float amax) { return kv8_pow2(amax, 0x600000u, 8); }    // c = 448 = 1.75 * 2^8
CS_DEV float kv8_scale127(float amax) { return kv8_pow2(amax, 0x7e0000u, 6); }    // c = 127 = 1.984375 * 2^6
// 1 / s of a power of two with its exponent in [-100, 120]
CS_DEV float kv8_inverse(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// |x|, or 0 where x is not finite.
CS_DEV float kv8_finite_abs(float x) {
  const float a = fabsf(x);
  return a <= 3.4028235e38f ? a : 0.f;
}

// x * inv, NaN where x is not finite: an infinity has no code, and the conversion would hold it as the
// largest one.
CS_DEV float kv8_scaled(float x, float inv) { return fmaf(x, inv, x * 0.f); }
// Values within a scale to e4m3, round to nearest even, NaN to NaN; the first in the lowest byte.
CS_DEV uint32_t kv8_pack4(const float (&x)[4]) {
  uint32_t r;
  asm("{\n .reg .b16 l, h;\n cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n"
      " mov.b32 %0, {l, h};\n}\n"
      : "=r"(r)
      : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]));
  return r;
}
// The two codes of `w`'s low half as f16 (exact).
CS_DEV uint32_t kv8_f16x2(uint32_t w) {
  uint32_t r;
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.rn.f16x2.e4m3x2 %0, l;\n}\n" : "=r"(r) : "r"(w));
  return r;
}
CS_DEV uint32_t kv8_f16x2_hi(uint32_t w) {
  uint32_t r;
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.rn.f16x2.e4m3x2 %0, h;\n}\n" : "=r"(r) : "r"(w));
  return r;
}
CS_DEV float2 kv8_floats(uint32_t w) {       // the low half's codes
  const uint32_t h = kv8_f16x2(w);
  float2 f;
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}\n"
      : "=f"(f.x), "=f"(f.y)
      : "r"(h));
  return f;
}
CS_DEV void kv8_floats4(uint32_t w, float (&f)[4]) {
  const float2 a = kv8_floats(w), b = kv8_floats(w >> 16);
  f[0] = a.x;
  f[1] = a.y;
  f[2] = b.x;
  f[3] = b.y;
}

// 16 bytes to shared memory, asynchronously, past L1; a warp's copies are counted in groups.  (Against bulk copies of
// whole page-heads with a barrier each: the same times, and nothing that could be waited for in vain.)
CS_DEV void kv8_copy16(uint32_t dst, const void* src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
CS_DEV void kv8_copy_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
CS_DEV void kv8_copy_wait() {               // all but the newest N groups have landed
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

CS_DEV uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
CS_DEV void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
CS_DEV void mma_f16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) { mma_f16(c, a[0], a[1], a[2], a[3], b0, b1); }
// A power of two, -126 <= k <= 127 (0 for -127), and the exponent of one (of 0: -127).
CS_DEV float kv8_two_to(int k) { return __uint_as_float((uint32_t)(127 + k) << 23); }
CS_DEV float kv8_exponent(float s) { return (float)((int)(__float_as_uint(s) >> 23) - 127); }
// Four codes as bf16 (exact), the lower two in `a`.
CS_DEV void kv8_codes_bf16(uint32_t w, uint32_t& a, uint32_t& b) {
  float x[4];
  kv8_floats4(w, x);
  a = pack_bf16(x[0], x[1]);
  b = pack_bf16(x[2], x[3]);
}

// Two bf16 with 0 in the place of infinities and NaN.
CS_DEV uint32_t kv8_finite_bf16x2(uint32_t w) { return w & ~__vcmpeq2(w & 0x7f807f80u, 0x7f807f80u); }

// Four bf16 of a 16-bit row.
CS_DEV void kv8_floats_of(uint2 u, float (&x)[4]) {
  x[0] = __uint_as_float(u.x << 16);
  x[1] = __uint_as_float(u.x & 0xffff0000u);
  x[2] = __uint_as_float(u.y << 16);
  x[3] = __uint_as_float(u.y & 0xffff0000u);
}
CS_DEV void kv8_store4(__nv_bfloat16* p, const float (&x)[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
}

}  // namespace cospec
