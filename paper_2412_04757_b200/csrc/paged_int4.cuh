// Cached rows of 4 bits an element (LTRI_TYPE_INT4): the numbers -7 to 7 as number + 8, two a byte, and for every 32 elements a
// scale of 8 bits, which are the upper half of a half without its sign (5 bits of exponent, 3 of mantissa), up to 480.
//
// value = number * scale has at most 7 significant bits.  As halves the values carry a factor 2^-3 (kI4Back undoes it): n times
// the largest scale is then 420, and what the number's offset costs below, 129 times the scale's half, 61920.
#pragma once

#include "paged.cuh"

namespace ltri {

constexpr int kI4Block = 32;            // elements that share a scale
constexpr unsigned kI4Largest = 0xBF;   // byte of the largest scale, 480
constexpr unsigned kI4Nan = 0xFC;       // of a block that holds a NaN
constexpr float kI4Back = 8.f;

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t i4_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t i4_mul(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// Two scales as halves: byte `lo` of a in the lower half, byte `hi` of b in the upper one.
__device__ __forceinline__ uint32_t i4_scales(uint32_t a, int lo, uint32_t b, int hi) {
  return (__byte_perm(a, b, lo | (4 + hi) << 8) & 0x00ff00ffu) << 7;
}
__device__ __forceinline__ float2 i4_scales_f32(uint32_t a, int lo, uint32_t b, int hi) {
  const uint32_t x = i4_scales(a, lo, b, hi);
  return __half22float2(*reinterpret_cast<const __half2*>(&x));
}

// Numbers to values.  Four bits below an exponent of 2^10 are 1024 + number + 8, or 1024 + 16 (number + 8) where they stand four
// places higher: a multiply-add takes the offset away and the scale in, exactly (1032 and 1152 times a scale's four significant
// bits have no more than eleven).
struct __align__(16) I4Scale {
  uint32_t s0, c0, s1, c1;
};
__device__ __forceinline__ I4Scale i4_factors(uint32_t halves) {
  I4Scale f;
  f.s0 = i4_mul(halves, 0x30003000u);  // 2^-3
  f.c0 = i4_mul(halves, 0xD808D808u);  // -1032 * 2^-3 = -129
  f.s1 = i4_mul(halves, 0x20002000u);  // 2^-7
  f.c1 = i4_mul(halves, 0xC880C880u);  // -1152 * 2^-7 = -9
  return f;
}
// (x & MASK) | 0x64006400, one instruction
template <uint32_t MASK>
__device__ __forceinline__ uint32_t i4_raised(uint32_t x) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(x), "n"(MASK), "r"(0x64006400u));
  return d;
}
// Elements i and i + 4 of the eight in w (of two rows' four each, the same element of both), for i = 0 to 3.
__device__ __forceinline__ void i4_values(uint32_t (&v)[4], uint32_t w, const I4Scale& f) {
  const uint32_t u = w >> 8;
  v[0] = i4_fma(i4_raised<0x000f000fu>(w), f.s0, f.c0);
  v[1] = i4_fma(i4_raised<0x00f000f0u>(w), f.s1, f.c1);
  v[2] = i4_fma(i4_raised<0x000f000fu>(u), f.s0, f.c0);
  v[3] = i4_fma(i4_raised<0x00f000f0u>(u), f.s1, f.c1);
}

// The scale nearest to x >= 0, ties to even, as its byte.  (An infinity may have become NaN in products: both are the largest one.)
__device__ __forceinline__ unsigned i4_scale_byte(float x) {
  x = fminf(x, 480.f);
  const unsigned u = __float_as_uint(x);
  // below 2^-14 the scales lie 2^-17 apart, as fp32's numbers from 64 to 128 do
  const float s = x < 0x1p-14f ? __fadd_rn(__fadd_rn(x, 96.f), -96.f)
                               : __uint_as_float((u + 0x7ffffu + (u >> 20 & 1u)) & 0xfff00000u);
  return __half_as_ushort(__float2half_rn(s)) >> 7;
}

__device__ __forceinline__ unsigned long long i4_pair(float a, float b) {
  unsigned long long x;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a), "f"(b));
  return x;
}
// (number + 8 of a value's quotient in the last bits, over 1.5 * 2^23) of a pair
__device__ __forceinline__ void i4_numbers(uint32_t& a, uint32_t& b, float2 x, float r, float rest) {
  unsigned long long y;
  asm("{\n.reg .b64 t;\nmul.rn.f32x2 t, %1, %3;\nfma.rn.f32x2 t, %1, %2, t;\nadd.rn.f32x2 %0, t, %4;\n}\n"
      : "=l"(y)
      : "l"(i4_pair(x.x, x.y)), "l"(i4_pair(r, r)), "l"(i4_pair(rest, rest)), "l"(i4_pair(12582920.f, 12582920.f)));
  asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(y));
}

// Eight elements of `type` by the four lanes of a block (neighbours, all of them here): their numbers, element i in bits 4i,
// and the block's scale.
// Quotients are products with a reciprocal in two terms, whose rounding is the quotient's where that is a midpoint: of two numbers,
// or of two scales (a quotient of up to eleven bits by 7 or by a scale is one, or further from it than fp32's rounding).
// (With divisions, clamps of every element and masks: 22700 tokens of eight KV heads of 128 40 us.)
__device__ __forceinline__ uint32_t i4_quantise(int type, const uint4& x, unsigned& scale) {
  const unsigned lanes = 0xfu << (threadIdx.x & 28);
  uint4 in = x;
  // magnitudes are ordered as their bits are, NaN above all
  uint32_t most = __vmaxu2(__vmaxu2(in.x & 0x7fff7fffu, in.y & 0x7fff7fffu), __vmaxu2(in.z & 0x7fff7fffu, in.w & 0x7fff7fffu));
  most = __vmaxu2(most, __shfl_xor_sync(lanes, most, 1));
  most = __vmaxu2(most, __shfl_xor_sync(lanes, most, 2));
  most = max(most & 0xffffu, most >> 16);
  if (most > (type == LTRI_TYPE_BF16 ? 0x7f80u : 0x7c00u)) {
    scale = kI4Nan;
    return 0x88888888u;
  }
  constexpr float kR7 = 1.f / 7.f, kRest7 = (float)(1.0 / 7.0 - (double)kR7);
  const float m = paged_unpack(type, most).x;
  scale = i4_scale_byte(__fmaf_rn(m, kR7, m * kRest7));
  const float s = __half2float(__ushort_as_half((unsigned short)(scale << 7)));
  if (s == 0.f) return 0x88888888u;
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
  const float rest = __fmaf_rn(-s, r, 1.f) * r;
  if (m >= 7.5f * s) {
    // beyond the largest scale, or between the smallest ones: elements are clamped (elsewhere m / s is 7.4375 at most)
    const float lim = 7.f * s;
    auto clamped = [&](uint32_t y) {
      const float2 f = paged_unpack(type, y);
      return paged_pack(type, fminf(fmaxf(f.x, -lim), lim), fminf(fmaxf(f.y, -lim), lim));
    };
    in = make_uint4(clamped(in.x), clamped(in.y), clamped(in.z), clamped(in.w));
  }
  uint32_t n[8];
  i4_numbers(n[0], n[1], paged_unpack(type, in.x), r, rest);
  i4_numbers(n[2], n[3], paged_unpack(type, in.y), r, rest);
  i4_numbers(n[4], n[5], paged_unpack(type, in.z), r, rest);
  i4_numbers(n[6], n[7], paged_unpack(type, in.w), r, rest);
  // their sum at distances of four bits, less what stands in front of the numbers
  uint32_t got = n[7];
#pragma unroll
  for (int i = 6; i >= 0; --i) got = got * 16u + n[i];
  return got - 0x4b400000u * 0x11111111u;
}
#endif

}  // namespace ltri
