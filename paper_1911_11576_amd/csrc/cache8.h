// Codes of a paged cache in 8 bits on the device: e4m3 (four exponent bits, three behind the first one, up to 448, NaN 0x7f and 0xff, no
// infinity) and whole numbers from -127 to 127.
#pragma once
#include "dev_common.h"
#include "paged.h"

namespace fs {

typedef short s16x2 __attribute__((ext_vector_type(2)));

template <typename T> constexpr float kLargest = __is_same(T, f16_t) ? 65504.f : __is_same(T, bf16_t) ? 0x1.fep+127f : 0x1.fffffep+127f;

struct E4m3 {
  // The largest number that a code over 2^power stands for and that is one of T: beyond, rounding could end at infinity.
  template <typename T> static __device__ __forceinline__ float most(int power) {
    const float x = __builtin_ldexpf(kLargest<T>, -power);      // (codes lie 2^-9 apart below 2^-6, else an eighth of a power of two)
    return __builtin_ldexpf(x < 0x1p-6f ? floorf(x * 512.f) * 0x1p-9f : fminf(as_f32(as_u32(x) & 0xfff00000u), 448.f), power);
  }
  // the least power of two that reaches x with a code of 448 = 1.75 * 2^8; 0 and subnormal numbers: one of -126 and less
  static __device__ __forceinline__ int power(float x) { return (int)(as_u32(x) >> 23) - 135 + ((as_u32(x) & 0x7fffffu) > 0x600000u); }
  // the codes of four numbers over 2^power (pack), of four of T as they lie in memory (pack_words): rounded once, to the nearest and the even one of two
  static __device__ __forceinline__ uint32_t pack(float a, float b, float c, float d, int power) {
    const float s = __builtin_ldexpf(1.f, power);
    const s16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s16x2{0, 0}, a, b, s, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, c, d, s, true));
  }
  template <typename T> static __device__ __forceinline__ uint32_t pack_words(uint32_t a, uint32_t b, int power) {
    const float s = __builtin_ldexpf(1.f, power);
    if constexpr (__is_same(T, bf16_t)) {
      const s16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(s16x2{0, 0}, __builtin_bit_cast(bf16x2, a), s, false);
      return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_bit_cast(bf16x2, b), s, true));
    } else {
      const s16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(s16x2{0, 0}, __builtin_bit_cast(f16x2, a), s, false);
      return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(lo, __builtin_bit_cast(f16x2, b), s, true));
    }
  }
  static __device__ __forceinline__ void unpack(uint32_t c, float (&x)[4]) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
  }
  // Four codes times `ratio`, as codes.  A product of 28 bits is rounded to the one of its two neighbours in fp32 whose last bit is 1, so that the rounding to a
  // code's four bits is that of the product itself, next to the middle of two codes too.
  static __device__ __forceinline__ uint32_t times(uint32_t c, float ratio) {
    float x[4];
    unpack(c, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = x[i] * ratio, left = fmaf(x[i], ratio, -p);
      const uint32_t u = as_u32(p);
      if (left != 0.f && !(u & 1)) x[i] = as_f32((left > 0.f) == (p > 0.f) ? u + 1 : u - 1);
      else x[i] = p;
    }
    return pack(x[0], x[1], x[2], x[3], 0);
  }
};

struct Int8 {
  template <typename T> static __device__ __forceinline__ float most(int power) { return __builtin_ldexpf(fminf(floorf(__builtin_ldexpf(kLargest<T>, -power)), 127.f), power); }
  // 127 = 1.984375 * 2^6
  static __device__ __forceinline__ int power(float x) { return (int)(as_u32(x) >> 23) - 133 + ((as_u32(x) & 0x7fffffu) > 0x7e0000u); }
  // four numbers times s, rounded once: 1.5 * 2^23 more leaves the nearest whole number, the even one of two, in the number's last bits
  static __device__ __forceinline__ uint32_t whole(float a, float b, float c, float d, float s) {
    const uint32_t w0 = as_u32(fmaf(a, s, 0x1.8p23f)), w1 = as_u32(fmaf(b, s, 0x1.8p23f)), w2 = as_u32(fmaf(c, s, 0x1.8p23f)), w3 = as_u32(fmaf(d, s, 0x1.8p23f));
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w3, w2, 0x0c0c0400u), __builtin_amdgcn_perm(w1, w0, 0x0c0c0400u), 0x05040100u);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b, float c, float d, int power) { return whole(a, b, c, d, __builtin_ldexpf(1.f, -power)); }
  template <typename T> static __device__ __forceinline__ uint32_t pack_words(uint32_t a, uint32_t b, int power) {
    if constexpr (__is_same(T, bf16_t)) return pack(bf16_to_f32(a & 0xffffu), as_f32(a & 0xffff0000u), bf16_to_f32(b & 0xffffu), as_f32(b & 0xffff0000u), power);
    else return pack(f16_to_f32(a & 0xffffu), f16_to_f32(a >> 16), f16_to_f32(b & 0xffffu), f16_to_f32(b >> 16), power);
  }
  static __device__ __forceinline__ void unpack(uint32_t c, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(c >> (8 * i));
  }
  static __device__ __forceinline__ uint32_t times(uint32_t c, float ratio) {
    float x[4];
    unpack(c, x);
    return whole(x[0], x[1], x[2], x[3], ratio);
  }
};

// Eight codes as numbers of T for the matrix unit: as they stand (plain: exact in both types), or the first four times s0 and the others times s1, rounded
// to T (scaled).  One instruction makes two numbers of e4m3 codes and takes a power of two with it: its scales are powers of two (power_of), and what
// is left of a scale (rest_of: 1 for what the store writes) goes into the dot's other operand or its result.  Whole numbers are multiplied in fp32.
__device__ __forceinline__ float power_of(float s) {
  const uint32_t e = as_u32(s) & 0x7f800000u;
  return e == 0 || e == 0x7f800000u ? 1.f : as_f32(e);
}
__device__ __forceinline__ float rest_of(float s) {
  const uint32_t e = as_u32(s) & 0x7f800000u;
  return e == 0 || e == 0x7f800000u ? s : as_f32((as_u32(s) & 0x807fffffu) | 0x3f800000u);
}

template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (__is_same(T, bf16_t)) return pack2_bf16(a, b);
  else return pack2_f16(a, b);
}

template <class Code, typename T> struct Numbers;
template <typename T> struct Numbers<E4m3, T> {
  template <bool HI> static __device__ __forceinline__ uint32_t two(uint32_t c, float s) {
    if constexpr (__is_same(T, bf16_t)) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, HI));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, s, HI));
  }
  static __device__ __forceinline__ u32x4 scaled(u32x2 c, float s0, float s1) {
    return u32x4{two<false>(c[0], s0), two<true>(c[0], s0), two<false>(c[1], s1), two<true>(c[1], s1)};
  }
  static __device__ __forceinline__ u32x4 plain(u32x2 c) { return scaled(c, 1.f, 1.f); }
  // all eight times one scale: one that takes() says, fast; or any, rounded to T
  static __device__ __forceinline__ bool takes(float s) { return power_of(s) == s; }
  static __device__ __forceinline__ u32x4 fast(u32x2 c, float s) { return scaled(c, s, s); }
  static __device__ __forceinline__ u32x4 rounded(u32x2 c, float s) {
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float x[4];
      E4m3::unpack(c[i], x);
      out[2 * i] = pack2<T>(x[0] * s, x[1] * s);
      out[2 * i + 1] = pack2<T>(x[2] * s, x[3] * s);
    }
    return out;
  }
};
template <typename T> struct Numbers<Int8, T> {
  static __device__ __forceinline__ u32x4 scaled(u32x2 c, float s0, float s1) {
    float x[4], y[4];
    Int8::unpack(c[0], x);
    Int8::unpack(c[1], y);
    return u32x4{pack2<T>(x[0] * s0, x[1] * s0), pack2<T>(x[2] * s0, x[3] * s0), pack2<T>(y[0] * s1, y[1] * s1), pack2<T>(y[2] * s1, y[3] * s1)};
  }
  static __device__ __forceinline__ u32x4 rounded(u32x2 c, float s) { return scaled(c, s, s); }
  // fp16: bytes without their sign, 128 more each, as the last bits of 1024 + them; less 1152, and times a power of two, in one instruction for two
  static __device__ __forceinline__ u32x4 in_halves(u32x2 c, float s) {
    const f16x2 f = {(_Float16)s, (_Float16)s}, off = {(_Float16)(-1152.f * s), (_Float16)(-1152.f * s)};
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = __builtin_amdgcn_perm(0x64646464u, c[i / 2] ^ 0x80808080u, i & 1 ? 0x04030402u : 0x04010400u);
      out[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, w), f, off));
    }
    return out;
  }
  static __device__ __forceinline__ u32x4 plain(u32x2 c) {
    if constexpr (__is_same(T, bf16_t)) return scaled(c, 1.f, 1.f);
    else return in_halves(c, 1.f);
  }
  // powers of two that fp16 holds, and 1152 times which
  static __device__ __forceinline__ bool takes(float s) { return __is_same(T, f16_t) && power_of(s) == s && s >= 0x1p-24f && s <= 0x1p5f; }
  static __device__ __forceinline__ u32x4 fast(u32x2 c, float s) { return in_halves(c, s); }
};

}  // namespace fs
