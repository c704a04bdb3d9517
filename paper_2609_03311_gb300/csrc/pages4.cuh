// pages4.cuh -- rows of the paged cache in 4 bits: 32 elements of a head that follow one another (a group) share a scale s and
// are held as whole numbers c from -7 to 7, an element as c s.
//
// A scale is a byte, five bits of exponent above three of mantissa: the upper bits of the fp16 number, so bits << 7 is that
// number.  Its four bits and the three of |c| make seven: c s is exact in fp16 and in bf16, and products of the tensor cores
// take the very values that are held.  Finer scales would hold the rows better by at most the 6 % that rounding a scale up
// costs on the mean, and round every value on its way to a product.
//
// s is the smallest scale that is at least max |x| / 7, at most SCALE_MAX; then |x - c s| <= s / 2 up to 7 SCALE_MAX = 64512.
//
// A page of a kv head lies in one piece: its rows' codes, then their scales.  Codes are c + 8, in 32-bit words of eight: element
// 2 i of the eight at bits 4 i, element 2 i + 1 at 16 + 4 i, so that a mask over a word takes out a pair of elements that follow
// one another, each in its half of the word.
#pragma once

#include <type_traits>

#include "device_common.cuh"

namespace dopr {
namespace pages4 {

constexpr int GROUP = 32;
constexpr uint32_t SCALE_LAST = 0xe1;      // the largest scale's byte; those above stand for NaN
constexpr float SCALE_MAX = 9216.f;
constexpr uint32_t SCALE_NAN = 0xff;
constexpr float HELD_MAX = 65504.f;        // rows above are refused, as by the library's other fp16 stores

template <int D>
constexpr int CODE_BYTES = D / 2;          // of a row
template <int D>
constexpr int SCALE_BYTES = D / GROUP;
__host__ __device__ inline int64_t page_bytes(int page, int head_dim) { return static_cast<int64_t>(page) * (head_dim / 2 + head_dim / GROUP); }

// The scale of a group with the largest magnitude `most`: its byte.  `inverse`: what elements are multiplied by, a little more
// than 1 / s: an element half way between two codes goes to the larger one, and no other crosses a border by it (x / s, x of 11
// bits and s of 4, is half way or at least 2^-13 off; the factor is 2^-20 off, give or take 2^-22).
__device__ __forceinline__ uint32_t scale_byte(float most, float& inverse) {
  // s = t steps, steps of three bits of mantissa, of 2^-17 at the low end: the smallest whole t with 7 t >= most / step.  The product
  // with 1 / 7 is off by less than 2^-18, so its ceiling less that is t or one below.
  const float want = __fmul_rn(most, 1.f / 7.f);
  const int e = max(static_cast<int>(__float_as_uint(want) >> 23) - 127 - 3, -17);
  const float step = __uint_as_float(static_cast<uint32_t>(e + 127) << 23), per = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  float t = fmaxf(ceilf(__fmaf_rn(want, per, -0x1p-18f)), 0.f);
  if (__fmul_rn(7.f, t) < __fmul_rn(most, per)) t += 1.f;
  const float s = fminf(t * step, SCALE_MAX);
  if (!(most <= HELD_MAX)) {  // a NaN, an infinity, too large
    inverse = 0.f;
    return SCALE_NAN;
  }
  inverse = s > 0.f ? __fmul_rn(__fdividef(1.f, s), 1.f + 0x1p-20f) : 0.f;
  return static_cast<uint32_t>(__half_as_ushort(__float2half_rn(s))) >> 7;
}
// The word of eight elements.  The fused product with 2^23 + 2^22 + 8 is rounded to a whole number, c + 8 in its low bits; what stands
// above them is zero in the lower 16 bits, where sums of four with 1, 16, 256, 4096 put the codes in order.
__device__ __forceinline__ uint32_t codes_of(const float* x, float inverse) {
  uint32_t n[8], half[2];
#pragma unroll
  for (int j = 0; j < 8; ++j) n[j] = __float_as_uint(__fmaf_rn(x[j], inverse, 12582912.f + 8.f));
#pragma unroll
  for (int j = 0; j < 2; ++j) half[j] = n[j] + 16 * n[2 + j] + 256 * n[4 + j] + 4096 * n[6 + j];
  return __byte_perm(half[0], half[1], 0x5410);
}

// Codes to the products' type T, in units of 1 / UNIT.  fp16: a nibble n put into the mantissa of a power of two is the number 2^p + n;
// less 2^p + 8 and times s it is c s, which a fused step gives exactly: 2^p + 8 times s fits the type where p is chosen so.  Such a
// product with a large scale leaves the range, so values come as 1 / 64 of what they are: s / 64 and all of its products are
// multiples of 2^-23.
template <typename T>
struct Widen;
template <>
struct Widen<__half> {
  static constexpr float UNIT = 64.f;
  __half2 s, from256, from16;
  // bytes: the scale of the words' lower halves in bits 0 .. 7, of the upper in 16 .. 23
  __device__ __forceinline__ explicit Widen(uint32_t bytes) {
    const uint32_t h = bytes << 7;
    s = __hmul2(reinterpret_cast<const __half2&>(h), __float2half2_rn(1.f / UNIT));
    from256 = __hmul2(s, __float2half2_rn(-264.f));
    from16 = __hmul2(s, __float2half2_rn(-24.f));
  }
  static __device__ __forceinline__ __half2 put(uint32_t w, uint32_t mask, uint32_t power) {
    const uint32_t x = (w & mask) | power;
    return reinterpret_cast<const __half2&>(x);
  }
  // v[k]: the pair of nibbles at 4 k and 16 + 4 k
  __device__ __forceinline__ void operator()(uint32_t w, uint32_t (&v)[4]) const {
    const uint32_t a = w << 2, b = w >> 6;  // nibbles at bits 2 and 6: beside powers 256 and 16
    const __half2 r[4] = {__hfma2(put(a, 0x003c003cu, 0x5c005c00u), s, from256), __hfma2(put(a, 0x03c003c0u, 0x4c004c00u), s, from16),
                          __hfma2(put(b, 0x003c003cu, 0x5c005c00u), s, from256), __hfma2(put(b, 0x03c003c0u, 0x4c004c00u), s, from16)};
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = reinterpret_cast<const uint32_t&>(r[k]);
  }
};
// bf16's lowest numbers lie on steps of 2^-133 up to bit 7, where the exponent begins: nibbles at bits 0 and 4 are such numbers as they
// stand, and 2^127 is as far from there as a factor has to be for values of 2^-22 of what they are (four shifts a word, one to
// each pair, below a power of two as fp16's: 2,048 rows on 16,384 keys 418 us, so 411).
template <>
struct Widen<__nv_bfloat16> {
  static constexpr float UNIT = 0x1p22f;
  __nv_bfloat162 low, high, from;
  __device__ __forceinline__ explicit Widen(uint32_t bytes) {
    // the byte's exponent is 112 below; s 2^111 for n 2^-133, s 2^107 for 16 n 2^-133
    const uint32_t h = bytes << 4, up = 0x77807780u, to_low = 0x77007700u, to_high = 0x75007500u, to_from = 0xb600b600u;
    const __nv_bfloat162 s = __hmul2(reinterpret_cast<const __nv_bfloat162&>(h), reinterpret_cast<const __nv_bfloat162&>(up));
    low = __hmul2(s, reinterpret_cast<const __nv_bfloat162&>(to_low));
    high = __hmul2(s, reinterpret_cast<const __nv_bfloat162&>(to_high));
    from = __hmul2(s, reinterpret_cast<const __nv_bfloat162&>(to_from));
  }
  __device__ __forceinline__ void operator()(uint32_t w, uint32_t (&v)[4]) const {
    const uint32_t x[4] = {w & 0x000f000fu, w & 0x00f000f0u, w >> 8 & 0x000f000fu, w >> 8 & 0x00f000f0u};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __nv_bfloat162 r = __hfma2(reinterpret_cast<const __nv_bfloat162&>(x[k]), k & 1 ? high : low, from);
      v[k] = reinterpret_cast<const uint32_t&>(r);
    }
  }
};

}  // namespace pages4
}  // namespace dopr
