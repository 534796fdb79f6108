// The 4-bit cache: blocks of 32 coordinates of a row, each coordinate a code of
// one sign, two exponent and one mantissa bit (0, 0.5, 1, 1.5, 2, 3, 4, 6), and
// one byte e + 127 a block; a value is code 2^e.  Coordinate i of a row is in byte
// i / 2, even ones in its low half.  gfx950 turns two codes into bf16 or fp32
// values, times the power of two, in one instruction, and every value is exact
// in either (two significant bits).
#pragma once

#include "device_common.h"

namespace bkv {
namespace mx {

constexpr int kBlock = 32;
// e + 127: subnormal coordinates fall below half of the smallest code, and the
// largest code stays finite.
constexpr int kLeast = 3, kMost = 252;
// The byte of a block that held an infinity or a NaN: the conversions make NaNs of
// all of its codes.  There is no code for either, and a number in their place
// would hide them.
constexpr unsigned kNan = 255;

template <int D>
struct Row {
    static constexpr int kCodes = D / 2;        // bytes
    static constexpr int kScales = D / kBlock;  // bytes
};

// Where a unit's keys or values lie, from one of its rows on.
struct Src {
    const uint8_t* c;  // codes
    const uint8_t* s;  // bytes
};
template <int D>
__device__ __forceinline__ Src rows(const void* codes, const uint8_t* bytes, long long row) {
    return {static_cast<const uint8_t*>(codes) + row * Row<D>::kCodes, bytes + row * Row<D>::kScales};
}

// Whether a cache has all of its arrays, aligned.
inline bool whole(const bkv_mx_cache& c) {
    const uintptr_t all[] = {(uintptr_t)c.K, (uintptr_t)c.KS, (uintptr_t)c.V, (uintptr_t)c.VS};
    for (uintptr_t p : all)
        if (!p || (p & 15u)) return false;
    return true;
}

// 2^e of a block's byte.
__device__ __forceinline__ float scale(unsigned byte) { return __uint_as_float(byte << 23); }

// The byte of a block whose largest magnitude has the bits `top`: the smallest e
// with top <= 7 2^e.  7 rounds to 6, no worse than the half step between 4 and 6,
// and from there on the next power is the closer one.  Magnitudes are ordered as
// their bits are, infinities and then NaNs last.
__device__ __forceinline__ unsigned scale_byte(unsigned top) {
    const int e = (int)((top + 0x1fffffu) >> 23) - 2;
    return top >= 0x7f800000u ? kNan : (unsigned)min(max(e, kLeast), kMost);
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Values of byte B of `codes`: two bf16 in a word, or two floats.
template <int B>
__device__ __forceinline__ unsigned pair_bf16(unsigned codes, float scale) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}
template <int B>
__device__ __forceinline__ f32x2 pair_f32(unsigned codes, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, B);
}
// All eight of a word.
__device__ __forceinline__ dev::u32x4 eight_bf16(unsigned codes, float scale) {
    return dev::u32x4{pair_bf16<0>(codes, scale), pair_bf16<1>(codes, scale), pair_bf16<2>(codes, scale),
                      pair_bf16<3>(codes, scale)};
}

// The high halves of two floats, and what they leave of them: three cuts take all
// of their 24 bits, as bf16 terms.
__device__ __forceinline__ unsigned cut(float& x, float& y) {
    const unsigned w = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
    x -= __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    y -= __uint_as_float(__float_as_uint(y) & 0xffff0000u);
    return w;
}

}  // namespace mx
}  // namespace bkv
