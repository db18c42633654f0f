// Device-side arithmetic of the microscaled 4-bit floating-point format
// (include/uq.h, "Microscaled 4-bit floating point"): blocks of 32 elements
// with one scale byte, elements of one sign bit above a 3-bit code for the
// magnitudes 0, 1, 2, 3, 4, 6, 8 and 12 in half units of the block's scale.
#pragma once

#include "uq_device.hpp"

namespace uq {

constexpr int kMxBlock = 32;         // elements that share a scale byte
constexpr int kMxBlockBytes = 16;    // their codes
constexpr uint32_t kMxNaN = 255;     // the scale byte of a block holding a NaN or an infinity

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Matrix element types as template arguments (the values of enum uq_type).
constexpr int kF32 = 0, kBF16 = 1, kF16 = 2;
template <int T> constexpr int kElemBytes = T == kF32 ? 4 : 2;

// Flat unit -> (row, unit in row) by one high multiply: for units per row
// n >= 1 and u < 2^31, u / n = (u * mul) >> (32 + shift) with
// shift = ceil(log2 n) - 1 and mul = ceil(2^(32 + shift) / n) < 2^32 (the
// round-up method of Granlund and Montgomery, "Division by invariant integers
// using multiplication", PLDI'94: mul * n exceeds 2^(32 + shift) by less than
// n <= 2^(shift + 1), so the quotient is exact for u < 2^31).  n = 1 is
// passed through.
struct RowDiv {
    uint32_t n, mul, shift;
};

inline RowDiv row_div(uint32_t n)
{
    RowDiv r;
    r.n = n;
    r.mul = 0;
    r.shift = 0;
    if (n > 1) {
        uint32_t lg = 0;
        while ((uint64_t(1) << lg) < n)
            ++lg;
        r.shift = lg - 1;
        r.mul = static_cast<uint32_t>(((uint64_t(1) << (32 + r.shift)) + n - 1) / n);
    }
    return r;
}

__device__ __forceinline__ uint32_t div_row(uint32_t u, const RowDiv& d)
{
    return d.n == 1 ? u : __umulhi(u, d.mul) >> d.shift;
}

// The scale byte of a block from the bits of its largest |x| as binary32
// (NaNs order above infinity): the least e >= -126 with max <= 6 * 2^e, plus
// 127.  With max = 1.f * 2^E, 6 * 2^e = 1.5 * 2^(e + 2), so e is E - 2, and
// one more when the fraction exceeds .5 (0x400000): an add that carries then.
__device__ __forceinline__ uint32_t mx4_byte(uint32_t top)
{
    const uint32_t t = (top + 0x3FFFFFu) >> 23;
    return top >= 0x7F800000u ? kMxNaN : (t > 3u ? t : 3u) - 2u;
}

// 2^(1 - e) for a byte of 1 .. 254 (a binary32 normal number): |x| times it is
// |x| in half units.  0 for the NaN byte; a byte of 0, which the rule above
// never forms, is read as 1.
__device__ __forceinline__ float mx4_half_units(uint32_t byte)
{
    return byte == kMxNaN ? 0.0f : __uint_as_float((255u - (byte > 1u ? byte : 1u)) << 23);
}

// Largest over the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t v)
{
    const uint32_t a = __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, true);  // lanes 1 0 3 2
    v = v > a ? v : a;
    const uint32_t b = __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, true);  // lanes 2 3 0 1
    return v > b ? v : b;
}

__device__ __forceinline__ uint32_t max3_u32(uint32_t a, uint32_t b, uint32_t c)
{
    const uint32_t m = a > b ? a : b;
    return m > c ? m : c;
}

// Bits of the largest |x| of eight.
__device__ __forceinline__ uint32_t octet_max(const float (&x)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; j += 2)
        m = max3_u32(m, __float_as_uint(x[j]) & 0x7FFFFFFFu, __float_as_uint(x[j + 1]) & 0x7FFFFFFFu);
    return m;
}

// Eight 4-bit fields to the nearest code, ties to the even one: the
// converter divides by the scale's power of two exactly and rounds once
// (checked against that rule for every 16-bit value and around every
// boundary in binary32).  byte is 1 .. 253.
__device__ __forceinline__ uint32_t mx4_nearest(const float (&x)[8], uint32_t byte)
{
    const float s = __uint_as_float(byte << 23);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
    return r;
}

// Stochastic code of one element from the whole of its uniform word r: with
// y = |x| in half units (exact: a power of two times x; results below 2^-126
// round far below any threshold), at most 12 (beyond it only on a byte that
// was not formed from x), and the grid's step at y, l = floor(y / step),
// t = floor((y / step - l) * 2^32), the code is that of l, or the next one when
// r < t.  step = 2^max(floor(log2 y) - 1, 0), which adds 2 to the code each
// time it doubles.
__device__ __forceinline__ uint32_t mx4_exact(float x, float to_half, uint32_t r)
{
    const float y = fminf(fabsf(x) * to_half, 12.0f);
    uint32_t sb = __float_as_uint(y) & 0x7F800000u;
    sb = sb > 0x40000000u ? sb : 0x40000000u;
    const float q = y * __uint_as_float(0x7F800000u - sb);  // y / step, at most 4
    const float l = floorf(q);
    const uint32_t t = static_cast<uint32_t>((q - l) * 4294967296.0f);
    return static_cast<uint32_t>(l) + (sb >> 22) - 256u + (r < t ? 1u : 0u);
}

// |code| in half units.
__device__ __forceinline__ int32_t mx4_half_value(uint32_t code)
{
    return code < 2u ? static_cast<int32_t>(code) : static_cast<int32_t>((2u | (code & 1u)) << ((code >> 1) - 1u));
}

// Half h of a Philox block's words (uq.h: bits 16*(h / 4) .. +15 of word h mod 4).
__device__ __forceinline__ uint32_t philox_half(const uint4& w, int h)
{
    const uint32_t v = (h & 3) == 0 ? w.x : (h & 3) == 1 ? w.y : (h & 3) == 2 ? w.z : w.w;
    return h < 4 ? v & 0xFFFFu : v >> 16;
}

}  // namespace uq
