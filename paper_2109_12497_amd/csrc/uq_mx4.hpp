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

// The largest of |a|, |b| and |c| in one instruction; a NaN if one is.
__device__ __forceinline__ float max3_abs(float a, float b, float c)
{
    float r;
    __asm__("v_maximum3_f32 %0, |%1|, |%2|, |%3|" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Bits of the largest |x| of eight, and of `most`; at or above 0x7F800000 if
// one of them is a NaN or an infinity.
__device__ __forceinline__ uint32_t octet_max(const float (&x)[8], uint32_t most = 0)
{
    float m = max3_abs(__uint_as_float(most), x[0], x[1]);
    m = max3_abs(m, x[2], x[3]);
    m = max3_abs(m, x[4], x[5]);
    return __float_as_uint(max3_abs(m, x[6], x[7]));
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

// The stochastic code of one element from the high half of its uniform word,
// without the division into steps: with y = |x| in half units, m = y + max(y, 2)
// is the code's place in binary32, for its bits 22 and up are 256 plus the code
// (y < 2: 2 + y has the codes 0 and 1 a half apart; beyond, 2 y keeps one bit
// below the leading one) and the 22 bits below are the fraction.  m is formed
// in x's own units, |x| + max(|x|, 2^e), and the power of two between them
// added to its exponent.  Adding the complement of the high half on the
// fraction's upper 16 bits carries into the code exactly when the half is
// below them.  What is returned is the sum shifted up by two: the code is its
// top byte.  The sum's fraction tells where that decided wrongly
// (mx4_undecided): the halves were equal, or m, which rounds where y < 2,
// carried into the fraction's upper 16 bits.  From byte kMxTop on m may pass
// the largest binary32; those blocks are decided by whole words alone.
constexpr uint32_t kMxTop = 252;
struct Mx4Place {
    float least;      // 2^e
    uint32_t to_half; // what to add to m's bits, shifted by two as they are
};
__device__ __forceinline__ Mx4Place mx4_places(uint32_t byte)
{
    return {__uint_as_float(byte << 23), (128u - byte) << 25};
}
// `halves`: a word of the complement; HALF picks the 16 bits.  x as it is: at
// most 6 * 2^e.
template <int HALF>
__device__ __forceinline__ uint32_t mx4_carry(float x, Mx4Place p, uint32_t halves)
{
    // One instruction each: fmaxf would first make x canonical, and the
    // compiler takes the sum with a shifted byte apart.
    float m;
    uint32_t place, r;
    __asm__("v_max_f32 %0, |%1|, %2" : "=v"(m) : "v"(x), "v"(p.least));
    m += fabsf(x);
    __asm__("v_lshl_add_u32 %0, %1, 2, %2" : "=v"(place) : "v"(m), "v"(p.to_half));
    if constexpr (HALF == 0)
        __asm__("v_mad_u32_u16 %0, %1, %2, %3" : "=v"(r) : "v"(halves), "s"(256), "v"(place));
    else
        __asm__("v_mad_u32_u16 %0, %1, %2, %3 op_sel:[1,0,0,0]" : "=v"(r) : "v"(halves), "s"(256), "v"(place));
    return r;
}
// Below kUndecided where the fraction of a sum lies within 64 of a carry.
constexpr uint32_t kUndecided = 128u << 10;
__device__ __forceinline__ uint32_t mx4_undecided(uint32_t sum)
{
    return (sum + 256u) << 8;
}

// The top bytes of four words.
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_amdgcn_perm(b, a, 0x0C0C0703u) | __builtin_amdgcn_perm(d, c, 0x07030C0Cu);
}

// Fields from eight sums (codes in their top bytes) and the elements' signs.
__device__ __forceinline__ uint32_t mx4_pack(const uint32_t (&sum)[8], const float (&x)[8])
{
    const auto bits = [&](int j) { return __float_as_uint(x[j]); };
    const uint32_t even = top_bytes(sum[0], sum[2], sum[4], sum[6]), odd = top_bytes(sum[1], sum[3], sum[5], sum[7]);
    const uint32_t se = top_bytes(bits(0), bits(2), bits(4), bits(6)), so = top_bytes(bits(1), bits(3), bits(5), bits(7));
    return (even | odd << 4) | ((se >> 4) & 0x08080808u) | (so & 0x80808080u);
}

// Sums over rows of eight signed codes in half units, biased by 12 a row and
// held as bytes (even and odd elements apart): at most 24 a row, so up to
// kMxByteRows rows.  A byte permutation looks a code's value up for four
// elements at a time, in one table for each sign.
constexpr int kMxByteRows = 8;
struct Mx4Bytes {
    uint32_t even = 0, odd = 0;

    __device__ __forceinline__ void add(const uint32_t (&sum)[8], const float (&x)[8])
    {
        const auto bits = [&](int j) { return __float_as_uint(x[j]); };
        even += values(top_bytes(sum[0], sum[2], sum[4], sum[6]), signs(bits(0), bits(2), bits(4), bits(6)));
        odd += values(top_bytes(sum[1], sum[3], sum[5], sum[7]), signs(bits(1), bits(3), bits(5), bits(7)));
    }
    // The sum of element j over `rows` rows.
    __device__ __forceinline__ int32_t total(int j, int rows) const
    {
        const uint32_t w = j & 1 ? odd : even;
        return static_cast<int32_t>((w >> (8 * (j >> 1))) & 0xFFu) - 12 * rows;
    }

  private:
    // 0xFF in the byte of a word whose top bit is set
    static __device__ __forceinline__ uint32_t signs(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
    {
        return __builtin_amdgcn_perm(b, a, 0x0C0C0B09u) | __builtin_amdgcn_perm(d, c, 0x0B090C0Cu);
    }
    static __device__ __forceinline__ uint32_t values(uint32_t codes, uint32_t negative)
    {
        const uint32_t plus = __builtin_amdgcn_perm(0x18141210u, 0x0F0E0D0Cu, codes);   // 24 20 18 16 15 14 13 12
        const uint32_t minus = __builtin_amdgcn_perm(0x00040608u, 0x090A0B0Cu, codes);  // 0 4 6 8 9 10 11 12
        return (plus & ~negative) | (minus & negative);
    }
};

// Half h of a Philox block's words (uq.h: bits 16*(h / 4) .. +15 of word h mod 4).
__device__ __forceinline__ uint32_t philox_half(const uint4& w, int h)
{
    const uint32_t v = (h & 3) == 0 ? w.x : (h & 3) == 1 ? w.y : (h & 3) == 2 ? w.z : w.w;
    return h < 4 ? v & 0xFFFFu : v >> 16;
}

}  // namespace uq
