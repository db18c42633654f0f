// Microscaled 4-bit floating point: quantisation, reading back and the
// aggregation step on that format (include/uq.h).
#include "uq_launch.hpp"
#include "uq_mx4.hpp"

namespace uq {
namespace {

// Eight elements as they lie in memory.
template <int T>
struct Octet {
    u32x4 part[T == kF32 ? 2 : 1];
};

// A whole octet in 16-byte pieces.
template <int T, bool NT = false>
__device__ __forceinline__ Octet<T> read_octet(const void* at)
{
    Octet<T> o;
#pragma unroll
    for (int i = 0; i < (T == kF32 ? 2 : 1); ++i)
        o.part[i] = NT ? load_nt(static_cast<const uint32_t*>(at) + 4 * i) : static_cast<const u32x4*>(at)[i];
    return o;
}

// The `left` first elements of an octet one by one, zeros past them.
template <int T>
__device__ __forceinline__ Octet<T> read_ragged(const void* at, int64_t left)
{
    Octet<T> o;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t e = 0;
        if constexpr (T == kF32) {
            if (j < left)
                e = static_cast<const uint32_t*>(at)[j];
            o.part[j / 4][j % 4] = e;
        } else {
            if (j < left)
                e = static_cast<const uint16_t*>(at)[j];
            o.part[0][j / 2] = j % 2 ? o.part[0][j / 2] | e << 16 : e;
        }
    }
    return o;
}

template <int T, bool NT = false>
__device__ __forceinline__ Octet<T> read_some(const void* at, int64_t left)
{
    return left >= 8 ? read_octet<T, NT>(at) : read_ragged<T>(at, left);
}

template <int T>
__device__ __forceinline__ void unpack_octet(const Octet<T>& o, float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (T == kF32) {
            x[j] = __uint_as_float(o.part[j / 4][j % 4]);
        } else {
            const uint32_t pair = o.part[0][j / 2];
            if constexpr (T == kBF16)
                x[j] = __uint_as_float(j % 2 ? pair & 0xFFFF0000u : pair << 16);
            else
                x[j] = static_cast<float>(__builtin_bit_cast(f16x2, pair)[j % 2]);
        }
    }
}

// Elements col .. col + 7 of one row as binary32 (zeros past cols; rows start
// on 16-byte boundaries and nothing past cols is read).
template <int T, bool NT = false>
__device__ __forceinline__ void load_octet(const void* row, int64_t col, int64_t cols, float (&x)[8])
{
    unpack_octet<T>(read_some<T, NT>(static_cast<const char*>(row) + col * kElemBytes<T>, cols - col), x);
}

// Eight stochastic codes of row `row`, octet `oct`, in the top bytes of sum,
// from the complement of the block of their words' high halves; the low
// halves' block is formed only where the high ones leave one of the eight
// undecided (once in 4096).
__device__ __forceinline__ void mx4_codes(const float (&x)[8], uint32_t byte, const uint4& halves, uint64_t oct,
                                          uint32_t row, uint64_t seed, uint32_t (&sum)[8])
{
    const Mx4Place place = mx4_places(byte);
    const uint32_t w[4] = {halves.x, halves.y, halves.z, halves.w};
    uint32_t least = ~0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        sum[j] = mx4_carry<0>(x[j], place, w[j]);
        sum[4 + j] = mx4_carry<1>(x[4 + j], place, w[j]);
        const uint32_t a = mx4_undecided(sum[j]), b = mx4_undecided(sum[4 + j]);
        const uint32_t c = a < b ? a : b;
        least = least < c ? least : c;
    }
    if (least < kUndecided || byte >= kMxTop) {
        const uint4 lo = philox4x32_10(static_cast<uint32_t>(oct), static_cast<uint32_t>(oct >> 32), row, 1,
                                       static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t hi = ~(j < 4 ? w[j & 3] << 16 : w[j & 3]) & 0xFFFF0000u;
            sum[j] = mx4_exact(x[j], mx4_half_units(byte), hi | philox_half(lo, j)) << 24;
        }
    }
}

// The same as eight fields.
__device__ __forceinline__ uint32_t mx4_stochastic(const float (&x)[8], uint32_t byte, const uint4& halves,
                                                   uint32_t oct, uint32_t row, uint64_t seed)
{
    uint32_t sum[8];
    mx4_codes(x, byte, halves, oct, row, seed, sum);
    return mx4_pack(sum, x);
}

// The start of row `row`: strides are multiples of 16 bytes, and in those
// units one 32 x 32 -> 64 bit product forms the offset.
__device__ __forceinline__ int64_t row_start(uint32_t row, uint32_t stride16)
{
    return static_cast<int64_t>((static_cast<uint64_t>(row) * stride16) << 4);
}

// Codes along the rows: one thread per octet, the four threads of a block's
// octets share its maximum.  A unit of the grid is an octet of the padded rows.
template <int T, bool SR>
__global__ __launch_bounds__(kBlock) void k_mx4_rows(const void* x, int64_t cols, uint32_t ldx16, uint64_t seed,
                                                     uint8_t* codes, uint32_t ldc16, uint8_t* scales, uint32_t lds16,
                                                     uint32_t row0, uint32_t units, RowDiv div)
{
    const uint32_t u = blockIdx.x * kBlock + threadIdx.x;
    if (u >= units)
        return;
    const uint32_t in = div_row(u, div);
    const uint32_t oct = u - in * div.n;
    const uint32_t row = row0 + in;
    float v[8];
    load_octet<T>(static_cast<const char*>(x) + row_start(row, ldx16), int64_t(oct) * 8, cols, v);
    uint4 halves;
    if constexpr (SR) {
        const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
        halves = philox_tail_not(row_key(0, row, k0), lane_key(oct, 0, k1), k0, k1);
    }
    const uint32_t byte = mx4_byte(quad_max(octet_max(v)));
    uint32_t w;
    if constexpr (SR)
        w = mx4_stochastic(v, byte, halves, oct, row, seed);
    else
        w = mx4_nearest(v, byte);
    w = byte == kMxNaN ? 0u : w;
    *reinterpret_cast<uint32_t*>(codes + row_start(row, ldc16) + int64_t(oct) * 4) = w;
    if ((oct & 3) == 0)
        scales[row_start(row, lds16) + oct / 4] = static_cast<uint8_t>(byte);
}

// Codes of the transposed matrix, and with ROWS of the rows too, from one
// read: a block takes 128 rows by 64 columns through LDS.  A thread first
// holds octets of four rows (32 apart, the same columns, so that their Philox
// blocks share the lane's part), forms the rows' codes from them and leaves
// the elements in LDS together with the complements of their words' high
// halves; then a thread takes 32 rows of one column, a whole block.  Four
// lanes take a column's four blocks, 64 contiguous bytes of its codes.
// Columns are turned by 16 every 32 rows: those four lanes then read
// different banks.
constexpr int kTileRows = 128, kTileCols = 64;

__device__ __forceinline__ int tile_at(int row, int col)
{
    return row * kTileCols + ((col + 16 * (row >> 5)) & (kTileCols - 1));
}

// Block -> tile.  Blocks go to the eight XCDs in turn, and each XCD has its own
// L2: eight blocks that one XCD takes in a row cover 2 tiles down and 4 across,
// so that the 128-byte lines which they write in part, two blocks' codes of a
// column and four blocks' codes of a row, leave it whole (8192 x 8192 bf16
// to the nearest, both ways, one matrix each time: 37 us, 42 with the tiles of
// a column in turn).
constexpr int kSuperDown = 2, kSuperAcross = 4, kSuper = kSuperDown * kSuperAcross, kXcds = 8;

__host__ __device__ __forceinline__ int64_t super_blocks(int64_t down, int64_t across)
{
    const int64_t all = ((down + kSuperDown - 1) / kSuperDown) * ((across + kSuperAcross - 1) / kSuperAcross);
    return (all + kXcds - 1) / kXcds * kXcds * kSuper;
}
__device__ __forceinline__ bool place_tile(int64_t block, int32_t down, int32_t across, int64_t* tr, int64_t* tc)
{
    const int64_t turn = block / kXcds, super = turn / kSuper * kXcds + block % kXcds;
    const int in = static_cast<int>(turn % kSuper), per_row = (across + kSuperAcross - 1) / kSuperAcross;
    const int64_t row = super / per_row;
    *tr = row * kSuperDown + in / kSuperAcross;
    *tc = (super - row * per_row) * kSuperAcross + in % kSuperAcross;
    return *tr < down && *tc < across;
}

template <int T, bool SR, bool ROWS>
__global__ __launch_bounds__(kBlock) void k_mx4_tiles(const void* x, int64_t rows, int64_t cols, int64_t ldx,
                                                      uint64_t seed, uint8_t* codes, int64_t ldc, uint8_t* scales,
                                                      int64_t lds, uint8_t* codes_t, int64_t ldct, uint8_t* scales_t,
                                                      int64_t ldst, int64_t first, int32_t down, int32_t across)
{
    // 16-bit types: half | element << 16; binary32: the halves apart
    __shared__ __attribute__((aligned(16))) uint32_t elems[kTileRows * kTileCols];
    __shared__ __attribute__((aligned(16))) uint16_t apart[T == kF32 && SR ? kTileRows * kTileCols : 1];
    int64_t tr, tc;
    if (!place_tile(first + blockIdx.x, down, across, &tr, &tc))
        return;
    const int64_t row0 = tr * kTileRows, col0 = tc * kTileCols;
    const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    {
        const int oc = threadIdx.x & 7, r0 = threadIdx.x >> 3;
        const uint32_t oct = static_cast<uint32_t>(col0 / 8) + oc;
        const int64_t row1 = row0 + r0;
        const char* at = static_cast<const char*>(x) + (row1 * ldx + col0 + oc * 8) * kElemBytes<T>;
        Octet<T> raw[4];
        if (row0 + kTileRows <= rows && col0 + kTileCols <= cols) {  // the same in the whole block
#pragma unroll
            for (int i = 0; i < 4; ++i)
                raw[i] = read_octet<T>(at + i * 32 * ldx * kElemBytes<T>);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                raw[i] = read_some<T>(at + i * 32 * ldx * kElemBytes<T>, row1 + 32 * i < rows ? cols - col0 - oc * 8 : 0);
        }
        uint8_t* const code_row = ROWS ? codes + row1 * ldc + int64_t(oct) * 4 : nullptr;
        uint8_t* const scale_row = ROWS ? scales + row1 * lds + oct / 4 : nullptr;
        const bool col_ok = col0 + (oc & ~3) * 8 < cols;
        LaneKey lk;
        if constexpr (SR)
            lk = lane_key(oct, 0, k1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + 32 * i;
            const uint32_t row = static_cast<uint32_t>(row0 + r);
            float v[8];
            unpack_octet<T>(raw[i], v);
            uint4 halves = make_uint4(0, 0, 0, 0);
            if constexpr (SR)
                halves = philox_tail_not(row_key(0, row, k0), lk, k0, k1);
            if constexpr (ROWS) {
                const uint32_t byte = mx4_byte(quad_max(octet_max(v)));
                uint32_t w;
                if constexpr (SR)
                    w = mx4_stochastic(v, byte, halves, oct, row, seed);
                else
                    w = mx4_nearest(v, byte);
                if (col_ok && row1 + 32 * i < rows) {
                    *reinterpret_cast<uint32_t*>(code_row + i * 32 * ldc) = byte == kMxNaN ? 0u : w;
                    if ((oct & 3) == 0)
                        scale_row[i * 32 * lds] = static_cast<uint8_t>(byte);
                }
            }
            const uint32_t h[4] = {halves.x, halves.y, halves.z, halves.w};
            const int to = tile_at(r, oc * 8);
            uint32_t d[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t e = __float_as_uint(v[j]);
                if constexpr (T == kF16) {
                    const _Float16 f = static_cast<_Float16>(v[j]);
                    e = static_cast<uint32_t>(__builtin_bit_cast(uint16_t, f)) << 16;
                }
                if constexpr (T != kF32 && SR)  // bytes 2, 3 of the element, 0, 1 or 2, 3 of the word
                    e = __builtin_amdgcn_perm(e, h[j & 3], j < 4 ? 0x07060100u : 0x07060302u);
                d[j] = e;
            }
            *reinterpret_cast<u32x4*>(elems + to) = u32x4{d[0], d[1], d[2], d[3]};
            *reinterpret_cast<u32x4*>(elems + to + 4) = u32x4{d[4], d[5], d[6], d[7]};
            if constexpr (T == kF32 && SR)
                *reinterpret_cast<u32x4*>(apart + to) =
                    u32x4{(h[0] & 0xFFFFu) | h[1] << 16, (h[2] & 0xFFFFu) | h[3] << 16, h[0] >> 16 | (h[1] & 0xFFFF0000u),
                          h[2] >> 16 | (h[3] & 0xFFFF0000u)};
        }
    }
    __syncthreads();
    const int q = threadIdx.x & 3, c = threadIdx.x >> 2;
    const int64_t col = col0 + c, blk = row0 / kMxBlock + q;
    if (col >= cols || blk * kMxBlock >= rows)
        return;
    const auto value = [](uint32_t d) {
        if constexpr (T == kF16) {
            const uint16_t e = static_cast<uint16_t>(d >> 16);
            return static_cast<float>(__builtin_bit_cast(_Float16, e));
        } else {
            return __uint_as_float(T == kF32 || !SR ? d : d & 0xFFFF0000u);
        }
    };
    uint32_t d[4][8], top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            d[i][j] = elems[tile_at(32 * q + 8 * i + j, c)];
            // bf16: the largest has the largest upper half, whatever lies below
            v[j] = T == kF16 ? value(d[i][j]) : __uint_as_float(d[i][j]);
        }
        top = octet_max(v, top);
    }
    if constexpr (T == kBF16 && SR)
        top &= 0xFFFF0000u;
    const uint32_t byte = mx4_byte(top);
    scales_t[col * ldst + blk] = static_cast<uint8_t>(byte);
    const Mx4Place place = mx4_places(byte);
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = value(d[i][j]);
        if constexpr (SR) {
            uint32_t sum[8], least = ~0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum[j] = mx4_carry<0>(v[j], place, T == kF32 ? apart[tile_at(32 * q + 8 * i + j, c)] : d[i][j]);
                const uint32_t a = mx4_undecided(sum[j]);
                least = least < a ? least : a;
            }
            w[i] = mx4_pack(sum, v);
            if (least < kUndecided || byte >= kMxTop) {
#pragma unroll 1
                for (int j = 0; j < 8; ++j) {  // each element has a block of low halves of its own
                    const int r = 32 * q + 8 * i + j, at = tile_at(r, c);
                    const uint32_t e = elems[at], half = T == kF32 ? apart[at] : e;
                    if (byte < kMxTop && mx4_undecided(mx4_carry<0>(value(e), place, half)) >= kUndecided)
                        continue;  // (all eight formed: 5% more time at 8192 x 8192)
                    const uint4 lo = philox4x32_10(static_cast<uint32_t>(col >> 3), 0, static_cast<uint32_t>(row0) + r,
                                                   1, k0, k1);
                    const uint32_t hi = ~half << 16;
                    const uint32_t code = mx4_exact(value(e), mx4_half_units(byte), hi | philox_half(lo, col & 7));
                    w[i] = (w[i] & ~(7u << (4 * j))) | code << (4 * j);
                }
            }
        } else {
            w[i] = mx4_nearest(v, byte);
        }
    }
    if (byte == kMxNaN)
        w = u32x4{0, 0, 0, 0};
    *reinterpret_cast<u32x4*>(codes_t + col * ldct + blk * kMxBlockBytes) = w;
}

// 16 bytes of values a thread (four in binary32, else eight): the codes of
// those and the block's byte in.  The converters decode, scale and round
// once, and give NaN for the scale byte 255.  Values leave nontemporally:
// 16384 x 8192 bf16 47.4 us, 63.6 with plain stores; 4096^2 5.9 and 7.5.
template <int T>
__global__ __launch_bounds__(kBlock) void k_mx4_read(const uint8_t* codes, uint32_t ldc16, const uint8_t* scales,
                                                     uint32_t lds16, int64_t cols, void* out, uint32_t ldo16,
                                                     uint32_t row0, uint32_t units, RowDiv div)
{
    constexpr int kEach = 16 / kElemBytes<T>;
    const uint32_t u = blockIdx.x * kBlock + threadIdx.x;
    if (u >= units)
        return;
    const uint32_t in = div_row(u, div);
    const uint32_t at = u - in * div.n;
    const uint32_t row = row0 + in;
    const int64_t col = int64_t(at) * kEach;
    const float s = __uint_as_float(static_cast<uint32_t>(scales[row_start(row, lds16) + at / (kMxBlock / kEach)]) << 23);
    const uint8_t* from = codes + row_start(row, ldc16) + int64_t(at) * (kEach / 2);
    u32x4 v;
    if constexpr (T == kF32) {
        const uint32_t w = *reinterpret_cast<const uint16_t*>(from);
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
        v = u32x4{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])};
    } else {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(from);
        if constexpr (T == kBF16) {
            v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
            v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
            v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
            v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
        } else {
            v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0));
            v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1));
            v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2));
            v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3));
        }
    }
    char* to = static_cast<char*>(out) + row_start(row, ldo16) + col * kElemBytes<T>;
    if (col + kEach <= cols) {
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(to));
        return;
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (col + j < cols) {
            if constexpr (T == kF32)
                reinterpret_cast<uint32_t*>(to)[j] = v[j];
            else
                reinterpret_cast<uint16_t*>(to)[j] = static_cast<uint16_t>(v[j / 2] >> (16 * (j % 2)));
        }
}

// Bytes shared by `rows` gradients (and, with accumulate, the bytes held):
// the rule is monotone in the maximum, so the shared byte is that of the
// largest |g| over the rows.
__global__ __launch_bounds__(kBlock) void k_mx4_shared(const float* g, int64_t d, int32_t rows, int64_t ldg,
                                                       int32_t accumulate, uint8_t* scales, int64_t oct0,
                                                       int64_t octs)
{
    const int64_t o = oct0 + int64_t(blockIdx.x) * kBlock + threadIdx.x;
    if (o >= octs)
        return;
    uint32_t top = 0;
    for (int32_t m = 0; m < rows; ++m) {
        float v[8];
        load_octet<kF32>(g + m * ldg, o * 8, d, v);
        top = octet_max(v, top);
    }
    uint32_t byte = mx4_byte(quad_max(top));
    if ((o & 3) == 0) {
        if (accumulate) {
            const uint32_t held = scales[o / 4];
            byte = byte > held ? byte : held;
        }
        scales[o / 4] = static_cast<uint8_t>(byte);
    }
}

// What the mean divides by: the workers and RN64 of their reciprocal.
struct Mx4Mean {
    double m, inv_m;
};

// sum * 2^(e - 1) / M, rounded to binary32 once (NaN for the NaN byte): the
// quotient in binary64, corrected by its remainder so that it is exact where 64
// bits hold it, then an exact power of two.  Other quotients of these integers
// are further from every midpoint of binary32 than binary64 is off (1 / (M j) of
// themselves for a midpoint of 25 bits j, above 2^-52.5 while 12 M < 2^31).  In
// binary32, with 2^(e - 1) / M as one factor, the mean was off by up to a whole step
// for M that are no powers of two, half a step more than the format costs; the
// time is that of the memory either way (ResNet-50, 8 workers: 178 us both).
__device__ __forceinline__ float mx4_mean(int32_t sum, double half, const Mx4Mean& by)
{
    const double s = sum, q = s * by.inv_m;
    return static_cast<float>(__builtin_fma(__builtin_fma(-q, by.m, s), by.inv_m, q) * half);
}
// 2^(byte - 128) for a byte of 1 and up.
__device__ __forceinline__ double mx4_half(uint32_t byte)
{
    const uint64_t bits = byte == kMxNaN ? 0x7FF8000000000000u : static_cast<uint64_t>(byte + 1023u - 128u) << 52;
    return __builtin_bit_cast(double, bits);
}

// Eight results of each lane, stored: a wave's 512 coordinates from `first` on.
// Lanes 32 apart exchange a half of theirs, so that each of the two stores
// covers 1 KiB without gaps (16 bytes a lane 32 bytes apart took twice the
// time as nontemporal stores).
template <bool NT, typename V>
__device__ __forceinline__ void store_octets(V* to, int64_t first, int64_t d, int lane, const uint32_t (&r)[8])
{
    if (first + 512 <= d) {
        u32x4 a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const u32x2 p = __builtin_amdgcn_permlane32_swap(r[j], r[4 + j], false, false);
            a[j] = p[0];  // coordinates j of octet lane, or 4 + j of octet lane - 32
            b[j] = p[1];  // coordinates j of octet lane + 32, or 4 + j of octet lane
        }
        uint32_t* o = reinterpret_cast<uint32_t*>(to) + first + (lane & 31) * 8 + (lane >> 5) * 4;
        if constexpr (NT) {
            __builtin_nontemporal_store(a, reinterpret_cast<u32x4*>(o));
            __builtin_nontemporal_store(b, reinterpret_cast<u32x4*>(o + 256));
        } else {
            reinterpret_cast<u32x4*>(o)[0] = a;
            reinterpret_cast<u32x4*>(o + 256)[0] = b;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (first + lane * 8 + j < d)
            reinterpret_cast<uint32_t*>(to)[first + lane * 8 + j] = r[j];
}

// The mean (with out) of the sums and their stores.
template <bool NT>
__device__ __forceinline__ void finish_octet(const int32_t (&total)[8], uint32_t byte, const Mx4Mean& by, int64_t first,
                                             int64_t d, int lane, int32_t* sum, float* out)
{
    uint32_t r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        r[j] = static_cast<uint32_t>(total[j]);
    store_octets<NT>(sum, first, d, lane, r);
    if (out == nullptr)
        return;
    const double half = mx4_half(byte);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        r[j] = __float_as_uint(mx4_mean(total[j], half, by));
    store_octets<NT>(out, first, d, lane, r);
}

// The whole step for up to ROWS rows: a lane holds its octet of every row in
// registers, so each gradient is read once.  A wave takes 512 coordinates.
// LOADS: gradients read nontemporally.
template <int ROWS, bool NT, bool LOADS>
__global__ __launch_bounds__(kBlock) void k_mx4_step(const float* g, int64_t d, int32_t rows, int64_t ldg,
                                                     uint64_t seed, uint8_t* scales, int32_t* sum, Mx4Mean by,
                                                     float* out, int64_t oct0, int64_t octs)
{
    const int lane = threadIdx.x & 63;
    const int64_t o = oct0 + int64_t(blockIdx.x) * kBlock + threadIdx.x;
    float v[ROWS][8];
    uint32_t top = 0;
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
        if (m < rows)
            load_octet<kF32, LOADS>(g + m * ldg, o * 8, d, v[m]);
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
        if (m < rows)
            top = octet_max(v[m], top);
    const uint32_t byte = mx4_byte(quad_max(top));
    if ((o & 3) == 0 && o < octs)
        scales[o / 4] = static_cast<uint8_t>(byte);
    const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    const LaneKey lk = lane_key(static_cast<uint32_t>(o), 0, k1);
    // the counter's high word is the same in the whole block: 2^32 is a multiple of its octets
    const uint32_t high = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(o >> 32));
    int32_t total[8] = {};
#pragma unroll
    for (int from = 0; from < ROWS; from += kMxByteRows) {
        Mx4Bytes bytes;
#pragma unroll
        for (int m = from; m < from + kMxByteRows && m < ROWS; ++m)
            if (m < rows) {
                uint32_t codes[8];
                mx4_codes(v[m], byte, philox_tail_not(row_key(high, m, k0), lk, k0, k1), o, m, seed, codes);
                bytes.add(codes, v[m]);
            }
        const int held = rows - from < 0 ? 0 : rows - from < kMxByteRows ? rows - from : kMxByteRows;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            total[j] += bytes.total(j, held);
    }
    if (byte == kMxNaN) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            total[j] = 0;
    }
    finish_octet<NT>(total, byte, by, (o - lane) * 8, d, lane, sum, out);
}

// The whole step with the rows of 512 coordinates spread over a block's four
// waves (wave w takes w, w + 4, ...), which share their maxima and add their
// sums through LDS.  1000 coordinates of 8 workers 3.4 us, 6.4 with a wave for
// all rows.
__global__ __launch_bounds__(kBlock) void k_mx4_step_spread(const float* g, int64_t d, int32_t rows, int64_t ldg,
                                                         uint64_t seed, uint8_t* scales, int32_t* sum, Mx4Mean by,
                                                         float* out, int64_t oct0, int64_t octs)
{
    constexpr int kWaves = kBlock / 64, kEach = 16 / kWaves;
    __shared__ uint32_t tops[kWaves][64];
    __shared__ u32x2 sums[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t o = oct0 + int64_t(blockIdx.x) * 64 + lane;
    float v[kEach][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (wave + kWaves * i < rows)
            load_octet<kF32>(g + (wave + kWaves * i) * ldg, o * 8, d, v[i]);
    const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    const LaneKey lk = lane_key(static_cast<uint32_t>(o), 0, k1);
    uint4 halves[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i)  // while the rows arrive
        halves[i] = philox_tail_not(row_key(static_cast<uint32_t>(o >> 32), wave + kWaves * i, k0), lk, k0, k1);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (wave + kWaves * i < rows)
            top = octet_max(v[i], top);
    tops[wave][lane] = top;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w)
        top = top > tops[w][lane] ? top : tops[w][lane];
    const uint32_t byte = mx4_byte(quad_max(top));
    Mx4Bytes bytes;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (wave + kWaves * i < rows) {
            uint32_t codes[8];
            mx4_codes(v[i], byte, halves[i], o, wave + kWaves * i, seed, codes);
            bytes.add(codes, v[i]);
        }
    sums[wave][lane] = u32x2{bytes.even, bytes.odd};
    __syncthreads();
    if (wave != 0)
        return;
    if ((o & 3) == 0 && o < octs)
        scales[o / 4] = static_cast<uint8_t>(byte);
    int32_t total[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        total[j] = bytes.total(j, rows);
    for (int w = 1; w < kWaves; ++w) {
        bytes.even = sums[w][lane][0];
        bytes.odd = sums[w][lane][1];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            total[j] += bytes.total(j, 0);
    }
    if (byte == kMxNaN) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            total[j] = 0;
    }
    finish_octet<false>(total, byte, by, (o - lane) * 8, d, lane, sum, out);
}

// The rows' codes on given bytes, added into sum (= or +=), and with out the mean.
template <bool NT>
__global__ __launch_bounds__(kBlock) void k_mx4_sum(const float* g, int64_t d, int32_t rows, int64_t ldg,
                                                    int32_t worker0, const uint8_t* scales, uint64_t seed,
                                                    int32_t accumulate, int32_t* sum, Mx4Mean by, float* out,
                                                    int64_t oct0, int64_t octs)
{
    const int lane = threadIdx.x & 63;
    const int64_t o = oct0 + int64_t(blockIdx.x) * kBlock + threadIdx.x;
    uint32_t byte = o < octs ? scales[o / 4] : 1u;
    byte = byte > 1u ? byte : 1u;
    int32_t total[8] = {};
    if (accumulate) {
        float held[8];
        load_octet<kF32>(sum, o * 8, d, held);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            total[j] = __float_as_int(held[j]);
    }
    const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    const LaneKey lk = lane_key(static_cast<uint32_t>(o), 0, k1);
    const uint32_t high = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(o >> 32));
    const float most = __uint_as_float(byte << 23) * 6.0f;
    for (int32_t from = 0; from < rows; from += kMxByteRows) {
        Mx4Bytes bytes;
        const int held = rows - from < kMxByteRows ? rows - from : kMxByteRows;
        for (int m = 0; m < held; ++m) {
            float v[8];
            load_octet<kF32>(g + (from + m) * ldg, o * 8, d, v);
#pragma unroll
            for (int j = 0; j < 8; ++j)  // the byte may not be this row's: no more than the largest code
                v[j] = copysignf(fminf(fabsf(v[j]), most), v[j]);
            uint32_t codes[8];
            const uint32_t id = static_cast<uint32_t>(worker0 + from + m);
            mx4_codes(v, byte, philox_tail_not(row_key(high, id, k0), lk, k0, k1), o, id, seed, codes);
            bytes.add(codes, v);
        }
        if (byte != kMxNaN) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                total[j] += bytes.total(j, held);
        }
    }
    finish_octet<NT>(total, byte, by, (o - lane) * 8, d, lane, sum, out);
}

int64_t blocks_for(int64_t units, int64_t per)
{
    return (units + per - 1) / per;
}

// A row stride (below 2^36 bytes, as the ABI layer checks) in 16-byte units.
uint32_t in16(int64_t bytes)
{
    return static_cast<uint32_t>(bytes / 16);
}

// Rows [row0, rows) in launches of at most `cap` blocks and 2^31 units.
template <typename F>
hipError_t over_rows(int64_t rows, int64_t per_row, F launch)
{
    const int64_t most = one_shot_cap() * kBlock;  // at most 2^30 units
    const int64_t step = most / per_row < 1 ? 1 : most / per_row;
    for (int64_t r = 0; r < rows; r += step) {
        const int64_t n = rows - r < step ? rows - r : step;
        launch(static_cast<uint32_t>(r), static_cast<uint32_t>(n * per_row));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

struct QuantiseArgs {
    const void* x;
    int64_t rows, cols, ldx;
    uint64_t seed;
    uint8_t* codes;
    int64_t ldc;
    uint8_t* scales;
    int64_t lds;
    uint8_t* codes_t;
    int64_t ldct;
    uint8_t* scales_t;
    int64_t ldst;
};

template <int T, bool SR>
hipError_t quantise(const QuantiseArgs& a, hipStream_t stream)
{
    if (a.codes_t == nullptr) {
        const int64_t per_row = blocks_for(a.cols, kMxBlock) * 4;
        const RowDiv div = row_div(static_cast<uint32_t>(per_row));
        return over_rows(a.rows, per_row, [&](uint32_t row0, uint32_t units) {
            k_mx4_rows<T, SR><<<static_cast<unsigned>(blocks_for(units, kBlock)), kBlock, 0, stream>>>(
                a.x, a.cols, in16(a.ldx * kElemBytes<T>), a.seed, a.codes, in16(a.ldc), a.scales, in16(a.lds), row0, units,
                div);
        });
    }
    const int32_t down = static_cast<int32_t>(blocks_for(a.rows, kTileRows));
    const int32_t across = static_cast<int32_t>(blocks_for(a.cols, kTileCols));
    const int64_t tiles = super_blocks(down, across);
    const int64_t cap = one_shot_cap();
    const auto kernel = a.codes != nullptr ? k_mx4_tiles<T, SR, true> : k_mx4_tiles<T, SR, false>;
    for (int64_t t = 0; t < tiles; t += cap) {
        kernel<<<static_cast<unsigned>(tiles - t < cap ? tiles - t : cap), kBlock, 0, stream>>>(
            a.x, a.rows, a.cols, a.ldx, a.seed, a.codes, a.ldc, a.scales, a.lds, a.codes_t, a.ldct, a.scales_t, a.ldst,
            t, down, across);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_mx4_quantize(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ldx, bool stochastic,
                               uint64_t seed, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                               uint8_t* codes_t, int64_t ldct, uint8_t* scales_t, int64_t ldst, hipStream_t stream)
{
    if (rows == 0 || cols == 0)
        return hipSuccess;
    const QuantiseArgs a = {x, rows, cols, ldx, seed, codes, ldc, scales, lds, codes_t, ldct, scales_t, ldst};
    if (stochastic)
        return type == kF32 ? quantise<kF32, true>(a, stream)
                            : type == kBF16 ? quantise<kBF16, true>(a, stream) : quantise<kF16, true>(a, stream);
    return type == kF32 ? quantise<kF32, false>(a, stream)
                        : type == kBF16 ? quantise<kBF16, false>(a, stream) : quantise<kF16, false>(a, stream);
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int64_t rows,
                                 int64_t cols, int32_t type, void* out, int64_t ldo, hipStream_t stream)
{
    if (rows == 0 || cols == 0)
        return hipSuccess;
    const int64_t per_row = blocks_for(cols, type == kF32 ? 4 : 8);
    const RowDiv div = row_div(static_cast<uint32_t>(per_row));
    return over_rows(rows, per_row, [&](uint32_t row0, uint32_t units) {
        const unsigned grid = static_cast<unsigned>(blocks_for(units, kBlock));
        const auto f = type == kF32 ? k_mx4_read<kF32> : type == kBF16 ? k_mx4_read<kBF16> : k_mx4_read<kF16>;
        f<<<grid, kBlock, 0, stream>>>(codes, in16(ldc), scales, in16(lds), cols, out, in16(ldo * (type == kF32 ? 4 : 2)),
                                       row0, units, div);
    });
}

// Octets of d coordinates, `each` to a block of threads, in launches of at
// most the cap.
template <typename F>
static hipError_t over_octets(int64_t d, int64_t each, F launch)
{
    const int64_t octs = blocks_for(d, kMxBlock) * 4, most = one_shot_cap() * each;
    for (int64_t o = 0; o < octs; o += most) {
        launch(o, octs, static_cast<unsigned>(blocks_for(octs - o < most ? octs - o : most, each)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

hipError_t launch_mx4_shared_scale(const float* g, int64_t d, int32_t rows, int64_t ldg, int32_t accumulate,
                                   uint8_t* scales, hipStream_t stream)
{
    return over_octets(d, kBlock, [&](int64_t o, int64_t octs, unsigned grid) {
        k_mx4_shared<<<grid, kBlock, 0, stream>>>(g, d, rows, ldg, accumulate, scales, o, octs);
    });
}

// Sums and outputs beyond this many bytes of each leave nontemporally.
constexpr int64_t kMxNontemporalBytes = int64_t(46) << 20;

hipError_t launch_mx4_quantize_sum(const float* g, int64_t d, int32_t rows, int64_t ldg, int32_t worker0,
                                   const uint8_t* scales, uint64_t seed, int32_t accumulate, int32_t* sum, int32_t M,
                                   float* out, hipStream_t stream)
{
    const Mx4Mean by = {static_cast<double>(M), out != nullptr ? 1.0 / M : 0.0};
    const auto kernel = 4 * d > kMxNontemporalBytes ? k_mx4_sum<true> : k_mx4_sum<false>;
    return over_octets(d, kBlock, [&](int64_t o, int64_t octs, unsigned grid) {
        kernel<<<grid, kBlock, 0, stream>>>(g, d, rows, ldg, worker0, scales, seed, accumulate, sum, by, out, o,
                                            octs);
    });
}

// Gradients beyond this many bytes, the Infinity Cache's size, are read
// nontemporally: 8 workers of 25.6 M coordinates 176.6 us, 181.1 otherwise; 2 of
// them (204 MB) 68.8 and 59.3.
constexpr int64_t kMxStreamBytes = int64_t(256) << 20;
// The rows are spread over a block's waves for 5 rows and more until the
// outputs leave nontemporally, and for fewer up to this many coordinates: 8 rows
// of 262,144 coordinates 4.2 us, 5.5 otherwise, of 11.2 M 80.3 and 85.4, of 25.6 M
// 181.0 and 176.6; 2 rows of 262,144 3.0 either way, of 1.05 M 5.4 and 4.3.
constexpr int64_t kMxSpread = int64_t(1) << 18;

// MOST: the rows that calls of these stores and loads have.
template <bool NT, bool LOADS, int MOST>
static auto step_kernel(int32_t rows)
{
    if constexpr (MOST > 8)
        if (rows > 8)
            return k_mx4_step<16, NT, LOADS>;
    if constexpr (MOST > 4)
        if (rows > 4)
            return k_mx4_step<8, NT, LOADS>;
    return rows > 2 ? k_mx4_step<4, NT, LOADS> : k_mx4_step<2, NT, LOADS>;
}

hipError_t launch_mx4_aggregate(const float* g, int64_t d, int32_t M, int64_t ldg, uint64_t seed, uint8_t* scales,
                                int32_t* sum, float* out, hipStream_t stream)
{
    const Mx4Mean by = {static_cast<double>(M), 1.0 / M};
    const bool spread = 4 * d <= kMxNontemporalBytes && (M >= 5 || d <= kMxSpread);
    // not spread, plain stores: at most 4 rows; outputs past 46 MiB and gradients
    // up to 256 MiB: at most 5
    static_assert(6 * kMxNontemporalBytes >= kMxStreamBytes, "six rows past the one are past the other");
    const auto kernel = spread ? k_mx4_step_spread
                      : 4 * d <= kMxNontemporalBytes ? step_kernel<false, false, 4>(M)
                      : 4 * d * M <= kMxStreamBytes ? step_kernel<true, false, 5>(M) : step_kernel<true, true, 16>(M);
    return over_octets(d, spread ? 64 : kBlock, [&](int64_t o, int64_t octs, unsigned grid) {
        kernel<<<grid, kBlock, 0, stream>>>(g, d, M, ldg, seed, scales, sum, by, out, o, octs);
    });
}

}  // namespace uq
