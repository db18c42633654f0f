// Microscaled 4-bit floating point: quantisation, reading back and the
// aggregation step on that format (include/uq.h).
#include "uq_launch.hpp"
#include "uq_mx4.hpp"

namespace uq {
namespace {

// Elements 8 * octet .. + 7 of one row as binary32 (zeros past cols).  Whole
// octets are read in 16-byte pieces (rows start on 16-byte boundaries), the
// last ragged one element by element: nothing past cols is read.
template <int T>
__device__ __forceinline__ void load_octet(const void* row, int64_t col, int64_t cols, float (&x)[8])
{
    if (col + 8 <= cols) {
        if constexpr (T == kF32) {
            const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(row) + col);
            const f32x4 a = p[0], b = p[1];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = a[j];
                x[4 + j] = b[j];
            }
        } else {
            const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(row) + col);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (T == kBF16) {
                    x[2 * j] = __uint_as_float(v[j] << 16);
                    x[2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u);
                } else {
                    const uint32_t pair = v[j];
                    const f16x2 h = __builtin_bit_cast(f16x2, pair);
                    x[2 * j] = static_cast<float>(h[0]);
                    x[2 * j + 1] = static_cast<float>(h[1]);
                }
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = 0.0f;
        if (col + j < cols) {
            if constexpr (T == kF32)
                x[j] = static_cast<const float*>(row)[col + j];
            else if constexpr (T == kBF16)
                x[j] = __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(row)[col + j]) << 16);
            else
                x[j] = static_cast<float>(static_cast<const _Float16*>(row)[col + j]);
        }
    }
}

// Eight stochastic fields of row `worker`, octet `oct`.
__device__ __forceinline__ uint32_t mx4_stochastic(const float (&x)[8], uint32_t byte, uint64_t oct, uint32_t worker,
                                                   uint64_t seed)
{
    const float to_half = mx4_half_units(byte);
    const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    const uint32_t c0 = static_cast<uint32_t>(oct), c1 = static_cast<uint32_t>(oct >> 32);
    const uint4 hi = philox4x32_10(c0, c1, worker, 0, k0, k1), lo = philox4x32_10(c0, c1, worker, 1, k0, k1);
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t r = (philox_half(hi, j) << 16) | philox_half(lo, j);
        w |= (mx4_exact(x[j], to_half, r) | (__float_as_uint(x[j]) >> 31 << 3)) << (4 * j);
    }
    return w;
}

// Codes along the rows: one thread per octet, the four threads of a block's
// octets share its maximum.  A unit of the grid is an octet of the padded rows.
template <int T, bool SR>
__global__ __launch_bounds__(kBlock) void k_mx4_rows(const void* x, int64_t cols, int64_t ldx, uint64_t seed,
                                                     uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                                                     uint32_t row0, uint32_t units, RowDiv div)
{
    const uint32_t u = blockIdx.x * kBlock + threadIdx.x;
    if (u >= units)
        return;
    const uint32_t in = div_row(u, div);
    const uint32_t oct = u - in * div.n;
    const uint32_t row = row0 + in;
    float v[8];
    load_octet<T>(static_cast<const char*>(x) + row * ldx * kElemBytes<T>, int64_t(oct) * 8, cols, v);
    const uint32_t byte = mx4_byte(quad_max(octet_max(v)));
    uint32_t w = SR ? mx4_stochastic(v, byte, oct, row, seed) : mx4_nearest(v, byte);
    w = byte == kMxNaN ? 0u : w;
    *reinterpret_cast<uint32_t*>(codes + row * ldc + int64_t(oct) * 4) = w;
    if ((oct & 3) == 0)
        scales[row * lds + oct / 4] = static_cast<uint8_t>(byte);
}

// Codes of the transposed matrix: one thread per column and block of 32 rows.
template <int T, bool SR>
__global__ __launch_bounds__(kBlock) void k_mx4_cols(const void* x, int64_t rows, int64_t cols, int64_t ldx,
                                                     uint64_t seed, uint8_t* codes, int64_t ldc, uint8_t* scales,
                                                     int64_t lds, int64_t unit0, int64_t units, int64_t col_units)
{
    const int64_t u = unit0 + int64_t(blockIdx.x) * kBlock + threadIdx.x;
    if (u >= units)
        return;
    const int64_t blk = u / col_units, col = u - blk * col_units;
    if (col >= cols)
        return;
    float v[4][8];
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const int64_t row = blk * 32 + j;
        float t = 0.0f;
        if (row < rows) {
            if constexpr (T == kF32)
                t = static_cast<const float*>(x)[row * ldx + col];
            else if constexpr (T == kBF16)
                t = __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(x)[row * ldx + col]) << 16);
            else
                t = static_cast<float>(static_cast<const _Float16*>(x)[row * ldx + col]);
        }
        v[j / 8][j % 8] = t;
        const uint32_t b = __float_as_uint(t) & 0x7FFFFFFFu;
        top = top > b ? top : b;
    }
    const uint32_t byte = mx4_byte(top);
    u32x4 w;
    for (int q = 0; q < 4; ++q) {
        if constexpr (SR) {
            const float to_half = mx4_half_units(byte);
            const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
            const uint32_t c0 = static_cast<uint32_t>(col / 8), c1 = static_cast<uint32_t>((col / 8) >> 32);
            uint32_t f = 0;
            for (int j = 0; j < 8; ++j) {
                const uint32_t row = static_cast<uint32_t>(blk * 32 + q * 8 + j);
                const uint4 hi = philox4x32_10(c0, c1, row, 0, k0, k1), lo = philox4x32_10(c0, c1, row, 1, k0, k1);
                const uint32_t r = (philox_half(hi, col & 7) << 16) | philox_half(lo, col & 7);
                f |= (mx4_exact(v[q][j], to_half, r) | (__float_as_uint(v[q][j]) >> 31 << 3)) << (4 * j);
            }
            w[q] = f;
        } else {
            w[q] = mx4_nearest(v[q], byte);
        }
    }
    if (byte == kMxNaN)
        w = u32x4{0, 0, 0, 0};
    *reinterpret_cast<u32x4*>(codes + col * ldc + blk * kMxBlockBytes) = w;
    scales[col * lds + blk] = static_cast<uint8_t>(byte);
}

// One thread per octet: 4 bytes of codes and the block's byte in, eight
// values out.  The converters decode, scale and round once, and give NaN for
// the scale byte 255.
template <int T>
__global__ __launch_bounds__(kBlock) void k_mx4_read(const uint8_t* codes, int64_t ldc, const uint8_t* scales,
                                                     int64_t lds, int64_t cols, void* out, int64_t ldo,
                                                     uint32_t row0, uint32_t units, RowDiv div)
{
    const uint32_t u = blockIdx.x * kBlock + threadIdx.x;
    if (u >= units)
        return;
    const uint32_t in = div_row(u, div);
    const uint32_t oct = u - in * div.n;
    const uint32_t row = row0 + in;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + row * ldc + int64_t(oct) * 4);
    const float s = __uint_as_float(static_cast<uint32_t>(scales[row * lds + oct / 4]) << 23);
    const int64_t col = int64_t(oct) * 8;
    if constexpr (T == kF32) {
        const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3)};
        float* o = static_cast<float*>(out) + row * ldo + col;
        if (col + 8 <= cols) {
            reinterpret_cast<f32x4*>(o)[0] = f32x4{p[0][0], p[0][1], p[1][0], p[1][1]};
            reinterpret_cast<f32x4*>(o)[1] = f32x4{p[2][0], p[2][1], p[3][0], p[3][1]};
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < cols)
                    o[j] = p[j / 2][j % 2];
        }
    } else {
        u32x4 v;
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
        uint16_t* o = static_cast<uint16_t*>(out) + row * ldo + col;
        if (col + 8 <= cols) {
            *reinterpret_cast<u32x4*>(o) = v;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < cols)
                    o[j] = static_cast<uint16_t>(v[j / 2] >> (16 * (j % 2)));
        }
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
        const uint32_t t = octet_max(v);
        top = top > t ? top : t;
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

// 2^(e - 1) / M as one binary32 factor (rounded once; NaN for the NaN byte).
__device__ __forceinline__ float mx4_mean_factor(uint32_t byte, float inv_m)
{
    // 2^(byte - 128) = 2^(byte - 1 - 127): exact, below 2^-126 as a denormal
    const float half = byte > 1u ? __uint_as_float((byte - 1u) << 23) : __uint_as_float(byte == 1u ? 0x00400000u
                                                                                               : 0x00200000u);
    return byte == kMxNaN ? __uint_as_float(0x7FC00000u) : half * inv_m;
}

// The rows' codes in half units on the given bytes, added into sum, and with
// out the mean.  FORM: the bytes are formed from the rows first and stored.
template <bool FORM>
__global__ __launch_bounds__(kBlock) void k_mx4_sum(const float* g, int64_t d, int32_t rows, int64_t ldg,
                                                    int32_t worker0, uint8_t* scales, uint64_t seed,
                                                    int32_t accumulate, int32_t* sum, float inv_m, float* out,
                                                    int64_t oct0, int64_t octs)
{
    const int64_t o = oct0 + int64_t(blockIdx.x) * kBlock + threadIdx.x;
    if (o >= octs)
        return;
    uint32_t byte;
    if constexpr (FORM) {
        uint32_t top = 0;
        for (int32_t m = 0; m < rows; ++m) {
            float v[8];
            load_octet<kF32>(g + m * ldg, o * 8, d, v);
            const uint32_t t = octet_max(v);
            top = top > t ? top : t;
        }
        byte = mx4_byte(quad_max(top));
        if ((o & 3) == 0)
            scales[o / 4] = static_cast<uint8_t>(byte);
    } else {
        byte = scales[o / 4];
    }
    const float to_half = mx4_half_units(byte);
    int32_t acc[8] = {};
    const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    const uint32_t c0 = static_cast<uint32_t>(o), c1 = static_cast<uint32_t>(o >> 32);
    if (byte != kMxNaN)
        for (int32_t m = 0; m < rows; ++m) {
            float v[8];
            load_octet<kF32>(g + m * ldg, o * 8, d, v);
            const uint32_t id = static_cast<uint32_t>(worker0 + m);
            const uint4 hi = philox4x32_10(c0, c1, id, 0, k0, k1), lo = philox4x32_10(c0, c1, id, 1, k0, k1);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t r = (philox_half(hi, j) << 16) | philox_half(lo, j);
                const int32_t h = mx4_half_value(mx4_exact(v[j], to_half, r));
                acc[j] += v[j] < 0.0f ? -h : h;
            }
        }
    const float deq = mx4_mean_factor(byte, inv_m);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t i = o * 8 + j;
        if (i < d) {
            const int32_t s = acc[j] + (accumulate ? sum[i] : 0);
            sum[i] = s;
            if (out != nullptr)
                out[i] = static_cast<float>(s) * deq;
        }
    }
}

int64_t blocks_for(int64_t units, int64_t per)
{
    return (units + per - 1) / per;
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

template <int T>
hipError_t quantise(const void* x, int64_t rows, int64_t cols, int64_t ldx, bool sr, uint64_t seed, uint8_t* codes,
                    int64_t ldc, uint8_t* scales, int64_t lds, uint8_t* codes_t, int64_t ldct, uint8_t* scales_t,
                    int64_t ldst, hipStream_t stream)
{
    hipError_t e = hipSuccess;
    if (codes != nullptr) {
        const int64_t per_row = blocks_for(cols, kMxBlock) * 4;
        const RowDiv div = row_div(static_cast<uint32_t>(per_row));
        e = over_rows(rows, per_row, [&](uint32_t row0, uint32_t units) {
            const unsigned grid = static_cast<unsigned>(blocks_for(units, kBlock));
            if (sr)
                k_mx4_rows<T, true><<<grid, kBlock, 0, stream>>>(x, cols, ldx, seed, codes, ldc, scales, lds, row0,
                                                                units, div);
            else
                k_mx4_rows<T, false><<<grid, kBlock, 0, stream>>>(x, cols, ldx, seed, codes, ldc, scales, lds, row0,
                                                                 units, div);
        });
    }
    if (e == hipSuccess && codes_t != nullptr) {
        const int64_t col_units = blocks_for(cols, 64) * 64;
        const int64_t units = blocks_for(rows, kMxBlock) * col_units;
        const int64_t cap = one_shot_cap() * kBlock;
        for (int64_t u = 0; u < units && e == hipSuccess; u += cap) {
            const unsigned grid = static_cast<unsigned>(blocks_for(units - u < cap ? units - u : cap, kBlock));
            if (sr)
                k_mx4_cols<T, true><<<grid, kBlock, 0, stream>>>(x, rows, cols, ldx, seed, codes_t, ldct, scales_t,
                                                                ldst, u, units, col_units);
            else
                k_mx4_cols<T, false><<<grid, kBlock, 0, stream>>>(x, rows, cols, ldx, seed, codes_t, ldct, scales_t,
                                                                 ldst, u, units, col_units);
            e = hipGetLastError();
        }
    }
    return e;
}

}  // namespace

hipError_t launch_mx4_quantize(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ldx, bool stochastic,
                               uint64_t seed, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                               uint8_t* codes_t, int64_t ldct, uint8_t* scales_t, int64_t ldst, hipStream_t stream)
{
    if (rows == 0 || cols == 0)
        return hipSuccess;
    const auto f = type == kF32 ? quantise<kF32> : type == kBF16 ? quantise<kBF16> : quantise<kF16>;
    return f(x, rows, cols, ldx, stochastic, seed, codes, ldc, scales, lds, codes_t, ldct, scales_t, ldst, stream);
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int64_t rows,
                                 int64_t cols, int32_t type, void* out, int64_t ldo, hipStream_t stream)
{
    if (rows == 0 || cols == 0)
        return hipSuccess;
    const int64_t per_row = blocks_for(cols, 8);
    const RowDiv div = row_div(static_cast<uint32_t>(per_row));
    return over_rows(rows, per_row, [&](uint32_t row0, uint32_t units) {
        const unsigned grid = static_cast<unsigned>(blocks_for(units, kBlock));
        if (type == kF32)
            k_mx4_read<kF32><<<grid, kBlock, 0, stream>>>(codes, ldc, scales, lds, cols, out, ldo, row0, units, div);
        else if (type == kBF16)
            k_mx4_read<kBF16><<<grid, kBlock, 0, stream>>>(codes, ldc, scales, lds, cols, out, ldo, row0, units, div);
        else
            k_mx4_read<kF16><<<grid, kBlock, 0, stream>>>(codes, ldc, scales, lds, cols, out, ldo, row0, units, div);
    });
}

// Octets of d coordinates, four to a block, in launches of at most the cap.
template <typename F>
static hipError_t over_octets(int64_t d, F launch)
{
    const int64_t octs = blocks_for(d, kMxBlock) * 4, most = one_shot_cap() * kBlock;
    for (int64_t o = 0; o < octs; o += most) {
        launch(o, octs, static_cast<unsigned>(blocks_for(octs - o < most ? octs - o : most, kBlock)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

hipError_t launch_mx4_shared_scale(const float* g, int64_t d, int32_t rows, int64_t ldg, int32_t accumulate,
                                   uint8_t* scales, hipStream_t stream)
{
    return over_octets(d, [&](int64_t o, int64_t octs, unsigned grid) {
        k_mx4_shared<<<grid, kBlock, 0, stream>>>(g, d, rows, ldg, accumulate, scales, o, octs);
    });
}

hipError_t launch_mx4_quantize_sum(const float* g, int64_t d, int32_t rows, int64_t ldg, int32_t worker0,
                                   const uint8_t* scales, uint64_t seed, int32_t accumulate, int32_t* sum, int32_t M,
                                   float* out, hipStream_t stream)
{
    const float inv_m = out != nullptr ? 1.0f / static_cast<float>(M) : 0.0f;
    return over_octets(d, [&](int64_t o, int64_t octs, unsigned grid) {
        k_mx4_sum<false><<<grid, kBlock, 0, stream>>>(g, d, rows, ldg, worker0, const_cast<uint8_t*>(scales), seed,
                                                      accumulate, sum, inv_m, out, o, octs);
    });
}

hipError_t launch_mx4_aggregate(const float* g, int64_t d, int32_t M, int64_t ldg, uint64_t seed, uint8_t* scales,
                                int32_t* sum, float* out, hipStream_t stream)
{
    const float inv_m = 1.0f / static_cast<float>(M);
    return over_octets(d, [&](int64_t o, int64_t octs, unsigned grid) {
        k_mx4_sum<true><<<grid, kBlock, 0, stream>>>(g, d, M, ldg, 0, scales, seed, 0, sum, inv_m, out, o, octs);
    });
}

}  // namespace uq
