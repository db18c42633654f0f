// The product of two microscaled 4-bit matrices (include/uq.h): the matrix
// cores multiply the 4-bit fields, apply both scale bytes and accumulate in
// binary32.
#include "uq_launch.hpp"
#include "uq_mx4.hpp"

namespace uq {
namespace {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kFp4 = 4;  // the matrix instructions' operand format

template <int T>
__device__ __forceinline__ void store_out(void* out, int64_t at, float v, bool accumulate)
{
    if constexpr (T == kF32) {
        float* o = static_cast<float*>(out) + at;
        *o = accumulate ? *o + v : v;
    } else if constexpr (T == kBF16) {
        __bf16* o = static_cast<__bf16*>(out) + at;
        *o = static_cast<__bf16>(accumulate ? static_cast<float>(*o) + v : v);
    } else {
        _Float16* o = static_cast<_Float16*>(out) + at;
        *o = static_cast<_Float16>(accumulate ? static_cast<float>(*o) + v : v);
    }
}

__device__ __forceinline__ i32x8 operand(i32x4 v)
{
    return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0};
}

// One wave per 32 x 32 outputs: lane l holds row l % 32 of both operands and
// every second block of 32 along k.
template <int T>
__global__ __launch_bounds__(kBlock) void k_mx4_matmul(const uint8_t* a, int64_t lda, const uint8_t* as, int64_t ldas,
                                                       const uint8_t* b, int64_t ldb, const uint8_t* bs, int64_t ldbs,
                                                       int64_t m, int64_t n, int64_t nkb, void* out, int64_t ldo,
                                                       int32_t accumulate, int64_t tile0, int64_t tiles_n)
{
    const int64_t tile = tile0 + blockIdx.x;
    const int64_t tm = tile / tiles_n, tn = tile - tm * tiles_n;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = tm * 64 + (wave >> 1) * 32 + (lane & 31), col = tn * 64 + (wave & 1) * 32 + (lane & 31);
    const bool row_ok = row < m, col_ok = col < n;
    f32x16 acc = {};
    for (int64_t kb = lane >> 5; kb < ((nkb + 1) & ~int64_t(1)); kb += 2) {
        i32x4 va = {0, 0, 0, 0}, vb = {0, 0, 0, 0};
        int sa = 127, sb = 127;
        if (row_ok && kb < nkb) {
            va = *reinterpret_cast<const i32x4*>(a + row * lda + kb * kMxBlockBytes);
            sa = as[row * ldas + kb];
        }
        if (col_ok && kb < nkb) {
            vb = *reinterpret_cast<const i32x4*>(b + col * ldb + kb * kMxBlockBytes);
            sb = bs[col * ldbs + kb];
        }
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(va), operand(vb), acc, kFp4, kFp4, 0, sa, 0, sb);
    }
    if (!col_ok)
        return;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int64_t i = tm * 64 + (wave >> 1) * 32 + (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5);
        if (i < m)
            store_out<T>(out, i * ldo + col, acc[r], accumulate != 0);
    }
}

}  // namespace

size_t mx4_matmul_workspace_bytes(int64_t, int64_t, int64_t)
{
    return 256;
}

hipError_t launch_mx4_matmul(const uint8_t* a, int64_t lda, const uint8_t* as, int64_t ldas, const uint8_t* b,
                             int64_t ldb, const uint8_t* bs, int64_t ldbs, int64_t m, int64_t n, int64_t k,
                             int32_t type, void* out, int64_t ldo, int32_t accumulate, void*, hipStream_t stream)
{
    if (m == 0 || n == 0)
        return hipSuccess;
    const int64_t tiles_n = (n + 63) / 64, tiles = (m + 63) / 64 * tiles_n, nkb = (k + 31) / 32;
    const int64_t cap = one_shot_cap();
    for (int64_t t = 0; t < tiles; t += cap) {
        const unsigned grid = static_cast<unsigned>(tiles - t < cap ? tiles - t : cap);
        const auto f = type == kF32 ? k_mx4_matmul<kF32> : type == kBF16 ? k_mx4_matmul<kBF16> : k_mx4_matmul<kF16>;
        f<<<grid, kBlock, 0, stream>>>(a, lda, as, ldas, b, ldb, bs, ldbs, m, n, nkb, out, ldo, accumulate, t,
                                       tiles_n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace uq
