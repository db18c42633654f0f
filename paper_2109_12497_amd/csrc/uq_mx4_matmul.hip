// The product of two microscaled 4-bit matrices (include/uq.h): the matrix
// cores multiply the 4-bit fields, apply both scale bytes and accumulate in
// binary32.
#include <type_traits>

#include "uq_launch.hpp"
#include "uq_mx4.hpp"

namespace uq {
namespace {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kFp4 = 4;    // the matrix instructions' operand format
constexpr int kBatch = 4;  // stages of 256 along k whose scale bytes a tile loads together

// Which form a product takes; it goes by the sizes alone, and so does the
// order of its sums.
struct MatmulPlan {
    enum Form { kRows, kTiles64, kTiles128, kTiles256 } form;
    int32_t parts;   // of k, added afterwards (kTiles64, kTiles128)
    int32_t mt, nt;  // 16 rows of a and of b that a block takes (kRows)
};

constexpr int64_t kMostParted = int64_t(1) << 24;

constexpr int64_t kUnits = 256;  // compute units

int64_t tile_blocks(int64_t m, int64_t n, MatmulPlan::Form form)
{
    const int64_t high = form == MatmulPlan::kTiles64 ? 64 : form == MatmulPlan::kTiles128 ? 128 : 256;
    const int64_t wide = form == MatmulPlan::kTiles256 ? 256 : 128;
    return ((m + high - 1) / high) * ((n + wide - 1) / wide);
}

// The nanoseconds that each form takes, fitted on one MI355X over 460 products
// (1 to 4096 x 64 to 65536 x 32 to 65536, operands in the caches and not) so
// that the least of them picks the fastest form: within 0.6% of it in the mean,
// 18% at most.
//
// Tiles, `stages` stages of 256 deep: a stage costs more with more compute units
// at work, for they share the caches' bandwidth and then run slower.  8192^3
// 260 us in tiles of 256 x 256; 2048^3 10.7 us in 128 x 128, 19 in 256 x 256; 192 x
// 4096 x 4096 10.9 in 64 x 128, 14.0 in 128 x 128.
double tiles_ns(int64_t m, int64_t n, int64_t stages, int64_t parts, MatmulPlan::Form form)
{
    const int64_t blocks = tile_blocks(m, n, form) * parts;
    const double deep = static_cast<double>(stages), share = static_cast<double>(blocks) / kUnits;
    // the parts are written, read again by another launch, and added: 200 x 1000
    // x 20000 36 us in one part, 24, 17.5 and 16 in two, four and eight
    const double join = parts > 1 ? 2700.0 + 0.001 * static_cast<double>(m * n) * static_cast<double>(parts) : 0.0;
    switch (form) {
    case MatmulPlan::kTiles64: return join + deep * (350.0 + 150.0 * share) + 4900.0;
    case MatmulPlan::kTiles128: {
        if (blocks <= kUnits)
            return join + deep * (520.0 + 280.0 * share) + 4900.0;
        const int64_t rounds = blocks / (2 * kUnits), rest = blocks % (2 * kUnits);
        const double last = rest > 0 ? deep * 1500.0 * (0.5 + 0.5 * static_cast<double>(rest) / (2 * kUnits)) + 5700.0 : 0.0;
        return join + static_cast<double>(rounds) * (deep * 1500.0 + 5700.0) + last;
    }
    default:
        return static_cast<double>((blocks + kUnits - 1) / kUnits) *
               (deep * (1200.0 + 600.0 * (share < 1.0 ? share : 1.0)) + 11000.0);
    }
}

// Few rows: a block reads mt fragments of a and nt of b.  What takes the time
// is the loads that a compute unit issues, so the rows that a unit's blocks
// read decide, those of a, which stay in the caches, by half: 64 x 10001 x 5003
// 13.7 us with nt = 3 (209 blocks), 18.0 with 4 (157), 21.2 with 2 (313, two to
// a unit) and 25.7 with 1; 48 x 8192 x 8192 17.2 with 2 (256 blocks), 19.5, 21.6
// and 23.6 with 3, 4 and 1; 32 x 4096 x 4096 6.6 with 1, 7.6, 8.9 and 10.0 with
// 2, 3 and 4; 32 x 28672 x 8192 38.9 with 4 (448), 48.3, 49.0 and 56.7 with 3, 2
// and 1.  Three beside one fragment of a never were the best (16 x 10001 x 5003
// 14.8, with 1 11.5), and four beside four, which do not fit the registers, nowhere
// by more than 3% before tiles.
MatmulPlan rows_plan(int64_t m, int64_t n)
{
    MatmulPlan best = {MatmulPlan::kRows, 1, m <= 16 ? 1 : m <= 32 ? 2 : m <= 48 ? 3 : 4, 1};
    const int64_t down = (m + 16 * best.mt - 1) / (16 * best.mt), a = m < 16 * best.mt ? m : 16 * best.mt;
    double least = 0.0;
    for (int32_t nt = 1; nt <= 4; ++nt) {
        if ((nt == 3 && best.mt == 1) || (nt == 4 && best.mt == 4))
            continue;
        const int64_t blocks = down * ((n + 16 * nt - 1) / (16 * nt));
        const double rows = static_cast<double>((blocks + 255) / 256) * (0.5 * static_cast<double>(a) + 16.0 * nt);
        if (nt == 1 || rows < least) {
            least = rows;
            best.nt = nt;
        }
    }
    return best;
}

// The rows that a compute unit reads, over k, and what its blocks add up and
// store (all of a unit's blocks start together, so a last round that fills few
// units costs half of one).
double rows_ns(const MatmulPlan& plan, int64_t m, int64_t n, int64_t k)
{
    const int64_t down = (m + 16 * plan.mt - 1) / (16 * plan.mt), a = m < 16 * plan.mt ? m : 16 * plan.mt;
    const int64_t blocks = down * ((n + 16 * plan.nt - 1) / (16 * plan.nt));
    const double share = static_cast<double>(blocks) / 256.0;
    const double rounds = 0.5 * (static_cast<double>((blocks + 255) / 256) + (share < 1.0 ? 1.0 : share));
    const double read = (0.5 * static_cast<double>(a) + 16.0 * plan.nt) * static_cast<double>(k);
    return 1800.0 + rounds * (0.02 * read + 220.0 * plan.mt * plan.nt);
}

// One form for the whole product; *ns is the time it takes.
MatmulPlan one_plan(int64_t m, int64_t n, int64_t k, double* ns)
{
    // 64 x 4096 x 4096 8.9 us as few rows, 10.4 in tiles; 64 x 28672 x 8192 58 and
    // 31; 256 x 1000 x 20000 22 and 16 (eight parts)
    MatmulPlan best = rows_plan(m, n);
    double& least = *ns;
    least = rows_ns(best, m, n, k);
    if (k == 0)
        return best;
    const int64_t stages = (k + 255) / 256, batches = (stages + kBatch - 1) / kBatch;
    // parts of more outputs than this never pay, and bound the workspace (512 MB)
    const int32_t most = m * n <= kMostParted ? 8 : 1;
    for (int32_t parts = 1; parts <= most && parts <= batches; parts *= 2) {
        const int64_t deep = parts == 1 ? stages : (batches + parts - 1) / parts * kBatch;
        for (const auto form : {MatmulPlan::kTiles64, MatmulPlan::kTiles128}) {
            // tiles of 64 x 128 are for a single round: 1024 x 4096 x 4096 20.1
            // us in two, 16.5 in one of 128 x 128
            if (form == MatmulPlan::kTiles64 && tile_blocks(m, n, form) * parts > kUnits)
                continue;
            const double t = tiles_ns(m, n, deep, parts, form);
            if (t < least) {
                least = t;
                best = {form, parts, 0, 0};
            }
        }
    }
    const double t = tiles_ns(m, n, stages, 1, MatmulPlan::kTiles256);
    if (t < least) {
        least = t;
        best = {MatmulPlan::kTiles256, 1, 0, 0};
    }
    return best;
}

// A product in one form, or its first rows (or columns) in tiles that fill
// whole rounds and the others in a form of their own.
struct MatmulSplit {
    MatmulPlan first, rest;
    int64_t m, n;  // of the first
};

// 2304 x 8497 x 13601 in 306 tiles of 256 x 256 takes two rounds for a round
// and a fifth, 216 us; 252 tiles and then 1329 columns 182.  2112 x 7854 x 7168 98.6
// and 71.9 us.
MatmulSplit matmul_plan(int64_t m, int64_t n, int64_t k)
{
    double least;
    MatmulSplit best = {one_plan(m, n, k, &least), {}, m, n};
    if (m == 0 || n == 0 || k == 0)
        return best;
    constexpr double kLaunch = 2000.0;  // the second launch
    const int64_t stages = (k + 255) / 256;
    for (const auto form : {MatmulPlan::kTiles128, MatmulPlan::kTiles256}) {
        const int64_t side = form == MatmulPlan::kTiles128 ? 128 : 256;
        const int64_t round = form == MatmulPlan::kTiles128 ? 2 * kUnits : kUnits;
        const int64_t down = (m + side - 1) / side, across = (n + side - 1) / side;
        const int64_t full = down * across / round * round;  // tiles in whole rounds
        for (const bool by_rows : {false, true}) {
            const int64_t lines = full / (by_rows ? across : down);
            if (lines == 0 || lines >= (by_rows ? down : across))
                continue;
            const int64_t m1 = by_rows ? lines * side : m, n1 = by_rows ? n : lines * side;
            double rest;
            const MatmulPlan plan = one_plan(by_rows ? m - m1 : m, by_rows ? n : n - n1, k, &rest);
            const double t = tiles_ns(m1, n1, stages, 1, form) + rest + kLaunch;
            if (t < least) {
                least = t;
                best = {{form, 1, 0, 0}, plan, m1, n1};
            }
        }
    }
    return best;
}

// The element at `at` of the output, of type `type` (the same for the whole launch).
__device__ __forceinline__ float load_out(int32_t type, const void* out, int64_t at)
{
    return type == kF32 ? static_cast<const float*>(out)[at]
         : type == kBF16 ? static_cast<float>(static_cast<const __bf16*>(out)[at])
                         : static_cast<float>(static_cast<const _Float16*>(out)[at]);
}

__device__ __forceinline__ void store_out(int32_t type, void* out, int64_t at, float v)
{
    if (type == kF32)
        static_cast<float*>(out)[at] = v;
    else if (type == kBF16)
        static_cast<__bf16*>(out)[at] = static_cast<__bf16>(v);
    else
        static_cast<_Float16*>(out)[at] = static_cast<_Float16>(v);
}

// Four columns of the output as they lie in memory, and their values.
template <int T>
using Four = std::conditional_t<T == kF32, f32x4, u32x2>;

template <int T>
__device__ __forceinline__ f32x4 values(Four<T> x)
{
    if constexpr (T == kF32)
        return x;
    const uint32_t x0 = x[0], x1 = x[1];
    if constexpr (T == kBF16)
        return f32x4{__uint_as_float(x0 << 16), __uint_as_float(x0 & 0xFFFF0000u), __uint_as_float(x1 << 16),
                     __uint_as_float(x1 & 0xFFFF0000u)};
    const f16x2 a = __builtin_bit_cast(f16x2, x0), b = __builtin_bit_cast(f16x2, x1);
    return f32x4{static_cast<float>(a[0]), static_cast<float>(a[1]), static_cast<float>(b[0]), static_cast<float>(b[1])};
}

// Columns col .. col + 3 (a multiple of 4) of the row that starts at `row`, of
// n; `old` is what load_four read there before.  PAST, past: nontemporally.
template <int T, bool PAST>
__device__ __forceinline__ Four<T> load_four(const void* out, int64_t row, int64_t col, int64_t n)
{
    using Element = std::conditional_t<T == kF32, float, uint16_t>;
    const auto* at = reinterpret_cast<const Four<T>*>(static_cast<const Element*>(out) + row + col);
    return col + 4 > n ? Four<T>{} : PAST ? __builtin_nontemporal_load(at) : *at;
}

template <typename V>
__device__ __forceinline__ void store_past(bool past, V v, V* at)
{
    if (past) {  // empty statements keep the compiler from merging the stores into a plain one
        asm volatile("");
        __builtin_nontemporal_store(v, at);
        asm volatile("");
    } else {
        *at = v;
    }
}

template <int T>
__device__ __forceinline__ void store_four(void* out, int64_t row, int64_t col, int64_t n, f32x4 v, bool accumulate,
                                           Four<T> old, bool past)
{
    if (col + 4 > n) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < n)
                store_out(T, out, row + col + j, accumulate ? load_out(T, out, row + col + j) + v[j] : v[j]);
        return;
    }
    if (accumulate)
        v += values<T>(old);
    if constexpr (T == kF32) {
        store_past(past, v, reinterpret_cast<f32x4*>(static_cast<float*>(out) + row + col));
    } else {
        u32x2* o = reinterpret_cast<u32x2*>(static_cast<uint16_t*>(out) + row + col);
        if constexpr (T == kBF16) {
            const bf16x2 a = {static_cast<__bf16>(v[0]), static_cast<__bf16>(v[1])};
            const bf16x2 b = {static_cast<__bf16>(v[2]), static_cast<__bf16>(v[3])};
            store_past(past, u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)}, o);
        } else {
            const f16x2 a = {static_cast<_Float16>(v[0]), static_cast<_Float16>(v[1])};
            const f16x2 b = {static_cast<_Float16>(v[2]), static_cast<_Float16>(v[3])};
            store_past(past, u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)}, o);
        }
    }
}

__device__ __forceinline__ i32x8 operand(i32x4 v)
{
    return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0};
}

// ---------------------------------------------------------------------------
// Tiles staged through LDS.
// ---------------------------------------------------------------------------
constexpr int kStageBlocks = 8;                             // blocks of 32 along k in a stage
constexpr int kStageBytes = kStageBlocks * kMxBlockBytes;   // of one row's codes: a cache line
constexpr uint32_t kPast = 0x80000000u;                     // a buffer offset past every operand (reads as 0)

__device__ __forceinline__ i32x4 buffer_of(const uint8_t* p, int64_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    return i32x4{static_cast<int>(at), static_cast<int>((at >> 32) & 0xFFFF), static_cast<int>(bytes > 0 ? bytes : 0),
                 0x00027000};
}

// A load straight into LDS: lane i's 16 bytes go to lds + 16 i.  It has no
// register result; the waits on such loads are the caller's (vmcnt), and the
// compiler, which does not know of them, can only wait for more than it needs.
// The s_nop is the wait state between a write of m0 and a load that uses it;
// nothing else in these kernels uses m0 (a reserved register, which the
// compiler takes in no clobber list).
__device__ __forceinline__ void load_lds16(i32x4 r, uint32_t off, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(r)
                 : "memory");
}
struct MatmulArgs {
    const uint8_t *a, *as, *b, *bs;
    int64_t lda, ldas, ldb, ldbs;
    int64_t m, n, nkb;
    void* out;
    int64_t ldo;
    int32_t type, accumulate;
    int32_t tiles_m, tiles_n;
    int64_t part_blocks;  // blocks along k of a part (all of them: one part)
    int64_t part_bytes;   // between the parts' outputs
    int32_t first;        // the launch's first block
    bool past;            // tiles' outputs are stored nontemporally
};

// Block -> tile.  Blocks go to the eight XCDs in turn, and each XCD has its
// own L2: an XCD's blocks take a run of tiles, and a run goes down kBand tiles
// of a column before it goes to the next, so that the 32 blocks an XCD holds
// at a time share 8 bands of rows and 4 of columns.
constexpr int kXcds = 8, kBand = 8;

__device__ __forceinline__ void place(int block, int tiles_m, int tiles_n, int* tm, int* tn)
{
    const int all = tiles_m * tiles_n, per = all / kXcds, more = all % kXcds, xcd = block % kXcds;
    const int tile = xcd * per + (xcd < more ? xcd : more) + block / kXcds;
    const int band = tile / (kBand * tiles_n), first = band * kBand;
    const int high = tiles_m - first < kBand ? tiles_m - first : kBand, in = tile - first * tiles_n;
    *tn = in / high;
    *tm = first + (in - *tn * high);
}

// One operand in LDS.  A stage's codes are ROWS rows of kStageBytes, the
// 16-byte piece c of row r at slot c ^ ((r / 2) & 7): sixteen rows of one
// piece then lie in all the banks.  Scale bytes come a batch of four stages at
// a time, ROWS rows of 32 bytes (loads of a row's 8 bytes of each stage cost
// as much time as the codes, for they touch as many lines: 1.01 us a stage of
// 256 + 256 rows against 0.58 without), piece p of row r at slot
// p ^ ((r / 8) & 1).
constexpr int kBatchBytes = kBatch * kStageBlocks;

template <int ROWS, int W>
struct Operand {
    static constexpr int kCodes = ROWS * kStageBytes, kScales = ROWS * kBatchBytes;
    static constexpr int kStep = 8 * W, kLoads = ROWS / kStep;  // of a wave, a stage's codes
    // and a batch's scales, 32 rows at a time (waves past the rows load what
    // others do)
    static constexpr int kScaleWaves = ROWS / 32 < W ? ROWS / 32 : W;
    static constexpr int kScaleStep = 32 * kScaleWaves, kScaleLoads = ROWS / kScaleStep;
    static_assert(ROWS % kStep == 0 && ROWS % kScaleStep == 0, "every load is whole");

    const uint8_t *p, *s;
    uint32_t ld, ld_s, to, to_s;  // to, to_s: where this wave's parts go in LDS
    int64_t bytes, bytes_s;       // of the rows there are; the rest read as 0
    uint32_t off, off_s;

    __device__ __forceinline__ Operand(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds,
                                       int64_t row0, int64_t rows, int64_t kb0, uint32_t lds_codes,
                                       uint32_t lds_scales, int wave, int lane)
    {
        const int64_t have = rows - row0 < ROWS ? rows - row0 : ROWS;
        p = codes + row0 * ldc + kb0 * kMxBlockBytes;
        s = scales + row0 * lds + kb0;
        ld = static_cast<uint32_t>(ldc);
        ld_s = static_cast<uint32_t>(lds);
        bytes = have * ldc - kb0 * kMxBlockBytes;
        bytes_s = have * lds - kb0;
        const int row = wave * 8 + (lane >> 3), srow = wave % kScaleWaves * 32 + (lane >> 1);
        off = row * ld + (((lane & 7) ^ ((row >> 1) & 7)) << 4);
        off_s = srow * ld_s + (((lane & 1) ^ ((srow >> 3) & 1)) << 4);
        to = lds_codes + wave * 8 * kStageBytes;
        to_s = lds_scales + wave % kScaleWaves * 32 * kBatchBytes;
    }
    // Blocks past the last (nkb) read as 0.
    __device__ __forceinline__ uint32_t offset(int64_t kb, int64_t nkb, int wave, int lane) const
    {
        const int row = wave * 8 + (lane >> 3), c = (lane & 7) ^ ((row >> 1) & 7);
        return kb + c < nkb ? off : kPast;
    }
    __device__ __forceinline__ i32x4 codes_from(int64_t kb) const
    {
        return buffer_of(p + kb * kMxBlockBytes, bytes - kb * kMxBlockBytes);
    }
    __device__ __forceinline__ i32x4 scales_from(int64_t kb) const
    {
        return buffer_of(s + kb, bytes_s - kb);
    }

    static __device__ __forceinline__ i32x4 piece(const uint8_t* lds, int row, int c)
    {
        return *reinterpret_cast<const i32x4*>(lds + row * kStageBytes + ((c ^ ((row >> 1) & 7)) << 4));
    }
    static __device__ __forceinline__ uint32_t scale(const uint8_t* lds, int row, int stage, int half)
    {
        const int slot = ((stage >> 1) & 1) ^ ((row >> 3) & 1);
        return *reinterpret_cast<const uint32_t*>(lds + row * kBatchBytes + slot * 16 + (stage & 1) * 8 + half * 4);
    }
};

// A block of WM x WN waves forms a tile of 32 WM FM x 32 WN FN outputs; a wave
// holds FM x FN accumulators of 32 x 32.  Lane l holds row l % 32 of an
// operand's fragment and the blocks 4 (l / 32) + t of a stage for its
// instruction t = 0..3: any order of the blocks along k gives the same
// products as long as both operands keep to it, and in this one a lane's four
// scale bytes are one dword.
//   What bounds it, 8192^3 to bf16 on one MI355X: 261 us, 4210 TFLOP/s (three
// sets of operands in turn, the card warm; 257 to 265 from card to card).  The
// card lowers its clock by the data: on zeros the same instructions take 187
// us (5890), and matrix instructions alone reach 6540 on random codes and 9000
// on zeros.  The rest is the loads into LDS (without them, on random codes, 15%
// less), and the outputs, which all compute units store at once (4%).  Eight
// waves of 128 x 64 against four of 128 x 128: 1% less time.
template <int T, int WM, int WN, int FM, int FN, int NS>
__global__ __launch_bounds__(64 * WM * WN, 1) void k_mx4_tiles(MatmulArgs g)
{
    constexpr int W = WM * WN, BM = 32 * WM * FM, BN = 32 * WN * FN;
    using A = Operand<BM, W>;
    using B = Operand<BN, W>;
    constexpr int kStage = A::kCodes + B::kCodes, kScaleBatch = A::kScales + B::kScales;
    __shared__ __attribute__((aligned(128))) uint8_t smem[NS * kStage + 2 * kScaleBatch];
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(
        (__attribute__((address_space(3))) uint8_t*)smem));
    constexpr int kScalesAt = NS * kStage;

    const int tiles = g.tiles_m * g.tiles_n, block = g.first + blockIdx.x, part = __builtin_amdgcn_readfirstlane(block / tiles);
    int tm, tn;
    place(block - part * tiles, g.tiles_m, g.tiles_n, &tm, &tn);
    // the buffers' addresses have to be scalar for the loads that take them
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    const int64_t kb0 = part * g.part_blocks;
    const int64_t nkb = g.nkb - kb0 < g.part_blocks ? g.nkb - kb0 : g.part_blocks;
    char* const out = static_cast<char*>(g.out) + part * g.part_bytes;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row0 = int64_t(tm) * BM, col0 = int64_t(tn) * BN;
    const int wm = wave / WN, wn = wave % WN, half = lane >> 5;
    const int ar = wm * 32 * FM + (lane & 31), br = wn * 32 * FN + (lane & 31);
    const A a(g.a, g.lda, g.as, g.ldas, row0, g.m, kb0, lds0, lds0 + kScalesAt, wave, lane);
    const B b(g.b, g.ldb, g.bs, g.ldbs, col0, g.n, kb0, lds0 + A::kCodes, lds0 + kScalesAt + A::kScales, wave, lane);
    const int64_t stages = (nkb + kStageBlocks - 1) / kStageBlocks;

    // The loads of stage `stage`'s codes, one at a time.
    struct Codes {
        i32x4 ra, rb;
        uint32_t oa, ob, buf;
    };
    const auto codes_of = [&](int64_t stage) {
        const int64_t kb = stage * kStageBlocks;
        return Codes{a.codes_from(kb), b.codes_from(kb), a.offset(kb, nkb, wave, lane), b.offset(kb, nkb, wave, lane),
                     static_cast<uint32_t>(stage & (NS - 1)) * kStage};
    };
    const auto load_codes = [&](const Codes& c, int j) {
        if (j < A::kLoads)
            load_lds16(c.ra, c.oa + j * A::kStep * a.ld, a.to + c.buf + j * A::kStep * kStageBytes);
        else
            load_lds16(c.rb, c.ob + (j - A::kLoads) * B::kStep * b.ld,
                       b.to + c.buf + (j - A::kLoads) * B::kStep * kStageBytes);
    };
    // Load i of the scales of batch `batch`.
    constexpr int kScaleLoads = A::kScaleLoads + B::kScaleLoads;
    static_assert(kScaleLoads <= kBatch, "a batch's scales are loaded one a stage");
    const auto load_scales = [&](int64_t batch, int i) {
        const int64_t kb = batch * kBatchBytes;
        const bool of_b = i >= A::kScaleLoads;
        const int j = of_b ? i - A::kScaleLoads : i;
        const uint32_t buf = static_cast<uint32_t>(batch & 1) * kScaleBatch;
        load_lds16(of_b ? b.scales_from(kb) : a.scales_from(kb),
                   of_b ? b.off_s + j * B::kScaleStep * b.ld_s : a.off_s + j * A::kScaleStep * a.ld_s,
                   (of_b ? b.to_s : a.to_s) + buf + j * A::kScaleStep * kBatchBytes);
    };
    // every load into LDS but the last `later` and every read of it by this
    // wave is done, then the other waves' are
    const auto sync = [](auto later) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(later)::value) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    f32x16 acc[FM][FN] = {};
    i32x4 fa[2][FM], fb[2][FN];
    uint32_t sa[2][FM], sb[2][FN];
    const auto read_a = [&](int64_t stage, int t, int i) {
        return A::piece(smem + (stage & (NS - 1)) * kStage, ar + 32 * i, 4 * half + t);
    };
    const auto read_b = [&](int64_t stage, int t, int j) {
        return B::piece(smem + (stage & (NS - 1)) * kStage + A::kCodes, br + 32 * j, 4 * half + t);
    };
    const auto read_scales = [&](int64_t stage, uint32_t(&xa)[FM], uint32_t(&xb)[FN]) {
        const uint8_t* l = smem + kScalesAt + ((stage / kBatch) & 1) * kScaleBatch;
        const int at = static_cast<int>(stage % kBatch);
#pragma unroll
        for (int i = 0; i < FM; ++i)
            xa[i] = A::scale(l, ar + 32 * i, at, half);
#pragma unroll
        for (int j = 0; j < FN; ++j)
            xb[j] = B::scale(l + A::kScales, br + 32 * j, at, half);
    };
    // Bytes of blocks past the last (their codes are 0) must not be NaN's.
    const auto keep_scales = [&](int64_t stage, uint32_t(&xa)[FM], uint32_t(&xb)[FN]) {
        const int64_t left = nkb - stage * kStageBlocks - 4 * half;
        const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
        for (int i = 0; i < FM; ++i)
            xa[i] &= keep;
#pragma unroll
        for (int j = 0; j < FN; ++j)
            xb[j] &= keep;
    };

    // A stage is four instructions' depth; each is cut into FM groups of FN
    // instructions, with a group's share of the next depth's reads and of the
    // loads of a later stage between them: a wave waits for its loads to be
    // taken, so they are spread.  LDS holds NS stages; the loads go into the
    // part that the current stage leaves at its fourth depth, start there and
    // end two depths into the next stage.  Stages past the last read as zeros,
    // past every operand's end, and enter no product.
    constexpr int kLoads = A::kLoads + B::kLoads, kSlots = 3 * FM, kPer = (kLoads + kSlots - 1) / kSlots;
    Codes next = codes_of(0);
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i)
        load_scales(0, i);
    load_scales(1, 0);
#pragma unroll
    for (int st = 0; st < NS - 1; ++st) {
        next = codes_of(st);
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
            load_codes(next, l);
    }
    next = codes_of(NS - 1);
    constexpr int kFirst = FM * kPer < kLoads ? FM * kPer : kLoads;  // at a stage's fourth depth
#pragma unroll
    for (int l = 0; l < kFirst; ++l)
        load_codes(next, l);
    sync(std::integral_constant<int, (NS - 2) * kLoads + kFirst>{});
    read_scales(0, sa[0], sb[0]);
    keep_scales(0, sa[0], sb[0]);
#pragma unroll
    for (int i = 0; i < FM; ++i)
        fa[0][i] = read_a(0, 0, i);
#pragma unroll
    for (int j = 0; j < FN; ++j)
        fb[0][j] = read_b(0, 0, j);
    const auto depth = [&](auto sub, int64_t s) {
        constexpr int t = decltype(sub)::value, tn = (t + 1) & 3;
        const int64_t from = t == 3 ? s + 1 : s;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            fa[tn & 1][i] = read_a(from, tn, i);
#pragma unroll
            for (int j = i * FN / FM; j < (i + 1) * FN / FM; ++j)
                fb[tn & 1][j] = read_b(from, tn, j);
            if (t != 2) {
                const int slot = ((t + 1) & 3) * FM + i;
#pragma unroll
                for (int l = slot * kPer; l < (slot + 1) * kPer && l < kLoads; ++l)
                    load_codes(next, l);
            }
#pragma unroll
            for (int j = 0; j < FN; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                    operand(fa[t & 1][i]), operand(fb[t & 1][j]), acc[i][j], kFp4, kFp4, t, sa[0][i], t, sb[0][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int64_t s = 0; s < stages; ++s) {
        depth(std::integral_constant<int, 0>{}, s);
        depth(std::integral_constant<int, 1>{}, s);
        depth(std::integral_constant<int, 2>{}, s);
        // stage s has been read whole, stage s + 1 has arrived
        sync(std::integral_constant<int, (NS - 2) * kLoads>{});
        next = codes_of(s + NS);
        // (with two stages a batch's loads are repeated rather than skipped: all
        // have arrived before they are read, and the branch costs registers)
        if (NS == 2 || (s + 1) % kBatch < kScaleLoads)
            load_scales((s + 1) / kBatch + 1, static_cast<int>((s + 1) % kBatch) % kScaleLoads);
        read_scales(s + 1, sa[1], sb[1]);
        depth(std::integral_constant<int, 3>{}, s);
        keep_scales(s + 1, sa[1], sb[1]);
#pragma unroll
        for (int i = 0; i < FM; ++i)
            sa[0][i] = sa[1][i];
#pragma unroll
        for (int j = 0; j < FN; ++j)
            sb[0][j] = sb[1][j];
    }
    // Out through LDS, 32 rows of the wave's columns at a time, so that a lane
    // stores four columns.  Rows are kPitch floats apart: the two halves of a
    // wave, four rows apart, then write different banks.  What the sums are
    // added to is read 64 rows ahead (4096 x 4096 x 8192 to fp32 88 us, 95 where a
    // row's are read before its store).
    constexpr int kCols = 32 * FN, kPitch = kCols + 8, kLanes = kCols / 4, kTurns = 32 * kLanes / 64;
    static_assert(W * 32 * kPitch * 4 <= sizeof(smem) && kPitch % 16 == 8, "the waves' parts fit the stages");
    sync(std::integral_constant<int, 0>{});
    float* mine = reinterpret_cast<float*>(smem) + wave * 32 * kPitch;
    const int64_t col = col0 + wn * kCols + (lane % kLanes) * 4, first = row0 + wm * 32 * FM + lane / kLanes;
    const bool add = g.accumulate != 0;
    Four<T> old[3][kTurns];
    // Large tiles read them nontemporally (8192^3 added to bf16, outputs in turn,
    // 291 us, 312 otherwise, one output each time 289 and 281; 4096 x 4096 x 8192 to
    // fp32 87 and 82 either way), small ones not (1000 x 3000 x 700 11.7 and 10.5).
    constexpr bool kReadPast = BM * BN >= 256 * 256;
    const auto load_old = [&](int i) {
#pragma unroll
        for (int r = 0; r < kTurns; ++r) {
            const int64_t row = first + 32 * i + r * (64 / kLanes);
            if (row < g.m)
                old[i % 3][r] = load_four<T, kReadPast>(out, row * g.ldo, col, g.n);
        }
    };
    if (add) {
        load_old(0);
        if constexpr (FM > 1)
            load_old(1);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        if (add && i + 2 < FM)
            load_old(i + 2);
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                mine[((r & 3) + 8 * (r >> 2) + 4 * half) * kPitch + 32 * j + (lane & 31)] = acc[i][j][r];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r = 0; r < kTurns; ++r) {
            const int at = r * (64 / kLanes);
            const f32x4 v = *reinterpret_cast<const f32x4*>(mine + (at + lane / kLanes) * kPitch + (lane % kLanes) * 4);
            const int64_t row = first + 32 * i + at;
            if (row < g.m)
                store_four<T>(out, row * g.ldo, col, g.n, v, add, old[i % 3][r], g.past);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// out = the parts' sum, in their order (+ out): one thread per four columns.
template <int T>
__global__ __launch_bounds__(kBlock) void k_mx4_join(const float* parts, int32_t count, int64_t m, int64_t n,
                                                     int64_t ldp, void* out, int64_t ldo, int32_t accumulate,
                                                     uint32_t row0, uint32_t units, RowDiv div)
{
    const uint32_t u = blockIdx.x * kBlock + threadIdx.x;
    if (u >= units)
        return;
    const uint32_t in = div_row(u, div);
    const int64_t row = row0 + in, col = int64_t(u - in * div.n) * 4;
    const Four<T> old = accumulate != 0 ? load_four<T, false>(out, row * ldo, col, n) : Four<T>{};
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int32_t c = 0; c < count; ++c)
        v += *reinterpret_cast<const f32x4*>(parts + (c * m + row) * ldp + col);
    store_four<T>(out, row * ldo, col, n, v, accumulate != 0, old, false);
}

// ---------------------------------------------------------------------------
// Few rows of a, or few outputs: both operands go straight into registers.  Up
// to 64 rows of a every row of b is read once.
// ---------------------------------------------------------------------------
// A block forms 16 MT x 16 NT outputs; its waves share k in chunks of 16
// blocks (512 elements), and add their sums through LDS in the waves' order.
// Lane l holds row l % 16 of a fragment and, for instruction t = 0..3 of a
// chunk, its block 4 t + l / 16: an instruction's load then covers 64
// contiguous bytes of each row, a chunk's four 256.
constexpr int kChunk = 16;

template <int N>
struct Fragments {
    i32x4 v[N][4];
    u32x4 s[N];

    template <bool WHOLE>
    __device__ __forceinline__ void load(const uint8_t* const (&p)[N], const uint8_t* const (&ps)[N], int64_t chunk,
                                         int64_t nkb, int q)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = *reinterpret_cast<const u32x4*>(ps[i] + chunk * kChunk);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int64_t kb = chunk * kChunk + 4 * t + q;
                if (WHOLE || kb < nkb)
                    v[i][t] = *reinterpret_cast<const i32x4*>(p[i] + kb * kMxBlockBytes);
                else
                    v[i][t] = i32x4{0, 0, 0, 0};
            }
        }
    }
    // The scale byte of this lane's block in instruction t; of blocks past the
    // last (their codes are 0) not a NaN's.
    template <bool WHOLE>
    __device__ __forceinline__ uint32_t scale(int i, int t, int64_t chunk, int64_t nkb, int q) const
    {
        const uint32_t b = s[i][t] >> (8 * q);
        return WHOLE || chunk * kChunk + 4 * t + q < nkb ? b : 0u;
    }
};

constexpr int kRowWaves = 8;

template <int MT, int NT>
__global__ __launch_bounds__(64 * kRowWaves) void k_mx4_rows_by(MatmulArgs g)
{
    __shared__ f32x4 part[kRowWaves][MT][NT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
    const int waves = blockDim.x >> 6;
    const int block = g.first + blockIdx.x, tm = block % g.tiles_m, tn = block / g.tiles_m;
    const int64_t row0 = int64_t(tm) * 16 * MT, col0 = int64_t(tn) * 16 * NT;
    const uint8_t *pa[MT], *sa[MT], *pb[NT], *sb[NT];
    // rows past the end are read as the last one; what they give is not stored
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t r = row0 + 16 * i + (lane & 15) < g.m ? row0 + 16 * i + (lane & 15) : g.m - 1;
        pa[i] = g.a + r * g.lda;
        sa[i] = g.as + r * g.ldas;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t r = col0 + 16 * j + (lane & 15) < g.n ? col0 + 16 * j + (lane & 15) : g.n - 1;
        pb[j] = g.b + r * g.ldb;
        sb[j] = g.bs + r * g.ldbs;
    }
    f32x4 acc[MT][NT] = {};
    const int64_t nkb = g.nkb, chunks = (nkb + kChunk - 1) / kChunk, whole = nkb / kChunk;
    const auto multiply = [&](auto all, const Fragments<MT>& fa, const Fragments<NT>& fb, int64_t c) {
        constexpr bool W = decltype(all)::value;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const uint32_t s = fb.template scale<W>(j, t, c, nkb, q);
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        operand(fa.v[i][t]), operand(fb.v[j][t]), acc[i][j], kFp4, kFp4, 0,
                        fa.template scale<W>(i, t, c, nkb, q), 0, s);
            }
    };
    int64_t c = wave;
    // two chunks' loads at a time where the registers hold them (37 x 10001 x
    // 5003, 3 and 4 fragments: 10.4 us with two, 9.4 with one)
    for (; MT + NT <= 6 && c + waves < whole; c += 2 * waves) {
        Fragments<NT> b0, b1;
        Fragments<MT> a0, a1;
        b0.template load<true>(pb, sb, c, nkb, q);
        b1.template load<true>(pb, sb, c + waves, nkb, q);
        a0.template load<true>(pa, sa, c, nkb, q);
        a1.template load<true>(pa, sa, c + waves, nkb, q);
        multiply(std::true_type{}, a0, b0, c);
        multiply(std::true_type{}, a1, b1, c + waves);
    }
    for (; c < chunks; c += waves) {
        Fragments<NT> b0;
        Fragments<MT> a0;
        b0.template load<false>(pb, sb, c, nkb, q);
        a0.template load<false>(pa, sa, c, nkb, q);
        multiply(std::false_type{}, a0, b0, c);
    }
    const int held = chunks < 1 ? 1 : chunks < waves ? static_cast<int>(chunks) : waves;  // waves with a share of k
    if (wave < held)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
                part[wave][i][j][lane] = acc[i][j];
    __syncthreads();
    for (int f = wave; f < MT * NT; f += waves) {
        const int i = f / NT, j = f % NT;
        const int64_t row = row0 + 16 * i + 4 * q, col = col0 + 16 * j + (lane & 15);
        f32x4 v = part[0][i][j][lane];
        for (int w = 1; w < held; ++w)
            v += part[w][i][j][lane];
        // all four are read before one is stored
        const auto finish = [&](auto type) {
            constexpr int T = decltype(type)::value;
            float old[4];
            if (g.accumulate != 0) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    old[r] = row + r < g.m && col < g.n ? load_out(T, g.out, (row + r) * g.ldo + col) : 0.0f;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    v[r] += old[r];
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (row + r < g.m && col < g.n)
                    store_out(T, g.out, (row + r) * g.ldo + col, v[r]);
        };
        if (g.type == kF32)
            finish(std::integral_constant<int, kF32>{});
        else if (g.type == kBF16)
            finish(std::integral_constant<int, kBF16>{});
        else
            finish(std::integral_constant<int, kF16>{});
    }
}

// `blocks` blocks of `threads`, in launches of at most the cap.
template <typename F>
hipError_t over_blocks(F kernel, MatmulArgs g, int64_t blocks, unsigned threads, hipStream_t stream)
{
    const int64_t cap = one_shot_cap();
    for (int64_t b = 0; b < blocks; b += cap) {
        g.first = static_cast<int32_t>(b);
        kernel<<<static_cast<unsigned>(blocks - b < cap ? blocks - b : cap), threads, 0, stream>>>(g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

template <int T, int WM, int WN, int FM, int FN, int NS>
hipError_t tiles(MatmulArgs g, int32_t parts, float* ws, hipStream_t stream)
{
    constexpr int BM = 32 * WM * FM, BN = 32 * WN * FN;
    g.tiles_m = static_cast<int32_t>((g.m + BM - 1) / BM);
    g.tiles_n = static_cast<int32_t>((g.n + BN - 1) / BN);
    if (parts == 1) {
        g.part_blocks = g.nkb;
        g.part_bytes = 0;
        return over_blocks(k_mx4_tiles<T, WM, WN, FM, FN, NS>, g, int64_t(g.tiles_m) * g.tiles_n, 64 * WM * WN, stream);
    }
    constexpr int64_t kUnit = kBatch * kStageBlocks;
    MatmulArgs p = g;
    p.part_blocks = ((g.nkb + kUnit - 1) / kUnit + parts - 1) / parts * kUnit;
    p.ldo = (g.n + 3) / 4 * 4;
    p.part_bytes = g.m * p.ldo * 4;
    p.out = ws;
    p.accumulate = 0;
    hipError_t e = over_blocks(k_mx4_tiles<kF32, WM, WN, FM, FN, NS>, p, int64_t(g.tiles_m) * g.tiles_n * parts,
                               64 * WM * WN, stream);
    const int64_t per_row = p.ldo / 4, most = (int64_t(1) << 30) / per_row < 1 ? 1 : (int64_t(1) << 30) / per_row;
    const RowDiv div = row_div(static_cast<uint32_t>(per_row));
    for (int64_t r = 0; r < g.m && e == hipSuccess; r += most) {
        const uint32_t units = static_cast<uint32_t>((g.m - r < most ? g.m - r : most) * per_row);
        k_mx4_join<T><<<(units + kBlock - 1) / kBlock, kBlock, 0, stream>>>(
            ws, parts, g.m, g.n, p.ldo, g.out, g.ldo, g.accumulate, static_cast<uint32_t>(r), units, div);
        e = hipGetLastError();
    }
    return e;
}

template <int MT, int NT>
hipError_t rows_by(MatmulArgs g, hipStream_t stream)
{
    g.tiles_m = static_cast<int32_t>((g.m + 16 * MT - 1) / (16 * MT));
    g.tiles_n = static_cast<int32_t>((g.n + 16 * NT - 1) / (16 * NT));
    const int64_t chunks = (g.nkb + kChunk - 1) / kChunk;
    // a wave for a chunk, or more to store the fragments (40 x 16000 x 2 6.6 us
    // by one wave, 3.9 by eight)
    const int64_t most = chunks > MT * NT ? chunks : MT * NT;
    const unsigned waves = most < kRowWaves ? static_cast<unsigned>(most) : kRowWaves;
    return over_blocks(k_mx4_rows_by<MT, NT>, g, int64_t(g.tiles_m) * g.tiles_n, 64 * waves, stream);
}

template <int MT>
hipError_t rows_by(const MatmulArgs& g, int32_t nt, hipStream_t stream)
{
    if (nt == 1)
        return rows_by<MT, 1>(g, stream);
    if (nt == 2)
        return rows_by<MT, 2>(g, stream);
    if constexpr (MT > 1)
        if (nt == 3)
            return rows_by<MT, 3>(g, stream);
    if constexpr (MT < 4)
        return rows_by<MT, 4>(g, stream);
    return hipErrorInvalidValue;  // rows_plan gives no other
}

// Two stages of 128 x 128 leave room for another block on the compute unit,
// four are faster where there is none: 126 x 1628 x 13400 40 us with four, 53 with
// two (13 blocks); 1024 x 8192 x 8192 57 and 53 (512 blocks).  Eight waves of 64
// x 32 outputs take 14.0 us for 192 x 4096 x 4096, four of 64 x 64 14.8; of 64 x 128
// outputs, four of 32 x 64 10.9, two of 64 x 64 14.2.
template <int T>
hipError_t tiles(const MatmulArgs& g, const MatmulPlan& plan, float* ws, hipStream_t stream)
{
    switch (plan.form) {
    case MatmulPlan::kTiles64: return tiles<T, 2, 2, 1, 2, 4>(g, plan.parts, ws, stream);
    case MatmulPlan::kTiles128:
        return tile_blocks(g.m, g.n, plan.form) * plan.parts <= kUnits ? tiles<T, 2, 4, 2, 1, 4>(g, plan.parts, ws, stream)
                                                                 : tiles<T, 2, 2, 2, 2, 2>(g, plan.parts, ws, stream);
    default: return tiles<T, 2, 4, 4, 2, 2>(g, 1, ws, stream);
    }
}

hipError_t product(const MatmulArgs& g, const MatmulPlan& plan, float* ws, hipStream_t stream)
{
    if (plan.form != MatmulPlan::kRows)
        return g.type == kF32 ? tiles<kF32>(g, plan, ws, stream)
                              : g.type == kBF16 ? tiles<kBF16>(g, plan, ws, stream) : tiles<kF16>(g, plan, ws, stream);
    switch (plan.mt) {
    case 1: return rows_by<1>(g, plan.nt, stream);
    case 2: return rows_by<2>(g, plan.nt, stream);
    case 3: return rows_by<3>(g, plan.nt, stream);
    default: return rows_by<4>(g, plan.nt, stream);
    }
}

}  // namespace

// Outputs from half the Infinity Cache's size on pass it by.  With three outputs
// in turn 8192^3 to bf16 (134 MB) takes 261 us, 277 otherwise, added to 291 and 304,
// 65536 x 1024 x 1024 60 and 75, 8192 x 4096 x 4096 added to fp32 (134 MB) 122 and 127; one
// output each time 259 and 263, 289 and 280, 59 and 64, 122 and 107.  What loses
// is a product added to one output again and again with nothing in between; a
// layer of 8192 x 8192 and 8192 rows (bf16, its own y and dw each time, dw added to)
// takes 310 us forward, 335 otherwise, and 681 backward, 717.  4096 x 4096 x 8192 (67 MB)
// lost 5% with one output and gained nothing with three.
constexpr double kPastBytes = 128.0 * (1 << 20);

static size_t parts_bytes(const MatmulPlan& plan, int64_t m, int64_t n)
{
    return plan.parts > 1 ? align256(static_cast<size_t>(plan.parts) * m * ((n + 3) / 4 * 4) * sizeof(float)) : 256;
}

size_t mx4_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    const MatmulSplit s = matmul_plan(m, n, k);
    const size_t first = parts_bytes(s.first, s.m, s.n);
    const size_t rest = s.m < m ? parts_bytes(s.rest, m - s.m, n) : s.n < n ? parts_bytes(s.rest, m, n - s.n) : 0;
    return first > rest ? first : rest;
}

hipError_t launch_mx4_matmul(const uint8_t* a, int64_t lda, const uint8_t* as, int64_t ldas, const uint8_t* b,
                             int64_t ldb, const uint8_t* bs, int64_t ldbs, int64_t m, int64_t n, int64_t k,
                             int32_t type, void* out, int64_t ldo, int32_t accumulate, void* ws, hipStream_t stream)
{
    if (m == 0 || n == 0)
        return hipSuccess;
    constexpr int64_t kMostLd = 1 << 23;  // a tile's rows lie within a buffer's 2^31 bytes
    const int64_t size = type == kF32 ? 4 : 2;
    MatmulArgs g = {a, as, b, bs, lda, ldas, ldb, ldbs, m, n, (k + 31) / 32, out, ldo, type, accumulate,
                    0, 0, 0, 0, 0, static_cast<double>(m) * static_cast<double>(n * size) >= kPastBytes};
    if (lda > kMostLd || ldb > kMostLd || ldas > kMostLd || ldbs > kMostLd)
        return product(g, rows_plan(m, n), nullptr, stream);
    const MatmulSplit s = matmul_plan(m, n, k);
    g.m = s.m;
    g.n = s.n;
    const hipError_t e = product(g, s.first, static_cast<float*>(ws), stream);
    if (e != hipSuccess || (s.m == m && s.n == n))
        return e;
    if (s.m < m) {
        g.m = m - s.m;
        g.a += s.m * lda;
        g.as += s.m * ldas;
        g.out = static_cast<char*>(out) + s.m * ldo * size;
    } else {
        g.n = n - s.n;
        g.b += s.n * ldb;
        g.bs += s.n * ldbs;
        g.out = static_cast<char*>(out) + s.n * size;
    }
    return product(g, s.rest, static_cast<float*>(ws), stream);
}

}  // namespace uq
