// Products of microscaled 4-bit matrices.
//
// v_mfma_scale_f32_16x16x128 multiplies 16 x 128 by 128 x 16 values of 4 bits with a scale per 32 of them: lane g * 16 + r holds the 16 bytes of
// block g of row r, and that block's scale in a byte of a word.  Its result has, in lane g * 16 + c, the rows 4 g .. 4 g + 3 of column c.  The rows are those of
// b here and the columns those of a, so that a lane has four consecutive outputs of one row.
#include "mx_internal.h"

namespace mc {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

template <int QA, int QB>
__device__ __forceinline__ v4f mma(v4i x, v4i y, v4f acc, int sx, int sy)
{
    const v8i X = {x[0], x[1], x[2], x[3], 0, 0, 0, 0}, Y = {y[0], y[1], y[2], y[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(X, Y, acc, 4, 4, QA, sx, QB, sy);
}

template <class T>
__device__ __forceinline__ void finish(const MxProduct &p, uint32_t i, uint32_t j, v4f acc)
{
    if (i >= p.a.rows || j >= p.b.rows) return;
    const global_ptr<T> row = in_global(static_cast<T *>(p.out)) + (int64_t)i * p.stride;
    const int32_t hi = (int32_t)p.b.rows;
    float y[4] = {acc[0], acc[1], acc[2], acc[3]};
    if (p.bias) {
        float b[4];
        load_some<4, float, false>(in_global(p.bias), (int32_t)j, 0, hi, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] += b[e];
    }
    if (p.accumulate) {
        float o[4];
        load_some<4, T, false>(row, (int32_t)j, 0, hi, o);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] += o[e];
    }
    store_some<4, T>(row, (int32_t)j, 0, hi, y);
}

// 128 x 128 outputs to a block of four wavefronts of 64 x 64, operands straight from memory.
template <class T>
__global__ __launch_bounds__(kBlock) void mx_matmul_k(MxProduct p, uint64_t first, uint32_t tiles_b)
{
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    const uint32_t ti = (uint32_t)((first + blockIdx.x) / tiles_b) * 2u + wave / 2u, tj = (uint32_t)((first + blockIdx.x) % tiles_b) * 2u + wave % 2u;        // tiles of 64
    if (ti * 64u >= p.a.rows || tj * 64u >= p.b.rows) return;
    const uint32_t last_a = (p.a.rows - 1u) / 16u, last_b = (p.b.rows - 1u) / 16u, steps = p.a.steps;
    global_ptr<const v4i> at[4], bt[4];
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) {           // (tiles beyond the last row stand for the last one: what they give is not stored)
        const uint32_t ra = ti * 4u + q < last_a ? ti * 4u + q : last_a, rb = tj * 4u + q < last_b ? tj * 4u + q : last_b;
        at[q] = (global_ptr<const v4i>)in_global(p.a.codes + (size_t)ra * steps * kMxCodes) + lane;
        bt[q] = (global_ptr<const v4i>)in_global(p.b.codes + (size_t)rb * steps * kMxCodes) + lane;
    }
    const global_ptr<const int> as = (global_ptr<const int>)in_global(p.a.scales + (size_t)ti * steps * kMxScales) + lane;
    const global_ptr<const int> bs = (global_ptr<const int>)in_global(p.b.scales + (size_t)tj * steps * kMxScales) + lane;
    v4f acc[4][4] = {};
    for (uint32_t s = 0; s < steps; ++s) {
        v4i x[4], y[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) { x[q] = at[q][s * 64u]; y[q] = bt[q][s * 64u]; }
        const int sx = as[s * 64u], sy = bs[s * 64u];
#define MC_ROW(q)                                              \
        acc[q][0] = mma<0, q>(y[0], x[q], acc[q][0], sy, sx);  \
        acc[q][1] = mma<1, q>(y[1], x[q], acc[q][1], sy, sx);  \
        acc[q][2] = mma<2, q>(y[2], x[q], acc[q][2], sy, sx);  \
        acc[q][3] = mma<3, q>(y[3], x[q], acc[q][3], sy, sx);
        MC_ROW(0) MC_ROW(1) MC_ROW(2) MC_ROW(3)
#undef MC_ROW
    }
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q)
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r)
            finish<T>(p, ti * 64u + q * 16u + (lane & 15u), tj * 64u + r * 16u + (lane >> 4) * 4u, acc[q][r]);
}

// ---- many rows -----------------------------------------------------------------------------------------------------------
// Operands through LDS: a block of four wavefronts has SIDE x SIDE outputs, a wavefront a quarter of them.  A step's codes and scales are copied straight
// to LDS, three steps ahead; a wavefront reads the next step's operands while it multiplies this one's.
typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));
// What a buffer's loads go by: beyond `bytes` they give 0.
__device__ __forceinline__ rsrc_t buffer_at(const uint8_t *p, uint64_t bytes)
{
    const uint64_t at = (uint64_t)(uintptr_t)p;
    const uint32_t size = bytes < 0xffffffffull ? (uint32_t)bytes : 0xffffffffu;
    return rsrc_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)), (uint32_t)__builtin_amdgcn_readfirstlane((int)size), 0x00020000u};
}
// 16 (4) bytes a lane from its offset `from` to LDS at `to` + 16 (4) * lane.  The compiler does not count these loads: copied() waits.  (The whole offset
// is the lane's: it is that which is checked against the buffer's size.)
__device__ __forceinline__ void copy16(uint32_t to, rsrc_t r, uint32_t from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(from), "s"(r) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, rsrc_t r, uint32_t from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(from), "s"(r) : "memory");
}
// All but the last N of this wavefront's copies are done, and all that it has read from LDS is there; and the same of the block's other wavefronts.
template <int N>
__device__ __forceinline__ void copied()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// v_mfma_scale_f32_32x32x64: lane 32 k + r holds the 16 bytes of block k of row r of 32 rows by 64 columns, half a step of two tiles; of its result lane
// 32 k + c holds, four at a time, the rows 4 k + 8 n .. 4 k + 8 n + 3 of column c.  One wavefront alone keeps the matrix unit busy with it (32 cycles, 9.2 PFLOP/s of all
// units; with 16x16x128, 16 cycles' work, every 29.5 cycles, 5.2 PFLOP/s).
typedef float v16f __attribute__((ext_vector_type(16)));
template <int QX, int QY>
__device__ __forceinline__ v16f mma32(v4i x, v4i y, v16f acc, int sx, int sy)
{
    const v8i X = {x[0], x[1], x[2], x[3], 0, 0, 0, 0}, Y = {y[0], y[1], y[2], y[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(X, Y, acc, 4, 4, QX, sx, QY, sy);
}
// A wavefront's operands for half a step: of either matrix PAIRS pairs of tiles, and a word of scales for two pairs (the first's in byte 0, the second's in byte 2).
template <int PAIRS> struct Operands {
    v4i a[PAIRS], b[PAIRS];
    int sa[PAIRS / 2], sb[PAIRS / 2];
};
// Products in groups of four, and behind each one what `also` issues for its number: instructions leave a wavefront in order, and what stands in front of
// the products in a row keeps the matrix unit waiting.
template <int PAIRS, class Also>
__device__ __forceinline__ void multiply(const Operands<PAIRS> &o, v16f (&acc)[PAIRS][PAIRS], Also also)
{
    uint32_t i = 0;
#define MC_ONE(dq, dr)                                                                                                        \
    acc[q + dq][r + dr] = mma32<2 * dr, 2 * dq>(o.b[r + dr], o.a[q + dq], acc[q + dq][r + dr], o.sb[r / 2], o.sa[q / 2]);      \
    also(i++);                                                                                                                \
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < PAIRS; q += 2)
#pragma unroll
        for (int r = 0; r < PAIRS; r += 2) {
            MC_ONE(0, 0) MC_ONE(0, 1) MC_ONE(1, 0) MC_ONE(1, 1)
        }
#undef MC_ONE
}

template <class T, int PAIRS>
__global__ __launch_bounds__(kBlock, PAIRS == 4 ? 1 : 2) void mx_matmul_lds_k(MxProduct p, uint32_t tiles_a, uint32_t tiles_b)
{
    constexpr uint32_t kTiles = 4 * PAIRS, kStages = 4;             // tiles of 16 rows to a block
    constexpr uint32_t kCodesA = 0, kCodesB = kTiles * kMxCodes, kScalesA = 2 * kCodesB, kScalesB = kScalesA + kTiles / 4 * kMxScales,
                       kStage = kScalesB + kTiles / 4 * kMxScales;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kStages * kStage];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    // Blocks go to the eight dies in turn: each die gets a run of tiles, eight rows of them by as many columns as that takes.
    uint32_t ti, tj;
    {
        constexpr uint32_t kDies = 8, kHigh = 8;
        const uint32_t all = tiles_a * tiles_b, die = blockIdx.x % kDies, each = all / kDies, more = all % kDies;
        const uint32_t t = die * each + (die < more ? die : more) + blockIdx.x / kDies;
        const uint32_t band = t / (kHigh * tiles_b), in = t % (kHigh * tiles_b), high = tiles_a - band * kHigh < kHigh ? tiles_a - band * kHigh : kHigh;
        ti = band * kHigh + in % high;
        tj = in / high;
    }
    const uint32_t steps = p.a.steps;
    const uint64_t first_a = (uint64_t)ti * kTiles, first_b = (uint64_t)tj * kTiles;                // tiles of 16
    const uint64_t line = (uint64_t)steps * kMxCodes, line_s = (uint64_t)steps * kMxScales;
    const rsrc_t codes_a = buffer_at(p.a.codes + first_a * line, ((p.a.rows + 15u) / 16u - first_a) * line);
    const rsrc_t codes_b = buffer_at(p.b.codes + first_b * line, ((p.b.rows + 15u) / 16u - first_b) * line);
    const rsrc_t scales_a = buffer_at(p.a.scales + first_a / 4u * line_s, ((p.a.rows + 63u) / 64u - first_a / 4u) * line_s);
    const rsrc_t scales_b = buffer_at(p.b.scales + first_b / 4u * line_s, ((p.b.rows + 63u) / 64u - first_b / 4u) * line_s);
    const uint32_t lane16 = lane * 16u, lane4 = lane * 4u, at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    // A wavefront copies a quarter of the step's tiles of either operand, and of the scales (PAIRS == 2: each wavefront one tile of the four).
    constexpr uint32_t kMine = kTiles / 4, kCopies = 2 * kMine + kTiles / 8;
    // the k-th of a wavefront's copies for step s
    const auto copy = [&](uint32_t s, uint32_t k) {
        const uint32_t to = at + s % kStages * kStage;
        if (k < 2u * kMine) {
            const uint32_t t = wave * kMine + k / 2u;
            if (k % 2u == 0) copy16(to + kCodesA + t * kMxCodes, codes_a, (t * steps + s) * kMxCodes + lane16);
            else copy16(to + kCodesB + t * kMxCodes, codes_b, (t * steps + s) * kMxCodes + lane16);
        } else if constexpr (PAIRS == 4) {
            if (k % 2u == 0) copy4(to + kScalesA + wave * kMxScales, scales_a, (wave * steps + s) * kMxScales + lane4);
            else copy4(to + kScalesB + wave * kMxScales, scales_b, (wave * steps + s) * kMxScales + lane4);
        } else if (wave < 2u) copy4(to + kScalesA + wave * kMxScales, scales_a, (wave * steps + s) * kMxScales + lane4);
        else copy4(to + kScalesB + (wave - 2u) * kMxScales, scales_b, ((wave - 2u) * steps + s) * kMxScales + lane4);
    };
    const auto copies = [&](uint32_t s, uint32_t from, uint32_t n) {
#pragma unroll
        for (uint32_t k = from; k < n; ++k) copy(s, k);
    };
    const uint32_t half_a = wave / 2u, half_b = wave % 2u;               // of the block
    const uint32_t other = lane >> 4 & 1u;                               // which tile of a pair the lane's row is of
    const uint32_t mine16 = other * kMxCodes + (lane >> 5) * 256u + (lane & 15u) * 16u, mine4 = (lane >> 5) * 64u + (lane & 15u) * 4u;
    // the k-th read of half a step's operands
    constexpr uint32_t kReads = 3 * PAIRS;
    const auto read = [&](uint32_t s, uint32_t half, Operands<PAIRS> &o, uint32_t k) {
        const uint8_t *from = lds + s % kStages * kStage;
        if (k < PAIRS) {
            const uint32_t q = k / 2u;
            if (k % 2u == 0) o.sa[q] = *reinterpret_cast<const int *>(from + kScalesA + (half_a * (PAIRS / 2) + q) * kMxScales + half * 128u + mine4) >> (8u * other);
            else o.sb[q] = *reinterpret_cast<const int *>(from + kScalesB + (half_b * (PAIRS / 2) + q) * kMxScales + half * 128u + mine4) >> (8u * other);
        } else {
            const uint32_t q = (k - PAIRS) / 2u;
            if (k % 2u == 0) o.b[q] = *reinterpret_cast<const v4i *>(from + kCodesB + (half_b * PAIRS + q) * 2u * kMxCodes + half * 512u + mine16);
            else o.a[q] = *reinterpret_cast<const v4i *>(from + kCodesA + (half_a * PAIRS + q) * 2u * kMxCodes + half * 512u + mine16);
        }
    };
    v16f acc[PAIRS][PAIRS] = {};
    Operands<PAIRS> first, second;
    // (Steps behind the last are copied too, from the next rows or as zeros, so that the number of copies under way is always the same; nothing multiplies them.)
    constexpr uint32_t kEarly = kCopies / 2, kProducts = PAIRS * PAIRS;
    copies(0, 0, kCopies);
    copies(1, 0, kCopies);
    copied<kCopies>();
    copies(2, 0, kEarly);
#pragma unroll
    for (uint32_t k = 0; k < kReads; ++k) read(0, 0, first, k);
    for (uint32_t s = 0; s < steps; ++s) {
        multiply<PAIRS>(first, acc, [&](uint32_t i) {
#pragma unroll
            for (uint32_t k = i * kReads / kProducts; k < (i + 1) * kReads / kProducts; ++k) read(s, 1, second, k);
#pragma unroll
            for (uint32_t k = i * (kCopies - kEarly) / kProducts; k < (i + 1) * (kCopies - kEarly) / kProducts; ++k) copy(s + 2, kEarly + k);
        });
        // step s + 1 is there, and every wavefront has read step s - 1, whose place step s + 3 takes
        copied<kCopies>();
        multiply<PAIRS>(second, acc, [&](uint32_t i) {
#pragma unroll
            for (uint32_t k = i * kReads / kProducts; k < (i + 1) * kReads / kProducts; ++k) read(s + 1, 0, first, k);
#pragma unroll
            for (uint32_t k = i * kEarly / kProducts; k < (i + 1) * kEarly / kProducts; ++k) copy(s + 3, k);
        });
    }
    copied<0>();                         // (no copy outlives the block, and no wavefront reads operands any more)
    // Results by rows: each wavefront turns its 32 x 32 PAIRS of them round in a part of LDS of its own, so that what a wavefront stores are whole lines.
    constexpr uint32_t kWide = 32 * PAIRS, kPitch = kWide + 4;           // floats to a row
    static_assert(4 * 32 * kPitch * sizeof(float) <= sizeof(lds), "a part of LDS for each wavefront");
    float *const own = reinterpret_cast<float *>(lds) + wave * 32u * kPitch;
    const uint32_t row0 = ((uint32_t)first_a + half_a * PAIRS * 2u) * 16u, col0 = ((uint32_t)first_b + half_b * PAIRS * 2u) * 16u;
#pragma unroll
    for (uint32_t q = 0; q < PAIRS; ++q) {
#pragma unroll
        for (uint32_t r = 0; r < PAIRS; ++r)
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n)
                *reinterpret_cast<v4f *>(own + (lane & 31u) * kPitch + r * 32u + n * 8u + (lane >> 5) * 4u) =
                    v4f{acc[q][r][4 * n], acc[q][r][4 * n + 1], acc[q][r][4 * n + 2], acc[q][r][4 * n + 3]};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        constexpr uint32_t kLanes = kWide / 4u, kRows = 64u / kLanes;    // four columns a lane
#pragma unroll 4
        for (uint32_t i = 0; i < 32u; i += kRows) {
            const uint32_t r = i + lane / kLanes, c = lane % kLanes * 4u;
            finish<T>(p, row0 + q * 32u + r, col0 + c, *reinterpret_cast<const v4f *>(own + r * kPitch + c));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

template <class T>
static void matmul_of(const LaunchCtx &lc, const MxProduct &p)
{
    if (p.a.rows > 128u && p.a.steps < (1u << 16)) {
        const uint32_t ta = (p.a.rows + 255u) / 256u, tb = (p.b.rows + 255u) / 256u;
        if ((uint64_t)ta * tb < (1u << 23)) {
            launch(mx_matmul_lds_k<T, 4>, dim3(ta * tb), dim3(kBlock), lc.stream, p, ta, tb);
            return;
        }
    }
    const uint32_t tiles_a = (p.a.rows + 127u) / 128u, tiles_b = (p.b.rows + 127u) / 128u;
    in_launches((uint64_t)tiles_a * tiles_b, [&](uint64_t first, uint32_t n) { launch(mx_matmul_k<T>, dim3(n), dim3(kBlock), lc.stream, p, first, tiles_b); });
}
void launch_mx_matmul(const LaunchCtx &lc, int dtype, const MxProduct &p)
{
    if (dtype == MC_DTYPE_F32) matmul_of<float>(lc, p);
    else if (dtype == MC_DTYPE_BF16) matmul_of<__bf16>(lc, p);
    else matmul_of<_Float16>(lc, p);
}

}  // namespace mc
