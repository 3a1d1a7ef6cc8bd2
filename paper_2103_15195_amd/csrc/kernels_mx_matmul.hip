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
// A wavefront's operands for half a step: PA and PB pairs of tiles, and a word of scales for two pairs (the first's in byte 0, the second's in byte 2).
template <int PA, int PB> struct Operands {
    v4i a[PA], b[PB];
    int sa[PA / 2], sb[PB / 2];
};
// Products, and behind each one what `also` issues for its number: instructions leave a wavefront in order, and what stands in front of the
// products in a row keeps the matrix unit waiting.
template <int PA, int PB, class Also>
__device__ __forceinline__ void multiply(const Operands<PA, PB> &o, v16f (&acc)[PA][PB], Also also)
{
    uint32_t i = 0;
#define MC_ONE(dq, dr)                                                                                                        \
    acc[q + dq][r + dr] = mma32<2 * dr, 2 * dq>(o.b[r + dr], o.a[q + dq], acc[q + dq][r + dr], o.sb[r / 2], o.sa[q / 2]);      \
    also(i++);                                                                                                                \
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < PA; q += 2)
#pragma unroll
        for (int r = 0; r < PB; r += 2) {
            MC_ONE(0, 0) MC_ONE(0, 1) MC_ONE(1, 0) MC_ONE(1, 1)
        }
#undef MC_ONE
}
// N sums of a row, to memory as T.
template <class T, int N>
__device__ __forceinline__ void store_sums(global_ptr<T> to, const float (&x)[N])
{
    typedef typename VecOf<T, N>::type vec;
    vec v;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (T)x[e];
    __builtin_nontemporal_store(v, (global_ptr<vec>)to);
}

template <class T, int PA, int PB, int STAGES, int BLOCKS>
__global__ __launch_bounds__(kBlock, BLOCKS) void mx_matmul_lds_k(MxProduct p, uint32_t tiles_a, uint32_t tiles_b)
{
    constexpr uint32_t kTilesA = 4 * PA, kTilesB = 4 * PB, kStages = STAGES;             // tiles of 16 rows to a block
    constexpr uint32_t kCodesA = 0, kCodesB = kTilesA * kMxCodes, kScalesA = kCodesB + kTilesB * kMxCodes, kScalesB = kScalesA + kTilesA / 4 * kMxScales,
                       kStage = kScalesB + kTilesB / 4 * kMxScales;
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
    const uint64_t first_a = (uint64_t)ti * kTilesA, first_b = (uint64_t)tj * kTilesB;                // tiles of 16
    const uint64_t line = (uint64_t)steps * kMxCodes, line_s = (uint64_t)steps * kMxScales;
    const rsrc_t codes_a = buffer_at(p.a.codes + first_a * line, ((p.a.rows + 15u) / 16u - first_a) * line);
    const rsrc_t codes_b = buffer_at(p.b.codes + first_b * line, ((p.b.rows + 15u) / 16u - first_b) * line);
    const rsrc_t scales_a = buffer_at(p.a.scales + first_a / 4u * line_s, ((p.a.rows + 63u) / 64u - first_a / 4u) * line_s);
    const rsrc_t scales_b = buffer_at(p.b.scales + first_b / 4u * line_s, ((p.b.rows + 63u) / 64u - first_b / 4u) * line_s);
    const uint32_t lane16 = lane * 16u, lane4 = lane * 4u, at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    // A wavefront copies a quarter of the step's tiles of either operand, a tile of a's scales and one of b's.
    static_assert(PA == 4 && PB <= 4, "a tile of scales to a wavefront");
    constexpr uint32_t kMineA = kTilesA / 4, kMineB = kTilesB / 4, kCopies = kMineA + kMineB + 2;
    // the k-th of a wavefront's copies for step s
    const auto copy = [&](uint32_t s, uint32_t k) {
        const uint32_t to = at + s % kStages * kStage;
        if (k < kMineA) {
            const uint32_t t = wave * kMineA + k;
            copy16(to + kCodesA + t * kMxCodes, codes_a, (t * steps + s) * kMxCodes + lane16);
        } else if (k < kMineA + kMineB) {
            const uint32_t t = wave * kMineB + k - kMineA;
            copy16(to + kCodesB + t * kMxCodes, codes_b, (t * steps + s) * kMxCodes + lane16);
        } else if (k == kMineA + kMineB) {
            copy4(to + kScalesA + wave * kMxScales, scales_a, (wave * steps + s) * kMxScales + lane4);
        } else {                         // (of two tiles the second is copied three times: the same bytes, and the same number of copies in each wavefront)
            const uint32_t t = wave < PB ? wave : PB - 1u;
            copy4(to + kScalesB + t * kMxScales, scales_b, (t * steps + s) * kMxScales + lane4);
        }
    };
    const auto copies = [&](uint32_t s, uint32_t from, uint32_t n) {
#pragma unroll
        for (uint32_t k = from; k < n; ++k) copy(s, k);
    };
    const uint32_t half_a = wave / 2u, half_b = wave % 2u;               // of the block
    const uint32_t other = lane >> 4 & 1u;                               // which tile of a pair the lane's row is of
    const uint32_t mine16 = other * kMxCodes + (lane >> 5) * 256u + (lane & 15u) * 16u, mine4 = (lane >> 5) * 64u + (lane & 15u) * 4u;
    // the k-th read of half a step's operands
    constexpr uint32_t kReads = PA / 2 + PB / 2 + PA + PB;
    const auto read = [&](uint32_t s, uint32_t half, Operands<PA, PB> &o, uint32_t k) {
        const uint8_t *from = lds + s % kStages * kStage;
        if (k < PA / 2) {
            o.sa[k] = *reinterpret_cast<const int *>(from + kScalesA + (half_a * (PA / 2) + k) * kMxScales + half * 128u + mine4) >> (8u * other);
        } else if (k < PA / 2 + PB / 2) {
            const uint32_t q = k - PA / 2;
            o.sb[q] = *reinterpret_cast<const int *>(from + kScalesB + (half_b * (PB / 2) + q) * kMxScales + half * 128u + mine4) >> (8u * other);
        } else if (k < PA / 2 + PB / 2 + PB) {
            const uint32_t q = k - PA / 2 - PB / 2;
            o.b[q] = *reinterpret_cast<const v4i *>(from + kCodesB + (half_b * PB + q) * 2u * kMxCodes + half * 512u + mine16);
        } else {
            const uint32_t q = k - PA / 2 - PB / 2 - PB;
            o.a[q] = *reinterpret_cast<const v4i *>(from + kCodesA + (half_a * PA + q) * 2u * kMxCodes + half * 512u + mine16);
        }
    };
    v16f acc[PA][PB] = {};
    Operands<PA, PB> first, second;
    // (Steps behind the last are copied too, from the next rows or as zeros, so that the number of copies under way is always the same; nothing multiplies them.)
    // With four stages a step's copies are issued half before and half behind a barrier, with three all behind it.
    constexpr uint32_t kAhead = kStages - 1, kEarly = kStages == 4 ? kCopies / 2 : kCopies, kProducts = PA * PB;
    copies(0, 0, kCopies);
    copies(1, 0, kStages == 4 ? kCopies : 0);
    copied<kStages == 4 ? kCopies : 0>();
    copies(kAhead - 1, 0, kEarly);
#pragma unroll
    for (uint32_t k = 0; k < kReads; ++k) read(0, 0, first, k);
    for (uint32_t s = 0; s < steps; ++s) {
        multiply<PA, PB>(first, acc, [&](uint32_t i) {
#pragma unroll
            for (uint32_t k = i * kReads / kProducts; k < (i + 1) * kReads / kProducts; ++k) read(s, 1, second, k);
#pragma unroll
            for (uint32_t k = i * (kCopies - kEarly) / kProducts; k < (i + 1) * (kCopies - kEarly) / kProducts; ++k) copy(s + kAhead - 1, kEarly + k);
        });
        // step s + 1 is there, and every wavefront has read step s - 1, whose place the next copies take
        copied<kStages == 4 ? kCopies : 0>();
        multiply<PA, PB>(second, acc, [&](uint32_t i) {
#pragma unroll
            for (uint32_t k = i * kReads / kProducts; k < (i + 1) * kReads / kProducts; ++k) read(s + 1, 0, first, k);
#pragma unroll
            for (uint32_t k = i * kEarly / kProducts; k < (i + 1) * kEarly / kProducts; ++k) copy(s + kAhead, k);
        });
    }
    copied<0>();                         // (no copy outlives the block, and no wavefront reads operands any more)
    // Results by rows: each wavefront turns its sets of 32 rows round in a part of LDS of its own, so that what a wavefront stores are whole lines.
    constexpr uint32_t kWide = 32 * PB, kPitch = kWide + 4;              // floats to a row
    static_assert(4 * 32 * kPitch * sizeof(float) <= sizeof(lds), "a part of LDS for each wavefront");
    float *const own = reinterpret_cast<float *>(lds) + wave * 32u * kPitch;
    const uint32_t row0 = ((uint32_t)first_a + half_a * PA * 2u) * 16u, col0 = ((uint32_t)first_b + half_b * PB * 2u) * 16u;
    constexpr int N = 16 / (int)sizeof(T);                               // columns of a lane
    constexpr uint32_t kLanes = kWide / N, kRows = 64u / kLanes;
    const uint32_t mine = lane % kLanes * N;
    const bool whole = col0 + kWide <= p.b.rows;
    float bias[N];
#pragma unroll
    for (int e = 0; e < N; ++e) bias[e] = 0.0f;
    if (p.bias && whole) {
#pragma unroll
        for (int e = 0; e < N; ++e) bias[e] = in_global(p.bias)[col0 + mine + e];
    }
#pragma unroll
    for (uint32_t q = 0; q < PA; ++q) {
#pragma unroll
        for (uint32_t r = 0; r < PB; ++r)
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n)
                *reinterpret_cast<v4f *>(own + (lane & 31u) * kPitch + r * 32u + n * 8u + (lane >> 5) * 4u) =
                    v4f{acc[q][r][4 * n], acc[q][r][4 * n + 1], acc[q][r][4 * n + 2], acc[q][r][4 * n + 3]};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const uint32_t top = row0 + q * 32u;
        if (whole && top + 32u <= p.a.rows && !p.accumulate) {
            global_ptr<T> to = in_global(static_cast<T *>(p.out)) + (int64_t)(top + lane / kLanes) * p.stride + col0 + mine;
#pragma unroll
            for (uint32_t i = 0; i < 32u; i += kRows, to += kRows * p.stride) {
                float x[N];
#pragma unroll
                for (int e = 0; e < N; e += 4) {
                    const v4f y = *reinterpret_cast<const v4f *>(own + (i + lane / kLanes) * kPitch + mine + e);
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[e + k] = y[k] + bias[e + k];
                }
                store_sums<T, N>(to, x);
            }
        } else {
#pragma unroll 1
            for (uint32_t i = 0; i < 32u; i += kRows)
#pragma unroll 1
                for (uint32_t e = 0; e < N; e += 4)
                    finish<T>(p, top + i + lane / kLanes, col0 + mine + e, *reinterpret_cast<const v4f *>(own + (i + lane / kLanes) * kPitch + mine + e));
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
            if (getenv("T4")) { const uint32_t tb = (p.b.rows + 127u) / 128u; launch(mx_matmul_lds_k<T, 4, 2, 3, 2>, dim3(ta * tb), dim3(kBlock), lc.stream, p, ta, tb); }
            else launch(mx_matmul_lds_k<T, 4, 4, 4, 1>, dim3(ta * tb), dim3(kBlock), lc.stream, p, ta, tb);
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
