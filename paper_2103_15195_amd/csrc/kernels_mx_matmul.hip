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

// ---- few rows -------------------------------------------------------------------------------------------------------------
// Operands straight from memory, b's past the caches: a block of eight wavefronts has 16 MT rows by 16 NT columns of outputs, which its wavefronts sum over steps
// of their own (the w-th over the w-th, w + 8-th ... step, so that they read b's tiles in one run), and SPLITS blocks share the steps where they are very many.
constexpr uint32_t kFewWaves = 8;
template <int MT, int NT> struct FewStep {   // operands of one step
    v4i a[MT], b[NT];
    int sa, sb;
};
template <int MT, int NT, int Q = 0, int R = 0>
__device__ __forceinline__ void few_products(const FewStep<MT, NT> &o, v4f (&acc)[MT][NT])
{
    if constexpr (Q < MT) {
        acc[Q][R] = mma<R, Q>(o.b[R], o.a[Q], acc[Q][R], o.sb, o.sa);
        few_products<MT, NT, R + 1 < NT ? Q : Q + 1, R + 1 < NT ? R + 1 : 0>(o, acc);
    }
}
template <class T, int MT, int NT>
__global__ __launch_bounds__(kFewWaves * 64) void mx_matmul_few_k(MxProduct p, uint64_t first, uint32_t tiles_b, uint32_t splits)
{
    constexpr int kDeep = MT * NT <= 4 ? 4 : 2;      // steps on their way at once
    __shared__ v4f sums[kFewWaves][MT * NT][64];
    const uint32_t waves = blockDim.x / 64u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    const uint64_t at = (first + blockIdx.x) / splits;
    const uint32_t split = (uint32_t)((first + blockIdx.x) % splits), ti = (uint32_t)(at / tiles_b), tj = (uint32_t)(at % tiles_b), steps = p.a.steps;
    const uint32_t from = (uint32_t)((uint64_t)steps * split / splits), to = (uint32_t)((uint64_t)steps * (split + 1u) / splits);
    const uint32_t last_a = (p.a.rows - 1u) / 16u, last_b = (p.b.rows - 1u) / 16u;
    global_ptr<const v4i> ap[MT], bp[NT];
#pragma unroll
    for (uint32_t q = 0; q < MT; ++q) {              // (tiles beyond the last row stand for the last one: what they give is not stored)
        const uint32_t r = ti * MT + q < last_a ? ti * MT + q : last_a;
        ap[q] = (global_ptr<const v4i>)in_global(p.a.codes + (size_t)r * steps * kMxCodes) + lane;
    }
#pragma unroll
    for (uint32_t q = 0; q < NT; ++q) {
        const uint32_t r = tj * NT + q < last_b ? tj * NT + q : last_b;
        bp[q] = (global_ptr<const v4i>)in_global(p.b.codes + (size_t)r * steps * kMxCodes) + lane;
    }
    const global_ptr<const int> as = (global_ptr<const int>)in_global(p.a.scales + (size_t)(ti * MT / 4u) * steps * kMxScales) + lane;
    const global_ptr<const int> bs = (global_ptr<const int>)in_global(p.b.scales + (size_t)(tj * NT / 4u) * steps * kMxScales) + lane;
    const uint32_t turn_a = ti * MT % 4u * 8u, turn_b = tj * NT % 4u * 8u;               // which bytes of a word of scales are the tiles'
    v4f acc[MT][NT] = {};
    for (uint32_t s = from + wave; s < to; s += kDeep * waves) {
        FewStep<MT, NT> o[kDeep];
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const uint32_t n = s + k * waves < to ? s + k * waves : to - 1u;             // (again, where there are no more)
#pragma unroll
            for (int q = 0; q < NT; ++q) o[k].b[q] = __builtin_nontemporal_load(bp[q] + n * 64u);
            o[k].sb = bs[n * 64u] >> turn_b;
#pragma unroll
            for (int q = 0; q < MT; ++q) o[k].a[q] = ap[q][n * 64u];
            o[k].sa = as[n * 64u] >> turn_a;
        }
#pragma unroll
        for (int k = 0; k < kDeep; ++k) if (s + k * waves < to) few_products<MT, NT>(o[k], acc);
    }
#pragma unroll
    for (int q = 0; q < MT; ++q)
#pragma unroll
        for (int r = 0; r < NT; ++r) sums[wave][q * NT + r][lane] = acc[q][r];
    __syncthreads();
    // Tile f of MT NT belongs to wavefront f % waves; sums are taken in the order of the wavefronts.
    p.out = static_cast<T *>(p.out) + split * p.apart;
    const uint32_t row = ti * 16u * MT + (lane & 15u), col = tj * 16u * NT + (lane >> 4) * 4u;
    for (uint32_t f = wave; f < MT * NT; f += waves) {
        v4f x = sums[0][f][lane];
        for (uint32_t w = 1; w < waves; ++w) x += sums[w][f][lane];
        finish<T>(p, row + f / NT * 16u, col + f % NT * 16u, x);
    }
}

// ---- many rows -----------------------------------------------------------------------------------------------------------
// Operands through LDS: four wavefronts have 64 PA x 64 PB outputs, each a quarter of them.  A step's codes and scales are copied straight to LDS, three steps
// ahead; a wavefront reads the operands of the next half step while it multiplies this one's.  With GROUPS = 2 a block has two such fours, which take
// half of the steps each.  256 x 256 outputs to a block and 128 x 128 read 4.2 and 8.3 bytes of operands for a thousand products (17/32 a value); a step of 128 takes a block of
// the first kind 0.9 us (a third of it waits; the clock falls to 1.6 GHz), of the second 0.39 for both of its groups.
typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));
// What a buffer's loads go by: beyond `bytes` they give 0.
__device__ __forceinline__ rsrc_t buffer_at(const uint8_t *p, uint64_t bytes)
{
    const uint64_t at = (uint64_t)(uintptr_t)p;
    const uint32_t size = bytes < 0xffffffffull ? (uint32_t)bytes : 0xffffffffu;
    return rsrc_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)), (uint32_t)__builtin_amdgcn_readfirstlane((int)size), 0x00020000u};
}
// 16 (4) bytes a lane from its offset `from` to LDS at `to` + 16 (4) * lane.  The compiler does not count these loads: copied() waits.  (The whole offset
// is the lane's: it is that which is checked against the buffer's size.  LDS's place is in m0, which the compiler is told and writes itself; the wait behind
// it is here, since it does not see what reads it.)
__device__ __forceinline__ void copy16(uint32_t to, rsrc_t r, uint32_t from)
{
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(to), "v"(from), "s"(r) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, rsrc_t r, uint32_t from)
{
    asm volatile("s_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"{m0}"(to), "v"(from), "s"(r) : "memory");
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
// N sums of a row, to memory as T, past the caches (4096 x 32064 outputs over 128: 66 us, through them 78).
template <class T, int N>
__device__ __forceinline__ void store_sums(global_ptr<T> to, const float (&x)[N])
{
    typedef typename VecOf<T, N>::type vec;
    vec v;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = (T)x[e];
    __builtin_nontemporal_store(v, (global_ptr<vec>)to);
}

template <class T, int PA, int PB, int GROUPS>
__global__ __launch_bounds__(kBlock * GROUPS, GROUPS == 1 ? 1 : 2) void mx_matmul_lds_k(MxProduct p, uint32_t tiles_a, uint32_t tiles_b, uint32_t splits)
{
    constexpr uint32_t kTilesA = 4 * PA, kTilesB = 4 * PB, kStages = 4;             // tiles of 16 rows to a block
    constexpr uint32_t kCodesA = 0, kCodesB = kTilesA * kMxCodes, kScalesA = kCodesB + kTilesB * kMxCodes, kScalesB = kScalesA + kTilesA / 4 * kMxScales,
                       kStage = kScalesB + kTilesB / 4 * kMxScales;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[GROUPS * kStages * kStage];
    const uint32_t group = __builtin_amdgcn_readfirstlane(threadIdx.x / kBlock), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % 4u, lane = threadIdx.x & 63u;
    // Blocks go to the eight dies in turn: each die gets a run of tiles, eight rows of them by as many columns as that takes.
    uint32_t ti, tj, split;
    {
        constexpr uint32_t kDies = 8, kHigh = 8;
        const uint32_t all = tiles_a * tiles_b * splits, die = blockIdx.x % kDies, each = all / kDies, more = all % kDies;
        const uint32_t n = die * each + (die < more ? die : more) + blockIdx.x / kDies, t = n / splits;
        split = n % splits;
        const uint32_t band = t / (kHigh * tiles_b), in = t % (kHigh * tiles_b), high = tiles_a - band * kHigh < kHigh ? tiles_a - band * kHigh : kHigh;
        ti = band * kHigh + in % high;
        tj = in / high;
    }
    const uint32_t steps = p.a.steps, parts = splits * GROUPS, part = split * GROUPS + group;
    const uint32_t begin = (uint32_t)((uint64_t)steps * part / parts), end = (uint32_t)((uint64_t)steps * (part + 1u) / parts);
    const uint32_t turns = (steps + parts - 1u) / parts;                 // the most steps that a part has
    const uint64_t first_a = (uint64_t)ti * kTilesA, first_b = (uint64_t)tj * kTilesB;                // tiles of 16
    const uint64_t line = (uint64_t)steps * kMxCodes, line_s = (uint64_t)steps * kMxScales;
    const rsrc_t codes_a = buffer_at(p.a.codes + first_a * line, ((p.a.rows + 15u) / 16u - first_a) * line);
    const rsrc_t codes_b = buffer_at(p.b.codes + first_b * line, ((p.b.rows + 15u) / 16u - first_b) * line);
    const rsrc_t scales_a = buffer_at(p.a.scales + first_a / 4u * line_s, ((p.a.rows + 63u) / 64u - first_a / 4u) * line_s);
    const rsrc_t scales_b = buffer_at(p.b.scales + first_b / 4u * line_s, ((p.b.rows + 63u) / 64u - first_b / 4u) * line_s);
    const uint32_t lane16 = lane * 16u, lane4 = lane * 4u, at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds + group * (kStages * kStage);
    // A wavefront copies a quarter of the step's tiles of either operand, and of the PA + PB tiles of scales one or two.
    static_assert(PA == PB, "scales are handed out evenly");
    constexpr uint32_t kMineA = kTilesA / 4, kMineB = kTilesB / 4, kCopies = kMineA + kMineB + PA / 2;
    const bool of_b = PA == 2 && wave >= 2u;
    const uint32_t tile_s = of_b ? wave - 2u : wave, scales_to = (of_b ? kScalesB : kScalesA) + tile_s * kMxScales;
    const rsrc_t scales_1 = of_b ? scales_b : scales_a;
    // the k-th of a wavefront's copies for step s
    const auto copy = [&](uint32_t s, uint32_t k) {
        const uint32_t to = at + s % kStages * kStage;
        if (k < kMineA) {
            const uint32_t t = wave * kMineA + k;
            copy16(to + kCodesA + t * kMxCodes, codes_a, (t * steps + s) * kMxCodes + lane16);
        } else if (k < kMineA + kMineB) {
            const uint32_t t = wave * kMineB + k - kMineA;
            copy16(to + kCodesB + t * kMxCodes, codes_b, (t * steps + s) * kMxCodes + lane16);
        } else if (k == kMineA + kMineB) copy4(to + scales_to, scales_1, (tile_s * steps + s) * kMxScales + lane4);
        else copy4(to + kScalesB + wave * kMxScales, scales_b, (wave * steps + s) * kMxScales + lane4);
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
        const uint8_t *from = lds + group * (kStages * kStage) + s % kStages * kStage;
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
    // A step's copies are issued half behind one barrier and half before the next.
    constexpr uint32_t kEarly = kCopies / 2, kProducts = PA * PB;
    copies(begin, 0, kCopies);
    copies(begin + 1, 0, kCopies);
    copied<kCopies>();
    copies(begin + 2, 0, kEarly);
#pragma unroll
    for (uint32_t k = 0; k < kReads; ++k) read(begin, 0, first, k);
    for (uint32_t s = begin; s < begin + turns; ++s) {
        const bool any = GROUPS == 1 || s < end;                         // (a group may have a step less than the other: it only waits)
        if (any) multiply<PA, PB>(first, acc, [&](uint32_t i) {
#pragma unroll
            for (uint32_t k = i * kReads / kProducts; k < (i + 1) * kReads / kProducts; ++k) read(s, 1, second, k);
#pragma unroll
            for (uint32_t k = i * (kCopies - kEarly) / kProducts; k < (i + 1) * (kCopies - kEarly) / kProducts; ++k) copy(s + 2, kEarly + k);
        });
        // step s + 1 is there, and every wavefront has read step s - 1, whose place the next copies take
        copied<kCopies>();
        if (any) multiply<PA, PB>(second, acc, [&](uint32_t i) {
#pragma unroll
            for (uint32_t k = i * kReads / kProducts; k < (i + 1) * kReads / kProducts; ++k) read(s + 1, 0, first, k);
#pragma unroll
            for (uint32_t k = i * kEarly / kProducts; k < (i + 1) * kEarly / kProducts; ++k) copy(s + 3, k);
        });
    }
    copied<0>();                         // (no copy outlives the block, and no wavefront reads operands any more)
    constexpr uint32_t kKept = PA / GROUPS;                              // sets of 32 rows that a group finishes
    const uint32_t kept = group * kKept;
    v16f (&sum)[kKept][PB] = reinterpret_cast<v16f (&)[kKept][PB]>(acc);
    if constexpr (GROUPS == 2) {         // each group gives the other its sums of the rows that the other finishes
        v4f *const place = reinterpret_cast<v4f *>(lds);
#pragma unroll
        for (uint32_t f = 0; f < kKept * PB * 4u; ++f) {
            const uint32_t q = f / (PB * 4u), r = f / 4u % PB, n = f % 4u;
            const v16f x = group ? acc[q][r] : acc[kKept + q][r];
            place[((group * 4u + wave) * kKept * PB * 4u + f) * 64u + lane] = v4f{x[4 * n], x[4 * n + 1], x[4 * n + 2], x[4 * n + 3]};
        }
        __syncthreads();
#pragma unroll
        for (uint32_t f = 0; f < kKept * PB * 4u; ++f) {
            const uint32_t q = f / (PB * 4u), r = f / 4u % PB, n = f % 4u;
            const v4f y = place[(((1u - group) * 4u + wave) * kKept * PB * 4u + f) * 64u + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[q][r][4 * n + e] = (group ? acc[kKept + q][r][4 * n + e] : acc[q][r][4 * n + e]) + y[e];
        }
        __syncthreads();
    }
    p.out = static_cast<T *>(p.out) + split * p.apart;
    // Results by rows: each wavefront turns its sets of 32 rows round in a part of LDS of its own, so that what a wavefront stores are whole lines (4096 x 32064
    // outputs over 4096: 290 us; stored from where the products leave them, eight bytes to a row, 810).
    constexpr uint32_t kWide = 32 * PB, kPitch = kWide + 4;              // floats to a row
    static_assert(GROUPS * 4 * 32 * kPitch * sizeof(float) <= sizeof(lds), "a part of LDS for each wavefront");
    float *const own = reinterpret_cast<float *>(lds) + (group * 4u + wave) * 32u * kPitch;
    const uint32_t row0 = ((uint32_t)first_a + (half_a * PA + kept) * 2u) * 16u, col0 = ((uint32_t)first_b + half_b * PB * 2u) * 16u;
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
    for (uint32_t q = 0; q < kKept; ++q) {
#pragma unroll
        for (uint32_t r = 0; r < PB; ++r)
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n)
                *reinterpret_cast<v4f *>(own + (lane & 31u) * kPitch + r * 32u + n * 8u + (lane >> 5) * 4u) =
                    v4f{sum[q][r][4 * n], sum[q][r][4 * n + 1], sum[q][r][4 * n + 2], sum[q][r][4 * n + 3]};
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

// ---- splits ---------------------------------------------------------------------------------------------------------------
// The parts' sums, in their order, and what else a result has: a thread to four columns of a row.
template <class T>
__global__ __launch_bounds__(kBlock) void mx_join_k(MxProduct p, uint64_t first, uint32_t splits, uint32_t wide)
{
    const uint64_t at = (first + blockIdx.x) * kBlock + threadIdx.x;
    const uint32_t row = (uint32_t)(at / wide), col = (uint32_t)(at % wide) * 4u;
    if (row >= p.a.rows) return;
    const global_ptr<const v4f> from = (global_ptr<const v4f>)in_global(p.partial + ((size_t)row * wide * 4u + col));
    v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t k = 0; k < splits; k += 4u) {      // (four on their way at once)
        v4f y[4];
#pragma unroll
        for (uint32_t j = 0; j < 4u; ++j) y[j] = from[(size_t)(k + j < splits ? k + j : splits - 1u) * (p.apart / 4u)];
#pragma unroll
        for (uint32_t j = 0; j < 4u; ++j) if (k + j < splits) x += y[j];
    }
    finish<T>(p, row, col, x);
}
// A product whose steps `splits` blocks share: `parts` takes it as one of 32-bit results into the scratch, a part behind the other.
template <class T, class Parts, class Whole>
static void shared_by(const LaunchCtx &lc, const MxProduct &p, uint32_t splits, Parts parts, Whole whole)
{
    if (splits == 1u) {
        whole(p);
        return;
    }
    const uint32_t wide = (p.b.rows + 3u) / 4u;
    MxProduct q = p;
    q.out = p.partial;
    q.bias = nullptr;
    q.accumulate = false;
    q.stride = (int64_t)wide * 4;
    q.apart = (size_t)p.a.rows * wide * 4u;
    parts(q);
    MxProduct j = p;
    j.apart = q.apart;
    in_launches(((uint64_t)p.a.rows * wide + kBlock - 1u) / kBlock, [&](uint64_t first, uint32_t n) { launch(mx_join_k<T>, dim3(n), dim3(kBlock), lc.stream, j, first, splits, wide); });
}

// How many blocks share a tile's steps: the power of two whose estimate is the shortest, from what was measured: 3 us for a round of 256 blocks to begin and end,
// `step` us for each of its steps; for the parts' pass 3 us, and 2 us for a million of their elements.  (512 x 1024 outputs over 12 544: 24.8 us
// without splits, 15.5 with the four that this takes; 256 x 256 over 65 536 104 and 21.4; 2048 x 2048 over 4096 14.7 with none.  Parts that the last block of a tile to come adds
// up, through memory and counts, took 25 us for the first.  Its estimate is 15.2, but 8.0 for the product, which takes 12.3, and 7.2 for the parts' pass, which takes
// 4.0: that every die fetches all of a, 36 MB together where the operands have 10, is not in it.)
static uint32_t splits_for(const MxProduct &p, uint64_t tiles, double step)
{
    const uint64_t part = (uint64_t)p.a.rows * ((p.b.rows + 3u) / 4u * 4u);
    uint32_t best = 1;
    double least = 0.0;
    for (uint32_t n = 1; n <= 64u && n <= p.a.steps && (n == 1u || n * part <= kMxPartial); n *= 2u) {
        const double t = (double)((tiles * n + 255u) / 256u) * (3.0 + step * ((p.a.steps + n - 1u) / n)) + (n == 1u ? 0.0 : 3.0 + (double)(n * part) * 2e-6);
        if (n == 1u || t < least) {
            least = t;
            best = n;
        }
    }
    return best;
}
template <class T, int MT, int NT>
static void few_of(const LaunchCtx &lc, const MxProduct &p)
{
    const uint64_t tiles_b = (p.b.rows + 16u * NT - 1u) / (16u * NT), tiles = (p.a.rows + 16u * MT - 1u) / (16u * MT) * tiles_b;
    const uint32_t waves = p.a.steps < kFewWaves ? p.a.steps : kFewWaves, splits = splits_for(p, tiles, 0.04);
    const auto go = [&](auto k, const MxProduct &q) {
        in_launches(tiles * splits, [&](uint64_t first, uint32_t n) { launch(k, dim3(n), dim3(waves * 64u), lc.stream, q, first, (uint32_t)tiles_b, splits); });
    };
    shared_by<T>(lc, p, splits, [&](const MxProduct &q) { go(mx_matmul_few_k<float, MT, NT>, q); }, [&](const MxProduct &q) { go(mx_matmul_few_k<T, MT, NT>, q); });
}
template <class T, int PAIRS, int GROUPS>
static bool lds_of(const LaunchCtx &lc, const MxProduct &p, uint64_t least)
{
    constexpr uint32_t kSide = 64 * PAIRS;
    const uint64_t ta = (p.a.rows + kSide - 1u) / kSide, tb = (p.b.rows + kSide - 1u) / kSide;
    if (ta * tb < least || ta * tb >= (1u << 22) || p.a.steps >= (1u << 16)) return false;
    const uint32_t splits = PAIRS == 4 ? 1u : splits_for(p, ta * tb, 0.2);
    const auto go = [&](auto k, const MxProduct &q) {
        launch(k, dim3((uint32_t)(ta * tb) * splits), dim3(kBlock * GROUPS), lc.stream, q, (uint32_t)ta, (uint32_t)tb, splits);
    };
    shared_by<T>(lc, p, splits, [&](const MxProduct &q) { go(mx_matmul_lds_k<float, PAIRS, PAIRS, GROUPS>, q); },
                 [&](const MxProduct &q) { go(mx_matmul_lds_k<T, PAIRS, PAIRS, GROUPS>, q); });
    return true;
}
// Which form takes a product (us, 16-bit results):
//   256 x 256 outputs to a block    where that makes 110 blocks: 2048 x 2560 (80) over 4096 32 and 25 by the next form, 3328 x 2560 (130) over 2048 23 and 26
//   128 x 128                       from 65 rows on, with more to do than 4800 steps of 64 x 16 outputs: 128 x 4096 over 4096 (16 384) 11.3, and 14 to 20 by the
//                                   next form, 1024 x 1024 over 1024 (8192) 6.7 and 8.6, over 512 (4096) 6.0 and 5.3, 256 x 1000 over 2048 (4032) 8.7 and 6.2, 512 x
//                                   512 over 512 (1024) 5.6 and 3.3
//   straight from memory            64 columns to a block above 12 800 of them (more than 200 such blocks: 1 x 32064 over 4096 13.6, 5 TB/s), else 16, or for up to 16 rows 32
//                                   above 6400: 16 x 4096 over 4096 7.0, and 10 with 64
// Both sides of the border of 12 800, over 4096 (three sets of operands in turn, which the last-level cache holds): 16 rows by 12 736 and 12 800 (400 blocks of 32 columns) 8.0 to 8.7
// and by 12 864 (201 of 64) 8.9; 17, 32 and 64 rows by 12 800 (800 of 16) 11.2, 11.5 and 15.9, by 12 864 9.1, 9.2 and 10.7: for more than 16 rows it lies too high.  (By 8192: 7.3, 7.7
// and 9.1.)
// The count of 256 x 256 blocks takes them as full: 65, 128, 192 and 256 rows by 32 064 over 4096, 126 blocks that are a quarter to wholly filled, take 31.4, 35.1, 35.2
// and 35.3, where the bytes are 14 to 17's; 512 x 16 384 27.7, 32 064 x 128 29.6.
template <class T>
static void matmul_of(const LaunchCtx &lc, const MxProduct &p)
{
    const uint64_t much = (uint64_t)((p.a.rows + 63u) / 64u) * ((p.b.rows + 15u) / 16u) * p.a.steps;
    if (p.a.rows > 64u && much > 4800u && (lds_of<T, 4, 1>(lc, p, 110u) || lds_of<T, 2, 2>(lc, p, 1u))) return;
    const bool wide = p.b.rows > 64u * 200u;
    if (p.a.rows <= 16u) {
        if (wide) few_of<T, 1, 4>(lc, p);
        else if (p.b.rows > 32u * 200u) few_of<T, 1, 2>(lc, p);
        else few_of<T, 1, 1>(lc, p);
    } else if (p.a.rows <= 32u) {
        if (wide) few_of<T, 2, 4>(lc, p);
        else few_of<T, 2, 1>(lc, p);
    } else {
        if (wide) few_of<T, 4, 4>(lc, p);
        else few_of<T, 4, 1>(lc, p);
    }
}
void launch_mx_matmul(const LaunchCtx &lc, int dtype, const MxProduct &p)
{
    if (dtype == MC_DTYPE_F32) matmul_of<float>(lc, p);
    else if (dtype == MC_DTYPE_BF16) matmul_of<__bf16>(lc, p);
    else matmul_of<_Float16>(lc, p);
}

}  // namespace mc
