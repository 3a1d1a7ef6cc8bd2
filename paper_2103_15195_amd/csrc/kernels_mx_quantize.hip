// Matrices to microscaled 4-bit floating point.
//
// A stream: what bounds it is the memory's rate.  A lane loads 16 bytes of a row, eight or four elements, so that a row's 128 columns are 16 or 32
// lanes and a block of 32 four or eight of them, whose largest magnitude takes two or three exchanges between neighbours.  Along the columns a lane
// holds all 32 rows of its block in registers: no exchange at all, and the rows' blocks are taken from the same registers.
#include "mx_internal.h"

namespace mc {

typedef uint32_t codes4 __attribute__((ext_vector_type(4)));
typedef uint16_t halves __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <class T> constexpr int kHas = 16 / (int)sizeof(T);             // elements of a lane
template <class T> constexpr uint32_t kRowLanes = kMxStep / kHas<T>;     // lanes to a row's 128 columns
template <class T> constexpr uint32_t kBlockLanes = kMxBlock / kHas<T>;  // lanes to a block of 32

__device__ __forceinline__ float float_of(uint32_t bits) { return __builtin_bit_cast(float, bits); }

// ---- a lane's part of a row: WORDS words ----------------------------------------------------------------------------------
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
template <int WORDS> struct Words;
template <> struct Words<2> { typedef words2 type; };
template <> struct Words<4> { typedef codes4 type; };
template <class T, int WORDS>
__device__ __forceinline__ typename Words<WORDS>::type load_words(const T *row, uint32_t col, uint32_t cols, bool full)
{
    typedef typename Words<WORDS>::type vec;
    typedef vec vec_any __attribute__((aligned(2)));
    typedef vec vec_word __attribute__((aligned(4)));
    if (full) {
        if constexpr (sizeof(T) == 4) return *(global_ptr<const vec_word>)(in_global(row) + col);
        else return *(global_ptr<const vec_any>)(in_global(row) + col);
    }
    vec w = {};
#pragma unroll
    for (int e = 0; e < 4 * WORDS / (int)sizeof(T); ++e) {
        if (col + e >= cols) continue;
        if constexpr (sizeof(T) == 4) w[e] = __builtin_bit_cast(uint32_t, in_global(row)[col + e]);
        else w[e / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, in_global(row)[col + e]) << (16 * (e % 2));
    }
    return w;
}
template <class T, int WORDS>
__device__ __forceinline__ void store_words(T *row, uint32_t col, uint32_t cols, typename Words<WORDS>::type w)
{
    typedef typename Words<WORDS>::type vec;
    typedef vec vec_any __attribute__((aligned(2)));
    typedef vec vec_word __attribute__((aligned(4)));
    constexpr int kEach = 4 * WORDS / (int)sizeof(T);
    if (col + kEach <= cols) {
        if constexpr (sizeof(T) == 4) __builtin_nontemporal_store(w, (global_ptr<vec_word>)(in_global(row) + col));
        else __builtin_nontemporal_store(w, (global_ptr<vec_any>)(in_global(row) + col));
        return;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (col + e >= cols) continue;
        if constexpr (sizeof(T) == 4) in_global(row)[col + e] = float_of(w[e]);
        else in_global(row)[col + e] = __builtin_bit_cast(T, (uint16_t)(w[e / 2] >> (16 * (e % 2))));
    }
}
// Magnitudes compare as whole numbers, and so do two of 16 bits in a word.
template <class T>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t w)
{
    if constexpr (sizeof(T) == 4) {
        w &= 0x7fffffffu;
        return a > w ? a : w;
    } else {
        const halves x = __builtin_bit_cast(halves, a), y = __builtin_bit_cast(halves, w & 0x7fff7fffu);
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
    }
}
// A magnitude of T's, of 16 bits in the low half, as a 32-bit one's bits.
template <class T>
__device__ __forceinline__ uint32_t bits_of(uint32_t a)
{
    if constexpr (std::is_same_v<T, __bf16>) return a << 16;
    else if constexpr (std::is_same_v<T, _Float16>) return __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)a));
    else return a;
}
// Two elements to codes in byte AT of a word.
template <class T, int AT>
__device__ __forceinline__ uint32_t pair_codes(uint32_t old, uint32_t w, float p)
{
    if constexpr (std::is_same_v<T, __bf16>) return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, w), p, AT);
    else return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(f16x2, w), p, AT);
}

// ---- scales ------------------------------------------------------------------------------------------------------------
// The scale's byte of a block whose largest magnitude has these bits.  fraction * 2^E with a fraction up to 1.75 gets 2^(E - 2), of which it is up to 7
// times as much; a larger one 2^(E - 1).  (Of normal values 1.25 percent of the square are lost, with 2^(E - 2) for all 1.32, with 2^(E - 1)
// wherever 6 would be exceeded 1.33; of uniform ones 0.98, 2.07 and 0.98.)
__device__ __forceinline__ uint32_t scale_of(uint32_t top)
{
    const int32_t e = (int32_t)((top + 0x1fffffu) >> 23) - 2;            // (fractions above 1.75 carry)
    return top >= 0x7f800000u ? 255u : e < 0 ? 0u : (uint32_t)e;
}
__device__ __forceinline__ float power_of(uint32_t scale) { return __builtin_bit_cast(float, scale ? scale << 23 : 0x00400000u); }

template <int CTRL>
__device__ __forceinline__ uint32_t neighbour(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false); }
constexpr int kOther = 0xB1, kOtherPair = 0x4E, kMirrored = 0x141, kMirrored16 = 0x140;       // lane ^ 1, ^ 2, ^ 7, ^ 15
// The largest of the lanes that a block of 32 columns is spread over.
template <uint32_t LANES>
__device__ __forceinline__ uint32_t block_max(uint32_t x)
{
    uint32_t y = neighbour<kOther>(x);
    x = x > y ? x : y;
    y = neighbour<kOtherPair>(x);
    x = x > y ? x : y;
    if constexpr (LANES >= 8) {
        y = neighbour<kMirrored>(x);
        x = x > y ? x : y;
    }
    if constexpr (LANES == 16) {
        y = neighbour<kMirrored16>(x);
        x = x > y ? x : y;
    }
    return x;
}

// ---- a lane's codes --------------------------------------------------------------------------------------------------------
// The block's scale, and the lane's codes, four bits an element.
template <class T, int WORDS>
__device__ __forceinline__ uint32_t row_codes(typename Words<WORDS>::type w, uint32_t &scale)
{
    constexpr uint32_t kEach = 4 * WORDS / sizeof(T);
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < WORDS; ++k) top = larger<T>(top, w[k]);
    if constexpr (sizeof(T) == 2) top = (top & 0xffffu) > top >> 16 ? top & 0xffffu : top >> 16;
    scale = scale_of(block_max<kMxBlock / kEach>(bits_of<T>(top)));
    const float p = power_of(scale);
    uint32_t c = 0;
    if constexpr (sizeof(T) == 2) {
        c = pair_codes<T, 0>(c, w[0], p);
        c = pair_codes<T, 1>(c, w[1], p);
        if constexpr (WORDS == 4) {
            c = pair_codes<T, 2>(c, w[2], p);
            c = pair_codes<T, 3>(c, w[3], p);
        }
    } else {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, float_of(w[0]), float_of(w[1]), p, 0);
        if constexpr (WORDS == 4) c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, float_of(w[2]), float_of(w[3]), p, 1);
    }
    return scale == 255u ? 0u : c;
}
// What codes stand for, within the range of T.
template <class T, int WORDS>
__device__ __forceinline__ typename Words<WORDS>::type values_of(uint32_t c, uint32_t scale)
{
    constexpr float most = std::is_same_v<T, _Float16> ? 65504.0f : std::is_same_v<T, __bf16> ? 0x1.fep127f : 0x1.fffffep127f;
    const float p = power_of(scale), keep = scale == 255u ? __builtin_nanf("") : 1.0f;
    const f32x2 x[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, p, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, p, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, p, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, p, 3)};
    typename Words<WORDS>::type w;
#pragma unroll
    for (int k = 0; k < 2 * WORDS / (int)sizeof(T); ++k) {
        const float a = __builtin_amdgcn_fmed3f(x[k][0], -most, most) * keep, b = __builtin_amdgcn_fmed3f(x[k][1], -most, most) * keep;
        if constexpr (sizeof(T) == 4) {
            w[2 * k] = __builtin_bit_cast(uint32_t, a);
            w[2 * k + 1] = __builtin_bit_cast(uint32_t, b);
        } else if constexpr (std::is_same_v<T, __bf16>) {
            w[k] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
        } else {
            w[k] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
        }
    }
    return w;
}
__device__ __forceinline__ size_t codes_at(const MxView &m, uint32_t row, uint32_t step, uint32_t group)
{
    return (((size_t)(row / 16u) * m.steps + step) * 64u + group * 16u + row % 16u) * 16u;
}
__device__ __forceinline__ size_t scales_at(const MxView &m, uint32_t row, uint32_t step, uint32_t group)
{
    return (((size_t)(row / 64u) * m.steps + step) * 64u + group * 16u + row % 16u) * 4u;
}
// A lane's codes of one row; `lane`: its place in the row.
template <class T>
__device__ __forceinline__ void put_codes(const MxView &m, uint32_t row, uint32_t step, uint32_t lane, uint32_t c)
{
    const global_ptr<uint8_t> to = in_global(m.codes) + codes_at(m, row, step, lane / kBlockLanes<T>) + lane % kBlockLanes<T> * (16u / kBlockLanes<T>);
    if constexpr (sizeof(T) == 2) *(global_ptr<uint32_t>)to = c;
    else *(global_ptr<uint16_t>)to = (uint16_t)c;
}

// ---- along the rows ----------------------------------------------------------------------------------------------------
// 64 rows by 128 columns to a block.  A thread has the same columns of the same row of each of the four tiles of 16 rows, so that it has a word of scales
// together.
template <class T> constexpr uint32_t kRowsThreads = 16u * kRowLanes<T>;
template <class T, bool VALUES>
__global__ __launch_bounds__(kRowsThreads<T>) void mx_rows_k(MxSource s, uint64_t first, uint32_t steps)
{
    const uint64_t at = first + blockIdx.x;
    const uint32_t step = (uint32_t)(at % steps), lane = threadIdx.x % kRowLanes<T>, col = step * kMxStep + lane * kHas<T>;
    const uint32_t row0 = (uint32_t)(at / steps) * 64u + threadIdx.x / kRowLanes<T>;
    const T *x = static_cast<const T *>(s.x);
    const bool full = step * kMxStep + kMxStep <= s.cols;                // (of columns)
    codes4 w[4];
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) {
        w[q] = codes4{0u, 0u, 0u, 0u};
        if (row0 + q * 16u < s.rows) w[q] = load_words<T, 4>(x + (int64_t)(row0 + q * 16u) * s.stride, col, s.cols, full);
    }
    uint32_t scales = 0, scale;
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) {
        const uint32_t row = row0 + q * 16u, c = row_codes<T, 4>(w[q], scale);
        scales |= scale << (8u * q);
        if (row >= s.rows) continue;
        if (s.by_rows.codes) put_codes<T>(s.by_rows, row, step, lane, c);
        if constexpr (VALUES) store_words<T, 4>(static_cast<T *>(s.values) + (int64_t)row * s.values_stride, col, s.cols, values_of<T, 4>(c, scale));
    }
    if (s.by_rows.codes && lane % kBlockLanes<T> == 0 && row0 < s.rows) {
        const global_ptr<uint8_t> to = in_global(s.by_rows.scales) + scales_at(s.by_rows, row0, step, lane / kBlockLanes<T>);
        if (row0 + 48u < s.rows) *(global_ptr<uint32_t>)to = scales;
        else for (uint32_t q = 0; q < 4; ++q) if (row0 + q * 16u < s.rows) to[q] = (uint8_t)(scales >> (8u * q));
    }
}

// ---- along the columns, and along the rows with them -----------------------------------------------------------------------
// A lane has WORDS words of 32 rows in registers: the columns' blocks without any exchange, and the rows' from the same registers.  A wavefront has 128 columns of as
// many sets of 32 rows as its lanes make.
template <class T, int WORDS, bool ROWS, bool VALUES>
__global__ __launch_bounds__(kBlock) void mx_cols_k(MxSource s, uint64_t first, uint64_t tiles, uint32_t across)
{
    constexpr uint32_t kEach = 4 * WORDS / sizeof(T), kInRow = kMxStep / kEach, kSets = 64u / kInRow, kHigh = kSets * 32u;      // elements of a lane, lanes to a row, rows
    const uint64_t at = (first + blockIdx.x) * (kBlock / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (at >= tiles) return;
    const uint32_t step = (uint32_t)(at % across), lane = threadIdx.x & 63u, in_row = lane % kInRow;
    const uint32_t top = (uint32_t)(at / across) * kHigh, row0 = top + lane / kInRow * 32u, col = step * kMxStep + in_row * kEach;
    const T *x = static_cast<const T *>(s.x);
    typename Words<WORDS>::type w[32];
    if (top + kHigh <= s.rows && step * kMxStep + kMxStep <= s.cols) {
        const T *p = x + (int64_t)row0 * s.stride;
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) w[i] = load_words<T, WORDS>(p + (int64_t)i * s.stride, col, s.cols, true);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) {
            w[i] = {};
            if (row0 + i < s.rows) w[i] = load_words<T, WORDS>(x + (int64_t)(row0 + i) * s.stride, col, s.cols, false);
        }
    }
    // ---- columns: row0 is a multiple of 32 and the rows are the transposed matrix's columns
    const uint32_t group = row0 % kMxStep / 32u;
    const MxView &m = s.by_cols;
#pragma unroll
    for (uint32_t k = 0; k < WORDS; ++k) {
        uint32_t most = 0;
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) most = larger<T>(most, w[i][k]);
#pragma unroll
        for (uint32_t h = 0; h < 4u / sizeof(T); ++h) {                  // a word has one column, or two
            const uint32_t c = col + k * (4u / sizeof(T)) + h;
            const uint32_t scale = scale_of(bits_of<T>(sizeof(T) == 2 ? (h ? most >> 16 : most & 0xffffu) : most));
            const float p = power_of(scale);
            codes4 codes = {0u, 0u, 0u, 0u};
#pragma unroll
            for (uint32_t i = 0; i < 32; i += 8) {
                uint32_t o = 0;
                if constexpr (sizeof(T) == 2) {
                    const uint32_t pick = h ? 0x07060302u : 0x05040100u;                     // the same half of two words
                    o = pair_codes<T, 0>(o, __builtin_amdgcn_perm(w[i + 1][k], w[i][k], pick), p);
                    o = pair_codes<T, 1>(o, __builtin_amdgcn_perm(w[i + 3][k], w[i + 2][k], pick), p);
                    o = pair_codes<T, 2>(o, __builtin_amdgcn_perm(w[i + 5][k], w[i + 4][k], pick), p);
                    o = pair_codes<T, 3>(o, __builtin_amdgcn_perm(w[i + 7][k], w[i + 6][k], pick), p);
                } else {
#define MC_PAIR(n) o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, float_of(w[i + 2 * n][k]), float_of(w[i + 2 * n + 1][k]), p, n)
                    MC_PAIR(0); MC_PAIR(1); MC_PAIR(2); MC_PAIR(3);
#undef MC_PAIR
                }
                codes[i / 8] = scale == 255u ? 0u : o;
            }
            if (c < s.cols) {
                *(global_ptr<codes4>)(in_global(m.codes) + codes_at(m, c, row0 / kMxStep, group)) = codes;
                in_global(m.scales)[scales_at(m, c, row0 / kMxStep, group) + c / 16u % 4u] = (uint8_t)scale;
            }
        }
    }
    if constexpr (ROWS || VALUES) {
        // 32 rows are two tiles of 16, and of one tile's 64 rows of scales.  Lanes that share a word of codes give theirs to the first of them.
        constexpr uint32_t kShare = 8u / kEach, kInBlock = kMxBlock / kEach;
        const uint32_t block = in_row / kInBlock;
        global_ptr<uint8_t> codes = {}, scales = {};
        if constexpr (ROWS) {
            codes = in_global(s.by_rows.codes) + codes_at(s.by_rows, row0, step, block) + in_row % kInBlock * (kEach / 2u);
            scales = in_global(s.by_rows.scales) + scales_at(s.by_rows, row0, step, block) + row0 / 16u % 4u;
        }
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) {
            uint32_t both = 0;                           // the scales of rows i and i + 16 lie side by side
#pragma unroll
            for (uint32_t j = i; j < 32; j += 16u) {
                asm volatile("" : "+v"(w[j]));           // (or the magnitudes that the columns took from it are kept, in as many registers again)
                uint32_t scale, c = row_codes<T, WORDS>(w[j], scale);
                both |= scale << (j / 16u * 8u);
                const uint32_t mine = c;
                if constexpr (kShare >= 2u) c |= neighbour<kOther>(c) << (4u * kEach);
                if constexpr (kShare == 4u) c |= neighbour<kOtherPair>(c) << (8u * kEach);
                if (row0 + j >= s.rows) continue;
                if constexpr (ROWS) {
                    if (in_row % kShare == 0) *(global_ptr<uint32_t>)(codes + (j / 16u ? (size_t)s.by_rows.steps * kMxCodes : 0u) + i * 16u) = c;
                }
                if constexpr (VALUES) store_words<T, WORDS>(static_cast<T *>(s.values) + (int64_t)(row0 + j) * s.values_stride, col, s.cols, values_of<T, WORDS>(mine, scale));
            }
            if constexpr (ROWS) {
                if (in_row % kInBlock == 0) {
                    if (row0 + i + 16u < s.rows) *(global_ptr<uint16_t>)(scales + i * 4u) = (uint16_t)both;
                    else if (row0 + i < s.rows) scales[i * 4u] = (uint8_t)both;
                }
            }
        }
    }
}

template <class T>
static void quantize_of(const LaunchCtx &lc, const MxSource &s)
{
    const uint32_t steps = (s.cols + kMxStep - 1u) / kMxStep;
    if (s.by_cols.codes) {
        // (whole steps of 128 rows: the padding along the transposed matrix's rows is written too)
        constexpr int W = 2;                       // (four: 4096 x 8192 of 16 bits in both directions 33 us, two 31; along the columns alone 20 and 17)
        const uint64_t tiles = (uint64_t)((s.rows + kMxStep - 1u) / kMxStep) * (kMxStep / (64u * W / (128u / 4u * sizeof(T)) * 32u)) * steps;
        auto k = s.by_rows.codes ? (s.values ? mx_cols_k<T, W, true, true> : mx_cols_k<T, W, true, false>) : s.values ? mx_cols_k<T, W, false, true> : mx_cols_k<T, W, false, false>;
        in_launches((tiles + kBlock / 64 - 1) / (kBlock / 64), [&](uint64_t first, uint32_t n) { launch(k, dim3(n), dim3(kBlock), lc.stream, s, first, tiles, steps); });
    } else {
        auto k = s.values ? mx_rows_k<T, true> : mx_rows_k<T, false>;
        in_launches((uint64_t)((s.rows + 63u) / 64u) * steps, [&](uint64_t first, uint32_t n) { launch(k, dim3(n), dim3(kRowsThreads<T>), lc.stream, s, first, steps); });
    }
}
void launch_mx_quantize(const LaunchCtx &lc, int dtype, const MxSource &s)
{
    if (dtype == MC_DTYPE_F32) quantize_of<float>(lc, s);
    else if (dtype == MC_DTYPE_BF16) quantize_of<__bf16>(lc, s);
    else quantize_of<_Float16>(lc, s);
}

}  // namespace mc
