// Matrices to microscaled 4-bit floating point.
//
// A lane quantises a whole block of 32 values, so that its largest magnitude needs no other lane, and its 16 bytes of codes are one
// store; lane g * 16 + r has the block g of row r of a tile, which is where the layout has it: a wavefront's codes are 1024 bytes
// in a row.
#include "mx_internal.h"

namespace mc {

typedef uint32_t codes4 __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));

// The scale's byte of a block whose largest magnitude has these bits.  fraction * 2^E with a fraction up to 1.75 gets 2^(E - 2), of which it is up to 7
// times as much; a larger one 2^(E - 1).  (Of normal values 1.25 percent of the square are lost, with 2^(E - 2) for all 1.32, with 2^(E - 1)
// wherever 6 would be exceeded 1.33; of uniform ones 0.98, 2.07 and 0.98.)
__device__ __forceinline__ uint32_t scale_of(uint32_t top)
{
    if (top >= 0x7f800000u) return 255u;
    const int32_t e = (int32_t)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u);
    return e < 0 ? 0u : (uint32_t)e;
}
__device__ __forceinline__ float power_of(uint32_t scale) { return __builtin_bit_cast(float, scale ? scale << 23 : 0x00400000u); }

// 32 values to their codes, and the scale's byte.
__device__ __forceinline__ codes4 quantised(const float (&x)[32], uint32_t &scale)
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
        const uint32_t a = __builtin_bit_cast(uint32_t, x[e]) & 0x7fffffffu;
        top = a > top ? a : top;
    }
    scale = scale_of(top);
    codes4 c = {0u, 0u, 0u, 0u};
    if (scale == 255u) return c;
    const float p = power_of(scale);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[8 * k], x[8 * k + 1], p, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[8 * k + 2], x[8 * k + 3], p, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[8 * k + 4], x[8 * k + 5], p, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[8 * k + 6], x[8 * k + 7], p, 3);
        c[k] = w;
    }
    return c;
}
// What codes stand for, within the range of T.
template <class T>
__device__ __forceinline__ void values_of(codes4 c, uint32_t scale, float (&x)[32])
{
    const float p = scale == 255u ? __builtin_nanf("") : power_of(scale);
    constexpr float most = std::is_same_v<T, _Float16> ? 65504.0f : std::is_same_v<T, __bf16> ? 0x1.fep127f : 0x1.fffffep127f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t code = c[k] >> (4 * e) & 15u, size = code & 7u;
            // twice the value: 0 1 2 3 4 6 8 12, as a nibble each
            const float v = (float)(int32_t)(0xC8643210u >> (4 * size) & 15u) * 0.5f * p;
            const float held = v > most ? most : v;                 // (NaN passes)
            x[8 * k + e] = code & 8u ? -held : held;
        }
    }
}
__device__ __forceinline__ void put(const MxView &m, uint32_t tile, uint32_t step, uint32_t lane, codes4 c, uint32_t scale)
{
    *(global_ptr<codes4>)(in_global(m.codes) + ((size_t)tile * m.steps + step) * kMxCodes + lane * 16u) = c;
    in_global(m.scales)[(((size_t)(tile / 4u) * m.steps + step) * 64u + lane) * 4u + tile % 4u] = (uint8_t)scale;
}
template <class T, int N>
__device__ __forceinline__ void load_row(const T *row, int32_t from, int32_t cols, float (&x)[32])
{
#pragma unroll
    for (int k = 0; k < 32 / N; ++k) {
        float y[N];
        load_some<N, T, false>(in_global(row), from + N * k, 0, cols, y);
#pragma unroll
        for (int e = 0; e < N; ++e) x[N * k + e] = y[e];
    }
}
template <class T, int N>
__device__ __forceinline__ void store_row(T *row, int32_t from, int32_t cols, const float (&x)[32])
{
#pragma unroll
    for (int k = 0; k < 32 / N; ++k) {
        float y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = x[N * k + e];
        store_some<N, T>(in_global(row), from + N * k, 0, cols, y);
    }
}

// Along the rows: a wavefront to a tile of 16 rows by 128 columns.
template <class T, bool VALUES>
__global__ __launch_bounds__(kBlock) void mx_rows_k(MxSource s, uint64_t first, uint64_t tiles)
{
    constexpr int N = 16 / (int)sizeof(T);
    const uint64_t t = (first + blockIdx.x) * (kBlock / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (t >= tiles) return;
    const uint32_t steps = (s.cols + kMxStep - 1u) / kMxStep, tile = (uint32_t)(t / steps), step = (uint32_t)(t % steps);
    const uint32_t lane = threadIdx.x & 63u, row = tile * 16u + (lane & 15u);
    const int32_t from = (int32_t)(step * kMxStep + (lane >> 4) * kMxBlock);
    if (row >= s.rows) return;
    float x[32];
    load_row<T, N>(static_cast<const T *>(s.x) + (int64_t)row * s.stride, from, (int32_t)s.cols, x);
    uint32_t scale;
    const codes4 c = quantised(x, scale);
    if (s.by_rows.codes) put(s.by_rows, tile, step, lane, c, scale);
    if constexpr (VALUES) {
        values_of<T>(c, scale, x);
        store_row<T, N>(static_cast<T *>(s.values) + (int64_t)row * s.values_stride, from, (int32_t)s.cols, x);
    }
}

// Along the columns too: a block has 128 rows by 128 columns in LDS, of which it takes tiles of either direction.
template <class T, bool ROWS, bool VALUES>
__global__ __launch_bounds__(kBlock) void mx_cols_k(MxSource s, uint64_t first)
{
    constexpr int N = 16 / (int)sizeof(T);
    constexpr uint32_t kSide = 128, kPitch = kSide + 16 / sizeof(T);
    __shared__ T held[kSide * kPitch];
    const uint32_t across = (s.cols + kSide - 1u) / kSide;
    const uint32_t br = (uint32_t)((first + blockIdx.x) / across), bc = (uint32_t)((first + blockIdx.x) % across), r0 = br * kSide, c0 = bc * kSide;
    {
        constexpr uint32_t wide = kSide / N;
        for (uint32_t i = threadIdx.x; i < kSide * wide; i += kBlock) {
            const uint32_t r = i / wide, c = i % wide * N;
            float y[N];
            if (r0 + r < s.rows) load_some<N, T, false>(in_global(static_cast<const T *>(s.x) + (int64_t)(r0 + r) * s.stride), (int32_t)(c0 + c), 0, (int32_t)s.cols, y);
            else for (int e = 0; e < N; ++e) y[e] = 0.0f;
#pragma unroll
            for (int e = 0; e < N; ++e) held[r * kPitch + c + e] = (T)y[e];
        }
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, in16 = lane & 15u, group = lane >> 4;
    for (uint32_t k = wave; k < kSide / 16u; k += kBlock / 64u) {
        float x[32];
        uint32_t scale;
        if constexpr (ROWS || VALUES) {
            const uint32_t r = k * 16u + in16;
            if (r0 + r < s.rows) {
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = (float)held[r * kPitch + group * 32u + e];
                const codes4 c = quantised(x, scale);
                if constexpr (ROWS) put(s.by_rows, br * 8u + k, bc, lane, c, scale);
                if constexpr (VALUES) {
                    values_of<T>(c, scale, x);
                    store_row<T, N>(static_cast<T *>(s.values) + (int64_t)(r0 + r) * s.values_stride, (int32_t)(c0 + group * 32u), (int32_t)s.cols, x);
                }
            }
        }
        const uint32_t col = k * 16u + in16;
        if (c0 + col < s.cols) {
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = (float)held[(group * 32u + e) * kPitch + col];
            const codes4 c = quantised(x, scale);
            put(s.by_cols, bc * 8u + k, br, lane, c, scale);
        }
    }
}

template <class T>
static void quantize_of(const LaunchCtx &lc, const MxSource &s)
{
    const uint32_t steps = (s.cols + kMxStep - 1u) / kMxStep;
    if (s.by_cols.codes) {
        const uint64_t blocks = (uint64_t)((s.rows + 127u) / 128u) * ((s.cols + 127u) / 128u);
        auto k = s.by_rows.codes ? (s.values ? mx_cols_k<T, true, true> : mx_cols_k<T, true, false>) : s.values ? mx_cols_k<T, false, true> : mx_cols_k<T, false, false>;
        in_launches(blocks, [&](uint64_t first, uint32_t n) { launch(k, dim3(n), dim3(kBlock), lc.stream, s, first); });
    } else {
        const uint64_t tiles = (uint64_t)((s.rows + 15u) / 16u) * steps, blocks = (tiles + kBlock / 64 - 1) / (kBlock / 64);
        auto k = s.values ? mx_rows_k<T, true> : mx_rows_k<T, false>;
        in_launches(blocks, [&](uint64_t first, uint32_t n) { launch(k, dim3(n), dim3(kBlock), lc.stream, s, first, tiles); });
    }
}
void launch_mx_quantize(const LaunchCtx &lc, int dtype, const MxSource &s)
{
    if (dtype == MC_DTYPE_F32) quantize_of<float>(lc, s);
    else if (dtype == MC_DTYPE_BF16) quantize_of<__bf16>(lc, s);
    else quantize_of<_Float16>(lc, s);
}

}  // namespace mc
