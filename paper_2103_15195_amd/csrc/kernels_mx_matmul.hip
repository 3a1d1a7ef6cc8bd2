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

template <class T>
static void matmul_of(const LaunchCtx &lc, const MxProduct &p)
{
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
