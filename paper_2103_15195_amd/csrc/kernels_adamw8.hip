// AdamW with moments in 8 bits.
//
// A stream, like AdamW in 32 bits, of 16 bytes an element instead of 28.  A thread has eight consecutive elements, so that a block of
// 128 that shares a scale is a row of 16 lanes, whose largest magnitude is found without LDS.
#include "mx_internal.h"

namespace mc {

// The largest of each row of 16 lanes, in all of them.
template <int ROTATE>
__device__ __forceinline__ float rotated_max(float x)
{
    const float y = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x120 + ROTATE, 0xf, 0xf, false));
    return fmaxf(x, y);
}
__device__ __forceinline__ float row_max(float x)
{
    return rotated_max<1>(rotated_max<2>(rotated_max<4>(rotated_max<8>(x))));
}

typedef uint32_t codes8 __attribute__((ext_vector_type(2)));
typedef codes8 codes8_any __attribute__((aligned(1)));
typedef float float2v __attribute__((ext_vector_type(2)));

// Eight consecutive elements of a thread, of a whole block's (FULL) or of those below `hi`.  A whole block's accesses depend on nothing, so that all of them
// travel together.
template <bool FULL>
__device__ __forceinline__ codes8 load_codes(global_ptr<const uint8_t> p, int32_t i, int32_t hi)
{
    if (FULL || i + 8 <= hi) return __builtin_nontemporal_load((global_ptr<const codes8_any>)(p + i));
    codes8 c = {0u, 0u};
    for (int e = 0; e < 8; ++e) if (i + e < hi) c[e / 4] |= (uint32_t)p[i + e] << (8 * (e % 4));
    return c;
}
template <bool FULL>
__device__ __forceinline__ void store_codes(global_ptr<uint8_t> p, int32_t i, int32_t hi, codes8 c)
{
    if (FULL || i + 8 <= hi) __builtin_nontemporal_store(c, (global_ptr<codes8_any>)(p + i));
    else for (int e = 0; e < 8; ++e) if (i + e < hi) p[i + e] = (uint8_t)(c[e / 4] >> (8 * (e % 4)));
}
template <bool FULL, class T>
__device__ __forceinline__ void load8(global_ptr<const T> p, int32_t i, int32_t hi, float (&x)[8])
{
    constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
    for (int k = 0; k < 8 / N; ++k) {
        float y[N];
        load_some<N, T>(p, i + N * k, 0, FULL ? (int32_t)kPiece8 : hi, y);
#pragma unroll
        for (int e = 0; e < N; ++e) x[N * k + e] = y[e];
    }
}
template <bool FULL, class T>
__device__ __forceinline__ void store8(global_ptr<T> p, int32_t i, int32_t hi, const float (&x)[8])
{
    constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
    for (int k = 0; k < 8 / N; ++k) {
        float y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = x[N * k + e];
        store_some<N, T>(p, i + N * k, 0, FULL ? (int32_t)kPiece8 : hi, y);
    }
}
__device__ __forceinline__ void held(codes8 c, float scale, float (&x)[8])
{
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[k], true);
        x[4 * k] = lo[0] * scale; x[4 * k + 1] = lo[1] * scale; x[4 * k + 2] = hi[0] * scale; x[4 * k + 3] = hi[1] * scale;
    }
}
// Values to codes under the largest finite magnitude of their block; returns the scale.  A NaN stays one, an infinity becomes one (the conversion
// has no infinity, and rounds what is up to half a step above 448 to 448, which the quotient's own rounding needs).
template <bool ROOT>
__device__ __forceinline__ float hold8(const float (&x)[8], codes8 &c)
{
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));           // (of a NaN: what was there)
    if (__builtin_expect(__any(top == __builtin_huge_valf()), 0)) {
        top = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]) < __builtin_huge_valf() ? fabsf(x[e]) : 0.0f);
    }
    top = row_max(top);
    const float scale = top >= 0x1p-100f ? top * (1.0f / 448.0f) : 0.0f, back = scale > 0.0f ? 1.0f / scale : 0.0f;
    // Roots above this are at least the least code: those above 0, and none in a block without a scale, where an infinity's 0 * infinity has to stay the NaN that it
    // is (a maximum would drop it).
    const float above = scale > 0.0f ? 0.0f : __builtin_huge_valf();
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        y[e] = x[e] * back;
        if (ROOT) y[e] = x[e] > above ? fmaxf(y[e], 0x1p-9f) : y[e];     // (not of a NaN, which is above nothing)
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k], y[4 * k + 1], 0, false);
        c[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k + 2], y[4 * k + 3], lo, true);
    }
    return scale;
}

struct NoCopy8 {};
template <class T>
__device__ __forceinline__ global_ptr<T> list8(const Step8View &v, uint32_t list, uint32_t tensor)
{
    return in_global(reinterpret_cast<T *>(ld_uniform(v.addr + (size_t)list * v.tensors + tensor)));
}
// The square root, rounded correctly from 2^-96 on (below, by up to a unit in the last place), by Tuckerman's test (Agarwal et al., New scalar and vector elementary functions for the
// IBM System/370, 1986): s, off by at most a unit u, is the root's rounding where s (s - u) < x <= s (s + u), else it is the neighbour on that side.  A fused multiply-add has the
// sign of either difference without an error.
__device__ __forceinline__ float root_of(float x)
{
    const float s = __builtin_amdgcn_sqrtf(x);
    const float under = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, s) - 1u), over = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, s) + 1u);
    float r = __builtin_fmaf(-under, s, x) <= 0.0f ? under : s;
    r = __builtin_fmaf(-over, s, x) > 0.0f ? over : r;
    return x >= 0x1p-126f && x < __builtin_huge_valf() ? r : s;
}
// The moments are rounded after every operation, as their formulas stand, so that their codes do not depend on how a compiler joins them: a unit in the last place can
// decide between two codes.  The weights' quotient is the hardware's reciprocal, off by such a unit.
// (All accesses under conditions of their own, library root and division: 25.6 M elements in 32 bits 119 us, 160 M of mixed precision 652.  So: 80 (5.2 TB/s) and 467
// (5.5 TB/s), which is the memory's rate: AdamW in 32 bits moves 5.5 and 5.8 TB/s.  With the hardware's root and fused sums 80 and 471.)
template <class T, class M, bool FULL>
__device__ __forceinline__ void adamw8_piece(const Step8View &v, const AdamwArgs &a, uint32_t name, uint32_t index, int32_t hi)
{
    const float coef = a.coef ? ld_uniform(a.coef) : 1.0f;
    const uint32_t tensor = name & ~kNoDecay;
    const int64_t from = (int64_t)index * kPiece8;
    const global_ptr<const T> grad = list8<const T>(v, MC_LIST8_GRADS, tensor) + from;
    const global_ptr<float> param = list8<float>(v, MC_LIST8_PARAMS, tensor) + from;
    const global_ptr<uint8_t> avg = list8<uint8_t>(v, MC_LIST8_EXP_AVG, tensor) + from, avg_sq = list8<uint8_t>(v, MC_LIST8_EXP_AVG_SQ, tensor) + from;
    const int64_t first = (int64_t)index * (kPiece8 / kBlock8) + threadIdx.x / (kBlock8 / 8);
    const global_ptr<float> avg_scale = list8<float>(v, MC_LIST8_EXP_AVG_SCALE, tensor) + first, avg_sq_scale = list8<float>(v, MC_LIST8_EXP_AVG_SQ_SCALE, tensor) + first;
    const int32_t i = (int32_t)threadIdx.x * 8;
    const bool mine = FULL || (i & ~(int32_t)(kBlock8 - 1)) < hi;        // the block of 128 holds elements
    const float decay = name & kNoDecay ? 1.0f : a.decay;
    float g[8], w[8], m[8], r[8];
    load8<FULL, T>(grad, i, hi, g);
    load8<FULL, float>(param, i, hi, w);
    const codes8 cm = load_codes<FULL>(avg, i, hi), cr = load_codes<FULL>(avg_sq, i, hi);
    const float sm = mine ? *avg_scale : 0.0f, sr = mine ? *avg_sq_scale : 0.0f;
    if (coef == 0.0f) return;            // (looked at behind the loads, which need not wait for it)
    held(cm, sm, m);
    held(cr, sr, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        g[e] *= coef;
        m[e] = a.beta1 * m[e] + a.one_minus_beta1 * g[e];
        r[e] = root_of(a.beta2 * (r[e] * r[e]) + a.one_minus_beta2 * (g[e] * g[e]));
        // (the least normal number, so that its reciprocal is finite)
        const float under = __builtin_fmaf(r[e], a.root, a.eps), q = m[e] * __builtin_amdgcn_rcpf(under < 0x1p-126f ? 0x1p-126f : under);
        w[e] = __builtin_fmaf(-a.rate, q, decay * w[e]);
        asm volatile("" : "+v"(w[e]));   // (the model's copy is this rounded, not the sum: the compiler has an instruction for that)
    }
    store8<FULL, float>(param, i, hi, w);
    if constexpr (!std::is_same_v<M, NoCopy8>) store8<FULL, M>(list8<M>(v, MC_LIST8_MODEL, tensor) + from, i, hi, w);
    codes8 c;
    const float tm = hold8<false>(m, c);
    store_codes<FULL>(avg, i, hi, c);
    const float tr = hold8<true>(r, c);
    store_codes<FULL>(avg_sq, i, hi, c);
    if (mine && threadIdx.x % (kBlock8 / 8) == 0) {
        *avg_scale = tm;
        *avg_sq_scale = tr;
    }
}
template <class T, class M>
__global__ __launch_bounds__(kBlock) void adamw8_k(Step8View v, AdamwArgs a)
{
    const uint32_t name = ld_uniform(&v.pieces[blockIdx.x].tensor), index = ld_uniform(&v.pieces[blockIdx.x].index);
    const int32_t hi = ld_uniform(&v.pieces[blockIdx.x].left);
    if (hi == (int32_t)kPiece8) adamw8_piece<T, M, true>(v, a, name, index, hi);
    else adamw8_piece<T, M, false>(v, a, name, index, hi);
}

template <class T>
static void adamw8_of(const LaunchCtx &lc, int model_dtype, const Step8View &v, const AdamwArgs &a)
{
    auto k = model_dtype == MC_DTYPE_NONE ? adamw8_k<T, NoCopy8> : model_dtype == MC_DTYPE_BF16 ? adamw8_k<T, __bf16> : adamw8_k<T, _Float16>;
    in_launches(v.npieces, [&](uint64_t first, uint32_t n) { launch(k, dim3(n), dim3(kBlock), lc.stream, Step8View{v.pieces + first, v.addr, n, v.tensors}, a); });
}
void launch_adamw8(const LaunchCtx &lc, int dtype, int model_dtype, const Step8View &v, const AdamwArgs &a)
{
    if (dtype == MC_DTYPE_F32) adamw8_of<float>(lc, model_dtype, v, a);
    else if (dtype == MC_DTYPE_BF16) adamw8_of<__bf16>(lc, model_dtype, v, a);
    else adamw8_of<_Float16>(lc, model_dtype, v, a);
}

}  // namespace mc
