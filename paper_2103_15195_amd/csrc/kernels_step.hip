// Kernels over a model's list of tensors: global gradient norm, clipping, AdamW.
//
// All three are streams: what bounds them is the memory's rate.  The norm reads its gradients through the caches, because what
// follows it reads them again: of a gradient that the last-level cache holds in part, clipping of 178 MB takes 80 us instead of 91, the norm and AdamW of
// 102 MB 134 instead of 150, of 320 MB in 16 bits 847 instead of 896 (a norm that nothing follows loses up to a tenth: 268 MB
// 43 -> 47 us).  Everything else is read and written past them (AdamW of 102 MB through them: 161 us).
#include "step_internal.h"

namespace mc {

// A piece, and the elements lo .. hi - 1 from `from` on of its tensor that are this block's, with `from` on a line of the list at `list`.
struct Span {
    uint32_t tensor;
    int32_t lo, hi;
    int64_t from;
};
template <class T>
__device__ __forceinline__ Span span_of(const StepView &v, uint32_t i, uint32_t list)
{
    const uint32_t name = ld_uniform(&v.pieces[i].tensor), index = ld_uniform(&v.pieces[i].index);
    const int32_t left = ld_uniform(&v.pieces[i].left);
    const uintptr_t at = ld_uniform(v.addr + (size_t)list * v.tensors + (name & ~kNoDecay));
    const int32_t shift = (int32_t)((uint32_t)at % kLine / (uint32_t)sizeof(T));
    const int32_t hi = left < (int32_t)kPiece ? left + shift : (int32_t)kPiece;
    return {name, index ? 0 : shift, hi < (int32_t)kPiece ? hi : (int32_t)kPiece, (int64_t)index * kPiece - shift};
}
template <class T>
__device__ __forceinline__ global_ptr<T> span_in(const StepView &v, uint32_t list, const Span &s)
{
    return in_global(reinterpret_cast<T *>(ld_uniform(v.addr + (size_t)list * v.tensors + (s.tensor & ~kNoDecay)))) + s.from;
}

// All pieces, in launches of fewer than 2^32 threads.
template <class Body>
static void in_launches(StepView v, Body body)
{
    constexpr uint32_t most = 1u << 21;
    for (uint32_t left = v.npieces; left; left -= v.npieces, v.pieces += v.npieces) {
        v.npieces = left < most ? left : most;
        body(v);
    }
}

// ---- norm -----------------------------------------------------------------------------------------------------------
// Squares are summed in binary64: of binary32 values they are exact there, and neither overflow nor vanish.  Blocks take pieces in
// turn, and the last one to be done adds up what all have left: one launch (with the sums added up by a second one 7.0 instead of 4.8 us
// for 272 474 elements in 65 tensors).
// 25.6 M elements in 161 tensors 19.3 us (5.3 TB/s), 120 M of 16 bits 43.0 (5.6 TB/s).  1024 blocks of 512 threads: of 256 threads 53.4 of
// the latter, 2048 of 256 20.2 of the former and 43.4.
constexpr int kNormThreads = 512;
template <class T>
__global__ __launch_bounds__(kNormThreads) void grad_norm_k(StepView v, double *partial, uint32_t *counts, float scale, float max_norm, float *out)
{
    constexpr int N = 16 / (int)sizeof(T), STEPS = (int)kPiece / (kNormThreads * N);
    __shared__ double lds[kNormThreads / 64];
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < v.npieces; c += gridDim.x) {
        const Span s = span_of<T>(v, c, MC_LIST_GRADS);
        const global_ptr<const T> g = span_in<const T>(v, MC_LIST_GRADS, s);
        float x[STEPS][N];
#pragma unroll
        for (int k = 0; k < STEPS; ++k) load_some<N, T, false>(g, (int32_t)(k * kNormThreads + threadIdx.x) * N, s.lo, s.hi, x[k]);
#pragma unroll
        for (int k = 0; k < STEPS; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) sum = __builtin_fma((double)x[k][e], (double)x[k][e], sum);
    }
    sum = block_sum<kNormThreads / 64>(sum, lds);
    if (threadIdx.x >= 64u) return;
    if (threadIdx.x == 0) leave_sum(partial + blockIdx.x, sum);
    if (!arrives_last(counts)) return;
    sum = 0.0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += 64u * 8u) {
        double x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = i + 64u * k < gridDim.x ? left_sum(partial + i + 64u * k) : 0.0;
        sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    }
    sum = wave_sum(sum);
    if (threadIdx.x != 0) return;
    const double norm = (double)scale * sqrt(sum);
    out[0] = (float)norm;
    out[1] = isfinite(sum) ? (float)((double)scale * fmin(1.0, (double)max_norm / (norm + 1e-6))) : 0.0f;
}

void launch_grad_norm(const LaunchCtx &lc, int dtype, const StepView &v, double *partial, uint32_t *counts, float scale, float max_norm, float *out)
{
    const uint32_t blocks = v.npieces < 1u ? 1u : v.npieces < kNormBlocks ? v.npieces : kNormBlocks;
    auto k = dtype == MC_DTYPE_F32 ? grad_norm_k<float> : dtype == MC_DTYPE_BF16 ? grad_norm_k<__bf16> : grad_norm_k<_Float16>;
    launch(k, dim3(blocks), dim3(kNormThreads), lc.stream, v, partial, counts, scale, max_norm, out);
}

// ---- clipping ---------------------------------------------------------------------------------------------------------
// A block to a piece (a block to a quarter of one: 83 instead of 81 us for 178 MB, 127 instead of 108 for 240 MB of 16 bits).  Behind the
// norm it finds part of the gradient in the last-level cache (pieces taken last first, so that those read last come first, gained
// nothing: 85.6 and 81.4 us).
template <class T>
__global__ __launch_bounds__(kBlock) void grad_clip_k(StepView v, uint32_t to_list, const float *coef)
{
    constexpr int N = 16 / (int)sizeof(T);
    const Span s = span_of<T>(v, blockIdx.x, to_list);
    const global_ptr<const T> g = span_in<const T>(v, MC_LIST_GRADS, s);
    const global_ptr<T> to = span_in<T>(v, to_list, s);
    const float c = *coef;
#pragma unroll
    for (int32_t k = 0; k < (int32_t)kPiece; k += kBlock * N) {
        const int32_t i = k + (int32_t)threadIdx.x * N;
        float x[N];
        load_some<N, T>(g, i, s.lo, s.hi, x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = c == 0.0f ? 0.0f : x[e] * c;
        store_some<N, T>(to, i, s.lo, s.hi, x);
    }
}

void launch_grad_clip(const LaunchCtx &lc, int dtype, const StepView &v, uint32_t to_list, const float *coef)
{
    auto k = dtype == MC_DTYPE_F32 ? grad_clip_k<float> : dtype == MC_DTYPE_BF16 ? grad_clip_k<__bf16> : grad_clip_k<_Float16>;
    in_launches(v, [&](const StepView &w) { launch(k, dim3(w.npieces), dim3(kBlock), lc.stream, w, to_list, coef); });
}

// ---- AdamW --------------------------------------------------------------------------------------------------------------
// Four elements a thread: 16 bytes of each 32-bit list, 8 of a 16-bit one.  A block has a quarter of a piece and is done when its
// one load of each list is: with the norm before it 25.6 M elements in 32 bits take 130 us (5.5 TB/s), 160 M of mixed precision 770 (5.8 TB/s);
// a block to a piece, four loads of each list a thread, 133 and 846.
struct NoCopy {};
constexpr uint32_t kAdamwSpan = kBlock * 4, kAdamwShares = kPiece / kAdamwSpan;
template <class T, class M>
__global__ __launch_bounds__(kBlock) void adamw_k(StepView v, AdamwArgs a)
{
    constexpr int N = 4;
    const float coef = a.coef ? ld_uniform(a.coef) : 1.0f;
    const Span s = span_of<float>(v, blockIdx.x / kAdamwShares, MC_LIST_PARAMS);
    const global_ptr<const T> grad = span_in<const T>(v, MC_LIST_GRADS, s);
    const global_ptr<float> param = span_in<float>(v, MC_LIST_PARAMS, s), avg = span_in<float>(v, MC_LIST_EXP_AVG, s),
                            avg_sq = span_in<float>(v, MC_LIST_EXP_AVG_SQ, s);
    const float decay = s.tensor & kNoDecay ? 1.0f : a.decay;
    const int32_t i = (int32_t)(blockIdx.x % kAdamwShares * kAdamwSpan + threadIdx.x * N);
    float g[N], w[N], m[N], q[N];
    load_some<N, T>(grad, i, s.lo, s.hi, g);
    load_some<N, float>(param, i, s.lo, s.hi, w);
    load_some<N, float>(avg, i, s.lo, s.hi, m);
    load_some<N, float>(avg_sq, i, s.lo, s.hi, q);
    if (coef == 0.0f) return;            // (looked at behind the loads, which need not wait for it)
#pragma unroll
    for (int e = 0; e < N; ++e) {
        g[e] *= coef;
        m[e] = a.beta1 * m[e] + a.one_minus_beta1 * g[e];
        q[e] = a.beta2 * q[e] + a.one_minus_beta2 * (g[e] * g[e]);
        w[e] = decay * w[e] - a.rate * (m[e] / (sqrtf(q[e]) * a.root + a.eps));
    }
    store_some<N, float>(param, i, s.lo, s.hi, w);
    store_some<N, float>(avg, i, s.lo, s.hi, m);
    store_some<N, float>(avg_sq, i, s.lo, s.hi, q);
    if constexpr (!std::is_same_v<M, NoCopy>) store_some<N, M>(span_in<M>(v, MC_LIST_MODEL, s), i, s.lo, s.hi, w);
}

template <class T>
static void adamw_of(const LaunchCtx &lc, int model_dtype, const StepView &v, const AdamwArgs &a)
{
    auto k = model_dtype == MC_DTYPE_NONE ? adamw_k<T, NoCopy> : model_dtype == MC_DTYPE_BF16 ? adamw_k<T, __bf16> : adamw_k<T, _Float16>;
    in_launches(v, [&](const StepView &w) { launch(k, dim3(w.npieces * kAdamwShares), dim3(kBlock), lc.stream, w, a); });
}
void launch_adamw(const LaunchCtx &lc, int dtype, int model_dtype, const StepView &v, const AdamwArgs &a)
{
    if (dtype == MC_DTYPE_F32) adamw_of<float>(lc, model_dtype, v, a);
    else if (dtype == MC_DTYPE_BF16) adamw_of<__bf16>(lc, model_dtype, v, a);
    else adamw_of<_Float16>(lc, model_dtype, v, a);
}

}  // namespace mc
