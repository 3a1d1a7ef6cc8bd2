// Kernels over a model's list of tensors: global gradient norm, clipping, AdamW.
#include "step_internal.h"

namespace mc {

template <class T> __device__ __forceinline__ global_ptr<T> piece_of(const StepView &v, uint32_t list, const Piece &p)
{
    const uintptr_t at = ld_uniform(v.addr + (size_t)list * v.tensors + (p.tensor & ~kNoDecay));
    return in_global(reinterpret_cast<T *>(at)) + (size_t)p.index * kPiece;
}
__device__ __forceinline__ Piece piece(const StepView &v, uint32_t i)
{
    Piece p;
    p.tensor = ld_uniform(&v.pieces[i].tensor);
    p.index = ld_uniform(&v.pieces[i].index);
    p.count = ld_uniform(&v.pieces[i].count);
    return p;
}

// ---- norm -----------------------------------------------------------------------------------------------------------
template <class T>
__global__ __launch_bounds__(kBlock) void grad_norm_k(StepView v, double *partial)
{
    constexpr int N = 16 / (int)sizeof(T);
    __shared__ double lds[kWavesPerBlock];
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < v.npieces; c += gridDim.x) {
        const Piece p = piece(v, c);
        const global_ptr<const T> g = piece_of<const T>(v, MC_LIST_GRADS, p);
#pragma unroll
        for (uint32_t s = 0; s < kPiece; s += kBlock * N) {
            float x[N];
            load_some<N, T>(g, s + threadIdx.x * N, p.count, x);
#pragma unroll
            for (int e = 0; e < N; ++e) sum = __builtin_fma((double)x[e], (double)x[e], sum);
        }
    }
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kBlock) void norm_finish_k(const double *partial, uint32_t count, float scale, float max_norm, float *out)
{
    __shared__ double lds[kWavesPerBlock];
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < count; i += kBlock) sum += partial[i];
    sum = block_sum(sum, lds);
    if (threadIdx.x != 0) return;
    const double norm = (double)scale * sqrt(sum);
    out[0] = (float)norm;
    out[1] = isfinite(sum) ? (float)((double)scale * fmin(1.0, (double)max_norm / (norm + 1e-6))) : 0.0f;
}

void launch_grad_norm(const LaunchCtx &lc, int dtype, const StepView &v, double *partial, float scale, float max_norm, float *out)
{
    const uint32_t blocks = v.npieces < kNormBlocks ? v.npieces : kNormBlocks;
    if (blocks) {
        auto k = dtype == MC_DTYPE_F32 ? grad_norm_k<float> : dtype == MC_DTYPE_BF16 ? grad_norm_k<__bf16> : grad_norm_k<_Float16>;
        launch(k, dim3(blocks), dim3(kBlock), lc.stream, v, partial);
    }
    launch(norm_finish_k, dim3(1), dim3(kBlock), lc.stream, partial, blocks, scale, max_norm, out);
}

// ---- clipping ---------------------------------------------------------------------------------------------------------
template <class T>
__global__ __launch_bounds__(kBlock) void grad_clip_k(StepView v, uint32_t to_list, const float *coef)
{
    constexpr int N = 16 / (int)sizeof(T);
    const Piece p = piece(v, blockIdx.x);
    const global_ptr<const T> g = piece_of<const T>(v, MC_LIST_GRADS, p);
    const global_ptr<T> to = piece_of<T>(v, to_list, p);
    const float c = *coef;
#pragma unroll
    for (uint32_t s = 0; s < kPiece; s += kBlock * N) {
        float x[N];
        load_some<N, T>(g, s + threadIdx.x * N, p.count, x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = c == 0.0f ? 0.0f : x[e] * c;
        store_some<N, T>(to, s + threadIdx.x * N, p.count, x);
    }
}

void launch_grad_clip(const LaunchCtx &lc, int dtype, const StepView &v, uint32_t to_list, const float *coef)
{
    if (!v.npieces) return;
    auto k = dtype == MC_DTYPE_F32 ? grad_clip_k<float> : dtype == MC_DTYPE_BF16 ? grad_clip_k<__bf16> : grad_clip_k<_Float16>;
    launch(k, dim3(v.npieces), dim3(kBlock), lc.stream, v, to_list, coef);
}

// ---- AdamW --------------------------------------------------------------------------------------------------------------
struct NoCopy {};
template <class T, class M>
__global__ __launch_bounds__(kBlock) void adamw_k(StepView v, AdamwArgs a)
{
    constexpr int N = 4;
    const float coef = a.coef ? *a.coef : 1.0f;
    if (coef == 0.0f) return;
    const Piece p = piece(v, blockIdx.x);
    const global_ptr<const T> grad = piece_of<const T>(v, MC_LIST_GRADS, p);
    const global_ptr<float> param = piece_of<float>(v, MC_LIST_PARAMS, p), avg = piece_of<float>(v, MC_LIST_EXP_AVG, p),
                            avg_sq = piece_of<float>(v, MC_LIST_EXP_AVG_SQ, p);
    const float decay = p.tensor & kNoDecay ? 1.0f : a.decay;
#pragma unroll
    for (uint32_t s = 0; s < kPiece; s += kBlock * N) {
        const uint32_t i = s + threadIdx.x * N;
        float g[N], w[N], m[N], q[N];
        load_some<N, T>(grad, i, p.count, g);
        load_some<N, float>(param, i, p.count, w);
        load_some<N, float>(avg, i, p.count, m);
        load_some<N, float>(avg_sq, i, p.count, q);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            g[e] *= coef;
            m[e] = a.beta1 * m[e] + a.one_minus_beta1 * g[e];
            q[e] = a.beta2 * q[e] + a.one_minus_beta2 * (g[e] * g[e]);
            w[e] = decay * w[e] - a.rate * (m[e] / (sqrtf(q[e]) * a.root + a.eps));
        }
        store_some<N, float>(param, i, p.count, w);
        store_some<N, float>(avg, i, p.count, m);
        store_some<N, float>(avg_sq, i, p.count, q);
        if constexpr (!std::is_same_v<M, NoCopy>) store_some<N, M>(piece_of<M>(v, MC_LIST_MODEL, p), i, p.count, w);
    }
}

template <class T>
static void adamw_of(const LaunchCtx &lc, int model_dtype, const StepView &v, const AdamwArgs &a)
{
    auto k = model_dtype == MC_DTYPE_NONE ? adamw_k<T, NoCopy> : model_dtype == MC_DTYPE_BF16 ? adamw_k<T, __bf16> : adamw_k<T, _Float16>;
    launch(k, dim3(v.npieces), dim3(kBlock), lc.stream, v, a);
}
void launch_adamw(const LaunchCtx &lc, int dtype, int model_dtype, const StepView &v, const AdamwArgs &a)
{
    if (!v.npieces) return;
    if (dtype == MC_DTYPE_F32) adamw_of<float>(lc, model_dtype, v, a);
    else if (dtype == MC_DTYPE_BF16) adamw_of<__bf16>(lc, model_dtype, v, a);
    else adamw_of<_Float16>(lc, model_dtype, v, a);
}

}  // namespace mc
