// Host <-> kernel-launcher interface of the operators in mergecomp_step.h, and what their kernels share.
#pragma once
#include "../../include/mergecomp_step.h"
#include "mc_internal.h"

namespace mc {

// ---- lists of tensors ---------------------------------------------------------------------------------------------
// Work is handed out in pieces of at most kPiece consecutive elements of one tensor.
constexpr uint32_t kPiece = 4096;
constexpr uint32_t kNoDecay = 0x80000000u;
struct alignas(16) Piece {
    uint32_t tensor;             // its place in the lists of addresses; kNoDecay: not decayed
    uint32_t index;              // the piece begins at element kPiece * index of it
    uint32_t count;
    uint32_t pad;
};
// A handle's lists as the kernels see them: the addresses of list l are addr[l * tensors ..].
struct StepView {
    const Piece *pieces;
    const uintptr_t *addr;
    uint32_t npieces, tensors;
};
// blocks of the norm's first pass, at most, and the scratch that they leave their sums in
constexpr uint32_t kNormBlocks = 2048;

struct AdamwArgs {
    const float *coef;           // null: 1
    float beta1, one_minus_beta1, beta2, one_minus_beta2;
    float decay;                 // 1 - lr weight_decay
    float rate;                  // lr / (1 - beta1^step)
    float root;                  // 1 / sqrt(1 - beta2^step)
    float eps;
};

void launch_grad_norm(const LaunchCtx &lc, int dtype, const StepView &v, double *partial, float scale, float max_norm, float *out);
void launch_grad_clip(const LaunchCtx &lc, int dtype, const StepView &v, uint32_t to_list, const float *coef);
void launch_adamw(const LaunchCtx &lc, int dtype, int model_dtype, const StepView &v, const AdamwArgs &a);

// ---- rows of logits -----------------------------------------------------------------------------------------------
constexpr int kLossSums = 7;                 // five sums and two counts
constexpr uint32_t kLossBlocks = 2048;
struct LossArgs {
    const void *logits;
    const int64_t *labels;
    const float *old_logp, *advantages, *weights, *ref_logp;
    float *sums, *logp;
    void *dlogits;
    int64_t stride, dstride;
    uint32_t rows, vocab;
    float to_base2, to_base2_rest;           // log2(e) / temperature, in two parts
    float inv_t, lo, hi, kl_coef, gscale;    // gscale: grad_scale / temperature
    double *partial;
};
void launch_token_logp(const LaunchCtx &lc, int dtype, const LossArgs &a);
void launch_policy_loss(const LaunchCtx &lc, int dtype, const LossArgs &a);

// ---- values of 32 and 16 bits ---------------------------------------------------------------------------------------
template <class T, int N> struct VecOf;
#define MC_VEC(T, N, ALIGN) template <> struct VecOf<T, N> { typedef T type __attribute__((ext_vector_type(N), aligned(ALIGN))); }
MC_VEC(float, 4, 4);
MC_VEC(__bf16, 4, 2);
MC_VEC(__bf16, 8, 2);
MC_VEC(_Float16, 4, 2);
MC_VEC(_Float16, 8, 2);
#undef MC_VEC

// N consecutive elements from p + i, those from `count` on as `fill`
template <int N, class T>
__device__ __forceinline__ void load_some(global_ptr<const T> p, uint32_t i, uint32_t count, float (&v)[N], float fill = 0.0f)
{
    typedef typename VecOf<T, N>::type vec;
    if (i + (uint32_t)N <= count) {
        const vec x = __builtin_nontemporal_load((global_ptr<const vec>)(p + i));
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (float)x[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = i + (uint32_t)e < count ? (float)p[i + e] : fill;
    }
}
template <int N, class T>
__device__ __forceinline__ void store_some(global_ptr<T> p, uint32_t i, uint32_t count, const float (&v)[N])
{
    typedef typename VecOf<T, N>::type vec;
    if (i + (uint32_t)N <= count) {
        vec x;
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = (T)v[e];
        __builtin_nontemporal_store(x, (global_ptr<vec>)(p + i));
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) if (i + (uint32_t)e < count) p[i + e] = (T)v[e];
    }
}

}  // namespace mc
