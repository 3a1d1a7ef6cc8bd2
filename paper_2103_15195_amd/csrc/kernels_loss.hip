// Kernels over rows of logits: token log-probabilities, and the clipped policy loss with its gradient.
#include "step_internal.h"

namespace mc {

// exp((x - top) / temperature) for logits of type T.  The difference comes first, so that a row of nothing but the type's lowest
// value is as good as any other.  With logits of 32 bits the factor has a second part: rounded to 24 bits it moves
// exp(-10) by 4e-7 (what is infinite already stays away from that part: times 0 or a negative number it would be NaN).
template <class T>
__device__ __forceinline__ float row_exp(const LossArgs &a, float x, float top)
{
    const float d = x - top;
    if constexpr (sizeof(T) < 4) return __builtin_amdgcn_exp2f(d * a.to_base2);
    return __builtin_amdgcn_exp2f(__builtin_fmaf(d, a.to_base2, fmaxf(d, -1e30f) * a.to_base2_rest));
}
// where a maximum of minus infinity (nothing seen so far) stands for exponents: any finite number
__device__ __forceinline__ float base_of(float top) { return top == -__builtin_inff() ? 0.0f : top; }

// What a row adds to the sums, and the slope of its loss by its log-probability.
struct RowTerms { float policy, kl, cut, slope; };
__device__ __forceinline__ RowTerms row_terms(const LossArgs &a, uint32_t r, float logp)
{
    RowTerms t;
    const float adv = a.advantages[r], rho = expf(logp - a.old_logp[r]);
    const float free = -adv * rho, held = -adv * fminf(fmaxf(rho, a.lo), a.hi);
    const bool is_free = !(free < held);              // (NaN: the ratio's)
    t.policy = is_free ? free : held;
    t.slope = is_free ? free : 0.0f;
    t.cut = is_free ? 0.0f : 1.0f;
    t.kl = 0.0f;
    if (a.ref_logp) {
        const float d = a.ref_logp[r] - logp, ed = expf(d);
        t.kl = ed - d - 1.0f;
        t.slope += a.kl_coef * (1.0f - ed);
    }
    return t;
}

// One block to a row, two passes over it: the running maximum and sum, then the gradient.
template <class T, bool LOSS>
__global__ __launch_bounds__(kBlock) void loss_rows_k(LossArgs a)
{
    constexpr int N = 16 / (int)sizeof(T);
    __shared__ float lds[2 * kWavesPerBlock];
    double sums[kLossSums] = {};
    for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t label = a.labels[r];
        const float w = LOSS ? (a.weights ? a.weights[r] : 1.0f) : 1.0f;
        const bool valid = label >= 0 && label < (int64_t)a.vocab, taken = valid && w != 0.0f;
        const global_ptr<const T> x = in_global(static_cast<const T *>(a.logits)) + (int64_t)r * a.stride;
        const global_ptr<T> dx = in_global(static_cast<T *>(a.dlogits)) + (int64_t)r * a.dstride;
        if (!taken) {
            if (LOSS && threadIdx.x == 0 && w != 0.0f) sums[6] += 1.0;
            if (threadIdx.x == 0 && a.logp) a.logp[r] = 0.0f;
            if (LOSS && a.dlogits) {
                const float zero[N] = {};
                for (uint32_t i = threadIdx.x * N; i < a.vocab; i += kBlock * N) store_some<N, T>(dx, i, a.vocab, zero);
            }
            continue;
        }
        const float xa = (float)x[label];
        float top = -__builtin_inff(), sum = 0.0f;
        for (uint32_t i = threadIdx.x * N; i < a.vocab; i += kBlock * N) {
            float v[N], most;
            load_some<N, T>(x, i, a.vocab, v, -__builtin_inff());
            most = v[0];
#pragma unroll
            for (int e = 1; e < N; ++e) most = fmaxf(most, v[e]);
            if (most > top) { sum *= row_exp<T>(a, top, most); top = most; }
            const float base = base_of(top);
#pragma unroll
            for (int e = 0; e < N; ++e) sum += row_exp<T>(a, v[e], base);
        }
        const float wtop = wave_max(top);
        sum *= row_exp<T>(a, top, base_of(wtop));
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) sum += __shfl_xor(sum, m, 64);
        if ((threadIdx.x & 63u) == 0) { lds[threadIdx.x >> 6] = wtop; lds[kWavesPerBlock + (threadIdx.x >> 6)] = sum; }
        __syncthreads();
        top = lds[0];
#pragma unroll
        for (int k = 1; k < kWavesPerBlock; ++k) top = fmaxf(top, lds[k]);
        top = base_of(top);
        sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kWavesPerBlock; ++k) sum += lds[kWavesPerBlock + k] * row_exp<T>(a, lds[k], top);
        __syncthreads();
        const float logp = (xa - top) * a.inv_t - logf(sum);
        if (threadIdx.x == 0 && a.logp) a.logp[r] = logp;
        if (!LOSS) continue;
        const RowTerms t = row_terms(a, r, logp);
        if (threadIdx.x == 0) {
            const double wd = w;
            sums[0] += wd * ((double)t.policy + (double)a.kl_coef * t.kl);
            sums[1] += wd * t.policy; sums[2] += wd * t.kl; sums[3] += wd * t.cut; sums[4] += wd; sums[5] += 1.0;
        }
        if (!a.dlogits) continue;
        const float slope = w * t.slope * a.gscale, part = -slope / sum;
        for (uint32_t i = threadIdx.x * N; i < a.vocab; i += kBlock * N) {
            float v[N];
            load_some<N, T>(x, i, a.vocab, v, -__builtin_inff());
#pragma unroll
            for (int e = 0; e < N; ++e) {
                v[e] = part * row_exp<T>(a, v[e], top);
                if (i + (uint32_t)e == (uint32_t)label) v[e] += slope;
            }
            store_some<N, T>(dx, i, a.vocab, v);
        }
    }
    if (LOSS && threadIdx.x == 0)
#pragma unroll
        for (int k = 0; k < kLossSums; ++k) a.partial[(size_t)blockIdx.x * kLossSums + k] = sums[k];
}

__global__ __launch_bounds__(kBlock) void loss_finish_k(const double *partial, uint32_t count, float *out)
{
    __shared__ double lds[kWavesPerBlock];
    for (int k = 0; k < kLossSums; ++k) {
        double sum = 0.0;
        for (uint32_t i = threadIdx.x; i < count; i += kBlock) sum += partial[(size_t)i * kLossSums + k];
        sum = block_sum(sum, lds);
        if (threadIdx.x == 0) out[k] = k < 5 ? (float)sum : __int_as_float((int)sum);
    }
    if (threadIdx.x == 0) out[7] = 0.0f;
}

template <class T>
static void loss_of(const LaunchCtx &lc, const LossArgs &a, bool loss)
{
    const uint32_t blocks = a.rows < kLossBlocks ? a.rows : kLossBlocks;
    if (blocks) launch(loss ? loss_rows_k<T, true> : loss_rows_k<T, false>, dim3(blocks), dim3(kBlock), lc.stream, a);
    if (loss) launch(loss_finish_k, dim3(1), dim3(kBlock), lc.stream, a.partial, blocks, a.sums);
}
static void loss_by(const LaunchCtx &lc, int dtype, const LossArgs &a, bool loss)
{
    if (dtype == MC_DTYPE_F32) loss_of<float>(lc, a, loss);
    else if (dtype == MC_DTYPE_BF16) loss_of<__bf16>(lc, a, loss);
    else loss_of<_Float16>(lc, a, loss);
}
void launch_token_logp(const LaunchCtx &lc, int dtype, const LossArgs &a) { loss_by(lc, dtype, a, false); }
void launch_policy_loss(const LaunchCtx &lc, int dtype, const LossArgs &a) { loss_by(lc, dtype, a, true); }

}  // namespace mc
