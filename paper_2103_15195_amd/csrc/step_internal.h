// Host <-> kernel-launcher interface of the operators in mergecomp_step.h, and what their kernels share.
#pragma once
#include "../../include/mergecomp_step.h"
#include "mc_internal.h"

namespace mc {

// ---- lists of tensors ---------------------------------------------------------------------------------------------
// Work is handed out in pieces of kPiece elements of a tensor, counted from the 128-byte line that the tensor begins in (in the list
// that a kernel writes): every piece but the first then begins on a line, wherever the tensors lie, and a piece more than
// the elements need stands ready for those that the beginning takes.
constexpr uint32_t kPiece = 4096, kLine = 128, kMostShift = kLine / 2 - 1;       // (elements of 16 bits)
constexpr uint32_t kNoDecay = 0x80000000u;
struct alignas(16) Piece {
    uint32_t tensor;             // its place in the lists of addresses; kNoDecay: not decayed
    uint32_t index;              // which of the tensor's pieces
    int32_t left;                // elements from kPiece * index on, if that many are within reach (below 0: the one more)
    uint32_t pad;
};
// A handle's lists as the kernels see them: the addresses of list l are addr[l * tensors ..].
struct StepView {
    const Piece *pieces;
    const uintptr_t *addr;
    uint32_t npieces, tensors;
};
// blocks of the norm's first pass, at most, and the scratch that they leave their sums in
constexpr uint32_t kNormBlocks = 1024;

struct AdamwArgs {
    const float *coef;           // null: 1
    float beta1, one_minus_beta1, beta2, one_minus_beta2;
    float decay;                 // 1 - lr weight_decay
    float rate;                  // lr / (1 - beta1^step)
    float root;                  // 1 / sqrt(1 - beta2^step)
    float eps;
};

void launch_grad_norm(const LaunchCtx &lc, int dtype, const StepView &v, double *partial, uint32_t *counts, float scale, float max_norm,
                      float *out);
void launch_grad_clip(const LaunchCtx &lc, int dtype, const StepView &v, uint32_t to_list, const float *coef);
void launch_adamw(const LaunchCtx &lc, int dtype, int model_dtype, const StepView &v, const AdamwArgs &a);

// ---- rows of logits -----------------------------------------------------------------------------------------------
constexpr int kLossSums = 6;                 // four sums and two counts
// What a row adds to them.
struct alignas(16) Term {
    float policy, kl, weight;
    uint32_t kind;
};
enum TermKind { TERM_NONE = 0, TERM_FREE = 1, TERM_CUT = 2, TERM_LEFT_OUT = 3 };      // takes no part; does; does and the clamp decides; has a weight, but no valid label
constexpr uint32_t kTermRows = 1u << 17;     // rows that there is room for: more of them are taken so many at a time
constexpr uint32_t kTermBlock = 2048;        // rows per block of the kernel that adds them up
constexpr uint32_t kLossPartials = kTermRows / kTermBlock;
// The parts of a row that several blocks share.
constexpr uint32_t kPartRows = 128, kMostParts = 64;
struct PartsOfRow {
    float top[kMostParts], sum[kMostParts];
    float label;                             // the label's logit
    float pad[31];
};
struct LossArgs {
    const void *logits;
    const int64_t *labels;
    const float *old_logp, *advantages, *weights, *ref_logp;
    float *sums, *logp;
    void *dlogits;
    int64_t stride, dstride;
    uint32_t rows, vocab;
    float to_base2, to_base2_rest;           // log2(e) / temperature, in two parts
    float least;                             // below 0: the largest number whose product with the second part is finite
    double inv_t;
    float lo, hi, kl_coef, gscale;           // gscale: grad_scale / temperature
    Term *terms;                             // kTermRows
    PartsOfRow *parts;                       // kPartRows
    double *partial;                         // kLossSums lists of kLossPartials sums, then the sums of the rows before these
    uint32_t *counts;                        // kArriveBytes
    uint32_t line;                           // bytes: what rows' vectors are counted from a multiple of
    bool more;                               // there are rows before these
};
void launch_token_logp(const LaunchCtx &lc, int dtype, const LossArgs &a);
void launch_policy_loss(const LaunchCtx &lc, int dtype, const LossArgs &a);

// ---- sums over all blocks of a launch -----------------------------------------------------------------------------
// Every block leaves its sums and adds one to a count; the block that finds all others' additions there combines them, in an order that
// does not depend on which block that is.  Additions to one line take 30 ns each where the blocks sit on different dies: up to
// kArriveFlat blocks share one count, more of them are counted in kArriveGroups groups, each on a line of its own, whose last
// blocks are counted in turn.  All counts are 0 again when the launch is over.
constexpr uint32_t kArriveFlat = 48, kArriveGroups = 32, kArriveLine = 32;           // (words between counts)
constexpr size_t kArriveBytes = (kArriveGroups + 1) * kArriveLine * sizeof(uint32_t);
__device__ __forceinline__ void leave_sum(double *p, double v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double left_sum(const double *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// One wavefront, whose lanes have left the block's sums: whether this is the last block.
__device__ __forceinline__ bool arrives_last(uint32_t *counts)
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0);               // the sums are written through before a count says so
    uint32_t last = 0;
    if ((threadIdx.x & 63u) == 0) {
        const uint32_t blocks = gridDim.x, groups = blocks <= kArriveFlat ? 1u : kArriveGroups, g = blockIdx.x % groups;
        const uint32_t members = (blocks - g + groups - 1u) / groups;
        uint32_t *mine = counts + (1u + g) * kArriveLine;
        last = __hip_atomic_fetch_add(mine, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == members - 1u;
        if (last) {
            __hip_atomic_store(mine, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (groups > 1u) {
                last = __hip_atomic_fetch_add(counts, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == groups - 1u;
                if (last) __hip_atomic_store(counts, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");       // (the sums are read past the caches, but not before the count)
    return __builtin_amdgcn_readfirstlane((int)last) != 0;
}

// ---- values of 32 and 16 bits ---------------------------------------------------------------------------------------
template <class T, int N> struct VecOf;
#define MC_VEC(T, N, ALIGN) template <> struct VecOf<T, N> { typedef T type __attribute__((ext_vector_type(N), aligned(ALIGN))); }
MC_VEC(float, 4, 4);
MC_VEC(__bf16, 4, 2);
MC_VEC(__bf16, 8, 2);
MC_VEC(_Float16, 4, 2);
MC_VEC(_Float16, 8, 2);
#undef MC_VEC

// N consecutive elements from p + i, of those from `lo` to `hi` (the others: 0).  STREAM: not to be kept in the caches.
template <int N, class T, bool STREAM = true>
__device__ __forceinline__ void load_some(global_ptr<const T> p, int32_t i, int32_t lo, int32_t hi, float (&v)[N])
{
    typedef typename VecOf<T, N>::type vec;
    if (i >= lo && i + N <= hi) {
        const global_ptr<const vec> q = (global_ptr<const vec>)(p + i);
        const vec x = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (float)x[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = i + e >= lo && i + e < hi ? (float)p[i + e] : 0.0f;
    }
}
template <int N, class T>
__device__ __forceinline__ void store_some(global_ptr<T> p, int32_t i, int32_t lo, int32_t hi, const float (&v)[N])
{
    typedef typename VecOf<T, N>::type vec;
    if (i >= lo && i + N <= hi) {
        vec x;
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = (T)v[e];
        __builtin_nontemporal_store(x, (global_ptr<vec>)(p + i));
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) if (i + e >= lo && i + e < hi) p[i + e] = (T)v[e];
    }
}

}  // namespace mc
