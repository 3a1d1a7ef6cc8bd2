// Kernels over rows of logits: token log-probabilities, and the clipped policy loss with its gradient.
#include "step_internal.h"

namespace mc {

constexpr float kNone = -__builtin_inff();

// exp((x - top) / temperature) for logits of type T.  The difference comes first, so that a row of nothing but the type's lowest
// value is as good as any other.  With logits of 32 bits the factor has a second part: rounded to 24 bits it moves
// exp(-10) by 4e-7 (the product with it is kept finite: an infinite one of the other sign would make NaN of the sum).
template <class T>
__device__ __forceinline__ float row_exp(const LossArgs &a, float x, float top)
{
    const float d = x - top;
    if constexpr (sizeof(T) < 4) return __builtin_amdgcn_exp2f(d * a.to_base2);
    return __builtin_amdgcn_exp2f(__builtin_fmaf(d, a.to_base2, fmaxf(d, a.least) * a.to_base2_rest));
}
// where a maximum of minus infinity (nothing seen so far) stands for exponents: any finite number
__device__ __forceinline__ float base_of(float top) { return top == kNone ? 0.0f : top; }
// log(x), x >= 0, beyond binary32: the exponent and the logarithm of what is between 1/2 and 1
__device__ __forceinline__ double log_wide(float x)
{
    if (!(x > 0.0f && x < __builtin_inff())) return (double)logf(x);
    int e;
    const float f = frexpf(x, &e);
    return (double)e * 0.693147180559945309 + (double)logf(f);
}

// What a row is besides its logits, all asked for at once.  Where a wavefront has one row, this comes through the scalar cache and stays in scalar
// registers.
struct Row {
    int64_t label;
    float weight, adv, old, ref;
    __device__ __forceinline__ bool valid(const LossArgs &a) const { return label >= 0 && label < (int64_t)a.vocab; }
    __device__ __forceinline__ bool taken(const LossArgs &a) const { return valid(a) && weight != 0.0f; }
};
template <bool ONE, class T>
__device__ __forceinline__ T of_row(const T *p, uint32_t r)
{
    if constexpr (ONE) return ld_uniform(p + r);
    return in_global(p)[r];
}
template <bool LOSS, bool ONE>
__device__ __forceinline__ Row row_of(const LossArgs &a, uint32_t r)
{
    Row row{of_row<ONE>(a.labels, r), 1.0f, 0.0f, 0.0f, 0.0f};
    if (LOSS) {
        row.adv = of_row<ONE>(a.advantages, r);
        row.old = of_row<ONE>(a.old_logp, r);
        if (a.weights) row.weight = of_row<ONE>(a.weights, r);
        if (a.ref_logp) row.ref = of_row<ONE>(a.ref_logp, r);
    }
    return row;
}

// exp(d) - d - 1, with em = exp(d) - 1: near 0, where the difference would be d^2 / 2 of two numbers of size d, by its series (of which
// the first term left out is less than a twentieth of a unit in the last place).
__device__ __forceinline__ float kl_term(float d, float em)
{
    float p = 1.0f / 362880.0f;
    for (const float c : {1.0f / 40320.0f, 1.0f / 5040.0f, 1.0f / 720.0f, 1.0f / 120.0f, 1.0f / 24.0f, 1.0f / 6.0f, 0.5f}) p = __builtin_fmaf(p, d, c);
    return fabsf(d) < 0.5f ? d * d * p : em - d;
}
// What a row adds to the sums, and the slope of its loss by its log-probability l.
struct RowTerms { float policy, kl, slope; bool cut; };
__device__ __forceinline__ RowTerms row_terms(const LossArgs &a, const Row &row, double l)
{
    RowTerms t;
    const float adv = row.adv, rho = expf((float)(l - (double)row.old));
    // (without an advantage 0 times the ratio, which may be beyond binary32)
    const float free = adv == 0.0f && rho > a.hi ? 0.0f : -adv * rho, held = -adv * fminf(fmaxf(rho, a.lo), a.hi);
    const bool is_free = !(free < held);              // (NaN: the ratio's)
    t.policy = is_free ? free : held;
    t.slope = is_free ? free : 0.0f;
    t.cut = !is_free;
    t.kl = 0.0f;
    if (a.ref_logp) {
        const float d = (float)((double)row.ref - l), em = expm1f(d);
        t.kl = kl_term(d, em);
        t.slope -= a.kl_coef * em;
    }
    return t;
}

// ---- sums over rows ---------------------------------------------------------------------------------------------------
// The rows' kernels leave a Term for every row.  In launches of few threads the last block adds them up; in larger ones, where that
// block would find thousands of them and every block would wait for its terms to be written through, a kernel behind them does (4.6 us of its own).
struct Sums {
    double at[4] = {};           // weight times policy term, KL term, whether the clamp decides, 1
    uint32_t taken = 0, left_out = 0;
    __device__ __forceinline__ void add(const Term &t)
    {
        const bool is_taken = t.kind == TERM_FREE || t.kind == TERM_CUT;
        const double w = is_taken ? (double)t.weight : 0.0;
        at[0] = __builtin_fma(w, is_taken ? (double)t.policy : 0.0, at[0]);
        at[1] = __builtin_fma(w, is_taken ? (double)t.kl : 0.0, at[1]);
        at[2] += t.kind == TERM_CUT ? w : 0.0;
        at[3] += w;
        taken += is_taken;
        left_out += t.kind == TERM_LEFT_OUT;
    }
    // Over a wavefront, the sum with the number sum_of_lane() in every lane.  Lanes hand each other half of what they have, and go on with the other half.
    __device__ __forceinline__ double join()
    {
        const bool odd = threadIdx.x & 1u, odd2 = threadIdx.x & 2u;
        double a = (odd ? at[2] : at[0]) + __shfl_xor(odd ? at[0] : at[2], 1, 64), b = (odd ? at[3] : at[1]) + __shfl_xor(odd ? at[1] : at[3], 1, 64);
        a = (odd2 ? b : a) + __shfl_xor(odd2 ? a : b, 2, 64);
#pragma unroll
        for (int m = 4; m <= 32; m <<= 1) a += __shfl_xor(a, m, 64);
        taken = wave_sum_u32(taken);
        left_out = wave_sum_u32(left_out);
        return a;
    }
};
__device__ __forceinline__ uint32_t sum_of_lane() { return (threadIdx.x & 1u) * 2u + (threadIdx.x >> 1 & 1u); }
// by a wavefront whose lane k < 4 has sum k, and lane 0 the counts
__device__ __forceinline__ void put_sums(const LossArgs &a, double sum, uint32_t taken, uint32_t left_out)
{
    const double policy = __shfl(sum, 0, 64), kl = __shfl(sum, 1, 64);
    if (threadIdx.x < 4u) a.sums[1u + threadIdx.x] = (float)sum;
    if (threadIdx.x != 0) return;
    a.sums[0] = (float)(a.ref_logp ? policy + (double)a.kl_coef * kl : policy);
    a.sums[5] = __int_as_float((int)taken);
    a.sums[6] = __int_as_float((int)left_out);
    a.sums[7] = 0.0f;
}
// a term past the caches, to a block that may sit on another die, and there
__device__ __forceinline__ void leave_term(Term *to, const Term &t)
{
    uint64_t from[2], *p = reinterpret_cast<uint64_t *>(to);
    __builtin_memcpy(from, &t, sizeof t);
    __hip_atomic_store(p, from[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(p + 1, from[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Term left_term(const Term *from)
{
    const uint64_t *p = reinterpret_cast<const uint64_t *>(from);
    const uint64_t x[2] = {__hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), __hip_atomic_load(p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)};
    Term t;
    __builtin_memcpy(&t, x, sizeof t);
    return t;
}
// By all of a block's threads, behind their rows: the last block adds up the terms of all.  In launches of at most so many threads over at most so many
// rows.  (So and by a kernel behind, us: 600 x 8000 bf16 8.9 and 12.0, 4096 x 1000 10.3 and 12.0, 512 x 32000 14.4 and 14.8; beyond the
// lines 1024 x 32000 25.8 and 23.7, 1024 x 16000 17.6 and 16.3, 8192 x 1000 15.3 and 12.5, 16384 x 100 17.2 and 12.1, but 2048 x 8000 15.6 and 16.0.)
constexpr uint64_t kFewThreads = 1u << 19;
constexpr uint32_t kFewRows = 4096;
static bool sums_here(const LossArgs &a, uint32_t blocks, uint32_t threads) { return (uint64_t)blocks * threads <= kFewThreads && a.rows <= kFewRows && !a.more; }
template <int THREADS>
__device__ __forceinline__ void sum_here(const LossArgs &a)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ double lds[WAVES][kLossSums];
    __shared__ uint32_t last;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0);               // each wavefront for the term that it has left: the barrier does not wait for stores
    __syncthreads();
    if (threadIdx.x < 64u) {
        const bool mine = arrives_last(a.counts);
        if (threadIdx.x == 0) last = mine;
    }
    __syncthreads();
    if (!last) return;
    const uint32_t lane = threadIdx.x & 63u;
    Sums s;
    for (uint32_t i = threadIdx.x; i < a.rows; i += THREADS * 4u) {
        Term t[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) if (i + (uint32_t)(THREADS * k) < a.rows) t[k] = left_term(a.terms + i + (uint32_t)(THREADS * k)); else t[k].kind = TERM_NONE;
#pragma unroll
        for (int k = 0; k < 4; ++k) s.add(t[k]);
    }
    const double mine = s.join();
    double *w = lds[threadIdx.x >> 6];
    if (lane < 4u) w[sum_of_lane()] = mine;
    if (lane == 0) { w[4] = (double)s.taken; w[5] = (double)s.left_out; }
    __syncthreads();
    if (threadIdx.x >= 64u) return;
    double sum = 0.0;
    if (lane < (uint32_t)kLossSums)
#pragma unroll
        for (int k = 0; k < WAVES; ++k) sum += lds[k][lane];
    const uint32_t taken = (uint32_t)__shfl(sum, 4, 64), left_out = (uint32_t)__shfl(sum, 5, 64);
    put_sums(a, sum, taken, left_out);
}
// A block for every kTermBlock rows, all of whose terms it asks for at once.  The sums of the rows of earlier launches stand behind the parts.
constexpr int kTermThreads = 512;
__global__ __launch_bounds__(kTermThreads) void loss_sums_k(LossArgs a)
{
    constexpr int EACH = kTermBlock / kTermThreads, WAVES = kTermThreads / 64;
    __shared__ double lds[WAVES][kLossSums];
    const uint32_t first = blockIdx.x * kTermBlock + threadIdx.x, lane = threadIdx.x & 63u;
    Term t[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) if (first + (uint32_t)(kTermThreads * k) < a.rows) t[k] = a.terms[first + (uint32_t)(kTermThreads * k)]; else t[k].kind = TERM_NONE;
    Sums s;
#pragma unroll
    for (int k = 0; k < EACH; ++k) s.add(t[k]);
    const double mine = s.join();
    double *w = lds[threadIdx.x >> 6];
    if (lane < 4u) w[sum_of_lane()] = mine;
    if (lane == 0) { w[4] = (double)s.taken; w[5] = (double)s.left_out; }
    __syncthreads();
    if (threadIdx.x >= 64u) return;
    const bool has = lane < (uint32_t)kLossSums;
    double sum = 0.0;
    if (has)
#pragma unroll
        for (int k = 0; k < WAVES; ++k) sum += lds[k][lane];
    double *behind = a.partial + (size_t)kLossSums * kLossPartials;
    if (gridDim.x > 1u) {
        if (has) leave_sum(a.partial + (size_t)lane * kLossPartials + blockIdx.x, sum);
        if (!arrives_last(a.counts)) return;
        sum = 0.0;
        for (uint32_t i = 0; has && i < gridDim.x; i += 16u) {
            double x[16];
#pragma unroll
            for (uint32_t k = 0; k < 16u; ++k) x[k] = i + k < gridDim.x ? left_sum(a.partial + (size_t)lane * kLossPartials + i + k) : 0.0;
#pragma unroll
            for (uint32_t k = 0; k < 16u; ++k) sum += x[k];
        }
    }
    if (has && a.more) sum += behind[lane];
    if (has) behind[lane] = sum;
    const uint32_t taken = (uint32_t)__shfl(sum, 4, 64), left_out = (uint32_t)__shfl(sum, 5, 64);
    put_sums(a, sum, taken, left_out);
}

// ---- rows that fit the registers of those who share them ----------------------------------------------------------------
// 16 bytes of a row, and its elements.
template <class T> struct Raw;
template <> struct Raw<float> {
    static constexpr int N = 4;
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
    float x[4];
    __device__ __forceinline__ void none() { for (int e = 0; e < N; ++e) x[e] = kNone; }
    __device__ __forceinline__ void take(vec v) { for (int e = 0; e < N; ++e) x[e] = v[e]; }
    __device__ __forceinline__ void load(global_ptr<const float> p) { take(__builtin_nontemporal_load((global_ptr<const vec>)p)); }
    __device__ __forceinline__ void load_cached(global_ptr<const float> p) { take(*(global_ptr<const vec>)p); }
    __device__ __forceinline__ float at(int e) const { return x[e]; }
    __device__ __forceinline__ void forget() { for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(x[e])); }
};
// The largest of values seen.
template <class T> struct Largest;
template <> struct Largest<float> {
    float top = kNone;
    __device__ __forceinline__ void see(const Raw<float> &r) { top = fmaxf(fmaxf(fmaxf(top, r.x[0]), r.x[1]), fmaxf(r.x[2], r.x[3])); }
    __device__ __forceinline__ float get() const { return top; }
};
// Of 16 bits, two to a word.  Read as integers, values from 0 on are in order, and those below 0 in reverse and below all
// others: the largest signed integer if that is not below 0, else the smallest unsigned one.  That takes two packed
// instructions for two elements, and no conversion.
typedef short short2v __attribute__((ext_vector_type(2)));
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
template <class T> struct Raw {
    static constexpr int N = 8;
    typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
    uint32_t x[4];
    // what has been computed from the elements so far is not kept for later (it would take twice the registers)
    __device__ __forceinline__ void forget() { for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(x[e])); }
    static constexpr uint32_t kNoneBits = std::is_same_v<T, __bf16> ? 0xFF80FF80u : 0xFC00FC00u;
    __device__ __forceinline__ void none() { for (int e = 0; e < 4; ++e) x[e] = kNoneBits; }
    __device__ __forceinline__ void take(vec v) { for (int e = 0; e < 4; ++e) x[e] = v[e]; }
    __device__ __forceinline__ void load(global_ptr<const T> p) { take(__builtin_nontemporal_load((global_ptr<const vec>)p)); }
    __device__ __forceinline__ void load_cached(global_ptr<const T> p) { take(*(global_ptr<const vec>)p); }
    __device__ __forceinline__ float at(int e) const
    {
        if constexpr (std::is_same_v<T, __bf16>) return __uint_as_float(e & 1 ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16);
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(e & 1 ? x[e >> 1] >> 16 : x[e >> 1]));
    }
};
template <class T> struct Largest {
    short2v high = {-32768, -32768};
    ushort2v low = {65535, 65535};
    __device__ __forceinline__ void see(const Raw<T> &r)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            high = __builtin_elementwise_max(high, __builtin_bit_cast(short2v, r.x[e]));
            low = __builtin_elementwise_min(low, __builtin_bit_cast(ushort2v, r.x[e]));
        }
    }
    __device__ __forceinline__ float get() const
    {
        const short h = high[0] > high[1] ? high[0] : high[1];
        const unsigned short l = low[0] < low[1] ? low[0] : low[1];
        return (float)__builtin_bit_cast(T, h >= 0 ? (unsigned short)h : l);
    }
};

// Over the SHARE (or, of more than a wavefront, 64) lanes that share a row.
template <int SHARE>
__device__ __forceinline__ float share_max(float x)
{
#pragma unroll
    for (int m = (SHARE < 64 ? SHARE : 64) / 2; m >= 1; m >>= 1) x = fmaxf(x, __shfl_xor(x, m, 64));
    return x;
}
template <int SHARE>
__device__ __forceinline__ float share_sum(float x)
{
#pragma unroll
    for (int m = (SHARE < 64 ? SHARE : 64) / 2; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
    return x;
}

// Where a row's vectors lie.  They are counted from the boundary (a.line bytes: a cache line, or 16) before the row of logits, so that a wavefront's
// accesses go to whole lines wherever a row begins (those of the gradient too where it is laid out like the logits; by the gradient's own
// boundary, the sums of a call without it would have other last bits).  What is left of the row before its first whole vector
// and behind its last, fewer than N elements each, is its edge, an element each for lanes 0 to 7 and 8 to 15.
template <class T>
struct RowSpan {
    static constexpr uint32_t N = 16 / sizeof(T);
    int32_t shift;               // elements between the boundary and the row
    uint32_t first, end;         // the whole vectors' numbers
    uint32_t edge;               // this lane's edge element, or vocab
    __device__ __forceinline__ RowSpan(const LossArgs &a, uintptr_t at, uint32_t lane)
    {
        shift = (int32_t)(((uint32_t)at & (a.line - 1u)) / (uint32_t)sizeof(T));
        first = ((uint32_t)shift + N - 1u) / N;
        end = ((uint32_t)shift + a.vocab) / N;
        const uint32_t head = min(first * N - (uint32_t)shift, a.vocab);         // (first may lie behind end: a row inside one vector)
        const uint32_t tail = end > first ? end * N - (uint32_t)shift : head;
        edge = lane < 8u ? (lane < head ? lane : a.vocab) : lane < 16u ? min(tail + lane - 8u, a.vocab) : a.vocab;
    }
    // the lane that has an element
    template <int SHARE>
    __device__ __forceinline__ uint32_t owner(uint32_t i) const
    {
        const uint32_t head = first * N - (uint32_t)shift, v = (i + (uint32_t)shift) / N;
        return i < head ? i : v < end ? v % SHARE : 8u + i - (end > first ? end * N - (uint32_t)shift : head);
    }
};

// SHARE threads to a row, each with up to NV 16-byte vectors of it, which are read once, and perhaps an element of its edge.
// KEEP: the exponentials stay in registers between the sum and the gradient, else the logits do.  HERE: the last block adds up
// the rows' terms.  Rows of one wavefront or less share a block of kBlock threads; those of more have one to themselves, since they meet at a barrier.
template <int SHARE> constexpr int held_threads() { return SHARE <= 64 ? kBlock : SHARE; }
template <class T, int SHARE, int NV, bool KEEP, bool LOSS, bool HERE>
__global__ __launch_bounds__(held_threads<SHARE>(), NV <= 4 || SHARE <= 512 ? 8 : 4) void loss_held_k(LossArgs a)
{
    constexpr int THREADS = held_threads<SHARE>(), N = Raw<T>::N, WAVES = SHARE / 64;
    constexpr bool ONE = SHARE >= 64;
    typedef typename VecOf<T, N>::type out_vec;
    __shared__ float at[2 * WAVES + 1];
    const uint32_t lane = threadIdx.x % SHARE, mine = threadIdx.x / SHARE;
    const uint32_t r = blockIdx.x * (THREADS / SHARE) + (ONE ? (uint32_t)__builtin_amdgcn_readfirstlane(mine) : mine);
    auto body = [&] {
        const Row row = row_of<LOSS, ONE>(a, r);
        const T *rx = static_cast<const T *>(a.logits) + (int64_t)r * a.stride;
        T *rd = static_cast<T *>(a.dlogits) + (int64_t)r * a.dstride;
        const bool slopes = LOSS && a.dlogits != nullptr;
        const RowSpan<T> span(a, (uintptr_t)rx, lane);
        const global_ptr<const T> x = in_global(rx);
        const global_ptr<T> dx = in_global(rd);
        auto whole = [&](int k) { const uint32_t i = (uint32_t)k * SHARE + lane; return i >= span.first && i < span.end; };
        auto place = [&](int k) { return (int64_t)((uint32_t)k * SHARE + lane) * N - span.shift; };
        auto put = [&](const Term &t) { if (HERE) leave_term(a.terms + r, t); else a.terms[r] = t; };
        if (!row.taken(a)) {
            if (lane == 0) {
                if (LOSS) put({0.0f, 0.0f, row.weight, row.weight != 0.0f ? (uint32_t)TERM_LEFT_OUT : (uint32_t)TERM_NONE});
                if (a.logp) a.logp[r] = 0.0f;
            }
            if (slopes) {
                const out_vec zero = {};
#pragma unroll
                for (int k = 0; k < NV; ++k) if (whole(k)) __builtin_nontemporal_store(zero, (global_ptr<out_vec>)(dx + place(k)));
                if (span.edge < a.vocab) dx[span.edge] = (T)0.0f;
            }
            return;
        }
        Raw<T> raw[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) if (whole(k)) raw[k].load(x + place(k)); else raw[k].none();
        const float edge = span.edge < a.vocab ? (float)x[span.edge] : kNone;
        float xa = (float)x[row.label];
        Largest<T> seen;
#pragma unroll
        for (int k = 0; k < NV; ++k) seen.see(raw[k]);
        const float wtop = share_max<SHARE>(fmaxf(seen.get(), edge)), wbase = base_of(wtop);
        if (sizeof(T) < 4)
#pragma unroll
            for (int k = 0; k < NV; ++k) raw[k].forget();
        float e[KEEP ? NV * N : 1], sum = row_exp<T>(a, edge, wbase);
        const float eedge = sum;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float y = row_exp<T>(a, raw[k].at(j), wbase);
                if (KEEP) e[k * N + j] = y;
                sum += y;
            }
        sum = share_sum<SHARE>(sum);
        // The wavefronts' maxima and sums, and the label's logit as the first wavefront has read it: where the gradient takes the
        // logits' place, another one may have overwritten it behind the barrier.
        float top = wbase, part = 1.0f;
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63u) == 0) { at[lane >> 6] = wtop; at[WAVES + (lane >> 6)] = sum; }
            if (lane == 0) at[2 * WAVES] = xa;
            __syncthreads();
            xa = at[2 * WAVES];
            const float m = at[lane % WAVES];
            top = base_of(share_max<WAVES>(m));
            sum = share_sum<WAVES>(at[WAVES + lane % WAVES] * row_exp<T>(a, m, top));
            part = row_exp<T>(a, wtop, top);
        }
        const double l = ((double)xa - (double)top) * a.inv_t - log_wide(sum);
        if (lane == 0 && a.logp) a.logp[r] = (float)l;
        if (!LOSS) return;
        const RowTerms t = row_terms(a, row, l);
        if (lane == 0) put({t.policy, t.kl, row.weight, t.cut ? (uint32_t)TERM_CUT : (uint32_t)TERM_FREE});
        if (!slopes) return;
        const float slope = row.weight * t.slope * a.gscale;
        part *= -slope / sum;
        if (!KEEP)
#pragma unroll
            for (int k = 0; k < NV; ++k) raw[k].forget();
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            out_vec v;
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = (T)(part * (KEEP ? e[k * N + j] : row_exp<T>(a, raw[k].at(j), wbase)));
            if (whole(k)) __builtin_nontemporal_store(v, (global_ptr<out_vec>)(dx + place(k)));
        }
        if (span.edge < a.vocab) dx[span.edge] = (T)(part * eedge);
        // the label's own element, by the thread that has stored it with the others
        if (lane == span.template owner<SHARE>((uint32_t)row.label)) dx[row.label] = (T)(part * row_exp<T>(a, xa, wbase) + slope);
    };
    if (r < a.rows) body();
    if (HERE) sum_here<THREADS>(a);
}

// ---- longer rows --------------------------------------------------------------------------------------------------------------
// As above, by 1024 threads, of which each holds NV vectors; what lies behind those is read twice, by way of the caches: with a block to a compute
// unit, 256 rows of 400 KB are under way, and what is read again of them stays in the last-level cache.  1024 rows of 200001 bf16 138 us, 256 of 262144
// fp32 97 (with 8 vectors held 147 and 97, two read ahead instead of four 144 and 97; 256 threads that held nothing 245 and 333).
template <class T, bool LOSS, bool HERE>
__global__ __launch_bounds__(1024, LOSS ? 4 : 8) void loss_long_k(LossArgs a)
{
    constexpr int SHARE = 1024, NV = LOSS ? 16 : 4, AHEAD = 4, N = Raw<T>::N, WAVES = SHARE / 64;
    typedef typename VecOf<T, N>::type out_vec;
    __shared__ float at[2 * WAVES + 1];
    const uint32_t lane = threadIdx.x, r = blockIdx.x;
    auto body = [&] {
        const Row row = row_of<LOSS, true>(a, r);
        const T *rx = static_cast<const T *>(a.logits) + (int64_t)r * a.stride;
        T *rd = static_cast<T *>(a.dlogits) + (int64_t)r * a.dstride;
        const bool slopes = LOSS && a.dlogits != nullptr;
        const RowSpan<T> span(a, (uintptr_t)rx, lane);
        const global_ptr<const T> x = in_global(rx);
        const global_ptr<T> dx = in_global(rd);
        auto place = [&](uint32_t i) { return (int64_t)i * N - span.shift; };
        auto put = [&](const Term &t) { if (HERE) leave_term(a.terms + r, t); else a.terms[r] = t; };
        if (!row.taken(a)) {
            if (lane == 0) {
                if (LOSS) put({0.0f, 0.0f, row.weight, row.weight != 0.0f ? (uint32_t)TERM_LEFT_OUT : (uint32_t)TERM_NONE});
                if (a.logp) a.logp[r] = 0.0f;
            }
            if (slopes) {
                const out_vec zero = {};
                for (uint32_t i = lane; i < span.end; i += SHARE) if (i >= span.first) __builtin_nontemporal_store(zero, (global_ptr<out_vec>)(dx + place(i)));
                if (span.edge < a.vocab) dx[span.edge] = (T)0.0f;
            }
            return;
        }
        Raw<T> raw[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const uint32_t i = (uint32_t)k * SHARE + lane;
            if (i >= span.first && i < span.end) raw[k].load(x + place(i)); else raw[k].none();
        }
        const float edge = span.edge < a.vocab ? (float)x[span.edge] : kNone;
        float xa = (float)x[row.label];
        // the running maximum and sum of what is not held
        float top = kNone, sum = 0.0f;
        for (uint32_t i = (uint32_t)NV * SHARE + lane; i < span.end; i += SHARE * AHEAD) {
            Raw<T> next[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) if (i + SHARE * k < span.end) next[k].load_cached(x + place(i + SHARE * k)); else next[k].none();
            Largest<T> seen;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) seen.see(next[k]);
            const float most = seen.get();
            if (!(most <= top)) { sum *= row_exp<T>(a, top, base_of(most)); top = most; }
            const float base = base_of(top);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) sum += row_exp<T>(a, next[k].at(j), base);
        }
        Largest<T> seen;
#pragma unroll
        for (int k = 0; k < NV; ++k) seen.see(raw[k]);
        const float wtop = share_max<64>(fmaxf(fmaxf(seen.get(), edge), top)), wbase = base_of(wtop);
        const float eedge = row_exp<T>(a, edge, wbase);
        sum = sum * row_exp<T>(a, top, wbase) + eedge;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            raw[k].forget();
#pragma unroll
            for (int j = 0; j < N; ++j) sum += row_exp<T>(a, raw[k].at(j), wbase);
        }
        sum = share_sum<64>(sum);
        if ((threadIdx.x & 63u) == 0) { at[lane >> 6] = wtop; at[WAVES + (lane >> 6)] = sum; }
        if (lane == 0) at[2 * WAVES] = xa;              // (see above)
        __syncthreads();
        xa = at[2 * WAVES];
        const float m = at[lane % WAVES];
        top = base_of(share_max<WAVES>(m));
        sum = share_sum<WAVES>(at[WAVES + lane % WAVES] * row_exp<T>(a, m, top));
        const double l = ((double)xa - (double)top) * a.inv_t - log_wide(sum);
        if (lane == 0 && a.logp) a.logp[r] = (float)l;
        if (!LOSS) return;
        const RowTerms t = row_terms(a, row, l);
        if (lane == 0) put({t.policy, t.kl, row.weight, t.cut ? (uint32_t)TERM_CUT : (uint32_t)TERM_FREE});
        if (!slopes) return;
        const float slope = row.weight * t.slope * a.gscale, part = -slope / sum;
        auto store = [&](uint32_t i, const Raw<T> &v) {
            out_vec o;
#pragma unroll
            for (int j = 0; j < N; ++j) o[j] = (T)(part * row_exp<T>(a, v.at(j), top));
            __builtin_nontemporal_store(o, (global_ptr<out_vec>)(dx + place(i)));
        };
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            raw[k].forget();
            const uint32_t i = (uint32_t)k * SHARE + lane;
            if (i >= span.first && i < span.end) store(i, raw[k]);
        }
        for (uint32_t i = (uint32_t)NV * SHARE + lane; i < span.end; i += SHARE * AHEAD) {
            Raw<T> next[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) if (i + SHARE * k < span.end) next[k].load(x + place(i + SHARE * k));
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) if (i + SHARE * k < span.end) store(i + SHARE * k, next[k]);
        }
        if (span.edge < a.vocab) dx[span.edge] = (T)(part * row_exp<T>(a, edge, top));
        if (lane == span.template owner<SHARE>((uint32_t)row.label)) dx[row.label] = (T)(part * row_exp<T>(a, xa, top) + slope);
    };
    body();
    if (HERE) sum_here<1024>(a);
}

// ---- few rows -----------------------------------------------------------------------------------------------------------------
// A row by as many blocks as it has parts of kPartVecs vectors: each finds its part's maximum and sum, and a second launch, where they
// are joined, reads the part again, which the caches still hold, and writes the gradient.
constexpr int kPartSteps = 4;
constexpr uint32_t kPartVecs = kPartSteps * kBlock;
template <class T>
__global__ __launch_bounds__(kBlock) void loss_parts_k(LossArgs a, uint32_t parts)
{
    __shared__ float at[2 * kWavesPerBlock];
    const uint32_t r = blockIdx.x / parts, part = blockIdx.x % parts, lane = threadIdx.x;
    const Row row = row_of<false, true>(a, r);
    if (!row.valid(a) || (a.weights && ld_uniform(a.weights + r) == 0.0f)) return;
    const T *rx = static_cast<const T *>(a.logits) + (int64_t)r * a.stride;
    const global_ptr<const T> x = in_global(rx);
    const RowSpan<T> span(a, (uintptr_t)rx, lane);
    Raw<T> raw[kPartSteps];
#pragma unroll
    for (int k = 0; k < kPartSteps; ++k) {
        const uint32_t i = part * kPartVecs + (uint32_t)k * kBlock + lane;
        if (i >= span.first && i < span.end) raw[k].load_cached(x + ((int64_t)i * Raw<T>::N - span.shift)); else raw[k].none();
    }
    const float edge = part == 0 && span.edge < a.vocab ? (float)x[span.edge] : kNone;
    if (part == 0 && lane == 0) a.parts[r].label = (float)x[row.label];
    Largest<T> seen;
#pragma unroll
    for (int k = 0; k < kPartSteps; ++k) seen.see(raw[k]);
    const float wtop = share_max<64>(fmaxf(seen.get(), edge)), wbase = base_of(wtop);
    float sum = row_exp<T>(a, edge, wbase);
#pragma unroll
    for (int k = 0; k < kPartSteps; ++k)
#pragma unroll
        for (int j = 0; j < Raw<T>::N; ++j) sum += row_exp<T>(a, raw[k].at(j), wbase);
    sum = share_sum<64>(sum);
    if ((lane & 63u) == 0) { at[lane >> 6] = wtop; at[kWavesPerBlock + (lane >> 6)] = sum; }
    __syncthreads();
    const float m = at[lane % kWavesPerBlock], top = share_max<kWavesPerBlock>(m);
    sum = share_sum<kWavesPerBlock>(at[kWavesPerBlock + lane % kWavesPerBlock] * row_exp<T>(a, m, base_of(top)));
    if (lane == 0) { a.parts[r].top[part] = top; a.parts[r].sum[part] = sum; }
}
// LOSS: a block to a part again; else one to a row.
template <class T, bool LOSS>
__global__ __launch_bounds__(kBlock) void loss_join_k(LossArgs a, uint32_t parts)
{
    constexpr int N = Raw<T>::N;
    typedef typename VecOf<T, N>::type out_vec;
    const uint32_t r = LOSS ? blockIdx.x / parts : blockIdx.x, part = LOSS ? blockIdx.x % parts : 0u, lane = threadIdx.x;
    auto body = [&] {
        const Row row = row_of<LOSS, true>(a, r);
        const T *rx = static_cast<const T *>(a.logits) + (int64_t)r * a.stride;
        T *rd = static_cast<T *>(a.dlogits) + (int64_t)r * a.dstride;
        const bool slopes = LOSS && a.dlogits != nullptr;
        const RowSpan<T> span(a, (uintptr_t)rx, lane);
        const global_ptr<const T> x = in_global(rx);
        const global_ptr<T> dx = in_global(rd);
        auto number = [&](int k) { return part * kPartVecs + (uint32_t)k * kBlock + lane; };
        auto whole = [&](int k) { const uint32_t i = number(k); return i >= span.first && i < span.end; };
        auto place = [&](int k) { return (int64_t)number(k) * N - span.shift; };
        const bool edges = part == 0 && span.edge < a.vocab, first = part == 0 && lane == 0;
        if (!row.taken(a)) {
            if (first && LOSS) leave_term(a.terms + r, {0.0f, 0.0f, row.weight, row.weight != 0.0f ? (uint32_t)TERM_LEFT_OUT : (uint32_t)TERM_NONE});
            if (first && a.logp) a.logp[r] = 0.0f;
            if (slopes) {
                const out_vec zero = {};
#pragma unroll
                for (int k = 0; k < kPartSteps; ++k) if (whole(k)) __builtin_nontemporal_store(zero, (global_ptr<out_vec>)(dx + place(k)));
                if (edges) dx[span.edge] = (T)0.0f;
            }
            return;
        }
        Raw<T> raw[kPartSteps];
        float edge = kNone;
        if (slopes) {
#pragma unroll
            for (int k = 0; k < kPartSteps; ++k) if (whole(k)) raw[k].load(x + place(k)); else raw[k].none();
            if (edges) edge = (float)x[span.edge];
        }
        const PartsOfRow &of = a.parts[r];
        const float xa = of.label, m = (lane & 63u) < parts ? of.top[lane & 63u] : kNone, s = (lane & 63u) < parts ? of.sum[lane & 63u] : 0.0f;
        const float top = base_of(share_max<64>(m)), sum = share_sum<64>(s * row_exp<T>(a, m, top));
        const double l = ((double)xa - (double)top) * a.inv_t - log_wide(sum);
        if (first && a.logp) a.logp[r] = (float)l;
        if (!LOSS) return;
        const RowTerms t = row_terms(a, row, l);
        if (first) leave_term(a.terms + r, {t.policy, t.kl, row.weight, t.cut ? (uint32_t)TERM_CUT : (uint32_t)TERM_FREE});
        if (!slopes) return;
        const float slope = row.weight * t.slope * a.gscale, scale = -slope / sum;
#pragma unroll
        for (int k = 0; k < kPartSteps; ++k) {
            out_vec v;
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = (T)(scale * row_exp<T>(a, raw[k].at(j), top));
            if (whole(k)) __builtin_nontemporal_store(v, (global_ptr<out_vec>)(dx + place(k)));
        }
        if (edges) dx[span.edge] = (T)(scale * row_exp<T>(a, edge, top));
        // the label's own element, by the thread that has stored it with the others
        const uint32_t i = ((uint32_t)row.label + (uint32_t)span.shift) / N;
        const bool in_vector = i >= span.first && i < span.end;
        if (part == (in_vector ? i / kPartVecs : 0u) && lane == span.template owner<kBlock>((uint32_t)row.label)) dx[row.label] = (T)(scale * row_exp<T>(a, xa, top) + slope);
    };
    body();
    if (LOSS) sum_here<kBlock>(a);
}

// ---- launches -----------------------------------------------------------------------------------------------------------------
template <class T, int SHARE, int NV, bool KEEP, bool LOSS>
static bool held(const LaunchCtx &lc, const LossArgs &a)
{
    constexpr uint32_t THREADS = held_threads<SHARE>(), each = THREADS / SHARE;
    const uint32_t blocks = (a.rows + each - 1) / each;
    const bool here = LOSS && sums_here(a, blocks, THREADS);
    launch(here ? loss_held_k<T, SHARE, NV, KEEP, LOSS, LOSS> : loss_held_k<T, SHARE, NV, KEEP, LOSS, false>, dim3(blocks), dim3(THREADS), lc.stream, a);
    return here;
}
// Vectors that the longest row may reach over, counted from a boundary of `line` bytes.
template <class T>
static uint32_t reach(const LossArgs &a, uint32_t line)
{
    const uintptr_t at = (uintptr_t)a.logits, step = (uintptr_t)a.stride * sizeof(T);
    const uintptr_t shift = step % line == 0 || a.rows == 1u ? at % line : line - sizeof(T);
    return (uint32_t)((shift / sizeof(T) + a.vocab) / Raw<T>::N);
}
// At most kTermRows rows; whether their terms are added up.
// Threads to a row, and vectors that each holds: several rows to a wavefront where rows are short (32768 x 200 / 500 / 1000 bf16 with 16, 32 and 64
// threads to a row: 12.9 / 21.5 / 27.9, 15.2 / 19.8 / 31.1 and 19.7 / 22.2 / 27.7 us), then so that few of the threads have less to hold than others, in at most the 64 registers
// that let 32 wavefronts share a compute unit (up to 65536 elements of 16 bits; for longer rows twice those).  80 M logits in rows of 10000 / 12000 / 14000 / 16000 bf16 by
// 1024 threads of two vectors 65 / 57 / 53 / 52 us, by 512 of three or four 51 / 51 / 53 / 53; 2000 / 8000 by 64 / 256 of four 56 / 52, by 128 / 512 of two 55 / 51.
// Without a gradient to write fewer threads with more to read are ahead: rows of 10000 / 16000 by 1024 of two 39 / 28, by 256 of eight 25 / 21.
// Rates of the policy loss in bf16 (TB/s): 4096 x 32064 5.5, 32003 (rows begin anywhere) 5.5, both with one row in eight masked; with 40 %
// masked 4096 x 32064 5.3, 8192 x 8192 5.0, 16384 x 4096 5.1, 32768 x 1000 3.9, 65536 x 100 1.4, 2048 x 65536 5.1, 2048 x 128259 5.3, 1024 x 200001 5.0.
template <class T, bool LOSS>
static bool loss_of(const LaunchCtx &lc, LossArgs a)
{
    a.line = kLine;
    // (A row that would need twice the registers for it, or the next of the forms below, is not moved to a line.  1536 and 3072 are limits of the policy loss
    // alone; the log-probabilities go by the same list.)
    const uint32_t close = reach<T>(a, 16u);
    uint32_t vecs = reach<T>(a, kLine);
    for (uint32_t room : {16u, 32u, 64u, 128u, 256u, 384u, 512u, 768u, 1024u, 1536u, 2048u, 3072u, 4096u, 8192u, 16384u}) if (close <= room && room < vecs) { a.line = 16u; vecs = close; }
    // Few long rows are shared by blocks.  (Policy loss so and with a block to each, us: rows of 128256 bf16, 1 / 64 / 128 / 200 of them 11.4 / 14.0 / 19.1 / 27.0
    // and 19.3 / 21.6 / 22.3 / 24.2; of 262144 fp32 11.4 / 30.3 / 56.8 / 87.9 and 43.5 / 52.2 / 69.8 / 95.8; of 70000 bf16, 64 / 128 / 200 11.6 / 15.0 / 17.6 and
    // 17.9 / 18.1 / 19.0.  Below 8192 vectors the gain is no more than what the host takes for a second launch, which is from 0.5 to 2 us from one machine to another:
    // 1 / 64 of 64000 bf16 11.3 / 11.0 and 12.2 / 14.5, on a slower host 13.5 / 13.3 and 11.8 / 14.0; their log-probabilities alone 7.8 / 7.6 and 6.3 / 7.4.)
    const uint32_t parts = (reach<T>(a, kLine) + kPartVecs - 1u) / kPartVecs;
    if (a.rows <= kPartRows && parts <= kMostParts && vecs > 1024 * 8 && !a.more) {
        a.line = kLine;
        launch(loss_parts_k<T>, dim3(a.rows * parts), dim3(kBlock), lc.stream, a, parts);
        launch(loss_join_k<T, LOSS>, dim3(LOSS ? a.rows * parts : a.rows), dim3(LOSS ? kBlock : 64), lc.stream, a, parts);
        return LOSS;
    }
    if (vecs <= 16 * 1) return held<T, 16, 1, true, LOSS>(lc, a);
    if (vecs <= 16 * 2) return held<T, 16, 2, true, LOSS>(lc, a);
    if (vecs <= 32 * 2) return held<T, 32, 2, true, LOSS>(lc, a);
    if (vecs <= 64 * 2) return held<T, 64, 2, true, LOSS>(lc, a);
    if constexpr (LOSS) {
        if (vecs <= 128 * 2) return held<T, 128, 2, true, LOSS>(lc, a);
        if (vecs <= 128 * 3) return held<T, 128, 3, true, LOSS>(lc, a);
        if (vecs <= 256 * 2) return held<T, 256, 2, true, LOSS>(lc, a);
        if (vecs <= 256 * 3) return held<T, 256, 3, true, LOSS>(lc, a);
        if (vecs <= 512 * 2) return held<T, 512, 2, true, LOSS>(lc, a);
        if (vecs <= 512 * 3) return held<T, 512, 3, true, LOSS>(lc, a);
        if (vecs <= 1024 * 2) return held<T, 1024, 2, true, LOSS>(lc, a);
        if (vecs <= 1024 * 3) return held<T, 1024, 3, true, LOSS>(lc, a);
        if (vecs <= 1024 * 4) return held<T, 1024, 4, true, LOSS>(lc, a);
        if (vecs <= 1024 * 8) return held<T, 1024, 8, false, LOSS>(lc, a);
        if (vecs <= 1024 * 16) return held<T, 1024, 16, false, LOSS>(lc, a);
    } else {
        // (log-probabilities alone are read once in any case: 2048 rows of 128259 62 us held, 56 not)
        if (vecs <= 64 * 4) return held<T, 64, 4, true, LOSS>(lc, a);
        if (vecs <= 128 * 3) return held<T, 128, 3, true, LOSS>(lc, a);
        if (vecs <= 128 * 4) return held<T, 128, 4, true, LOSS>(lc, a);
        if (vecs <= 256 * 3) return held<T, 256, 3, true, LOSS>(lc, a);
        if (vecs <= 256 * 4) return held<T, 256, 4, true, LOSS>(lc, a);
        if (vecs <= 256 * 8) return held<T, 256, 8, false, LOSS>(lc, a);
        if (vecs <= 512 * 8) return held<T, 512, 8, false, LOSS>(lc, a);
    }
    const bool here = LOSS && sums_here(a, a.rows, 1024u);
    launch(here ? loss_long_k<T, LOSS, LOSS> : loss_long_k<T, LOSS, false>, dim3(a.rows), dim3(1024), lc.stream, a);
    return here;
}
// the sums of no rows
__global__ void no_rows_k(float *sums) { if (threadIdx.x < 8u) sums[threadIdx.x] = 0.0f; }

template <bool LOSS>
static void loss_by(const LaunchCtx &lc, int dtype, LossArgs a)
{
    const uintptr_t size = dtype == MC_DTYPE_F32 ? 4u : 2u;
    for (uint32_t left = a.rows; left;) {
        a.rows = left < kTermRows ? left : kTermRows;
        const bool done = dtype == MC_DTYPE_F32 ? loss_of<float, LOSS>(lc, a) : dtype == MC_DTYPE_BF16 ? loss_of<__bf16, LOSS>(lc, a) : loss_of<_Float16, LOSS>(lc, a);
        if (LOSS && !done) launch(loss_sums_k, dim3((a.rows + kTermBlock - 1) / kTermBlock), dim3(kTermThreads), lc.stream, a);
        left -= a.rows;
        a.more = true;
        a.logits = static_cast<const char *>(a.logits) + (int64_t)a.rows * a.stride * size;
        if (a.dlogits) a.dlogits = static_cast<char *>(a.dlogits) + (int64_t)a.rows * a.dstride * size;
        a.labels += a.rows;
        if (a.logp) a.logp += a.rows;
        if (!LOSS) continue;
        a.old_logp += a.rows;
        a.advantages += a.rows;
        if (a.weights) a.weights += a.rows;
        if (a.ref_logp) a.ref_logp += a.rows;
    }
}
void launch_token_logp(const LaunchCtx &lc, int dtype, const LossArgs &a) { loss_by<false>(lc, dtype, a); }
void launch_policy_loss(const LaunchCtx &lc, int dtype, const LossArgs &a)
{
    if (a.rows) loss_by<true>(lc, dtype, a);
    else launch(no_rows_k, dim3(1), dim3(64), lc.stream, a.sums);
}

}  // namespace mc
