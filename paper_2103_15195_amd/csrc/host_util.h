// What the host sides of the operators around a step share: types, errors, memory on a handle's device, and whether arguments overlap.
#pragma once
#include <cmath>

#include "step_internal.h"

namespace mc {

inline bool known(int32_t dtype) { return dtype == MC_DTYPE_F32 || dtype == MC_DTYPE_BF16 || dtype == MC_DTYPE_F16; }
inline uintptr_t size_of(int32_t dtype) { return dtype == MC_DTYPE_F32 ? 4u : 2u; }
inline bool off(const void *p, uintptr_t align) { return (reinterpret_cast<uintptr_t>(p) & (align - 1u)) != 0; }
inline int launched() { return hipGetLastError() == hipSuccess ? MC_OK : MC_ERR_DEVICE; }
inline LaunchCtx on(void *stream)
{
    (void)hipGetLastError();
    return LaunchCtx{static_cast<hipStream_t>(stream), nullptr, nullptr, nullptr};
}

// The kernels' numbers of one AdamW update; false: an argument that mc_adamw refuses.
inline bool adamw_args(const mc_adamw_config *c, const float *coef, AdamwArgs &a)
{
    if (!c || off(coef, 4) || c->step < 1) return false;
    if (!(c->beta1 >= 0.0 && c->beta1 < 1.0 && c->beta2 >= 0.0 && c->beta2 < 1.0 && c->eps > 0.0 && std::isfinite(c->eps))) return false;
    if (!(c->lr >= 0.0 && std::isfinite(c->lr) && c->weight_decay >= 0.0 && std::isfinite(c->weight_decay))) return false;
    a.coef = coef;
    a.beta1 = (float)c->beta1; a.one_minus_beta1 = (float)(1.0 - c->beta1);
    a.beta2 = (float)c->beta2; a.one_minus_beta2 = (float)(1.0 - c->beta2);
    a.decay = (float)(1.0 - c->lr * c->weight_decay);
    a.rate = (float)(c->lr / (1.0 - std::pow(c->beta1, (double)c->step)));
    a.root = (float)(1.0 / std::sqrt(1.0 - std::pow(c->beta2, (double)c->step)));
    a.eps = (float)c->eps;
    // (an eps of 0 there would make 0 / 0 of what has never had a gradient, an infinite rate 0 * infinity)
    return a.eps > 0.0f && std::isfinite(a.eps) && std::isfinite(a.decay) && std::isfinite(a.rate) && std::isfinite(a.root);
}

struct OnDevice {                         // makes a handle's device current where something is freed
    int prev = -1;
    bool switched = false;
    explicit OnDevice(int device)
    {
        if (hipGetDevice(&prev) == hipSuccess && prev != device) switched = hipSetDevice(device) == hipSuccess;
    }
    ~OnDevice() { if (switched) (void)hipSetDevice(prev); }
};

template <class T>
inline int grab(T **p, size_t bytes)
{
    void *q = nullptr;
    if (hipMalloc(&q, bytes) != hipSuccess) { (void)hipGetLastError(); return MC_ERR_ALLOC; }
    *p = static_cast<T *>(q);
    return MC_OK;
}

inline int grab_counts(uint32_t **p)
{
    const int rc = grab(p, kArriveBytes);
    if (rc != MC_OK) return rc;
    // (done before work on any stream)
    return hipMemset(*p, 0, kArriveBytes) == hipSuccess && hipDeviceSynchronize() == hipSuccess ? MC_OK : MC_ERR_DEVICE;
}

// ---- whether two things in memory share a byte
struct Extent {
    uintptr_t at;
    uint64_t bytes;
};
inline Extent extent(const void *p, uint64_t bytes) { return {reinterpret_cast<uintptr_t>(p), p ? bytes : 0u}; }
inline bool meet(Extent a, Extent b) { return a.bytes && b.bytes && a.at < b.at + b.bytes && b.at < a.at + a.bytes; }
// The rows of a matrix: `rows` of them, `bytes` each (not 0), `step` from one to the next.
struct RowsAt {
    uintptr_t at;
    uint64_t rows, bytes, step;
    // (a step that no address space holds stands for all longer ones, so that sums of an address and a step stay below 2^64)
    RowsAt(const void *p, int64_t n, int64_t vocab, int64_t stride, uintptr_t size)
        : at(reinterpret_cast<uintptr_t>(p)), rows(p ? (uint64_t)n : 0u), bytes((uint64_t)vocab * size), step((uint64_t)(stride < (int64_t(1) << 58) ? stride : int64_t(1) << 58) * size) {}
    Extent all() const { return {at, rows ? (rows > (uint64_t(1) << 62) / step ? uint64_t(1) << 62 : (rows - 1u) * step) + bytes : 0u}; }
};
inline bool meet(Extent a, const RowsAt &m)
{
    if (!meet(a, m.all())) return false;
    const uint64_t k = a.at > m.at ? (a.at - m.at) / m.step : 0u;                 // the last row that begins at a or before it, or the first
    return meet(a, Extent{m.at + k * m.step, m.bytes}) || (k + 1u < m.rows && meet(a, Extent{m.at + (k + 1u) * m.step, m.bytes}));
}
// (of as many rows)
inline bool meet(const RowsAt &a, const RowsAt &b)
{
    if (!meet(a.all(), b.all())) return false;
    if (a.step != b.step) {            // (and in one another's reach: no layout that a program would choose)
        for (uint64_t k = 0; k < a.rows; ++k) if (meet(Extent{a.at + k * a.step, a.bytes}, b)) return true;
        return false;
    }
    // rows of one step lie on each other where the distance of the two is closer to a multiple of it than a row is long
    const uint64_t distance = a.at > b.at ? a.at - b.at : b.at - a.at, k = distance / a.step, behind = distance % a.step;
    return (k < a.rows && behind < a.bytes) || (k + 1u < a.rows && a.step - behind < a.bytes);
}

}  // namespace mc
