// Host side of the C ABI declared in include/mergecomp_step.h: handles, argument checks and launches.
#include <cfloat>
#include <cmath>
#include <new>
#include <vector>

#include "host_util.h"
#include "step_internal.h"

using namespace mc;

struct mc_step {
    int device = 0;
    int32_t grad_dtype = 0, model_dtype = MC_DTYPE_NONE;
    std::vector<int32_t> live;           // tensors that hold elements
    int32_t tensors = 0;
    uint32_t npieces = 0;
    Piece *d_pieces = nullptr;
    uintptr_t *d_addr = nullptr;         // MC_LISTS lists of the live tensors' addresses
    double *d_partial = nullptr;
    uint32_t *d_counts = nullptr;        // 0 between calls
    std::vector<uintptr_t> want;         // a list on its way to the device (reserved at creation)
    bool bound[MC_LISTS] = {};
};
struct mc_loss {
    int device = 0;
    Term *d_terms = nullptr;
    PartsOfRow *d_parts = nullptr;
    double *d_partial = nullptr;
    uint32_t *d_counts = nullptr;        // 0 between calls
};

namespace {

StepView view(const mc_step *h) { return {h->d_pieces, h->d_addr, h->npieces, (uint32_t)h->live.size()}; }
bool ready(const mc_step *h, int32_t list) { return h->bound[list] || h->live.empty(); }

}  // namespace

extern "C" {

int mc_step_destroy(mc_step *h)
{
    if (!h) return MC_ERR_INVALID_ARG;
    {
        OnDevice guard(h->device);
        (void)hipDeviceSynchronize();
        if (h->d_pieces) (void)hipFree(h->d_pieces);
        if (h->d_addr) (void)hipFree(h->d_addr);
        if (h->d_partial) (void)hipFree(h->d_partial);
        if (h->d_counts) (void)hipFree(h->d_counts);
    }
    delete h;
    return MC_OK;
}

int mc_step_create(mc_step **out, const int64_t *numel, int32_t n_tensors, int32_t grad_dtype, int32_t model_dtype, const uint8_t *no_decay)
{
    if (!out) return MC_ERR_INVALID_ARG;
    *out = nullptr;
    if (!numel || n_tensors < 1 || !known(grad_dtype)) return MC_ERR_INVALID_ARG;
    if (model_dtype != MC_DTYPE_NONE && model_dtype != MC_DTYPE_BF16 && model_dtype != MC_DTYPE_F16) return MC_ERR_INVALID_ARG;
    uint64_t pieces = 0;
    for (int32_t t = 0; t < n_tensors; ++t) {
        if (numel[t] < 0) return MC_ERR_INVALID_ARG;
        if (numel[t] >= (int64_t(1) << 39)) return MC_ERR_RANGE;
        pieces += numel[t] ? ((uint64_t)numel[t] + kMostShift + kPiece - 1) / kPiece : 0;
        if (pieces > (uint64_t(1) << 27)) return MC_ERR_RANGE;
    }
    mc_step *h = new (std::nothrow) mc_step();
    if (!h) return MC_ERR_ALLOC;
    if (hipGetDevice(&h->device) != hipSuccess) { (void)hipGetLastError(); delete h; return MC_ERR_DEVICE; }
    int rc = MC_OK;
    try {
        h->grad_dtype = grad_dtype;
        h->model_dtype = model_dtype;
        h->tensors = n_tensors;
        h->npieces = (uint32_t)pieces;
        std::vector<Piece> table;
        table.reserve(pieces);
        for (int32_t t = 0; t < n_tensors; ++t) {
            if (numel[t] == 0) continue;
            const uint32_t name = (uint32_t)h->live.size() | (no_decay && no_decay[t] ? kNoDecay : 0u);
            h->live.push_back(t);
            for (int64_t at = 0, i = 0; at < numel[t] + (int64_t)kMostShift; at += kPiece, ++i)
                table.push_back({name, (uint32_t)i, (int32_t)(numel[t] - at < (int64_t)kPiece ? numel[t] - at : kPiece), 0u});
        }
        h->want.reserve(h->live.size());
        rc = grab(&h->d_partial, kNormBlocks * sizeof(double));
        if (rc == MC_OK) rc = grab_counts(&h->d_counts);
        if (rc == MC_OK && pieces) rc = grab(&h->d_pieces, table.size() * sizeof(Piece));
        if (rc == MC_OK && pieces) rc = grab(&h->d_addr, (size_t)MC_LISTS * h->live.size() * sizeof(uintptr_t));
        if (rc == MC_OK && pieces && hipMemcpy(h->d_pieces, table.data(), table.size() * sizeof(Piece), hipMemcpyHostToDevice) != hipSuccess) rc = MC_ERR_DEVICE;
    } catch (const std::bad_alloc &) {
        rc = MC_ERR_ALLOC;
    }
    if (rc != MC_OK) { (void)hipGetLastError(); mc_step_destroy(h); return rc; }
    *out = h;
    return MC_OK;
}

int mc_step_bind(mc_step *h, int32_t list, const void *const *ptrs, void *stream)
{
    if (!h || !ptrs || list < 0 || list >= MC_LISTS || (list == MC_LIST_MODEL && h->model_dtype == MC_DTYPE_NONE)) return MC_ERR_INVALID_ARG;
    const uintptr_t align = list <= MC_LIST_CLIPPED ? size_of(h->grad_dtype) : list == MC_LIST_MODEL ? size_of(h->model_dtype) : 4u;
    for (int32_t t : h->live) if (!ptrs[t] || off(ptrs[t], align)) return MC_ERR_INVALID_ARG;
    h->want.clear();                                      // (capacity reserved: no allocation)
    for (int32_t t : h->live) h->want.push_back(reinterpret_cast<uintptr_t>(ptrs[t]));
    const LaunchCtx lc = on(stream);
    if (!h->want.empty()) launch_upload_ptrs(lc, h->want.data(), h->d_addr + (size_t)list * h->want.size(), (uint32_t)h->want.size());
    const int rc = launched();
    h->bound[list] = rc == MC_OK;
    return rc;
}

static int norm_args(const mc_step *h, float scale, float max_norm, const float *out)
{
    if (!h || !out || off(out, 4) || !std::isfinite(scale) || !(scale > 0.0f) || !(max_norm > 0.0f)) return MC_ERR_INVALID_ARG;
    return ready(h, MC_LIST_GRADS) ? MC_OK : MC_ERR_INVALID_ARG;
}

int mc_grad_norm(mc_step *h, float scale, float max_norm, float *out, void *stream)
{
    const int rc = norm_args(h, scale, max_norm, out);
    if (rc != MC_OK) return rc;
    launch_grad_norm(on(stream), h->grad_dtype, view(h), h->d_partial, h->d_counts, scale, max_norm, out);
    return launched();
}

int mc_grad_clip(mc_step *h, float scale, float max_norm, float *out, void *stream)
{
    const int rc = norm_args(h, scale, max_norm, out);
    if (rc != MC_OK) return rc;
    const LaunchCtx lc = on(stream);
    launch_grad_norm(lc, h->grad_dtype, view(h), h->d_partial, h->d_counts, scale, max_norm, out);
    launch_grad_clip(lc, h->grad_dtype, view(h), h->bound[MC_LIST_CLIPPED] ? MC_LIST_CLIPPED : MC_LIST_GRADS, out + 1);
    return launched();
}

int mc_adamw(mc_step *h, const mc_adamw_config *c, const float *coef, void *stream)
{
    AdamwArgs a;
    if (!h || !adamw_args(c, coef, a)) return MC_ERR_INVALID_ARG;
    for (int32_t list : {MC_LIST_GRADS, MC_LIST_PARAMS, MC_LIST_EXP_AVG, MC_LIST_EXP_AVG_SQ}) if (!ready(h, list)) return MC_ERR_INVALID_ARG;
    if (h->model_dtype != MC_DTYPE_NONE && !ready(h, MC_LIST_MODEL)) return MC_ERR_INVALID_ARG;
    launch_adamw(on(stream), h->grad_dtype, h->model_dtype, view(h), a);
    return launched();
}

int mc_loss_destroy(mc_loss *h)
{
    if (!h) return MC_ERR_INVALID_ARG;
    {
        OnDevice guard(h->device);
        (void)hipDeviceSynchronize();
        if (h->d_terms) (void)hipFree(h->d_terms);
        if (h->d_parts) (void)hipFree(h->d_parts);
        if (h->d_partial) (void)hipFree(h->d_partial);
        if (h->d_counts) (void)hipFree(h->d_counts);
    }
    delete h;
    return MC_OK;
}

int mc_loss_create(mc_loss **out)
{
    if (!out) return MC_ERR_INVALID_ARG;
    *out = nullptr;
    mc_loss *h = new (std::nothrow) mc_loss();
    if (!h) return MC_ERR_ALLOC;
    if (hipGetDevice(&h->device) != hipSuccess) { (void)hipGetLastError(); delete h; return MC_ERR_DEVICE; }
    int rc = grab(&h->d_partial, (size_t)(kLossPartials + 1) * kLossSums * sizeof(double));
    if (rc == MC_OK) rc = grab(&h->d_terms, (size_t)kTermRows * sizeof(Term));
    if (rc == MC_OK) rc = grab(&h->d_parts, (size_t)kPartRows * sizeof(PartsOfRow));
    if (rc == MC_OK) rc = grab_counts(&h->d_counts);
    if (rc != MC_OK) { mc_loss_destroy(h); return rc; }
    *out = h;
    return MC_OK;
}

static int logits_args(const mc_loss *h, const mc_logits *x, LossArgs &a)
{
    if (!h || !x || !known(x->dtype) || x->rows < 0 || x->vocab < 1 || x->stride < x->vocab) return MC_ERR_INVALID_ARG;
    if (!(x->temperature > 0.0f) || !std::isfinite(x->temperature)) return MC_ERR_INVALID_ARG;
    if (x->rows > 0 && (!x->logits || !x->labels)) return MC_ERR_INVALID_ARG;
    if (off(x->logits, size_of(x->dtype)) || off(x->labels, 8)) return MC_ERR_INVALID_ARG;
    if (x->vocab >= (int64_t(1) << 31) - (1 << 16) || x->rows >= (int64_t(1) << 31)) return MC_ERR_RANGE;
    a = LossArgs{};
    a.logits = x->logits;
    a.labels = x->labels;
    a.stride = x->stride;
    a.rows = (uint32_t)x->rows;
    a.vocab = (uint32_t)x->vocab;
    const double base2 = 1.4426950408889634 / (double)x->temperature;
    a.to_base2 = (float)base2;
    if (!std::isfinite(a.to_base2)) return MC_ERR_INVALID_ARG;          // (a temperature below 4.3e-39)
    a.to_base2_rest = (float)(base2 - (double)a.to_base2);
    // (The first part is at least 2^24 times the second: with a second part above 1 the exponential of a difference beyond this is 0 whatever is
    // added, and with a smaller one nothing finite lies beyond it but the last thousandth of binary32's range.)
    a.least = -(float)(0.999 * FLT_MAX / std::fmax(1.0, std::fabs((double)a.to_base2_rest)));
    a.inv_t = 1.0 / (double)x->temperature;
    a.partial = h->d_partial;
    a.terms = h->d_terms;
    a.parts = h->d_parts;
    a.counts = h->d_counts;
    return MC_OK;
}

int mc_token_logp(mc_loss *h, const mc_logits *x, float *logp, void *stream)
{
    LossArgs a;
    const int rc = logits_args(h, x, a);
    if (rc != MC_OK) return rc;
    if ((a.rows && !logp) || off(logp, 4)) return MC_ERR_INVALID_ARG;
    const Extent to = extent(logp, 4u * (uint64_t)a.rows);
    if (meet(to, extent(x->labels, 8u * (uint64_t)a.rows)) || meet(to, RowsAt(x->logits, x->rows, x->vocab, x->stride, size_of(x->dtype)))) return MC_ERR_INVALID_ARG;
    a.logp = logp;
    launch_token_logp(on(stream), x->dtype, a);
    return launched();
}

// Whether anything that a call writes lies over something else of it.  Wavefronts and blocks that share a row read and write what the row has in no order, so
// that a log-probability in the place of an old one, say, could be taken for it.  The sums come behind the rows whose terms they hold, so they may lie over what
// is read, unless there are more rows to come.
static bool overlaps(const mc_logits *x, const mc_policy *p)
{
    const uint64_t n = (uint64_t)x->rows;
    const Extent logp = extent(p->logp, 4u * n), sums = extent(p->sums, 32u);
    const RowsAt logits(x->logits, x->rows, x->vocab, x->stride, size_of(x->dtype)), slopes(p->dlogits, x->rows, x->vocab, p->dlogits_stride, size_of(x->dtype));
    for (const Extent s : {extent(x->labels, 8u * n), extent(p->old_logp, 4u * n), extent(p->advantages, 4u * n), extent(p->weights, 4u * n), extent(p->ref_logp, 4u * n)})
        if (meet(logp, s) || meet(s, slopes) || (n > kTermRows && meet(sums, s))) return true;
    if (meet(logp, sums) || meet(logp, logits) || meet(logp, slopes) || meet(sums, slopes) || (n > kTermRows && meet(sums, logits))) return true;
    return p->dlogits != x->logits && meet(slopes, logits);
}

int mc_policy_loss(mc_loss *h, const mc_logits *x, const mc_policy *p, void *stream)
{
    LossArgs a;
    const int rc = logits_args(h, x, a);
    if (rc != MC_OK) return rc;
    if (!p || !p->sums || (a.rows && (!p->old_logp || !p->advantages))) return MC_ERR_INVALID_ARG;
    for (const void *q : {(const void *)p->old_logp, (const void *)p->advantages, (const void *)p->weights, (const void *)p->ref_logp, (const void *)p->sums,
                          (const void *)p->logp}) if (off(q, 4)) return MC_ERR_INVALID_ARG;
    if (p->dlogits && (off(p->dlogits, size_of(x->dtype)) || p->dlogits_stride < x->vocab)) return MC_ERR_INVALID_ARG;
    if (p->dlogits == x->logits && p->dlogits && p->dlogits_stride != x->stride) return MC_ERR_INVALID_ARG;
    if (overlaps(x, p)) return MC_ERR_INVALID_ARG;
    if (!(p->clip_low >= 0.0f && p->clip_low <= 1.0f && p->clip_high >= 0.0f && p->kl_coef >= 0.0f)) return MC_ERR_INVALID_ARG;
    if (!std::isfinite(p->clip_high) || !std::isfinite(p->kl_coef) || !std::isfinite(p->grad_scale)) return MC_ERR_INVALID_ARG;
    a.old_logp = p->old_logp; a.advantages = p->advantages; a.weights = p->weights; a.ref_logp = p->ref_logp;
    a.sums = p->sums; a.logp = p->logp; a.dlogits = p->dlogits; a.dstride = p->dlogits_stride;
    a.lo = 1.0f - p->clip_low; a.hi = 1.0f + p->clip_high; a.kl_coef = p->kl_coef;
    a.gscale = (float)((double)p->grad_scale / (double)x->temperature);
    if (!std::isfinite(a.gscale)) return MC_ERR_INVALID_ARG;
    launch_policy_loss(on(stream), x->dtype, a);
    return launched();
}

}  // extern "C"
