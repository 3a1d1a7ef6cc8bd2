// Host side of the C ABI declared in include/mergecomp_mx.h: handles, argument checks and launches.
#include <new>
#include <vector>

#include "host_util.h"
#include "mx_internal.h"

using namespace mc;

struct mc_step8 {
    int device = 0;
    int32_t grad_dtype = 0, model_dtype = MC_DTYPE_NONE;
    std::vector<int32_t> live;           // tensors that hold elements
    uint32_t npieces = 0;
    Piece *d_pieces = nullptr;
    uintptr_t *d_addr = nullptr;         // MC_LISTS8 lists of the live tensors' addresses
    std::vector<uintptr_t> want;         // a list on its way to the device (reserved at creation)
    bool bound[MC_LISTS8] = {};
};
struct mc_mx {
    int device = 0;
    float *d_partial = nullptr;
};

namespace {

constexpr int64_t kMost = (int64_t(1) << 31) - (1 << 16);

bool ready(const mc_step8 *h, int32_t list) { return h->bound[list] || h->live.empty(); }
uint64_t steps_of(int64_t cols) { return ((uint64_t)cols + kMxStep - 1) / kMxStep; }
// Whether a matrix can be one: sizes, and buffers on their boundaries (none where it has no rows).
int matrix_args(const mc_mx_matrix *m)
{
    if (!m || m->rows < 0 || m->cols < 1) return MC_ERR_INVALID_ARG;
    if (m->rows >= kMost || m->cols >= kMost) return MC_ERR_RANGE;
    if (m->rows > 0 && (!m->codes || !m->scales)) return MC_ERR_INVALID_ARG;
    return off(m->codes, 16) || off(m->scales, 4) ? MC_ERR_INVALID_ARG : MC_OK;
}
MxView view(const mc_mx_matrix *m)
{
    return {static_cast<uint8_t *>(m->codes), static_cast<uint8_t *>(m->scales), (uint32_t)m->rows, (uint32_t)steps_of(m->cols)};
}
Extent codes_at(const mc_mx_matrix *m) { return extent(m->codes, mc_mx_code_bytes(m->rows, m->cols)); }
Extent scales_at(const mc_mx_matrix *m) { return extent(m->scales, mc_mx_scale_bytes(m->rows, m->cols)); }

}  // namespace

extern "C" {

int mc_step8_destroy(mc_step8 *h)
{
    if (!h) return MC_ERR_INVALID_ARG;
    {
        OnDevice guard(h->device);
        (void)hipDeviceSynchronize();
        if (h->d_pieces) (void)hipFree(h->d_pieces);
        if (h->d_addr) (void)hipFree(h->d_addr);
    }
    delete h;
    return MC_OK;
}

int mc_step8_create(mc_step8 **out, const int64_t *numel, int32_t n_tensors, int32_t grad_dtype, int32_t model_dtype, const uint8_t *no_decay)
{
    if (!out) return MC_ERR_INVALID_ARG;
    *out = nullptr;
    if (!numel || n_tensors < 1 || !known(grad_dtype)) return MC_ERR_INVALID_ARG;
    if (model_dtype != MC_DTYPE_NONE && model_dtype != MC_DTYPE_BF16 && model_dtype != MC_DTYPE_F16) return MC_ERR_INVALID_ARG;
    uint64_t pieces = 0;
    for (int32_t t = 0; t < n_tensors; ++t) {
        if (numel[t] < 0) return MC_ERR_INVALID_ARG;
        if (numel[t] >= (int64_t(1) << 39)) return MC_ERR_RANGE;
        pieces += ((uint64_t)numel[t] + kPiece8 - 1) / kPiece8;
        if (pieces > (uint64_t(1) << 28)) return MC_ERR_RANGE;
    }
    mc_step8 *h = new (std::nothrow) mc_step8();
    if (!h) return MC_ERR_ALLOC;
    if (hipGetDevice(&h->device) != hipSuccess) { (void)hipGetLastError(); delete h; return MC_ERR_DEVICE; }
    int rc = MC_OK;
    try {
        h->grad_dtype = grad_dtype;
        h->model_dtype = model_dtype;
        h->npieces = (uint32_t)pieces;
        std::vector<Piece> table;
        table.reserve(pieces);
        for (int32_t t = 0; t < n_tensors; ++t) {
            if (numel[t] == 0) continue;
            const uint32_t name = (uint32_t)h->live.size() | (no_decay && no_decay[t] ? kNoDecay : 0u);
            h->live.push_back(t);
            for (int64_t at = 0, i = 0; at < numel[t]; at += kPiece8, ++i)
                table.push_back({name, (uint32_t)i, (int32_t)(numel[t] - at < (int64_t)kPiece8 ? numel[t] - at : kPiece8), 0u});
        }
        h->want.reserve(h->live.size());
        if (pieces) rc = grab(&h->d_pieces, table.size() * sizeof(Piece));
        if (rc == MC_OK && pieces) rc = grab(&h->d_addr, (size_t)MC_LISTS8 * h->live.size() * sizeof(uintptr_t));
        if (rc == MC_OK && pieces && hipMemcpy(h->d_pieces, table.data(), table.size() * sizeof(Piece), hipMemcpyHostToDevice) != hipSuccess) rc = MC_ERR_DEVICE;
    } catch (const std::bad_alloc &) {
        rc = MC_ERR_ALLOC;
    }
    if (rc != MC_OK) { (void)hipGetLastError(); mc_step8_destroy(h); return rc; }
    *out = h;
    return MC_OK;
}

int mc_step8_bind(mc_step8 *h, int32_t list, const void *const *ptrs, void *stream)
{
    if (!h || !ptrs || list < 0 || list >= MC_LISTS8 || (list == MC_LIST8_MODEL && h->model_dtype == MC_DTYPE_NONE)) return MC_ERR_INVALID_ARG;
    const uintptr_t align = list == MC_LIST8_GRADS ? size_of(h->grad_dtype) : list == MC_LIST8_MODEL ? size_of(h->model_dtype) :
                            list == MC_LIST8_EXP_AVG || list == MC_LIST8_EXP_AVG_SQ ? 1u : 4u;
    for (int32_t t : h->live) if (!ptrs[t] || off(ptrs[t], align)) return MC_ERR_INVALID_ARG;
    h->want.clear();                                      // (capacity reserved: no allocation)
    for (int32_t t : h->live) h->want.push_back(reinterpret_cast<uintptr_t>(ptrs[t]));
    const LaunchCtx lc = on(stream);
    if (!h->want.empty()) launch_upload_ptrs(lc, h->want.data(), h->d_addr + (size_t)list * h->want.size(), (uint32_t)h->want.size());
    const int rc = launched();
    h->bound[list] = rc == MC_OK;
    return rc;
}

int mc_adamw8(mc_step8 *h, const mc_adamw_config *c, const float *coef, void *stream)
{
    AdamwArgs a;
    if (!h || !adamw_args(c, coef, a)) return MC_ERR_INVALID_ARG;
    for (int32_t list = 0; list < MC_LISTS8; ++list)
        if (!ready(h, list) && !(list == MC_LIST8_MODEL && h->model_dtype == MC_DTYPE_NONE)) return MC_ERR_INVALID_ARG;
    launch_adamw8(on(stream), h->grad_dtype, h->model_dtype, {h->d_pieces, h->d_addr, h->npieces, (uint32_t)h->live.size()}, a);
    return launched();
}

size_t mc_mx_code_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 1 || rows >= kMost || cols >= kMost) return 0;
    return ((size_t)rows + 15) / 16 * steps_of(cols) * kMxCodes;
}
size_t mc_mx_scale_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 1 || rows >= kMost || cols >= kMost) return 0;
    return ((size_t)rows + 63) / 64 * steps_of(cols) * kMxScales;
}

int mc_mx_destroy(mc_mx *h)
{
    if (!h) return MC_ERR_INVALID_ARG;
    {
        OnDevice guard(h->device);
        (void)hipDeviceSynchronize();
        if (h->d_partial) (void)hipFree(h->d_partial);
    }
    delete h;
    return MC_OK;
}

int mc_mx_create(mc_mx **out)
{
    if (!out) return MC_ERR_INVALID_ARG;
    *out = nullptr;
    mc_mx *h = new (std::nothrow) mc_mx();
    if (!h) return MC_ERR_ALLOC;
    if (hipGetDevice(&h->device) != hipSuccess) { (void)hipGetLastError(); delete h; return MC_ERR_DEVICE; }
    int rc = grab(&h->d_partial, kMxPartial * sizeof(float));
    if (rc != MC_OK) { (void)hipGetLastError(); mc_mx_destroy(h); return rc; }
    *out = h;
    return MC_OK;
}

int mc_mx_quantize(mc_mx *h, const mc_mx_source *x, const mc_mx_matrix *by_rows, const mc_mx_matrix *by_cols, void *values, int64_t values_stride, void *stream)
{
    if (!h || !x || !known(x->dtype) || x->rows < 0 || x->cols < 1 || x->stride < x->cols) return MC_ERR_INVALID_ARG;
    if (x->rows >= kMost || x->cols >= kMost) return MC_ERR_RANGE;
    if (!by_rows && !by_cols && !values) return MC_ERR_INVALID_ARG;
    if ((x->rows > 0 && !x->data) || off(x->data, size_of(x->dtype)) || off(values, size_of(x->dtype))) return MC_ERR_INVALID_ARG;
    if (values && (values_stride < x->cols || (values == x->data && values_stride != x->stride))) return MC_ERR_INVALID_ARG;
    if (by_rows && (matrix_args(by_rows) != MC_OK || by_rows->rows != x->rows || by_rows->cols != x->cols)) return MC_ERR_INVALID_ARG;
    // (a transposed matrix has the source's rows for columns, and nothing is quantised where there are none)
    if (by_cols && x->rows > 0 && (matrix_args(by_cols) != MC_OK || by_cols->rows != x->cols || by_cols->cols != x->rows)) return MC_ERR_INVALID_ARG;
    if (x->rows == 0) return MC_OK;
    const RowsAt from(x->data, x->rows, x->cols, x->stride, size_of(x->dtype)), to(values, x->rows, x->cols, values ? values_stride : x->stride, size_of(x->dtype));
    if (values && values != x->data && meet(from, to)) return MC_ERR_INVALID_ARG;
    Extent written[4];
    int n = 0;
    for (const mc_mx_matrix *m : {by_rows, by_cols}) if (m) { written[n++] = codes_at(m); written[n++] = scales_at(m); }
    for (int i = 0; i < n; ++i) {
        if (meet(written[i], from) || (values && meet(written[i], to))) return MC_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j) if (meet(written[i], written[j])) return MC_ERR_INVALID_ARG;
    }
    MxSource s = {};
    s.x = x->data; s.values = values;
    s.stride = x->stride; s.values_stride = values_stride;
    s.rows = (uint32_t)x->rows; s.cols = (uint32_t)x->cols;
    if (by_rows) s.by_rows = view(by_rows);
    if (by_cols) s.by_cols = view(by_cols);
    launch_mx_quantize(on(stream), x->dtype, s);
    return launched();
}

int mc_mx_matmul(mc_mx *h, const mc_mx_matrix *a, const mc_mx_matrix *b, const mc_mx_result *y, void *stream)
{
    if (!h || !y) return MC_ERR_INVALID_ARG;
    for (const mc_mx_matrix *m : {a, b}) {
        const int rc = matrix_args(m);
        if (rc != MC_OK) return rc;
    }
    if (a->cols != b->cols || !known(y->dtype) || off(y->out, size_of(y->dtype)) || off(y->bias, 4)) return MC_ERR_INVALID_ARG;
    if (a->rows == 0 || b->rows == 0) return MC_OK;
    if (!y->out || y->stride < b->rows) return MC_ERR_INVALID_ARG;
    const RowsAt to(y->out, a->rows, b->rows, y->stride, size_of(y->dtype));
    for (const Extent e : {codes_at(a), scales_at(a), codes_at(b), scales_at(b), extent(y->bias, 4u * (uint64_t)b->rows)})
        if (meet(e, to)) return MC_ERR_INVALID_ARG;
    MxProduct p = {};
    p.a = view(a); p.b = view(b);
    p.out = y->out; p.bias = y->bias; p.stride = y->stride; p.accumulate = y->accumulate != 0;
    p.partial = h->d_partial;
    launch_mx_matmul(on(stream), y->dtype, p);
    return launched();
}

}  // extern "C"
