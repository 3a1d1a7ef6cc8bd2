// Host <-> kernel-launcher interface of the operators in mergecomp_mx.h, and what their kernels share.
#pragma once
#include "../../include/mergecomp_mx.h"
#include "step_internal.h"

namespace mc {

// ---- lists of tensors with moments in 8 bits -------------------------------------------------------------------------
constexpr uint32_t kBlock8 = 128;            // elements that share a scale
constexpr uint32_t kPiece8 = 2048;           // elements of a tensor that a block takes: eight a thread
struct Step8View {
    const Piece *pieces;                     // index: which of the tensor's pieces; left: elements from kPiece8 * index on, at most kPiece8
    const uintptr_t *addr;                   // those of list l: addr[l * tensors ..]
    uint32_t npieces, tensors;
};
void launch_adamw8(const LaunchCtx &lc, int dtype, int model_dtype, const Step8View &v, const AdamwArgs &a);

// ---- microscaled matrices --------------------------------------------------------------------------------------------
constexpr uint32_t kMxBlock = 32, kMxStep = 128, kMxCodes = 1024, kMxScales = 256;        // elements to a scale, columns, bytes to a tile's codes and scales
struct MxView {
    uint8_t *codes, *scales;
    uint32_t rows, steps;                    // columns padded: kMxStep * steps
};
struct MxSource {
    const void *x;
    void *values;                            // null: none
    int64_t stride, values_stride;
    uint32_t rows, cols;
    MxView by_rows, by_cols;                 // codes null: none
};
void launch_mx_quantize(const LaunchCtx &lc, int dtype, const MxSource &s);

struct MxProduct {
    MxView a, b;
    void *out;
    const float *bias;                       // null: none
    int64_t stride;
    bool accumulate;
    float *partial;                          // kMxPartial floats
    size_t apart;                            // elements from a part's result to the next one's
};
constexpr size_t kMxPartial = size_t(1) << 24;
void launch_mx_matmul(const LaunchCtx &lc, int dtype, const MxProduct &p);

// Blocks of up to 512 threads in launches of fewer than 2^32 threads: body(first block, blocks).
template <class Body>
inline void in_launches(uint64_t blocks, Body body)
{
    constexpr uint64_t most = 1u << 22;
    for (uint64_t first = 0; first < blocks; first += most) body(first, (uint32_t)(blocks - first < most ? blocks - first : most));
}

}  // namespace mc
