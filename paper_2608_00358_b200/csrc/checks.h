// Checks that the C entry points of the expert layers share.
#pragma once
#include "experts.cuh"
#include "plan.hpp"

namespace hccl {
hccl_status_t note_cuda_error(cudaError_t e, const char* what);  // executor.cu
}

namespace {

bool aligned(const void* p, int64_t bytes) { return ((uintptr_t)p) % (uintptr_t)bytes == 0; }
// rows * ld may not wrap: every offset the kernels form stays below 2^62 bytes
bool sane(int64_t rows, int64_t ld, int64_t width) { return rows >= 0 && width >= 0 && (rows <= 1 || ld >= width) && ld >= 0 && (ld == 0 || rows < (INT64_C(1) << 60) / ld); }

hccl_status_t done(cudaError_t e, const char* what) { return e == cudaSuccess ? HCCL_OK : hccl::note_cuda_error(e, what); }

// What the rows' movers read of a routing.
hccl_status_t check_routing(const hccl_routing_t* r) {
    if (!r || r->tokens < 0 || r->top_k < 1 || r->top_k > HCCL_MAX_TOP_K || r->experts < 1 || r->experts > HCCL_MAX_EXPERTS) return HCCL_ERR_INVALID_ARG;
    if (r->tokens >= (INT64_C(1) << 31) / r->top_k) return HCCL_ERR_INVALID_ARG;
    if (!r->offsets || (r->tokens && !r->slots)) return HCCL_ERR_INVALID_ARG;
    if (!aligned(r->offsets, 4) || !aligned(r->slots, 4)) return HCCL_ERR_ALIGNMENT;
    return HCCL_OK;
}

hccl_status_t check_matrix(const void* p, int64_t rows, int64_t ld, int64_t width, int dt) {
    if (!sane(rows, ld, width)) return HCCL_ERR_INVALID_ARG;
    if (rows && width && !p) return HCCL_ERR_INVALID_ARG;
    return aligned(p, hccl::elem_bytes(dt)) ? HCCL_OK : HCCL_ERR_ALIGNMENT;
}

#define TRY(x)                               \
    do {                                     \
        const hccl_status_t st_ = (x);       \
        if (st_ != HCCL_OK) return st_;      \
    } while (0)

}  // namespace
