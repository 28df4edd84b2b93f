// C entry points of the expert-layer operators: argument checks and launches.
#include <cstring>

#include "checks.h"

using namespace hccl::experts;

namespace {

hccl_status_t check_router(const hccl_router_t* r, int64_t tokens) {
    if (!r || tokens < 0) return HCCL_ERR_INVALID_ARG;
    if (r->experts < 1 || r->experts > HCCL_MAX_EXPERTS) return HCCL_ERR_INVALID_ARG;
    if (r->top_k < 1 || r->top_k > HCCL_MAX_TOP_K || r->top_k > r->experts) return HCCL_ERR_INVALID_ARG;
    if (r->score != HCCL_SCORE_SOFTMAX && r->score != HCCL_SCORE_SIGMOID) return HCCL_ERR_INVALID_ARG;
    if (r->groups < 0) return HCCL_ERR_INVALID_ARG;
    if (r->groups > 1) {
        if (r->experts % r->groups || r->top_groups < 1 || r->top_groups > r->groups) return HCCL_ERR_INVALID_ARG;
        if (r->group_best != 1 && r->group_best != 2) return HCCL_ERR_INVALID_ARG;
    }
    if (tokens >= (INT64_C(1) << 31) / r->top_k) return HCCL_ERR_INVALID_ARG;
    return HCCL_OK;
}

RouteParams route_params(const hccl_router_t* c, const void* logits, int64_t ld, const float* bias, const uint8_t* mask, const hccl_routing_t* r) {
    RouteParams p = {};
    p.logits = logits;
    p.ld = ld;
    p.bias = bias;
    p.mask = mask;
    p.tokens = r->tokens;
    p.E = c->experts;
    p.K = c->top_k;
    p.groups = c->groups > 1 ? c->groups : 1;
    p.per_group = c->experts / p.groups;
    p.top_groups = c->top_groups;
    p.group_best = c->group_best;
    p.sigmoid = c->score == HCCL_SCORE_SIGMOID;
    p.renorm = c->renormalise != 0;
    p.scale = c->scale;
    p.ids = r->ids;
    p.weights = r->weights;
    p.counts = (long long*)r->counts;
    p.offsets = r->offsets;
    p.slots = r->slots;
    p.source = r->source;
    return p;
}

hccl_status_t check_route_inputs(const hccl_router_t* c, const void* logits, int64_t ld, hccl_dtype_t dt, const float* bias, const hccl_routing_t* r) {
    if (!r) return HCCL_ERR_INVALID_ARG;
    TRY(check_router(c, r->tokens));
    if (!hccl::valid_dtype(dt)) return HCCL_ERR_DTYPE;
    if (r->experts != c->experts || r->top_k != c->top_k) return HCCL_ERR_COUNT_MISMATCH;
    TRY(check_matrix(logits, r->tokens, ld, c->experts, dt));
    if (!aligned(bias, 4)) return HCCL_ERR_ALIGNMENT;
    if (r->tokens && !r->ids) return HCCL_ERR_INVALID_ARG;
    return aligned(r->ids, 4) ? HCCL_OK : HCCL_ERR_ALIGNMENT;
}

hccl_status_t check_matmul(const hccl_matmul_i8_t* m) {
    if (!m || m->M < 0 || m->N < 0 || m->K < 0 || m->groups < 0 || m->groups > HCCL_MAX_EXPERTS) return HCCL_ERR_INVALID_ARG;
    if (!hccl::valid_dtype(m->dtype)) return HCCL_ERR_DTYPE;
    if (m->K > HCCL_MAX_I8_K) return HCCL_ERR_INVALID_ARG;
    const int64_t g = m->groups ? m->groups : 1;
    if (m->M > HCCL_MAX_I8_ROWS || m->N > HCCL_MAX_I8_ROWS / g) return HCCL_ERR_INVALID_ARG;
    if (!sane(m->M, m->lda, m->K) || !sane(m->N * g, m->ldw, m->K)) return HCCL_ERR_INVALID_ARG;
    if (m->groups && !m->offsets) return HCCL_ERR_INVALID_ARG;
    if (m->M && m->N) {
        if ((m->K && (!m->a || !m->w)) || !m->a_scale || !m->w_scale) return HCCL_ERR_INVALID_ARG;
        TRY(check_matrix(m->y, m->M, m->ldy, m->N, m->dtype));
    }
    if (!aligned(m->a, 16) || !aligned(m->w, 16) || m->lda % 16 || m->ldw % 16) return HCCL_ERR_ALIGNMENT;
    if (!aligned(m->a_scale, 4) || !aligned(m->w_scale, 4) || !aligned(m->bias, 4) || !aligned(m->offsets, 4) || !aligned(m->dev_status, 4)) return HCCL_ERR_ALIGNMENT;
    return HCCL_OK;
}

MatmulParams matmul_params(const hccl_matmul_i8_t* m) {
    MatmulParams p = {};
    p.M = m->M;
    p.N = m->N;
    p.K = m->K;
    p.lda = m->lda;
    p.ldw = m->ldw;
    p.ldy = m->ldy;
    p.groups = m->groups;
    p.a = m->a;
    p.w = m->w;
    p.a_scale = m->a_scale;
    p.w_scale = m->w_scale;
    p.bias = m->bias;
    p.offsets = m->offsets;
    p.y = m->y;
    p.status = m->dev_status;
    return p;
}

hccl_status_t quant_params(QuantParams* p, const void* x, int64_t ldx, int64_t M, int64_t K, hccl_dtype_t dt, const hccl_routing_t* r, int8_t* q,
                           int64_t ldq, int64_t n_q, float* scale) {
    if (!hccl::valid_dtype(dt)) return HCCL_ERR_DTYPE;
    if (K < 0 || K > HCCL_MAX_I8_K || M < 0 || n_q < 0) return HCCL_ERR_INVALID_ARG;
    TRY(check_matrix(x, M, ldx, K, dt));
    if (!sane(n_q, ldq, K)) return HCCL_ERR_INVALID_ARG;
    if (n_q && ((K && !q) || !scale)) return HCCL_ERR_INVALID_ARG;
    if (!aligned(scale, 4)) return HCCL_ERR_ALIGNMENT;
    if (r) {
        TRY(check_routing(r));
        if (M != r->tokens) return HCCL_ERR_COUNT_MISMATCH;
    } else if (n_q < M) {
        return HCCL_ERR_COUNT_MISMATCH;
    }
    *p = {};
    p->x = x;
    p->ldx = ldx;
    p->M = M;
    p->K = K;
    p->ldq = ldq;
    p->n_q = n_q;
    p->q = q;
    p->scale = scale;
    p->slots = r ? r->slots : nullptr;
    p->top_k = r ? r->top_k : 1;
    return HCCL_OK;
}

}  // namespace

extern "C" {

hccl_status_t hccl_route_workspace_bytes(const hccl_router_t* c, int64_t tokens, size_t* bytes) {
    TRY(check_router(c, tokens));
    if (!bytes) return HCCL_ERR_INVALID_ARG;
    *bytes = route_workspace(c->experts, tokens);
    return HCCL_OK;
}

hccl_status_t hccl_route(const hccl_router_t* c, const void* logits, int64_t ld, hccl_dtype_t dt, const float* bias, const uint8_t* mask,
                         const hccl_routing_t* out, void* workspace, size_t bytes, void* stream) {
    TRY(check_route_inputs(c, logits, ld, dt, bias, out));
    if (!out->counts || !out->offsets) return HCCL_ERR_INVALID_ARG;
    if (out->tokens && (!out->weights || !out->slots || !out->source)) return HCCL_ERR_INVALID_ARG;
    if (!aligned(out->weights, 4) || !aligned(out->counts, 8) || !aligned(out->offsets, 4) || !aligned(out->slots, 4) || !aligned(out->source, 4)) return HCCL_ERR_ALIGNMENT;
    if (bytes < route_workspace(c->experts, out->tokens)) return HCCL_ERR_WORKSPACE;
    if (!workspace) return HCCL_ERR_INVALID_ARG;
    if (!aligned(workspace, 16)) return HCCL_ERR_ALIGNMENT;
    RouteParams p = route_params(c, logits, ld, bias, mask, out);
    p.hist = (uint8_t*)workspace;
    return done(launch_route(dt, p, (cudaStream_t)stream), "hccl_route");
}

hccl_status_t hccl_route_backward(const hccl_router_t* c, const void* logits, int64_t ld, hccl_dtype_t dt, const float* bias, const uint8_t* mask,
                                  const hccl_routing_t* r, const float* dweights, void* dlogits, int64_t ldd, void* stream) {
    TRY(check_route_inputs(c, logits, ld, dt, bias, r));
    TRY(check_matrix(dlogits, r->tokens, ldd, c->experts, dt));
    if (r->tokens && !dweights) return HCCL_ERR_INVALID_ARG;
    if (!aligned(dweights, 4)) return HCCL_ERR_ALIGNMENT;
    RouteGradParams p = {};
    p.r = route_params(c, logits, ld, bias, mask, r);
    p.dweights = dweights;
    p.dlogits = dlogits;
    p.ldd = ldd;
    return done(launch_route_grad(dt, p, (cudaStream_t)stream), "hccl_route_backward");
}

static hccl_status_t rows_params(RowsParams* p, const hccl_routing_t* r, int64_t n_rows, int64_t H, hccl_dtype_t dt) {
    TRY(check_routing(r));
    if (!hccl::valid_dtype(dt)) return HCCL_ERR_DTYPE;
    if (n_rows < 0 || H < 0) return HCCL_ERR_INVALID_ARG;
    *p = {};
    p->tokens = r->tokens;
    p->n_rows = n_rows;
    p->H = H;
    p->K = r->top_k;
    p->E = r->experts;
    p->slots = r->slots;
    p->offsets = r->offsets;
    return HCCL_OK;
}

hccl_status_t hccl_dispatch(const void* x, int64_t ldx, int64_t H, hccl_dtype_t dt, const hccl_routing_t* r, void* rows, int64_t ldr,
                            int64_t n_rows, void* stream) {
    RowsParams p;
    TRY(rows_params(&p, r, n_rows, H, dt));
    TRY(check_matrix(x, p.tokens, ldx, H, dt));
    TRY(check_matrix(rows, n_rows, ldr, H, dt));
    p.x = x;
    p.ldx = ldx;
    p.rows_out = rows;
    p.ldro = ldr;
    return done(launch_dispatch(dt, p, (cudaStream_t)stream), "hccl_dispatch");
}

static hccl_status_t combine(const void* rows, int64_t ldr, int64_t n_rows, int64_t H, hccl_dtype_t dt, const hccl_routing_t* r, const float* weights,
                             void* y, int64_t ldy, void* stream, const char* what) {
    RowsParams p;
    TRY(rows_params(&p, r, n_rows, H, dt));
    TRY(check_matrix(rows, n_rows, ldr, H, dt));
    TRY(check_matrix(y, p.tokens, ldy, H, dt));
    if (!aligned(weights, 4)) return HCCL_ERR_ALIGNMENT;
    p.rows = rows;
    p.ldr = ldr;
    p.y = y;
    p.ldy = ldy;
    p.weights = weights;
    return done(launch_combine(dt, p, (cudaStream_t)stream), what);
}

hccl_status_t hccl_dispatch_backward(const void* drows, int64_t ldr, int64_t n_rows, int64_t H, hccl_dtype_t dt, const hccl_routing_t* r, void* dx,
                                     int64_t ldx, void* stream) {
    return combine(drows, ldr, n_rows, H, dt, r, nullptr, dx, ldx, stream, "hccl_dispatch_backward");
}

hccl_status_t hccl_combine(const void* rows, int64_t ldr, int64_t n_rows, int64_t H, hccl_dtype_t dt, const hccl_routing_t* r, const float* weights,
                           void* y, int64_t ldy, void* stream) {
    if (r && r->tokens && !weights) return HCCL_ERR_INVALID_ARG;
    return combine(rows, ldr, n_rows, H, dt, r, weights, y, ldy, stream, "hccl_combine");
}

hccl_status_t hccl_combine_backward(const void* dy, int64_t ldy, const void* rows, int64_t ldr, int64_t n_rows, int64_t H, hccl_dtype_t dt,
                                    const hccl_routing_t* r, const float* weights, void* drows, int64_t ldd, float* dweights, void* stream) {
    RowsParams p;
    TRY(rows_params(&p, r, n_rows, H, dt));
    if (p.tokens && (!weights || !dweights)) return HCCL_ERR_INVALID_ARG;
    TRY(check_matrix(dy, p.tokens, ldy, H, dt));
    TRY(check_matrix(rows, n_rows, ldr, H, dt));
    TRY(check_matrix(drows, n_rows, ldd, H, dt));
    if (!aligned(weights, 4) || !aligned(dweights, 4)) return HCCL_ERR_ALIGNMENT;
    p.x = dy;
    p.ldx = ldy;
    p.rows = rows;
    p.ldr = ldr;
    p.rows_out = drows;
    p.ldro = ldd;
    p.weights = weights;
    p.dweights = dweights;
    return done(launch_combine_grad(dt, p, (cudaStream_t)stream), "hccl_combine_backward");
}

hccl_status_t hccl_quantize_rows_i8(const void* x, int64_t ldx, int64_t M, int64_t K, hccl_dtype_t dt, const hccl_routing_t* r, int8_t* q, int64_t ldq,
                                    int64_t n_q, float* scale, void* stream) {
    QuantParams p;
    TRY(quant_params(&p, x, ldx, M, K, dt, r, q, ldq, n_q, scale));
    return done(launch_quantise(dt, p, (cudaStream_t)stream), "hccl_quantize_rows_i8");
}

hccl_status_t hccl_matmul_i8(const hccl_matmul_i8_t* m, void* stream) {
    TRY(check_matmul(m));
    return done(launch_matmul_i8(m->dtype, matmul_params(m), (cudaStream_t)stream), "hccl_matmul_i8");
}

hccl_status_t hccl_linear_i8(const hccl_matmul_i8_t* in, const void* x, int64_t ldx, hccl_dtype_t dt, const hccl_routing_t* r, void* stream) {
    if (!in) return HCCL_ERR_INVALID_ARG;
    hccl_matmul_i8_t m = *in;
    if (r) {
        TRY(check_routing(r));
        m.groups = r->experts;
        m.offsets = r->offsets;
    }
    TRY(check_matmul(&m));
    QuantParams p;
    TRY(quant_params(&p, x, ldx, r ? r->tokens : m.M, m.K, dt, r, (int8_t*)m.a, m.lda, m.M, (float*)m.a_scale));
    MatmulParams mm = matmul_params(&m);
    if (mm.M && mm.N && few_rows(mm) && few_rows_quantise(mm)) return done(launch_linear_i8_few(m.dtype, mm, p, dt, (cudaStream_t)stream), "hccl_linear_i8");
    const cudaError_t e = launch_quantise(dt, p, (cudaStream_t)stream);
    if (e != cudaSuccess) return hccl::note_cuda_error(e, "hccl_linear_i8");
    mm.dependent = p.M > 0;
    return done(launch_matmul_i8(m.dtype, mm, (cudaStream_t)stream), "hccl_linear_i8");
}

// For the Python binding: it packs an array in one step, which takes half the time of handing over ten arguments one by one.
hccl_status_t hccl_call_packed(int32_t call, const int64_t* a) {
    if (!a) return HCCL_ERR_INVALID_ARG;
    const auto at = [&](int i) { return (void*)(uintptr_t)a[i]; };
    const auto dt = [&](int i) { return (hccl_dtype_t)a[i]; };
    const auto matmul = [&] {
        hccl_matmul_i8_t m = {};
        m.M = a[0], m.N = a[1], m.K = a[2], m.groups = (int32_t)a[3], m.dtype = (int32_t)a[4];
        m.a = (const int8_t*)at(5), m.lda = a[6], m.a_scale = (const float*)at(7);
        m.w = (const int8_t*)at(8), m.ldw = a[9], m.w_scale = (const float*)at(10);
        m.bias = (const float*)at(11), m.offsets = (const int32_t*)at(12);
        m.y = at(13), m.ldy = a[14], m.dev_status = (int32_t*)at(15);
        return m;
    };
    const auto f32 = [&](int i) {
        const uint32_t bits = (uint32_t)a[i];
        float f;
        memcpy(&f, &bits, 4);
        return f;
    };
    const auto matmul_fp4 = [&] {
        hccl_matmul_fp4_t m = {};
        m.M = a[0], m.N = a[1], m.K = a[2], m.groups = (int32_t)a[3], m.dtype = (int32_t)a[4], m.format = (int32_t)a[5], m.x_wide = f32(6);
        m.w = (const uint8_t*)at(7), m.ldw = a[8], m.w_scale = at(9), m.w_wide = (const float*)at(10);
        m.bias = (const float*)at(11), m.offsets = (const int32_t*)at(12);
        m.y = at(13), m.ldy = a[14], m.scratch = at(15), m.scratch_bytes = a[16];
        m.dev_status = (int32_t*)at(17);
        return m;
    };
    const auto activation = [&] {
        hccl_activation_t f = {};
        f.act = (int32_t)a[0], f.gated = (int32_t)a[1];
        memcpy(&f.p, &a[2], 8);
        f.seed = (const int64_t*)at(3);
        return f;
    };
    switch (call) {
        case HCCL_CALL_ROUTE:
            return hccl_route((const hccl_router_t*)at(0), at(1), a[2], dt(3), (const float*)at(4), (const uint8_t*)at(5), (const hccl_routing_t*)at(6), at(7), (size_t)a[8], at(9));
        case HCCL_CALL_ROUTE_BACKWARD:
            return hccl_route_backward((const hccl_router_t*)at(0), at(1), a[2], dt(3), (const float*)at(4), (const uint8_t*)at(5), (const hccl_routing_t*)at(6),
                                       (const float*)at(7), at(8), a[9], at(10));
        case HCCL_CALL_DISPATCH:
            return hccl_dispatch(at(0), a[1], a[2], dt(3), (const hccl_routing_t*)at(4), at(5), a[6], a[7], at(8));
        case HCCL_CALL_DISPATCH_BACKWARD:
            return hccl_dispatch_backward(at(0), a[1], a[2], a[3], dt(4), (const hccl_routing_t*)at(5), at(6), a[7], at(8));
        case HCCL_CALL_COMBINE:
            return hccl_combine(at(0), a[1], a[2], a[3], dt(4), (const hccl_routing_t*)at(5), (const float*)at(6), at(7), a[8], at(9));
        case HCCL_CALL_COMBINE_BACKWARD:
            return hccl_combine_backward(at(0), a[1], at(2), a[3], a[4], a[5], dt(6), (const hccl_routing_t*)at(7), (const float*)at(8), at(9), a[10], (float*)at(11), at(12));
        case HCCL_CALL_QUANTIZE_ROWS_I8:
            return hccl_quantize_rows_i8(at(0), a[1], a[2], a[3], dt(4), (const hccl_routing_t*)at(5), (int8_t*)at(6), a[7], a[8], (float*)at(9), at(10));
        case HCCL_CALL_MATMUL_I8: {
            const hccl_matmul_i8_t m = matmul();
            return hccl_matmul_i8(&m, at(16));
        }
        case HCCL_CALL_LINEAR_I8: {
            const hccl_matmul_i8_t m = matmul();
            return hccl_linear_i8(&m, at(16), a[17], dt(18), (const hccl_routing_t*)at(19), at(20));
        }
        case HCCL_CALL_QUANTIZE_ROWS_FP4:
            return hccl_quantize_rows_fp4(at(0), a[1], a[2], a[3], dt(4), (int32_t)a[5], f32(6), (const hccl_routing_t*)at(7), (uint8_t*)at(8), a[9], (uint8_t*)at(10), a[11], a[12], at(13));
        case HCCL_CALL_DEQUANTIZE_ROWS_FP4:
            return hccl_dequantize_rows_fp4((const uint8_t*)at(0), a[1], (const uint8_t*)at(2), a[3], a[4], a[5], (int32_t)a[6], f32(7), at(8), a[9], dt(10), at(11));
        case HCCL_CALL_MATMUL_FP4: {
            const hccl_matmul_fp4_t m = matmul_fp4();
            return hccl_matmul_fp4(&m, (const uint8_t*)at(18), a[19], (const uint8_t*)at(20), a[21], at(22));
        }
        case HCCL_CALL_LINEAR_FP4: {
            const hccl_matmul_fp4_t m = matmul_fp4();
            return hccl_linear_fp4(&m, at(18), a[19], dt(20), (const hccl_routing_t*)at(21), at(22));
        }
        case HCCL_CALL_EXPERT_LAYER_FP4:
            return hccl_expert_layer_fp4((const hccl_experts_fp4_t*)at(0), at(1), a[2], dt(3), (const hccl_routing_t*)at(4), at(5), a[6], at(7), (size_t)a[8], (int32_t*)at(9), at(10));
        case HCCL_CALL_ACTIVATE: {
            const hccl_activation_t f = activation();
            return hccl_activate(&f, at(4), a[5], a[6], a[7], dt(8), (const int32_t*)at(9), (int32_t)a[10], at(11), a[12], at(13));
        }
        case HCCL_CALL_ACTIVATE_BACKWARD: {
            const hccl_activation_t f = activation();
            return hccl_activate_backward(&f, at(4), a[5], at(6), a[7], a[8], a[9], dt(10), (const int32_t*)at(11), (int32_t)a[12], at(13), a[14], at(15));
        }
        default:
            return HCCL_ERR_INVALID_ARG;
    }
}

}  // extern "C"
