// C entry points of the operators in 4-bit floating point: argument checks and launches.
#include <cmath>

#include "activate.cuh"
#include "checks.h"
#include "fp4.cuh"

using namespace hccl::experts;

namespace {

constexpr int64_t PITCH = 16;  // bytes: what TMA asks of the distance between rows

int64_t up_to(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
int64_t stages(int64_t K) { return (K + 255) / 256; }

bool valid_format(int32_t f) { return f == HCCL_NVFP4 || f == HCCL_MXFP4; }
bool valid_wide(float g) { return g >= 1e-30f && g <= 1e30f; }  // (NaN fails)

hccl_status_t check_shape(int64_t rows, int64_t K, int32_t format) {
    if (!valid_format(format)) return HCCL_ERR_DTYPE;
    return K < 0 || K > HCCL_MAX_FP4_K || rows < 0 || rows > HCCL_MAX_I8_ROWS ? HCCL_ERR_INVALID_ARG : HCCL_OK;
}

// Rows of codes and of scales.
hccl_status_t check_rows(const uint8_t* q, int64_t ldq, const uint8_t* scale, int64_t lds, int64_t rows, int64_t K, int32_t format) {
    if (!sane(rows, ldq, (K + 1) / 2) || !sane(rows, lds, (K + block_of(format) - 1) / block_of(format))) return HCCL_ERR_INVALID_ARG;
    return rows && K && (!q || !scale) ? HCCL_ERR_INVALID_ARG : HCCL_OK;
}

// TMA counts atoms in 32 bits.
bool few_atoms(int64_t tiles, int64_t K, int format) { return tiles * stages(K) * stage_atoms(format) < (INT64_C(1) << 31); }

hccl_status_t check_weights(int64_t N, int64_t K, int32_t groups, int32_t format) {
    TRY(check_shape(N, K, format));
    if (groups < 0 || groups > 2 * HCCL_MAX_EXPERTS) return HCCL_ERR_INVALID_ARG;
    const int64_t g = groups ? groups : 1;
    if (N > HCCL_MAX_I8_ROWS / g || !few_atoms((N + 127) / 128 * g, K, format)) return HCCL_ERR_INVALID_ARG;
    return HCCL_OK;
}
int64_t weight_scale_bytes(int64_t N, int64_t K, int32_t groups, int32_t format) {
    return (N + 127) / 128 * (groups ? groups : 1) * stages(K) * stage_atoms(format) * ATOM;
}

struct Scratch {
    int64_t ldq, scales, bytes;  // the rows come first, at `scales` their scales in tiles
    int wide;                    // 128-row atoms to a tile
};
Scratch scratch_of(int64_t M, int64_t K, int32_t groups, int32_t format, int tn) {
    Scratch s;
    s.wide = tn > 128 ? tn / 128 : 1;
    s.ldq = up_to((K + 1) / 2, PITCH);
    s.scales = up_to(M * s.ldq, ATOM);
    s.bytes = s.scales + ((M + tn - 1) / tn + (groups ? groups : 1)) * s.wide * stages(K) * stage_atoms(format) * ATOM;
    return s;
}
hccl_status_t check_product(int64_t M, int64_t N, int64_t K, int32_t groups, int32_t format) {
    TRY(check_weights(N, K, groups, format));
    if (M < 0 || M > HCCL_MAX_I8_ROWS || groups > HCCL_MAX_EXPERTS) return HCCL_ERR_INVALID_ARG;
    const int tn = choose_fp4(M, N, K, groups).tn;
    return few_atoms(((M + tn - 1) / tn + (groups ? groups : 1)) * (tn > 128 ? 2 : 1), K, format) ? HCCL_OK : HCCL_ERR_INVALID_ARG;
}

hccl_status_t check_matmul(const hccl_matmul_fp4_t* m) {
    if (!m) return HCCL_ERR_INVALID_ARG;
    TRY(check_product(m->M, m->N, m->K, m->groups, m->format));
    if (!hccl::valid_dtype(m->dtype)) return HCCL_ERR_DTYPE;
    const int64_t g = m->groups ? m->groups : 1;
    if (!sane(m->N * g, m->ldw, (m->K + 1) / 2)) return HCCL_ERR_INVALID_ARG;
    if (m->format == HCCL_NVFP4 ? !valid_wide(m->x_wide) : m->x_wide != 1.f) return HCCL_ERR_INVALID_ARG;
    if (m->groups && !m->offsets) return HCCL_ERR_INVALID_ARG;
    if (m->M && m->N) {
        if ((m->K && (!m->w || !m->w_scale)) || !m->w_wide) return HCCL_ERR_INVALID_ARG;
        TRY(check_matrix(m->y, m->M, m->ldy, m->N, m->dtype));
        if (m->K && (!m->scratch || m->scratch_bytes < scratch_of(m->M, m->K, m->groups, m->format, choose_fp4(m->M, m->N, m->K, m->groups).tn).bytes)) return HCCL_ERR_WORKSPACE;
    }
    if (!aligned(m->w, 16) || m->ldw % 16 || !aligned(m->w_scale, 16) || !aligned(m->scratch, 128)) return HCCL_ERR_ALIGNMENT;
    if (!aligned(m->w_wide, 4) || !aligned(m->bias, 4) || !aligned(m->offsets, 4) || !aligned(m->dev_status, 4)) return HCCL_ERR_ALIGNMENT;
    return HCCL_OK;
}

MatmulFp4 matmul_params(const hccl_matmul_fp4_t* m) {
    MatmulFp4 p = {};
    p.M = m->M;
    p.N = m->N;
    p.K = m->K;
    p.ldw = m->ldw;
    p.ldy = m->ldy;
    p.groups = m->groups;
    p.format = m->format;
    p.w = m->w;
    p.w_scale = (const uint8_t*)m->w_scale;
    p.w_wide = m->w_wide;
    p.x_wide = m->x_wide;
    p.bias = m->bias;
    p.offsets = m->offsets;
    p.y = m->y;
    p.status = m->dev_status;
    const TileChoice c = choose_fp4(m->M, m->N, m->K, m->groups);
    p.tn = c.tn;
    p.splits = c.splits;
    return p;
}

hccl_status_t quant_params(Fp4Rows* p, const void* x, int64_t ldx, int64_t M, int64_t K, hccl_dtype_t dt, int32_t format, float wide, const hccl_routing_t* r, uint8_t* q,
                           int64_t ldq, int64_t n_q) {
    TRY(check_shape(M, K, format));
    if (!hccl::valid_dtype(dt)) return HCCL_ERR_DTYPE;
    if (n_q < 0 || n_q > HCCL_MAX_I8_ROWS || (format == HCCL_NVFP4 && !valid_wide(wide))) return HCCL_ERR_INVALID_ARG;
    TRY(check_matrix(x, M, ldx, K, dt));
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
    p->wide = wide;
    p->six = 6.f * wide;
    p->sixth = 1.f / p->six;
    p->q = q;
    p->ldq = ldq;
    p->n_q = n_q;
    p->slots = r ? r->slots : nullptr;
    p->top_k = r ? r->top_k : 1;
    return HCCL_OK;
}

}  // namespace

extern "C" {

hccl_status_t hccl_quantize_rows_fp4(const void* x, int64_t ldx, int64_t M, int64_t K, hccl_dtype_t dt, int32_t format, float wide, const hccl_routing_t* r, uint8_t* q,
                                     int64_t ldq, uint8_t* scale, int64_t lds, int64_t n_q, void* stream) {
    Fp4Rows p;
    TRY(quant_params(&p, x, ldx, M, K, dt, format, wide, r, q, ldq, n_q));
    TRY(check_rows(q, ldq, scale, lds, n_q, K, format));
    p.scale = scale;
    p.lds = lds;
    return done(launch_quantise_fp4(dt, format, p, (cudaStream_t)stream), "hccl_quantize_rows_fp4");
}

hccl_status_t hccl_dequantize_rows_fp4(const uint8_t* q, int64_t ldq, const uint8_t* scale, int64_t lds, int64_t M, int64_t K, int32_t format, float wide, void* y,
                                       int64_t ldy, hccl_dtype_t dt, void* stream) {
    TRY(check_shape(M, K, format));
    if (!hccl::valid_dtype(dt)) return HCCL_ERR_DTYPE;
    if (format == HCCL_NVFP4 && !valid_wide(wide)) return HCCL_ERR_INVALID_ARG;
    TRY(check_rows(q, ldq, scale, lds, M, K, format));
    TRY(check_matrix(y, M, ldy, K, dt));
    Fp4Values p = {};
    p.q = q;
    p.ldq = ldq;
    p.scale = scale;
    p.lds = lds;
    p.M = M;
    p.K = K;
    p.y = y;
    p.ldy = ldy;
    p.wide = wide;
    return done(launch_dequantise_fp4(dt, format, p, (cudaStream_t)stream), "hccl_dequantize_rows_fp4");
}

hccl_status_t hccl_fp4_weight_scale_bytes(int64_t N, int64_t K, int32_t groups, int32_t format, size_t* bytes) {
    TRY(check_weights(N, K, groups, format));
    if (!bytes) return HCCL_ERR_INVALID_ARG;
    *bytes = (size_t)weight_scale_bytes(N, K, groups, format);
    return HCCL_OK;
}

hccl_status_t hccl_fp4_weight_scales(const uint8_t* scale, int64_t lds, int64_t N, int64_t K, int32_t groups, int32_t format, void* out, void* stream) {
    TRY(check_weights(N, K, groups, format));
    const int64_t g = groups ? groups : 1, blocks = (K + block_of(format) - 1) / block_of(format);
    if (!sane(N * g, lds, blocks)) return HCCL_ERR_INVALID_ARG;
    if (N == 0 || K == 0) return HCCL_OK;
    if (!scale || !out) return HCCL_ERR_INVALID_ARG;
    if (!aligned(out, 16)) return HCCL_ERR_ALIGNMENT;
    // rows beyond N in a group's last tile: their sums are not used, but what is not set could differ from run to run
    const cudaError_t e = cudaMemsetAsync(out, 0, (size_t)weight_scale_bytes(N, K, groups, format), (cudaStream_t)stream);
    if (e != cudaSuccess) return done(e, "hccl_fp4_weight_scales");
    Fp4Scales p = {};
    p.scale = scale;
    p.lds = lds;
    p.N = N;
    p.blocks = blocks;
    p.out = (uint8_t*)out;
    p.tn = 128;
    p.atoms = (int)(stages(K) * stage_atoms(format));
    p.groups = (int)g;
    return done(launch_tile_scales_fp4(p, (cudaStream_t)stream), "hccl_fp4_weight_scales");
}

hccl_status_t hccl_fp4_scratch_bytes(int64_t M, int64_t N, int64_t K, int32_t groups, int32_t format, size_t* bytes) {
    TRY(check_product(M, N, K, groups, format));
    if (!bytes) return HCCL_ERR_INVALID_ARG;
    *bytes = (size_t)scratch_of(M, K, groups, format, choose_fp4(M, N, K, groups).tn).bytes;
    return HCCL_OK;
}

hccl_status_t hccl_matmul_fp4(const hccl_matmul_fp4_t* m, const uint8_t* q, int64_t ldq, const uint8_t* scale, int64_t lds, void* stream) {
    TRY(check_matmul(m));
    TRY(check_rows(q, ldq, scale, lds, m->M, m->K, m->format));
    if (!aligned(q, 16) || ldq % 16) return HCCL_ERR_ALIGNMENT;
    if (m->M == 0 || m->N == 0) return HCCL_OK;
    MatmulFp4 p = matmul_params(m);
    p.q = q;
    p.ldq = ldq;
    if (m->K) {
        const Scratch s = scratch_of(m->M, m->K, m->groups, m->format, p.tn);
        p.q_scale = (uint8_t*)m->scratch + s.scales;
        Fp4Scales t = {};
        t.scale = scale;
        t.lds = lds;
        t.N = m->M;
        t.blocks = (m->K + block_of(m->format) - 1) / block_of(m->format);
        t.out = (uint8_t*)p.q_scale;
        t.tn = p.tn;
        t.atoms = (int)(stages(m->K) * stage_atoms(m->format));
        t.groups = m->groups ? m->groups : 1;
        t.offsets = m->groups ? m->offsets : nullptr;
        const cudaError_t e = launch_tile_scales_fp4(t, (cudaStream_t)stream);
        if (e != cudaSuccess) return done(e, "hccl_matmul_fp4");
    }
    return done(launch_matmul_fp4(m->dtype, p, (cudaStream_t)stream), "hccl_matmul_fp4");
}

hccl_status_t hccl_linear_fp4(const hccl_matmul_fp4_t* in, const void* x, int64_t ldx, hccl_dtype_t dt, const hccl_routing_t* r, void* stream) {
    if (!in) return HCCL_ERR_INVALID_ARG;
    hccl_matmul_fp4_t m = *in;
    if (r) {
        TRY(check_routing(r));
        m.groups = r->experts;
        m.offsets = r->offsets;
    }
    TRY(check_matmul(&m));
    Fp4Rows p;
    TRY(quant_params(&p, x, ldx, r ? r->tokens : m.M, m.K, dt, m.format, m.x_wide, r, (uint8_t*)m.scratch, 0, m.M));
    if (m.M == 0 || m.N == 0) return HCCL_OK;
    MatmulFp4 mm = matmul_params(&m);
    if (m.K) {
        const Scratch s = scratch_of(m.M, m.K, m.groups, m.format, mm.tn);
        p.ldq = mm.ldq = s.ldq;
        mm.q = p.q;
        mm.q_scale = p.scale = p.q + s.scales;
        p.tn = mm.tn;
        while (1 << p.shift < p.tn) p.shift++;
        p.atoms = (int)(stages(m.K) * stage_atoms(m.format));
        p.offsets = m.groups ? m.offsets : nullptr;
        p.groups = m.groups;
        const cudaError_t e = launch_quantise_fp4(dt, m.format, p, (cudaStream_t)stream);
        if (e != cudaSuccess) return done(e, "hccl_linear_fp4");
        mm.dependent = p.M > 0;
    }
    return done(launch_matmul_fp4(m.dtype, mm, (cudaStream_t)stream), "hccl_linear_fp4");
}

static hccl_status_t check_experts(const hccl_experts_fp4_t* e, int64_t tokens, int32_t top_k) {
    if (!e || tokens < 0 || tokens > HCCL_MAX_FEW_TOKENS || top_k < 1 || top_k > HCCL_MAX_TOP_K) return HCCL_ERR_INVALID_ARG;
    if (e->experts < 1 || e->experts > HCCL_MAX_EXPERTS || e->H < 1 || e->I < 1 || e->I > HCCL_MAX_FP4_K) return HCCL_ERR_INVALID_ARG;
    if (e->act != HCCL_ACT_SILU && e->act != HCCL_ACT_GELU && e->act != HCCL_ACT_RELU) return HCCL_ERR_INVALID_ARG;
    TRY(check_weights(e->I, e->H, e->gated ? 2 * e->experts : e->experts, e->format));
    return check_weights(e->H, e->I, e->experts, e->format);
}

hccl_status_t hccl_expert_layer_scratch_bytes(const hccl_experts_fp4_t* e, int64_t tokens, int32_t top_k, size_t* bytes) {
    TRY(check_experts(e, tokens, top_k));
    if (!bytes) return HCCL_ERR_INVALID_ARG;
    *bytes = few_fp4_scratch(tokens, e->H, e->I, top_k, e->gated != 0);
    return HCCL_OK;
}

hccl_status_t hccl_expert_layer_fp4(const hccl_experts_fp4_t* e, const void* x, int64_t ldx, hccl_dtype_t dt, const hccl_routing_t* r, void* y, int64_t ldy, void* scratch,
                                    size_t bytes, int32_t* dev_status, void* stream) {
    TRY(check_routing(r));
    TRY(check_experts(e, r->tokens, r->top_k));
    if (!hccl::valid_dtype(dt)) return HCCL_ERR_DTYPE;
    if (r->experts != e->experts) return HCCL_ERR_COUNT_MISMATCH;
    TRY(check_matrix(x, r->tokens, ldx, e->H, dt));
    TRY(check_matrix(y, r->tokens, ldy, e->H, dt));
    const int64_t N = e->gated ? 2 * e->I : e->I;
    if (!sane(N * e->experts, e->ld_up, (e->H + 1) / 2) || !sane(e->H * e->experts, e->ld_down, (e->I + 1) / 2)) return HCCL_ERR_INVALID_ARG;
    if (!e->up || !e->up_scale || !e->up_wide || !e->down || !e->down_scale || !e->down_wide) return HCCL_ERR_INVALID_ARG;
    if (!aligned(e->up, 16) || e->ld_up % 16 || !aligned(e->up_scale, 16) || !aligned(e->down, 16) || e->ld_down % 16 || !aligned(e->down_scale, 16)) return HCCL_ERR_ALIGNMENT;
    if (!aligned(e->up_wide, 4) || !aligned(e->up_bias, 4) || !aligned(e->down_wide, 4) || !aligned(e->down_bias, 4) || !aligned(dev_status, 4)) return HCCL_ERR_ALIGNMENT;
    if (r->tokens == 0) return HCCL_OK;
    if (!r->weights || !r->source) return HCCL_ERR_INVALID_ARG;
    if (!aligned(r->weights, 4) || !aligned(r->source, 4)) return HCCL_ERR_ALIGNMENT;
    if (!scratch || bytes < few_fp4_scratch(r->tokens, e->H, e->I, r->top_k, e->gated != 0)) return HCCL_ERR_WORKSPACE;
    if (!aligned(scratch, 128)) return HCCL_ERR_ALIGNMENT;
    FewFp4 p = {};
    p.T = r->tokens;
    p.H = e->H;
    p.I = e->I;
    p.ldx = ldx;
    p.ldy = ldy;
    p.top_k = r->top_k;
    p.experts = e->experts;
    p.format = e->format;
    p.act = e->act;
    p.gated = e->gated != 0;
    p.x = x;
    p.y = y;
    p.offsets = r->offsets;
    p.source = r->source;
    p.weights = r->weights;
    p.up = e->up;
    p.up_scale = (const uint8_t*)e->up_scale;
    p.ld_up = e->ld_up;
    p.up_wide = e->up_wide;
    p.up_bias = e->up_bias;
    p.down = e->down;
    p.down_scale = (const uint8_t*)e->down_scale;
    p.ld_down = e->ld_down;
    p.down_wide = e->down_wide;
    p.down_bias = e->down_bias;
    p.scratch = (char*)scratch;
    p.status = dev_status;
    return done(launch_few_fp4(dt, p, (cudaStream_t)stream), "hccl_expert_layer_fp4");
}

static hccl_status_t activate_params(ActivateParams* q, const hccl_activation_t* a, const void* x, int64_t ldx, int64_t M, int64_t I, hccl_dtype_t dt, const int32_t* offsets,
                                     int32_t groups) {
    if (!a || M < 0 || I < 0 || I > (INT64_C(1) << 40) || groups < 0) return HCCL_ERR_INVALID_ARG;
    if (a->act != HCCL_ACT_SILU && a->act != HCCL_ACT_GELU && a->act != HCCL_ACT_RELU) return HCCL_ERR_INVALID_ARG;
    if (!(a->p >= 0 && a->p < 1)) return HCCL_ERR_INVALID_ARG;
    if (!hccl::valid_dtype(dt)) return HCCL_ERR_DTYPE;
    if ((a->p > 0 && M && I && !a->seed) || (groups && !offsets)) return HCCL_ERR_INVALID_ARG;
    TRY(check_matrix(x, M, ldx, a->gated ? 2 * I : I, dt));
    if (!aligned(a->seed, 8) || !aligned(offsets, 4)) return HCCL_ERR_ALIGNMENT;
    *q = {};
    q->x = x;
    q->ldx = ldx;
    q->M = M;
    q->I = I;
    q->seed = (const long long*)a->seed;
    q->offsets = groups ? offsets : nullptr;
    q->groups = groups;
    q->act = a->act;
    q->gated = a->gated != 0;
    q->drop = a->p > 0;
    const double at = nearbyint(a->p * 4294967296.0);
    q->threshold = at > 4294967295.0 ? 4294967295u : (unsigned)at;
    q->keep = (float)(1.0 / (1.0 - a->p));
    return HCCL_OK;
}

hccl_status_t hccl_activate(const hccl_activation_t* a, const void* x, int64_t ldx, int64_t M, int64_t I, hccl_dtype_t dt, const int32_t* offsets, int32_t groups, void* y,
                            int64_t ldy, void* stream) {
    ActivateParams p;
    TRY(activate_params(&p, a, x, ldx, M, I, dt, offsets, groups));
    TRY(check_matrix(y, M, ldy, I, dt));
    p.out = y;
    p.ldo = ldy;
    return done(launch_activate(dt, p, (cudaStream_t)stream), "hccl_activate");
}

hccl_status_t hccl_activate_backward(const hccl_activation_t* a, const void* dy, int64_t lddy, const void* x, int64_t ldx, int64_t M, int64_t I, hccl_dtype_t dt,
                                     const int32_t* offsets, int32_t groups, void* dx, int64_t lddx, void* stream) {
    ActivateParams p;
    TRY(activate_params(&p, a, x, ldx, M, I, dt, offsets, groups));
    TRY(check_matrix(dy, M, lddy, I, dt));
    TRY(check_matrix(dx, M, lddx, a->gated ? 2 * I : I, dt));
    p.dy = dy;
    p.ldy = lddy;
    p.out = dx;
    p.ldo = lddx;
    return done(launch_activate_grad(dt, p, (cudaStream_t)stream), "hccl_activate_backward");
}

}  // extern "C"
