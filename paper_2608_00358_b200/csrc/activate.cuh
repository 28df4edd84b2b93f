// Activations of expert layers and their slopes, in 32 bits.
#pragma once
#include "two.cuh"

namespace hccl {
namespace experts {

// 1 / x within 1 ulp.
__device__ __forceinline__ float reciprocal(float x) {
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// 1 / (1 + exp(-x)), by an exponential that is never infinite.
__device__ __forceinline__ float logistic(float x) {
    const float e = expf(-fabsf(x)), r = reciprocal(1.f + e);
    return x >= 0.f ? r : e * r;
}
__device__ __forceinline__ float activation(int act, float g) {
    if (act == HCCL_ACT_SILU) return g * logistic(g);
    if (act == HCCL_ACT_GELU) return g * normcdff(g);
    return g > 0.f || g != g ? g : 0.f;
}
// And its derivative; of the rectifier at 0: 0.
__device__ __forceinline__ void activation_slope(int act, float g, float* a, float* slope) {
    if (act == HCCL_ACT_SILU) {
        const float s = logistic(g);
        *a = g * s;
        *slope = fmaf(*a, 1.f - s, s);
    } else if (act == HCCL_ACT_GELU) {
        const float phi = normcdff(g);
        *a = g * phi;
        *slope = phi + g * expf(-0.5f * g * g) * 0.39894228f;
    } else {
        *a = g > 0.f || g != g ? g : 0.f;
        *slope = g > 0.f ? 1.f : 0.f;
    }
}

struct ActivateParams {
    const void *x, *dy;  // [M, 2 I] (not gated: [M, I]); the gradient of the result [M, I]
    void* out;
    long long ldx, ldy, ldo, M, I;
    const long long* seed;  // key and call
    const int* offsets;     // null: all rows
    int groups, act, gated, drop;
    unsigned threshold;     // of a 32-bit word
    float keep;             // 1 / (1 - p)
};
cudaError_t launch_activate(int dt, const ActivateParams& p, cudaStream_t s);
cudaError_t launch_activate_grad(int dt, const ActivateParams& p, cudaStream_t s);

}  // namespace experts
}  // namespace hccl
