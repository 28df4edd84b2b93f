// From elements to bytes: what the quantiser and the product of few rows share. scale = max|x| / 127, q = round(x * (1 / max|x| * 127)).
#pragma once
#include "experts.cuh"

namespace hccl {
namespace experts {

constexpr float TINY = 1e-30f;  // below it 1 / max could overflow

// 16 bytes of a row as they lie in memory, beyond K zeros.
template <typename T> struct Sixteen {
    static constexpr int N = 16 / sizeof(T);
    unsigned w[4];
    __device__ __forceinline__ void load(const T* x, int i, int K, bool vec) {
        if (vec && i + N <= K) {
            const uint4 v = *(const uint4*)(x + i);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else {
#pragma unroll
            for (int u = 0; u < 4; u++) {
                w[u] = 0;
#pragma unroll
                for (int j = 0; j < N / 4; j++) {
                    const int at = i + u * (N / 4) + j;
                    if (at < K) w[u] |= (sizeof(T) == 4 ? ((const unsigned*)x)[at] : (unsigned)((const unsigned short*)x)[at]) << (16 * j);
                }
            }
        }
    }
    // The largest magnitude, as the bits of a number that is not negative: they are in the numbers' order, with NaN above infinity, so that it sticks.
    __device__ __forceinline__ unsigned magnitude() const;
    __device__ __forceinline__ float value(int j) const;
};
template <> __device__ __forceinline__ unsigned Sixteen<float>::magnitude() const {
    return max(max(w[0] & 0x7fffffffu, w[1] & 0x7fffffffu), max(w[2] & 0x7fffffffu, w[3] & 0x7fffffffu));
}
template <> __device__ __forceinline__ float Sixteen<float>::value(int j) const { return __uint_as_float(w[j]); }
template <> __device__ __forceinline__ unsigned Sixteen<__nv_bfloat16>::magnitude() const {
    __nv_bfloat162 m[4];
#pragma unroll
    for (int u = 0; u < 4; u++) {
        const unsigned a = w[u] & 0x7fff7fffu;
        m[u] = *(const __nv_bfloat162*)&a;
    }
    const __nv_bfloat162 r = __hmax2_nan(__hmax2_nan(m[0], m[1]), __hmax2_nan(m[2], m[3]));
    return max(__float_as_uint(__low2float(r)), __float_as_uint(__high2float(r))) & 0x7fffffffu;
}
template <> __device__ __forceinline__ float Sixteen<__nv_bfloat16>::value(int j) const { return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16); }
template <> __device__ __forceinline__ unsigned Sixteen<__half>::magnitude() const {
    __half2 m[4];
#pragma unroll
    for (int u = 0; u < 4; u++) {
        const unsigned a = w[u] & 0x7fff7fffu;
        m[u] = *(const __half2*)&a;
    }
    const __half2 r = __hmax2_nan(__hmax2_nan(m[0], m[1]), __hmax2_nan(m[2], m[3]));
    return max(__float_as_uint(__low2float(r)) & 0x7fffffffu, __float_as_uint(__high2float(r)) & 0x7fffffffu);
}
template <> __device__ __forceinline__ float Sixteen<__half>::value(int j) const {
    const unsigned short h = (unsigned short)(j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu);
    return __half2float(__ushort_as_half(h));
}

// Four numbers within [-127.5, 127.5] to bytes. Adding 1.5 * 2^23 leaves the number, rounded half to even, in the low bits.
__device__ __forceinline__ unsigned four_bytes(float a, float b, float c, float d) {
    const float big = 12582912.f;
    const unsigned lo = __byte_perm(__float_as_uint(__fadd_rn(a, big)), __float_as_uint(__fadd_rn(b, big)), 0x0040);
    const unsigned hi = __byte_perm(__float_as_uint(__fadd_rn(c, big)), __float_as_uint(__fadd_rn(d, big)), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
}

// The factor and the scale of a row from the bits of its largest magnitude. Factor 0: the row's bytes are zero.
__device__ __forceinline__ void row_scale(unsigned bits, float* factor, float* scale) {
    const float top = __uint_as_float(bits);
    const bool finite = top < INFINITY, some = finite && top >= TINY;
    *factor = some ? __fmul_rn(1.f / top, 127.f) : 0.f;
    *scale = !finite ? __int_as_float(0x7fc00000) : some ? top / 127.f : 0.f;
}
// Four elements of a piece, from the j-th on.
template <typename T> __device__ __forceinline__ unsigned quantised(const Sixteen<T>& v, int j, float factor) {
    if (factor == 0.f) return 0u;  // an infinity times 0 would be NaN
    return four_bytes(__fmul_rn(v.value(j), factor), __fmul_rn(v.value(j + 1), factor), __fmul_rn(v.value(j + 2), factor), __fmul_rn(v.value(j + 3), factor));
}

}  // namespace experts
}  // namespace hccl
