// Rows to 8-bit integers with a scale for each row: scale = max|x| / 127, q = round(x * (1 / max|x| * 127)). With a routing the row
// is written to every place that the token was sent to, so it is read and quantised once. Memory is the bound: a block
// holds its row in registers between the maximum and the rounding, so every element is read once.
#include <algorithm>

#include "experts.cuh"

namespace hccl {
namespace experts {
namespace {

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

// A thread holds P pieces of 16 bytes; rows longer than the block holds are read a second time.
template <typename T, int P> __global__ void __launch_bounds__(512) hccl_quantise_rows(const __grid_constant__ QuantParams p) {
    constexpr int N = Sixteen<T>::N;
    __shared__ unsigned part[2][16];
    asm volatile("griddepcontrol.launch_dependents;");  // the product may start to fetch its weights
    const int threads = blockDim.x, warps = threads / 32, K = (int)p.K, span = threads * N * P, copies = p.slots ? p.top_k : 1;
    int turn = 0;
    for (long long m = blockIdx.x; m < p.M; m += gridDim.x, turn ^= 1) {
        const T* x = (const T*)p.x + m * p.ldx;
        Sixteen<T> v[P];
        unsigned bits = 0;
        for (int at = 0; at < K; at += span) {
#pragma unroll
            for (int u = 0; u < P; u++) v[u].load(x, at + (u * threads + (int)threadIdx.x) * N, K, p.vec);
#pragma unroll
            for (int u = 0; u < P; u++) bits = max(bits, v[u].magnitude());
        }
        bits = __reduce_max_sync(0xffffffffu, bits);
        if (warps > 1) {  // two places in turn: a warp may be a row ahead of another's reading, not two
            if (threadIdx.x % 32 == 0) part[turn][threadIdx.x / 32] = bits;
            __syncthreads();
            bits = __reduce_max_sync(0xffffffffu, threadIdx.x % 32 < warps ? part[turn][threadIdx.x % 32] : 0u);
        }
        const float top = __uint_as_float(bits);
        const bool finite = top < INFINITY, some = finite && top >= TINY;
        const float inv = some ? __fmul_rn(1.f / top, 127.f) : 0.f;
        const float scale = !finite ? __int_as_float(0x7fc00000) : some ? top / 127.f : 0.f;
        for (int at = 0; at < K; at += span) {
            unsigned o[P][N / 4];
#pragma unroll
            for (int u = 0; u < P; u++) {
                if (span < K) v[u].load(x, at + (u * threads + (int)threadIdx.x) * N, K, p.vec);
#pragma unroll
                for (int j = 0; j < N / 4; j++)
                    o[u][j] = some ? four_bytes(__fmul_rn(v[u].value(4 * j), inv), __fmul_rn(v[u].value(4 * j + 1), inv), __fmul_rn(v[u].value(4 * j + 2), inv),
                                                __fmul_rn(v[u].value(4 * j + 3), inv))
                                   : 0u;
            }
            for (int c = 0; c < copies; c++) {
                const long long row = p.slots ? p.slots[m * p.top_k + c] : m;
                if (row < 0 || row >= p.n_q) continue;
                int8_t* q = p.q + row * p.ldq;
#pragma unroll
                for (int u = 0; u < P; u++) {
                    const int i = at + (u * threads + (int)threadIdx.x) * N;
                    if (p.vec_q && i + N <= K) {
                        if constexpr (N == 8) *(uint2*)(q + i) = make_uint2(o[u][0], o[u][N / 4 - 1]);
                        else *(unsigned*)(q + i) = o[u][0];
                    } else {
#pragma unroll
                        for (int j = 0; j < N; j++)
                            if (i + j < K) q[i + j] = (int8_t)(o[u][j / 4] >> (8 * (j & 3)));
                    }
                }
                if (at == 0 && threadIdx.x == 0) p.scale[row] = scale;
            }
        }
        if (K == 0 && threadIdx.x == 0)
            for (int c = 0; c < copies; c++) {
                const long long row = p.slots ? p.slots[m * p.top_k + c] : m;
                if (row >= 0 && row < p.n_q) p.scale[row] = 0.f;
            }
    }
}

template <typename T> cudaError_t quant_launch(const QuantParams& in, cudaStream_t s) {
    QuantParams p = in;
    if (p.M == 0) return cudaSuccess;
    constexpr int N = Sixteen<T>::N;
    p.vec = (uintptr_t)p.x % 16 == 0 && (p.ldx * sizeof(T)) % 16 == 0;
    p.vec_q = (uintptr_t)p.q % 8 == 0 && p.ldq % 8 == 0;
    int threads = 32;  // two pieces to a thread, up to 512 threads; then eight
    while (threads < 512 && threads * N * 2 < p.K) threads *= 2;
    const int blocks = (int)std::min<long long>(p.M, (long long)SMS * (2048 / threads));
    if (p.K <= 512 * N * 2) hccl_quantise_rows<T, 2><<<blocks, threads, 0, s>>>(p);
    else hccl_quantise_rows<T, 8><<<blocks, threads, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_quantise(int dt, const QuantParams& p, cudaStream_t s) {
    if (dt == HCCL_FP32) return quant_launch<float>(p, s);
    if (dt == HCCL_BF16) return quant_launch<__nv_bfloat16>(p, s);
    return quant_launch<__half>(p, s);
}

}  // namespace experts
}  // namespace hccl
