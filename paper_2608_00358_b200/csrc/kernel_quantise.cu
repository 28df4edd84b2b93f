// Rows to 8-bit integers with a scale for each row: scale = max|x| / 127, q = round(x * (1 / max|x| * 127)). With a routing the row
// is written to every place that the token was sent to, so it is read and quantised once. Memory is the bound: a block
// holds its row in registers between the maximum and the rounding, so every element is read once.
#include <algorithm>

#include "experts.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr float TINY = 1e-30f;  // below it 1 / max could overflow

template <typename T, int N> __device__ __forceinline__ void load_piece(const T* x, long long i, long long K, bool vec, float (&v)[N]) {
    if (vec && i + N <= K) {
        if (sizeof(T) == 4) {  // 16 elements: four loads
#pragma unroll
            for (int u = 0; u < N / 4; u++) {
                const float4 f = *(const float4*)(x + i + 4 * u);
                v[4 * u] = f.x, v[4 * u + 1] = f.y, v[4 * u + 2] = f.z, v[4 * u + 3] = f.w;
            }
        } else {
#pragma unroll
            for (int u = 0; u < N / 8; u++) {
                Pack<T, 16 / sizeof(T)> p;
                p.raw = *(const uint4*)(x + i + 8 * u);
#pragma unroll
                for (int j = 0; j < 8; j++) v[8 * u + j] = to_f32<T>(p.v[j % (16 / sizeof(T))]);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; j++) v[j] = i + j < K ? to_f32<T>(x[i + j]) : 0.f;
    }
}

__device__ __forceinline__ float keep_nan_max(float a, float b) { return b > a || isnan(b) ? b : a; }  // of numbers that are not negative; NaN sticks

// A thread holds P pieces of 16 elements; rows longer than the block holds are read a second time.
template <typename T, int P> __global__ void __launch_bounds__(512) hccl_quantise_rows(const __grid_constant__ QuantParams p) {
    __shared__ float part[16];
    asm volatile("griddepcontrol.launch_dependents;");  // the product may start to fetch its weights
    const int threads = blockDim.x, warps = threads / 32;
    const bool held = (long long)threads * 16 * P >= p.K;
    for (long long m = blockIdx.x; m < p.M; m += gridDim.x) {
        const T* x = (const T*)p.x + m * p.ldx;
        float v[P][16], top = 0.f;
        for (long long at = 0; at < p.K; at += (long long)threads * 16 * P) {
#pragma unroll
            for (int u = 0; u < P; u++) {
                load_piece<T, 16>(x, at + ((long long)u * threads + threadIdx.x) * 16, p.K, p.vec, v[u]);
#pragma unroll
                for (int j = 0; j < 16; j++) top = keep_nan_max(top, fabsf(v[u][j]));
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) top = keep_nan_max(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (warps > 1) {
            if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = top;
            __syncthreads();
            top = part[0];
            for (int i = 1; i < warps; i++) top = keep_nan_max(top, part[i]);
            __syncthreads();
        }
        const bool finite = top < INFINITY, some = finite && top >= TINY;
        const float inv = some ? __fmul_rn(1.f / top, 127.f) : 0.f;
        const float scale = !finite ? __int_as_float(0x7fc00000) : some ? top / 127.f : 0.f;
        const int copies = p.slots ? p.top_k : 1;
        for (long long at = 0; at < p.K; at += (long long)threads * 16 * P) {
#pragma unroll
            for (int u = 0; u < P; u++) {
                const long long i = at + ((long long)u * threads + threadIdx.x) * 16;
                if (i >= p.K) continue;
                if (!held) load_piece<T, 16>(x, i, p.K, p.vec, v[u]);
                union {
                    uint4 raw;
                    int8_t b[16];
                } o;
#pragma unroll
                for (int j = 0; j < 16; j++) o.b[j] = finite ? (int8_t)__float2int_rn(v[u][j] * inv) : (int8_t)0;
                for (int c = 0; c < copies; c++) {
                    const long long row = p.slots ? p.slots[m * p.top_k + c] : m;
                    if (row < 0 || row >= p.n_q) continue;
                    int8_t* q = p.q + row * p.ldq + i;
                    if (p.vec_q && i + 16 <= p.K) *(uint4*)q = o.raw;
                    else
#pragma unroll
                        for (int j = 0; j < 16; j++)
                            if (i + j < p.K) q[j] = o.b[j];
                }
            }
        }
        for (int c = threadIdx.x; c < copies; c += threads) {
            const long long row = p.slots ? p.slots[m * p.top_k + c] : m;
            if (row >= 0 && row < p.n_q) p.scale[row] = scale;
        }
    }
}

template <typename T> cudaError_t quant_launch(const QuantParams& in, cudaStream_t s) {
    QuantParams p = in;
    if (p.M == 0) return cudaSuccess;
    p.vec = (uintptr_t)p.x % 16 == 0 && (p.ldx * sizeof(T)) % 16 == 0;
    p.vec_q = (uintptr_t)p.q % 16 == 0 && p.ldq % 16 == 0;
    // a warp for every 512 elements while a thread holds one piece, up to 512 threads; then two pieces each
    int threads = 32;
    while (threads < 512 && threads * 16 < p.K) threads *= 2;
    const int blocks = (int)std::min<long long>(p.M, (long long)SMS * (2048 / threads));
    if (p.K <= 512 * 16) hccl_quantise_rows<T, 1><<<blocks, threads, 0, s>>>(p);
    else hccl_quantise_rows<T, 2><<<blocks, threads, 0, s>>>(p);
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
