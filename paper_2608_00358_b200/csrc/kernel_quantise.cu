// Rows to 8-bit integers with a scale for each row: scale = max|x| / 127, q = round(x * (1 / max|x| * 127)). With a routing the row
// is written to every place that the token was sent to, so it is read and quantised once. Memory is the bound: a block
// holds its row in registers between the maximum and the rounding, so every element is read once.
#include <algorithm>

#include "rows_i8.cuh"

namespace hccl {
namespace experts {
namespace {

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
        float factor, scale;
        row_scale(bits, &factor, &scale);
        for (int at = 0; at < K; at += span) {
            unsigned o[P][N / 4];
#pragma unroll
            for (int u = 0; u < P; u++) {
                if (span < K) v[u].load(x, at + (u * threads + (int)threadIdx.x) * N, K, p.vec);
#pragma unroll
                for (int j = 0; j < N / 4; j++) o[u][j] = quantised(v[u], 4 * j, factor);
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
    const int blocks = (int)std::min<long long>(p.M, 1 << 30);  // one for each row: the hardware hands out the next one where one has ended
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
