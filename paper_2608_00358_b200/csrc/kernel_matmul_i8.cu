// Product of 8-bit integers with scales for each row of both operands, sums exact in 32-bit integers.
#include "experts.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int TM = 64, TN = 64, TK = 64, MM_THREADS = 256;

// One block forms 64 rows x 64 columns; each thread 4 x 4 of them, four products at a time.
template <typename T> __global__ void __launch_bounds__(MM_THREADS) hccl_matmul_i8_simple(const __grid_constant__ MatmulParams p) {
    __shared__ int as[TM][TK / 4 + 1], ws[TN][TK / 4 + 1];
    // which rows: tiles are counted group by group
    long long m0 = 0, m1 = p.M;
    int g = 0;
    long long tile = blockIdx.y;
    if (p.groups) {
        for (g = 0; g < p.groups; g++) {
            m0 = max(0ll, (long long)p.offsets[g]);
            m1 = min(p.M, (long long)p.offsets[g + 1]);
            const long long n = m1 > m0 ? (m1 - m0 + TM - 1) / TM : 0;
            if (tile < n) break;
            tile -= n;
        }
        if (g == p.groups) return;
    }
    m0 += tile * TM;
    const long long n0 = (long long)blockIdx.x * TN;
    const int8_t* w = p.w + ((long long)g * p.N) * p.ldw;
    int acc[4][4] = {};
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (long long k0 = 0; k0 < p.K; k0 += TK) {
        for (int i = threadIdx.x; i < TM * TK; i += MM_THREADS) {
            const int r = i / TK, c = i % TK;
            const bool k_in = k0 + c < p.K;
            ((int8_t*)as[r])[c] = (k_in && m0 + r < m1) ? p.a[(m0 + r) * p.lda + k0 + c] : 0;
            ((int8_t*)ws[r])[c] = (k_in && n0 + r < p.N) ? w[(n0 + r) * p.ldw + k0 + c] : 0;
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < TK / 4; c++)
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] = __dp4a(as[ty + 16 * i][c], ws[tx + 16 * j][c], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; i++)
        for (int j = 0; j < 4; j++) {
            const long long m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m >= m1 || n >= p.N) continue;
            float v = (float)acc[i][j] * p.a_scale[m] * p.w_scale[(long long)g * p.N + n];
            if (p.bias) v += p.bias[(long long)g * p.N + n];
            ((T*)p.y)[m * p.ldy + n] = from_f32<T>(v);
        }
}

template <typename T> cudaError_t matmul_launch(const MatmulParams& p, cudaStream_t s) {
    const long long tiles = (p.M + TM - 1) / TM + p.groups;
    hccl_matmul_i8_simple<T><<<dim3((unsigned)((p.N + TN - 1) / TN), (unsigned)tiles), MM_THREADS, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_matmul_i8(int dt, const MatmulParams& p, cudaStream_t s) {
    if (p.M == 0 || p.N == 0) return cudaSuccess;
    if (dt == HCCL_FP32) return matmul_launch<float>(p, s);
    if (dt == HCCL_BF16) return matmul_launch<__nv_bfloat16>(p, s);
    return matmul_launch<__half>(p, s);
}

}  // namespace experts
}  // namespace hccl
