// Rows to 8-bit integers with a scale for each row: scale = max|x| / 127, q = round(x * (1 / max|x| * 127)). One block holds a row;
// with a routing the row is written to every place that the token was sent to, so it is read and quantised once.
#include "experts.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int QUANT_THREADS = 256;
constexpr float TINY = 1e-30f;  // below it 127 / max could overflow

template <typename T> __global__ void __launch_bounds__(QUANT_THREADS) hccl_quantise_rows(const __grid_constant__ QuantParams p) {
    __shared__ float part[QUANT_THREADS / 32];
    asm volatile("griddepcontrol.launch_dependents;");  // the product may start to fetch its weights
    for (long long m = blockIdx.x; m < p.M; m += gridDim.x) {
        const T* x = (const T*)p.x + m * p.ldx;
        float top = 0.f;
        for (long long k = threadIdx.x; k < p.K; k += QUANT_THREADS) {
            const float v = fabsf(to_f32<T>(x[k]));
            top = v > top || isnan(v) ? v : top;  // NaN sticks
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const float v = __shfl_xor_sync(0xffffffffu, top, o);
            top = v > top || isnan(v) ? v : top;
        }
        if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = top;
        __syncthreads();
        top = part[0];
        for (int i = 1; i < QUANT_THREADS / 32; i++) top = part[i] > top || isnan(part[i]) ? part[i] : top;
        __syncthreads();
        const bool finite = top < INFINITY;
        const float inv = finite && top >= TINY ? __fmul_rn(1.f / top, 127.f) : 0.f;
        const float scale = !finite ? __int_as_float(0x7fc00000) : top >= TINY ? top / 127.f : 0.f;
        const int copies = p.slots ? p.top_k : 1;
        for (int c = 0; c < copies; c++) {
            const long long row = p.slots ? p.slots[m * p.top_k + c] : m;
            if (row < 0 || row >= p.n_q) continue;
            int8_t* q = p.q + row * p.ldq;
            for (long long k = threadIdx.x; k < p.K; k += QUANT_THREADS) q[k] = finite ? (int8_t)__float2int_rn(to_f32<T>(x[k]) * inv) : 0;
            if (threadIdx.x == 0) p.scale[row] = scale;
        }
    }
}

template <typename T> cudaError_t quant_launch(const QuantParams& p, cudaStream_t s) {
    const long long most = SMS * 8;
    const int blocks = (int)(p.M < most ? p.M : most);
    if (blocks == 0) return cudaSuccess;
    hccl_quantise_rows<T><<<blocks, QUANT_THREADS, 0, s>>>(p);
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
