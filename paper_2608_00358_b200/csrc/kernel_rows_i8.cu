// Products in 8-bit integers for at most 8 rows: the weights are read once and their bytes are the time, so a call's fixed cost is what can
// be saved. Against the kernel of tiles (tensor memory, tensor maps, a cluster that adds its parts, the quantiser's launch before it) this one
// starts loading weights with its first instruction and quantises the rows itself where they are short.
//
// mma.sync m16n8k32: 16 channels x 8 rows. A warp takes 128 bytes of K of 16 channels at a time, straight from memory to the registers of
// the instruction: of each half, lane 4g + t loads bytes 16t .. 16t + 15 of channels g and g + 8, two instructions' worth. That hands the instruction its
// columns of K in another order than they have in memory, the same for both operands, and a sum does not mind. Four such items (8 KB) are in flight for
// each warp, across the end of a group of channels. The 8 warps of a block share K and add their sums, exact integers, in shared memory.
//
// Measured (B200, weights not in the L2): one row, 8192 x 4096 9 us with the quantising = 3.7 TB/s (the tiles: 12.6), 16384 x 8192 25 us = 5.2 TB/s; 8 rows, 8192 x 4096 10.5 us
// (the tiles: 11.4 for 16).
#include <algorithm>
#include <atomic>

#include "rows_i8.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int FEW_THREADS = 256, FEW_WARPS = FEW_THREADS / 32, DEEP = 4, ITEM = 128 /* bytes of K */;

struct FewParams {
    MatmulParams m;
    const void* x;  // null: m.a and m.a_scale hold the rows in 8 bits
    long long ldx;
    int x_dt, x_vec, q_stride;
};

template <typename X> __device__ __forceinline__ void largest(const FewParams& p, unsigned* top) {
    constexpr int N = Sixteen<X>::N;
    const int K = (int)p.m.K, pieces = (K + N - 1) / N;
    for (int r = 0; r < (int)p.m.M; r++) {
        unsigned bits = 0;
        for (int i = threadIdx.x; i < pieces; i += FEW_THREADS) {
            Sixteen<X> v;
            v.load((const X*)p.x + r * p.ldx, i * N, K, p.x_vec);
            bits = max(bits, v.magnitude());
        }
        bits = __reduce_max_sync(0xffffffffu, bits);
        if (threadIdx.x % 32 == 0) atomicMax(&top[r], bits);
    }
}
template <typename X> __device__ __forceinline__ void quantise(const FewParams& p, const unsigned* top, float* scale, char* q) {
    constexpr int N = Sixteen<X>::N;
    const int K = (int)p.m.K, pieces = (p.q_stride - 16) / N;  // zeros beyond K
    for (int r = 0; r < (int)p.m.M; r++) {
        float factor, s;
        row_scale(top[r], &factor, &s);
        if (threadIdx.x == 0) scale[r] = s;
        for (int i = threadIdx.x; i < pieces; i += FEW_THREADS) {
            Sixteen<X> v;
            v.load((const X*)p.x + r * p.ldx, i * N, K, p.x_vec);
            unsigned* to = (unsigned*)(q + r * p.q_stride + i * N);
#pragma unroll
            for (int j = 0; j < N / 4; j++) to[j] = quantised(v, 4 * j, factor);
        }
    }
}

__device__ __forceinline__ uint4 load_once(const int8_t* at) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(at));
    return v;
}
__device__ __forceinline__ void mma(int (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename T> __global__ void __launch_bounds__(FEW_THREADS, 2) hccl_matmul_i8_few(const __grid_constant__ FewParams p) {
    extern __shared__ __align__(16) char q[];  // [M][q_stride] rows in 8 bits
    __shared__ unsigned top[8];
    __shared__ float scale[8];
    __shared__ int part[2][FEW_WARPS][128];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const int K = (int)p.m.K, M = (int)p.m.M, N = (int)p.m.N;
    const int groups = (N + 15) / 16, per = (K + ITEM * FEW_WARPS - 1) / (ITEM * FEW_WARPS);  // items of a warp in a group of channels
    const int mine = (groups - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x, items = mine * per;
    const int k_first = warp * ITEM + t * 16;

    // Item i: bytes from (warp + 8 (i % per)) * ITEM on of the block's channel group i / per. Pieces beyond K or beyond the items are zero.
    int asked = 0, ask_k = k_first, ask_n = 0, ask_group = (int)blockIdx.x;
    const int8_t *lo_row = p.m.w + (long long)min(ask_group * 16 + g, N - 1) * p.m.ldw, *hi_row = p.m.w + (long long)min(ask_group * 16 + 8 + g, N - 1) * p.m.ldw;
    const auto fetch = [&](uint4 (&v)[4]) {
        const bool some = asked < items;
        v[0] = v[1] = v[2] = v[3] = make_uint4(0, 0, 0, 0);
        if (some && ask_k < K) v[0] = load_once(lo_row + ask_k), v[1] = load_once(hi_row + ask_k);
        if (some && ask_k + 64 < K) v[2] = load_once(lo_row + ask_k + 64), v[3] = load_once(hi_row + ask_k + 64);
        asked++;
        ask_k += ITEM * FEW_WARPS;
        if (++ask_n == per) {
            ask_n = 0;
            ask_k = k_first;
            ask_group += (int)gridDim.x;
            lo_row = p.m.w + (long long)min(ask_group * 16 + g, N - 1) * p.m.ldw;
            hi_row = p.m.w + (long long)min(ask_group * 16 + 8 + g, N - 1) * p.m.ldw;
        }
    };
    uint4 v[DEEP][4];
#pragma unroll
    for (int u = 0; u < DEEP; u++) fetch(v[u]);

    if (threadIdx.x < 8) top[threadIdx.x] = 0;
    if (p.m.dependent) asm volatile("griddepcontrol.wait;" ::: "memory");
    if (p.x) {
        __syncthreads();
        if (p.x_dt == HCCL_FP32) largest<float>(p, top);
        else if (p.x_dt == HCCL_BF16) largest<__nv_bfloat16>(p, top);
        else largest<__half>(p, top);
        __syncthreads();
        if (p.x_dt == HCCL_FP32) quantise<float>(p, top, scale, q);
        else if (p.x_dt == HCCL_BF16) quantise<__nv_bfloat16>(p, top, scale, q);
        else quantise<__half>(p, top, scale, q);
    } else {
        const int pieces = (p.q_stride - 16) / 16;
        for (int i = threadIdx.x; i < M * pieces; i += FEW_THREADS) {
            const int r = i / pieces, k = i % pieces * 16;
            const int8_t* row = p.m.a + r * p.m.lda;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (k < K) {
                v = *(const uint4*)(row + k);
                if (k + 16 > K) {  // what the row's last 16 bytes hold beyond K
                    unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int j = 0; j < 16; j++)
                        if (k + j >= K) w[j / 4] &= ~(0xffu << (8 * (j & 3)));
                    v = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            *(uint4*)(q + r * p.q_stride + k) = v;
        }
        if (threadIdx.x < M) scale[threadIdx.x] = p.m.a_scale[threadIdx.x];
    }
    __syncthreads();

    int acc[4] = {0, 0, 0, 0}, n = 0, at = warp * ITEM, group = (int)blockIdx.x, turn = 0;
    const char* row = q + min(g, M - 1) * p.q_stride + t * 16;
    for (int i0 = 0; i0 < items; i0 += DEEP) {
#pragma unroll
        for (int u = 0; u < DEEP; u++) {
            if (i0 + u >= items) break;
            uint4 b0 = make_uint4(0, 0, 0, 0), b1 = b0;
            if (g < M && at < p.q_stride - 16) b0 = *(const uint4*)(row + at), b1 = *(const uint4*)(row + at + 64);
            mma(acc, v[u][0].x, v[u][1].x, v[u][0].y, v[u][1].y, b0.x, b0.y);
            mma(acc, v[u][0].z, v[u][1].z, v[u][0].w, v[u][1].w, b0.z, b0.w);
            mma(acc, v[u][2].x, v[u][3].x, v[u][2].y, v[u][3].y, b1.x, b1.y);
            mma(acc, v[u][2].z, v[u][3].z, v[u][2].w, v[u][3].w, b1.z, b1.w);
            fetch(v[u]);
            at += ITEM * FEW_WARPS;
            if (++n == per) {  // the same for all warps
                n = 0;
                at = warp * ITEM;
                int* to = part[turn][warp];  // [channel][row]
                *(int2*)(to + g * 8 + 2 * t) = make_int2(acc[0], acc[1]);
                *(int2*)(to + (g + 8) * 8 + 2 * t) = make_int2(acc[2], acc[3]);
                acc[0] = acc[1] = acc[2] = acc[3] = 0;
                __syncthreads();
                if (threadIdx.x < 128) {
                    const int c = threadIdx.x % 16, r = threadIdx.x / 16, chan = group * 16 + c;
                    if (chan < N && r < M) {
                        int sum = 0;
#pragma unroll
                        for (int w = 0; w < FEW_WARPS; w++) sum += part[turn][w][c * 8 + r];
                        float v = __fmul_rn(__fmul_rn((float)sum, scale[r]), p.m.w_scale[chan]);
                        if (p.m.bias) v = __fadd_rn(v, p.m.bias[chan]);
                        ((T*)p.m.y)[r * p.m.ldy + chan] = from_f32<T>(v);
                    }
                }
                turn ^= 1;  // the next group's sums go elsewhere: they are not written over before the barrier after next
                group += (int)gridDim.x;
            }
        }
    }
}

// Shared memory for the rows: a third of an SM's, so that two blocks fit with room to spare.
constexpr long long FEW_SMEM = 72 * 1024;
int few_stride(long long K) { return (int)((K + ITEM - 1) / ITEM * ITEM + 16); }  // 16: the rows of a quarter warp start on different banks

template <typename T> cudaError_t few_launch(const FewParams& in, cudaStream_t s) {
    FewParams p = in;
    p.q_stride = few_stride(p.m.K);
    const size_t smem = (size_t)p.m.M * p.q_stride;
    if (smem > 40 * 1024) {
        static std::atomic<bool> ready[64];
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev >= 64 || !ready[dev]) {
            e = cudaFuncSetAttribute(hccl_matmul_i8_few<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)FEW_SMEM);
            if (e != cudaSuccess) return e;
            if (dev < 64) ready[dev] = true;
        }
    }
    const long long groups = (p.m.N + 15) / 16;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min<long long>(groups, 2 * SMS));
    cfg.blockDim = dim3(FEW_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = p.m.dependent ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, hccl_matmul_i8_few<T>, p);
}

cudaError_t few(int dt, const FewParams& p, cudaStream_t s) {
    if (dt == HCCL_FP32) return few_launch<float>(p, s);
    if (dt == HCCL_BF16) return few_launch<__nv_bfloat16>(p, s);
    return few_launch<__half>(p, s);
}

}  // namespace

bool few_rows(const MatmulParams& p) { return p.groups == 0 && p.M <= 8 && p.K > 0 && p.M * few_stride(p.K) <= FEW_SMEM; }

// Rows short enough for every block to quantise them again: two passes over them out of the L2 are hidden behind the weights then.
bool few_rows_quantise(const MatmulParams& p) { return p.M * p.K <= 8192; }

cudaError_t launch_matmul_i8_few(int dt, const MatmulParams& m, cudaStream_t s) {
    FewParams p = {};
    p.m = m;
    return few(dt, p, s);
}

cudaError_t launch_linear_i8_few(int dt, const MatmulParams& m, const QuantParams& x, int x_dt, cudaStream_t s) {
    FewParams p = {};
    p.m = m;
    p.x = x.x;
    p.ldx = x.ldx;
    p.x_dt = x_dt;
    const int es = x_dt == HCCL_FP32 ? 4 : 2;
    p.x_vec = (uintptr_t)x.x % 16 == 0 && (x.ldx * es) % 16 == 0;
    return few(dt, p, s);
}

}  // namespace experts
}  // namespace hccl
