// Kernels of the expert-layer operators (routing, exchange of rows, products in 8-bit integers): parameter records,
// launchers, and the few device helpers that they share. experts.cu holds the C entry points and their checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/hccl.h"

namespace hccl {
namespace experts {

constexpr int SMS = 148;

// ---------------------------------------------------------------- element access
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);  // one rounding to nearest even
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// A piece of a row: BYTES at once (16, 8, 4, or one element).
template <int BYTES> struct Piece;
template <> struct Piece<16> { using type = uint4; };
template <> struct Piece<8> { using type = uint2; };
template <> struct Piece<4> { using type = unsigned int; };
template <> struct Piece<2> { using type = unsigned short; };

template <typename A, typename B> struct Same {
    static constexpr bool value = false;
};
template <typename A> struct Same<A, A> {
    static constexpr bool value = true;
};

template <typename T, int N> union Pack {
    typename Piece<N * sizeof(T)>::type raw;
    T v[N];
    unsigned w[N * sizeof(T) >= 4 ? N * sizeof(T) / 4 : 1];
    __device__ __forceinline__ Pack() {}
    // Two 16-bit elements of a word at a time, where there are two.
    __device__ __forceinline__ void get(float (&f)[N]) const {
        if constexpr (sizeof(T) == 2 && N >= 2) {
#pragma unroll
            for (int i = 0; i < N / 2; i++) two(w[i], f[2 * i], f[2 * i + 1]);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) f[i] = to_f32<T>(v[i]);
        }
    }
    __device__ __forceinline__ void set(const float (&f)[N]) {
        if constexpr (sizeof(T) == 2 && N >= 2) {
#pragma unroll
            for (int i = 0; i < N / 2; i++) w[i] = word(f[2 * i], f[2 * i + 1]);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) v[i] = from_f32<T>(f[i]);
        }
    }
    static __device__ __forceinline__ void two(unsigned w, float& a, float& b) {
        if constexpr (sizeof(T) == 2) {
            if constexpr (BF) {
                a = __uint_as_float(w << 16);
                b = __uint_as_float(w & 0xffff0000u);
            } else {
                const float2 f = __half22float2(*(const __half2*)&w);
                a = f.x;
                b = f.y;
            }
        }
    }
    static __device__ __forceinline__ unsigned word(float a, float b) {
        if constexpr (BF) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
            return *(const unsigned*)&h;
        } else {
            const __half2 h = __floats2half2_rn(a, b);
            return *(const unsigned*)&h;
        }
    }
    static constexpr bool BF = Same<T, __nv_bfloat16>::value;
};

// ---------------------------------------------------------------- routing
struct RouteParams {
    const void* logits;
    const float* bias;
    const uint8_t* mask;
    long long ld, tokens;
    int E, K, groups, per_group, top_groups, group_best, sigmoid, renorm;
    float scale;
    int per4, magic;     // quads of experts lie in one group each; e * magic >> 20 = e / per_group
    int segment;         // quads of a group, if they are 1, 2, 4, .. lanes side by side; 0 otherwise
    int vec;             // rows of logits can be read four elements at once
    int warps;           // per block
    int chunk, chunks;   // tokens counted together; chunks of them (1: a single block does everything)
    int* ids;
    float* weights;
    long long* counts;
    int *offsets, *slots, *source;
    uint8_t* hist;       // [chunks][E rounded up to 16] rows of each expert in each chunk
};

struct RouteGradParams {
    RouteParams r;  // logits, bias, mask, sizes, ids
    const float* dweights;
    void* dlogits;
    long long ldd;
    int vec;
};

size_t route_workspace(int E, long long tokens);
cudaError_t launch_route(int dt, const RouteParams& p, cudaStream_t s);
cudaError_t launch_route_grad(int dt, const RouteGradParams& p, cudaStream_t s);

// ---------------------------------------------------------------- exchange of rows
struct RowsParams {
    const void* x;        // [tokens, H]: dispatch's input, combine_backward's dy
    void* y;              // [tokens, H]: combine's output
    const void* rows;     // [n_rows, H]
    void* rows_out;       // [n_rows, H]
    long long ldx, ldy, ldr, ldro, tokens, n_rows, H;
    int K, E;
    const int* slots;
    const int* offsets;
    const float* weights; // null: 1
    float* dweights;
};

cudaError_t launch_dispatch(int dt, const RowsParams& p, cudaStream_t s);
cudaError_t launch_combine(int dt, const RowsParams& p, cudaStream_t s);
cudaError_t launch_combine_grad(int dt, const RowsParams& p, cudaStream_t s);

// ---------------------------------------------------------------- products in 8-bit integers
struct QuantParams {
    const void* x;
    long long ldx, M, K, ldq, n_q;
    int8_t* q;
    float* scale;
    int vec, vec_q;    // 16 bytes at a time
    const int* slots;  // null: row m of x to row m of q
    int top_k;
};
cudaError_t launch_quantise(int dt, const QuantParams& p, cudaStream_t s);

struct MatmulParams {
    long long M, N, K, lda, ldw, ldy;
    int groups;  // 0: one matrix
    const int8_t *a, *w;
    const float *a_scale, *w_scale, *bias;
    const int* offsets;
    void* y;
    int* status;
    int dependent;  // launched behind the quantiser, which lets it start early
};
cudaError_t launch_matmul_i8(int dt, const MatmulParams& p, cudaStream_t s);

// At most 8 rows (kernel_rows_i8.cu): whether the kernel takes them, and whether it quantises them itself.
bool few_rows(const MatmulParams& p);
bool few_rows_quantise(const MatmulParams& p);
cudaError_t launch_matmul_i8_few(int dt, const MatmulParams& p, cudaStream_t s);
cudaError_t launch_linear_i8_few(int dt, const MatmulParams& p, const QuantParams& x, int x_dt, cudaStream_t s);

}  // namespace experts
}  // namespace hccl
