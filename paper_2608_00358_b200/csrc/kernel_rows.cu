// Exchange of rows between token order and expert order: dispatch (copy), combine (weighted sum) and the gradient of
// combine. All three walk tokens, so that a token's row is read (or written) once and each of its top_k rows in
// expert order is touched once, without atomics: a row belongs to one choice.
#include "experts.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int ROWS_THREADS = 256;

// The row of choice k of token t, or -1.
__device__ __forceinline__ long long slot_of(const RowsParams& p, long long t, int k) {
    const long long s = p.slots[t * p.K + k];
    return (s >= 0 && s < p.n_rows) ? s : -1;
}

// Rows from offsets[E] to n_rows belong to no choice: zero.
template <typename T, int N> __device__ __forceinline__ void clear_tail(const RowsParams& p) {
    const long long used = max(0ll, (long long)p.offsets[p.E]);
    for (long long r = used + blockIdx.x; r < p.n_rows; r += gridDim.x) {
        Pack<T, N> z;
#pragma unroll
        for (int i = 0; i < N; i++) z.v[i] = from_f32<T>(0.f);
        auto* out = (typename Piece<N * sizeof(T)>::type*)((T*)p.rows_out + r * p.ldro);
        for (long long c = threadIdx.x; c < p.H / N; c += blockDim.x) out[c] = z.raw;
    }
}

template <typename T, int N> __global__ void __launch_bounds__(ROWS_THREADS) hccl_rows_dispatch(const __grid_constant__ RowsParams p) {
    using P = typename Piece<N * sizeof(T)>::type;
    const long long cols = p.H / N;
    for (long long t = blockIdx.x; t < p.tokens; t += gridDim.x) {
        const P* x = (const P*)((const T*)p.x + t * p.ldx);
        for (long long c = threadIdx.x; c < cols; c += blockDim.x) {
            const P v = x[c];
            for (int k = 0; k < p.K; k++) {
                const long long s = slot_of(p, t, k);
                if (s >= 0) ((P*)((T*)p.rows_out + s * p.ldro))[c] = v;
            }
        }
    }
    clear_tail<T, N>(p);
}

template <typename T, int N> __global__ void __launch_bounds__(ROWS_THREADS) hccl_rows_combine(const __grid_constant__ RowsParams p) {
    using P = typename Piece<N * sizeof(T)>::type;
    const long long cols = p.H / N;
    for (long long t = blockIdx.x; t < p.tokens; t += gridDim.x) {
        P* y = (P*)((T*)p.y + t * p.ldy);
        for (long long c = threadIdx.x; c < cols; c += blockDim.x) {
            float acc[N];
#pragma unroll
            for (int i = 0; i < N; i++) acc[i] = 0.f;
            for (int k = 0; k < p.K; k++) {
                const long long s = slot_of(p, t, k);
                if (s < 0) continue;
                const float w = p.weights ? p.weights[t * p.K + k] : 1.f;
                Pack<T, N> v;
                v.raw = ((const P*)((const T*)p.rows + s * p.ldr))[c];
#pragma unroll
                for (int i = 0; i < N; i++) acc[i] = fmaf(w, to_f32<T>(v.v[i]), acc[i]);
            }
            Pack<T, N> o;
#pragma unroll
            for (int i = 0; i < N; i++) o.v[i] = from_f32<T>(acc[i]);
            y[c] = o.raw;
        }
    }
}

template <typename T, int N> __global__ void __launch_bounds__(ROWS_THREADS) hccl_rows_combine_grad(const __grid_constant__ RowsParams p) {
    using P = typename Piece<N * sizeof(T)>::type;
    __shared__ float part[ROWS_THREADS / 32];
    const long long cols = p.H / N;
    const int warps = blockDim.x / 32;
    for (long long t = blockIdx.x; t < p.tokens; t += gridDim.x) {
        const P* dy = (const P*)((const T*)p.x + t * p.ldx);
        for (int k = 0; k < p.K; k++) {
            const long long s = slot_of(p, t, k);
            float dot = 0.f;
            if (s >= 0) {
                const float w = p.weights ? p.weights[t * p.K + k] : 1.f;
                const P* r = (const P*)((const T*)p.rows + s * p.ldr);
                P* out = (P*)((T*)p.rows_out + s * p.ldro);
                for (long long c = threadIdx.x; c < cols; c += blockDim.x) {
                    Pack<T, N> g, v, o;
                    g.raw = dy[c];
                    v.raw = r[c];
#pragma unroll
                    for (int i = 0; i < N; i++) {
                        dot = fmaf(to_f32<T>(g.v[i]), to_f32<T>(v.v[i]), dot);
                        o.v[i] = from_f32<T>(w * to_f32<T>(g.v[i]));
                    }
                    out[c] = o.raw;
                }
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
            if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = dot;
            __syncthreads();
            if (threadIdx.x == 0) {
                float sum = 0.f;
                for (int i = 0; i < warps; i++) sum += part[i];
                p.dweights[t * p.K + k] = sum;
            }
            __syncthreads();
        }
    }
    clear_tail<T, N>(p);
}

// Bytes that every row start and the row length allow to be moved at once.
int piece_bytes(int es, long long H, const void* const* ptr, const long long* ld, int n) {
    unsigned long long bits = (unsigned long long)H * es;
    for (int i = 0; i < n; i++) bits |= (unsigned long long)(uintptr_t)ptr[i] | (unsigned long long)(ld[i] * es);
    return bits % 16 == 0 ? 16 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 2;
}

enum { DISPATCH, COMBINE, COMBINE_GRAD };

template <typename T, int N> cudaError_t rows_launch(int what, const RowsParams& p, cudaStream_t s) {
    const long long cols = p.H / N;
    int threads = 32;
    while (threads < ROWS_THREADS && threads < cols) threads *= 2;
    const long long work = what == COMBINE ? p.tokens : (p.tokens > p.n_rows ? p.tokens : p.n_rows);
    const long long most = (long long)SMS * (2048 / threads);
    const int blocks = (int)(work < most ? work : most);
    if (blocks == 0) return cudaSuccess;
    if (what == DISPATCH) hccl_rows_dispatch<T, N><<<blocks, threads, 0, s>>>(p);
    else if (what == COMBINE) hccl_rows_combine<T, N><<<blocks, threads, 0, s>>>(p);
    else hccl_rows_combine_grad<T, N><<<blocks, threads, 0, s>>>(p);
    return cudaGetLastError();
}

template <typename T> cudaError_t rows_piece(int what, int bytes, const RowsParams& p, cudaStream_t s) {
    if (bytes == 16) return rows_launch<T, 16 / sizeof(T)>(what, p, s);
    if (bytes == 8) return rows_launch<T, 8 / sizeof(T)>(what, p, s);
    if (bytes == 4 || sizeof(T) == 4) return rows_launch<T, 4 / sizeof(T)>(what, p, s);
    return rows_launch<T, 1>(what, p, s);
}

cudaError_t rows_dtype(int what, int dt, int bytes, const RowsParams& p, cudaStream_t s) {
    if (dt == HCCL_FP32) return rows_piece<float>(what, bytes, p, s);
    if (dt == HCCL_BF16) return rows_piece<__nv_bfloat16>(what, bytes, p, s);
    return rows_piece<__half>(what, bytes, p, s);
}

}  // namespace

cudaError_t launch_dispatch(int dt, const RowsParams& p, cudaStream_t s) {
    const void* ptr[] = {p.x, p.rows_out};
    const long long ld[] = {p.ldx, p.ldro};
    return rows_dtype(DISPATCH, dt, piece_bytes(dt == HCCL_FP32 ? 4 : 2, p.H, ptr, ld, 2), p, s);
}
cudaError_t launch_combine(int dt, const RowsParams& p, cudaStream_t s) {
    const void* ptr[] = {p.rows, p.y};
    const long long ld[] = {p.ldr, p.ldy};
    return rows_dtype(COMBINE, dt, piece_bytes(dt == HCCL_FP32 ? 4 : 2, p.H, ptr, ld, 2), p, s);
}
cudaError_t launch_combine_grad(int dt, const RowsParams& p, cudaStream_t s) {
    const void* ptr[] = {p.x, p.rows, p.rows_out};
    const long long ld[] = {p.ldx, p.ldr, p.ldro};
    return rows_dtype(COMBINE_GRAD, dt, piece_bytes(dt == HCCL_FP32 ? 4 : 2, p.H, ptr, ld, 3), p, s);
}

}  // namespace experts
}  // namespace hccl
