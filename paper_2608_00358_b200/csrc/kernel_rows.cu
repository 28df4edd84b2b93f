// Exchange of rows between token order and expert order: dispatch (copy), combine (weighted sum) and the gradient of
// combine. All three walk tokens, so that a token's row is read (or written) once and each of its top_k rows in
// expert order is touched once, without atomics: a row belongs to one choice. Memory is the bound of all three; what
// costs is latency, so every thread asks for the pieces of eight choices before it uses the first.
#include <algorithm>

#include "experts.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int ROWS_THREADS = 256, BATCH = 8 /* choices at a time */;

// A warp's look at a token's choices: lane k holds the row of choice k (-1: none) and its weight.
struct Choices {
    long long slot;
    float w;
    __device__ __forceinline__ Choices(const RowsParams& p, long long t) : slot(-1), w(0.f) {
        const int k = threadIdx.x % 32;
        if (k < p.K) {
            const long long s = p.slots[t * p.K + k];
            if (s >= 0 && s < p.n_rows) {
                slot = s;
                w = p.weights ? p.weights[t * p.K + k] : 1.f;
            }
        }
    }
};

// Rows from offsets[E] to n_rows belong to no choice: zero.
template <typename T, int N> __device__ __forceinline__ void clear_tail(const RowsParams& p, long long block, long long blocks) {
    const long long used = max(0ll, (long long)p.offsets[p.E]);
    for (long long r = used + block; r < p.n_rows; r += blocks) {
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
        const Choices mine(p, t);
        const P* x = (const P*)((const T*)p.x + t * p.ldx);
        for (int k0 = 0; k0 < p.K; k0 += BATCH) {
            P* to[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; j++) {
                const long long s = k0 + j < p.K ? __shfl_sync(FULL, mine.slot, k0 + j) : -1;
                to[j] = s >= 0 ? (P*)((T*)p.rows_out + s * p.ldro) : nullptr;
            }
            for (long long c = threadIdx.x; c < cols; c += blockDim.x) {
                const P v = x[c];
#pragma unroll
                for (int j = 0; j < BATCH; j++)
                    if (to[j]) to[j][c] = v;
            }
        }
    }
    clear_tail<T, N>(p, blockIdx.x, gridDim.x);
}

// Dispatch of rows that start and end on 16-byte boundaries: a warp brings a piece of a row to shared memory and lets the bulk copy unit write it
// to each of its places, one instruction for each, from lane k for choice k. Two buffers: the next piece is on its way in while the
// last one's copies leave.
constexpr int BULK_WARPS = 4;
__device__ __forceinline__ void copy_in(char* to, const char* from, int bytes) {
    for (int i = threadIdx.x % 32 * 16; i < bytes; i += 32 * 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(to + i)), "l"(from + i) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int PIECE> __global__ void __launch_bounds__(32 * BULK_WARPS) hccl_rows_dispatch_bulk(const __grid_constant__ RowsParams p, long long bytes, long long x_step, long long row_step) {
    __shared__ __align__(128) char buf[BULK_WARPS][2][PIECE];
    const int warp = threadIdx.x / 32;
    const long long pieces = (bytes + PIECE - 1) / PIECE, items = p.tokens * pieces, step = (long long)gridDim.x * BULK_WARPS;
    const auto size_of = [&](long long i) { return (int)min((long long)PIECE, bytes - i % pieces * PIECE); };
    const auto bring = [&](long long i, int b) { copy_in(buf[warp][b], (const char*)p.x + i / pieces * x_step + i % pieces * PIECE, size_of(i)); };
    long long i = (long long)blockIdx.x * BULK_WARPS + warp;
    int b = 0;
    if (i < items) bring(i, 0);
    for (; i < items; i += step, b ^= 1) {
        const Choices mine(p, i / pieces);
        // the other buffer's copies have been read out of it
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
        if (i + step < items) {
            bring(i + step, b ^ 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // what arrived, before the copy unit reads it
        __syncwarp();
        if (mine.slot >= 0)
            asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"((char*)p.rows_out + mine.slot * row_step + i % pieces * PIECE),
                         "r"((unsigned)__cvta_generic_to_shared(buf[warp][b])), "r"(size_of(i))
                         : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    // rows without a choice
    const long long used = max(0ll, (long long)p.offsets[p.E]);
    for (long long r = used + blockIdx.x; r < p.n_rows; r += gridDim.x)
        for (long long c = threadIdx.x * 16ll; c < bytes; c += 32 * BULK_WARPS * 16) *(uint4*)((char*)p.rows_out + r * row_step + c) = make_uint4(0, 0, 0, 0);
}

// Block (x, y): columns [x * span, ...) of tokens y, y + gridDim.y, ...
template <typename T, int N> __global__ void __launch_bounds__(ROWS_THREADS) hccl_rows_combine(const __grid_constant__ RowsParams p, int span) {
    using P = typename Piece<N * sizeof(T)>::type;
    const long long cols = p.H / N, c0 = (long long)blockIdx.x * span, c1 = min(c0 + span, cols);
    for (long long t = blockIdx.y; t < p.tokens; t += gridDim.y) {
        const Choices mine(p, t);
        P* y = (P*)((T*)p.y + t * p.ldy);
        // (a thread's first column decides how often the warp goes round, so that all lanes take part in the shuffles)
        for (long long base = c0; base < c1; base += blockDim.x) {
            const long long c = base + threadIdx.x;
            float acc[N];
#pragma unroll
            for (int i = 0; i < N; i++) acc[i] = 0.f;
            for (int k0 = 0; k0 < p.K; k0 += BATCH) {
                Pack<T, N> v[BATCH];
                float w[BATCH];
                bool some[BATCH];
#pragma unroll
                for (int j = 0; j < BATCH; j++) {
                    const long long s = k0 + j < p.K ? __shfl_sync(FULL, mine.slot, k0 + j) : -1;
                    w[j] = __shfl_sync(FULL, mine.w, (k0 + j) & 31);
                    some[j] = s >= 0 && c < c1;
                    if (some[j]) v[j].raw = ((const P*)((const T*)p.rows + s * p.ldr))[c];
                }
#pragma unroll
                for (int j = 0; j < BATCH; j++)
                    if (some[j]) {
#pragma unroll
                        for (int i = 0; i < N; i++) acc[i] = fmaf(w[j], to_f32<T>(v[j].v[i]), acc[i]);
                    }
            }
            if (c < c1) {
                Pack<T, N> o;
#pragma unroll
                for (int i = 0; i < N; i++) o.v[i] = from_f32<T>(acc[i]);
                y[c] = o.raw;
            }
        }
    }
}

template <typename T, int N> __global__ void __launch_bounds__(ROWS_THREADS) hccl_rows_combine_grad(const __grid_constant__ RowsParams p) {
    using P = typename Piece<N * sizeof(T)>::type;
    __shared__ float part[2][ROWS_THREADS / 32][32];
    const long long cols = p.H / N;
    const int warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    int turn = 0;
    for (long long t = blockIdx.x; t < p.tokens; t += gridDim.x, turn ^= 1) {
        const Choices mine(p, t);
        const P* dy = (const P*)((const T*)p.x + t * p.ldx);
        float sums = 0.f;  // lane k: this warp's part of choice k
        for (int k0 = 0; k0 < p.K; k0 += BATCH) {
            const P* from[BATCH];
            P* to[BATCH];
            float w[BATCH], dot[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; j++) {
                const long long s = k0 + j < p.K ? __shfl_sync(FULL, mine.slot, k0 + j) : -1;
                w[j] = __shfl_sync(FULL, mine.w, (k0 + j) & 31);
                from[j] = s >= 0 ? (const P*)((const T*)p.rows + s * p.ldr) : nullptr;
                to[j] = s >= 0 ? (P*)((T*)p.rows_out + s * p.ldro) : nullptr;
                dot[j] = 0.f;
            }
            for (long long c = threadIdx.x; c < cols; c += blockDim.x) {
                Pack<T, N> g, v[BATCH];
                g.raw = dy[c];
#pragma unroll
                for (int j = 0; j < BATCH; j++)
                    if (from[j]) v[j].raw = from[j][c];
#pragma unroll
                for (int j = 0; j < BATCH; j++)
                    if (from[j]) {
                        Pack<T, N> o;
#pragma unroll
                        for (int i = 0; i < N; i++) {
                            dot[j] = fmaf(to_f32<T>(g.v[i]), to_f32<T>(v[j].v[i]), dot[j]);
                            o.v[i] = from_f32<T>(w[j] * to_f32<T>(g.v[i]));
                        }
                        to[j][c] = o.raw;
                    }
            }
#pragma unroll
            for (int j = 0; j < BATCH; j++) {
#pragma unroll
                for (int o = 16; o; o >>= 1) dot[j] += __shfl_xor_sync(FULL, dot[j], o);
                if (lane == k0 + j) sums = dot[j];
            }
        }
        if (warps > 1) {  // two places in turn: a warp may be a token ahead of the one that adds up, not two
            part[turn][warp][lane] = sums;
            __syncthreads();
            if (warp == 0) {
                sums = 0.f;
                for (int i = 0; i < warps; i++) sums += part[turn][i][lane];
            }
        }
        if (warp == 0 && lane < p.K) p.dweights[t * p.K + lane] = sums;
    }
    clear_tail<T, N>(p, blockIdx.x, gridDim.x);
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
    if (what == COMBINE) {
        if (p.tokens == 0) return cudaSuccess;
        while (threads < ROWS_THREADS && threads < cols) threads *= 2;
        // a block takes two rounds of columns where tokens fill the SMs, one where they do not
        const int span = threads * (p.tokens >= SMS * 4 ? 2 : 1);
        const unsigned across = (unsigned)std::max<long long>(1, (cols + span - 1) / span);
        hccl_rows_combine<T, N><<<dim3(across, (unsigned)std::min<long long>(p.tokens, 65535)), threads, 0, s>>>(p, span);
        return cudaGetLastError();
    }
    const long long work = std::max(p.tokens, p.n_rows);
    if (work == 0) return cudaSuccess;
    const int a_thread = what == COMBINE_GRAD ? 4 : 2;  // pieces of a thread, about
    while (threads < ROWS_THREADS && threads * a_thread < cols) threads *= 2;
    const int blocks = (int)std::min<long long>(work, (long long)SMS * (2048 / threads));
    if (what == DISPATCH) hccl_rows_dispatch<T, N><<<blocks, threads, 0, s>>>(p);
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
    const int es = dt == HCCL_FP32 ? 4 : 2;
    const void* ptr[] = {p.x, p.rows_out};
    const long long ld[] = {p.ldx, p.ldro};
    const int piece = piece_bytes(es, p.H, ptr, ld, 2);
    if (piece == 16 && p.tokens && p.H) {
        const long long bytes = p.H * es, items = p.tokens * ((bytes + 4095) / 4096);
        const int blocks = (int)std::min<long long>((items + BULK_WARPS - 1) / BULK_WARPS, SMS * 6);
        hccl_rows_dispatch_bulk<4096><<<blocks, 32 * BULK_WARPS, 0, s>>>(p, bytes, p.ldx * es, p.ldro * es);
        return cudaGetLastError();
    }
    return rows_dtype(DISPATCH, dt, piece, p, s);
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
