// Exchange of rows between token order and expert order: dispatch (copy), combine (weighted sum) and the gradient of
// combine. They walk tokens (the gradient: choices, token by token), so that each row in expert order is touched once and a token's row
// comes from memory once, without atomics: a row belongs to one choice. Memory is the bound of all three; what
// costs is latency, so every thread asks for the pieces of several choices before it uses the first.
//
// Measured (B200, copy peak 6.5 TB/s): dispatch 8192 x 4096 bf16 to 8 places 102 us = 5.9 TB/s; combine back 100 us = 6.0 TB/s, its gradient 173 us = 6.6 TB/s;
// gradient 4099 x 2056 of 6 (rows of 4112 bytes) 40 us = 5.5 TB/s; combine of 32 tokens 3 us, a launch and two latencies.
#include <algorithm>

#include "experts.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int ROWS_THREADS = 256, COMBINE_THREADS = 128 /* 8192 x 4096 of 8: 100 us, 109 with 256: the last round of the blocks is shorter */, BATCH = 8 /* choices at a time */;

// A token belongs to a team of `team` warps (1, 2, 4 or 8) of a block.
struct Team {
    int lanes, rank;          // threads of the team, this thread's place in it
    long long first, step;    // tokens first, first + step, ...
    __device__ __forceinline__ explicit Team(int warps) : lanes(32 * warps), rank((int)threadIdx.x % lanes) {
        const int per = (int)blockDim.x / lanes;
        first = (long long)blockIdx.x * per + (int)threadIdx.x / lanes;
        step = (long long)gridDim.x * per;
    }
};

// A warp's look at a token's choices: lane k holds the row of choice k (-1: none) and its weight.
struct Choices {
    int slot;
    float w;
    __device__ __forceinline__ Choices(const RowsParams& p, long long t) : slot(-1), w(0.f) {
        const int k = threadIdx.x % 32;
        if (k < p.K) {
            const int s = p.slots[t * p.K + k];
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

template <typename T, int N> __global__ void __launch_bounds__(ROWS_THREADS) hccl_rows_dispatch(const __grid_constant__ RowsParams p, int team) {
    using P = typename Piece<N * sizeof(T)>::type;
    const int cols = (int)(p.H / N);
    const Team m(team);
    for (long long t = m.first; t < p.tokens; t += m.step) {
        const Choices mine(p, t);
        const P* x = (const P*)((const T*)p.x + t * p.ldx);
        for (int k0 = 0; k0 < p.K; k0 += BATCH) {
            P* to[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; j++) {
                const int s = k0 + j < p.K ? __shfl_sync(FULL, mine.slot, k0 + j) : -1;
                to[j] = s >= 0 ? (P*)((T*)p.rows_out + s * p.ldro) : nullptr;
            }
            for (int c = m.rank; c < cols; c += m.lanes) {
                const P v = x[c];
#pragma unroll
                for (int j = 0; j < BATCH; j++)
                    if (to[j]) to[j][c] = v;
            }
        }
    }
    clear_tail<T, N>(p, blockIdx.x, gridDim.x);
}

// Dispatch of rows that start and end on 16-byte boundaries (8192 x 4096 to 8: 102 us, 112 with the stores above): a warp brings a piece of a row to shared memory and lets the bulk copy unit write it
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
            asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"((char*)p.rows_out + (long long)mine.slot * row_step + i % pieces * PIECE),
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

// KB: choices at a time, the least of 2, 4 and 8 that is not below K, or 8. blockIdx.y: which span of the columns.
template <typename T, int N, int KB> __global__ void __launch_bounds__(COMBINE_THREADS) hccl_rows_combine(const __grid_constant__ RowsParams p, int team, int span) {
    using P = typename Piece<N * sizeof(T)>::type;
    const int cols = (int)(p.H / N), c0 = (int)blockIdx.y * span, c1 = min(c0 + span, cols);
    const Team m(team);
    for (long long t = m.first; t < p.tokens; t += m.step) {
        const Choices mine(p, t);
        P* y = (P*)((T*)p.y + t * p.ldy);
        const P* from[KB];
        float w[KB];
        const auto take = [&](int k0) {
#pragma unroll
            for (int j = 0; j < KB; j++) {
                const int s = k0 + j < p.K ? __shfl_sync(FULL, mine.slot, k0 + j) : -1;
                w[j] = __shfl_sync(FULL, mine.w, (k0 + j) & 31);
                from[j] = s >= 0 ? (const P*)((const T*)p.rows + s * p.ldr) : nullptr;
            }
        };
        take(0);
        // (the team's first column decides how often a warp goes round, so that all lanes take part in the shuffles)
        for (int base = c0; base < c1; base += m.lanes) {
            const int c = base + m.rank;
            float acc[N];
#pragma unroll
            for (int i = 0; i < N; i++) acc[i] = 0.f;
            for (int k0 = 0; k0 < p.K; k0 += KB) {
                if (p.K > KB) take(k0);
                if (c < c1) {
                    Pack<T, N> v[KB];
#pragma unroll
                    for (int j = 0; j < KB; j++)
                        if (from[j]) v[j].raw = from[j][c];
#pragma unroll
                    for (int j = 0; j < KB; j++)
                        if (from[j]) {
                            float f[N];
                            v[j].get(f);
#pragma unroll
                            for (int i = 0; i < N; i++) acc[i] = fmaf(w[j], f[i], acc[i]);
                        }
                }
            }
            if (c < c1) {
                Pack<T, N> o;
                o.set(acc);
                y[c] = o.raw;
            }
        }
    }
}

// A warp for each choice: it reads the token's gradient (the block's other warps read the same, from the L1) and the choice's row, once, and writes the row's
// gradient. Four pieces of both are asked for at a time. (Teams of warps that held a token's gradient for all its choices took 50 us for 4099 x 2056 of 6 and 188 for
// 8192 x 4096 of 8.)
template <typename T, int N> __global__ void __launch_bounds__(ROWS_THREADS) hccl_rows_combine_grad(const __grid_constant__ RowsParams p) {
    using P = typename Piece<N * sizeof(T)>::type;
    constexpr int U = 4;
    const int cols = (int)(p.H / N), lane = threadIdx.x % 32;
    const long long pairs = p.tokens * p.K, step = (long long)gridDim.x * (ROWS_THREADS / 32);
    for (long long i = (long long)blockIdx.x * (ROWS_THREADS / 32) + threadIdx.x / 32; i < pairs; i += step) {
        const int s = p.slots[i];
        float dot = 0.f;
        if (s >= 0 && s < p.n_rows) {
            const float w = p.weights[i];
            const P *dy = (const P*)((const T*)p.x + i / p.K * p.ldx), *row = (const P*)((const T*)p.rows + s * p.ldr);
            P* out = (P*)((T*)p.rows_out + s * p.ldro);
            for (int c0 = lane; c0 < cols; c0 += 32 * U) {
                Pack<T, N> g[U], v[U];
#pragma unroll
                for (int u = 0; u < U; u++)
                    if (c0 + 32 * u < cols) {
                        g[u].raw = dy[c0 + 32 * u];
                        v[u].raw = row[c0 + 32 * u];
                    }
#pragma unroll
                for (int u = 0; u < U; u++)
                    if (c0 + 32 * u < cols) {
                        float d[N], f[N];
                        g[u].get(d);
                        v[u].get(f);
#pragma unroll
                        for (int n = 0; n < N; n++) {
                            dot = fmaf(d[n], f[n], dot);
                            d[n] *= w;
                        }
                        Pack<T, N> o;
                        o.set(d);
                        out[c0 + 32 * u] = o.raw;
                    }
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) dot += __shfl_xor_sync(FULL, dot, o);
        if (lane == 0) p.dweights[i] = dot;
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

// Warps for each token: one (combine 8192 x 4096 of 8, 4099 x 2056 of 6, 2000 x 1024 of 4, bf16, in blocks of 256: 109, 30 and 5 us; 112, 37 and 5 with four); with few tokens as many as make 16 warps
// for each SM.
int team_of(long long tokens, long long cols, int most) {
    int w = 1;
    while (w < most && tokens * w < SMS * 16 && cols > 32 * w) w *= 2;
    return w;
}

template <typename T, int N> cudaError_t rows_launch(int what, const RowsParams& p, cudaStream_t s) {
    const long long cols = p.H / N;
    if (cols > 1 << 30) return cudaErrorInvalidValue;
    const int warps_of = (what == COMBINE ? COMBINE_THREADS : ROWS_THREADS) / 32, team = team_of(p.tokens, cols, warps_of), per = warps_of / team;
    const long long whole = (p.tokens + per - 1) / per;  // a block for each `per` tokens: the hardware hands out the next one where one has ended
    const unsigned blocks = (unsigned)std::min<long long>(std::max<long long>(whole, what == COMBINE ? 1 : SMS), 1 << 30);
    if (what == COMBINE) {
        if (p.tokens == 0 || p.H == 0) return cudaSuccess;
        // few tokens: a row's columns go to several blocks, one round for each
        const long long rounds = (cols + 32 * team - 1) / (32 * team);
        const unsigned across = (unsigned)std::min<long long>(rounds, std::max<long long>(1, SMS * 4 / std::max<long long>(whole, 1)));
        const int span = (int)((rounds + across - 1) / across) * 32 * team;
        const dim3 grid(blocks, across);
        if (p.K <= 2) hccl_rows_combine<T, N, 2><<<grid, COMBINE_THREADS, 0, s>>>(p, team, span);
        else if (p.K <= 4) hccl_rows_combine<T, N, 4><<<grid, COMBINE_THREADS, 0, s>>>(p, team, span);
        else hccl_rows_combine<T, N, 8><<<grid, COMBINE_THREADS, 0, s>>>(p, team, span);
        return cudaGetLastError();
    }
    if (p.tokens == 0 && p.n_rows == 0) return cudaSuccess;
    if (what == DISPATCH) {
        hccl_rows_dispatch<T, N><<<blocks, ROWS_THREADS, 0, s>>>(p, team);
    } else {
        const long long warps = ROWS_THREADS / 32, all = (p.tokens * p.K + warps - 1) / warps;
        hccl_rows_combine_grad<T, N><<<(unsigned)std::min<long long>(std::max<long long>(all, SMS), 1 << 30), ROWS_THREADS, 0, s>>>(p);
    }
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
    // (a copy through shared memory has its own latency: below some 4 MB of rows, plain stores; 50 x 2048 to 8 places 4.8 us by bulk copies)
    if (piece == 16 && p.tokens * p.K * p.H * es >= 4 << 20) {
        const long long bytes = p.H * es, items = p.tokens * ((bytes + 4095) / 4096);
        // Warps: 32 KB of buffers on each SM, as many bytes of rows as it takes (8192 x 4096 to 8 places: 102 us with one block on each SM, 108-111
        // with two to six; 131 with half the bytes), and no more warps than bring every one to the same number of pieces.
        const long long per_sm = std::min<long long>(8, std::max<long long>(1, 4096 / bytes)), most = std::min<long long>(items, SMS * per_sm * BULK_WARPS);
        const long long rounds = (items + most - 1) / most, warps = (items + rounds - 1) / rounds;
        const int blocks = (int)((warps + BULK_WARPS - 1) / BULK_WARPS);
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
