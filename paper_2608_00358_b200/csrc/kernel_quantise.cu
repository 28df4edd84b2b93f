// Rows to 8-bit integers with a scale for each row: scale = max|x| / 127, q = round(x * (1 / max|x| * 127)). With a routing the row
// is written to every place that the token was sent to, so it is read and quantised once. Memory is the bound: a block
// holds its row in registers between the maximum and the rounding, so every element is read once.
//
// Measured (B200, copy peak 6.5 TB/s): 8192 x 8192 bf16 40 us = 5.0 TB/s; 8192 x 4096 bf16 to 8 places 57 us = 5.9 TB/s; one row of 4096 2 us.
#include <algorithm>
#include <atomic>

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

// Many long rows (aligned, at most 32 KB): teams of 32 to 256 threads walk rows, each with RING rows on their way into shared memory. A thread fetches
// and reads the same 16-byte pieces, so that nothing but the row's maximum needs a barrier; between rows nothing stops the stream of loads, which is what the
// kernel above loses (8192 x 8192 bf16: 50 us).
constexpr int RING = 3, HELD = 8 /* pieces of a thread */;
template <typename T> __global__ void __launch_bounds__(256) hccl_quantise_ring(const __grid_constant__ QuantParams p, int team) {
    constexpr int N = Sixteen<T>::N;
    extern __shared__ __align__(16) uint4 ring[];  // [threads][RING][HELD], a thread's own pieces side by side in turns of the block
    __shared__ unsigned part[2][8];
    asm volatile("griddepcontrol.launch_dependents;");
    const int threads = blockDim.x, rank = (int)threadIdx.x % team, K = (int)p.K;
    const long long teams = threads / team, first = (long long)blockIdx.x * teams + threadIdx.x / team, step = (long long)gridDim.x * teams;
    const auto place = [&](int turn, int u) { return ring + (turn * HELD + u) * threads + threadIdx.x; };
    const auto fetch = [&](long long m, int turn) {
        if (m < p.M) {
            const char* x = (const char*)((const T*)p.x + m * p.ldx);
#pragma unroll
            for (int u = 0; u < HELD; u++) {
                const int i = (u * team + rank) * N, bytes = min(16, (K - i) * (int)sizeof(T));
                if (bytes > 0)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((unsigned)__cvta_generic_to_shared(place(turn, u))), "l"(x + (long long)i * sizeof(T)), "r"(bytes) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int r = 0; r < RING; r++) fetch(first + r * step, r);
    int turn = 0, half = 0;
    for (long long m = first; m < p.M; m += step, half ^= 1) {
        asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");
        Sixteen<T> v[HELD];
        unsigned bits = 0;
#pragma unroll
        for (int u = 0; u < HELD; u++) {
            uint4 w = make_uint4(0, 0, 0, 0);
            if ((u * team + rank) * N < K) w = *place(turn, u);
            v[u].w[0] = w.x, v[u].w[1] = w.y, v[u].w[2] = w.z, v[u].w[3] = w.w;
        }
#pragma unroll
        for (int u = 0; u < HELD; u++) bits = max(bits, v[u].magnitude());
        bits = __reduce_max_sync(0xffffffffu, bits);
        if (team > 32) {  // two places in turn: a warp may be a row ahead of another's reading, not two
            const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, lead = warp - rank / 32;
            if (lane == 0) part[half][warp] = bits;
            asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / team), "r"(team) : "memory");
            bits = __reduce_max_sync(0xffffffffu, lane < team / 32 ? part[half][lead + lane] : 0u);
        }
        fetch(m + RING * step, turn);  // into the places just read
        turn = turn + 1 == RING ? 0 : turn + 1;
        float factor, scale;
        row_scale(bits, &factor, &scale);
        unsigned o[HELD][N / 4];
#pragma unroll
        for (int u = 0; u < HELD; u++)
#pragma unroll
            for (int j = 0; j < N / 4; j++) o[u][j] = quantised(v[u], 4 * j, factor);
        int8_t* q = p.q + m * p.ldq;
#pragma unroll
        for (int u = 0; u < HELD; u++) {
            const int i = (u * team + rank) * N;
            if (p.vec_q && i + N <= K) {
                if constexpr (N == 8) *(uint2*)(q + i) = make_uint2(o[u][0], o[u][N / 4 - 1]);
                else *(unsigned*)(q + i) = o[u][0];
            } else {
#pragma unroll
                for (int j = 0; j < N; j++)
                    if (i + j < K) q[i + j] = (int8_t)(o[u][j / 4] >> (8 * (j & 3)));
            }
        }
        if (rank == 0) p.scale[m] = scale;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <typename T> cudaError_t ring_launch(const QuantParams& p, cudaStream_t s) {
    const long long bytes = p.K * (long long)sizeof(T);
    int team = 32;
    while (team * HELD * 16 < bytes) team *= 2;
    const int threads = team == 256 ? 256 : 128, smem = threads * RING * HELD * 16;
    static std::atomic<bool> ready[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev]) {
        e = cudaFuncSetAttribute(hccl_quantise_ring<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 256 * RING * HELD * 16);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev] = true;
    }
    // as many blocks as fit at once (48 KB of an SM's shared memory for 128 threads), and no more than bring every team to the same number of rows
    const long long rows = threads / team, work = (p.M + rows - 1) / rows, most = std::min<long long>(work, SMS * (threads == 256 ? 2 : 4)), rounds = (work + most - 1) / most;
    hccl_quantise_ring<T><<<(int)((work + rounds - 1) / rounds), threads, smem, s>>>(p, team);
    return cudaGetLastError();
}

template <typename T> cudaError_t quant_launch(const QuantParams& in, cudaStream_t s) {
    QuantParams p = in;
    if (p.M == 0) return cudaSuccess;
    constexpr int N = Sixteen<T>::N;
    p.vec = (uintptr_t)p.x % 16 == 0 && (p.ldx * sizeof(T)) % 16 == 0;
    p.vec_q = (uintptr_t)p.q % 8 == 0 && p.ldq % 8 == 0;
    // The ring where long rows come in large numbers: 8192 x 8192 bf16 40 us against 50, 8192 x 4096 bf16 23 against 25 and fp32 36 against 39; with rows of 2 KB
    // (65536 x 1024) 82 against 70, with few rows (64 x 4096) 3.4 against 2.7, with eight copies of each 59 against 57.
    const long long bytes = p.K * (long long)sizeof(T);
    if (p.vec && !p.slots && bytes >= 8192 && bytes <= 256 * HELD * 16 && p.M * bytes >= 32 << 20) return ring_launch<T>(p, s);
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
