// The gated activation between an expert's two products, with dropout: y[r, i] = act(x[r, i]) x[r, I + i] m[r, i], and its gradient. m is 0 or 1 / (1 - p), from a
// counter-based generator, and is formed anew wherever it is needed: nothing of it is stored. Without a gate y = act(x) m.
//
// The generator is Philox-4x32-10 (Salmon, Moraes, Dror, Shaw 2011): four 32-bit words from a 128-bit counter and a 64-bit key in ten rounds of two 32 x 32 bit
// products. Element i of the result (row * I + column) takes word i % 4 of the counter (i / 4, call); it is kept if the word is at least p 2^32.
#include <algorithm>

#include "activate.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int THREADS = 256;

struct Words {
    unsigned w[4];
};
__device__ __forceinline__ Words philox(unsigned long long counter, unsigned long long call, unsigned long long key) {
    unsigned c0 = (unsigned)counter, c1 = (unsigned)(counter >> 32), c2 = (unsigned)call, c3 = (unsigned)(call >> 32), k0 = (unsigned)key, k1 = (unsigned)(key >> 32);
#pragma unroll
    for (int r = 0; r < 10; r++) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(b >> 32) ^ c1 ^ k0;
        c1 = (unsigned)b;
        c2 = (unsigned)(a >> 32) ^ c3 ^ k1;
        c3 = (unsigned)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// The factors that dropout multiplies N neighbouring elements with, N a multiple of 4, the first being element `at` of the result. A counter's words begin within the
// elements where I is odd.
template <int N> __device__ __forceinline__ void factors(const ActivateParams& p, unsigned long long key, unsigned long long call, unsigned long long at, float (&f)[N]) {
    const unsigned o = (unsigned)at & 3u;
    if (o == 0) {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const Words w = philox(at / 4 + j / 4, call, key);
#pragma unroll
            for (int i = 0; i < 4; i++) f[j + i] = w.w[i] >= p.threshold ? p.keep : 0.f;
        }
    } else {
        Words w = philox(at / 4, call, key);
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const Words next = philox(at / 4 + j / 4 + 1, call, key);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const unsigned v = i + o == 1 ? w.w[1] : i + o == 2 ? w.w[2] : i + o == 3 ? w.w[3] : i + o == 4 ? next.w[0] : i + o == 5 ? next.w[1] : next.w[2];
                f[j + i] = v >= p.threshold ? p.keep : 0.f;
            }
            w = next;
        }
    }
}

// N elements, V at a time; from `left` on nothing is read (0) or written.
template <typename T, int N, int V> __device__ __forceinline__ void load(const T* x, int left, float (&v)[N]) {
#pragma unroll
    for (int u = 0; u < N / V; u++) {
        float part[V];
        if (V == N || u * V < left) {
            if constexpr (V == 1) {
                part[0] = to_f32<T>(x[u]);
            } else {
                Pack<T, V> q;
                q.raw = *(const typename Piece<V * sizeof(T)>::type*)(x + u * V);
                q.get(part);
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; j++) part[j] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < V; j++) v[u * V + j] = part[j];
    }
}
template <typename T, int N, int V> __device__ __forceinline__ void store(T* y, int left, const float (&v)[N]) {
#pragma unroll
    for (int u = 0; u < N / V; u++) {
        if (V == N || u * V < left) {
            if constexpr (V == 1) {
                y[u] = from_f32<T>(v[u]);
            } else {
                float part[V];
#pragma unroll
                for (int j = 0; j < V; j++) part[j] = v[u * V + j];
                Pack<T, V> q;
                q.set(part);
                *(typename Piece<V * sizeof(T)>::type*)(y + u * V) = q.raw;
            }
        }
    }
}

// A thread holds N elements of a row, V of them to an access (V < N: rows that do not start on 16 bytes or hold no whole pieces). `team` threads side by side walk a row.
// Rows from the last expert's end on are set to zero, and not read.
template <typename T, int N, int V, bool GRAD, int ACT> __global__ void __launch_bounds__(THREADS) hccl_activate_rows(const __grid_constant__ ActivateParams p, int team) {
    const int teams = THREADS / team, mine = (int)threadIdx.x / team, rank = (int)threadIdx.x % team;
    const long long rows = p.offsets ? min((long long)p.offsets[p.groups], p.M) : p.M;
    unsigned long long key = 0, call = 0;
    if (p.drop) key = (unsigned long long)p.seed[0], call = (unsigned long long)p.seed[1];
    for (long long r = (long long)blockIdx.x * teams + mine; r < p.M; r += (long long)gridDim.x * teams) {
        const T* x = (const T*)p.x + r * p.ldx;
        const T* dy = (const T*)p.dy + r * p.ldy;
        T* out = (T*)p.out + r * p.ldo;
        const unsigned long long at = (unsigned long long)r * (unsigned long long)p.I;
        for (long long c = (long long)rank * N; c < p.I; c += (long long)team * N) {
            const int left = (int)min((long long)N, p.I - c);
            float f[N], g[N], u[N], d[N];
            if (r >= rows) {
#pragma unroll
                for (int j = 0; j < N; j++) f[j] = 0.f;
                store<T, N, V>(out + c, left, f);
                if (GRAD && p.gated) store<T, N, V>(out + p.I + c, left, f);
                continue;
            }
            load<T, N, V>(x + c, left, g);
            if (p.gated) load<T, N, V>(x + p.I + c, left, u);
            if (GRAD) load<T, N, V>(dy + c, left, d);
            if (!p.gated)
#pragma unroll
                for (int j = 0; j < N; j++) u[j] = 1.f;
            if (p.drop) factors<N>(p, key, call, at + (unsigned long long)c, f);
            else
#pragma unroll
                for (int j = 0; j < N; j++) f[j] = 1.f;
            if constexpr (!GRAD) {
#pragma unroll
                for (int j = 0; j < N; j++) {
                    const float v = activation(ACT, g[j]) * u[j] * f[j];
                    g[j] = f[j] == 0.f ? 0.f : v;  // (dropped is 0, whatever it was)
                }
                store<T, N, V>(out + c, left, g);
            } else {
#pragma unroll
                for (int j = 0; j < N; j++) {
                    float a, slope;
                    activation_slope(ACT, g[j], &a, &slope);
                    const float dd = d[j] * f[j];
                    const bool off = f[j] == 0.f;
                    g[j] = off ? 0.f : dd * u[j] * slope;
                    u[j] = off ? 0.f : dd * a;
                }
                store<T, N, V>(out + c, left, g);
                if (p.gated) store<T, N, V>(out + p.I + c, left, u);
            }
        }
    }
}

template <typename T, int N, int V, bool GRAD, int ACT> cudaError_t launch(const ActivateParams& p, cudaStream_t s) {
    const long long pieces = (p.I + N - 1) / N;
    int team = 32;
    while (team < THREADS && team < pieces) team *= 2;
    const long long blocks = (p.M + THREADS / team - 1) / (THREADS / team);
    hccl_activate_rows<T, N, V, GRAD, ACT><<<(unsigned)std::max(1ll, std::min(blocks, (long long)SMS * 8)), THREADS, 0, s>>>(p, team);
    return cudaGetLastError();
}

// The widest accesses that every row's start and length allow: 16 bytes, two elements, or one.
template <typename T, bool GRAD, int ACT> cudaError_t aligned(const ActivateParams& p, cudaStream_t s) {
    constexpr int N = sizeof(T) == 2 ? 8 : 4, WIDE = 16 / sizeof(T);
    const auto whole = [&](const void* at, long long ld, int n) { return (uintptr_t)at % (n * sizeof(T)) == 0 && (p.M <= 1 || ld % n == 0); };
    const auto all = [&](int n) { return p.I % n == 0 && whole(p.x, p.ldx, n) && whole(p.out, p.ldo, n) && (!GRAD || whole(p.dy, p.ldy, n)); };
    if (all(WIDE)) return launch<T, N, WIDE, GRAD, ACT>(p, s);
    if (all(2)) return launch<T, N, 2, GRAD, ACT>(p, s);
    return launch<T, N, 1, GRAD, ACT>(p, s);
}

template <typename T, bool GRAD> cudaError_t typed(const ActivateParams& p, cudaStream_t s) {
    if (p.act == HCCL_ACT_SILU) return aligned<T, GRAD, HCCL_ACT_SILU>(p, s);
    if (p.act == HCCL_ACT_GELU) return aligned<T, GRAD, HCCL_ACT_GELU>(p, s);
    return aligned<T, GRAD, HCCL_ACT_RELU>(p, s);
}

template <bool GRAD> cudaError_t any(int dt, const ActivateParams& p, cudaStream_t s) {
    if (p.M == 0 || p.I == 0) return cudaSuccess;
    if (dt == HCCL_FP32) return typed<float, GRAD>(p, s);
    if (dt == HCCL_BF16) return typed<__nv_bfloat16, GRAD>(p, s);
    return typed<__half, GRAD>(p, s);
}

}  // namespace

cudaError_t launch_activate(int dt, const ActivateParams& p, cudaStream_t s) { return any<false>(dt, p, s); }
cudaError_t launch_activate_grad(int dt, const ActivateParams& p, cudaStream_t s) { return any<true>(dt, p, s); }

}  // namespace experts
}  // namespace hccl
