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

// A thread's N elements of a row: the factors that dropout multiplies them with. `at` = row * I + column.
template <int N> __device__ __forceinline__ void factors(const ActivateParams& p, unsigned long long key, unsigned long long call, unsigned long long at, float (&f)[N]) {
    if (!p.drop) {
#pragma unroll
        for (int j = 0; j < N; j++) f[j] = 1.f;
        return;
    }
    if (at % 4 == 0 || N == 1) {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const Words w = philox(at / 4 + j / 4, call, key);
            if constexpr (N == 1) {
                const unsigned o = (unsigned)(at % 4), v = o == 0 ? w.w[0] : o == 1 ? w.w[1] : o == 2 ? w.w[2] : w.w[3];
                f[0] = v >= p.threshold ? p.keep : 0.f;
            } else {
#pragma unroll
                for (int i = 0; i < 4; i++) f[j + i] = w.w[i] >= p.threshold ? p.keep : 0.f;
            }
        }
    } else if constexpr (N >= 4) {  // the elements begin inside a counter's words
        const int o = (int)(at % 4);
        Words w = philox(at / 4, call, key);
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const Words next = philox(at / 4 + j / 4 + 1, call, key);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const unsigned v = i + o == 0 ? w.w[0] : i + o == 1 ? w.w[1] : i + o == 2 ? w.w[2] : i + o == 3 ? w.w[3] : i + o == 4 ? next.w[0] : i + o == 5 ? next.w[1] : next.w[2];
                f[j + i] = v >= p.threshold ? p.keep : 0.f;
            }
            w = next;
        }
    }
}

template <typename T, int N> __device__ __forceinline__ void load(const T* x, float (&v)[N]) {
    if constexpr (N * sizeof(T) > 16) {
        constexpr int H = 16 / sizeof(T);
#pragma unroll
        for (int u = 0; u < N / H; u++) {
            Pack<T, H> q;
            float part[H];
            q.raw = ((const uint4*)x)[u];
            q.get(part);
#pragma unroll
            for (int j = 0; j < H; j++) v[u * H + j] = part[j];
        }
    } else if constexpr (N == 1) {
        v[0] = to_f32<T>(x[0]);
    } else {
        Pack<T, N> q;
        q.raw = *(const typename Piece<N * sizeof(T)>::type*)x;
        q.get(v);
    }
}
template <typename T, int N> __device__ __forceinline__ void store(T* y, const float (&v)[N]) {
    if constexpr (N * sizeof(T) > 16) {
        constexpr int H = 16 / sizeof(T);
#pragma unroll
        for (int u = 0; u < N / H; u++) {
            Pack<T, H> q;
            float part[H];
#pragma unroll
            for (int j = 0; j < H; j++) part[j] = v[u * H + j];
            q.set(part);
            ((uint4*)y)[u] = q.raw;
        }
    } else if constexpr (N == 1) {
        y[0] = from_f32<T>(v[0]);
    } else {
        Pack<T, N> q;
        q.set(v);
        *(typename Piece<N * sizeof(T)>::type*)y = q.raw;
    }
}

// N elements of a row at a time. Rows from the last expert's end on are set to zero, and not read.
template <typename T, int N, bool GRAD> __global__ void __launch_bounds__(THREADS) hccl_activate_rows(const __grid_constant__ ActivateParams p) {
    const long long pieces = (p.I + N - 1) / N, total = p.M * pieces, step = (long long)gridDim.x * THREADS;
    const long long rows = p.offsets ? p.offsets[p.groups] : p.M;
    unsigned long long key = 0, call = 0;
    if (p.drop) key = (unsigned long long)p.seed[0], call = (unsigned long long)p.seed[1];
    for (long long i = (long long)blockIdx.x * THREADS + threadIdx.x; i < total; i += step) {
        const long long r = i / pieces, c = (i - r * pieces) * N;
        T* out = (T*)p.out + r * p.ldo + c;
        float f[N], g[N], u[N], d[N];
        if (r >= rows) {
#pragma unroll
            for (int j = 0; j < N; j++) f[j] = 0.f;
            store<T, N>(out, f);
            if (GRAD && p.gated) store<T, N>(out + p.I, f);
            continue;
        }
        const T* x = (const T*)p.x + r * p.ldx + c;
        load<T, N>(x, g);
        if (p.gated) load<T, N>(x + p.I, u);
        if (GRAD) load<T, N>((const T*)p.dy + r * p.ldy + c, d);
        factors<N>(p, key, call, (unsigned long long)r * (unsigned long long)p.I + (unsigned long long)c, f);
        if constexpr (!GRAD) {
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float a = activation(p.act, g[j]);
                f[j] = f[j] == 0.f ? 0.f : (p.gated ? a * u[j] : a) * f[j];  // (dropped is 0, whatever it was)
            }
            store<T, N>(out, f);
        } else {
#pragma unroll
            for (int j = 0; j < N; j++) {
                float a, slope;
                activation_slope(p.act, g[j], &a, &slope);
                const float dd = d[j] * f[j];
                const bool off = f[j] == 0.f;
                g[j] = off ? 0.f : dd * (p.gated ? u[j] : 1.f) * slope;
                u[j] = off ? 0.f : dd * a;
            }
            store<T, N>(out, g);
            if (p.gated) store<T, N>(out + p.I, u);
        }
    }
}

template <typename T, int N, bool GRAD> cudaError_t launch(const ActivateParams& p, cudaStream_t s) {
    const long long work = p.M * ((p.I + N - 1) / N);
    const unsigned grid = (unsigned)std::max(1ll, std::min((work + THREADS - 1) / THREADS, (long long)SMS * 8));
    hccl_activate_rows<T, N, GRAD><<<grid, THREADS, 0, s>>>(p);
    return cudaGetLastError();
}

// Eight (32-bit data: four) elements at once where every row starts on 16 bytes and holds whole pieces.
template <typename T, bool GRAD> cudaError_t typed(const ActivateParams& p, cudaStream_t s) {
    constexpr int N = 16 / sizeof(T);
    const auto whole = [&](const void* at, long long ld) { return (uintptr_t)at % 16 == 0 && (p.M <= 1 || ld % N == 0); };
    if (p.I % N == 0 && whole(p.x, p.ldx) && whole(p.out, p.ldo) && (!GRAD || whole(p.dy, p.ldy))) return launch<T, N, GRAD>(p, s);
    return launch<T, 1, GRAD>(p, s);
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
