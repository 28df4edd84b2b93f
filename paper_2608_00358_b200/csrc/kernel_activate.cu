// The gated activation between an expert's two products, with dropout: y[r, i] = act(x[r, i]) x[r, I + i] m[r, i], and its gradient. m is 0 or 1 / (1 - p), from a
// counter-based generator, and is formed anew wherever it is needed: nothing of it is stored. Without a gate y = act(x) m.
//
// The generator is Philox-4x32-10 (Salmon, Moraes, Dror, Shaw 2011): four 32-bit words from a 128-bit counter and a 64-bit key in ten rounds of two 32 x 32 bit
// products. Element i of the result (row * I + column) takes word i % 4 of the counter (i / 4, call); it is kept if the word is at least p 2^32.
//
// Measured (B200, copy peak 6.5 TB/s): SiLU, 32768 x 2048 bf16 without dropout 62 us, gradient 101; with dropout 92 and 107 (GELU 111 and 127): 32 instructions
// an element issue in two thirds of the cycles, about 10 of them the generator's (18 wide products for four elements, and what joins them).
#include <algorithm>

#include "activate.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int THREADS = 128;

struct Words {
    unsigned w[4];
};
// A call's generator. The keys of the ten rounds, and of the first two rounds what hangs on the call and on the counter's upper half alone, are formed once.
struct Generator {
    unsigned k[10][2], upper, c0, c1;
    unsigned long long a, call;
    __device__ __forceinline__ Generator(unsigned long long key, unsigned long long call) : call(call) {
#pragma unroll
        for (int r = 0; r < 10; r++) k[r][0] = (unsigned)key + r * 0x9E3779B9u, k[r][1] = (unsigned)(key >> 32) + r * 0xBB67AE85u;
        set(0);
    }
    __device__ __forceinline__ void set(unsigned u) {
        const unsigned long long b = (unsigned long long)(unsigned)call * 0xCD9E8D57u;
        upper = u;
        c0 = (unsigned)(b >> 32) ^ upper ^ k[0][0];
        c1 = (unsigned)b;
        a = (unsigned long long)c0 * 0xD2511F53u;
    }
    __device__ __forceinline__ Words at(unsigned long long counter) {
        if ((unsigned)(counter >> 32) != upper) set((unsigned)(counter >> 32));
        return beside((unsigned)counter);
    }
    // Of a counter whose upper half is that of the last one.
    __device__ __forceinline__ Words beside(unsigned counter) const {
        const unsigned long long first = (unsigned long long)counter * 0xD2511F53u;
        const unsigned d2 = (unsigned)(first >> 32) ^ (unsigned)(call >> 32) ^ k[0][1], d3 = (unsigned)first;
        const unsigned long long second = (unsigned long long)d2 * 0xCD9E8D57u;
        unsigned x0 = (unsigned)(second >> 32) ^ c1 ^ k[1][0], x1 = (unsigned)second, x2 = (unsigned)(a >> 32) ^ d3 ^ k[1][1], x3 = (unsigned)a;
#pragma unroll
        for (int r = 2; r < 10; r++) {
            const unsigned long long m = (unsigned long long)x0 * 0xD2511F53u, q = (unsigned long long)x2 * 0xCD9E8D57u;
            x0 = (unsigned)(q >> 32) ^ x1 ^ k[r][0];
            x1 = (unsigned)q;
            x2 = (unsigned)(m >> 32) ^ x3 ^ k[r][1];
            x3 = (unsigned)m;
        }
        return {{x0, x1, x2, x3}};
    }
};

// The random words of N neighbouring elements, N a multiple of 4, the first being element `at` of the result. WHOLE: `at` is a multiple of N; otherwise a counter's words may
// begin within the elements.
template <int N, bool WHOLE> __device__ __forceinline__ void words(Generator& gen, unsigned long long at, unsigned (&f)[N]) {
    const unsigned o = WHOLE ? 0u : (unsigned)at & 3u;
    if (o == 0) {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const Words w = WHOLE && j ? gen.beside((unsigned)(at / 4) + j / 4) : gen.at(at / 4 + j / 4);
#pragma unroll
            for (int i = 0; i < 4; i++) f[j + i] = w.w[i];
        }
    } else {
        Words w = gen.at(at / 4);
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const Words next = gen.at(at / 4 + j / 4 + 1);
#pragma unroll
            for (int i = 0; i < 4; i++) f[j + i] = i + o == 1 ? w.w[1] : i + o == 2 ? w.w[2] : i + o == 3 ? w.w[3] : i + o == 4 ? next.w[0] : i + o == 5 ? next.w[1] : next.w[2];
            w = next;
        }
    }
}

// For results of 16 bits. What the exponentials' arguments lose by rounding costs (|x| + 11) 2^-24 of SiLU, where expf takes four instructions to save that.
__device__ __forceinline__ Two exponentials(Two x) {  // 2^x
    float a, b;
    x.get(a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    return Two(a, b);
}
__device__ __forceinline__ Two reciprocals(Two x) {
    float a, b;
    x.get(a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return Two(a, b);
}
// 2^16 / (1 + exp(-x)): by the factor, which meets the exponential's argument, neither is infinite nor the quotient 0 before x times it is below 2^-126 (without it SiLU
// would be 0 from -88.7 on, where the result may still be of any size: -90 beside 1e38 gives -7). The sums one by one: as pairs the gradient is given 80 registers in the place of 94 and takes 111 us instead of 107.
__device__ __forceinline__ Two large_logistic(Two x) {
    float a, b;
    exponentials(fma2(x, Two(-1.44269504f), Two(-16.f))).get(a, b);
    return reciprocals(Two(a + 0x1p-16f, b + 0x1p-16f));
}
// The normal distribution times `part` (a power of two), and exp(-x^2 / 2). Below 0 the distribution is exp(-x^2 / 2) R(|x|); R, which falls from 1/2 as slowly as 1 / |x|, is a polynomial of degree 7 in 1 / (1 + 0.35 |x|), by
// least squares on Chebyshev's points, weighted anew until the relative error was even: 2^-21.4, and as it is evaluated here 2^-20.7, up to 13.2, where the exponential leaves the normal numbers and is taken as 0.
// The exponential's argument is rounded twice, which costs x^2 2^-24 of the result. (normcdff with expf takes four times the instructions, 32768 x 2048 bf16 with dropout 221 us, gradient 263.)
__device__ __forceinline__ Two normal(Two x, float part, Two* bell) {
    float a, b;
    x.get(a, b);
    const Two t = reciprocals(fma2(Two(fabsf(a), fabsf(b)), Two(0.35f), Two(1.f)));
    Two r = fma2(Two(4.88590253e-02f * part), t, Two(-2.01797222e-01f * part));
    r = fma2(r, t, Two(2.40131299e-01f * part));
    r = fma2(r, t, Two(-1.65972006e-02f * part));
    r = fma2(r, t, Two(1.55758767e-01f * part));
    r = fma2(r, t, Two(1.33409697e-01f * part));
    r = fma2(r, t, Two(1.40262654e-01f * part));
    r = fma2(r, t, Two(-2.68791464e-05f * part));
    *bell = exponentials(x * x * Two(-0.72134752f));
    const Two below = *bell * r;
    float u, v, c, d;
    below.get(u, v);
    fma2(below, Two(-1.f), Two(part)).get(c, d);
    return Two(a < 0.f ? u : c, b < 0.f ? v : d);
}

// N elements as they lie in memory, V to an access; from `left` on nothing is read.
template <typename T, int N, int V> struct Raw {
    Pack<T, V> q[N / V];
    __device__ __forceinline__ void load(const T* x, int left) {
#pragma unroll
        for (int u = 0; u < N / V; u++)
            if (V == N || u * V < left) q[u].raw = *(const typename Piece<V * sizeof(T)>::type*)(x + u * V);
    }
    __device__ __forceinline__ void get(float (&v)[N]) const {
#pragma unroll
        for (int u = 0; u < N / V; u++) {
            float part[V];
            q[u].get(part);
#pragma unroll
            for (int j = 0; j < V; j++) v[u * V + j] = part[j];
        }
    }
};
// The first `left` of them to memory.
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
// Where a piece is one access, RING pieces of each thread are on their way into shared memory, where it alone reads them: what the generator keeps busy cannot also keep enough loads in flight.
// Rows from the last expert's end on are set to zero, and not read.
constexpr int RING = 4;
template <typename T, int N, int V, bool GRAD, int ACT> __global__ void __launch_bounds__(THREADS) hccl_activate_rows(const __grid_constant__ ActivateParams p, int team) {
    constexpr bool SHORT = sizeof(T) == 2, RINGED = V == N;
    constexpr int INPUTS = GRAD ? 3 : 2;
    constexpr float PART = GRAD ? 0.5f : 1.f;
    extern __shared__ __align__(16) uint4 ring[];  // [RING][INPUTS][threads]
    const int teams = THREADS / team, mine = (int)threadIdx.x / team, rank = (int)threadIdx.x % team;
    const long long rows = p.offsets ? min((long long)p.offsets[p.groups], p.M) : p.M;
    // A thread has `n` pieces of each of its rows, the last with `end` elements.
    const long long step = (long long)gridDim.x * teams, across = (long long)team * N, c0 = (long long)rank * N, r0 = (long long)blockIdx.x * teams + mine;
    // (the same in all lanes, and by way of the shuffle known to be: the rounds' keys then take none of a thread's registers; 94 -> 91 us)
    const auto same = [](unsigned long long v) { return (unsigned long long)__shfl_sync(0xffffffffu, (unsigned)(v >> 32), 0) << 32 | __shfl_sync(0xffffffffu, (unsigned)v, 0); };
    Generator generator(same(p.drop ? (unsigned long long)p.seed[0] : 0), same(p.drop ? (unsigned long long)p.seed[1] : 0));
    if (c0 >= p.I) return;
    const int n = (int)((p.I - c0 + across - 1) / across), end = (int)min((long long)N, p.I - c0 - (n - 1) * across);
    const long long mine_read = rows > r0 ? (rows - r0 + step - 1) / step : 0;
    const int pieces = (int)(mine_read * n);
    Raw<T, N, V> raw[INPUTS] = {};  // gate, other half, gradient

    // Where the loads are (ringed: ahead of the work), and where the work is. From piece to piece it is `across` on, at a row's end a jump: indices formed anew for
    // each piece took a sixth of the instructions.
    const long long back = (n - 1) * across;
    const T *fx = (const T*)p.x + r0 * p.ldx + c0, *fd = (const T*)p.dy + r0 * p.ldy + c0;
    const long long x_jump = step * p.ldx - back, d_jump = step * p.ldy - back, o_jump = step * p.ldo - back, a_jump = step * p.I - back;
    T* out = (T*)p.out + r0 * p.ldo + c0;
    unsigned long long at = (unsigned long long)(r0 * p.I + c0);
    int fk = 0, ahead = 0, turn = 0, k = 0;
    const auto fetch = [&](int slot) {
        if (ahead++ < pieces) {
            const T* const from[3] = {fx, fx + p.I, fd};
#pragma unroll
            for (int i = 0; i < INPUTS; i++) {
                if (i == 1 && !p.gated) continue;
                if constexpr (RINGED)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(ring + (slot * INPUTS + i) * THREADS + threadIdx.x)), "l"(from[i]) : "memory");
                else
                    raw[i].load(from[i], fk == n - 1 ? end : N);
            }
        }
        if (RINGED) asm volatile("cp.async.commit_group;" ::: "memory");
        const bool over = ++fk == n;
        if (over) fk = 0;
        fx += over ? x_jump : across;
        if (GRAD) fd += over ? d_jump : across;
    };
    if (RINGED)
#pragma unroll
        for (int i = 0; i < RING - 1; i++) fetch(i);
    for (int i = 0; i < pieces; i++) {
        fetch(turn == 0 ? RING - 1 : turn - 1);
        if constexpr (RINGED) {
            asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");
#pragma unroll
            for (int j = 0; j < INPUTS; j++) raw[j].q[0].raw = ring[(turn * INPUTS + j) * THREADS + threadIdx.x];
            turn = turn == RING - 1 ? 0 : turn + 1;
        }
        const int left = RINGED || k != n - 1 ? N : end;
        float g[N], u[N], d[N];
        unsigned word[N];
        if (p.drop) words<N, RINGED>(generator, at, word);
        else
#pragma unroll
            for (int j = 0; j < N; j++) word[j] = 0xffffffffu;
        raw[0].get(g);
        if (p.gated) raw[1].get(u);
        else
#pragma unroll
            for (int j = 0; j < N; j++) u[j] = 1.f;
        if constexpr (GRAD) raw[INPUTS - 1].get(d);
        // What is dropped is 0, whatever it was. Of finite numbers no product on the way is infinite unless the result is: large numbers meet the activation first (-1e30 of a gate and
        // 1e30 of the other half are 0), 1 / (1 - p), which only makes larger, comes last, and a slope, up to 1.13, meets the gradient by its half (PART). (A product below 2^-126 is rounded
        // to 2^-149 before it grows.)
        if constexpr (SHORT && ACT != HCCL_ACT_RELU) {
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const Two x(g[j], g[j + 1]), o(u[j], u[j + 1]), grown(p.keep / PART);
                Two f, bell;  // act(x) = x f / PART
                if constexpr (ACT == HCCL_ACT_SILU) f = large_logistic(x) * Two(0x1p-16f * PART);
                else f = normal(x, PART, &bell);
                const Two act = x * f;
                if constexpr (!GRAD) {
                    (act * o * grown).get(g[j], g[j + 1]);
                } else {
                    const Two dd(d[j], d[j + 1]);
                    Two slope;
                    if constexpr (ACT == HCCL_ACT_SILU) slope = fma2(act, fma2(f, Two(-1.f / PART), Two(1.f)), f);
                    else slope = fma2(x * Two(0.39894228f * PART), bell, f);
                    (dd * slope * o * grown).get(g[j], g[j + 1]);
                    (dd * act * grown).get(u[j], u[j + 1]);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; j++) {
                if constexpr (!GRAD) {
                    g[j] = activation(ACT, g[j]) * u[j] * p.keep;
                } else {
                    float a, slope;
                    activation_slope(ACT, g[j], &a, &slope);
                    g[j] = d[j] * (PART * slope) * u[j] * (p.keep / PART);
                    u[j] = d[j] * a * p.keep;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < N; j++) {
            g[j] = word[j] >= p.threshold ? g[j] : 0.f;
            if (GRAD) u[j] = word[j] >= p.threshold ? u[j] : 0.f;
        }
        store<T, N, V>(out, left, g);
        if (GRAD && p.gated) store<T, N, V>(out + p.I, left, u);
        const bool over = ++k == n;
        if (over) k = 0;
        out += over ? o_jump : across;
        at += over ? a_jump : across;
    }
    // (out is where the rows that are not read begin)
    float none[N];
#pragma unroll
    for (int j = 0; j < N; j++) none[j] = 0.f;
    for (long long r = r0 + mine_read * step; r < p.M; r += step)
        for (k = 0; k < n; k++) {
            const int left = k == n - 1 ? end : N;
            store<T, N, V>(out, left, none);
            if (GRAD && p.gated) store<T, N, V>(out + p.I, left, none);
            out += k == n - 1 ? o_jump : across;
        }
}

template <typename T, int N, int V, bool GRAD, int ACT> cudaError_t launch(const ActivateParams& p, cudaStream_t s) {
    const long long pieces = (p.I + N - 1) / N;
    int team = 32;
    while (team < THREADS && team < pieces) team *= 2;
    // Fewer rounds of blocks where each forms keys first. (Blocks of 128 threads against 256: 1003 x 1410 fp32 10.4 and 12.4 us, 32768 x 2048 bf16 92 and 91, its gradient 105 and 109.)
    const long long blocks = (p.M + THREADS / team - 1) / (THREADS / team);
    hccl_activate_rows<T, N, V, GRAD, ACT><<<(unsigned)std::max(1ll, std::min(blocks, (long long)SMS * (p.drop ? 12 : 64))), THREADS, V == N ? RING * (GRAD ? 3 : 2) * THREADS * 16 : 0, s>>>(p, team);
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
