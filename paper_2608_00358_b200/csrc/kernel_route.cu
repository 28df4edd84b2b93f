// Routing of tokens to experts: scores, the choice of the top k, their weights, the layout of the rows in expert
// order, and the gradient of the scores.
//
// One warp holds one token's scores in registers, expert e in register e / 32 of lane e % 32. The keys that the choice
// goes by are mapped to unsigned integers in the same order (sign bit flipped, negative numbers complemented), so
// that a maximum over the warp is one redux instruction; 0 stands for "not eligible" and is below every key.
#include "experts.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int ROUTE_THREADS = 256, ROUTE_WARPS = ROUTE_THREADS / 32;

__device__ __forceinline__ unsigned ordered(float f) {
    const unsigned u = __float_as_uint(f + 0.0f);  // -0 becomes +0: they compare equal
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float unordered(unsigned k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}

// Scores of one token. On return s[] is the score's numerator (sigmoid: the score itself; softmax: exp(l - max)), key[] the ordered
// key or 0. Returns false for a token that cannot be scored. *total: the softmax's sum (1 for the sigmoid).
template <typename T, int V>
__device__ __forceinline__ bool score_token(const RouteParams& p, long long t, int lane, float (&s)[V], unsigned (&key)[V], float* total) {
    const T* row = (const T*)p.logits + t * p.ld;
    float l[V], b[V];
#pragma unroll
    for (int i = 0; i < V; i++) {
        const int e = i * 32 + lane;
        l[i] = e < p.E ? to_f32<T>(row[e]) : -INFINITY;
        b[i] = (p.bias && e < p.E) ? p.bias[e] : 0.f;
    }
    bool bad = false, off[V];
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; i++) {
        off[i] = l[i] == -INFINITY || b[i] == -INFINITY;
        if (!off[i]) {
            bad |= isnan(l[i]) || !(b[i] < INFINITY) || (!p.sigmoid && l[i] == INFINITY);
            m = fmaxf(m, l[i]);
        }
    }
    if (__any_sync(FULL, bad)) return false;
    if (p.sigmoid) {
#pragma unroll
        for (int i = 0; i < V; i++) {
            s[i] = off[i] ? 0.f : 1.f / (1.f + expf(-l[i]));
            key[i] = off[i] ? 0u : ordered(s[i] + b[i]);
        }
        *total = 1.f;
        return true;
    }
    m = unordered(__reduce_max_sync(FULL, ordered(m)));
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; i++) {
        s[i] = off[i] ? 0.f : expf(l[i] - m);  // l is finite and so is m, if any expert is eligible
        sum += s[i];
    }
    sum = warp_sum(sum);
    *total = sum;
#pragma unroll
    for (int i = 0; i < V; i++) key[i] = off[i] ? 0u : ordered(p.bias ? s[i] / sum + b[i] : l[i]);
    return true;
}

// Clears the keys of experts whose group is not among the best. Lane g keeps group g's score.
template <int V> __device__ __forceinline__ void keep_best_groups(const RouteParams& p, int lane, unsigned (&key)[V]) {
    // groups beyond 32 are walked in rounds of 32: lane j of round r holds group r * 32 + j
    unsigned mine[V];  // group score (ordered) of group r * 32 + lane
#pragma unroll
    for (int r = 0; r < V; r++) mine[r] = 0;
    for (int g = 0; g < p.groups; g++) {
        const int lo = g * p.per_group, hi = lo + p.per_group;
        unsigned k1 = 0, k2 = 0;
#pragma unroll
        for (int i = 0; i < V; i++) {
            if (i * 32 + 31 >= lo && i * 32 < hi) {
                const int e = i * 32 + lane;
                const unsigned k = (e >= lo && e < hi) ? key[i] : 0u;
                k2 = max(k2, min(k1, k));
                k1 = max(k1, k);
            }
        }
        const unsigned m1 = __reduce_max_sync(FULL, k1);
        unsigned score = m1;
        if (p.group_best == 2) {
            const int owner = __ffs(__ballot_sync(FULL, k1 == m1)) - 1;
            const unsigned m2 = __reduce_max_sync(FULL, lane == owner ? k2 : k1);
            if (m1 && m2) score = ordered(unordered(m1) + unordered(m2));
        }
#pragma unroll
        for (int r = 0; r < V; r++)
            if (g == r * 32 + lane) mine[r] = score;
    }
    unsigned chosen[V];  // bit g % 32 of word g / 32, the same in all lanes
#pragma unroll
    for (int r = 0; r < V; r++) chosen[r] = 0;
    for (int n = 0; n < p.top_groups; n++) {
        unsigned best = 0;
#pragma unroll
        for (int r = 0; r < V; r++) best = max(best, mine[r]);
        best = __reduce_max_sync(FULL, best);
        if (!best) break;
        bool done = false;
#pragma unroll
        for (int r = 0; r < V; r++) {
            const unsigned who = __ballot_sync(FULL, mine[r] == best);
            if (!done && who) {
                const int owner = __ffs(who) - 1;
                chosen[r] |= 1u << owner;
                if (lane == owner) mine[r] = 0;
                done = true;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; i++) {
        const int g = (i * 32 + lane) / p.per_group;
        unsigned word = 0;
#pragma unroll
        for (int r = 0; r < V; r++)
            if (g / 32 == r) word = chosen[r];
        if (!((word >> (g & 31)) & 1u)) key[i] = 0;
    }
}

// Layout of this block's tokens: base[e] (shared) = first row of expert e for this block; the rows of a block's
// tokens follow in token order. Each warp takes a run of the block's choices; a first walk counts them by expert, a second hands
// out the rows with match_any, so that the order does not depend on which warp is faster.
__device__ __forceinline__ void layout_block(const RouteParams& p, long long t0, long long t1, int* base, int* cnt, int threads) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = threads / 32;
    const long long first = t0 * p.K, n = (t1 - t0) * p.K;
    const long long per = ((n + warps - 1) / warps + 31) / 32 * 32;
    const long long lo = min((long long)warp * per, n), hi = min(lo + per, n);
    int* mine = cnt + (size_t)warp * p.E;
    for (int e = lane; e < p.E; e += 32) mine[e] = 0;
    __syncwarp();
    for (long long i = lo + lane; i < hi; i += 32) {
        const int e = p.ids[first + i];
        if (e >= 0) atomicAdd(&mine[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.E; e += threads) {  // counts become first rows
        int at = base[e];
        for (int w = 0; w < warps; w++) {
            const int c = cnt[(size_t)w * p.E + e];
            cnt[(size_t)w * p.E + e] = at;
            at += c;
        }
    }
    __syncthreads();
    for (long long b = lo; b < hi; b += 32) {
        const long long i = b + lane;
        const int e = i < hi ? p.ids[first + i] : -1;
        const unsigned same = __match_any_sync(FULL, e);
        int row = -1;
        if (e >= 0) row = mine[e] + __popc(same & ((1u << lane) - 1));
        __syncwarp();
        if (e >= 0 && (same >> lane) == 1u) mine[e] += __popc(same);  // the highest lane of its set moves the counter on
        __syncwarp();
        if (i < hi) {
            p.slots[first + i] = row;
            if (row >= 0) p.source[row] = (int)(first + i);
        }
    }
}

// Offsets of all experts from their totals, and this block's first rows. tot and base: shared, E ints each.
__device__ __forceinline__ void offsets_block(const RouteParams& p, int* tot, int* base, bool write, int threads) {
    // one warp scans the totals
    if (threadIdx.x < 32) {
        int run = 0;
        for (int b = 0; b < p.E; b += 32) {
            const int e = b + (int)threadIdx.x;
            const int c = e < p.E ? tot[e] : 0;
            int inc = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(FULL, inc, o);
                if ((int)threadIdx.x >= o) inc += v;
            }
            if (e < p.E) {
                const int start = run + inc - c;
                if (write) {
                    p.offsets[e] = start;
                    p.counts[e] = c;
                }
                base[e] += start;
            }
            run += __shfl_sync(FULL, inc, 31);
        }
        if (threadIdx.x == 0) {
            tot[p.E] = run;
            if (write) p.offsets[p.E] = run;
        }
    }
    __syncthreads();
}

template <typename T, int V>
__global__ void __launch_bounds__(ROUTE_THREADS) hccl_route_choose(const __grid_constant__ RouteParams p) {
    extern __shared__ int sm[];  // hist[E]
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    for (int e = threadIdx.x; e < p.E; e += ROUTE_THREADS) sm[e] = 0;
    __syncthreads();
    const long long t0 = (long long)blockIdx.x * p.chunk, t1 = min(t0 + p.chunk, p.tokens);
    for (long long t = t0 + warp; t < t1; t += ROUTE_WARPS) {
        int id = -1;       // of choice `lane`
        float w = 0.f;
        float s[V], total = 1.f;
        unsigned key[V];
        const bool live = !p.mask || p.mask[t];
        if (live) {
            if (!score_token<T, V>(p, t, lane, s, key, &total)) {
                w = __int_as_float(0x7fc00000);
            } else {
                if (p.groups > 1) keep_best_groups<V>(p, lane, key);
                for (int k = 0; k < p.K; k++) {
                    unsigned best = 0;
                    int at = 0;
                    float sv = 0.f;
#pragma unroll
                    for (int i = 0; i < V; i++)
                        if (key[i] > best) best = key[i], at = i, sv = s[i];
                    const unsigned m = __reduce_max_sync(FULL, best);
                    if (!m) break;
                    const int e = __reduce_min_sync(FULL, best == m ? at * 32 + lane : 0x7fffffff);
                    const float se = __shfl_sync(FULL, sv, e & 31);
#pragma unroll
                    for (int i = 0; i < V; i++)
                        if (e == i * 32 + lane) key[i] = 0;
                    if (lane == k) id = e, w = se;
                }
                // softmax: s is exp(l - max); the common divisor drops out of a renormalised weight
                const float div = p.renorm ? warp_sum(w) : total;
                w = div > 0.f ? w / div * p.scale : 0.f;
            }
        }
        if (lane < p.K) {
            p.ids[t * p.K + lane] = id;
            p.weights[t * p.K + lane] = w;
            if (id >= 0) atomicAdd(&sm[id], 1);
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.E; e += ROUTE_THREADS) p.hist[(size_t)blockIdx.x * p.E + e] = sm[e];
}

__global__ void __launch_bounds__(ROUTE_THREADS) hccl_route_layout(const __grid_constant__ RouteParams p) {
    extern __shared__ int sm[];  // tot[E + 1], base[E], cnt[ROUTE_WARPS][E]
    int *tot = sm, *base = sm + p.E + 1, *cnt = base + p.E;
    for (int e = threadIdx.x; e < p.E; e += ROUTE_THREADS) {
        int before = 0, all = 0;
        for (int b = 0; b < p.blocks; b++) {
            const int c = p.hist[(size_t)b * p.E + e];
            if (b < (int)blockIdx.x) before += c;
            all += c;
        }
        tot[e] = all;
        base[e] = before;
    }
    __syncthreads();
    offsets_block(p, tot, base, blockIdx.x == 0, ROUTE_THREADS);
    const long long t0 = (long long)blockIdx.x * p.chunk, t1 = min(t0 + p.chunk, p.tokens);
    if (t0 < t1) layout_block(p, t0, t1, base, cnt, ROUTE_THREADS);
    // rows that belong to no choice
    const long long n = p.tokens * p.K;
    for (long long i = tot[p.E] + (long long)blockIdx.x * ROUTE_THREADS + threadIdx.x; i < n; i += (long long)gridDim.x * ROUTE_THREADS) p.source[i] = -1;
}

// d of the logits. Weight j of the chosen has w_j = scale * s_j / S (S = sum of the chosen scores if renormalised, else 1), so
// ds_j = scale / S * (dw_j - sum_i dw_i s_i / S) or scale * dw_j; then the score's own derivative:
// sigmoid dl = ds s (1 - s), softmax dl_e = s_e (ds_e - sum_j ds_j s_j) over all experts.
template <typename T, int V>
__global__ void __launch_bounds__(ROUTE_THREADS) hccl_route_grad(const __grid_constant__ RouteGradParams q) {
    const RouteParams& p = q.r;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    for (long long t = (long long)blockIdx.x * ROUTE_WARPS + warp; t < p.tokens; t += (long long)gridDim.x * ROUTE_WARPS) {
        T* out = (T*)q.dlogits + t * q.ldd;
        float s[V], total = 1.f, d[V];
        unsigned key[V];
        const bool live = !p.mask || p.mask[t];
        bool ok = live;
        if (live) ok = score_token<T, V>(p, t, lane, s, key, &total);
        if (!ok) {
            const T v = from_f32<T>(live ? __int_as_float(0x7fc00000) : 0.f);
            for (int e = lane; e < p.E; e += 32) out[e] = v;
            continue;
        }
        const float inv = total > 0.f ? 1.f / total : 0.f;  // 0: no expert was eligible
        int id = -1;
        float dw = 0.f, c = 0.f;
        if (lane < p.K) {
            id = p.ids[t * p.K + lane];
            if (id >= p.E) id = -1;
            if (id >= 0) dw = q.dweights[t * p.K + lane] * p.scale;
        }
        // score of this lane's choice
        for (int k = 0; k < p.K; k++) {
            const int e = __shfl_sync(FULL, id, k);
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < V; i++)
                if (e == i * 32 + lane) v = s[i];
            v = __shfl_sync(FULL, v, e & 31);
            if (lane == k && e >= 0) c = v;
        }
        if (p.renorm) {
            const float S = warp_sum(c);
            const float r = S > 0.f ? 1.f / S : 0.f;
            dw = (dw - warp_sum(dw * c) * r) * r;  // the softmax's divisor has dropped out: d of exp(l - max)
            if (id < 0) dw = 0.f;
            // in terms of exp(l - max) the chain through the sum is already in: dl_e = exp_e * dw_e
        }
        const float dot = (!p.sigmoid && !p.renorm) ? warp_sum(dw * c) * inv : 0.f;
#pragma unroll
        for (int i = 0; i < V; i++) d[i] = 0.f;
        for (int k = 0; k < p.K; k++) {
            const int e = __shfl_sync(FULL, id, k);
            const float g = __shfl_sync(FULL, dw, k);
#pragma unroll
            for (int i = 0; i < V; i++)
                if (e == i * 32 + lane) d[i] = g;
        }
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int e = i * 32 + lane;
            if (e >= p.E) continue;
            float v;
            if (p.sigmoid) v = d[i] * s[i] * (1.f - s[i]);
            else if (p.renorm) v = d[i] * s[i];
            else v = s[i] * inv * (d[i] - dot);
            out[e] = from_f32<T>(v);
        }
    }
}

int route_blocks(long long tokens) {
    const long long b = (tokens + ROUTE_WARPS - 1) / ROUTE_WARPS;
    return (int)(b < 1 ? 1 : (b > SMS ? SMS : b));
}

template <typename T, int V> cudaError_t route_launch(const RouteParams& p, cudaStream_t s) {
    hccl_route_choose<T, V><<<p.blocks, ROUTE_THREADS, p.E * 4, s>>>(p);
    hccl_route_layout<<<p.blocks, ROUTE_THREADS, (2 * p.E + 1 + ROUTE_WARPS * p.E) * 4, s>>>(p);
    return cudaGetLastError();
}
template <typename T, int V> cudaError_t grad_launch(const RouteGradParams& p, cudaStream_t s) {
    const long long b = (p.r.tokens + ROUTE_WARPS - 1) / ROUTE_WARPS;
    hccl_route_grad<T, V><<<(int)(b > SMS * 8 ? SMS * 8 : b), ROUTE_THREADS, 0, s>>>(p);
    return cudaGetLastError();
}

#define ROUTE_PICK_V(FN, T, E, ...)                       \
    do {                                                  \
        const int v_ = ((E) + 31) / 32;                   \
        if (v_ <= 2) return FN<T, 2>(__VA_ARGS__);        \
        if (v_ <= 4) return FN<T, 4>(__VA_ARGS__);        \
        if (v_ <= 8) return FN<T, 8>(__VA_ARGS__);        \
        if (v_ <= 16) return FN<T, 16>(__VA_ARGS__);      \
        return FN<T, 32>(__VA_ARGS__);                    \
    } while (0)

}  // namespace

size_t route_workspace(int E, long long tokens) { return (size_t)route_blocks(tokens) * E * 4; }

cudaError_t launch_route(int dt, const RouteParams& in, cudaStream_t s) {
    RouteParams p = in;
    p.blocks = route_blocks(p.tokens);
    p.chunk = (int)((p.tokens + p.blocks - 1) / p.blocks);
    if (dt == HCCL_FP32) ROUTE_PICK_V(route_launch, float, p.E, p, s);
    if (dt == HCCL_BF16) ROUTE_PICK_V(route_launch, __nv_bfloat16, p.E, p, s);
    ROUTE_PICK_V(route_launch, __half, p.E, p, s);
}

cudaError_t launch_route_grad(int dt, const RouteGradParams& p, cudaStream_t s) {
    if (p.r.tokens == 0) return cudaSuccess;
    if (dt == HCCL_FP32) ROUTE_PICK_V(grad_launch, float, p.r.E, p, s);
    if (dt == HCCL_BF16) ROUTE_PICK_V(grad_launch, __nv_bfloat16, p.r.E, p, s);
    ROUTE_PICK_V(grad_launch, __half, p.r.E, p, s);
}

}  // namespace experts
}  // namespace hccl
