// Routing of tokens to experts: scores, the choice of the top k, their weights, the layout of the rows in expert
// order, and the gradient of the scores.
//
// The choice. L lanes share a token (8: four tokens to a warp; 32: one). Experts go to lanes in quads: quad q = experts 4q .. 4q + 3 belongs to
// lane q % L, as its quad q / L. Keys lie in shared memory and the largest key of each quad in a register, so a round of
// the top k costs a maximum over the lane's quads, one over the lanes, and a second look at one quad. Not eligible: -inf. What bounds it is
// the chain of the rounds, each a few dependent exchanges between lanes: 1.6 instructions a cycle of 4 at 37 % of the warps for 16384 x 256, some 500 instructions of a warp for each token.
//
// Measured (B200, replayed from a graph): 16384 x 256 bf16, sigmoid, 8 groups, top 8: 21.6 us, some 15 choosing and 6.5 of layout behind it; without groups 17.2, as softmax 17.3; 32768 x 128 20.8; one token of 256
// 4.7-5.1 us, 61 x 60 5.1-5.7 us, in one launch; the gradient of 32768 x 128 5.9-7.0 us = 2.7-3.2 TB/s, of a softmax that is not renormalised 18.3 us = 1.0 TB/s: a row is read three times there.
//
// Keys with a bias are good to a few 2^-24 (__expf and an approximate reciprocal), without one they are the logits; the weights of the chosen are formed anew with
// expf and a rounded division.
#include <algorithm>
#include <atomic>
#include <cfloat>

#include "experts.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr unsigned FULL = 0xffffffffu;
constexpr int LAYOUT_THREADS = 512;
constexpr int ONE_BLOCK_WARPS = 16, MANY_WARPS = 8;
constexpr int NOT_A_NUMBER = 0x7fc00000;

__host__ __device__ constexpr int round_up(int n, int m) { return (n + m - 1) / m * m; }
// floats from one token's keys to the next: 8 banks on, so that lanes of four tokens that walk their groups do not collide
__host__ __device__ __forceinline__ int key_stride(int E) { return round_up(E, 32) + 8; }
// Lines of threads that add up counts in the layout, at most 32.
__host__ __device__ __forceinline__ int layout_lines(int E) {
    const int n = LAYOUT_THREADS / (round_up(E, 16) / 16);
    return n < 32 ? n : 32;
}
__host__ __device__ __forceinline__ int token_floats(const RouteParams& p) { return key_stride(p.E) + (p.groups > 1 ? 2 * round_up(p.groups, 4) : 0) + round_up(p.K, 4); }

template <int L> __device__ __forceinline__ float lanes_max(float v) {
    if constexpr (L == 32) {
        float r;
        asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
        return r;
    } else {
#pragma unroll
        for (int o = L / 2; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(FULL, v, o));
        return v;
    }
}
// The largest value over the lanes, and of the quads that have it the lowest.
template <int L> __device__ __forceinline__ void lanes_best(float& v, int& quad) {
    if constexpr (L == 32) {
        const float m = lanes_max<32>(v);
        quad = __reduce_min_sync(FULL, v == m ? quad : 0x7fffffff);
        v = m;
    } else {
#pragma unroll
        for (int o = L / 2; o; o >>= 1) {
            const float u = __shfl_xor_sync(FULL, v, o);
            const int q = __shfl_xor_sync(FULL, quad, o);
            const bool take = (u > v) | ((u == v) & (q < quad));  // no branch: the chain of these is the latency of a round
            v = take ? u : v;
            quad = take ? q : quad;
        }
    }
}
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = L / 2; o; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}
template <int L> __device__ __forceinline__ bool lanes_any(bool v) {
    const unsigned b = __ballot_sync(FULL, v);
    return (b >> (threadIdx.x % 32 / L * L)) & (L == 32 ? FULL : (1u << (L % 32)) - 1);
}

__device__ __forceinline__ float quick_sigmoid(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Two scores added up from their logits k1 >= k2 (k2 may be -inf), m the token's largest: without a bias logits stand in the place of keys, which have the scores' order, but it is the scores that
// are added up. Softmax: by the logarithm of exp(k1) + exp(k2), over exp(m), so that a sum far below the largest does not vanish. Not inlined: seldom asked for, and
// a call for few tokens waits for its instructions (one token of 256 experts 4.72 us against 4.78).
__device__ __noinline__ float two_scores(float k1, float k2, float m, int sigmoid) {
    if (sigmoid) return 1.f / (1.f + expf(-k1)) + 1.f / (1.f + expf(-k2));
    return fmaxf((k1 - m) + log1pf(expf(k2 - k1)), -FLT_MAX);  // -inf is for groups without experts
}

// One token for each L lanes. keys: this token's shared memory (token_floats). sbias: the bias in shared memory, up to a multiple of 4 experts; odd: some of
// it is infinite or NaN. Writes ids and weights (ids to `kept` too, shared, unless null), counts the chosen in hist.
template <typename T, int Q, int L>
__device__ __forceinline__ void choose_token(const RouteParams& p, long long t, bool in, float* keys, const float* sbias, bool odd, int* hist, int* kept) {
    const int lane = threadIdx.x % 32, l = lane % L;
    const int stride = key_stride(p.E), gpad = p.groups > 1 ? round_up(p.groups, 4) : 0;
    float* gscore = keys + stride;
    int* gkeep = (int*)(gscore + gpad);
    int* chosen = (int*)(keys + stride + 2 * gpad);
    const bool live = in && (!p.mask || p.mask[t]);
    const T* row = (const T*)p.logits + (in ? t : 0) * p.ld;
    const auto bias_quad = [&](int i, float (&b)[4]) {
        const float4 b4 = *(const float4*)(sbias + (i * L + l) * 4);
        b[0] = b4.x, b[1] = b4.y, b[2] = b4.z, b[3] = b4.w;
    };

    float x[Q][4];
    if (p.vec) {  // whole quads, all asked for before the first is looked at
        Pack<T, 4> raw[Q];
#pragma unroll
        for (int i = 0; i < Q; i++) {
            raw[i].raw = {};
            if (live && (i * L + l) * 4 < p.E) raw[i].raw = ((const typename Piece<4 * sizeof(T)>::type*)row)[i * L + l];
        }
#pragma unroll
        for (int i = 0; i < Q; i++) {
            raw[i].get(x[i]);
            const float off = live && (i * L + l) * 4 < p.E ? 0.f : -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; j++) x[i][j] += off;
        }
    } else {
#pragma unroll
        for (int i = 0; i < Q; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int e = (i * L + l) * 4 + j;
                x[i][j] = -INFINITY;
                if (live && e < p.E) x[i][j] = to_f32<T>(row[e]);
            }
    }
    bool bad = false;
    if (odd) {
#pragma unroll
        for (int i = 0; i < Q; i++) {
            if ((i * L + l) * 4 >= p.E) continue;
            float b[4];
            bias_quad(i, b);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if (b[j] == -INFINITY) x[i][j] = -INFINITY;  // the expert is off, whatever its logit
                bad |= x[i][j] != -INFINITY && !(b[j] < INFINITY);
            }
        }
    }
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < Q; i++) m = max_or_nan(m, max_or_nan(max_or_nan(x[i][0], x[i][1]), max_or_nan(x[i][2], x[i][3])));
    bad |= isnan(m);
    m = lanes_max<L>(m);
    bad |= !p.sigmoid && m == INFINITY;
    bad = lanes_any<L>(bad);
    float total = 1.f;
    if (p.sigmoid) {  // (without a bias the logits are the keys: their order is the scores', also where those round to the same number)
        if (p.bias) {
#pragma unroll
            for (int i = 0; i < Q; i++) {
                float b[4] = {0.f, 0.f, 0.f, 0.f};
                if ((i * L + l) * 4 < p.E) bias_quad(i, b);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float off = x[i][j] == -INFINITY ? -INFINITY : b[j];  // (not around the sigmoid: that would be a branch for each)
                    x[i][j] = quick_sigmoid(x[i][j]) + off;
                }
            }
        }
    } else if (p.bias || !p.renorm) {
        const float base = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < Q; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) sum += __expf(x[i][j] - base);
        total = lanes_sum<L>(sum);
        if (p.bias) {
            const float r = total > 0.f ? __fdividef(1.f, total) : 0.f;  // nothing left: 0 * infinity would make keys that are not numbers
#pragma unroll
            for (int i = 0; i < Q; i++)
                if ((i * L + l) * 4 < p.E) {
                    float b[4];
                    bias_quad(i, b);
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const float off = x[i][j] == -INFINITY ? -INFINITY : b[j];
                        x[i][j] = __expf(x[i][j] - base) * r + off;
                    }
                }
        }
    }
    // x is the key now
#pragma unroll
    for (int i = 0; i < Q; i++)
        if ((i * L + l) * 4 < p.E) *(float4*)(keys + (i * L + l) * 4) = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
    const auto group_score = [&](float k1, float k2) {
        if (p.group_best != 2 || k1 == -INFINITY) return k1;
        if (!p.bias) return two_scores(k1, k2, m, p.sigmoid);
        return k2 == -INFINITY ? k1 : k1 + k2;
    };
    float top[Q];
#pragma unroll
    for (int i = 0; i < Q; i++) top[i] = fmaxf(fmaxf(x[i][0], x[i][1]), fmaxf(x[i][2], x[i][3]));
    if (p.groups > 1) {
        if (L == 32 && p.segment) {
            // A group's quads are neighbouring lanes' i-th (with 8 lanes this costs more instructions than it saves: 16384 x 256 27.5 us against 24.8): the two largest of each quad, then of the lanes by exchange, all quads side by side.
#pragma unroll
            for (int i = 0; i < Q; i++) {
                const float a1 = fmaxf(x[i][0], x[i][1]), a2 = fminf(x[i][0], x[i][1]), b1 = fmaxf(x[i][2], x[i][3]), b2 = fminf(x[i][2], x[i][3]);
                float k1 = fmaxf(a1, b1), k2 = fmaxf(fminf(a1, b1), fmaxf(a2, b2));
#pragma unroll
                for (int o = 1; o < L; o <<= 1) {
                    if (o >= p.segment) break;
                    const float o1 = __shfl_xor_sync(FULL, k1, o), o2 = __shfl_xor_sync(FULL, k2, o);
                    k2 = fmaxf(fminf(k1, o1), fmaxf(k2, o2));
                    k1 = fmaxf(k1, o1);
                }
                const int q = i * L + l;
                if ((l & (p.segment - 1)) == 0 && q * 4 < p.E) gscore[q >> (31 - __clz(p.segment))] = (p.group_best == 2 && k2 != -INFINITY) ? k1 + k2 : k1;
            }
        } else {
            __syncwarp();
            for (int g = l; g < p.groups; g += L) {
                float k1 = -INFINITY, k2 = -INFINITY, o1 = -INFINITY, o2 = -INFINITY;  // the two largest, of two halves: two chains of latencies side by side
                const auto seen = [&](float v) {
                    k2 = fmaxf(k2, fminf(k1, v));
                    k1 = fmaxf(k1, v);
                };
                const auto seen_too = [&](float v) {
                    o2 = fmaxf(o2, fminf(o1, v));
                    o1 = fmaxf(o1, v);
                };
                const float* k = keys + g * p.per_group;
                // lanes start at different places of their groups: different banks
                if (p.per4) {
                    const int quads = p.per_group / 4;
                    int at = min(l & 7, quads - 1);
                    for (int i = 0; i < quads; i += 4) {
                        float4 v[4];
#pragma unroll
                        for (int u = 0; u < 4; u++) {
                            v[u] = *(const float4*)(k + 4 * at);
                            at = at + 1 == quads ? 0 : at + 1;
                        }
#pragma unroll
                        for (int u = 0; u < 4; u++) {
                            if (i + u >= quads) v[u] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);  // round again: seen already
                            seen(v[u].x), seen_too(v[u].z), seen(v[u].y), seen_too(v[u].w);
                        }
                    }
                } else {
                    int at = g % p.per_group;
                    for (int i = 0; i < p.per_group; i++) {
                        seen(k[at]);
                        at = at + 1 == p.per_group ? 0 : at + 1;
                    }
                }
                seen(o1), seen(o2);
                gscore[g] = group_score(k1, k2);
            }
        }
        for (int g = p.groups + l; g < gpad; g += L) gscore[g] = -INFINITY;
        __syncwarp();
        for (int g = l; g < p.groups; g += L) {
            const float mine = gscore[g];
            int above = 0;
            for (int o = 0; o < gpad; o += 4) {
                const float4 v = *(const float4*)(gscore + o);
                above += (v.x > mine) | ((v.x == mine) & (o < g));
                above += (v.y > mine) | ((v.y == mine) & (o + 1 < g));
                above += (v.z > mine) | ((v.z == mine) & (o + 2 < g));
                above += (v.w > mine) | ((v.w == mine) & (o + 3 < g));
            }
            gkeep[g] = above < p.top_groups;
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < Q; i++) {
            const int e = (i * L + l) * 4;
            if (e >= p.E) continue;
            if (p.per4) {
                if (!gkeep[(e * p.magic) >> 20]) top[i] = -INFINITY;  // its keys are not looked at again
            } else {
                float4 v = *(const float4*)(keys + e);
                if (!gkeep[(e * p.magic) >> 20]) v.x = -INFINITY;
                if (e + 1 < p.E && !gkeep[((e + 1) * p.magic) >> 20]) v.y = -INFINITY;
                if (e + 2 < p.E && !gkeep[((e + 2) * p.magic) >> 20]) v.z = -INFINITY;
                if (e + 3 < p.E && !gkeep[((e + 3) * p.magic) >> 20]) v.w = -INFINITY;
                *(float4*)(keys + e) = v;
                top[i] = fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w));
            }
        }
    }
    __syncwarp();
    for (int k = 0; k < p.K; k++) {
        float tree[Q];  // the first of the largest, pair by pair
        int of[Q];
#pragma unroll
        for (int i = 0; i < Q; i++) tree[i] = top[i], of[i] = i;
#pragma unroll
        for (int step = 1; step < Q; step *= 2)
#pragma unroll
            for (int i = 0; i + step < Q; i += 2 * step)
                if (tree[i + step] > tree[i]) tree[i] = tree[i + step], of[i] = of[i + step];
        const int at = of[0], mine = at * L + l;
        // Each lane looks at its own best quad while the lanes find out whose it is.
        float* c = keys + min(mine * 4, stride - 4);
        const float4 v = *(const float4*)c;
        float win = tree[0];
        const int j = v.x == win ? 0 : v.y == win ? 1 : v.z == win ? 2 : 3;
        const float next = fmaxf(fmaxf(j == 0 ? -INFINITY : v.x, j == 1 ? -INFINITY : v.y), fmaxf(j == 2 ? -INFINITY : v.z, j == 3 ? -INFINITY : v.w));
        int quad = mine;
        lanes_best<L>(win, quad);
        const bool none = !(win > -INFINITY) || bad, owner = quad == mine && !none;  // NaN is none too: every place gets an id that some lane found
        if (owner) {
            chosen[k] = quad * 4 + j;
            c[j] = -INFINITY;
        }
        if (none && l == 0) chosen[k] = -1;
#pragma unroll
        for (int i = 0; i < Q; i++) top[i] = owner && at == i ? next : top[i];
    }
    __syncwarp();
    constexpr int R = 32 / L;  // at most 32 choices over L lanes
    float s[R], sum = 0.f;
    int id[R];
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int k = r * L + l;
        id[r] = k < p.K ? chosen[k] : -1;
        float v = p.sigmoid ? -INFINITY : m;
        if (id[r] >= 0) v = to_f32<T>(row[id[r]]);
        s[r] = p.sigmoid ? 1.f / (1.f + expf(-v)) : expf(v - m);  // softmax: the common divisor drops out of renormalised weights
        s[r] = id[r] >= 0 ? s[r] : 0.f;
        sum += s[r];
        if (r * L + L >= p.K) {
#pragma unroll
            for (int q = 0; q < R; q++)
                if (q > r) id[q] = -1, s[q] = 0.f;
            break;
        }
    }
    if (!p.sigmoid && p.renorm && p.bias) {
        // A bias may choose scores that are 0 against the row's largest: over the largest chosen one, as the gradient does. (Without a bias that is the row's, or, with groups, close to it.)
        float base = -INFINITY;
#pragma unroll
        for (int r = 0; r < R; r++)
            if (id[r] >= 0) base = fmaxf(base, to_f32<T>(row[id[r]]));
        base = lanes_max<L>(base);
        sum = 0.f;
#pragma unroll
        for (int r = 0; r < R; r++) {
            s[r] = id[r] >= 0 ? expf(to_f32<T>(row[id[r]]) - base) : 0.f;
            sum += s[r];
        }
    }
    const float div = p.renorm ? lanes_sum<L>(sum) : total;
    if (in) {
#pragma unroll
        for (int r = 0; r < R; r++) {
            const int k = r * L + l;
            if (k >= p.K) break;
            p.ids[t * p.K + k] = id[r];
            if (kept) kept[t * p.K + k] = id[r];
            p.weights[t * p.K + k] = (live && bad) ? __int_as_float(NOT_A_NUMBER) : (id[r] >= 0 && div > 0.f) ? s[r] / div * p.scale : 0.f;
            if (id[r] >= 0) atomicAdd(&hist[id[r]], 1);
        }
    }
    __syncwarp();
}

// Rows of the choices [first, first + n), whose experts are ids[0 .. n). base[e] (shared) = first row of expert e for them; rows follow in the order of the choices.
// Each warp takes a run of them; a first walk counts by expert, a second hands out the rows with match_any, so that the
// order does not depend on which warp is faster. cnt: shared, [warps][E], of at most 16 warps.
__device__ __forceinline__ void layout_choices(const RouteParams& p, const int* ids, long long first, int n, const int* base, int* cnt, int threads) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = threads / 32;
    const int per = round_up((n + warps - 1) / warps, 32);
    const int lo = min(warp * per, n), hi = min(lo + per, n);
    int* mine = cnt + warp * p.E;
    for (int e = lane; e < p.E; e += 32) mine[e] = 0;
    constexpr int HELD = 4;  // a run's first 128 choices stay in registers between the walks
    int id[HELD];
#pragma unroll
    for (int u = 0; u < HELD; u++) {
        const int i = lo + u * 32 + lane;
        id[u] = i < hi ? ids[i] : -1;
    }
    __syncwarp();
#pragma unroll
    for (int u = 0; u < HELD; u++)
        if (id[u] >= 0) atomicAdd(&mine[id[u]], 1);
    for (int i = lo + HELD * 32 + lane; i < hi; i += 32) {
        const int e = ids[i];
        if (e >= 0) atomicAdd(&mine[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.E; e += threads) {  // counts become first rows
        int at = base[e], c[16];
#pragma unroll
        for (int w = 0; w < 16; w++) c[w] = w < warps ? cnt[w * p.E + e] : 0;
#pragma unroll
        for (int w = 0; w < 16; w++) {
            if (w < warps) cnt[w * p.E + e] = at;
            at += c[w];
        }
    }
    __syncthreads();
    const auto place = [&](int i, int e) {
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
    };
#pragma unroll
    for (int u = 0; u < HELD; u++)
        if (lo + u * 32 < hi) place(lo + u * 32 + lane, id[u]);
    for (int b = lo + HELD * 32; b < hi; b += 32) place(b + lane, b + lane < hi ? ids[b + lane] : -1);
}

// Offsets of all experts from their totals tot[E] (shared); each expert's first row is added to base[e]. Returns the number of rows. A warp scans 32 experts,
// the warps' sums are added up by each; scratch: shared, 33 ints.
__device__ __forceinline__ int offsets_of(const RouteParams& p, const int* tot, int* base, int* scratch, bool write, int threads) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = threads / 32, parts = (p.E + 31) / 32;  // at most 32 parts
    for (int part = warp; part < parts; part += warps) {
        const int e = part * 32 + lane;
        const int sum = __reduce_add_sync(FULL, e < p.E ? tot[e] : 0);
        if (lane == 0) scratch[part] = sum;
    }
    __syncthreads();
    int used = 0;
    for (int part = warp; part < parts || part == warp; part += warps) {
        const int sums = lane < parts ? scratch[lane] : 0;
        used = __reduce_add_sync(FULL, sums);
        if (part >= parts) break;
        const int before = __reduce_add_sync(FULL, lane < part ? sums : 0);
        const int e = part * 32 + lane, c = e < p.E ? tot[e] : 0;
        int inc = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(FULL, inc, o);
            if (lane >= o) inc += v;
        }
        const int start = before + inc - c;
        if (e < p.E) {
            base[e] += start;
            if (write) {
                p.offsets[e] = start;
                p.counts[e] = c;
            }
        }
    }
    if (write && threadIdx.x == 0) p.offsets[p.E] = used;
    __syncthreads();
    return used;
}

// Four blocks to an SM (64 registers, a few of them spilled): the 512 blocks of 16384 tokens are on their way at once. With three, 444 are, and the rest wait for
// a whole chain of latencies (24.9 us against 22.6, when that was measured).
// A block chooses for one chunk of tokens and leaves its counts for the layout; a single block (ONE) goes on to the layout itself.
template <typename T, int Q, int L, bool ONE>
__global__ void __launch_bounds__(32 * (ONE ? ONE_BLOCK_WARPS : MANY_WARPS), ONE ? 1 : 4) hccl_route_choose(const __grid_constant__ RouteParams p) {
    extern __shared__ __align__(16) int sm[];  // hist[E16] bias[E16], a single block's ids, then the tokens' keys; a single block: its layout's counts in their place
    __shared__ int scratch[32];
    const int E16 = round_up(p.E, 16), threads = 32 * p.warps, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    int* hist = sm;
    float* sbias = (float*)(sm + E16);
    int* kept = ONE ? (int*)(sbias + E16) : nullptr;
    float* keys = sbias + E16 + (ONE ? round_up((int)p.tokens * p.K, 4) : 0);
    asm volatile("griddepcontrol.launch_dependents;");
    bool strange = false;
    for (int e = threadIdx.x; e < E16; e += threads) {
        hist[e] = 0;
        if (p.bias) {
            const float b = e < p.E ? p.bias[e] : 0.f;
            sbias[e] = b;
            strange |= !(fabsf(b) < INFINITY);
        }
    }
    const bool odd = __syncthreads_or(strange);
    const long long t0 = (long long)blockIdx.x * p.chunk, t1 = min(t0 + p.chunk, p.tokens);
    const int sub = lane / L, per = 32 / L;
    float* mine = keys + (warp * per + sub) * token_floats(p);
    for (long long t = t0 + warp * per; t < t1; t += p.warps * per) choose_token<T, Q, L>(p, t + sub, t + sub < t1, mine, sbias, odd, hist, kept);
    __syncthreads();
    if constexpr (!ONE) {
        for (int e = threadIdx.x; e < E16; e += threads) p.hist[(size_t)blockIdx.x * E16 + e] = (uint8_t)hist[e];
        return;
    }
    int *base = (int*)sbias, *cnt = (int*)keys;
    for (int e = threadIdx.x; e < p.E; e += threads) base[e] = 0;
    __syncthreads();
    const int used = offsets_of(p, hist, base, scratch, true, threads);
    const int n = (int)(p.tokens * p.K);
    if (n <= 32) {  // a lane for each choice: its row is the first of its expert's and as many further as choices of the same expert come before
        if (warp == 0) {
            const int e = lane < n ? kept[lane] : -1;
            const unsigned same = __match_any_sync(FULL, e);
            const int row = e < 0 ? -1 : base[e] + __popc(same & ((1u << lane) - 1));
            if (lane < n) {
                p.slots[lane] = row;
                if (row >= 0) p.source[row] = lane;
            }
        }
    } else {
        layout_choices(p, kept, 0, n, base, cnt, threads);
    }
    for (int i = used + (int)threadIdx.x; i < n; i += threads) p.source[i] = -1;
}

// Adds 16 counters of 8 bits to 16 sums of 16 bits: bytes 0 and 2 of word w to sum[2w], bytes 1 and 3 to sum[2w + 1].
__device__ __forceinline__ void add_bytes(uint4 v, unsigned (&sum)[8]) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        sum[2 * i] += w[i] & 0x00ff00ffu;
        sum[2 * i + 1] += (w[i] >> 8) & 0x00ff00ffu;
    }
}
// Each block lays out the choices of a run of chunks. How many rows of each expert lie before them, and in all, it adds up itself from the
// chunks' counts: 8 bits each (a chunk has at most 255 tokens, a token chooses an expert once), read 16 at a time and summed in 16 bits by a thread, in 32 bits over the threads.
__global__ void __launch_bounds__(LAYOUT_THREADS) hccl_route_layout(const __grid_constant__ RouteParams p) {
    extern __shared__ __align__(16) int sm[];  // tot[E16], base[E16], then sums[2][lines][E16 / 2] or, after them, cnt[warps][E]
    __shared__ int scratch[32];
    const int E16 = round_up(p.E, 16), columns = E16 / 16, lines = layout_lines(p.E);
    int *tot = sm, *base = sm + E16, *cnt = base + E16;
    unsigned* sums = (unsigned*)cnt;
    const int c0 = (int)((long long)p.chunks * blockIdx.x / gridDim.x), c1 = (int)((long long)p.chunks * (blockIdx.x + 1) / gridDim.x);
    const int col = (int)threadIdx.x % columns, line = (int)threadIdx.x / columns;
    for (int e = threadIdx.x; e < 2 * E16; e += LAYOUT_THREADS) tot[e] = 0;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint4* h = (const uint4*)p.hist + col;
    const int per_line = (p.chunks + lines - 1) / lines;  // a line adds up a run of chunks, 256 of them at a time: 257 bytes of 255 fill 16 bits
    for (int from = 0; from < per_line; from += 256) {
        unsigned below[8] = {}, rest[8] = {};
        if (line < lines) {
            const auto add_up = [&](int c, int end, unsigned (&sum)[8]) {
                for (; c < end; c += 8) {
                    uint4 v[8];
#pragma unroll
                    for (int u = 0; u < 8; u++) v[u] = c + u < end ? h[(size_t)(c + u) * columns] : make_uint4(0, 0, 0, 0);
                    if (p.chunk <= 63) {  // four of them still fit 8 bits
#pragma unroll
                        for (int u = 0; u < 8; u += 4)
                            add_bytes(make_uint4(v[u].x + v[u + 1].x + v[u + 2].x + v[u + 3].x, v[u].y + v[u + 1].y + v[u + 2].y + v[u + 3].y,
                                                 v[u].z + v[u + 1].z + v[u + 2].z + v[u + 3].z, v[u].w + v[u + 1].w + v[u + 2].w + v[u + 3].w), sum);
                    } else {
#pragma unroll
                        for (int u = 0; u < 8; u++) add_bytes(v[u], sum);
                    }
                }
            };
            const int lo = line * per_line + from, hi = min(min(lo + 256, (line + 1) * per_line), p.chunks);
            add_up(lo, min(hi, c0), below);
            add_up(max(lo, c0), hi, rest);
        }
        __syncthreads();
        if (line < lines) {
            uint4 *a = (uint4*)(sums + line * (E16 / 2) + col * 8), *b = (uint4*)(sums + (lines + line) * (E16 / 2) + col * 8);
            a[0] = make_uint4(below[0], below[1], below[2], below[3]);
            a[1] = make_uint4(below[4], below[5], below[6], below[7]);
            b[0] = make_uint4(rest[0], rest[1], rest[2], rest[3]);
            b[1] = make_uint4(rest[4], rest[5], rest[6], rest[7]);
        }
        __syncthreads();
        // word w of the sums before, or of the rest: two experts; the lines in `parts` shares
        const int parts = max(1, LAYOUT_THREADS / E16);
        for (int i = threadIdx.x; i < E16 * parts; i += LAYOUT_THREADS) {
            const int part = i / E16, at = i % E16;
            const bool before = at < E16 / 2;
            const int w = before ? at : at - E16 / 2, e = w / 8 * 16 + (w % 8) / 2 * 4 + (w & 1);
            const unsigned* from_lines = sums + (before ? 0 : lines * (E16 / 2)) + w;
            int lo = 0, hi = 0;
#pragma unroll 8
            for (int l = part; l < lines; l += parts) {
                const unsigned v = from_lines[l * (E16 / 2)];
                lo += v & 0xffffu;
                hi += v >> 16;
            }
            if (lo) atomicAdd(&tot[e], lo);
            if (hi) atomicAdd(&tot[e + 2], hi);
            if (before && lo) atomicAdd(&base[e], lo);
            if (before && hi) atomicAdd(&base[e + 2], hi);
        }
        __syncthreads();
    }
    const int used = offsets_of(p, tot, base, scratch, blockIdx.x == 0, LAYOUT_THREADS);
    const long long t0 = (long long)c0 * p.chunk, t1 = min((long long)c1 * p.chunk, p.tokens);
    if (t0 < t1) layout_choices(p, p.ids + t0 * p.K, t0 * p.K, (int)((t1 - t0) * p.K), base, cnt, LAYOUT_THREADS);
    const long long n = p.tokens * p.K;  // rows that belong to no choice
    for (long long i = used + (long long)blockIdx.x * LAYOUT_THREADS + threadIdx.x; i < n; i += (long long)gridDim.x * LAYOUT_THREADS) p.source[i] = -1;
}

// d of the logits. Weight j of the chosen has w_j = scale * s_j / S (S = sum of the chosen scores if renormalised, else 1), so
// ds_j = scale / S * (dw_j - sum_i dw_i s_i / S) or scale * dw_j; then the score's own derivative (with s_j / S formed first, which is a weight):
// sigmoid dl = ds s (1 - s), softmax dl_e = s_e (ds_e - sum_j ds_j s_j) over all experts. Where the weights are renormalised (the softmax's
// divisor drops out, and with it sum_j ds_j s_j = 0) or the scores are sigmoids, only the chosen have a gradient: their logits alone
// are read, and the row is zeros with k places filled, put together in shared memory. Memory is the bound.
template <typename T, int L>
__global__ void __launch_bounds__(256) hccl_route_grad(const __grid_constant__ RouteGradParams q) {
    const RouteParams& p = q.r;
    extern __shared__ __align__(16) char smem[];  // a row of T for each token of the block, rounded up to 16 bytes
    constexpr int R = 32 / L, V = 16 / sizeof(T);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, l = lane % L, per = 32 / L;
    const int row_elems = round_up(p.E, V);
    T* buf = (T*)smem + (size_t)(warp * per + lane / L) * row_elems;
    const bool whole_row = !p.sigmoid && !p.renorm;
    for (long long t0 = (long long)blockIdx.x * 8 * per; t0 < p.tokens; t0 += (long long)gridDim.x * 8 * per) {
        const long long t = t0 + warp * per + lane / L;
        const bool in = t < p.tokens, live = in && (!p.mask || p.mask[t]);
        const T* row = (const T*)p.logits + (in ? t : 0) * p.ld;
        int id[R];
        float dw[R], x[R], c[R];
        bool some = false;
#pragma unroll
        for (int r = 0; r < R; r++) {
            const int k = r * L + l;
            id[r] = -1, dw[r] = 0.f, x[r] = -INFINITY;
            if (live && k < p.K) {
                id[r] = p.ids[t * p.K + k];
                if (id[r] >= p.E) id[r] = -1;
                if (id[r] >= 0) {
                    dw[r] = q.dweights[t * p.K + k] * p.scale;
                    x[r] = to_f32<T>(row[id[r]]);
                    some = true;
                }
            }
        }
        some = lanes_any<L>(some);
        // what the row is filled with, where it is not one of the chosen
        float m = -INFINITY, total = 1.f, dot = 0.f, fill = 0.f;
        const bool walk = whole_row || !__all_sync(FULL, some || !live);  // a live token that chose nothing: were its scores numbers?
        bool bad = false;
        if (walk) {
            for (int e = l; e < p.E && live; e += L) {
                float v = to_f32<T>(row[e]);
                const float b = p.bias ? p.bias[e] : 0.f;
                if (b == -INFINITY) v = -INFINITY;
                bad |= isnan(v) || (v != -INFINITY && !(b < INFINITY));
                m = fmaxf(m, v);
            }
            m = lanes_max<L>(m);
            bad |= live && !p.sigmoid && m == INFINITY;
            bad = lanes_any<L>(bad);
            if (bad) fill = __int_as_float(NOT_A_NUMBER);
            if (whole_row) {
                float sum = 0.f;
                for (int e = l; e < p.E && live; e += L)
                    if (m != -INFINITY && !(p.bias && p.bias[e] == -INFINITY)) sum += expf(to_f32<T>(row[e]) - m);
                total = lanes_sum<L>(sum);
            }
        }
        if (!whole_row && !p.sigmoid) {
            m = -INFINITY;
#pragma unroll
            for (int r = 0; r < R; r++) m = fmaxf(m, x[r]);
            m = lanes_max<L>(m);
        }
        float sc = 0.f, sdc = 0.f;
#pragma unroll
        for (int r = 0; r < R; r++) {
            c[r] = id[r] < 0 ? 0.f : p.sigmoid ? 1.f / (1.f + expf(-x[r])) : expf(x[r] - m);
            sc += c[r];
            sdc += dw[r] * c[r];
        }
        if (p.renorm) {
            // By the weights c / S: (dw - sum dw c / S) / S would leave the range for sigmoids near 0, times c it is of the size of dw.
            const float S = lanes_sum<L>(sc), D = lanes_sum<L>(sdc), r1 = S > 0.f ? 1.f / S : 0.f;
#pragma unroll
            for (int r = 0; r < R; r++) dw[r] = (dw[r] - D * r1) * (c[r] * r1);
        } else if (whole_row) {
            const float r1 = total > 0.f ? 1.f / total : 0.f;
            dot = lanes_sum<L>(sdc) * r1;
            total = r1;
        }
        // the row
        if (!whole_row || bad) {
            for (int e = l; e < row_elems; e += L) buf[e] = from_f32<T>(fill);
        } else {
            for (int e = l; e < p.E && live; e += L) {
                const bool off = m == -INFINITY || (p.bias && p.bias[e] == -INFINITY);
                buf[e] = from_f32<T>(off ? 0.f : -expf(to_f32<T>(row[e]) - m) * total * dot);
            }
            if (!live)
                for (int e = l; e < row_elems; e += L) buf[e] = from_f32<T>(0.f);
        }
        __syncwarp();
#pragma unroll
        for (int r = 0; r < R; r++)
            if (id[r] >= 0 && !bad) buf[id[r]] = from_f32<T>(p.renorm ? (p.sigmoid ? dw[r] * (1.f - c[r]) : dw[r]) : p.sigmoid ? dw[r] * c[r] * (1.f - c[r]) : c[r] * total * (dw[r] - dot));
        __syncwarp();
        if (in) {
            T* out = (T*)q.dlogits + t * q.ldd;
            if (q.vec) {
                for (int v = l; v < p.E / V; v += L) ((uint4*)out)[v] = ((const uint4*)buf)[v];
            } else {
                for (int e = l; e < p.E; e += L) out[e] = buf[e];
            }
        }
        __syncwarp();
    }
}

// ---------------------------------------------------------------- host
// Lanes for a token. 8 do the least work in all (16384 x 256: 25 us against 36 with 32; 32 x 64: 4.5 against 5.8), 32 have the shorter chain of latencies where keys are many for each lane and
// tokens do not fill the SMs (1024 x 256: 10.0 us against 11.7, 64 x 256: 8.9 against 10.2, one token of 64: 3.7 against 4.2); beyond 256 experts 8 lanes would hold more than 8 quads each.
int lanes_for(long long tokens, int E) { return (tokens <= ONE_BLOCK_WARPS || E > 256 || (E > 128 && tokens <= 1024)) ? 32 : 8; }
bool one_block(long long tokens, int lanes) { return tokens <= ONE_BLOCK_WARPS * (32 / lanes) * 2; }

struct Cut {
    int lanes, warps, chunk, chunks;
};
Cut cut(long long tokens, int E) {
    Cut c;
    c.lanes = lanes_for(tokens, E);
    const int per = 32 / c.lanes;
    if (one_block(tokens, c.lanes)) {
        c.warps = (int)std::min<long long>(ONE_BLOCK_WARPS, std::max<long long>(4, (tokens + per - 1) / per));
        c.chunk = (int)tokens;
        c.chunks = 1;
        return c;
    }
    c.warps = MANY_WARPS;
    const int round = MANY_WARPS * per;  // tokens a block chooses for at once: 32 or 8
    long long want = (tokens + 16 * SMS - 1) / (16 * SMS);
    want = (want + round - 1) / round * round;
    c.chunk = (int)std::min<long long>(std::max<long long>(want, round), 255 / round * round);
    c.chunks = (int)((tokens + c.chunk - 1) / c.chunk);
    return c;
}

// Opt-in to large shared memory, once for each kernel and device. The most that a launch here asks for: one block for 32 tokens of 1024 experts in 1024 groups, top 32.
constexpr int MOST_SMEM = 4 * (2 * HCCL_MAX_EXPERTS + ONE_BLOCK_WARPS * (HCCL_MAX_EXPERTS + 8 + 2 * HCCL_MAX_EXPERTS + HCCL_MAX_TOP_K) + 2 * ONE_BLOCK_WARPS * HCCL_MAX_TOP_K);
static_assert(MOST_SMEM + 1024 <= 227 * 1024, "beyond a block's shared memory");
template <typename K> cudaError_t allow(K* kernel, size_t bytes, std::atomic<bool> (&ready)[64]) {
    if (bytes <= 48 * 1024) return cudaSuccess;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < 64 && ready[dev])) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST_SMEM);
    if (e == cudaSuccess && dev < 64) ready[dev] = true;
    return e;
}

template <typename T, int Q, int L, bool ONE> cudaError_t choose_launch(const RouteParams& p, cudaStream_t s) {
    size_t ints = (size_t)p.warps * (32 / L) * token_floats(p);
    if (ONE) ints = std::max(ints, (size_t)p.warps * p.E) + round_up((int)p.tokens * p.K, 4);
    const size_t smem = (2 * round_up(p.E, 16) + ints) * 4;
    static std::atomic<bool> ready[64];
    const cudaError_t e = allow(hccl_route_choose<T, Q, L, ONE>, smem, ready);
    if (e != cudaSuccess) return e;
    hccl_route_choose<T, Q, L, ONE><<<p.chunks, 32 * p.warps, smem, s>>>(p);
    return cudaGetLastError();
}

template <typename T, int Q, int L> cudaError_t route_launch(const RouteParams& p, cudaStream_t s) {
    const int E16 = round_up(p.E, 16);
    if (p.chunks == 1) return choose_launch<T, Q, L, true>(p, s);
    cudaError_t e = choose_launch<T, Q, L, false>(p, s);
    if (e != cudaSuccess) return e;
    static std::atomic<bool> ready2[64];
    cudaLaunchConfig_t cfg = {};
    cfg.dynamicSmemBytes = (size_t)(2 * E16 + std::max(LAYOUT_THREADS / 32 * p.E, layout_lines(p.E) * E16)) * 4;
    if ((e = allow(hccl_route_layout, cfg.dynamicSmemBytes, ready2)) != cudaSuccess) return e;
    cfg.gridDim = dim3((unsigned)std::min(p.chunks, SMS));
    cfg.blockDim = dim3(LAYOUT_THREADS);
    cfg.stream = s;
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, hccl_route_layout, p);
}

template <typename T> cudaError_t route_sizes(const RouteParams& p, int lanes, cudaStream_t s) {
    if (lanes == 8) {
        if (p.E <= 32) return route_launch<T, 1, 8>(p, s);
        if (p.E <= 64) return route_launch<T, 2, 8>(p, s);
        if (p.E <= 128) return route_launch<T, 4, 8>(p, s);
        return route_launch<T, 8, 8>(p, s);
    }
    if (p.E <= 128) return route_launch<T, 1, 32>(p, s);
    if (p.E <= 256) return route_launch<T, 2, 32>(p, s);
    if (p.E <= 512) return route_launch<T, 4, 32>(p, s);
    return route_launch<T, 8, 32>(p, s);
}

template <typename T, int L> cudaError_t grad_launch(const RouteGradParams& p, cudaStream_t s) {
    const int per_block = 8 * (32 / L);
    const size_t smem = (size_t)per_block * round_up(p.r.E, 16 / sizeof(T)) * sizeof(T);
    const long long blocks = (p.r.tokens + per_block - 1) / per_block;
    hccl_route_grad<T, L><<<(int)std::min<long long>(blocks, SMS * 8), 256, smem, s>>>(p);
    return cudaGetLastError();
}
template <typename T> cudaError_t grad_sizes(const RouteGradParams& p, cudaStream_t s) {
    return p.r.E <= 256 ? grad_launch<T, 8>(p, s) : grad_launch<T, 32>(p, s);
}

bool aligned_rows(const void* at, long long ld, int es, int bytes) { return (uintptr_t)at % bytes == 0 && (ld * es) % bytes == 0; }

}  // namespace

size_t route_workspace(int E, long long tokens) {
    const Cut c = cut(tokens, E);
    return c.chunks > 1 ? (size_t)c.chunks * round_up(E, 16) : HCCL_ROUTE_NO_WORKSPACE;  // (more than one chunk: more than that)
}

cudaError_t launch_route(int dt, const RouteParams& in, cudaStream_t s) {
    RouteParams p = in;
    const Cut c = cut(p.tokens, p.E);
    p.warps = c.warps;
    p.chunk = c.chunk;
    p.chunks = c.chunks;
    p.per4 = p.per_group % 4 == 0;
    p.magic = ((1 << 20) + p.per_group - 1) / p.per_group;
    const int es = dt == HCCL_FP32 ? 4 : 2;
    const int quads = p.per_group / 4;
    // (Sums of two scores without a bias are formed in the other walk alone: once in the code instead of once for each quad of a lane, which a single token would wait for.)
    const bool sums_of_scores = p.group_best == 2 && !p.bias;
    p.segment = p.per4 && quads <= c.lanes && (quads & (quads - 1)) == 0 && !sums_of_scores ? quads : 0;
    p.vec = aligned_rows(p.logits, p.ld, es, 4 * es) && p.E % 4 == 0;
    if (dt == HCCL_FP32) return route_sizes<float>(p, c.lanes, s);
    if (dt == HCCL_BF16) return route_sizes<__nv_bfloat16>(p, c.lanes, s);
    return route_sizes<__half>(p, c.lanes, s);
}

cudaError_t launch_route_grad(int dt, const RouteGradParams& in, cudaStream_t s) {
    RouteGradParams p = in;
    if (p.r.tokens == 0) return cudaSuccess;
    const int es = dt == HCCL_FP32 ? 4 : 2;
    p.vec = aligned_rows(p.dlogits, p.ldd, es, 16) && (p.r.E * es) % 16 == 0;
    if (dt == HCCL_FP32) return grad_sizes<float>(p, s);
    if (dt == HCCL_BF16) return grad_sizes<__nv_bfloat16>(p, s);
    return grad_sizes<__half>(p, s);
}

}  // namespace experts
}  // namespace hccl
