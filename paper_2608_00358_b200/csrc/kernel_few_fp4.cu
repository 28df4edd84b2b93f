// A whole expert layer for a few tokens in two kernels: y[t] = sum over j of w[t, j] down_e(act(up_e(x[t]))), weights in 4-bit floating point, activations not rounded.
//
// With few tokens the chosen experts' weights are read once and that is the time, so 4-bit activations would save nothing and cost accuracy. The tensor cores multiply 4-bit
// numbers by 4-bit numbers all the same: an activation goes in as a sum of eight of them. Of a block x of a row, q0 = e2m1(x / s0) is taken, of what is left q1, and so on,
// each with a scale of its own; a step leaves at most a sixth (powers of two as scales: a quarter) of the block's maximum, so eight leave 6^-8 (4^-8). Eight columns is
// also the least that an instruction computes: a token's eight pieces are its eight columns, and for one token they cost nothing. The sum over the pieces
// is taken in 32 bits. With e4m3 scales each row's part of K is first multiplied by a power of two that brings its largest element to 1024 .. 2048, near 448 x 6, the top of their range; what
// four pieces leave is less than 2048 x 0.178^4 = 2.1 (a rounded scale leaves up to 17 / 96 of a block's maximum) and is multiplied by 2^10, so that the last four have the whole range
// again and the scales' smallest step, 2^-9, is 2^-30 of the row's largest element.
//
// Work: units of 128 channels x `span` stages of 256 elements of K x a chunk of at most 8 of an expert's rows, in the order [chunk][part of K][channels]; every block takes an equal run of
// them. Within a chunk and a part of K the pieces are made once and stay in shared memory while the weights stream past them. A unit's sums go to memory as 32-bit partial
// sums, one for each part of K; the second kernel adds the first's up in their order, applies the activation and splits the result. Who finishes the last
// unit of 128 output channels adds up all partial sums of these channels in their order: results repeat bit for bit.
//
// Roles of a block (16 warps): warp 0 loads weights, warp 1 copies scales to tensor memory and issues the products, warp 2 owns the tensor memory, warp 3 lists the chunks, warps 4-7 take
// the sums out, warps 8-15 make the pieces, one part of K ahead.
#include <algorithm>
#include <atomic>

#include "activate.cuh"
#include "fp4.cuh"
#include "tensor.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int THREADS = 512, CH = 128, ROWS = 8 /* of a chunk */, PIECES = 8, SPAN = 4 /* stages of K at most */, COLS = 512;
constexpr int TN = ROWS * PIECES;
constexpr float LATER = 1024.f;  // e4m3 scales: what the last half of the pieces is larger by
constexpr int ENOUGH = 6;  // units for each block, below which K is cut finer
constexpr int SPLIT_WARPS = 8, SPLITTERS = 32 * SPLIT_WARPS, EACH = 8 /* elements of a thread */, TASKS = ROWS * SPAN * 256 / EACH / SPLITTERS;

template <int FORMAT> struct Shape {
    static constexpr int ATOMS = stage_atoms(FORMAT);
    static constexpr int STAGE = CH * KB + ATOMS * ATOM;
    static constexpr int STAGES = 6;
    static constexpr int PIECE_STAGE = TN * KB, PIECE_SCALES = SPAN * PIECE_STAGE;  // of a part of K: its rows by stages, then their scales
    static constexpr int PART = PIECE_SCALES + SPAN * ATOMS * ATOM;
    static constexpr int RING = (STAGES * STAGE + 1023) / 1024 * 1024;
    static constexpr int SMEM = RING + 2 * PART + 1024;
    // tensor memory: two accumulators, two parts' scales, the stages' scales
    static constexpr int X_SCALES = 2 * TN, W_SCALES = X_SCALES + 2 * SPAN * 4 * ATOMS;
    static_assert(W_SCALES + STAGES * 4 * ATOMS <= COLS, "tensor memory");
    static_assert(STAGE % 1024 == 0 && PART % 1024 == 0, "operands start on 1024-byte boundaries");
};

struct FewParams {
    CUtensorMap w, w_scale;
    const void* x;     // up: [T, K] in T; down: the first kernel's partial sums
    void* y;           // up: partial sums; down: [T, H]
    float* part;       // down: its partial sums
    int* arrived;      // [channel tiles of down]
    long long ldx, ldy;
    const int *offsets, *source, *slots;
    const float *weights, *wide, *bias;
    int* status;
    int K, N, I, k_blocks, chan_tiles, x_blocks, x_tiles /* down: of the first kernel */;
    int experts, top_k, T, rows /* T * top_k */, act, gated, half /* width of a row of the first kernel's sums, of the gate's and of the other half */, wide_y;
    int down_tiles, vec;
};

// How many stages of K a unit has, so that there are enough units to share out evenly. (Both kernels and the scratch's size go by it.)
__host__ __device__ __forceinline__ int span_of(int chunks, int tiles, int k_blocks, int blocks) {
    int span = SPAN;
    while (span > 1 && (long long)chunks * tiles * ((k_blocks + span - 1) / span) < (long long)ENOUGH * blocks) span /= 2;
    return span;
}

template <int FORMAT> __device__ __forceinline__ void mma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
#define HCCL_MMA(kind) \
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n tcgen05.mma.cta_group::1.kind::" kind " [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"(sa), "r"(sb), "r"(accumulate) : "memory")
    if constexpr (FORMAT == HCCL_NVFP4) HCCL_MMA("mxf4nvf4.block_scale.scale_vec::4X");
    else HCCL_MMA("mxf4.block_scale.scale_vec::2X");
#undef HCCL_MMA
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t addr) {
    const uint64_t from = (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(from) : "memory");
}
__device__ __forceinline__ void tmem_load8(uint32_t addr, float (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                 : "r"(addr));
}

// Eight elements of a row, zeros from K on.
template <typename T> __device__ __forceinline__ void load8(const T* x, int k, int K, bool vec, float (&v)[EACH]) {
    constexpr int H = 16 / sizeof(T);
    if (vec && k + EACH <= K) {
#pragma unroll
        for (int u = 0; u < EACH / H; u++) {
            Pack<T, H> q;
            float f[H];
            q.raw = ((const uint4*)(x + k))[u];
            q.get(f);
#pragma unroll
            for (int j = 0; j < H; j++) v[u * H + j] = f[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < EACH; j++) v[j] = k + j < K ? to_f32<T>(x[k + j]) : 0.f;
    }
}

// Whether all of `count` threads that meet at a barrier say so: a wait that gave up in one warp is known to all before the next barrier.
__device__ __forceinline__ bool all_of(bool ok, int barrier, int count) {
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.and.pred q, %2, %3, p;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"((uint32_t)ok), "r"(barrier), "r"(count) : "memory");
    return r != 0;
}

// A step that serves for a piece: whatever it is, what it leaves is exact and goes to the next piece, so that divisions need not be rounded to nearest.
template <int FORMAT> __device__ __forceinline__ Step some_step(unsigned top) {
    if constexpr (FORMAT == HCCL_MXFP4) return step_of<FORMAT>(top, 1.f, 6.f);
    Step r;
    unsigned short two;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(0.f), "f"(__uint_as_float(top) * (1.f / 6.f)));
    unsigned halves;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(halves) : "h"(two));
    r.byte = top >= 0x7f800000u ? 0x7fu : two & 0xffu;
    r.d = __low2float(*(const __half2*)&halves);
    r.inv = r.byte ? __fdividef(1.f, r.d) : 0.f;
    return r;
}

struct Unit {
    int expert, row, rows;  // a chunk: rows [row, row + rows) in expert order
    int kc, tile;
};

template <typename T, int FORMAT, bool DOWN> __global__ void __launch_bounds__(THREADS, 1) hccl_few_fp4(const __grid_constant__ FewParams p) {
    using S = Shape<FORMAT>;
    extern __shared__ char dynamic[];
    __shared__ __align__(8) unsigned long long bars[2 * S::STAGES + 8];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up, last_one;
    __shared__ int before[HCCL_MAX_EXPERTS + 1];
    __shared__ float unscale[2][ROWS];
    __shared__ unsigned top_of[2][ROWS];
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_addr(dynamic) + 1023) & ~1023u;
    char* const parts = dynamic + (base - smem_addr(dynamic)) + S::RING;
    const uint32_t bar0 = smem_addr(bars);
    const auto full = [&](int s) { return bar0 + 8 * s; };
    const auto empty = [&](int s) { return bar0 + 8 * (S::STAGES + s); };
    const auto acc_full = [&](int b) { return bar0 + 8 * (2 * S::STAGES + b); };
    const auto acc_empty = [&](int b) { return bar0 + 8 * (2 * S::STAGES + 2 + b); };
    const auto part_full = [&](int b) { return bar0 + 8 * (2 * S::STAGES + 4 + b); };
    const auto part_empty = [&](int b) { return bar0 + 8 * (2 * S::STAGES + 6 + b); };

    if (!DOWN) asm volatile("griddepcontrol.launch_dependents;");  // its blocks may start to fetch weights as this one's leave
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; s++) mbar_init(full(s), 1), mbar_init(empty(s), 1);
        for (int b = 0; b < 2; b++) mbar_init(acc_full(b), 1), mbar_init(acc_empty(b), 4), mbar_init(part_full(b), SPLIT_WARPS), mbar_init(part_empty(b), 5);
        gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (!DOWN)  // for the second kernel
        for (int i = (int)(blockIdx.x * THREADS + threadIdx.x); i < p.down_tiles; i += (int)gridDim.x * THREADS) p.arrived[i] = 0;
    if (threadIdx.x < 2 * ROWS) top_of[threadIdx.x / ROWS][threadIdx.x % ROWS] = 0;
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_at)), "n"(COLS));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (warp == 3) {
        int run = 0;
        for (int b = 0; b < p.experts; b += 32) {
            const int g = b + lane;
            int n = 0;
            if (g < p.experts) n = max(0, (min(p.rows, p.offsets[g + 1]) - max(0, p.offsets[g]) + ROWS - 1) / ROWS);
            int inc = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += v;
            }
            if (g < p.experts) before[g] = run + inc - n;
            run += __shfl_sync(0xffffffffu, inc, 31);
        }
        if (lane == 0) before[p.experts] = run;
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_at, 0);
    const int chunks = __shfl_sync(0xffffffffu, before[p.experts], 0), blocks = (int)gridDim.x;
    const int span = span_of(chunks, p.chan_tiles, p.k_blocks, blocks), parts_of_k = (p.k_blocks + span - 1) / span;
    const long long units = (long long)chunks * parts_of_k * p.chan_tiles;
    const int u0 = (int)(units * blockIdx.x / blocks), u1 = (int)(units * (blockIdx.x + 1) / blocks);
    const int filled = min(p.rows, max(0, p.offsets[p.experts]));  // rows that have sums: how far apart the parts of K lie

    int hint = 0;
    const auto unit_of = [&](int u) {
        Unit r;
        const int chunk = u / (parts_of_k * p.chan_tiles), rest = u - chunk * parts_of_k * p.chan_tiles;
        while (chunk >= before[hint + 1]) hint++;
        const int lo = max(0, p.offsets[hint]), hi = min(p.rows, p.offsets[hint + 1]), row = lo + (chunk - before[hint]) * ROWS;
        r.expert = __shfl_sync(0xffffffffu, hint, 0);
        r.row = __shfl_sync(0xffffffffu, row, 0);
        r.rows = __shfl_sync(0xffffffffu, min(ROWS, hi - row), 0);
        r.kc = __shfl_sync(0xffffffffu, rest / p.chan_tiles, 0);
        r.tile = __shfl_sync(0xffffffffu, rest % p.chan_tiles, 0);
        return r;
    };
    const auto stages_of = [&](int kc) { return min(span, p.k_blocks - kc * span); };
    const auto ends = [&](int u) { return u == u1 - 1 || (u + 1) % p.chan_tiles == 0; };  // the last unit of its part of K here
    int it = 0, acc = 0, turn = 0;  // stages, units and parts of K passed

    if (warp == 0) {
        for (int u = u0; u < u1; u++) {
            const Unit t = unit_of(u);
            const int n = stages_of(t.kc);
            for (int i = 0; i < n; i++, it++) {
                const int s = it % S::STAGES, kb = t.kc * span + i;
                if (!mbar_wait(empty(s), ((it / S::STAGES) & 1) ^ 1, &gave_up)) break;
                if (elected()) {
                    const uint32_t at = base + s * S::STAGE;
                    mbar_expect(full(s), S::STAGE);
                    tma_load<1>(at, &p.w, kb * KB, t.expert * p.N + t.tile * CH, full(s));
                    tma_load<1>(at + CH * KB, &p.w_scale, 0, ((t.expert * p.chan_tiles + t.tile) * p.k_blocks + kb) * S::ATOMS, full(s));
                }
                __syncwarp();
            }
            if (*(volatile int*)&gave_up) break;
        }
    } else if (warp == 1) {
        const int steps = (p.K + 63) / 64;
        bool ok = true;
        for (int u = u0; u < u1 && ok; u++, acc++) {
            const Unit t = unit_of(u);
            const int n = stages_of(t.kc), b = acc & 1, half = turn & 1;
            const uint32_t x_scales = tmem + S::X_SCALES + half * SPAN * 4 * S::ATOMS, pieces = base + S::RING + half * S::PART;
            const uint32_t desc = (1u << 7) | (1u << 10) | ((uint32_t)t.rows << 17) | (FORMAT == HCCL_MXFP4 ? 1u << 23 : 0u) | (1u << 27);  // 128 channels, rows * 8 columns
            if (u == u0 || t.tile == 0) {
                ok = mbar_wait(part_full(half), (turn >> 1) & 1, &gave_up);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (elected())
                    for (int i = 0; i < n * S::ATOMS; i++) copy_scales(x_scales + 4 * i, pieces + S::PIECE_SCALES + i * ATOM);
                __syncwarp();
            }
            ok = mbar_wait(acc_empty(b), ((acc >> 1) & 1) ^ 1, &gave_up);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (int i = 0; i < n; i++, it++) {
                const int s = it % S::STAGES, left = min(4, steps - 4 * (t.kc * span + i));
                ok = mbar_wait(full(s), (it / S::STAGES) & 1, &gave_up);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t at = base + s * S::STAGE, scales = tmem + S::W_SCALES + s * 4 * S::ATOMS;
                const uint64_t w = operand(at), x = operand(pieces + i * S::PIECE_STAGE);
                if (elected()) {
#pragma unroll
                    for (int a = 0; a < S::ATOMS; a++) copy_scales(scales + 4 * a, at + CH * KB + a * ATOM);
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        if (k >= left) break;
                        const int a = k * S::ATOMS / 4;
                        const uint32_t two = FORMAT == HCCL_MXFP4 ? 2u * (k & 1) : 0u;
                        mma_fp4<FORMAT>(tmem + b * TN, w + 2 * k, x + 2 * k, desc | (two << 4) | (two << 29), scales + 4 * a, x_scales + 4 * (i * S::ATOMS + a), (i > 0 || k > 0) ? 1u : 0u);
                    }
                    mma_commit<1>(empty(s));
                    if (i == n - 1) {
                        mma_commit<1>(acc_full(b));
                        if (ends(u)) mma_commit<1>(part_empty(half));
                    }
                }
                __syncwarp();
            }
            if (ends(u)) turn++;
        }
    } else if (warp >= 4 && warp < 8) {
        const int quarter = warp & 3;
        if (DOWN) asm volatile("griddepcontrol.wait;" ::: "memory");
        bool ok = true;
        // Adds up what the experts of each token have for 128 channels.
        const auto combine = [&](int tile) {
            const int chan = tile * CH + quarter * 32 + lane;
            const bool in = chan < p.N;
            constexpr int BATCH = 16;
            float sum = 0.f;
            for (int q0 = 0; q0 < p.rows; q0 += BATCH) {
                const int mine = q0 + lane < p.rows && lane < BATCH ? p.slots[q0 + lane] : -1;
                const float weight = q0 + lane < p.rows && lane < BATCH ? p.weights[q0 + lane] : 0.f;
                float z[BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; i++) z[i] = 0.f;
                for (int kc = 0; kc < parts_of_k; kc++) {
#pragma unroll
                    for (int i = 0; i < BATCH; i++) {
                        const int slot = __shfl_sync(0xffffffffu, mine, i);
                        if (in && slot >= 0 && slot < filled) z[i] += __ldcg(p.part + ((long long)kc * filled + slot) * p.wide_y + chan);
                    }
                }
#pragma unroll
                for (int i = 0; i < BATCH; i++) {
                    const int q = q0 + i, slot = __shfl_sync(0xffffffffu, mine, i);
                    const float f = __shfl_sync(0xffffffffu, weight, i);
                    if (q < p.rows) {
                        if (slot >= 0 && slot < filled) sum = fmaf(f, z[i], sum);
                        if ((q + 1) % p.top_k == 0) {
                            if (in) ((T*)p.y)[(long long)(q / p.top_k) * p.ldy + chan] = from_f32<T>(sum);
                            sum = 0.f;
                        }
                    }
                }
            }
        };
        if (DOWN && units == 0)
            for (int tile = blockIdx.x; tile < p.chan_tiles; tile += blocks) combine(tile);  // nobody has anything: zeros
        for (int u = u0; u < u1 && ok; u++, acc++) {
            const Unit t = unit_of(u);
            const int b = acc & 1, half = turn & 1, chan = t.tile * CH + quarter * 32 + lane;
            const bool in = chan < p.N;
            const float wide = p.wide[t.expert], bias = (in && p.bias && t.kc == 0) ? p.bias[(long long)t.expert * p.N + chan] : 0.f;
            ok = mbar_wait(part_full(half), (turn >> 1) & 1, &gave_up) && mbar_wait(acc_full(b), (acc >> 1) & 1, &gave_up);
            if (DOWN) ok = all_of(ok, 1, 128);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            float sums[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; r++) {
                if (r >= t.rows) break;
                float v[8];
                __syncwarp();
                tmem_load8(tmem + ((uint32_t)(quarter * 32) << 16) + b * TN + r * PIECES, v);
                tmem_arrived();
                float s = ((v[7] + v[6]) + v[5]) + v[4];  // the smallest first
                if (FORMAT == HCCL_NVFP4) s *= 1.f / LATER;
#pragma unroll
                for (int i = 3; i >= 0; i--) s += v[i];
                sums[r] = fmaf(s, unscale[half][r] * wide, bias);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(acc_empty(b));
                if (ends(u)) mbar_arrive(part_empty(half));
            }
            if (ends(u)) turn++;
            float* out = DOWN ? p.part : (float*)p.y;
            const int width = DOWN ? p.wide_y : (p.gated ? 2 : 1) * p.half, at = !DOWN && p.gated && chan >= p.I ? p.half + chan - p.I : chan;
            out += ((long long)t.kc * filled + t.row) * width + at;
            if (in)
#pragma unroll
                for (int r = 0; r < ROWS; r++)
                    if (r < t.rows) __stcg(out + (long long)r * width, sums[r]);
            if (DOWN) {
                // All four warps' sums are out before the unit is counted; who counts the last one sees the others'.
                __threadfence();
                asm volatile("bar.sync 1, 128;" ::: "memory");
                if (threadIdx.x == 128) {
                    const int n = chunks * parts_of_k;
                    last_one = atomicAdd(p.arrived + t.tile, 1) == n - 1;
                    __threadfence();
                }
                asm volatile("bar.sync 1, 128;" ::: "memory");
                if (last_one) combine(t.tile);
            }
        }
    } else if (warp >= 8) {
        const int me = (int)threadIdx.x - 256;
        if (DOWN) asm volatile("griddepcontrol.wait;" ::: "memory");
        const int x_span = DOWN ? span_of(chunks, p.x_tiles, p.x_blocks, blocks) : 0, x_parts = DOWN ? (p.x_blocks + x_span - 1) / x_span : 0;
        bool ok = true;
        for (int u = u0; u < u1 && ok; u = (u / p.chan_tiles + 1) * p.chan_tiles, turn++) {
            const Unit t = unit_of(u);
            const int half = turn & 1, k0 = t.kc * span * 256, wide = stages_of(t.kc) * 256 / EACH;  // threads to a row
            char* const part = parts + half * S::PART;
            // A thread's elements: those of task i of (row, eight elements), i = me, me + 256, ...
            float v[TASKS][EACH];
            const auto row_of = [&](int i) { return (me + i * SPLITTERS) / wide; };
            const auto k_of = [&](int i) { return k0 + (me + i * SPLITTERS) % wide * EACH; };
#pragma unroll
            for (int i = 0; i < TASKS; i++) {
                const int r = row_of(i), k = k_of(i);
                if (r >= t.rows) break;
                if constexpr (!DOWN) {
                    const int from = p.source[t.row + r];
                    load8<T>((const T*)p.x + (long long)(from / p.top_k) * p.ldx, k, (unsigned)from < (unsigned)p.rows ? p.K : 0, p.vec, v[i]);
                } else {
                    const int width = (p.gated ? 2 : 1) * p.half;
                    const float* from = (const float*)p.x + (long long)(t.row + r) * width;
                    float g[EACH] = {}, o[EACH] = {};
                    if (k < p.K)
                        for (int c = 0; c < x_parts; c++, from += (long long)filled * width) {
#pragma unroll
                            for (int j = 0; j < EACH; j += 4) {
                                const float4 a = __ldcg((const float4*)(from + k + j));
                                g[j] += a.x, g[j + 1] += a.y, g[j + 2] += a.z, g[j + 3] += a.w;
                                if (p.gated) {
                                    const float4 q = __ldcg((const float4*)(from + p.half + k + j));
                                    o[j] += q.x, o[j + 1] += q.y, o[j + 2] += q.z, o[j + 3] += q.w;
                                }
                            }
                        }
#pragma unroll
                    for (int j = 0; j < EACH; j++) v[i][j] = k + j < p.K ? (p.gated ? activation(p.act, g[j]) * o[j] : activation(p.act, g[j])) : 0.f;
                }
            }
            // (the buffers' last readers)
            ok = mbar_wait(part_empty(half), ((turn >> 1) & 1) ^ 1, &gave_up);
            if (FORMAT == HCCL_NVFP4) ok = all_of(ok, 2, SPLITTERS);
            if (!ok) break;
            // The largest magnitude of each row's part of K.
            if (FORMAT == HCCL_NVFP4) {
#pragma unroll
                for (int i = 0; i < TASKS; i++) {
                    const int r = row_of(i);
                    if (r >= t.rows) break;
                    unsigned top = 0;
#pragma unroll
                    for (int j = 0; j < EACH; j++) top = max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
                    top = __reduce_max_sync(0xffffffffu, top);
                    if (top) atomicMax(&top_of[half][r], top);
                }
                asm volatile("bar.sync 2, 256;" ::: "memory");
            }
#pragma unroll
            for (int i = 0; i < TASKS; i++) {
                const int r = row_of(i), k = k_of(i);
                if (r >= t.rows) break;
                float factor = 1.f, back = 1.f;
                if (FORMAT == HCCL_NVFP4) {
                    // 2^10 <= largest * factor < 2^11; both factors stay powers of two that are no subnormal numbers
                    const unsigned top = top_of[half][r];
                    const int e = (int)(top >> 23) - 127, up = min(max(10 - e, -126), 126);
                    factor = __uint_as_float((unsigned)(127 + up) << 23), back = __uint_as_float((unsigned)(127 - up) << 23);
                }
                if (k == k0) unscale[half][r] = back;
#pragma unroll
                for (int j = 0; j < EACH; j++) v[i][j] *= factor;
                const int kk = k - k0, stage = kk / 256, in_stage = kk % 256;
#pragma unroll
                for (int q = 0; q < PIECES; q++) {
                    if (FORMAT == HCCL_NVFP4 && q == PIECES / 2)
#pragma unroll
                        for (int j = 0; j < EACH; j++) v[i][j] *= LATER;
                    unsigned top = 0;
#pragma unroll
                    for (int j = 0; j < EACH; j++) top = max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
                    // a block's elements lie with two neighbouring lanes, or four
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    if (FORMAT == HCCL_MXFP4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const Step s = some_step<FORMAT>(top);
                    float quo[EACH], val[EACH];
#pragma unroll
                    for (int j = 0; j < EACH; j++) quo[j] = v[i][j] * s.inv;
                    const unsigned code = eight_codes(quo);
                    eight_values(__shfl_sync(0xffffffffu, code, lane), val);
#pragma unroll
                    for (int j = 0; j < EACH; j++) v[i][j] = fmaf(-val[j], s.d, v[i][j]);
                    const int n = r * PIECES + q, sixteen = in_stage / 32;
                    *(unsigned*)(part + stage * S::PIECE_STAGE + n * KB + ((sixteen ^ (n & 7)) * 16) + in_stage % 32 / 2) = code;
                    constexpr int B = block_of(FORMAT);
                    if (kk % B == 0) part[S::PIECE_SCALES + kk / (4 * B) * ATOM + atom_row(n) + kk / B % 4] = (char)s.byte;
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(part_full(half));
            if (FORMAT == HCCL_NVFP4) {
                // everyone has read the maxima: they start at zero when this half's turn comes again
                asm volatile("bar.sync 2, 256;" ::: "memory");
                if (me < ROWS) top_of[half][me] = 0;
            }
        }
    }
    // After a wait that gave up, loads may still be in flight: wait (with a limit) for the stages that were issued.
    if (warp == 0 && lane == 0 && *(volatile int*)&gave_up) {
        const unsigned long long t0 = now_ns();
        for (int i = max(0, it - S::STAGES); i < it; i++)
            while (!mbar_try(full(i % S::STAGES), (i / S::STAGES) & 1) && now_ns() - t0 < WAIT_NS) {}
        __nanosleep(1000000);  // and the instructions issued last, which end by themselves
        if (p.status) *p.status = HCCL_ERR_TIMEOUT;
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLS));
}

template <typename T, int FORMAT, bool DOWN> cudaError_t launch(const FewParams& p, cudaStream_t s) {
    using S = Shape<FORMAT>;
    static std::atomic<bool> ready[64];  // by device; setting it twice does no harm
    int dev = 0;
    cudaError_t e;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev]) {
        e = cudaFuncSetAttribute(hccl_few_fp4<T, FORMAT, DOWN>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(SMS);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = S::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = DOWN ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, hccl_few_fp4<T, FORMAT, DOWN>, p);
}

constexpr long long up_to(long long n, long long m) { return (n + m - 1) / m * m; }

// Floats of partial sums: [parts of K][rows][width]. With all SPAN stages to a unit there are that many parts; where span_of cuts finer, it does so because there are fewer than
// ENOUGH * SMS units of twice the size, each of 128 channels x at most 8 rows (width is at most 16 more than the channels).
long long partial_sums(long long rows, long long width, long long k_blocks) {
    const long long most = rows * k_blocks * width, fine = 2ll * ROWS * ENOUGH * SMS * (CH + 16), coarse = rows * ((k_blocks + SPAN - 1) / SPAN) * width;
    return up_to(std::max(coarse, std::min(most, fine)), 64);
}

struct Places {
    long long half, wide_up, wide_y, sums_up, sums_down, tiles;
};
Places places(long long rows, long long H, long long I, int gated) {
    Places a;
    a.half = up_to(I, 8);
    a.wide_up = (gated ? 2 : 1) * a.half;
    a.wide_y = H;
    a.sums_up = partial_sums(rows, a.wide_up, (H + 255) / 256);
    a.sums_down = partial_sums(rows, a.wide_y, (I + 255) / 256);
    a.tiles = (H + CH - 1) / CH;
    return a;
}

template <typename T, int FORMAT> cudaError_t few(const FewFp4& q, cudaStream_t s) {
    using S = Shape<FORMAT>;
    const long long rows = q.T * q.top_k, N = (q.gated ? 2 : 1) * q.I;
    const Places at = places(rows, q.H, q.I, q.gated);
    FewParams p = {};
    p.offsets = q.offsets;
    p.source = q.source;
    p.slots = q.slots;
    p.weights = q.weights;
    p.status = q.status;
    p.experts = q.experts;
    p.top_k = q.top_k;
    p.T = (int)q.T;
    p.rows = (int)rows;
    p.act = q.act;
    p.gated = q.gated;
    p.half = (int)at.half;
    p.I = (int)q.I;
    p.wide_y = (int)at.wide_y;
    p.down_tiles = (int)at.tiles;
    float* const sums = (float*)q.scratch;
    p.arrived = (int*)(sums + at.sums_up + at.sums_down);
    p.part = sums + at.sums_up;
    cudaError_t e;
    const auto maps = [&](const uint8_t* w, const uint8_t* scale, long long ld, long long n, long long k) {
        p.N = (int)n;
        p.K = (int)k;
        p.k_blocks = (int)((k + 255) / 256);
        p.chan_tiles = (int)((n + CH - 1) / CH);
        if ((e = make_map(&p.w, w, n * q.experts, (k + 1) / 2, ld, CH)) != cudaSuccess) return e;
        return make_atom_map(&p.w_scale, scale, (long long)q.experts * p.chan_tiles * p.k_blocks * S::ATOMS, S::ATOMS);
    };
    if ((e = maps(q.up, q.up_scale, q.ld_up, N, q.H)) != cudaSuccess) return e;
    p.x = q.x;
    p.ldx = q.ldx;
    p.vec = (uintptr_t)q.x % 16 == 0 && (q.T <= 1 || q.ldx * sizeof(T) % 16 == 0);
    p.y = sums;
    p.wide = q.up_wide;
    p.bias = q.up_bias;
    if ((e = launch<T, FORMAT, false>(p, s)) != cudaSuccess) return e;
    p.x_blocks = p.k_blocks;
    p.x_tiles = p.chan_tiles;
    if ((e = maps(q.down, q.down_scale, q.ld_down, q.H, q.I)) != cudaSuccess) return e;
    p.x = sums;
    p.y = q.y;
    p.ldy = q.ldy;
    p.wide = q.down_wide;
    p.bias = q.down_bias;
    return launch<T, FORMAT, true>(p, s);
}

}  // namespace

size_t few_fp4_scratch(long long T, long long H, long long I, int top_k, int gated) {
    const Places at = places(T * top_k, H, I, gated);
    return (size_t)((at.sums_up + at.sums_down) * 4 + up_to(at.tiles * 4, 128));
}

cudaError_t launch_few_fp4(int dt, const FewFp4& p, cudaStream_t s) {
    if (p.T == 0) return cudaSuccess;
    const bool nv = p.format == HCCL_NVFP4;
    if (dt == HCCL_FP32) return nv ? few<float, HCCL_NVFP4>(p, s) : few<float, HCCL_MXFP4>(p, s);
    if (dt == HCCL_BF16) return nv ? few<__nv_bfloat16, HCCL_NVFP4>(p, s) : few<__nv_bfloat16, HCCL_MXFP4>(p, s);
    return nv ? few<__half, HCCL_NVFP4>(p, s) : few<__half, HCCL_MXFP4>(p, s);
}

}  // namespace experts
}  // namespace hccl
