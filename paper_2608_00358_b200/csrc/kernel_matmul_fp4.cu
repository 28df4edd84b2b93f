// Products in 4-bit floating point with a scale for each block of both operands, on the fifth-generation tensor cores, which multiply the scales in.
//
// y[m, n] = (sum over blocks of (sum_k q[m, k] v[n, k]) s[m, b] t[n, b]) * x_wide * w_wide[group] (+ bias[n]), summed in 32-bit floating point. As in the products in
// 8-bit integers the weights are the instruction's 128-row operand and the tokens its columns. With CG = 2 two blocks on neighbouring SMs form a
// tile of 256 channels x 256 tokens; each has all 256 tokens' scales in its own tensor memory.
//
// Roles of a block (12 warps): warp 0 issues the TMA loads, warp 1 copies a stage's scales to tensor memory and issues the matrix instructions, warp 2 owns
// the tensor memory, warps 4-11 turn accumulators into results. A stage is 256 elements of K: 128 bytes of each row, and the scales' atoms. Every stage has
// columns of tensor memory of its own for its scales, so that they are not written again before the instructions that read them are done.
// A tile of 256 tokens leaves room for one accumulator: 16-bit results are taken out whole, into registers, and stored while the next tile is formed.
//
// Measured (B200; four times the bf16 library rate is 6.7 PFLOP/s): 8192^3 176-197 us on different machines = 5.6-6.3 PFLOP/s at the power limit, tensor cores active in 75 % of the cycles; a
// stage's products take 512 cycles and its bytes 594 of shared memory's (2 x 38 KB written and read at 128 a cycle), so shared memory is the next bound. 64 matrices 2048 x 4096: 65536 rows
// 241-265 us, 512 rows 52 us = 5.8 TB/s of weights. 997 x 4104 x 2064 12 us; 1 to 16 rows, 8192 x 4096, 10 to 11 us with cold weights (with the quantiser 10.3 us in replays of a graph, 14.4 after a flush
// of the caches), most of it set-up and the first stages' way.
#include <atomic>

#include "fp4.cuh"
#include "tensor.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int MM_THREADS = 384, CH = 128 /* channels of a tile */;

template <int TN, int CG, int FORMAT> struct Shape {
    static constexpr int ROWS = TN / CG;                   // token rows that a block holds
    static constexpr int BOX = ROWS < 64 ? ROWS : 64;      // of them, in one TMA load
    static constexpr int ATOMS = stage_atoms(FORMAT), WIDE = TN > 128 ? TN / 128 : 1;
    static constexpr int W_SCALE = (CH + ROWS) * KB, X_SCALE = W_SCALE + ATOMS * ATOM;  // places in a stage
    static constexpr int STAGE = X_SCALE + WIDE * ATOMS * ATOM;
    static constexpr int ACCS = TN > 128 ? 1 : 2;
    static constexpr int SCALE_COLS = 4 * ATOMS * (1 + WIDE);
    static constexpr int BY_SMEM = (200 * 1024) / STAGE, BY_TMEM = (512 - ACCS * TN) / SCALE_COLS;
    static constexpr int STAGES = BY_SMEM < BY_TMEM ? BY_SMEM : BY_TMEM;
    static constexpr int SMEM = STAGES * STAGE + 1024;
    static_assert(STAGE % 1024 == 0, "operands start on 1024-byte boundaries");
};
constexpr int COLS = 512;  // of tensor memory: all of it, one block to an SM

struct TileParams {
    CUtensorMap a, w, a_scale, w_scale;
    long long ldy;
    const float *w_wide, *bias;
    const int* offsets;
    void* y;
    int* status;
    float x_wide;
    int M, N, groups, steps /* of 64 elements */, k_blocks, n_tiles, chan_tiles, splits, dependent;
    int pairs;  // two neighbouring 16-bit results of a row can be written at once
};

// ---------------------------------------------------------------- instructions
template <int CG, int FORMAT> __device__ __forceinline__ void mma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
#define HCCL_MMA(cg, kind) \
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n tcgen05.mma.cta_group::" cg ".kind::" kind " [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"(sa), "r"(sb), "r"(accumulate) : "memory")
    if constexpr (FORMAT == HCCL_NVFP4) {
        if constexpr (CG == 2) HCCL_MMA("2", "mxf4nvf4.block_scale.scale_vec::4X");
        else HCCL_MMA("1", "mxf4nvf4.block_scale.scale_vec::4X");
    } else {
        if constexpr (CG == 2) HCCL_MMA("2", "mxf4.block_scale.scale_vec::2X");
        else HCCL_MMA("1", "mxf4.block_scale.scale_vec::2X");
    }
#undef HCCL_MMA
}
// An atom of scales to four columns of tensor memory, the same in each quarter of its lanes; with CG = 2 each block's from its own shared memory.
template <int CG> __device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t addr) {
    const uint64_t from = (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);  // 32 rows of 16 bytes, 8 of them in 128
    if constexpr (CG == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(from) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(from) : "memory");
}

// ---------------------------------------------------------------- tiles
struct Tile {
    int group, row, rows, chan;  // rows [row, row + rows) of the tokens, this block's channels from chan on
    int x_tile;                  // of the tokens' scales
};

// Tile t. before[g] = token tiles of the groups below g. Within a group 8 token tiles pass under one tile of channels
// before the next, so that the blocks of a wave share both operands in the L2.
template <int TN, int CG> __device__ __forceinline__ Tile tile_of(const TileParams& p, const int* before, int t, int rank, int* hint) {
    Tile r;
    int g = 0, lo = 0, hi = p.M;
    if (p.groups) {
        g = *hint;
        while (t >= before[g + 1] * p.n_tiles) g++;
        *hint = g;
        lo = max(0, p.offsets[g]);
        hi = min(p.M, p.offsets[g + 1]);
    }
    const int mt = p.groups ? before[g + 1] - before[g] : (p.M + TN - 1) / TN;
    const int i = t - (p.groups ? before[g] * p.n_tiles : 0);
    const int band = i / (8 * p.n_tiles), first = band * 8, deep = min(8, mt - first), j = i - band * 8 * p.n_tiles;
    // (the same in all lanes, and by way of the shuffle known to be)
    r.group = __shfl_sync(0xffffffffu, g, 0);
    r.row = __shfl_sync(0xffffffffu, lo + (first + j % deep) * TN, 0);
    r.rows = __shfl_sync(0xffffffffu, min(TN, hi - r.row), 0);
    r.chan = __shfl_sync(0xffffffffu, (j / deep) * CH * CG + rank * CH, 0);
    r.x_tile = __shfl_sync(0xffffffffu, (int)tile_base(lo, TN, g) + first + j % deep, 0);
    return r;
}

template <typename T, int TN, int CG, int FORMAT> __global__ void __launch_bounds__(MM_THREADS, 1) hccl_matmul_fp4_tiles(const __grid_constant__ TileParams p) {
    using S = Shape<TN, CG, FORMAT>;
    constexpr int ACCS = S::ACCS;
    extern __shared__ char dynamic[];
    __shared__ __align__(8) unsigned long long bars[2 * S::STAGES + 2 * ACCS];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up;
    __shared__ int before[HCCL_MAX_EXPERTS + 1];
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_addr(dynamic) + 1023) & ~1023u;
    const uint32_t bar0 = smem_addr(bars);
    const auto full = [&](int s) { return bar0 + 8 * s; };
    const auto empty = [&](int s) { return bar0 + 8 * (S::STAGES + s); };
    const auto acc_full = [&](int b) { return bar0 + 8 * (2 * S::STAGES + b); };
    const auto acc_empty = [&](int b) { return bar0 + 8 * (2 * S::STAGES + ACCS + b); };

    // Which blocks work together: a pair (CG = 2, on one tile), or p.splits blocks that share a tile's K, or each alone.
    const int splits = CG == 2 ? 1 : p.splits, team = CG == 2 ? 2 : p.splits;
    const int rank = (int)blockIdx.x % team, first = (int)blockIdx.x / team, step = (int)gridDim.x / team;
    const int pair_rank = CG == 2 ? rank : 0;
    const int k0 = CG == 2 ? 0 : (int)((long long)p.k_blocks * rank / splits), k1 = CG == 2 ? p.k_blocks : (int)((long long)p.k_blocks * (rank + 1) / splits);

    // A role's own state
    int it = 0, acc = 0, hint = 0;  // stages passed, tiles passed, group
    bool waited = !p.dependent;
    const auto rely = [&] {  // from here on reads what the kernel before this one wrote
        if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
        waited = true;
    };
    // Token rows that this block loads: all of the tile's, or, of a pair, a half of them, rounded up to 16.
    const auto half_of = [&](const Tile& t) { return CG == 2 ? ((t.rows + 31) / 32) * 16 : t.rows; };
    const auto full_at = [&](int s) { return CG == 2 ? of_rank(full(s), 0) : full(s); };
    // The next three by one lane.
    const auto load_w = [&](const Tile& t, int s, int kb) {
        const uint32_t at = base + s * S::STAGE;
        tma_load<CG>(at, &p.w, kb * KB, t.group * p.N + t.chan, full_at(s));
        tma_load<CG>(at + S::W_SCALE, &p.w_scale, 0, ((t.group * p.chan_tiles + t.chan / CH) * p.k_blocks + kb) * S::ATOMS, full_at(s));
    };
    const auto load_a = [&](const Tile& t, int s, int kb) {
        const uint32_t at = base + s * S::STAGE;
        const int half = half_of(t), boxes = (half + S::BOX - 1) / S::BOX;
        for (int i = 0; i < boxes; i++) tma_load<CG>(at + CH * KB + i * S::BOX * KB, &p.a, kb * KB, t.row + pair_rank * half + i * S::BOX, full_at(s));
#pragma unroll
        for (int i = 0; i < S::WIDE; i++)
            tma_load<CG>(at + S::X_SCALE + i * S::ATOMS * ATOM, &p.a_scale, 0, ((t.x_tile * S::WIDE + i) * p.k_blocks + kb) * S::ATOMS, full_at(s));
    };
    // The first block's barrier counts the bytes of both.
    const auto expect = [&](const Tile& t, int s) {
        if (pair_rank == 0) mbar_expect(full(s), (uint32_t)(CG * (CH * KB + (half_of(t) + S::BOX - 1) / S::BOX * S::BOX * KB + (1 + S::WIDE) * S::ATOMS * ATOM)));
    };

    int pre = 0;  // stages of the first tile whose weights are under way
    const auto prefetch = [&](const Tile& t) {
        pre = min(k1 - k0, S::STAGES);
        if (elected())
            for (int i = 0; i < pre; i++) {
                expect(t, i);
                load_w(t, i, k0 + i);
            }
        __syncwarp();
    };
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; s++) mbar_init(full(s), 1), mbar_init(empty(s), 1);
        for (int b = 0; b < ACCS; b++) mbar_init(acc_full(b), 1), mbar_init(acc_empty(b), 8 * CG);
        gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (CG == 2) cluster_sync();  // both blocks' barriers exist before either uses the other's
    // The weights do not hang on the kernel before, nor on the other warps: they are asked for at once.
    if (warp == 0 && !p.groups) prefetch(tile_of<TN, CG>(p, before, first, pair_rank, &hint));
    if (warp == 2) {
        if constexpr (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_at)), "n"(COLS));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_at)), "n"(COLS));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        }
    }
    if (warp == 3 && p.groups) {
        int run = 0;
        for (int b = 0; b < p.groups; b += 32) {
            const int g = b + lane;
            int n = 0;
            if (g < p.groups) n = max(0, (min(p.M, p.offsets[g + 1]) - max(0, p.offsets[g]) + TN - 1) / TN);
            int inc = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += v;
            }
            if (g < p.groups) before[g] = run + inc - n;
            run += __shfl_sync(0xffffffffu, inc, 31);
        }
        if (lane == 0) before[p.groups] = run;
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_at, 0);
    const int tiles = p.n_tiles * (p.groups ? before[p.groups] : (p.M + TN - 1) / TN);

    const auto produce = [&](const Tile& t) {
        if (!pre && !waited) prefetch(t);
        rely();
        if (elected())
            for (int i = 0; i < pre; i++) load_a(t, i, k0 + i);
        __syncwarp();
        it += pre;
        for (int kb = k0 + pre; kb < k1; kb++, it++) {
            const int s = it % S::STAGES;
            if (!mbar_wait(empty(s), ((it / S::STAGES) & 1) ^ 1, &gave_up)) return;
            if (elected()) {
                expect(t, s);
                load_w(t, s, kb);
                load_a(t, s, kb);
            }
            __syncwarp();
        }
        pre = 0;
    };
    const auto multiply = [&](const Tile& t) {
        const int b = acc % ACCS;
        const uint32_t cols = CG == 2 ? (uint32_t)((t.rows + 31) & ~31) : (uint32_t)((t.rows + 7) & ~7);
        // e2m1 operands, both with K innermost; scales e4m3 or powers of two
        const uint32_t desc = (1u << 7) | (1u << 10) | ((cols >> 3) << 17) | (FORMAT == HCCL_MXFP4 ? 1u << 23 : 0u) | ((uint32_t)(CH * CG >> 7) << 27);
        if (!mbar_wait(acc_empty(b), ((acc / ACCS) & 1) ^ 1, &gave_up)) return;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int kb = k0; kb < k1; kb++, it++) {
            const int s = it % S::STAGES;
            if (!mbar_wait(full(s), (it / S::STAGES) & 1, &gave_up)) return;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t at = base + s * S::STAGE, scales = tmem + ACCS * TN + s * S::SCALE_COLS;
            const uint64_t w = operand(at), a = operand(at + CH * KB);
            const int steps = min(4, p.steps - 4 * kb);
            if (elected()) {
#pragma unroll
                for (int i = 0; i < S::ATOMS; i++) copy_scales<CG>(scales + 4 * i, at + S::W_SCALE + i * ATOM);
#pragma unroll
                for (int i = 0; i < S::ATOMS; i++)
#pragma unroll
                    for (int j = 0; j < S::WIDE; j++) copy_scales<CG>(scales + 4 * S::ATOMS + 4 * (i * S::WIDE + j), at + S::X_SCALE + (j * S::ATOMS + i) * ATOM);
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    if (k >= steps) break;
                    const int i = k * S::ATOMS / 4;
                    const uint32_t half = FORMAT == HCCL_MXFP4 ? 2u * (k & 1) : 0u;  // two of an atom's four scales are a step's
                    mma_fp4<CG, FORMAT>(tmem + b * TN, w + 2 * k, a + 2 * k, desc | (half << 4) | (half << 29), scales + 4 * i, scales + 4 * S::ATOMS + 4 * i * S::WIDE,
                                        (kb > k0 || k > 0) ? 1u : 0u);
                }
                mma_commit<CG>(empty(s));
                if (kb == k1 - 1) mma_commit<CG>(acc_full(b));
            }
            __syncwarp();
        }
    };
    const auto scaled = [&](float sum, float factor, float bias) {
        const float v = __fmul_rn(sum, factor);
        return p.bias ? __fadd_rn(v, bias) : v;
    };
    const auto factor_of = [&](int group) { return __fmul_rn(p.w_wide[group], p.x_wide); };
    const auto free_acc = [&](int b) {
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            if (CG == 2) mbar_arrive_at(of_rank(acc_empty(b), 0));
            else mbar_arrive(acc_empty(b));
        }
    };
    const auto results = [&](const Tile& t) {
        const int b = acc % ACCS, quarter = warp & 3, chan = t.chan + quarter * 32 + lane;
        const bool in = chan < p.N;
        const float factor = factor_of(t.group), bias = (in && p.bias) ? p.bias[(long long)t.group * p.N + chan] : 0.f;
        // The tile's columns in blocks of 32, in turn to the two warps of a quarter (four warps instead: no difference at 256 tokens).
        constexpr int C = TN < 32 ? TN : 32, U = (TN + 63) / 64;
        constexpr bool WHOLE = ACCS == 1 && sizeof(T) == 2;  // everything out of tensor memory first
        const int half = (warp - 4) >> 2;
        if (p.k_blocks && !mbar_wait(acc_full(b), (acc / ACCS) & 1, &gave_up)) return;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + b * TN;
        const auto fetch = [&](int c0, float (&o)[C]) {
            int v[32];
            __syncwarp();
            if (p.k_blocks) {
                tmem_load(at + c0, *(int(*)[16])v);
                if (TN > 16) tmem_load(at + c0 + 16, *(int(*)[16])(v + 16));
                tmem_arrived();
            } else {
#pragma unroll
                for (int j = 0; j < 32; j++) v[j] = 0;
            }
#pragma unroll
            for (int j = 0; j < C; j++) o[j] = scaled(__int_as_float(v[j]), factor, bias);
        };
        // Results of a block of columns as words of two neighbouring tokens.
        const auto store_words = [&](int c0, const unsigned (&w)[C / 2]) {
            T* y = (T*)p.y + (long long)(t.row + c0) * p.ldy + chan;
            if (p.pairs && c0 + C <= t.rows && t.chan + quarter * 32 + 32 <= p.N) {
                // Two neighbouring lanes trade: the even one keeps row j of both channels, the odd one row j + 1, four bytes each, so that a store
                // instruction writes 64 bytes of two rows.
                const int odd = lane & 1;
                y += odd * p.ldy - odd;
#pragma unroll
                for (int j = 0; j < C / 2; j++, y += 2 * p.ldy) {
                    const unsigned other = __shfl_xor_sync(0xffffffffu, w[j], 1);
                    *(unsigned*)y = __byte_perm(w[j], other, odd ? 0x3276 : 0x5410);
                }
            } else if (in) {
#pragma unroll
                for (int j = 0; j < C; j++, y += p.ldy)
                    if (c0 + j < t.rows) *(unsigned short*)y = (unsigned short)(w[j / 2] >> (16 * (j & 1)));
            }
        };
        if constexpr (WHOLE) {
            unsigned w[U][C / 2];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int c0 = (2 * u + half) * 32;
                if (c0 < t.rows) {
                    float o[C];
                    fetch(c0, o);
#pragma unroll
                    for (int j = 0; j < C; j += 2) w[u][j / 2] = Pack<T, 2>::word(o[j], o[j + 1]);
                }
            }
            free_acc(b);
#pragma unroll
            for (int u = 0; u < U; u++)
                if ((2 * u + half) * 32 < t.rows) store_words((2 * u + half) * 32, w[u]);
        } else {
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int c0 = (2 * u + half) * 32;
                if (c0 >= t.rows) break;
                float o[C];
                fetch(c0, o);
                if constexpr (sizeof(T) == 2) {
                    unsigned w[C / 2];
#pragma unroll
                    for (int j = 0; j < C; j += 2) w[j / 2] = Pack<T, 2>::word(o[j], o[j + 1]);
                    store_words(c0, w);
                } else if (in) {
                    T* y = (T*)p.y + (long long)(t.row + c0) * p.ldy + chan;
#pragma unroll
                    for (int j = 0; j < C; j++, y += p.ldy)
                        if (c0 + j < t.rows) *y = from_f32<T>(o[j]);
                }
            }
            free_acc(b);
        }
    };
    const auto stopped = [&] { return *(volatile int*)&gave_up != 0; };

    if (splits == 1) {
        if (warp == 0) {
            if (p.k_blocks)
                for (int t = first; t < tiles && !stopped(); t += step) produce(tile_of<TN, CG>(p, before, t, pair_rank, &hint));
        } else if (warp == 1 && pair_rank == 0) {
            if (p.k_blocks)
                for (int t = first; t < tiles && !stopped(); t += step, acc++) multiply(tile_of<TN, CG>(p, before, t, pair_rank, &hint));
        } else if (warp >= 4) {
            rely();
            for (int t = first; t < tiles && !stopped(); t += step, acc++) results(tile_of<TN, CG>(p, before, t, pair_rank, &hint));
        }
    } else if constexpr (CG == 1 && TN <= 64) {
        // One tile at a time for the whole cluster. The partial sums go to shared memory (the stages are idle by then), column by
        // column; then each block adds a share of the outputs over all blocks of the cluster, in their order. Every block passes every barrier, also
        // after a wait that gave up.
        float* part = (float*)(dynamic + (base - smem_addr(dynamic)));
        for (int t = first; t < tiles; t += step, acc++) {
            const Tile tile = tile_of<TN, CG>(p, before, t, 0, &hint);
            if (warp == 0) produce(tile);
            if (warp == 1) multiply(tile);
            if (warp >= 4) {
                const int b = acc % ACCS, quarter = warp & 3;
                const bool ok = mbar_wait(acc_full(b), (acc / ACCS) & 1, &gave_up);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (ok)
                    for (int c0 = ((warp - 4) >> 2) * 16; c0 < tile.rows; c0 += 32) {
                        int v[16];
                        tmem_load(tmem + ((uint32_t)(quarter * 32) << 16) + b * TN + c0, v);
                        tmem_arrived();
#pragma unroll
                        for (int i = 0; i < 16; i++) part[(c0 + i) * CH + quarter * 32 + lane] = __int_as_float(v[i]);
                    }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(acc_empty(b));
            }
            rely();
            __syncwarp();
            cluster_sync();
            const float factor = factor_of(tile.group);
            const int total = tile.rows * (CH / 4), lo = total * rank / splits, hi = total * (rank + 1) / splits;  // four channels at a time
            for (int i = lo + (int)threadIdx.x; i < hi; i += MM_THREADS) {
                float sum[4] = {};
                for (int r = 0; r < splits; r++) {
                    const int4 v = cluster_load(base + 16 * i, r);
                    sum[0] += __int_as_float(v.x), sum[1] += __int_as_float(v.y), sum[2] += __int_as_float(v.z), sum[3] += __int_as_float(v.w);
                }
                const int chan = tile.chan + i % (CH / 4) * 4, row = tile.row + i / (CH / 4);
                T* y = (T*)p.y + (long long)row * p.ldy + chan;
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (chan + j < p.N) y[j] = from_f32<T>(scaled(sum[j], factor, p.bias ? p.bias[(long long)tile.group * p.N + chan + j] : 0.f));
            }
            // what the generic proxy read and wrote here, the next tile's loads will overwrite
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            cluster_sync();
        }
    }
    rely();
    // After a wait that gave up, loads may still be in flight: wait (with a limit) for the stages that were issued.
    if (warp == 0 && lane == 0 && stopped()) {
        const unsigned long long t0 = now_ns();
        if (pair_rank == 0)
            for (int i = max(0, it - S::STAGES); i < it; i++)
                while (!mbar_try(full(i % S::STAGES), (i / S::STAGES) & 1) && now_ns() - t0 < WAIT_NS) {}
        __nanosleep(1000000);  // and the instructions issued last, which end by themselves
        if (p.status) *p.status = HCCL_ERR_TIMEOUT;
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) cluster_sync();  // neither block leaves while the other's instructions or arrivals may still reach it
    if (warp == 2) {
        if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLS));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLS));
    }
}

// ---------------------------------------------------------------- host
template <typename T, int TN, int CG, int FORMAT> cudaError_t tiles_launch(const MatmulFp4& q, cudaStream_t s) {
    using S = Shape<TN, CG, FORMAT>;
    const long long G = q.groups ? q.groups : 1;
    TileParams p = {};
    p.ldy = q.ldy;
    p.w_wide = q.w_wide;
    p.x_wide = q.x_wide;
    p.bias = q.bias;
    p.offsets = q.offsets;
    p.y = q.y;
    p.status = q.status;
    p.M = (int)q.M;
    p.N = (int)q.N;
    p.groups = q.groups;
    p.steps = (int)((q.K + 63) / 64);
    p.k_blocks = (int)((q.K + 255) / 256);
    p.n_tiles = (int)((q.N + CH * CG - 1) / (CH * CG));
    p.chan_tiles = (int)((q.N + CH - 1) / CH);
    p.splits = q.splits;
    p.dependent = q.dependent;
    p.pairs = (uintptr_t)q.y % 4 == 0 && q.ldy % 2 == 0;
    cudaError_t e;
    if (q.K) {
        const long long bytes = (q.K + 1) / 2, x_tiles = (q.M + TN - 1) / TN + G;
        if ((e = make_map(&p.a, q.q, q.M, bytes, q.ldq, S::BOX)) != cudaSuccess) return e;
        if ((e = make_map(&p.w, q.w, q.N * G, bytes, q.ldw, CH)) != cudaSuccess) return e;
        if ((e = make_atom_map(&p.a_scale, q.q_scale, x_tiles * S::WIDE * p.k_blocks * S::ATOMS, S::ATOMS)) != cudaSuccess) return e;
        if ((e = make_atom_map(&p.w_scale, q.w_scale, G * p.chan_tiles * p.k_blocks * S::ATOMS, S::ATOMS)) != cudaSuccess) return e;
    }
    static std::atomic<bool> ready[64];  // by device; setting it twice does no harm
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev]) {
        e = cudaFuncSetAttribute(hccl_matmul_fp4_tiles<T, TN, CG, FORMAT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev] = true;
    }
    const long long tiles = (long long)p.n_tiles * ((q.M + TN - 1) / TN + q.groups);  // at most, with groups
    const int team = CG == 2 ? 2 : q.splits;
    const long long teams = SMS / team;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((tiles < teams ? tiles : teams) * team));
    cfg.blockDim = dim3(MM_THREADS);
    cfg.dynamicSmemBytes = S::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (team > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)team;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        n++;
    }
    if (q.dependent) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        n++;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, hccl_matmul_fp4_tiles<T, TN, CG, FORMAT>, p);
}

template <typename T, int FORMAT> cudaError_t matmul_launch(const MatmulFp4& p, cudaStream_t s) {
    switch (p.tn) {
        case 16: return tiles_launch<T, 16, 1, FORMAT>(p, s);
        case 32: return tiles_launch<T, 32, 1, FORMAT>(p, s);
        case 64: return tiles_launch<T, 64, 1, FORMAT>(p, s);
        case 128: return tiles_launch<T, 128, 1, FORMAT>(p, s);
        default: return tiles_launch<T, 256, 2, FORMAT>(p, s);
    }
}

}  // namespace

// Which tile, as for the products in 8-bit integers: tiles of TN tokens and a cluster of S blocks for each, by an estimate in microseconds: rounds of the blocks over the tiles, times stages, times a
// stage's time, and what does not overlap. Measured with the quantiser against every other choice on 18 shapes, TN,S (1 x 8192 x 4096 takes 10.4 us with 16,1 to 32,2; 1 x 2048 x 4096 8.3 with
// 16,4 and 10.3 with 32,2; 128 x 2048 x 8192 12.4 with 64,4 and 16.1 with 32,1; 512 x 4096 x 4096 13.3 with 128,1 and 17.3 with 64,1; 997 x 4104 x 2064 14.4 with 256,1 and 16.5 with 128,1); nowhere is
// the choice more than 8 % behind the best. Groups are uneven: tiles of twice the mean number of rows hold most groups whole, so that weights are read once.
TileChoice choose_fp4(long long M, long long N, long long K, int groups) {
    if (groups) {
        const long long twice = 2 * ((M + groups - 1) / groups);
        return {twice <= 16 ? 16 : twice <= 32 ? 32 : twice <= 64 ? 64 : twice <= 128 ? 128 : 256, 1};
    }
    const double k_blocks = (double)((K + 255) / 256);
    static const struct {
        int tn;
        double stage, last, exchange;
    } option[] = {{16, 0.17, 0.0, 1.4}, {32, 0.17, 0.1, 1.5}, {64, 0.18, 0.4, 2.4}, {128, 0.22, 1.2, 0}, {256, 0.30, 2.3, 0}};
    TileChoice best = {256, 1};
    double least = 1e30;
    for (const auto& o : option) {
        const bool pair = o.tn == 256;
        const long long tiles = (M + o.tn - 1) / o.tn * ((N + (pair ? 2 * CH : CH) - 1) / (pair ? 2 * CH : CH)), at_once = pair ? SMS / 2 : SMS;
        for (int s = 1; s <= (o.tn <= 64 ? 8 : 1); s *= 2) {
            if (s > 1 && (tiles * s > (s == 8 ? 64 : 128) || k_blocks < 4 * s)) break;
            const double t = (double)((tiles + at_once - 1) / at_once) * (k_blocks / s) * o.stage + o.last + (s > 1 ? o.exchange : 0);
            if (t < least) least = t, best = {o.tn, s};
        }
    }
    return best;
}

cudaError_t launch_matmul_fp4(int dt, const MatmulFp4& p, cudaStream_t s) {
    if (p.M == 0 || p.N == 0) return cudaSuccess;
    const bool nv = p.format == HCCL_NVFP4;
    if (dt == HCCL_FP32) return nv ? matmul_launch<float, HCCL_NVFP4>(p, s) : matmul_launch<float, HCCL_MXFP4>(p, s);
    if (dt == HCCL_BF16) return nv ? matmul_launch<__nv_bfloat16, HCCL_NVFP4>(p, s) : matmul_launch<__nv_bfloat16, HCCL_MXFP4>(p, s);
    return nv ? matmul_launch<__half, HCCL_NVFP4>(p, s) : matmul_launch<__half, HCCL_MXFP4>(p, s);
}

}  // namespace experts
}  // namespace hccl
