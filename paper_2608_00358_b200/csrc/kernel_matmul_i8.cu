// Products in 8-bit integers with scales for each row of both operands, on the fifth-generation tensor cores.
//
// y[m, n] = (sum_k a[m, k] w[n, k]) * a_scale[m] * w_scale[n] (+ bias[n]). The weights are the instruction's 128-row operand and the
// tokens its columns, so that one kernel serves a single token (N = 16 columns, the weights stream past them) and a
// long prompt (N = 256); the sum is exact in 32-bit integers, in any order.
//
// With CG = 2 two blocks on neighbouring SMs form one tile of 256 channels x 256 tokens: each holds its own 128 channels and half the
// tokens, and the first one's instructions read both. A stage then is 32 KB for each SM instead of 48 KB, which matters because
// shared memory is the bound: a block alone writes and reads 2 x 48 KB for 512 cycles of products, at 128 bytes a cycle.
//
// Roles of a block (12 warps): warp 0 issues the TMA loads, warp 1 the matrix instructions, warp 2 owns the tensor memory, warps 4-11 turn
// accumulators into results (two to each quarter of the tensor memory's lanes). Stages of 128 bytes of K pass from the loads to the instructions through mbarriers; two
// accumulators let the results of one tile leave while the next is formed. Blocks stay and walk tiles; where there are
// too few tiles for the SMs, a cluster of blocks shares a tile's K and adds its partial sums through distributed shared memory.
//
// Measured (B200; twice the bf16 library rate is 3.3 POP/s): 8192^3 308-345 us = 3.2-3.6 POP/s, 535 cycles for a stage whose products take 512, at the 1.5 GHz that the power
// limit leaves (1.9 GHz and 255 us on zeros): the tensor cores are the bound. 64 matrices 2048 x 4096: 512 rows 85 us = 6.1-6.3 TB/s of weights, 65536 rows 375-390 us. 16 rows, 8192 x 4096: 10.8 us = 3.1 TB/s.
// 997 x 2064 x 4104, one round of the blocks: 13.7 us, of which 0.8 set-up, 7 products (665 cycles a stage, fed from the L2), 3 results.
#include <cuda.h>

#include <atomic>

#include "experts.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int MM_THREADS = 384, CH = 128 /* channels of a tile */, KB = 128 /* bytes of K in a stage */;
constexpr unsigned long long WAIT_NS = 2000000000ull;  // bound of every wait

template <int TN, int CG> struct Shape {
    static constexpr int ROWS = TN / CG;               // token rows that a block holds
    static constexpr int BOX = ROWS < 64 ? ROWS : 64;  // of them, in one TMA load
    static constexpr int STAGE = (CH + ROWS) * KB;
    static constexpr int STAGES = (200 * 1024) / STAGE;
    static constexpr int COLS = 2 * TN < 32 ? 32 : 2 * TN;  // tensor memory columns: two accumulators
    static constexpr int SMEM = STAGES * STAGE + 1024;
};

struct TileParams {
    CUtensorMap a, w;
    long long ldy;
    const float *a_scale, *w_scale, *bias;
    const int* offsets;
    void* y;
    int* status;
    int M, N, groups, k_blocks, n_tiles, splits, dependent;
    int pairs;  // two neighbouring 16-bit results of a row can be written at once
};

// ---------------------------------------------------------------- instructions
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count)); }
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// One lane of a warp that is whole here. The matrix and copy instructions want their operands in uniform registers: issued behind
// `lane == 0` the compiler cannot tell that one lane is left and wraps each in a loop over lanes (169 cycles an instruction, measured, against
// 128 of products at 256 columns); behind this it can, if the operands come from values that are the same in all lanes.
__device__ __forceinline__ bool elected() {
    uint32_t e;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(e));
    return e;
}
// Waits for a phase to complete, by a whole warp. After WAIT_NS, or once another wait of this block has given up, it returns false.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
    const unsigned long long t0 = now_ns();
    for (;;) {
        for (int i = 0; i < 64; i++)
            if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
        if (now_ns() - t0 > WAIT_NS) *gave_up = 1;
        if (__any_sync(0xffffffffu, *gave_up)) return false;
    }
}
__device__ __forceinline__ uint32_t of_rank(uint32_t addr, uint32_t rank) {  // the same place in another block of the cluster
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
__device__ __forceinline__ void mbar_arrive_at(uint32_t cluster_bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory"); }
// bar: an address in the cluster's shared memory; with CG = 2 it may lie in the pair's other block.
template <int CG> __device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 2) {
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
        return;
    }
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// Shared-memory operand with 128-byte rows of K in the 128-byte swizzle: groups of 8 rows lie 1024 bytes apart.
__device__ __forceinline__ uint64_t operand(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
template <int CG> __device__ __forceinline__ void mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, uint32_t accumulate) {
    if constexpr (CG == 2)
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"(accumulate) : "memory");
}
// Arrives at the barrier, in both blocks of a pair, when the instructions issued so far are done.
template <int CG> __device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t addr, int (&v)[16]) {  // 16 columns of a warp's 32 lanes; tmem_arrived before use
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]),
                   "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_arrived() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int4 cluster_load(uint32_t addr, uint32_t rank) {
    int4 v;
    asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(of_rank(addr, rank)) : "memory");
    return v;
}

// The same value as (float)v, one rounding to nearest even, by way of its halves: 2^23 + h is a number whose low bits are the 16-bit h, so both
// halves become exact floating-point numbers by a byte permutation and a subtraction, and one fused multiply-add joins and rounds them.
// The conversion instruction runs at an eighth of the rate of these six; results take turns between the two.
__device__ __forceinline__ float by_halves(int v) {
    const unsigned up = (unsigned)v ^ 0x80000000u;  // high half + 2^15
    const float hi = __fadd_rn(__uint_as_float(__byte_perm(up, 0x4b000000u, 0x7632)), -8421376.f), lo = __fadd_rn(__uint_as_float(__byte_perm(up, 0x4b000000u, 0x7610)), -8388608.f);
    return __fmaf_rn(hi, 65536.f, lo);
}

// ---------------------------------------------------------------- tiles
struct Tile {
    int group, row, rows, chan;  // rows [row, row + rows) of the tokens, this block's channels from chan on
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
    return r;
}

template <typename T, int TN, int CG> __global__ void __launch_bounds__(MM_THREADS, 1) hccl_matmul_i8_tiles(const __grid_constant__ TileParams p) {
    using S = Shape<TN, CG>;
    extern __shared__ char dynamic[];
    __shared__ __align__(8) unsigned long long bars[2 * S::STAGES + 4];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up;
    __shared__ int before[HCCL_MAX_EXPERTS + 1];
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_addr(dynamic) + 1023) & ~1023u;
    const uint32_t bar0 = smem_addr(bars);
    const auto full = [&](int s) { return bar0 + 8 * s; };
    const auto empty = [&](int s) { return bar0 + 8 * (S::STAGES + s); };
    const auto acc_full = [&](int b) { return bar0 + 8 * (2 * S::STAGES + b); };
    const auto acc_empty = [&](int b) { return bar0 + 8 * (2 * S::STAGES + 2 + b); };

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
    const auto load_w = [&](const Tile& t, int s, int kb) { tma_load<CG>(base + s * S::STAGE, &p.w, kb * KB, t.group * p.N + t.chan, full_at(s)); };
    const auto load_a = [&](const Tile& t, int s, int kb) {
        const int half = half_of(t), boxes = (half + S::BOX - 1) / S::BOX;
        for (int i = 0; i < boxes; i++) tma_load<CG>(base + s * S::STAGE + CH * KB + i * S::BOX * KB, &p.a, kb * KB, t.row + pair_rank * half + i * S::BOX, full_at(s));
    };
    // The first block's barrier counts the bytes of both.
    const auto expect = [&](const Tile& t, int s) {
        if (pair_rank == 0) mbar_expect(full(s), (uint32_t)(CG * (CH * KB + (half_of(t) + S::BOX - 1) / S::BOX * S::BOX * KB)));
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
        for (int b = 0; b < 2; b++) mbar_init(acc_full(b), 1), mbar_init(acc_empty(b), 8 * CG);
        gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (CG == 2) cluster_sync();  // both blocks' barriers exist before either uses the other's
    // The weights do not hang on the kernel before, nor on the other warps: they are asked for at once.
    if (warp == 0 && !p.groups) prefetch(tile_of<TN, CG>(p, before, first, pair_rank, &hint));
    if (warp == 2) {
        if constexpr (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_at)), "n"(S::COLS));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_at)), "n"(S::COLS));
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
        const int b = acc & 1;
        const uint32_t cols = CG == 2 ? (uint32_t)((t.rows + 31) & ~31) : (uint32_t)((t.rows + 15) & ~15);
        // 32-bit accumulators, signed 8-bit operands, both with K innermost
        const uint32_t desc = (2u << 4) | (1u << 7) | (1u << 10) | ((cols >> 3) << 17) | ((uint32_t)(CH * CG >> 4) << 24);
        if (!mbar_wait(acc_empty(b), ((acc >> 1) & 1) ^ 1, &gave_up)) return;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int kb = k0; kb < k1; kb++, it++) {
            const int s = it % S::STAGES;
            if (!mbar_wait(full(s), (it / S::STAGES) & 1, &gave_up)) return;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t w = operand(base + s * S::STAGE), a = operand(base + s * S::STAGE + CH * KB);
            if (elected()) {
#pragma unroll
                for (int k = 0; k < KB / 32; k++) mma_i8<CG>(tmem + b * TN, w + 2 * k, a + 2 * k, desc, (kb > k0 || k > 0) ? 1u : 0u);
                mma_commit<CG>(empty(s));
                if (kb == k1 - 1) mma_commit<CG>(acc_full(b));
            }
            __syncwarp();
        }
    };
    // A sum passes 2^24 from K = 1024 on: its conversion to 32-bit floating point is a rounding, like each scale's product.
    const auto scaled = [&](float sum, float sa, float sw, float bias) {
        const float v = __fmul_rn(__fmul_rn(sum, sa), sw);
        return p.bias ? __fadd_rn(v, bias) : v;
    };
    const auto results = [&](const Tile& t) {
        const int b = acc & 1, quarter = warp & 3, chan = t.chan + quarter * 32 + lane;
        const bool in = chan < p.N;
        const long long gc = (long long)t.group * p.N + chan;
        const float sw = in ? p.w_scale[gc] : 0.f, bias = (in && p.bias) ? p.bias[gc] : 0.f;
        // The tile's columns in blocks of 32, in turn to the two warps of a quarter; the scale of a block's row 32 i + lane is loaded while the
        // products are formed.
        constexpr int C = TN < 32 ? TN : 32, U = (TN + 63) / 64;
        const int half = (warp - 4) >> 2;
        float sa[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int r = (2 * u + half) * 32 + lane;
            sa[u] = r < t.rows ? p.a_scale[t.row + r] : 0.f;
        }
        if (p.k_blocks && !mbar_wait(acc_full(b), (acc >> 1) & 1, &gave_up)) return;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + b * TN;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int c0 = (2 * u + half) * 32;
            if (c0 >= t.rows) break;
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
            float o[C];  // all of them before the first store: a branch for each would leave its chain of latencies bare
#pragma unroll
            for (int j = 0; j < C; j++) o[j] = scaled(j & 1 ? by_halves(v[j]) : (float)v[j], __shfl_sync(0xffffffffu, sa[u], j), sw, bias);
            T* y = (T*)p.y + (long long)(t.row + c0) * p.ldy + chan;
            if (sizeof(T) == 2 && p.pairs && c0 + C <= t.rows && t.chan + quarter * 32 + 32 <= p.N) {
                // Two neighbouring lanes trade: the even one keeps row j of both channels, the odd one row j + 1, four bytes each, so that a store
                // instruction writes 64 bytes of two rows.
                const int odd = lane & 1;
                y += odd * p.ldy - odd;
#pragma unroll
                for (int j = 0; j < C; j += 2, y += 2 * p.ldy) {
                    const unsigned mine = Pack<T, 2>::word(o[j], o[j + 1]), other = __shfl_xor_sync(0xffffffffu, mine, 1);
                    *(unsigned*)y = __byte_perm(mine, other, odd ? 0x3276 : 0x5410);
                }
            } else if (in) {
#pragma unroll
                for (int j = 0; j < C; j++, y += p.ldy)
                    if (c0 + j < t.rows) *y = from_f32<T>(o[j]);
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            if (CG == 2) mbar_arrive_at(of_rank(acc_empty(b), 0));
            else mbar_arrive(acc_empty(b));
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
    } else {
        // One tile at a time for the whole cluster. The partial sums go to shared memory (the stages are idle by then), column by
        // column; then each block adds a share of the outputs over all blocks of the cluster. Every block passes every barrier, also
        // after a wait that gave up.
        int* part = (int*)(dynamic + (base - smem_addr(dynamic)));
        for (int t = first; t < tiles; t += step, acc++) {
            const Tile tile = tile_of<TN, CG>(p, before, t, 0, &hint);
            if (warp == 0) produce(tile);
            if (warp == 1) multiply(tile);
            if (warp >= 4) {
                const int b = acc & 1, quarter = warp & 3;
                const bool ok = mbar_wait(acc_full(b), (acc >> 1) & 1, &gave_up);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (ok)
                    for (int c0 = ((warp - 4) >> 2) * 16; c0 < tile.rows; c0 += 32) {
                        int v[16];
                        tmem_load(tmem + ((uint32_t)(quarter * 32) << 16) + b * TN + c0, v);
                        tmem_arrived();
#pragma unroll
                        for (int i = 0; i < 16; i++) part[(c0 + i) * CH + quarter * 32 + lane] = v[i];
                    }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(acc_empty(b));
            }
            rely();
            __syncwarp();
            cluster_sync();
            const int total = tile.rows * (CH / 4), lo = total * rank / splits, hi = total * (rank + 1) / splits;  // four channels at a time
            for (int i = lo + (int)threadIdx.x; i < hi; i += MM_THREADS) {
                int4 part_of[8];
#pragma unroll
                for (int r = 0; r < 8; r++) part_of[r] = r < splits ? cluster_load(base + 16 * i, r) : make_int4(0, 0, 0, 0);
                int sum[4] = {};
#pragma unroll
                for (int r = 0; r < 8; r++) sum[0] += part_of[r].x, sum[1] += part_of[r].y, sum[2] += part_of[r].z, sum[3] += part_of[r].w;
                const int chan = tile.chan + i % (CH / 4) * 4, row = tile.row + i / (CH / 4);
                const long long gc = (long long)tile.group * p.N + chan;
                const float sa = p.a_scale[row];
                T* y = (T*)p.y + (long long)row * p.ldy + chan;
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (chan + j < p.N) y[j] = from_f32<T>(scaled((float)sum[j], sa, p.w_scale[gc + j], p.bias ? p.bias[gc + j] : 0.f));
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
        if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::COLS));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::COLS));
    }
}

// ---------------------------------------------------------------- host
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                             CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encoder() {
    static const EncodeFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) f = nullptr;
        return (EncodeFn)f;
    }();
    return fn;
}

// Rows of `ld` bytes of which K count; a box is 128 bytes wide. What lies beyond K or beyond the rows reads as zero.
cudaError_t make_map(CUtensorMap* m, const void* at, long long rows, long long K, long long ld, int box_rows) {
    const EncodeFn fn = encoder();
    if (!fn) return cudaErrorNotSupported;
    const long long least = (K + 15) / 16 * 16;
    const cuuint64_t dim[2] = {(cuuint64_t)K, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)(ld > least ? ld : least)};
    const cuuint32_t box[2] = {KB, (cuuint32_t)box_rows}, one[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(at), dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

template <typename T, int TN, int CG> cudaError_t tiles_launch(const MatmulParams& q, int splits, cudaStream_t s) {
    using S = Shape<TN, CG>;
    TileParams p = {};
    p.ldy = q.ldy;
    p.a_scale = q.a_scale;
    p.w_scale = q.w_scale;
    p.bias = q.bias;
    p.offsets = q.offsets;
    p.y = q.y;
    p.status = q.status;
    p.M = (int)q.M;
    p.N = (int)q.N;
    p.groups = q.groups;
    p.k_blocks = (int)((q.K + KB - 1) / KB);
    p.n_tiles = (int)((q.N + CH * CG - 1) / (CH * CG));
    p.splits = splits;
    p.dependent = q.dependent;
    p.pairs = (uintptr_t)q.y % 4 == 0 && q.ldy % 2 == 0;
    cudaError_t e;
    if (q.K) {
        if ((e = make_map(&p.a, q.a, q.M, q.K, q.lda, S::BOX)) != cudaSuccess) return e;
        if ((e = make_map(&p.w, q.w, q.N * (q.groups ? q.groups : 1), q.K, q.ldw, CH)) != cudaSuccess) return e;
    }
    static std::atomic<bool> ready[64];  // by device; setting it twice does no harm
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev]) {
        e = cudaFuncSetAttribute(hccl_matmul_i8_tiles<T, TN, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev] = true;
    }
    const long long tiles = (long long)p.n_tiles * ((q.M + TN - 1) / TN + q.groups);  // at most, with groups
    const int team = CG == 2 ? 2 : splits;
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
    return cudaLaunchKernelEx(&cfg, hccl_matmul_i8_tiles<T, TN, CG>, p);
}

// Which tile. Tiles of TN tokens and a cluster of S blocks for each, by an estimate in microseconds fitted to measurements on shapes from 16 x 8192 x 4096 to 2048^3 (measured against
// every other choice on 14 of them, TN,S: 16 x 8192 x 4096 takes 10.8 us with its 16,1 and 15.1 with 32,4; 16 x 2048 x 4096 6.7 with 16,4, the best is 6.6 with 32,4, 16,1 takes 9.9; 128 x 2048 x 8192 11.4 with 64,4 and 17.2
// with 64,1; 512 x 4096 x 4096 12.9 with 128,1 and 16.4 with 256,1; 997 x 4104 x 2064 13.7 with 256,1 and 18.3 with 128,1; nowhere is the choice more than 6 % behind the best):
// rounds of the blocks over the tiles, times the stages of one, times a stage's time (0.15 while fetching is the bound, 0.27 for a
// pair's 2 x 512 cycles of products), and what does not overlap: the last tile's results and the cluster's exchange. One round of a cluster may take 128 blocks at most: more
// than that do not find their neighbouring SMs free at once (measured: 16 x 8192 x 4096 with S = 4, 256 blocks, 15.2 us against 11.4 with S = 2).
struct Choice {
    int tn, splits;
};
Choice choose(const MatmulParams& p) {
    const double k_blocks = (double)((p.K + KB - 1) / KB);
    if (p.groups) {
        // Groups are uneven: tiles of twice the mean number of rows hold most groups whole, so that weights are read once
        // (64 groups, 512 rows, 2048 x 4096: 80 us with 16 to 64, 83 with 256; 4096 rows: 91 with 128, 128 with 32).
        const long long twice = 2 * ((p.M + p.groups - 1) / p.groups);
        return {twice <= 16 ? 16 : twice <= 32 ? 32 : twice <= 64 ? 64 : twice <= 128 ? 128 : 256, 1};
    }
    static const struct {
        int tn;
        double stage, last, exchange;
    } option[] = {{16, 0.15, 0.0, 1.0}, {32, 0.15, 0.1, 1.5}, {64, 0.16, 0.4, 2.4}, {128, 0.20, 1.2, 0}, {256, 0.27, 3.0, 0}};
    Choice best = {256, 1};
    double least = 1e30;
    for (const auto& o : option) {
        const bool pair = o.tn == 256;
        const long long tiles = (p.M + o.tn - 1) / o.tn * ((p.N + (pair ? 2 * CH : CH) - 1) / (pair ? 2 * CH : CH)), at_once = pair ? SMS / 2 : SMS;
        for (int s = 1; s <= (o.tn <= 64 ? 8 : 1); s *= 2) {
            if (s > 1 && (tiles * s > (s == 8 ? 64 : 128) || k_blocks < 4 * s)) break;
            const double t = (double)((tiles + at_once - 1) / at_once) * (k_blocks / s) * o.stage + o.last + (s > 1 ? o.exchange : 0);
            if (t < least) least = t, best = {o.tn, s};
        }
    }
    return best;
}

template <typename T> cudaError_t matmul_launch(const MatmulParams& p, cudaStream_t s) {
    const Choice c = choose(p);
    switch (c.tn) {
        case 16: return tiles_launch<T, 16, 1>(p, c.splits, s);
        case 32: return tiles_launch<T, 32, 1>(p, c.splits, s);
        case 64: return tiles_launch<T, 64, 1>(p, c.splits, s);
        case 128: return tiles_launch<T, 128, 1>(p, 1, s);
        default: return tiles_launch<T, 256, 2>(p, 1, s);
    }
}

}  // namespace

cudaError_t launch_matmul_i8(int dt, const MatmulParams& p, cudaStream_t s) {
    if (p.M == 0 || p.N == 0) return cudaSuccess;
    if (few_rows(p)) return launch_matmul_i8_few(dt, p, s);
    if (dt == HCCL_FP32) return matmul_launch<float>(p, s);
    if (dt == HCCL_BF16) return matmul_launch<__nv_bfloat16>(p, s);
    return matmul_launch<__half>(p, s);
}

}  // namespace experts
}  // namespace hccl
