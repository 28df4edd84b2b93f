// A whole expert layer for a few tokens in two kernels: y[t] = sum over j of w[t, j] down_e(act(up_e(x[t]))), weights in 4-bit floating point, activations as numbers of 22 bits.
//
// With few tokens the chosen experts' weights are read once and that is the time, so 4-bit activations would save nothing and cost accuracy. The tensor cores multiply 4-bit
// numbers by 4-bit numbers all the same: an activation goes in as the sum of eight of them. 1024 elements of a row (or what there is) are brought to whole numbers below 2^22 by a power of
// two, which leaves less than 2^-22 of their largest, and written with eight digits from -4 to 3 in base 8; half a digit is an e2m1 number, and its scale, a power of 8, the same for all blocks.
// Fewer bits than a 32-bit number's own, by choice: beside a row's largest element the others lose what a 32-bit sum with its product loses four times over (2^-22 of it against 2^-24), and more digits would
// be more columns. Four digits span what one byte's scale can: the last four columns have the scales of the first four again, and their sum 8^-4 of the weight. Eight columns is also the least that an
// instruction computes: a token's eight digits are its eight columns, and for one token they cost nothing. The sum over them is taken in 32 bits.
//
// Rows in expert order are taken in chunks of at most 8 rows of one expert. Both kernels run one block to an SM, and weights never wait for anything but room:
//
//   up    units of 128 channels x `span` stages of 256 elements of K x a chunk, in the order [chunk][1024 columns of the activated rows][part of K][channels]; every block takes an equal run
//         of them. For each chunk and part of K a block makes the pieces itself, one part ahead; a unit's sums go to memory, one 32-bit partial sum for each part of K. At its end a block counts its
//         units; whoever counts the last one of 1024 columns adds up their parts in their order, applies the activation and makes the pieces for the second kernel.
//   down  stages in the order [128 channels][chunk][K], every block an equal run of them. A chunk's sums over 1024 of K stay in tensor memory; weighted, they are added up in
//         shared memory over the chunks, [token][channel]. Where the channels' run ends within a block its sums are the result; otherwise the blocks that share the channels leave
//         partial sums, and whoever counts the last stage adds these up in the blocks' order.
//
// All sums have a fixed order: results repeat bit for bit.
//
// Measured (B200, copy peak 6.5 TB/s): one token through 8 of 64 experts of 4096 x 2048 35 us in replays of a graph, 45 to 47 after a flush of the caches; 8 experts of 8192 x 8192, one token 103 + 53 us
// = 5.9 TB/s of weights and 8 tokens 133 + 55; 19 tokens through 4 of 60 experts of 2056 x 1416 68 us. With many tokens and few channels the second kernel's last sums are the time: 50 tokens through 2 of
// 8 experts of 128 x 192 17 + 90 us. Of the 35 us the weights take 17 at the copy rate. The rest are latencies in a row: 5 until the first pieces are
// there, 1.5 to count, 5 for a block to finish others' sums, 3 to the second kernel's first product, 4 for its last sums, and a memory set and two launches.
#include <algorithm>
#include <atomic>

#include "activate.cuh"
#include "fp4.cuh"
#include "tensor.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int CH = 128, ROWS = 8 /* of a chunk */, PIECES = 8, SPAN = 4 /* stages of K in a part at most, of the second product in every one */, WIDE = SPAN * 256, GROUP = WIDE / CH /* channel tiles of a half in 1024 columns */, COLS = 512;
constexpr int TN = ROWS * PIECES;
constexpr float LATER = 4096.f;  // what the last half of the pieces is larger by
constexpr int ENOUGH = 6;  // units for each block, below which K is cut finer
constexpr int EACH = 8;  // elements of a thread that makes pieces
static_assert(ROWS * WIDE % EACH == 0, "");
constexpr int UP_THREADS = 512, SPLIT_WARPS = 8, SPLITTERS = 32 * SPLIT_WARPS, TASKS = ROWS * SPAN * 256 / EACH / SPLITTERS;
constexpr int DOWN_THREADS = 512;  // 8 warps at work, all of them in the last sums
constexpr int MAX_CHUNKS = HCCL_MAX_FEW_TOKENS * HCCL_MAX_TOP_K, OWN = (MAX_CHUNKS + SMS - 1) / SMS + 2;  // chunks in all, and in one block's run of the first kernel

template <int FORMAT> struct Shape {
    static constexpr int ATOMS = stage_atoms(FORMAT);
    static constexpr int STAGES = 7;
    // up: the ring of weights, two parts' pieces, and elements between their row's maximum and their pieces
    static constexpr int STAGE = CH * KB + ATOMS * ATOM;
    static constexpr int PIECE_STAGE = TN * KB, PART = SPAN * PIECE_STAGE;
    static constexpr int RING = STAGES * STAGE;
    static constexpr int HELD = ROWS * WIDE * 4;
    static constexpr int SMEM_UP = RING + 2 * PART + HELD + 1024;
    static_assert(STAGE % 1024 == 0 && PART % 1024 == 0, "operands start on 1024-byte boundaries");
    // down: a stage of weights, their scales, pieces; then [token][channel]
    static constexpr int D_STAGE = STAGE + PIECE_STAGE, D_SUMS = STAGES * D_STAGE;
    static constexpr int SMEM_DOWN = D_SUMS + HCCL_MAX_FEW_TOKENS * CH * 4 + 1024;
    // tensor memory: two accumulators, the pieces' scales, the stages' scales
    static constexpr int X_SCALES = 2 * TN, W_SCALES = X_SCALES + 4;
    static_assert(W_SCALES + STAGES * 4 * ATOMS <= COLS, "tensor memory");
};

struct FewParams {
    CUtensorMap w, w_scale, x;  // the last: down
    const void* in;        // up: [T, K] in T
    void* y;               // down: [T, N]
    float* sums;           // up: partial sums [part of K][row][width]
    uint8_t* pieces;       // [row][8][pitch]
    float* unscale;        // [row][part of the second product's K]
    float* part;           // down: two tiles of partial sums for each block, [token][channel]
    int *chunk_count, *tile_count;
    long long ldx, ldy, pitch;
    const int *offsets, *source;
    const float *weights, *wide, *bias;
    int* status;
    int K, N, I, k_blocks, down_parts /* parts of the second product's K */;
    int chan_tiles;        // up: of a half; down: of all channels
    int experts, top_k, T, rows /* T * top_k */, act, gated, half /* I, up to a multiple of 8 */, width /* of a row of sums: half, or both halves */, vec;
};

// How many stages of K a unit has at most, so that there are enough units to share out evenly. (The scratch's size goes by it.)
__device__ __forceinline__ int span_of(int chunks, int tiles, int k_blocks, int blocks) {
    int shift = 2;
    static_assert(SPAN == 1 << 2, "a shift");
    while (shift && (long long)chunks * tiles * ((k_blocks + (1 << shift) - 1) >> shift) < (long long)ENOUGH * blocks) shift--;
    return 1 << shift;
}
// a / b for numbers that are not negative and a quotient below 2^20: from an approximate one, off by one at most. Where a block's run begins hangs on ten divisions in a
// row, and a division in whole numbers takes 40 instructions, of 64 bits 150.
template <typename A> __device__ __forceinline__ int divide(A a, A b) {
    const int q = (int)__fdividef((float)a, (float)b);
    const A left = a - (A)q * b;
    return left < 0 ? q - 1 : left >= b ? q + 1 : q;
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

// What 1024 elements with this largest magnitude are multiplied with, a power of two, to become whole numbers below 2^22; and what half a digit of the first columns' scales stands for.
__device__ __forceinline__ void row_factor(unsigned top, float* factor, float* back) {
    const int e = (int)(top >> 23) - 127, up = min(21 - e, 126);  // (numbers near the smallest are cut at 2^-127)
    *factor = __uint_as_float((unsigned)(127 + up) << 23);
    *back = top >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : __uint_as_float((unsigned)(127 + 16 - up) << 23);  // 2 * 8^5 / factor
}
// The scale of piece q, as stored, four times: 64, 8, 1, 1/8, and again.
template <int FORMAT> __device__ __forceinline__ unsigned piece_scale(int q) {
    const unsigned e = 6 - 3 * (q & 3), byte = FORMAT == HCCL_NVFP4 ? (e + 7) << 3 : e + 127;
    return byte * 0x01010101u;
}
// Eight neighbouring elements to eight pieces of them; piece q's codes go to codes + q * pitch, there to the sixteen bytes number (sixteen ^ (q & swizzle)).
// One function for all places, since code that a warp passes for the first time is fetched line by line.
__device__ __noinline__ void make_pieces(float4 lo, float4 hi, float factor, char* codes, long long pitch, int sixteen, int swizzle) {
    const float v[EACH] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    unsigned a[EACH];
#pragma unroll
    for (int j = 0; j < EACH; j++) {
        // 1.5 * 2^23 + n has the whole number n in its low bits; with 44444444 in base 8 added, digit + 4 in every three of them.
        unsigned x = __float_as_uint(__fmaf_rn(v[j], factor, 12582912.f)) - 0x4b400000u + 044444444u;
        x = (x & 0xfffu) | (x << 4 & 0x0fff0000u);  // three bits to four
        x = (x & 0x003f003fu) | (x << 2 & 0x3f003f00u);
        x = (x & 0x07070707u) | (x << 1 & 0x70707070u);
        const unsigned n = ~x >> 2 & 0x11111111u;     // 1 where the digit is negative
        a[j] = ((x & 0x33333333u) ^ (n * 3)) + n * 9;  // half the digit: 0 .. 3 stay, -1 .. -4 become 9 .. 12
    }
    // Eight words of an element's eight digits to eight words of eight elements' digit.
    unsigned b[EACH];
#pragma unroll
    for (int j = 0; j < 4; j++) b[j] = __byte_perm(a[j], a[j + 4], 0x5410), b[j + 4] = __byte_perm(a[j], a[j + 4], 0x7632);
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
        for (int j = 0; j < 2; j++) a[4 * h + j] = __byte_perm(b[4 * h + j], b[4 * h + j + 2], 0x6240), a[4 * h + j + 2] = __byte_perm(b[4 * h + j], b[4 * h + j + 2], 0x7351);
#pragma unroll
    for (int h = 0; h < 4; h++) {  // a[2 h]: digits 2 h and 2 h + 1 of the even elements, a[2 h + 1]: of the odd ones
        const unsigned even = a[2 * h], odd = a[2 * h + 1];
        const int q = PIECES - 1 - 2 * h;  // the first piece is the highest digit
        *(unsigned*)(codes + q * pitch + (sixteen ^ (q & swizzle)) * 16) = (even & 0x0f0f0f0fu) | (odd << 4 & 0xf0f0f0f0u);
        *(unsigned*)(codes + (q - 1) * pitch + (sixteen ^ ((q - 1) & swizzle)) * 16) = (even >> 4 & 0x0f0f0f0fu) | (odd & 0xf0f0f0f0u);
    }
}
__device__ __forceinline__ void prefetch(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) { asm volatile("prefetch.tensormap [%0];" ::"l"(m)); }
// The eight columns of a row's pieces, as the products come out, to one sum: the smallest first.
__device__ __forceinline__ float sum_of_pieces(const float (&v)[8]) {
    float s = (((v[7] + v[6]) + v[5]) + v[4]) * (1.f / LATER);
#pragma unroll
    for (int i = 3; i >= 0; i--) s += v[i];
    return s;
}
// Chunks by expert, by one warp: each(chunk, packed) for every one. Returns how many.
struct Chunk {
    int expert, row, rows;  // rows [row, row + rows) in expert order
};
static_assert(OWN <= 32, "a lane each");
static_assert(HCCL_MAX_EXPERTS <= 1 << 11 && HCCL_MAX_FEW_TOKENS * HCCL_MAX_TOP_K <= 1 << 12 && ROWS < 1 << 4, "packed");
__device__ __forceinline__ int packed(int expert, int row, int rows) { return expert << 16 | row << 4 | rows; }
__device__ __forceinline__ Chunk unpacked(int c) {
    c = __shfl_sync(0xffffffffu, c, 0);  // (the same in all lanes, and by way of the shuffle known to be)
    return {c >> 16, c >> 4 & 0xfff, c & 15};
}
// Rows in expert order that have an expert. They may begin later than row 0 (an expert's share of a larger routing).
__device__ __forceinline__ int first_row(const FewParams& p) { return min(p.rows, max(0, p.offsets[0])); }
__device__ __forceinline__ int end_row(const FewParams& p) { return min(p.rows, max(0, p.offsets[p.experts])); }
template <typename Each> __device__ __forceinline__ int list_chunks(const FewParams& p, int lane, const Each& each) {
    int run = 0;
    const int first = first_row(p), end = end_row(p);
    for (int b = 0; b < p.experts; b += 32) {
        const int g = b + lane;
        int lo = 0, hi = 0;
        if (g < p.experts) lo = max(first, p.offsets[g]), hi = min(end, p.offsets[g + 1]);
        const int n = max(0, (hi - lo + ROWS - 1) / ROWS);
        int inc = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += v;
        }
        for (int i = 0; i < n; i++) each(run + inc - n + i, packed(g, lo + i * ROWS, min(ROWS, hi - lo - i * ROWS)));
        run += __shfl_sync(0xffffffffu, inc, 31);
    }
    return run;
}
__device__ __forceinline__ uint32_t instruction(int rows, int format) {  // e2m1 operands, 128 channels, rows * 8 columns
    return (1u << 7) | (1u << 10) | ((uint32_t)rows << 17) | (format == HCCL_MXFP4 ? 1u << 23 : 0u) | (1u << 27);
}
// After a wait that gave up, loads may still be in flight: wait (with a limit) for the stages that were issued.
template <typename Full> __device__ __forceinline__ void drain(const Full& full, int stages, int it, int* status) {
    const unsigned long long t0 = now_ns();
    for (int i = max(0, it - stages); i < it; i++)
        while (!mbar_try(full(i % stages), (i / stages) & 1) && now_ns() - t0 < WAIT_NS) {}
    __nanosleep(1000000);  // and the instructions issued last, which end by themselves
    if (status) *status = HCCL_ERR_TIMEOUT;
}

// Four elements of act(gate) * other from partial sums, `apart` fours apart; other: how far the other half is, 0: no gate.
__device__ __forceinline__ float4 activated(const float4* from, long long apart, int other, int parts, int act) {
    float4 g = make_float4(0.f, 0.f, 0.f, 0.f), o = g;
    if (from)
#pragma unroll 1
        for (int kc = 0; kc < parts; kc += 4) {
            float4 x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                x[i] = y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (kc + i < parts) x[i] = __ldcg(from + (kc + i) * apart), y[i] = __ldcg(from + (kc + i) * apart + other);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                g.x += x[i].x, g.y += x[i].y, g.z += x[i].z, g.w += x[i].w;
                o.x += y[i].x, o.y += y[i].y, o.z += y[i].z, o.w += y[i].w;
            }
        }
    if (!other) o = make_float4(1.f, 1.f, 1.f, 1.f);
    if (act == HCCL_ACT_SILU) g.x = activation(HCCL_ACT_SILU, g.x), g.y = activation(HCCL_ACT_SILU, g.y), g.z = activation(HCCL_ACT_SILU, g.z), g.w = activation(HCCL_ACT_SILU, g.w);
    else if (act == HCCL_ACT_GELU) g.x = activation(HCCL_ACT_GELU, g.x), g.y = activation(HCCL_ACT_GELU, g.y), g.z = activation(HCCL_ACT_GELU, g.z), g.w = activation(HCCL_ACT_GELU, g.w);
    else g.x = activation(HCCL_ACT_RELU, g.x), g.y = activation(HCCL_ACT_RELU, g.y), g.z = activation(HCCL_ACT_RELU, g.z), g.w = activation(HCCL_ACT_RELU, g.w);
    return make_float4(g.x * o.x, g.y * o.y, g.z * o.z, g.w * o.w);
}

// ---------------------------------------------------------------- first product, activation, pieces
// Where a block is in its run of units. index: among the `of` units with the same chunk, part and kc.
struct Unit {
    Chunk c;
    int u, chunk, part /* of the second product's K */, kc, half /* gate or other */, tile /* of the half */, index, of, group;
};

// Roles (16 warps): warp 0 loads weights, warp 1 copies scales to tensor memory and issues the products, warp 2 owns the tensor memory, warp 3 lists the chunks, warps 4-7 take
// the sums out, warps 8-15 make the pieces.
template <typename T, int FORMAT> __global__ void __launch_bounds__(UP_THREADS, 1) hccl_few_up(const __grid_constant__ FewParams p) {
    using S = Shape<FORMAT>;
    extern __shared__ char dynamic[];
    __shared__ __align__(8) unsigned long long bars[2 * S::STAGES + 8];
    __shared__ __align__(16) unsigned scale_atom[ATOM / 4];  // of the pieces: the same for all blocks
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up, completed;
    __shared__ int chunk_total, table[OWN];
    __shared__ float unscale[2][ROWS];
    __shared__ unsigned top_of[2][ROWS];
    __shared__ int job_row[ROWS], job_part[ROWS];
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_addr(dynamic) + 1023) & ~1023u;
    char* const parts = dynamic + (base - smem_addr(dynamic)) + S::RING;
    float4* const held = (float4*)(parts + 2 * S::PART);
    const uint32_t bar0 = smem_addr(bars);
    const auto full = [&](int s) { return bar0 + 8 * s; };
    const auto empty = [&](int s) { return bar0 + 8 * (S::STAGES + s); };
    const auto acc_full = [&](int b) { return bar0 + 8 * (2 * S::STAGES + b); };
    const auto acc_empty = [&](int b) { return bar0 + 8 * (2 * S::STAGES + 2 + b); };
    const auto part_full = [&](int b) { return bar0 + 8 * (2 * S::STAGES + 4 + b); };
    const auto part_empty = [&](int b) { return bar0 + 8 * (2 * S::STAGES + 6 + b); };

    if (threadIdx.x == 32) prefetch_map(&p.w), prefetch_map(&p.w_scale);
    asm volatile("griddepcontrol.launch_dependents;");  // the second kernel's blocks may start to fetch weights as this one's leave
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; s++) mbar_init(full(s), 1), mbar_init(empty(s), 1);
        for (int b = 0; b < 2; b++) mbar_init(acc_full(b), 1), mbar_init(acc_empty(b), 4), mbar_init(part_full(b), SPLIT_WARPS), mbar_init(part_empty(b), 5);
        gave_up = 0;
        completed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x < 2 * ROWS) top_of[threadIdx.x / ROWS][threadIdx.x % ROWS] = 0;
    if (threadIdx.x < 128) {
        scale_atom[atom_row((int)threadIdx.x) / 4] = piece_scale<FORMAT>((int)threadIdx.x % PIECES);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_at)), "n"(COLS));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    constexpr int blocks = SMS;
    if (warp >= 8) {
        // While the chunks are listed: what comes first from memory is asked for, a share by each block, and the code that makes pieces is fetched by running it (one token through 8 of 64
        // experts of 4096 x 2048 35.6 us, without 36.9).
        const int lines = (p.K * (int)sizeof(T) + 127) / 128;  // of a row (one that begins between two reaches into one more: that is fetched when it is needed)
        for (int i = (int)(blockIdx.x * SPLITTERS + threadIdx.x) - 256; i < lines * p.T; i += blocks * SPLITTERS) {
            const int t = divide(i, lines);
            prefetch((const char*)p.in + t * p.ldx * (long long)sizeof(T) + (i - t * lines) * 128);
        }
        if (blockIdx.x * SPLITTERS + threadIdx.x - 256 < p.rows) prefetch(p.source + (blockIdx.x * SPLITTERS + threadIdx.x - 256));
        make_pieces(make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f), 0.f, (char*)(held + threadIdx.x - 256), SPLITTERS * 16, 0, 0);
    }
    if (warp == 3) {
        // Chunks of a block's run: every chunk has the same number of units, so the run begins in chunk floor(chunks * block / blocks).
        int* const all = (int*)parts;  // (free until the first pieces)
        const int n = min(p.rows, list_chunks(p, lane, [&](int chunk, int c) {
            if (chunk < p.rows) all[chunk] = c;  // (never more than rows, if the offsets ascend)
        }));
        __syncwarp();
        const int own = n * (int)blockIdx.x / blocks;
        if (lane < OWN && own + lane < n) table[lane] = all[own + lane];
        if (lane == 0) chunk_total = n;
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_at, 0);
    const int chunks = __shfl_sync(0xffffffffu, chunk_total, 0), own = chunks * (int)blockIdx.x / blocks;
    const int halves = p.gated ? 2 : 1, span = span_of(chunks, halves * p.chan_tiles, p.k_blocks, blocks), parts_of_k = divide(p.k_blocks + span - 1, span);
    const int of_chunk = parts_of_k * halves * p.chan_tiles, of_part = parts_of_k * halves * GROUP;  // units; a chunk's last part may have fewer
    const long long units = (long long)chunks * of_chunk;
    const int u0 = (int)(units * blockIdx.x / blocks), u1 = (int)(units * (blockIdx.x + 1) / blocks);
    // Rows that have sums: how far apart the parts of K lie. Chunks of 8 hold them all, whatever the offsets are (they telescope), which is what the scratch's size goes by.
    const int first = first_row(p), filled = max(0, end_row(p) - first);

    const auto uniform = [](int v) { return __shfl_sync(0xffffffffu, v, 0); };
    const auto place = [&](Unit& t) { t.half = t.index >= t.group, t.tile = t.part * GROUP + t.index - t.half * t.group; };
    const auto in_part = [&](Unit& t) { t.group = min(GROUP, p.chan_tiles - t.part * GROUP), t.of = halves * t.group; };
    const auto unit_at = [&](int u) {
        Unit t = {};
        t.u = u;
        if (u >= u1) return t;
        t.chunk = uniform(divide(u, of_chunk));
        t.c = unpacked(table[t.chunk - own]);
        int rest = u - t.chunk * of_chunk;
        t.part = uniform(divide(rest, of_part));
        in_part(t);
        rest -= t.part * of_part;
        t.kc = uniform(divide(rest, t.of));
        t.index = uniform(rest - t.kc * t.of);
        place(t);
        return t;
    };
    const auto advance = [&](Unit& t) {
        t.u++;
        if (++t.index == t.of) {
            t.index = 0;
            if (++t.kc == parts_of_k) {
                t.kc = 0;
                if (++t.part == p.down_parts) {
                    t.part = 0;
                    t.chunk++;
                    if (t.u < u1) t.c = unpacked(table[t.chunk - own]);
                }
                in_part(t);
            }
        }
        place(t);
    };
    // With one part of K a chunk's pieces serve all its units.
    const auto begins = [&](const Unit& t) { return t.u == u0 || (t.index == 0 && (parts_of_k > 1 || t.part == 0)); };
    const auto ends = [&](const Unit& t) { return t.u == u1 - 1 || (t.index == t.of - 1 && (parts_of_k > 1 || t.part == p.down_parts - 1)); };
    const auto stage_of = [&](int kc) { return divide(p.k_blocks * kc, parts_of_k); };  // the first of a part of K; parts differ by one stage at most
    const auto stages_of = [&](int kc) { return stage_of(kc + 1) - stage_of(kc); };
    int it = 0, acc = 0, turn = 0;  // stages, units and parts of K passed

    if (warp == 0) {
        for (Unit t = unit_at(u0); t.u < u1; advance(t)) {
            const int n = stages_of(t.kc), kb0 = stage_of(t.kc);
            for (int i = 0; i < n; i++, it++) {
                const int s = it % S::STAGES, kb = kb0 + i;
                if (!mbar_wait(empty(s), ((it / S::STAGES) & 1) ^ 1, &gave_up)) break;
                if (elected()) {
                    const uint32_t at = base + s * S::STAGE;
                    mbar_expect(full(s), S::STAGE);
                    tma_load<1>(at, &p.w, kb * KB, t.c.expert * p.N + t.half * p.I + t.tile * CH, full(s));
                    tma_load<1>(at + CH * KB, &p.w_scale, 0, (((t.c.expert * halves + t.half) * p.chan_tiles + t.tile) * p.k_blocks + kb) * S::ATOMS, full(s));
                }
                __syncwarp();
            }
            if (*(volatile int*)&gave_up) break;
        }
    } else if (warp == 1) {
        const int steps = (p.K + 63) / 64;
        bool ok = true;
        if (elected()) copy_scales(tmem + S::X_SCALES, smem_addr(scale_atom));
        __syncwarp();
        for (Unit t = unit_at(u0); t.u < u1 && ok; advance(t), acc++) {
            const int n = stages_of(t.kc), kb0 = stage_of(t.kc), b = acc & 1, half = turn & 1;
            const uint32_t pieces = base + S::RING + half * S::PART;
            const uint32_t desc = instruction(t.c.rows, FORMAT);
            if (begins(t)) {
                ok = mbar_wait(part_full(half), (turn >> 1) & 1, &gave_up);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            }
            ok = mbar_wait(acc_empty(b), ((acc >> 1) & 1) ^ 1, &gave_up);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (int i = 0; i < n; i++, it++) {
                const int s = it % S::STAGES, left = min(4, steps - 4 * (kb0 + i));
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
                        mma_fp4<FORMAT>(tmem + b * TN, w + 2 * k, x + 2 * k, desc | (two << 4) | (two << 29), scales + 4 * a, tmem + S::X_SCALES, (i > 0 || k > 0) ? 1u : 0u);
                    }
                    mma_commit<1>(empty(s));
                    if (i == n - 1) {
                        mma_commit<1>(acc_full(b));
                        if (ends(t)) mma_commit<1>(part_empty(half));
                    }
                }
                __syncwarp();
            }
            if (ends(t)) turn++;
        }
    } else if (warp >= 4 && warp < 8) {
        const int quarter = warp & 3;
        bool ok = true;
        for (Unit t = unit_at(u0); t.u < u1 && ok; advance(t), acc++) {
            const int b = acc & 1, half = turn & 1, chan = t.tile * CH + quarter * 32 + lane;
            const bool in = chan < p.I;
            const float wide = p.wide[t.c.expert], bias = (in && p.bias && t.kc == 0) ? p.bias[(long long)t.c.expert * p.N + t.half * p.I + chan] : 0.f;
            ok = mbar_wait(part_full(half), (turn >> 1) & 1, &gave_up) && mbar_wait(acc_full(b), (acc >> 1) & 1, &gave_up);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            float sums[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; r++) {
                if (r >= t.c.rows) break;
                float v[8];
                __syncwarp();
                tmem_load8(tmem + ((uint32_t)(quarter * 32) << 16) + b * TN + r * PIECES, v);
                tmem_arrived();
                sums[r] = fmaf(sum_of_pieces(v), unscale[half][r] * wide, bias);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(acc_empty(b));
                if (ends(t)) mbar_arrive(part_empty(half));
            }
            if (ends(t)) turn++;
            float* out = p.sums + ((long long)t.kc * filled + t.c.row - first) * p.width + t.half * p.half + chan;
            if (in)
#pragma unroll
                for (int r = 0; r < ROWS; r++)
                    if (r < t.c.rows) __stcg(out + (long long)r * p.width, sums[r]);
        }
        __threadfence();  // the sums are out before this block counts its units
    } else if (warp >= 8) {
        const int me = (int)threadIdx.x - 256;
        bool ok = true;
        for (int u = u0, next; u < u1 && ok; u = next, turn++) {
            const Unit t = unit_at(u);
            next = parts_of_k > 1 ? u + t.of - t.index : (t.chunk + 1) * of_chunk;
            const int half = turn & 1, k0 = stage_of(t.kc) * 256, wide = stages_of(t.kc) * 256 / EACH;  // threads to a row
            char* const part = parts + half * S::PART;
            // A thread's elements, eight at a time, are those of task i of (row, eight elements), i = me, me + 256, ...
            const auto row_of = [&](int i) { return divide(me + i * SPLITTERS, wide); };
            const auto k_of = [&](int i, int r) { return k0 + (me + i * SPLITTERS - r * wide) * EACH; };
#pragma unroll 1
            for (int i = 0; i < TASKS; i++) {
                const int r = row_of(i), k = k_of(i, r);
                if (r >= t.c.rows) break;
                float v[EACH];
                const int from = p.source[t.c.row + r];
                load8<T>((const T*)p.in + (long long)divide(max(from, 0), p.top_k) * p.ldx, k, (unsigned)from < (unsigned)p.rows ? p.K : 0, p.vec, v);
                unsigned top = 0;  // the largest magnitude of each row's part of K
#pragma unroll
                for (int j = 0; j < EACH; j++) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
                top = __reduce_max_sync(0xffffffffu, top);
                if (lane == 0) atomicMax(&top_of[half][r], top);
                held[2 * i * SPLITTERS + me] = make_float4(v[0], v[1], v[2], v[3]);
                held[(2 * i + 1) * SPLITTERS + me] = make_float4(v[4], v[5], v[6], v[7]);
            }
            // (the buffers' last readers)
            ok = mbar_wait(part_empty(half), ((turn >> 1) & 1) ^ 1, &gave_up);
            ok = all_of(ok, 2, SPLITTERS);
            if (!ok) break;
#pragma unroll 1
            for (int i = 0; i < TASKS; i++) {
                const int r = row_of(i), k = k_of(i, r);
                if (r >= t.c.rows) break;
                float factor, back;
                row_factor(top_of[half][r], &factor, &back);
                if (k == k0) unscale[half][r] = back;
                const int kk = k - k0, in_stage = kk % 256;
                make_pieces(held[2 * i * SPLITTERS + me], held[(2 * i + 1) * SPLITTERS + me], factor, part + kk / 256 * S::PIECE_STAGE + r * PIECES * KB + in_stage % 32 / 2, KB, in_stage / 32, 7);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(part_full(half));
            // everyone has read the maxima: they start at zero when this half's turn comes again
            asm volatile("bar.sync 2, 256;" ::: "memory");
            if (me < ROWS) top_of[half][me] = 0;
        }
    }
    if (warp == 0 && lane == 0 && *(volatile int*)&gave_up) drain(full, S::STAGES, it, p.status);
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLS));
    if (*(volatile int*)&gave_up || u0 >= u1) return;

    // The block counts its units, all at once; parts of chunks that are complete with them are its own to finish.
    int* const list = (int*)parts;  // (its last readers are done)
    const auto part_at = [&](int u) {
        const int chunk = divide(u, of_chunk);
        return chunk * p.down_parts + divide(u - chunk * of_chunk, of_part);
    };
    for (int i = part_at(u0) + (int)threadIdx.x; i <= part_at(u1 - 1); i += UP_THREADS) {
        const int chunk = divide(i, p.down_parts), lo = chunk * of_chunk + (i - chunk * p.down_parts) * of_part, hi = min(lo + of_part, (chunk + 1) * of_chunk);
        const int n = min(u1, hi) - max(u0, lo);
        if (atomicAdd(p.chunk_count + i, n) + n == hi - lo) list[atomicAdd(&completed, 1)] = i;
    }
    __threadfence();
    __syncthreads();
    // As many of them at once as have ROWS rows together: a row's 1024 columns are a job for 128 threads' eights.
    float4* const h = held;  // [job][four columns]
    for (int l = 0; l < completed;) {
        int jobs = 0;
        for (; l < completed; l++) {  // (all threads the same; one of them writes it down)
            const int chunk = divide(list[l], p.down_parts), part = list[l] - chunk * p.down_parts;
            const Chunk c = unpacked(table[chunk - own]);
            if (jobs + c.rows > ROWS) break;
            for (int r = 0; r < c.rows; r++, jobs++)
                if (threadIdx.x == 0) job_row[jobs] = c.row + r, job_part[jobs] = part, top_of[0][jobs] = 0;
        }
        __syncthreads();
        const auto columns = [&](int job, int* from) {  // up to the end of the last instruction's 64 elements
            *from = job_part[job] * WIDE;
            return (min(WIDE, p.I - *from) + 63) & ~63;
        };
#pragma unroll 1
        for (int i = (int)threadIdx.x; i < jobs * (WIDE / 4); i += UP_THREADS) {
            int from;
            const int job = i / (WIDE / 4), col = i % (WIDE / 4) * 4;
            if (col >= columns(job, &from)) continue;
            const int k = from + col;
            const float4 x = activated(k < p.half ? (const float4*)(p.sums + (long long)(job_row[job] - first) * p.width + k) : nullptr, (long long)filled * p.width / 4, p.gated ? p.half / 4 : 0, parts_of_k, p.act);
            float v[4] = {x.x, x.y, x.z, x.w};
            unsigned top = 0;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if (k + j >= p.I) v[j] = 0.f;
                top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
            }
            if (top) atomicMax(&top_of[0][job], top);
            h[i] = make_float4(v[0], v[1], v[2], v[3]);
        }
        __syncthreads();
#pragma unroll 1
        for (int i = (int)threadIdx.x; i < jobs * (WIDE / EACH); i += UP_THREADS) {
            int from;
            const int job = i / (WIDE / EACH), col = i % (WIDE / EACH) * EACH;
            if (col >= columns(job, &from)) continue;
            float factor, back;
            row_factor(top_of[0][job], &factor, &back);
            if (col == 0) p.unscale[(long long)job_row[job] * p.down_parts + job_part[job]] = back;
            make_pieces(h[2 * i], h[2 * i + 1], factor, (char*)p.pieces + (long long)job_row[job] * PIECES * p.pitch + (from + col) / 2, p.pitch, 0, 0);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- second product, weighted sums
// Where a block is in its run of stages: a segment has one chunk and one part of K. g1: where it ends.
struct Segment {
    Chunk c;
    int g, g1, chunk, tile, k0, k1;  // stages of K
};

// Roles (the first 8 of 16 warps): warp 0 loads weights and pieces, warp 1 copies scales to tensor memory and issues the products, warp 2 owns the tensor memory, warp 3 lists the chunks, warps 4-7 take
// the sums out.
template <typename T, int FORMAT> __global__ void __launch_bounds__(DOWN_THREADS, 1) hccl_few_down(const __grid_constant__ FewParams p) {
    using S = Shape<FORMAT>;
    extern __shared__ char dynamic[];
    __shared__ __align__(8) unsigned long long bars[2 * S::STAGES + 4];
    __shared__ __align__(16) unsigned scale_atom[ATOM / 4];  // of the pieces: the same for all blocks
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up, completed, list[2];
    __shared__ int chunk_total, table[MAX_CHUNKS];
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t base = (smem_addr(dynamic) + 1023) & ~1023u;
    float* const sums = (float*)(dynamic + (base - smem_addr(dynamic)) + S::D_SUMS);
    const uint32_t bar0 = smem_addr(bars);
    const auto full = [&](int s) { return bar0 + 8 * s; };
    const auto empty = [&](int s) { return bar0 + 8 * (S::STAGES + s); };
    const auto acc_full = [&](int b) { return bar0 + 8 * (2 * S::STAGES + b); };
    const auto acc_empty = [&](int b) { return bar0 + 8 * (2 * S::STAGES + 2 + b); };

    if (threadIdx.x == 32) prefetch_map(&p.w), prefetch_map(&p.w_scale), prefetch_map(&p.x);
    if (threadIdx.x >= 128 && threadIdx.x < 256)  // what the sums are weighted with, a share by each block
        for (int i = (int)(blockIdx.x * 128 + threadIdx.x - 128); i < p.rows; i += SMS * 128) prefetch(p.source + i), prefetch(p.weights + i);
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; s++) mbar_init(full(s), 1), mbar_init(empty(s), 1);
        for (int b = 0; b < 2; b++) mbar_init(acc_full(b), 1), mbar_init(acc_empty(b), 4);
        gave_up = 0;
        completed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x < 128) {
        scale_atom[atom_row((int)threadIdx.x) / 4] = piece_scale<FORMAT>((int)threadIdx.x % PIECES);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_at)), "n"(COLS));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (warp == 3) {
        const int n = list_chunks(p, lane, [&](int chunk, int c) {
            if (chunk < p.rows) table[chunk] = c;
        });
        if (lane == 0) chunk_total = min(p.rows, n);  // (never more than rows, if the offsets ascend)
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_at, 0);
    const int chunks = __shfl_sync(0xffffffffu, chunk_total, 0);
    constexpr int blocks = SMS;
    const int of_tile = chunks * p.k_blocks;
    const long long total = (long long)of_tile * p.chan_tiles;
    const auto first_of = [&](int block) { return (int)(total * block / blocks); };
    const int g0 = first_of((int)blockIdx.x), g1 = first_of((int)blockIdx.x + 1), first_tile = of_tile ? divide(g0, of_tile) : 0;

    const auto uniform = [](int v) { return __shfl_sync(0xffffffffu, v, 0); };
    const auto bound = [&](Segment& t) {
        t.k1 = min(min(p.k_blocks, (t.k0 / SPAN + 1) * SPAN), t.k0 + g1 - t.g);
        t.g1 = t.g + t.k1 - t.k0;
    };
    const auto first_segment = [&] {
        Segment t = {};
        t.g = g0;
        if (g0 >= g1) return t;
        t.tile = uniform(first_tile);
        const int rest = g0 - t.tile * of_tile;
        t.chunk = uniform(divide(rest, p.k_blocks));
        t.k0 = rest - t.chunk * p.k_blocks;
        t.c = unpacked(table[t.chunk]);
        bound(t);
        return t;
    };
    const auto advance = [&](Segment& t) {
        t.g = t.g1;
        t.k0 = t.k1;
        if (t.k0 == p.k_blocks) {
            t.k0 = 0;
            if (++t.chunk == chunks) t.chunk = 0, t.tile++;
            t.c = unpacked(table[t.chunk]);
        }
        bound(t);
    };
    int it = 0, acc = 0;  // stages and segments passed

    if (warp == 0) {
        const auto expect = [&](const Segment& t, int s) { mbar_expect(full(s), (uint32_t)(S::STAGE + t.c.rows * PIECES * KB)); };
        const auto load_w = [&](const Segment& t, int s, int kb) {
            const uint32_t at = base + s * S::D_STAGE;
            tma_load<1>(at, &p.w, kb * KB, t.c.expert * p.N + t.tile * CH, full(s));
            tma_load<1>(at + CH * KB, &p.w_scale, 0, ((t.c.expert * p.chan_tiles + t.tile) * p.k_blocks + kb) * S::ATOMS, full(s));
        };
        const auto load_x = [&](const Segment& t, int s, int kb) {
            const uint32_t at = base + s * S::D_STAGE;
            for (int r = 0; r < t.c.rows; r++) tma_load<1>(at + S::STAGE + r * PIECES * KB, &p.x, kb * KB, (t.c.row + r) * PIECES, full(s));
        };
        // The first stages' weights do not hang on the first kernel's results.
        const auto first = [&](const auto& each) {
            int n = 0;
            for (Segment t = first_segment(); t.g < g1 && n < S::STAGES; advance(t)) {
                for (int kb = t.k0; kb < t.k1 && n < S::STAGES; kb++, n++)
                    if (elected()) each(t, n, kb);
                __syncwarp();
            }
            return n;
        };
        const int pre = first([&](const Segment& t, int s, int kb) {
            expect(t, s);
            load_w(t, s, kb);
        });
        asm volatile("griddepcontrol.wait;" ::: "memory");
        first(load_x);
        for (Segment t = first_segment(); t.g < g1; advance(t)) {
            for (int kb = t.k0; kb < t.k1; kb++, it++) {
                if (it < pre) continue;
                const int s = it % S::STAGES;
                if (!mbar_wait(empty(s), ((it / S::STAGES) & 1) ^ 1, &gave_up)) break;
                if (elected()) {
                    expect(t, s);
                    load_w(t, s, kb);
                    load_x(t, s, kb);
                }
                __syncwarp();
            }
            if (*(volatile int*)&gave_up) break;
        }
    } else if (warp == 1) {
        const int steps = (p.K + 63) / 64;
        bool ok = true;
        if (elected()) copy_scales(tmem + S::X_SCALES, smem_addr(scale_atom));
        __syncwarp();
        for (Segment t = first_segment(); t.g < g1 && ok; advance(t), acc++) {
            const int b = acc & 1;
            const uint32_t desc = instruction(t.c.rows, FORMAT);
            ok = mbar_wait(acc_empty(b), ((acc >> 1) & 1) ^ 1, &gave_up);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (int kb = t.k0; kb < t.k1; kb++, it++) {
                const int s = it % S::STAGES, left = min(4, steps - 4 * kb);
                ok = mbar_wait(full(s), (it / S::STAGES) & 1, &gave_up);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t at = base + s * S::D_STAGE, scales = tmem + S::W_SCALES + s * 4 * S::ATOMS;
                const uint64_t w = operand(at), x = operand(at + S::STAGE);
                if (elected()) {
#pragma unroll
                    for (int a = 0; a < S::ATOMS; a++) copy_scales(scales + 4 * a, at + CH * KB + a * ATOM);
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        if (k >= left) break;
                        const int a = k * S::ATOMS / 4;
                        const uint32_t two = FORMAT == HCCL_MXFP4 ? 2u * (k & 1) : 0u;
                        mma_fp4<FORMAT>(tmem + b * TN, w + 2 * k, x + 2 * k, desc | (two << 4) | (two << 29), scales + 4 * a, tmem + S::X_SCALES, (kb > t.k0 || k > 0) ? 1u : 0u);
                    }
                    mma_commit<1>(empty(s));
                    if (kb == t.k1 - 1) mma_commit<1>(acc_full(b));
                }
                __syncwarp();
            }
        }
    } else if (warp >= 4 && warp < 8) {
        const int quarter = warp & 3, me = quarter * 32 + lane;
        asm volatile("griddepcontrol.wait;" ::: "memory");
        for (int t = 0; t < p.T; t++) sums[t * CH + me] = 0.f;
        bool ok = true;
        // What a segment's sums are multiplied with, asked for one segment ahead: each lane below the number of rows holds one row's choice.
        struct Row {
            int token;
            float weight, back, wide, bias;
        };
        const auto row_of = [&](const Segment& t) {
            Row r = {-1, 0.f, 0.f, p.wide[t.c.expert], 0.f};  // (of no segment: nothing)
            if (p.bias && t.k0 == 0 && t.tile * CH + me < p.N) r.bias = p.bias[(long long)t.c.expert * p.N + t.tile * CH + me];
            if (lane < t.c.rows) {
                const int choice = p.source[t.c.row + lane];
                if ((unsigned)choice < (unsigned)p.rows) r.token = divide(choice, p.top_k), r.weight = p.weights[choice];
                r.back = __ldcg(p.unscale + (long long)(t.c.row + lane) * p.down_parts + t.k0 / SPAN);
            }
            return r;
        };
        Segment next = first_segment();
        Row row, next_row = row_of(next);
        while (next.g < g1 && ok) {
            const Segment t = next;
            row = next_row;
            advance(next);
            if (next.g < g1) next_row = row_of(next);
            const int b = acc & 1, chan = t.tile * CH + me;
            const bool in = chan < p.N;
            ok = mbar_wait(acc_full(b), (acc >> 1) & 1, &gave_up);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
            for (int r = 0; r < ROWS; r++) {
                if (r >= t.c.rows) break;
                float v[8];
                __syncwarp();
                tmem_load8(tmem + ((uint32_t)(quarter * 32) << 16) + b * TN + r * PIECES, v);
                tmem_arrived();
                const int to = __shfl_sync(0xffffffffu, row.token, r);
                const float z = fmaf(sum_of_pieces(v), __shfl_sync(0xffffffffu, row.back, r) * row.wide, row.bias), f = __shfl_sync(0xffffffffu, row.weight, r);
                if (to >= 0) sums[to * CH + me] = fmaf(f, z, sums[to * CH + me]);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty(b));
            acc++;
            if (t.g1 == g1 || t.g1 == (t.tile + 1) * of_tile) {  // the last of its channels here
                if (g0 <= t.tile * of_tile && t.g1 == (t.tile + 1) * of_tile) {
                    T* y = (T*)p.y + chan;
                    for (int i = 0; i < p.T; i++, y += p.ldy) {
                        if (in) *y = from_f32<T>(sums[i * CH + me]);
                        sums[i * CH + me] = 0.f;
                    }
                } else {
                    float* part = p.part + (long long)(2 * blockIdx.x + (t.tile == first_tile ? 0 : 1)) * p.T * CH + me;
                    for (int i = 0; i < p.T; i++, part += CH) {
                        __stcg(part, sums[i * CH + me]);
                        sums[i * CH + me] = 0.f;
                    }
                }
            }
        }
        __threadfence();  // the sums are out before this block counts its stages
    }
    if (warp == 0 && lane == 0 && *(volatile int*)&gave_up) drain(full, S::STAGES, it, p.status);
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLS));
    if (*(volatile int*)&gave_up) return;
    if (total == 0) {  // no token has an expert
        asm volatile("griddepcontrol.wait;" ::: "memory");
        for (long long i = (long long)blockIdx.x * DOWN_THREADS + threadIdx.x; i < (long long)p.T * p.N; i += (long long)blocks * DOWN_THREADS)
            ((T*)p.y)[i / p.N * p.ldy + i % p.N] = from_f32<T>(0.f);
        return;
    }
    if (threadIdx.x < 2 && g0 < g1) {  // the first and the last of this block's runs of channels, if others share them
        const int tile = threadIdx.x == 0 ? first_tile : divide(g1 - 1, of_tile), lo = max(g0, tile * of_tile), hi = min(g1, (tile + 1) * of_tile), n = hi - lo;
        if (n < of_tile && (threadIdx.x == 0 || tile != first_tile)) {
            if (atomicAdd(p.tile_count + tile, n) + n == of_tile) list[atomicAdd(&completed, 1)] = tile;
            __threadfence();
        }
    }
    __syncthreads();
    for (int i = warp; i < completed * p.T; i += DOWN_THREADS / 32) {
        const int token = divide(i, completed), tile = list[i - token * completed], chan = tile * CH + 4 * lane;
        const auto block_of_stage = [&](long long g) { return divide((g + 1) * blocks - 1, total); };
        const int from = block_of_stage((long long)tile * of_tile), to = block_of_stage((long long)(tile + 1) * of_tile - 1);
        float sum[4] = {};
#pragma unroll 8
        for (int b = from; b <= to; b++) {
            const int lo = first_of(b), which = lo >= tile * of_tile ? 0 : 1;
            const bool some = first_of(b + 1) > lo;  // (with fewer stages than blocks some have none)
            const float4 v = __ldcg((const float4*)(p.part + ((long long)(2 * b + which) * p.T + token) * CH) + lane);
            if (some) sum[0] += v.x, sum[1] += v.y, sum[2] += v.z, sum[3] += v.w;
        }
        T* y = (T*)p.y + (long long)token * p.ldy + chan;
#pragma unroll
        for (int c = 0; c < 4; c++)
            if (chan + c < p.N) y[c] = from_f32<T>(sum[c]);
    }
}

// ---------------------------------------------------------------- host
constexpr long long up_to(long long n, long long m) { return (n + m - 1) / m * m; }

// Floats of the first product's partial sums: [parts of K][rows][width]. With all SPAN stages to a unit there are that many parts; where span_of cuts finer, it does so because there
// are fewer than ENOUGH * SMS units of twice the size, each of 128 channels x at most 8 rows (width is at most 16 more than the channels).
long long partial_sums(long long rows, long long width, long long k_blocks) {
    const long long most = rows * k_blocks * width, fine = 2ll * ROWS * ENOUGH * SMS * (CH + 16), coarse = rows * ((k_blocks + SPAN - 1) / SPAN) * width;
    return std::max(coarse, std::min(most, fine));
}

struct Places {  // in the scratch, in bytes
    long long half, width, pitch, parts, counts, count_bytes, sums, unscale, pieces, part, end;
};
Places places(long long T, long long rows, long long H, long long I, int gated) {
    Places a;
    a.half = up_to(I, 8);
    a.width = (gated ? 2 : 1) * a.half;
    a.pitch = up_to(I, 256) / 2;
    long long at = 0;
    const auto take = [&](long long bytes) {
        const long long here = at;
        at += up_to(bytes, 512);
        return here;
    };
    a.parts = (I + WIDE - 1) / WIDE;
    a.count_bytes = 4 * (rows * a.parts + (H + CH - 1) / CH);  // of parts of chunks (there are at most as many chunks as rows) and of the second product's tiles
    a.counts = take(a.count_bytes);
    a.sums = take(4 * partial_sums(rows, a.width, (H + 255) / 256));
    a.unscale = take(4 * rows * a.parts);
    a.pieces = take(rows * PIECES * a.pitch);
    a.part = take(4 * 2ll * SMS * T * CH);
    a.end = at;
    return a;
}

template <typename Kernel> cudaError_t launch(Kernel* kernel, std::atomic<bool>* ready, int threads, int smem, bool dependent, const FewParams& p, cudaStream_t s) {
    int dev = 0;
    cudaError_t e;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev]) {
        if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return e;
        if (dev < 64) ready[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(SMS);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = dependent ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <typename T, int FORMAT> cudaError_t few(const FewFp4& q, cudaStream_t s) {
    using S = Shape<FORMAT>;
    const long long rows = q.T * q.top_k;
    const Places at = places(q.T, rows, q.H, q.I, q.gated);
    FewParams p = {};
    p.offsets = q.offsets;
    p.source = q.source;
    p.weights = q.weights;
    p.status = q.status;
    p.experts = q.experts;
    p.top_k = q.top_k;
    p.T = (int)q.T;
    p.rows = (int)rows;
    p.act = q.act;
    p.gated = q.gated;
    p.I = (int)q.I;
    p.half = (int)at.half;
    p.width = (int)at.width;
    p.pitch = at.pitch;
    p.down_parts = (int)at.parts;
    p.chunk_count = (int*)(q.scratch + at.counts);
    p.tile_count = p.chunk_count + rows * at.parts;
    p.sums = (float*)(q.scratch + at.sums);
    p.unscale = (float*)(q.scratch + at.unscale);
    p.pieces = (uint8_t*)(q.scratch + at.pieces);
    p.part = (float*)(q.scratch + at.part);
    cudaError_t e;
    const auto maps = [&](const uint8_t* w, const uint8_t* scale, long long ld, long long n, long long k, int halves) {
        p.N = (int)(n * halves);
        p.K = (int)k;
        p.k_blocks = (int)((k + 255) / 256);
        p.chan_tiles = (int)((n + CH - 1) / CH);
        if ((e = make_map(&p.w, w, n * halves * q.experts, (k + 1) / 2, ld, CH)) != cudaSuccess) return e;
        return make_atom_map(&p.w_scale, scale, (long long)q.experts * halves * p.chan_tiles * p.k_blocks * S::ATOMS, S::ATOMS);
    };
    if ((e = cudaMemsetAsync(p.chunk_count, 0, at.count_bytes, s)) != cudaSuccess) return e;
    if ((e = maps(q.up, q.up_scale, q.ld_up, q.I, q.H, q.gated ? 2 : 1)) != cudaSuccess) return e;
    p.in = q.x;
    p.ldx = q.ldx;
    p.vec = (uintptr_t)q.x % 16 == 0 && (q.T <= 1 || q.ldx * sizeof(T) % 16 == 0);
    p.wide = q.up_wide;
    p.bias = q.up_bias;
    static std::atomic<bool> up_ready[64], down_ready[64];  // by device; setting it twice does no harm
    if ((e = launch(hccl_few_up<T, FORMAT>, up_ready, UP_THREADS, S::SMEM_UP, false, p, s)) != cudaSuccess) return e;
    if ((e = maps(q.down, q.down_scale, q.ld_down, q.H, q.I, 1)) != cudaSuccess) return e;
    if ((e = make_map(&p.x, p.pieces, rows * PIECES, at.pitch, at.pitch, PIECES)) != cudaSuccess) return e;
    p.y = q.y;
    p.ldy = q.ldy;
    p.wide = q.down_wide;
    p.bias = q.down_bias;
    return launch(hccl_few_down<T, FORMAT>, down_ready, DOWN_THREADS, S::SMEM_DOWN, true, p, s);
}

}  // namespace

size_t few_fp4_scratch(long long T, long long H, long long I, int top_k, int gated) { return (size_t)places(T, T * top_k, H, I, gated).end; }

cudaError_t launch_few_fp4(int dt, const FewFp4& p, cudaStream_t s) {
    if (p.T == 0) return cudaSuccess;
    const bool nv = p.format == HCCL_NVFP4;
    if (dt == HCCL_FP32) return nv ? few<float, HCCL_NVFP4>(p, s) : few<float, HCCL_MXFP4>(p, s);
    if (dt == HCCL_BF16) return nv ? few<__nv_bfloat16, HCCL_NVFP4>(p, s) : few<__nv_bfloat16, HCCL_MXFP4>(p, s);
    return nv ? few<__half, HCCL_NVFP4>(p, s) : few<__half, HCCL_MXFP4>(p, s);
}

}  // namespace experts
}  // namespace hccl
