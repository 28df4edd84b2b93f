// Rows to 4-bit floating point in blocks with a scale each, and back; scales from rows to the tiles that the tensor cores take.
// Memory and instructions bound it at about the same time: an element is read once and everything that hangs on it stays in one thread's registers, 16 elements of a row, so that a block
// is one thread's (NVFP4) or two neighbours' (MXFP4). With a routing a token's row is quantised once and written to every place it was sent to.
//
// Measured (B200, copy peak 6.5 TB/s): 8192 x 8192 bf16 40 us = 4.4 TB/s (16 instructions an element issue in 79 % of the cycles); 8192 x 4096 to 8 places 51 us = 4.3 TB/s, to 4 places 30; the way
// back, 32768 x 4096 to bf16, 62 us = 5.5 TB/s; 1999 x 2057 fp32, rows on 4 bytes, 8 us there and 15 back.
#include <algorithm>

#include "fp4.cuh"
#include "rows_i8.cuh"

namespace hccl {
namespace experts {
namespace {

constexpr int EACH = 16, THREADS = 256;

// The group of a row in expert order: the last that begins at it or before; -1 where no group has it.
__device__ __forceinline__ int group_of(const int* offsets, int groups, long long row) {
    if (!offsets) return 0;
    if (row < offsets[0] || row >= offsets[groups]) return -1;
    int lo = 0, hi = groups - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (offsets[mid] <= row) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Where a row goes: its codes, and its scales, by rows or in tiles. row < 0: nowhere.
struct Place {
    long long row, scale;
};
__device__ __forceinline__ Place place_of(const Fp4Rows& p, long long row) {
    Place at = {row, -1};
    if (row < 0 || row >= p.n_q) {
        at.row = -1;
    } else if (!p.tn) {
        at.scale = row * p.lds;
    } else {
        // (rows are counted in 32 bits there, tn is a power of two)
        unsigned first = 0, g = 0;
        if (p.offsets) {
            const int of = group_of(p.offsets, p.groups, row);
            if (of < 0) return at;
            g = of, first = (unsigned)max(0, p.offsets[of]);
        }
        const unsigned r = (unsigned)row - first, in_tile = r & ((1u << p.shift) - 1), tile = (first >> p.shift) + g + (r >> p.shift);
        const unsigned atom = p.shift > 7 ? (tile << (p.shift - 7)) + (in_tile >> 7) : tile;
        at.scale = (long long)atom * (p.atoms * ATOM) + atom_row(in_tile & 127);
    }
    return at;
}

// A thread has 16 elements of a row, `team` threads side by side (8 to 256) a row, or, of long rows, a part of it; blocks come and go, which costs less than walking rows does in
// instructions, and those are the bound (8192 x 8192 bf16: 45 us; walked, with loads two pieces ahead, 55). WHOLE: rows start on 16 bytes. Otherwise a warp fetches its 512 elements
// one by one, lanes side by side, and hands them round through shared memory.
template <typename T, int FORMAT, bool WHOLE> __global__ void __launch_bounds__(THREADS) hccl_quantise_fp4(const __grid_constant__ Fp4Rows p, int team, int teams) {
    constexpr int N = Sixteen<T>::N, PARTS = EACH / N, SHARE = FORMAT == HCCL_NVFP4 ? 1 : 2 /* threads to a block */;
    extern __shared__ __align__(16) uint4 shared[];
    float* const handed = (float*)shared + threadIdx.x / 32 * (32 * 17);                              // [warp][lane][17], unless WHOLE
    Place* const places = (Place*)(shared + (WHOLE ? 0 : blockDim.x / 32 * (32 * 17 / 4)));  // [teams * copies], where rows have a routing
    asm volatile("griddepcontrol.launch_dependents;");  // the product may start to fetch its weights
    int mine = 0, rank = (int)threadIdx.x;
    if (teams > 1) mine = rank / team, rank -= mine * team;
    const int lane = threadIdx.x % 32, K = (int)p.K;
    const long long first = (long long)blockIdx.x * teams, m = first + mine;
    const int k = ((int)blockIdx.y * team + rank) * EACH, copies = p.slots ? p.top_k : 1;
    const bool in = m < p.M && k < ((K + 63) & ~63);
    Sixteen<T> v[PARTS];
    float f[EACH];  // negated
    unsigned top = 0;
    if constexpr (WHOLE) {
        const T* x = (const T*)p.x + m * p.ldx + k;
        if (in && k + EACH <= K) {
#pragma unroll
            for (int u = 0; u < PARTS; u++) {
                const uint4 w = ((const uint4*)x)[u];
                v[u].w[0] = w.x, v[u].w[1] = w.y, v[u].w[2] = w.z, v[u].w[3] = w.w;
            }
        } else {
#pragma unroll
            for (int u = 0; u < PARTS; u++) v[u].load(x, u * N, in ? K - k : 0, true);
        }
    }
    if (p.slots) {
        for (int i = (int)threadIdx.x; i < teams * copies; i += blockDim.x)
            if (first + i / copies < p.M) places[i] = place_of(p, p.slots[(first + i / copies) * p.top_k + i % copies]);
        __syncthreads();
    }
    if constexpr (WHOLE) {
#pragma unroll
        for (int u = 0; u < PARTS; u++) {
            top = max(top, v[u].magnitude());
#pragma unroll
            for (int i = 0; i < 4; i++) v[u].w[i] ^= sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
        }
#pragma unroll
        for (int j = 0; j < EACH; j++) f[j] = v[j / N].value(j % N);
    } else {
        const int col = ((int)blockIdx.y * team + rank / 32 * 32) * EACH + lane;  // (a warp has one row here)
        const T* x = (const T*)p.x + m * p.ldx;
#pragma unroll
        for (int i = 0; i < EACH; i++) handed[i * 32 + lane + 2 * i + lane / EACH] = m < p.M && col + i * 32 < K ? to_f32<T>(x[col + i * 32]) : 0.f;
        __syncwarp();
#pragma unroll
        for (int j = 0; j < EACH; j++) f[j] = -handed[lane * 17 + j], top = max(top, __float_as_uint(f[j]) & 0x7fffffffu);
    }
    if (FORMAT == HCCL_MXFP4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const Step s = step_of<FORMAT>(top, p.wide, p.six, p.sixth);
    unsigned code[2] = {0, 0};
    if (s.inv != 0.f) {
        // A saturated scale leaves quotients as large as the input: kept finite, so that the remainder is a number.
        if (FORMAT == HCCL_NVFP4 && s.byte == 0x7eu)
#pragma unroll
            for (int j = 0; j < EACH; j++) f[j] = fminf(fmaxf(f[j], -8.f * s.d), 8.f * s.d);
#pragma unroll
        for (int j = 0; j < EACH; j += 2) quotients<FORMAT>(Two(f[j], f[j + 1]), s).get(f[j], f[j + 1]);
        code[0] = eight_codes(f), code[1] = eight_codes(f + 8);
    }
    // A scale for each 16 or 32 elements; the first of four lanes (eight) has four to write.
    unsigned four = s.byte;
    four |= __shfl_down_sync(0xffffffffu, four, SHARE) << 8;
    four |= __shfl_down_sync(0xffffffffu, four, 2 * SHARE) << 16;
    if (!in) return;
    const int block = k / (SHARE * EACH), blocks = (K + SHARE * EACH - 1) / (SHARE * EACH);
    const auto put = [&](const Place& at) {
        if (at.row < 0) return;
        uint8_t* q = p.q + at.row * p.ldq + k / 2;
        if (p.vec_q && k + EACH <= K) {
            *(uint2*)q = make_uint2(code[0], code[1]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (k + 2 * j < K) q[j] = (uint8_t)(code[j / 4] >> (8 * (j & 3)));
        }
        if (lane % SHARE || at.scale < 0) return;
        if (!p.tn) {
            if (block < blocks) p.scale[at.scale + block] = (uint8_t)s.byte;
        } else if (block % 4 == 0) {
            *(unsigned*)(p.scale + at.scale + block / 4 * ATOM) = four;
        }
    };
    if (p.slots)
        for (int c = 0; c < copies; c++) put(places[mine * copies + c]);
    else
        put(place_of(p, m));  // (n_q is at least M)
}

// A thread has V elements at a time, 16 bytes of the result where rows start on them (WHOLE); `team` threads side by side a row, four pieces of each on their way at once. Otherwise an
// element, so that a warp's stores are side by side.
template <typename T, int FORMAT, bool WHOLE> __global__ void __launch_bounds__(THREADS) hccl_dequantise_fp4(const __grid_constant__ Fp4Values p, int team, int teams) {
    constexpr int V = WHOLE ? 16 / sizeof(T) : 1, U = 4;
    int mine = 0, rank = (int)threadIdx.x;
    if (teams > 1) mine = rank / team, rank -= mine * team;
    const int K = (int)p.K;
    for (long long m = (long long)blockIdx.x * teams + mine; m < p.M; m += (long long)gridDim.x * teams) {
        const uint8_t* const q = p.q + m * p.ldq;
        const uint8_t* const scale = p.scale + m * p.lds;
        T* const y = (T*)p.y + m * p.ldy;
        for (int base = 0; base < K; base += U * team * V) {
            unsigned w[U], byte[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int k = base + (u * team + rank) * V;
                w[u] = byte[u] = 0;
                if (k < K) {
                    if (!WHOLE || k + V > K) {
#pragma unroll
                        for (int j = 0; j < (V + 1) / 2; j++)
                            if (k + 2 * j < K) w[u] |= (unsigned)q[k / 2 + j] << (8 * j);
                        if (V == 1 && k % 2) w[u] >>= 4;
                    } else if constexpr (V == 8) {
                        w[u] = *(const unsigned*)(q + k / 2);
                    } else {
                        w[u] = *(const unsigned short*)(q + k / 2);
                    }
                    byte[u] = scale[k / block_of(FORMAT)];
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int k = base + (u * team + rank) * V;
                if (k >= K) break;
                const float d = step_value<FORMAT>(byte[u], p.wide);
                float v[8];
                eight_values(w[u], v);
#pragma unroll
                for (int j = 0; j < V; j++) v[j] = __fmul_rn(v[j], d);
                if (WHOLE && k + V <= K) {
                    if constexpr (WHOLE) {
                        Pack<T, V> o;
                        float part[V];
#pragma unroll
                        for (int j = 0; j < V; j++) part[j] = v[j];
                        o.set(part);
                        *(uint4*)(y + k) = o.raw;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < V; j++)
                        if (k + j < K) y[k + j] = from_f32<T>(v[j]);
                }
            }
        }
    }
}

// Four scales of a row to their place; also those beyond the last block, as zeros. 8192 x 8192 12 us, 65536 rows of 4096 over 64 experts 54: a division, four loads of bytes and, over experts, a search
// for each word. Weights pass here once; rows that arrive in 4 bits at each product.
__global__ void __launch_bounds__(THREADS) hccl_tile_scales_fp4(const __grid_constant__ Fp4Scales p) {
    const long long rows = p.N * (p.offsets ? 1 : p.groups), total = rows * p.atoms, step = (long long)gridDim.x * THREADS;
    for (long long i = (long long)blockIdx.x * THREADS + threadIdx.x; i < total; i += step) {
        const long long row = i / p.atoms;
        const int a = (int)(i % p.atoms);
        unsigned four = 0;
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (4 * a + j < p.blocks) four |= (unsigned)p.scale[row * p.lds + 4 * a + j] << (8 * j);
        long long tile, r;
        if (p.offsets) {
            const int g = group_of(p.offsets, p.groups, row);
            if (g < 0) continue;
            const long long first = max(0, p.offsets[g]);
            r = row - first;
            tile = tile_base(first, p.tn, g);
        } else {
            const long long g = row / p.N;
            r = row % p.N;
            tile = g * ((p.N + p.tn - 1) / p.tn);
        }
        tile += r / p.tn;
        const int in_tile = (int)(r % p.tn), wide = p.tn > 128 ? p.tn / 128 : 1;
        *(unsigned*)(p.out + ((tile * wide + in_tile / 128) * p.atoms + a) * ATOM + atom_row(in_tile % 128)) = four;
    }
}

unsigned grid_for(long long blocks) { return (unsigned)std::max(1ll, std::min(blocks, (long long)SMS * 8)); }

// Threads to a row: a power of two up to a warp, then whole warps.
int team_for(long long pieces, int least) {
    int team = least;
    while (team < 32 && team < pieces) team *= 2;
    return team < pieces ? (int)std::min((long long)THREADS, (pieces + 31) / 32 * 32) : team;
}

template <typename T, int FORMAT> cudaError_t quantise_launch(const Fp4Rows& q, cudaStream_t s) {
    Fp4Rows p = q;
    p.vec_q = (uintptr_t)p.q % 8 == 0 && p.ldq % 8 == 0;
    const bool whole = (uintptr_t)p.x % 16 == 0 && (p.ldx * sizeof(T) % 16 == 0 || p.M <= 1);
    const int team = team_for((p.K + EACH - 1) / EACH, whole ? 8 : 32), teams = THREADS / team, threads = teams * team;
    const int shared = (whole ? 0 : threads * 17 * 4) + (p.slots ? teams * p.top_k * (int)sizeof(Place) : 0);  // at most 17 and 16 KB
    const dim3 grid((unsigned)((p.M + teams - 1) / teams), (unsigned)((p.K + team * EACH - 1) / (team * EACH)));
    if (whole) hccl_quantise_fp4<T, FORMAT, true><<<grid, threads, shared, s>>>(p, team, teams);
    else hccl_quantise_fp4<T, FORMAT, false><<<grid, threads, shared, s>>>(p, team, teams);
    return cudaGetLastError();
}

template <typename T, int FORMAT> cudaError_t dequantise_launch(const Fp4Values& p, cudaStream_t s) {
    const bool whole = (uintptr_t)p.q % 4 == 0 && p.ldq % 4 == 0 && (uintptr_t)p.y % 16 == 0 && (p.ldy * sizeof(T) % 16 == 0 || p.M <= 1);
    const int V = whole ? 16 / (int)sizeof(T) : 1, team = team_for((p.K + 4 * V - 1) / (4 * V), 32), teams = THREADS / team;
    const unsigned grid = (unsigned)std::min((p.M + teams - 1) / teams, 1ll << 30);
    if (whole) hccl_dequantise_fp4<T, FORMAT, true><<<grid, teams * team, 0, s>>>(p, team, teams);
    else hccl_dequantise_fp4<T, FORMAT, false><<<grid, teams * team, 0, s>>>(p, team, teams);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_quantise_fp4(int dt, int format, const Fp4Rows& p, cudaStream_t s) {
    if (p.M == 0 || p.K == 0) return cudaSuccess;
    const bool nv = format == HCCL_NVFP4;
    if (dt == HCCL_FP32) return nv ? quantise_launch<float, HCCL_NVFP4>(p, s) : quantise_launch<float, HCCL_MXFP4>(p, s);
    if (dt == HCCL_BF16) return nv ? quantise_launch<__nv_bfloat16, HCCL_NVFP4>(p, s) : quantise_launch<__nv_bfloat16, HCCL_MXFP4>(p, s);
    return nv ? quantise_launch<__half, HCCL_NVFP4>(p, s) : quantise_launch<__half, HCCL_MXFP4>(p, s);
}

cudaError_t launch_dequantise_fp4(int dt, int format, const Fp4Values& p, cudaStream_t s) {
    if (p.M == 0 || p.K == 0) return cudaSuccess;
    const bool nv = format == HCCL_NVFP4;
    if (dt == HCCL_FP32) return nv ? dequantise_launch<float, HCCL_NVFP4>(p, s) : dequantise_launch<float, HCCL_MXFP4>(p, s);
    if (dt == HCCL_BF16) return nv ? dequantise_launch<__nv_bfloat16, HCCL_NVFP4>(p, s) : dequantise_launch<__nv_bfloat16, HCCL_MXFP4>(p, s);
    return nv ? dequantise_launch<__half, HCCL_NVFP4>(p, s) : dequantise_launch<__half, HCCL_MXFP4>(p, s);
}

cudaError_t launch_tile_scales_fp4(const Fp4Scales& p, cudaStream_t s) {
    const long long total = p.N * (p.offsets ? 1 : p.groups) * p.atoms;
    if (total == 0) return cudaSuccess;
    hccl_tile_scales_fp4<<<grid_for((total + THREADS - 1) / THREADS), THREADS, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace experts
}  // namespace hccl
