// Rows to 4-bit floating point in blocks with a scale each, and back; scales from rows to the tiles that the tensor cores take.
// Memory is the bound: an element is read once and everything that hangs on it stays in one thread's registers, 16 elements of a row, so that a block
// is one thread's (NVFP4) or two neighbours' (MXFP4). With a routing a token's row is quantised once and written to every place it was sent to.
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

// `lanes` neighbouring lanes (8, 16 or 32) share a row; longer rows are walked in pieces of 512 elements by one warp each.
template <typename T, int FORMAT> __global__ void __launch_bounds__(THREADS) hccl_quantise_fp4(const __grid_constant__ Fp4Rows p, int lanes, int pieces) {
    constexpr int N = Sixteen<T>::N, PARTS = EACH / N;
    asm volatile("griddepcontrol.launch_dependents;");  // the product may start to fetch its weights
    const int lane = threadIdx.x % 32, K = (int)p.K, per_warp = 32 / lanes, copies = p.slots ? p.top_k : 1;
    const long long tasks = (p.M + per_warp - 1) / per_warp * pieces, step = (long long)gridDim.x * (THREADS / 32);
    for (long long task = (long long)blockIdx.x * (THREADS / 32) + threadIdx.x / 32; task < tasks; task += step) {
        const long long m = task / pieces * per_warp + lane / lanes;
        const int k = ((int)(task % pieces) * lanes + lane % lanes) * EACH;
        const bool in = m < p.M;
        Sixteen<T> v[PARTS];
        unsigned top = 0;
        if (in) {
            const T* x = (const T*)p.x + m * p.ldx;
#pragma unroll
            for (int u = 0; u < PARTS; u++) v[u].load(x, k + u * N, K, p.vec);
#pragma unroll
            for (int u = 0; u < PARTS; u++) top = max(top, v[u].magnitude());
        }
        if (FORMAT == HCCL_MXFP4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        const Step s = step_of<FORMAT>(top, p.wide, p.six);
        unsigned code[2] = {0, 0};
        if (in && s.inv != 0.f) {
            // A saturated scale leaves quotients as large as the input: kept finite, so that the remainder is a number.
            const bool far = FORMAT == HCCL_NVFP4 && s.byte == 0x7eu;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                float q[8];
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    float x = v[(8 * h + j) / N].value((8 * h + j) % N);
                    if (far) x = fminf(fmaxf(x, -8.f * s.d), 8.f * s.d);
                    q[j] = quotient<FORMAT>(x, s);
                }
                code[h] = eight_codes(q);
            }
        }
        // A scale for each 16 or 32 elements; the first of four lanes (eight) has four to write.
        constexpr int SHARE = FORMAT == HCCL_NVFP4 ? 1 : 2;
        unsigned four = s.byte;
        four |= __shfl_down_sync(0xffffffffu, four, SHARE) << 8;
        four |= __shfl_down_sync(0xffffffffu, four, 2 * SHARE) << 16;
        const int block = k / (SHARE * EACH), blocks = (K + SHARE * EACH - 1) / (SHARE * EACH);
        if (!in || k >= ((K + 63) & ~63)) continue;
        for (int c = 0; c < copies; c++) {
            const long long row = p.slots ? p.slots[m * p.top_k + c] : m;
            if (row < 0 || row >= p.n_q) continue;
            uint8_t* q = p.q + row * p.ldq + k / 2;
            if (p.vec_q && k + EACH <= K) {
                *(uint2*)q = make_uint2(code[0], code[1]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; j++)
                    if (k + 2 * j < K) q[j] = (uint8_t)(code[j / 4] >> (8 * (j & 3)));
            }
            if (!p.tn) {
                if (lane % SHARE == 0 && block < blocks) p.scale[row * p.lds + block] = (uint8_t)s.byte;
            } else if (block % 4 == 0 && lane % SHARE == 0) {
                const int g = group_of(p.offsets, p.groups, row);
                if (g < 0) continue;
                const long long first = p.offsets ? max(0, p.offsets[g]) : 0, r = row - first;
                const long long tile = tile_base(first, p.tn, g) + r / p.tn;
                const int in_tile = (int)(r % p.tn), wide = p.tn > 128 ? p.tn / 128 : 1;
                *(unsigned*)(p.scale + ((tile * wide + in_tile / 128) * p.atoms + block / 4) * ATOM + atom_row(in_tile % 128)) = four;
            }
        }
    }
}

template <typename T, int FORMAT> __global__ void __launch_bounds__(THREADS) hccl_dequantise_fp4(const __grid_constant__ Fp4Values p, int pieces) {
    const long long total = p.M * pieces, step = (long long)gridDim.x * THREADS;
    const int K = (int)p.K;
    for (long long i = (long long)blockIdx.x * THREADS + threadIdx.x; i < total; i += step) {
        const long long m = i / pieces;
        const int k = (int)(i % pieces) * EACH;
        const uint8_t* q = p.q + m * p.ldq + k / 2;
        unsigned w[2] = {0, 0};
        if (p.vec && k + EACH <= K) {
            const uint2 both = *(const uint2*)q;
            w[0] = both.x, w[1] = both.y;
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (k + 2 * j < K) w[j / 4] |= (unsigned)q[j] << (8 * (j & 3));
        }
        const float d = step_value<FORMAT>(p.scale[m * p.lds + k / block_of(FORMAT)], p.wide);
        float v[EACH];
        eight_values(w[0], v);
        eight_values(w[1], v + 8);
#pragma unroll
        for (int j = 0; j < EACH; j++) v[j] = __fmul_rn(v[j], d);
        T* y = (T*)p.y + m * p.ldy + k;
        constexpr int N = 16 / sizeof(T);
        if (p.vec && k + EACH <= K) {
#pragma unroll
            for (int u = 0; u < EACH / N; u++) {
                Pack<T, N> o;
                float part[N];
#pragma unroll
                for (int j = 0; j < N; j++) part[j] = v[u * N + j];
                o.set(part);
                ((uint4*)y)[u] = o.raw;
            }
        } else {
#pragma unroll
            for (int j = 0; j < EACH; j++)
                if (k + j < K) y[j] = from_f32<T>(v[j]);
        }
    }
}

// Four scales of a row to their place; also those beyond the last block, as zeros.
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

template <typename T, int FORMAT> cudaError_t quantise_launch(const Fp4Rows& q, cudaStream_t s) {
    Fp4Rows p = q;
    p.vec = (uintptr_t)p.x % 16 == 0 && (p.ldx * sizeof(T) % 16 == 0 || p.M <= 1);
    p.vec_q = (uintptr_t)p.q % 8 == 0 && p.ldq % 8 == 0;
    const long long sixteens = (p.K + EACH - 1) / EACH;
    int lanes = 8;
    while (lanes < 32 && lanes < sixteens) lanes *= 2;
    const int pieces = (int)((sixteens + lanes - 1) / lanes);
    const long long warps = (p.M + 32 / lanes - 1) / (32 / lanes) * pieces;
    hccl_quantise_fp4<T, FORMAT><<<grid_for((warps + THREADS / 32 - 1) / (THREADS / 32)), THREADS, 0, s>>>(p, lanes, pieces);
    return cudaGetLastError();
}

template <typename T, int FORMAT> cudaError_t dequantise_launch(const Fp4Values& q, cudaStream_t s) {
    Fp4Values p = q;
    p.vec = (uintptr_t)p.q % 8 == 0 && p.ldq % 8 == 0 && (uintptr_t)p.y % 16 == 0 && p.ldy * sizeof(T) % 16 == 0;
    const int pieces = (int)((p.K + EACH - 1) / EACH);
    hccl_dequantise_fp4<T, FORMAT><<<grid_for((p.M * pieces + THREADS - 1) / THREADS), THREADS, 0, s>>>(p, pieces);
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
