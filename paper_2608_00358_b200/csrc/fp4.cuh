// 4-bit floating point in blocks: what quantising, the products and the few-token layer share.
//
// An element is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a byte, the earlier in the low half. A block has a step d that
// all its elements are multiples of. NVFP4: 16 elements, a byte s = e4m3(max|x| / (6 g)) and d = s g with a 32-bit g for the whole matrix. MXFP4: 32
// elements, a byte e, d = 2^(e - 127), the least e with max|x| <= 6 d (not OCP's floor(log2 max|x|) - 2,
// which cuts up to a quarter off a block's largest elements: nothing saturates here). q = e2m1(x / d), the quotient rounded to 32 bits, ties to even. A block with an infinity or a NaN has the scale NaN (0x7f, 0xff).
//
// Scales lie in two ways. By rows: [rows][blocks], for exchange and storage. In tiles, as the tensor cores take them: an atom of 512 bytes holds 128 rows x 4 blocks, the
// four bytes of row r at (r % 32) * 16 + (r / 32) * 4; atoms of a tile's successive blocks follow one another, up to whole stages of 256 elements.
#pragma once
#include "two.cuh"

namespace hccl {
namespace experts {

constexpr int ATOM = 512;
__host__ __device__ constexpr int block_of(int format) { return format == HCCL_NVFP4 ? 16 : 32; }
__host__ __device__ constexpr int stage_atoms(int format) { return format == HCCL_NVFP4 ? 4 : 2; }  // of 256 elements

// The place of a row's group of four blocks within its tile's first atom.
__host__ __device__ __forceinline__ int atom_row(int r) { return (r & 31) * 16 + (r >> 5) * 4; }

// The bytes of scales in tiles that a token row's tile of `tn` tokens takes: where the rows of group g begin, in tiles. Groups begin at
// any row; each is given a tile more than its rows before it fill, which is enough for the part-filled tile at its end.
__host__ __device__ __forceinline__ long long tile_base(long long first_row, int tn, int g) { return first_row / tn + g; }

struct Step {
    float d, inv;    // 1 / d, to nearest; 0: the block's elements are zeros
    unsigned byte;   // as stored
};
// top: the largest magnitude's bits; NaN is above infinity. six: 6 wide, and sixth its reciprocal, both to nearest.
template <int FORMAT> __device__ __forceinline__ Step step_of(unsigned top, float wide, float six, float sixth) {
    Step r;
    if constexpr (FORMAT == HCCL_NVFP4) {
        const float x = __uint_as_float(top), y = __fmul_rn(x, sixth);
        const float t = fminf(__fmaf_rn(-__fmaf_rn(y, six, -x), sixth, y), 448.f);  // x / six, as the quotients below; what is too large for that is NaN there and 448 here
        unsigned short two;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(0.f), "f"(t));
        r.byte = two & 0xffu;
        unsigned halves;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(halves) : "h"(two));
        r.d = __fmul_rn(__low2float(*(const __half2*)&halves), wide);
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(r.d));
        r.inv = r.byte ? __fmaf_rn(inv, __fmaf_rn(-r.d, inv, 1.f), inv) : 0.f;  // one step of Newton's: to nearest but for a few in a million, which the quotients' remainder makes up for
        if (top >= 0x7f800000u) r.byte = 0x7fu, r.inv = 0.f, r.d = __uint_as_float(0x7fffffffu);
    } else {
        const int code = max((int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u), 1);
        r.byte = (unsigned)code;
        r.d = __uint_as_float((unsigned)code << 23);
        r.inv = __uint_as_float((unsigned)(254 - code) << 23);  // exact
        if (top >= 0x7f800000u) r.byte = 0xffu, r.inv = 0.f, r.d = __uint_as_float(0x7fffffffu);
    }
    return r;
}
// x / d rounded to nearest, of -x (Markstein 1990: from the rounded reciprocal, by the quotient's exact remainder; in these signs a negative zero stays one); for MXFP4 a product with a
// power of two.
template <int FORMAT> __device__ __forceinline__ Two quotients(Two minus_x, const Step& s) {
    const Two inv(-s.inv), y = minus_x * inv;
    if constexpr (FORMAT == HCCL_MXFP4) return y;
    return fma2(fma2(y, Two(s.d), minus_x), inv, y);
}
// Eight quotients to four bytes, the first in the lowest half-byte; |q| > 6 becomes 6.
__device__ __forceinline__ unsigned eight_codes(const float* q) {
    unsigned r;
    asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
        " cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(r)
        : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
    return r;
}
// Eight codes to their values. A byte permutation looks four of them up: the upper byte of a magnitude as a 16-bit number is all that it has; its sign comes from a
// permutation of negative bytes, which a selector's fourth bit turns to ones. (The conversion instruction, given bytes of a register, was compiled wrongly in some places.)
__device__ __forceinline__ void eight_values(unsigned w, float* v) {
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const unsigned x = h ? w >> 16 : w;
        const unsigned four = __byte_perm(0x3e3c3800u, 0x46444240u, x & 0x7777u);  // 0, 0.5, 1, 1.5, 2, 3, 4, 6
        unsigned sign;
        asm("prmt.b32 %0, %1, %1, %2;" : "=r"(sign) : "r"(0x80808080u), "r"(x));  // 0xff where the code is negative, 0x80 elsewhere
        const unsigned signed_four = four | (sign << 1 & 0x80808080u);
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const unsigned two = __byte_perm(signed_four, 0u, i ? 0x3424 : 0x1404);
            const float2 f = __half22float2(*(const __half2*)&two);
            v[4 * h + 2 * i] = f.x, v[4 * h + 2 * i + 1] = f.y;
        }
    }
}
// The step that a stored byte stands for.
template <int FORMAT> __device__ __forceinline__ float step_value(unsigned byte, float wide) {
    if constexpr (FORMAT == HCCL_NVFP4) {
        unsigned halves;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(halves) : "h"((unsigned short)byte));
        return __fmul_rn(__low2float(*(const __half2*)&halves), wide);
    } else {
        return byte == 0xffu ? __uint_as_float(0x7fffffffu) : byte ? __uint_as_float(byte << 23) : __uint_as_float(0x400000u);
    }
}

// ---------------------------------------------------------------- parameter records and launchers
struct Fp4Rows {       // quantiser
    const void* x;
    long long ldx, M, K, ldq, n_q;
    uint8_t* q;
    uint8_t* scale;    // by rows (lds) or in tiles (tn > 0)
    long long lds;
    int tn, shift, atoms;  // tokens of a tile, 1 << shift; atoms of a row of tiles' blocks, up to whole stages
    float wide, six, sixth;
    int vec_q;
    const int* slots;  // null: row m of x to row m of q
    int top_k;
    const int* offsets;  // of the groups, where the scales go to tiles; null: one group
    int groups;
};
cudaError_t launch_quantise_fp4(int dt, int format, const Fp4Rows& p, cudaStream_t s);

struct Fp4Values {     // the way back
    const uint8_t *q, *scale;
    long long ldq, lds, M, K, ldy;
    void* y;
    float wide;
};
cudaError_t launch_dequantise_fp4(int dt, int format, const Fp4Values& p, cudaStream_t s);

struct Fp4Scales {     // scales by rows to scales in tiles; rows of `groups` groups of N, or by offsets
    const uint8_t* scale;
    long long lds, N, blocks;
    uint8_t* out;
    int tn, atoms, groups;
    const int* offsets;  // null: every group has N rows, and tiles of its own
};
cudaError_t launch_tile_scales_fp4(const Fp4Scales& p, cudaStream_t s);

struct MatmulFp4 {
    long long M, N, K, ldq, ldw, ldy;
    int groups, format;
    const uint8_t *q, *q_scale, *w, *w_scale;  // both scales in tiles
    const float *w_wide, *bias;
    float x_wide;
    const int* offsets;
    void* y;
    int* status;
    int dependent, tn, splits;
};
struct TileChoice {
    int tn, splits;
};
TileChoice choose_fp4(long long M, long long N, long long K, int groups);
cudaError_t launch_matmul_fp4(int dt, const MatmulFp4& p, cudaStream_t s);

struct FewFp4 {        // a whole expert layer for few tokens
    long long T, H, I, ldx, ldy;
    int top_k, experts, format, act, gated;
    const void* x;
    void* y;
    const int *offsets, *source;
    const float* weights;
    const uint8_t *up, *up_scale, *down, *down_scale;
    const float *up_wide, *down_wide, *up_bias, *down_bias;
    long long ld_up, ld_down;
    char* scratch;
    int* status;
};
size_t few_fp4_scratch(long long T, long long H, long long I, int top_k, int gated);
cudaError_t launch_few_fp4(int dt, const FewFp4& p, cudaStream_t s);

}  // namespace experts
}  // namespace hccl
