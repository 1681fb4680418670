// Microscaled 4-bit floating point: the two formats' sizes, where a block's scale byte lies, and the conversions.
//
// A value is e2m1 (0, .5, 1, 1.5, 2, 3, 4, 6 and signs), the even one of a pair in the low half of a byte.  BWLA_FP4_MX: 32 values
// share a scale 2^(byte - 127) (byte 255: NaN).  BWLA_FP4_NV: 16 values share an e4m3 scale, a row an fp32 one.  Scale bytes lie in
// tiles of 128 rows x 4 blocks, the 512 bytes that tcgen05.cp (32x128b) brings to tensor memory as tcgen05.mma wants them.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "bwla_common.cuh"

namespace bwla {

inline int fp4_block(int format) { return format == BWLA_FP4_NV ? 16 : 32; }
inline int64_t fp4_col_tiles(int64_t K, int format) { return (K / fp4_block(format) + 3) / 4; }      // tiles of 4 blocks along a row

// byte of block j of row r, given the row's number of tiles
__device__ __forceinline__ size_t fp4_scale_at(int64_t r, int j, int64_t col_tiles) {
    return ((size_t)(r >> 7) * (size_t)col_tiles + (size_t)(j >> 2)) * 512 + (size_t)((r & 31) * 16 + ((r >> 5) & 3) * 4 + (j & 3));
}

// 2^e for -127 <= e <= 127 (-127: the subnormal)
__device__ __forceinline__ float fp4_pow2(int e) { return __int_as_float(e > -127 ? (e + 127) << 23 : 0x00400000); }

// Eight values to their codes, v[0] lowest; to nearest, ties to the even code, beyond 6 to 6.
__device__ __forceinline__ uint32_t fp4_codes8(const float (&v)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// ... and back (exact)
__device__ __forceinline__ void fp4_values8(uint32_t codes, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

__device__ __forceinline__ uint32_t cvt_pair(float lo, float hi) {      // two bf16, rounded to nearest
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ uint32_t fp4_e4m3(float v) {              // to nearest even, beyond 448 to 448
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(r) : "f"(v), "f"(0.f));
    return r & 0xFFu;
}
__device__ __forceinline__ float fp4_from_e4m3(uint32_t byte) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)byte));
    return __half2float(__ushort_as_half((unsigned short)(h & 0xFFFFu)));
}
template <bool NV>
__device__ __forceinline__ float fp4_block_scale(uint32_t byte) {
    if (NV) return fp4_from_e4m3(byte);
    return byte == 255u ? __int_as_float(0x7FC00000) : fp4_pow2((int)byte - 127);
}

// x / d for a d of few bits, as precisely as the rounding to few bits behind it needs: where the quotient is no multiple of a short
// number the result is none either, and lies on the quotient's side of it.  inv: 1 / d, rounded.  One Newton step on the quotient with
// its exact residual (Markstein), then the residual's sign.
__device__ __forceinline__ float fp4_quotient(float x, float d, float inv) {
    float q = __fmul_rn(x, inv);
    q = __fmaf_rn(__fmaf_rn(-q, d, x), inv, q);
    const float r = __fmaf_rn(-q, d, x);
    const uint32_t bits = __float_as_uint(q);
    // (towards zero where the remainder has the other sign than the quotient)
    if (r != 0.f && (bits & 0xFFFFu) == 0u) q = __uint_as_float(((__float_as_uint(r) ^ bits) >> 31) ? bits - 1u : bits + 1u);
    return copysignf(q, x);                 // (of a negative zero the steps above lose the sign)
}

// Scale of a row whose largest magnitude is `top` (finite): the smallest power of two 2^E >= 2^-126 with top <= 6 * 448 * 2^E; 1 for a
// row of zeros.  A power of two costs the e4m3 scales none of their precision, and dividing by it is exact.
__device__ __forceinline__ int fp4_row_exponent(float top) {
    const uint32_t bits = __float_as_uint(top);
    if (bits == 0u) return 0;
    const int e = (int)(bits >> 23) - 127 - 11 + ((bits & 0x7FFFFFu) > 0x280000u ? 1 : 0);      // 2688 = 1.3125 * 2^11
    return max(e, -126);
}

// What a block's values are multiplied (MX) or divided (NV) by, and the scale byte, from the block's largest magnitude.
struct Fp4Block { float mul, div, inv; uint32_t byte; };
__device__ __forceinline__ Fp4Block fp4_block_mx(float top) {
    Fp4Block b;
    const uint32_t bits = __float_as_uint(top);
    const int e = max((int)(bits >> 23) - 127 - 2, -127);
    const bool finite = bits < 0x7F800000u;
    b.byte = finite ? (uint32_t)(e + 127) : 255u;
    b.mul = finite ? fp4_pow2(-e) : 0.f;
    return b;
}
// to_row: 2^-E of the row.  EXACT: top has 24 bits, else up to 11.  (1/6 in fp32 is above 1/6 by half of 2^-24 of it; see fp4_divide8.)
template <bool EXACT>
__device__ __forceinline__ Fp4Block fp4_block_nv(float top, float to_row) {
    Fp4Block b;
    const float t = __fmul_rn(top, to_row);
    const uint32_t byte = fp4_e4m3(EXACT ? fp4_quotient(t, 6.f, 1.f / 6.f) : __fmul_rz(t, 1.f / 6.f));
    b.byte = top == 0.f ? 0u : max(byte, 1u);
    b.div = fp4_from_e4m3(b.byte);
    // the reciprocal of a number of four bits to nearest: the hardware's estimate and one Newton step
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(b.div));
    r = __fmaf_rn(__fmaf_rn(-b.div, r, 1.f), r, r);
    b.inv = b.byte ? r : 0.f;
    return b;
}

// Eight values by their block's scale, for the rounding to e2m1; mul: 1 / (scale * 2^E).
// A code is decided against the middles T between codes, numbers of up to three bits, and 1 / scale, rounded, is never below the exact
// one: the scale has four bits, and 1/9 to 1/15 are all rounded up in fp32, by less than 2^-24 of themselves.  So where the quotient is
// T the product rounded towards zero is T.  Values of up to 11 bits (bf16, fp16) otherwise miss T by 2^-11 of it, and the product is all there
// is to do.  EXACT, for values of 24 bits: products within four units of a T are divided with the residual instead.
template <bool EXACT>
__device__ __forceinline__ void fp4_divide8(float (&f)[8], const Fp4Block& b, float mul, float to_row) {
    float q[8];
    bool near = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        q[i] = __fmul_rz(f[i], mul);
        if (EXACT) near = near || ((__float_as_uint(q[i]) + 4u) & 0x1FFFF8u) == 0u;
    }
    if (EXACT && near) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = fp4_quotient(__fmul_rn(f[i], to_row), b.div, b.inv);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = q[i];
}

int launch_fp4_quantize(const void* x, int dtype, int64_t M, int64_t K, int64_t ldx, int format, uint8_t* codes, uint8_t* scales, float* row_scales,
                        bool chained, cudaStream_t stream);
int launch_fp4_expand(const uint8_t* codes, const uint8_t* scales, const float* row_scales, int64_t M, int64_t K, int format, void* out, int dtype,
                      int64_t ldo, cudaStream_t stream);

struct Fp4GemmArgs {
    const uint8_t *a_codes, *a_scales; const float* a_rows;      // [M] rows
    const uint8_t *w_codes, *w_scales; const float* w_rows;      // [N] rows
    int64_t M, K, N;
    int format;
    __nv_bfloat16* out; int64_t ldo;
    uint32_t* status;
    float* parts; size_t part_bytes;      // room for sums of parts of tiles (fp4_pair.cu)
    bool prepared;                        // a layer's weights, complete before its kernels: read before griddepcontrol.wait
};
// Bytes of it that this product uses (fp4_part_bytes_up_to: any of up to so many tokens)
size_t fp4_gemm_part_bytes(int64_t M, int64_t K, int64_t N);
int launch_fp4_gemm(const Fp4GemmArgs& a, cudaStream_t stream);
int launch_fp4_pair(const Fp4GemmArgs& a, cudaStream_t stream);

// The maps of an operand: its codes as boxes of `box_rows` rows x 256 values (128 bytes, 128-byte swizzle), its scale tiles as boxes of
// `tile_rows` x 128 rows x 256 values.
struct Fp4Maps { CUtensorMap a, a_scales, w, w_scales; };
int fp4_operand_maps(CUtensorMap* codes, CUtensorMap* scales, const uint8_t* c, const uint8_t* s, int64_t rows, int64_t K, int format, int box_rows, int tile_rows);

}  // namespace bwla
