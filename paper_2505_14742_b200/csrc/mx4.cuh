// MXFP4 (OCP microscaling: blocks of 32 e2m1 elements under one e8m0 scale) - layout and device helpers shared by the
// quantization kernels, the product and the backward's expansion of the weight.
//
// Codes: [rows][pitch] bytes, two elements per byte, the even column in the low nibble; ceil(K / 32) * 16 bytes of a row
// are used (columns beyond K inside the last block hold code 0).
// Scales: tiles of 128 rows x 4 blocks, 512 bytes each, tiles of one row band one after the other.  Inside a tile the byte
// of row i, block b is at (i % 32) * 16 + (i / 32) * 4 + b: read as 32 rows of 16 bytes this is what tcgen05.cp 32x128b
// puts into tensor memory for a block-scaled tcgen05.mma.  Rows and blocks beyond the matrix hold 0 (2^-127).
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace quaff {

constexpr int kMx4Block = 32;          // elements under one scale
constexpr int kMx4TileRows = 128;      // rows of a scale tile
constexpr int kMx4TileBytes = 512;     // 128 rows x 4 blocks

inline int64_t mx4_row_bytes(int K) { return (int64_t)((K + kMx4Block - 1) / kMx4Block) * (kMx4Block / 2); }
inline int mx4_ktiles(int K) { return (K + 127) / 128; }
inline int mx4_row_tiles(int rows) { return rows / kMx4TileRows + (rows % kMx4TileRows != 0); }
inline size_t mx4_scale_bytes(int rows, int K) { return (size_t)mx4_row_tiles(rows) * mx4_ktiles(K) * kMx4TileBytes; }

__host__ __device__ __forceinline__ int64_t mx4_scale_offset(int row, int block, int ktiles) {
    return ((int64_t)(row >> 7) * ktiles + (block >> 2)) * kMx4TileBytes + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// e8m0 byte of a block from the exponent field of its largest magnitude: floor(log2 max) - 2 (e2m1's largest power of two
// is 2^2), not below 2^-127; 255 (NaN) when the block holds an infinity or a NaN.
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t exp_field) { return exp_field == 255u ? 255u : (exp_field < 2u ? 0u : exp_field - 2u); }
// 2^(127 - byte) as float; exact, byte <= 252 (a NaN block gets 0: its codes are 0)
__device__ __forceinline__ float mx4_inv_scale(uint32_t byte) { return byte == 255u ? 0.0f : __uint_as_float((254u - byte) << 23); }
// the value of an e8m0 byte
__device__ __forceinline__ float mx4_scale_value(uint32_t byte) {
    return byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte ? byte << 23 : 0x00400000u);
}

// eight floats (already divided by the scale) -> eight e2m1 codes, element 0 in the lowest nibble; nearest, ties to an even
// mantissa, magnitudes above 6 become 6
__device__ __forceinline__ uint32_t mx4_pack8(const float (&v)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// a block of 32 bf16 (four 16-byte words) -> its codes and scale byte
__device__ __forceinline__ void mx4_quantize_block(const uint4 (&v)[4], uint32_t (&c)[4], uint32_t& byte) {
    uint32_t m2 = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        m2 = __vmaxu2(__vmaxu2(m2, v[j].x & 0x7FFF7FFFu), v[j].y & 0x7FFF7FFFu);
        m2 = __vmaxu2(__vmaxu2(m2, v[j].z & 0x7FFF7FFFu), v[j].w & 0x7FFF7FFFu);
    }
    byte = mx4_scale_of(max(m2 & 0xFFFFu, m2 >> 16) >> 7);
    const float inv = mx4_inv_scale(byte);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float f[8] = {__fmul_rn(bf16_lo(v[j].x), inv), __fmul_rn(bf16_hi(v[j].x), inv), __fmul_rn(bf16_lo(v[j].y), inv), __fmul_rn(bf16_hi(v[j].y), inv),
                            __fmul_rn(bf16_lo(v[j].z), inv), __fmul_rn(bf16_hi(v[j].z), inv), __fmul_rn(bf16_lo(v[j].w), inv), __fmul_rn(bf16_hi(v[j].w), inv)};
        c[j] = byte == 255u ? 0u : mx4_pack8(f);          // infinity or NaN times 0 above
    }
}
// eight codes -> four f16x2 words (exact)
__device__ __forceinline__ void mx4_unpack8(uint32_t codes, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(codes));
}

// f32 -> the sum of bf16 parts, one call per part: what is returned is bf16 bits, v becomes what they leave.  An infinity is its first part
// and zeros (inf - inf would make the sum NaN); a number beyond the largest bf16 begins with that, not with infinity.
__device__ __forceinline__ uint32_t bf16_part(float& v) {
    constexpr uint32_t kMax = 0x7F7F0000u;
    const uint32_t u = __float_as_uint(v), a = u & 0x7FFFFFFFu;
    const float x = a > kMax && a < 0x7F800000u ? __uint_as_float(kMax | (u & 0x80000000u)) : v;
    const uint32_t bits = pack_bf16x2(x, 0.0f) & 0xFFFFu;
    v = a == 0x7F800000u ? 0.0f : __fsub_rn(v, bf16_bits_to_f32(bits));
    return bits;
}

// host side, shared between the translation units (arguments are validated by the entry points)
quaff_status_t mx4_quantize_launch(const void* X, int x_dtype, int64_t ldx, int M, int K, uint8_t* codes, int64_t ldc, uint8_t* scales,
                                   cudaStream_t st);
quaff_status_t mx4_dequantize_launch(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int M, int K, uint16_t* out, int64_t ldo,
                                     cudaStream_t st);
// a byte array as rows of 128 bytes, no swizzle: box = box_rows rows, contiguous in shared memory (bytes a multiple of 128)
quaff_status_t make_tmap_rows128(CUtensorMap* map, const void* base, uint64_t bytes, uint32_t box_rows);
// an output matrix [rows][cols] of 2- or 4-byte elements for stores of 32 rows x 128 bytes, 128-byte swizzle
quaff_status_t make_tmap_out(CUtensorMap* map, void* base, int elem_bytes, uint64_t rows, uint64_t cols, uint64_t ld);
enum { kSkinnyDown = 0, kSkinnyParts = 1, kSkinnyFold = 2, kSkinnyTurned = 3 };
// One skinny product (mx4_skinny.cuh): prepare builds the parameters, tensor maps included, and enqueues nothing
struct SkinnyParams {
    CUtensorMap map_a, map_b;
    int M, nst, per, ranks;         // output rows; stages of 64 contraction elements, of a rank; slices of the contraction
    int cols, rp, r, rot;           // accumulator columns (r rounded up to 16, times the parts of G); accumulators that TMEM holds (a power of two)
    uint32_t tx_bytes;
    float scale, bf16_scale;
    // T and G: bf16 result (G: optional) and scale x the sum in bf16 parts, [rows][parts rp];  dA, dB: f32 result
    uint16_t *bf16_out, *parts_out;
    int parts;
    float* f32_out;
    int accumulate;
    // T: the codes and scales of X on the way
    int K, ktiles;
    uint8_t* codes;
    int64_t ldc;
    uint8_t* scales;
    int32_t* status;
};
//   mode: kSkinnyParts  A [rows][kc] B [r][kc];  kSkinnyDown  A [rows][kc] B [kc][r];  kSkinnyFold, kSkinnyTurned  A [kc][rows] B [kc][cols]
quaff_status_t mx4_skinny_prepare(SkinnyParams& p, int mode, const void* A, int64_t lda, const void* B, int64_t ldb, int rows, int kc, int r, int cols,
                                  int32_t* status);
quaff_status_t mx4_skinny_launch(const SkinnyParams& p, int mode, cudaStream_t st);
// G, dB and the expanded weight in one launch (the weight: unless out is null).  prepare says whether the problem is small
// enough and divides the CTAs; it reads N, K, ktiles and out.
struct Mx4FrontParams {
    SkinnyParams g, db;
    const uint8_t* codes;
    int64_t ldc;
    const uint8_t* scales;
    int N, K, ktiles;
    uint16_t* out;
    int64_t ldo;
    int ranks, g_ctas, db_ctas, w_ctas, items;
};
bool mx4_front_prepare(Mx4FrontParams& p, int M, bool want_db);
quaff_status_t mx4_front_launch(const Mx4FrontParams& p, cudaStream_t st);
size_t mx4_fwd_workspace_bytes(int M, int K, int r);

}  // namespace quaff
