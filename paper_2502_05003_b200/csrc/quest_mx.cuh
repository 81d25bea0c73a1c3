// Microscaled (MX) tensors: layout, rounding of a block, and what the kernels that take them share.
//
// A block is 32 consecutive elements of a row: E2M1 codes (4 bits, two to a byte, element 0 in the low nibble) or E4M3
// bytes, under one scale 2^(s - 127), s a byte (UE8M0; 255 is NaN).  Scale bytes are stored as the tensor cores take them:
// tiles of 128 rows x 4 blocks, 512 bytes each, the tiles of a band of 128 rows one after another; row r, block j of a tile
// at byte 16 (r % 32) + 4 (r / 32) + j.  Rows and blocks that only fill up a tile have scale byte 0.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "quest_internal.cuh"

namespace quest {

constexpr int MX_BLOCK = 32;

// Shapes that the MX calls take.
inline bool mx_bits_ok(int bits) { return bits == 4 || bits == 8; }
inline bool mx_cols_ok(int64_t cols) { return cols >= 32 && cols <= 16384 && cols % 32 == 0; }
inline bool mx_rows_ok(int64_t rows) { return rows >= 0 && rows <= ((int64_t)1 << 24); }
inline bool mx_had_ok(int had_block) { return had_block == 1 || had_block == 32; }
inline size_t mx_scales_bytes(int64_t rows, int64_t cols) { return (size_t)((rows + 127) / 128) * (size_t)((cols + 127) / 128) * 512; }

// One tensor of a quantizer launch.
struct MxJob {
    const void *x;
    int64_t rows, ld;
    uint8_t *codes, *scales;
    int bits;
};
int launch_mx_quantize(const MxJob *jobs, int njobs, int dtype, int64_t cols, int had_block, cudaStream_t st);
// Codes and scales -> dense rows of `dtype`; ones (nullable): a bitmap of rows x cols / 8 bytes that is filled with ones.
struct MxDequantJob {
    const uint8_t *codes, *scales;
    int64_t rows;
    void *out;
    uint8_t *ones;
    int bits;
};
int launch_mx_dequantize(const MxDequantJob *jobs, int njobs, int dtype, int64_t cols, cudaStream_t st);
// y = x w^T over blocks: x 4 or 8 bits, w 4 bits (quest_mx_gemm.cu).
int launch_mx_gemm(const uint8_t *xq, const uint8_t *sx, int bits_x, const uint8_t *wq, const uint8_t *sw, int64_t M, int64_t N,
                   int64_t K, void *y, int y_dtype, int64_t ldy, cudaStream_t st);
// The same with the sides of the tensor cores' tiles exchanged and, where that fills the chip, K split (quest_mx_thin.cu).
int launch_mx_thin(const uint8_t *xq, const uint8_t *sx, int bits_x, const uint8_t *wq, const uint8_t *sw, int64_t M, int64_t N, int64_t K,
                   void *y, int y_dtype, int64_t ldy, cudaStream_t st);
// The product for a few rows of x (quest_mx_decode.cu), which are quantized on the way (x) or are given as codes (xq, sx).
int launch_mx_few_rows(const void *x, int x_dtype, int64_t ldx, const uint8_t *xq, const uint8_t *sx, int bits_x, int had_block,
                       const uint8_t *wq, const uint8_t *sw, int64_t M, int64_t N, int64_t K, void *y, int y_dtype, int64_t ldy,
                       cudaStream_t st);

// Which of the three.  Up to 32 rows go without tensor memory while w is small: its rows fill one round of CTAs, and K is short enough
// for one CTA to walk.  Time of the exchanged tiles over that kernel's, 8 and 4 bits: 8 x 2048 x 2048 1.13 / 0.96, x 4096 0.90 / 0.73,
// x 8192 0.70 / 0.55; 8 x 4096 x 2048 1.41 / 1.18, 8 x 8192 x 2048 0.73 / 0.54; 16 x 2048 x 2048 1.13 / 1.09, x 2560 1.01 / 0.89; 24 x 2048 x
// 1024 1.06 / 1.14, x 1536 0.96 / 1.01, x 2048 1.02 / 0.95; 32 x 2048 x 768 0.93 / 0.83; 32 x 32000 x 4096 0.22 / 0.20.
// Above, the exchanged tiles against pairs of CTAs on 256 rows of x: 64 x 4096 x 4096 0.71 / 0.87, 128 x 2048 x 8192 0.52 / 0.67;
// more than 128 rows 0.5 .. 1.04 where w fills a side of 128 and the tiles take half of the SMs (K is split) or one
// short round, else 0.8 .. 1.3.
enum class MxProduct { few, thin, wide };
constexpr int64_t MX_SMS = 148;
inline MxProduct mx_product(int64_t M, int64_t N, int64_t K, int bits_x) {
    const int64_t per_sm = M <= 8 ? 48 : M <= 16 ? 32 : 24;
    if (M <= 32 && N <= per_sm * MX_SMS && (M < 8 ? 8 : M) * K <= 32768) return MxProduct::few;
    const int64_t tiles = (N + 127) / 128 * ((M + 127) / 128);
    const bool fits = N >= 128 && (2 * tiles <= MX_SMS || (tiles <= MX_SMS && K <= (bits_x == 4 ? 2048 : 1024)));
    return M <= 128 || fits ? MxProduct::thin : MxProduct::wide;
}
// Whether the product of few rows quantizes x itself (quest_mx_codes_optional): up to eight of which a thread of the CTA takes one quarter of a block.  More, and
// a launch of the quantizer in front costs less (8 x 2048 x 2048: 7.7 us against 4.9; 1 x 2048 x 2048: 3.8 against 4.2, 2 x 2048 x 2048 4.2 against 4.3).
inline bool mx_fuses_quantizer(int64_t M, int64_t N, int64_t K) { return M <= 8 && M * K <= 4096 && N <= 48 * MX_SMS; }

#ifdef __CUDACC__

// Byte of the scale of (row, block); tiles = those of a band of 128 rows, (cols + 127) / 128.  Rows are at most 2^24, tiles 128: the
// number of a tile fits 32 bits, its place does not.
__device__ __forceinline__ long long mx_scale_at(int row, int block, int tiles) {
    return (long long)((row >> 7) * tiles + (block >> 2)) * 512 + (((row & 31) << 4) + (((row >> 5) & 3) << 2) + (block & 3));
}

__device__ __forceinline__ float mx_max_nan(float a, float b) {          // the larger magnitude; NaN if either is
    float r;
    asm("{\n\t.reg .f32 p, q;\n\tabs.f32 p, %1;\n\tabs.f32 q, %2;\n\tmax.NaN.f32 %0, p, q;\n\t}" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Scale byte of a block with largest magnitude amax: the exponent of amax less that of the element type's largest number
// (E2M1 2, E4M3 8), so that amax comes to lie in the type's top binade; what rounds beyond the largest number saturates.  0 for
// amax = 0, 255 where the block holds an infinity or a NaN.
template <int BITS>
__device__ __forceinline__ uint32_t mx_scale_byte(float amax) {
    const uint32_t e = __float_as_uint(amax) >> 23;                      // amax >= 0, or a NaN (of either sign bit)
    return (e & 255u) == 255u ? 255u : (uint32_t)max((int)e - (BITS == 4 ? 2 : 8), 0);
}
// 2^(127 - s): what the elements are multiplied with, exactly unless they vanish beside amax.  s = 255: 0.
__device__ __forceinline__ float mx_inverse_scale(uint32_t s) { return s == 255u ? 0.0f : __uint_as_float((254u - s) << 23); }
// 2^(s - 127) in binary32; s = 255: NaN.
__device__ __forceinline__ float mx_scale_f32(uint32_t s) {
    return __uint_as_float(s == 255u ? 0x7FC00000u : s == 0u ? 0x00400000u : s << 23);
}

// Eight elements -> a word of E2M1 codes; four elements -> a word of E4M3 bytes.  To nearest, ties to even, saturating.
__device__ __forceinline__ uint32_t mx_e2m1x8(const float *t) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(t[0]), "f"(t[1]), "f"(t[2]), "f"(t[3]), "f"(t[4]), "f"(t[5]), "f"(t[6]), "f"(t[7]));
    return r;
}
__device__ __forceinline__ uint32_t mx_e4m3x4(const float *t) {
    uint32_t r;
    asm("{\n\t.reg .b16 a, b;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
        "mov.b32 %0, {a, b};\n\t}"
        : "=r"(r)
        : "f"(t[0]), "f"(t[1]), "f"(t[2]), "f"(t[3]));
    return r;
}
// Two E2M1 codes (the low byte of w) or two E4M3 bytes (the low half of w) -> their values in binary32.
__device__ __forceinline__ float2 mx_values_e2m1(uint32_t w) {
    uint32_t h;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(h) : "r"(w));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
__device__ __forceinline__ float2 mx_values_e4m3(uint32_t w) {
    uint32_t h;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(h) : "r"(w));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

// In place: the orthonormal Walsh-Hadamard transform of 32 elements.  Strides from 16 down to 1, every sum rounded, then one
// product with 1 / sqrt(32): the order is part of the contract (codes are reproducible bit for bit).
__device__ __forceinline__ void mx_rotate(float *v) {
    float2 *p = reinterpret_cast<float2 *>(v);
    const float2 neg1 = make_float2(-1.0f, -1.0f);
#pragma unroll
    for (int s = 8; s >= 1; s >>= 1)                                    // strides 16 .. 2 in pairs of elements
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if ((i & s) == 0) {
                const float2 a = p[i], b = p[i + s];
                p[i] = __fadd2_rn(a, b);
                p[i + s] = __ffma2_rn(b, neg1, a);
            }
    const float2 sc = make_float2(0.17677669529663687f, 0.17677669529663687f);
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = __fmul2_rn(make_float2(__fadd_rn(p[i].x, p[i].y), __fsub_rn(p[i].x, p[i].y)), sc);
}
__device__ __forceinline__ float mx_amax(const float *v) {
    float m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = mx_max_nan(mx_max_nan(v[i], v[i + 8]), mx_max_nan(v[i + 16], v[i + 24]));
    return mx_max_nan(mx_max_nan(mx_max_nan(m[0], m[1]), mx_max_nan(m[2], m[3])),
                      mx_max_nan(mx_max_nan(m[4], m[5]), mx_max_nan(m[6], m[7])));
}
// One whole block in a thread -> its code words (4 or 8 of them) and its scale byte.  v is scaled in place.
template <int BITS>
__device__ __forceinline__ uint32_t mx_round_block(float *v, uint32_t *w) {
    const uint32_t s = mx_scale_byte<BITS>(mx_amax(v));
    const float inv = mx_inverse_scale(s);
    const float2 inv2 = make_float2(inv, inv);
    float2 *p = reinterpret_cast<float2 *>(v);
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = __fmul2_rn(p[i], inv2);
    if (s == 255u) {
#pragma unroll
        for (int i = 0; i < BITS; ++i) w[i] = 0u;
    } else if constexpr (BITS == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = mx_e2m1x8(v + 8 * i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = mx_e4m3x4(v + 4 * i);
    }
    return s;
}
// 32 elements of `dtype` from a 16-byte aligned address.
template <bool F32>
__device__ __forceinline__ void mx_load_block(const void *src, float *v) {
    if constexpr (F32) {
        uint32_t w[32];
        load_words<32>(src, w);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(w[i]);
    } else {
        uint32_t w[16];
        load_words<16>(src, w);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}
#endif

}  // namespace quest
