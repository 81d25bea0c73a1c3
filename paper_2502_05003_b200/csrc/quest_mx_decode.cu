// The microscaled product for a few rows of x and a small w (mx_product): y[m][n] = sum_k x[m][k] w[n][k], up to 32 rows m.
//
// Bound by reading w (4.25 bits an element) and, beside that, by the instructions that turn codes into operands, so it runs on
// mma.sync m16n8k16 with the rows of w as the 16-wide side: 128 rows of w a CTA, as the tcgen05 products take, would leave most SMs
// without one or cost sums over a cluster.  Codes become binary16 operands with the hardware conversions, two elements an
// instruction and exactly (E2M1 has 2 and E4M3 4 significant bits); their scales, which may pass binary16's range, stay out:
// a block of 32 is two products from zero, and its sums join the accumulators times one scale after the other in binary32:
//     acc[n][m] += 2^sw[n] (2^sx[m] sum_32 qw[n] qx[m])
// (the two scales alone may meet past 2^128 over sums that are 0, or less than 1).  A block's sum c is 0 or 2^-10 to 2^17 in steps
// of 2^-10, so times a scale below 2^111 it neither overflows nor loses a bit (steps of 2^-137 at least), and the rest is one
// rounding.  Warps (FUSED: CTAs) that meet a scale of x of 2^65 or more take their sums once more, the smaller scale of each pair first.
//
// A CTA takes 16 RT rows of w, its warps split K in groups of 128 elements.  w goes through shared memory (16-byte asynchronous
// copies, two groups a warp in flight, rows 80 bytes apart so that reads meet no bank twice), because the four lanes that share a row
// in a product each need a quarter of every block.  The contraction index only has to be the same on both sides: lane t of a
// row takes elements 8 t .. 8 t + 7 of a block.  The warps' partial sums meet in shared memory.
// FUSED (mx_fuses_quantizer): every CTA quantizes x while the first copies of w are under way, four
// threads to a block, and leaves operands and scale bytes in shared memory.  One launch, and the host pays for one.
//
// Device time back to back, weights out of L2: 1 x 2048 x 2048 3.7 us fused, 2.9 from codes (the floor of 2.3 MB is 0.35: launch,
// one round trip to memory, conversions and sums); 16 x 2048 x 2048 3.3 from codes, where conversions, products and scaling fill 30 % of
// the issue slots.  (bfloat16 operands unpacked with shifts and masks took 1.04 times the time of the conversions, and every CTA
// quantizing all of 24 rows of x 2.4 times, on 24 x 5504 x 2048, which the exchanged tiles take now.)
#include <algorithm>

#include "quest_mx.cuh"

namespace quest {
namespace {

constexpr int WARPS = 16;
constexpr int PITCH = 80;                        // bytes between the rows of a group (64 bytes of codes)
// floats between the tokens of a warp's partial sums: the 32 lanes of a store meet 32 banks
__host__ __device__ constexpr int part_pitch(int rt) { return 16 * rt + 4; }
// FUSED: bytes between the rows of x as operands; eight lanes read 64 bytes each of two rows without a conflict
__host__ __device__ constexpr int x_pitch(int tiles) { return 256 * tiles + 64; }

struct FewArgs {
    const void *x;                  // FUSED: [M x K], else
    const uint8_t *xq, *sx;         // its codes and scales
    long long ldx;
    const uint8_t *wq, *sw;
    int M, N, K, tiles;             // tiles: groups of 128 elements (scale tiles) of a row
    void *y;
    long long ldy;
    int x_f32, rotate, y_f32;
};

// c = a b, from zero
__device__ __forceinline__ void mma_f16_first(float *c, const uint32_t *a, const uint32_t *b) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]), "f"(0.0f));
}
__device__ __forceinline__ void mma_f16(float *c, const uint32_t *a, const uint32_t *b) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// Eight E2M1 codes -> four binary16 pairs; four E4M3 bytes -> two.
__device__ __forceinline__ void f16_of_e2m1x8(uint32_t w, uint32_t *h) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}
__device__ __forceinline__ void f16_of_e4m3x4(uint32_t w, uint32_t *h) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(h[0]), "=r"(h[1])
        : "r"(w));
}
// Scales of blocks b and b + 1 (b even) from a word of four scale bytes, as bfloat16, and one of them in binary32: exact, NaN for 255.
__device__ __forceinline__ uint32_t scale_pair(uint32_t bytes, int b) {
    uint32_t h;
    asm("{\n\t.reg .b16 p, q;\n\tmov.b32 {p, q}, %1;\n\tcvt.rn.bf16x2.ue8m0x2 %0, p;\n\t}" : "=r"(h) : "r"(b ? bytes >> 16 : bytes));
    return h;
}
__device__ __forceinline__ float scale_of(uint32_t pair, int b) { return __uint_as_float(b & 1 ? pair & 0xFFFF0000u : pair << 16); }

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool in) {       // zeros where not in
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}

// A quarter of a block of x in each of four lanes -> its operand words and the block's scale byte (the same in the four).
template <int XB>
__device__ __forceinline__ uint32_t quantize_quarter(float *v, bool rotate, int lane, uint32_t *h) {
    if (rotate) {
#pragma unroll
        for (int o = 2; o >= 1; o >>= 1)                                  // strides 16 and 8
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float p = __shfl_xor_sync(0xffffffffu, v[k], o);
                v[k] = (lane & o) ? __fsub_rn(p, v[k]) : __fadd_rn(v[k], p);
            }
#pragma unroll
        for (int o = 4; o >= 1; o >>= 1)
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if ((k & o) == 0) {
                    const float p = v[k], q = v[k + o];
                    v[k] = __fadd_rn(p, q);
                    v[k + o] = __fsub_rn(p, q);
                }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __fmul_rn(v[k], 0.17677669529663687f);
    }
    float m = mx_max_nan(mx_max_nan(mx_max_nan(v[0], v[1]), mx_max_nan(v[2], v[3])),
                         mx_max_nan(mx_max_nan(v[4], v[5]), mx_max_nan(v[6], v[7])));
    m = mx_max_nan(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = mx_max_nan(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const uint32_t s = mx_scale_byte<XB>(m);
    const float inv = mx_inverse_scale(s);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = __fmul_rn(v[k], inv);
    if constexpr (XB == 4) {
        f16_of_e2m1x8(s == 255u ? 0u : mx_e2m1x8(v), h);
    } else {
        f16_of_e4m3x4(s == 255u ? 0u : mx_e4m3x4(v), h);
        f16_of_e4m3x4(s == 255u ? 0u : mx_e4m3x4(v + 4), h + 2);
    }
    return s;
}

// The sums of a warp whatever the scales, into its place of the partial sums: 16 rows of w, eight of x and one block at a time, codes
// straight from memory.  The smaller of two scales cannot make a block's sum overflow unless the whole does; a NaN counts as the smaller.
// Not inlined: in between the kernel's own instructions it costs a lone call of 1 x 2048 x 2048 0.15 us.
template <int XB, int TT, int RT, bool FUSED>
__device__ __noinline__ void sums_of_any_scales(const FewArgs &a, const uint8_t *x_operands, const uint8_t *x_scales, float *mine) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int blocks = a.K / MX_BLOCK;
#pragma unroll 1
    for (int i = 0; i < RT * TT; ++i) {
        const int n = blockIdx.x * (16 * RT) + 16 * (i / TT) + g, m0 = 8 * (i % TT);
        float acc[4] = {};
#pragma unroll 1
        for (int block = 4 * warp; block < blocks; block = (block & 3) == 3 ? block + 4 * WARPS - 3 : block + 1) {
            uint32_t w[2][4], x[4];
            float sw[2], sx[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool in = n + 8 * h < a.N;
                const long long row = (long long)(n + 8 * h) * a.K;
                f16_of_e2m1x8(in ? __ldg(reinterpret_cast<const uint32_t *>(a.wq + (row + block * MX_BLOCK + 8 * t) / 2)) : 0u, w[h]);
                sw[h] = in ? mx_scale_f32(__ldg(a.sw + mx_scale_at(n + 8 * h, block, a.tiles))) : 0.0f;
                const int m = m0 + 2 * t + h;
                if constexpr (FUSED) sx[h] = m < a.M ? mx_scale_f32(x_scales[4 * (m * a.tiles) + block]) : 0.0f;
                else sx[h] = m < a.M ? mx_scale_f32(__ldg(a.sx + mx_scale_at(m, block, a.tiles))) : 0.0f;
            }
            const bool in = m0 + g < a.M;
            const long long at = (long long)(m0 + g) * a.K + block * MX_BLOCK + 8 * t;
            if constexpr (FUSED) {
                const uint4 q = in ? *reinterpret_cast<const uint4 *>(x_operands + g * x_pitch(a.tiles) + 64 * block + 16 * t) : make_uint4(0u, 0u, 0u, 0u);
                x[0] = q.x; x[1] = q.y; x[2] = q.z; x[3] = q.w;
            } else if constexpr (XB == 4) {
                f16_of_e2m1x8(in ? __ldg(reinterpret_cast<const uint32_t *>(a.xq + at / 2)) : 0u, x);
            } else {
                const uint2 q = in ? __ldg(reinterpret_cast<const uint2 *>(a.xq + at)) : make_uint2(0u, 0u);
                f16_of_e4m3x4(q.x, x);
                f16_of_e4m3x4(q.y, x + 2);
            }
            const uint32_t a0[4] = {w[0][0], w[1][0], w[0][1], w[1][1]}, a1[4] = {w[0][2], w[1][2], w[0][3], w[1][3]};
            float c[4];
            mma_f16_first(c, a0, x);
            mma_f16(c, a1, x + 2);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float least;
                asm("min.NaN.f32 %0, %1, %2;" : "=f"(least) : "f"(sx[k & 1]), "f"(sw[k >> 1]));
                acc[k] = __fmaf_rn(__fmul_rn(c[k], least), fmaxf(sx[k & 1], sw[k >> 1]), acc[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) mine[(m0 + 2 * t + (k & 1)) * part_pitch(RT) + 16 * (i / TT) + 8 * (k >> 1) + g] = acc[k];
    }
}

// Two CTAs to an SM where a round of them has that many (launch_mx_few_rows); elsewhere registers for one (16 x 2048 x 2048, 4 bits: 3.0 us
// with 102 of them, 4.6 with 64).
template <int XB, int TT, int RT, bool FUSED>
__global__ void __launch_bounds__(32 * WARPS, TT == 1 && RT == 1 ? 2 : 1)
mx_few_rows_kernel(const __grid_constant__ FewArgs a) {
    static_assert(!FUSED || TT == 1, "x is quantized on the way for up to eight rows");
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * (16 * RT), blocks = a.K / MX_BLOCK;
    if constexpr (TT == 1) {
        // the first group of w on its way into L2 while the kernel before this one still runs (1 x 2048 x 2048 fused 3.98 -> 3.77 us)
        if (lane < 16 && warp < a.tiles)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int n = n0 + 16 * r + lane;
                if (n < a.N) asm volatile("prefetch.global.L2 [%0];" ::"l"(a.wq + ((long long)n * a.K + warp * 128) / 2) : "memory");
            }
    }
    pdl_wait();
    constexpr int GROUP_BYTES = RT * 16 * PITCH;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (2 * GROUP_BYTES);
    const auto request = [&](int group, int slot) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = (lane >> 2) + 8 * i, n = n0 + 16 * r + row, block = 4 * group + t;
                const bool in = n < a.N && block < blocks;
                copy16(ring + slot * GROUP_BYTES + (16 * r + row) * PITCH + 16 * t,
                       a.wq + (in ? ((long long)n * a.K + block * MX_BLOCK) / 2 : 0), in);
            }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    float acc[RT][TT][4] = {};
    if (warp < a.tiles) request(warp, 0);
    // FUSED: operands of x, rows of whole groups, and behind them four scale bytes a group
    uint8_t *x_operands = smem + WARPS * 2 * GROUP_BYTES, *x_scales = x_operands + a.M * x_pitch(a.tiles);
    int any_large = 0;                           // a scale of x of 2^65 or more (or NaN)
    if constexpr (FUSED) {
        const int quarters = 16 * a.tiles;       // of a row
        for (int i = threadIdx.x; i < (a.M * quarters + 31) / 32 * 32; i += 32 * WARPS) {
            const int m = i / quarters, q = i - m * quarters;
            float v[8];
            const bool in = m < a.M && 8 * q < a.K;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.0f;
            if (in) {
                const long long at = m * a.ldx + 8 * q;
                if (a.x_f32) {
                    const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(a.x) + at);
                    const float4 p0 = __ldg(p), p1 = __ldg(p + 1);
                    v[0] = p0.x; v[1] = p0.y; v[2] = p0.z; v[3] = p0.w;
                    v[4] = p1.x; v[5] = p1.y; v[6] = p1.z; v[7] = p1.w;
                } else {
                    const uint4 w4 = __ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.x) + at));
                    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        v[2 * k] = __uint_as_float(w[k] << 16);
                        v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
                    }
                }
            }
            uint32_t h[4];
            const uint32_t s = quantize_quarter<XB>(v, a.rotate, lane, h);      // a block's four quarters are lanes of one warp
            if (m < a.M) {
                *reinterpret_cast<uint4 *>(x_operands + m * x_pitch(a.tiles) + 16 * q) = make_uint4(h[0], h[1], h[2], h[3]);
                any_large |= s >= 192u;
                if ((q & 3) == 0) x_scales[4 * (m * a.tiles) + (q >> 2)] = (uint8_t)s;
            }
        }
        any_large = __syncthreads_or(any_large);
    }
    uint32_t large = 0;                          // bit 7 of a byte: the same in the codes' scales
    int slot = 0;
    for (int group = warp; group < a.tiles; group += WARPS, slot ^= 1) {
        const bool more = group + WARPS < a.tiles;
        if (more) request(group + WARPS, slot ^ 1);
        uint32_t ws[RT][2];                      // four scale bytes of rows g and g + 8
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = n0 + 16 * r + 8 * h + g;
                ws[r][h] = n < a.N ? __ldg(reinterpret_cast<const uint32_t *>(a.sw + mx_scale_at(n, 4 * group, a.tiles))) : 0u;
            }
        // x: a quarter of each of the four blocks of token g; the scales that lane's columns of the accumulators take
        uint32_t xr[TT][4][XB / 4];              // codes, which become operands when their block's turn comes
        uint32_t xs[TT][2];
        if constexpr (FUSED) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
                xs[0][c] = 2 * t + c < a.M ? *reinterpret_cast<const uint32_t *>(x_scales + 4 * ((2 * t + c) * a.tiles + group)) : 0u;
        } else {
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) {
                const int m = 8 * tt + g;
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const bool in = m < a.M && 4 * group + b < blocks;
                    const long long at = (long long)m * a.K + (4 * group + b) * MX_BLOCK + 8 * t;
                    if constexpr (XB == 4) {
                        xr[tt][b][0] = in ? __ldg(reinterpret_cast<const uint32_t *>(a.xq + at / 2)) : 0u;
                    } else {
                        const uint2 q = in ? __ldg(reinterpret_cast<const uint2 *>(a.xq + at)) : make_uint2(0u, 0u);
                        xr[tt][b][0] = q.x;
                        xr[tt][b][1] = q.y;
                    }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int col = 8 * tt + 2 * t + c;
                    xs[tt][c] = col < a.M ? __ldg(reinterpret_cast<const uint32_t *>(a.sx + mx_scale_at(col, 4 * group, a.tiles))) : 0u;
                }
            }
        }
        if constexpr (!FUSED)
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) large |= (xs[tt][0] & (xs[tt][0] << 1)) | (xs[tt][1] & (xs[tt][1] << 1));
        if (more) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
        const uint8_t *mine = smem + warp * (2 * GROUP_BYTES) + slot * GROUP_BYTES + g * PITCH + 4 * t;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            float2 sx2[TT];
            uint32_t xb[TT][4];
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) {
                if constexpr (FUSED) {
                    const uint4 q = g < a.M ? *reinterpret_cast<const uint4 *>(x_operands + g * x_pitch(a.tiles) + 256 * group + 64 * b + 16 * t)
                                            : make_uint4(0u, 0u, 0u, 0u);
                    xb[tt][0] = q.x; xb[tt][1] = q.y; xb[tt][2] = q.z; xb[tt][3] = q.w;
                } else if constexpr (XB == 4) {
                    f16_of_e2m1x8(xr[tt][b][0], xb[tt]);
                } else {
                    f16_of_e4m3x4(xr[tt][b][0], xb[tt]);
                    f16_of_e4m3x4(xr[tt][b][1], xb[tt] + 2);
                }
                sx2[tt] = make_float2(scale_of(scale_pair(xs[tt][0], b & 2), b), scale_of(scale_pair(xs[tt][1], b & 2), b));
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                uint32_t lo[4], hi[4];
                f16_of_e2m1x8(*reinterpret_cast<const uint32_t *>(mine + 16 * r * PITCH + 16 * b), lo);
                f16_of_e2m1x8(*reinterpret_cast<const uint32_t *>(mine + (16 * r + 8) * PITCH + 16 * b), hi);
                const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
                const float s0 = scale_of(scale_pair(ws[r][0], b & 2), b), s1 = scale_of(scale_pair(ws[r][1], b & 2), b);
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) {
                    float c[4];
                    mma_f16_first(c, a0, xb[tt]);
                    mma_f16(c, a1, xb[tt] + 2);
                    float2 *p = reinterpret_cast<float2 *>(acc[r][tt]);
                    p[0] = __ffma2_rn(__fmul2_rn(make_float2(c[0], c[1]), sx2[tt]), make_float2(s0, s0), p[0]);
                    p[1] = __ffma2_rn(__fmul2_rn(make_float2(c[2], c[3]), sx2[tt]), make_float2(s1, s1), p[1]);
                }
            }
        }
        __syncwarp();                            // the next round's copies overwrite this slot
    }
    __syncthreads();                             // every warp has left the ring
    float *part = reinterpret_cast<float *>(smem);               // [warp][token][row of w]
    constexpr int ROWS = RT * 16, TOKENS = TT * 8, P = part_pitch(RT);
    if constexpr (!FUSED) any_large = __any_sync(0xffffffffu, (large & 0x80808080u) != 0);
    if (any_large) {
        sums_of_any_scales<XB, TT, RT, FUSED>(a, x_operands, x_scales, part + warp * TOKENS * P);     // (x lies behind the ring)
    } else {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    part[(warp * TOKENS + 8 * tt + 2 * t + (c & 1)) * P + 16 * r + 8 * (c >> 1) + g] = acc[r][tt][c];
    }
    __syncthreads();
    const int live = min(WARPS, a.tiles);
    for (int i = threadIdx.x; i < TOKENS * ROWS; i += 32 * WARPS) {
        const int m = i / ROWS, c = i - m * ROWS, n = n0 + c;
        if (m >= a.M || n >= a.N) continue;
        float s = 0.0f;
        for (int k = 0; k < live; ++k) s += part[(k * TOKENS + m) * P + c];
        if (a.y_f32) static_cast<float *>(a.y)[m * a.ldy + n] = s;
        else static_cast<__nv_bfloat16 *>(a.y)[m * a.ldy + n] = __float2bfloat16_rn(s);
    }
}

template <int XB, int TT, int RT, bool FUSED>
cudaError_t launch_shape(const FewArgs &a, cudaStream_t st) {
    constexpr int ring = WARPS * 2 * RT * 16 * PITCH, most = 232448;
    const int bytes = std::max(ring + (FUSED ? a.M * (x_pitch(a.tiles) + 4 * a.tiles) : 0), WARPS * TT * 8 * part_pitch(RT) * 4);
    static DynamicSmemOnce smem_attr;
    const cudaError_t e = smem_attr.set(mx_few_rows_kernel<XB, TT, RT, FUSED>, most);
    if (e != cudaSuccess) return e;
    return launch_pdl(mx_few_rows_kernel<XB, TT, RT, FUSED>, dim3((unsigned)((a.N + 16 * RT - 1) / (16 * RT))), dim3(32 * WARPS), (size_t)bytes, st, 1, a);
}
template <int XB, int TT, bool FUSED>
cudaError_t launch_rows(const FewArgs &a, int rt, cudaStream_t st) {
    if (rt == 1) return launch_shape<XB, TT, 1, FUSED>(a, st);
    if constexpr (TT == 1) return launch_shape<XB, TT, 3, FUSED>(a, st);
    else return launch_shape<XB, TT, 2, FUSED>(a, st);
}
template <int XB>
cudaError_t launch_tokens(const FewArgs &a, int rt, cudaStream_t st) {
    if (a.x) return launch_rows<XB, 1, true>(a, rt, st);
    return a.M <= 8 ? launch_rows<XB, 1, false>(a, rt, st) : a.M <= 16 ? launch_rows<XB, 2, false>(a, rt, st)
         : a.M <= 24 ? launch_rows<XB, 3, false>(a, rt, st) : launch_rows<XB, 4, false>(a, rt, st);
}

}  // namespace

int launch_mx_few_rows(const void *x, int x_dtype, int64_t ldx, const uint8_t *xq, const uint8_t *sx, int bits_x, int had_block,
                       const uint8_t *wq, const uint8_t *sw, int64_t M, int64_t N, int64_t K, void *y, int y_dtype, int64_t ldy,
                       cudaStream_t st) {
    const FewArgs a = {x, xq, sx, (long long)ldx, wq, sw, (int)M, (int)N, (int)K, (int)((K + 127) / 128), y, (long long)ldy,
                       x_dtype == QUEST_F32, had_block == 32, y_dtype == QUEST_F32};
    // rows of w a CTA: as few as one round of CTAs allows, for up to eight rows of x two 16-row CTAs to an SM.  From codes, us with 16 rows a
    // CTA and with more: 1 x 4736 x 2048 3.3, 48 rows 3.9; 1 x 5504 x 2048 4.7, 3.9; 8 x 4096 x 4096 5.4, 6.1; 8 x 5504 x 4096 8.1, 6.2;
    // 16 x 2368 x 2048 3.5, 32 rows 4.0; 16 x 2400 x 2048 5.6, 4.3; 24 x 2400 x 1280 5.8, 4.8.  Longer w does not come here (mx_product)
    const int64_t sms = num_sms();
    const int rt = M <= 8 ? (N <= 32 * sms ? 1 : 3) : N <= 16 * sms ? 1 : 2;
    const cudaError_t e = bits_x == 4 ? launch_tokens<4>(a, rt, st) : launch_tokens<8>(a, rt, st);
    return e == cudaSuccess ? QUEST_OK : cuda_fail(e);
}

}  // namespace quest
