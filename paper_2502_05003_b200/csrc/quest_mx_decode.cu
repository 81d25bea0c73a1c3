// The microscaled product for a few rows of x (a decoding step): y[m][n] = sum_k x[m][k] w[n][k], up to 32 rows m.
//
// Bound by reading w (4.25 bits an element), not by arithmetic, so it runs on mma.sync m16n8k16 with the rows of w as the
// 16-wide side: a tcgen05 tile would be empty but for these rows, and 128 rows of w a CTA would leave most SMs without one.
// Both operands are turned into bfloat16 with their scales multiplied in, which is exact (E2M1 has 2 and E4M3 4 significant
// bits, the exponents fit), so products are exact and sums binary32, as on the block-scaled path.
//
// A CTA takes 16 RT rows of w, its warps split K.  In a warp, lane (g, t) = (lane / 4, lane % 4) reads whole blocks: of 128
// elements of K block t of rows g and g + 8 of w and of row g of x.  The contraction index of an m16n8k16 product only has to
// be the same on both sides, so each of eight products takes four elements of every lane's block, in the order in which the
// nibbles of a word unpack (element p beside p + 4): nothing is exchanged between lanes, and a lane that quantizes x has
// all 32 elements under one scale.  The warps' partial sums meet in shared memory.
#include "quest_mx.cuh"

namespace quest {
namespace {

constexpr int WARPS = 8;

struct FewArgs {
    const void *x;                  // [M x K], to be quantized; or NULL and
    const uint8_t *xq, *sx;         // its codes and scales
    long long ldx;
    const uint8_t *wq, *sw;
    int M, N, K, tiles;             // tiles: scale tiles of a row
    void *y;
    long long ldy;
    int x_f32, rotate, y_f32;
};

__device__ __forceinline__ void mma_bf16(float *c, const uint32_t *a, const uint32_t *b) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// Nibbles p and p + 4 of a word of E2M1 codes -> bfloat16 pair times `scale`.  Sign, exponent and mantissa bit go to the
// places that bfloat16 has for them, which reads 2^-126 times the value (zero and 0.5 as subnormals); the factor 2^126 and the scale
// are two products because together they may pass 2^127.
template <int P>
__device__ __forceinline__ uint32_t unpack_e2m1(uint32_t w, uint32_t scale) {
    const uint32_t mag = (P == 0 ? w << 6 : P == 1 ? w << 2 : P == 2 ? w >> 2 : w >> 6) & 0x01C001C0u;
    const uint32_t sign = (P == 0 ? w << 12 : P == 1 ? w << 8 : P == 2 ? w << 4 : w) & 0x80008000u;
    return mul_bf16x2(mul_bf16x2(mag | sign, 0x7E807E80u), scale);
}
// A block of x in the order of the products: word 2 i + j of f holds elements 8 q + p and 8 q + p + 4, q = i / 2, p = 2 (i % 2) + j.
template <int XB>
__device__ __forceinline__ void quantized_fragments(float *v, uint32_t *f) {
    const uint32_t s = mx_scale_byte<XB>(mx_amax(v));
    const float inv = mx_inverse_scale(s), sc = mx_scale_f32(s);
    const float2 inv2 = make_float2(inv, inv), sc2 = make_float2(sc, sc);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const float2 t = __fmul2_rn(make_float2(v[8 * q + p], v[8 * q + p + 4]), inv2);
            uint32_t h;
            if constexpr (XB == 4)
                asm("{\n\t.reg .b8 a;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}"
                    : "=r"(h) : "f"(t.x), "f"(t.y));
            else
                asm("{\n\t.reg .b16 a;\n\tcvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}"
                    : "=r"(h) : "f"(t.x), "f"(t.y));
            const float2 u = __fmul2_rn(__half22float2(*reinterpret_cast<const __half2 *>(&h)), sc2);
            f[4 * q + p] = s == 255u ? 0x7FC07FC0u : pack_bf16x2(u.x, u.y);
        }
}
template <int XB>
__device__ __forceinline__ void stored_fragments(const uint8_t *codes, uint32_t s, uint32_t *f) {
    if constexpr (XB == 4) {
        const uint4 c = __ldg(reinterpret_cast<const uint4 *>(codes));
        const uint32_t w[4] = {c.x, c.y, c.z, c.w}, sc = mx_scale_bf16x2(s);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            f[4 * q] = unpack_e2m1<0>(w[q], sc); f[4 * q + 1] = unpack_e2m1<1>(w[q], sc);
            f[4 * q + 2] = unpack_e2m1<2>(w[q], sc); f[4 * q + 3] = unpack_e2m1<3>(w[q], sc);
        }
    } else {
        uint32_t w[8];
        load_words<8>(codes, w);
        const float sc = mx_scale_f32(s);
        const float2 sc2 = make_float2(sc, sc);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const float2 u = __fmul2_rn(mx_values_e4m3(__byte_perm(w[2 * q], w[2 * q + 1], p | (p + 4) << 4)), sc2);
                f[4 * q + p] = pack_bf16x2(u.x, u.y);
            }
    }
}

template <int XB, int TT, int RT>
__global__ void __launch_bounds__(32 * WARPS)
mx_few_rows_kernel(const __grid_constant__ FewArgs a) {
    __shared__ float part[WARPS][TT * 8][RT * 16];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * (16 * RT), blocks = a.K / MX_BLOCK;
    float acc[RT][TT][4] = {};
    for (int group = warp; group < a.tiles; group += WARPS) {
        const int block = 4 * group + t;
        const bool in_k = block < blocks;
        uint4 w[RT][2];
        uint32_t ws[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = n0 + 16 * r + 8 * h + g;
                const bool in = in_k && n < a.N;
                w[r][h] = in ? __ldg(reinterpret_cast<const uint4 *>(a.wq + ((long long)n * a.K + block * MX_BLOCK) / 2)) : make_uint4(0u, 0u, 0u, 0u);
                ws[r][h] = in ? __ldg(a.sw + mx_scale_at(n, block, a.tiles)) : 0u;
            }
        uint32_t xf[TT][16];
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) {
            const int m = 8 * tt + g;
            if (!in_k || m >= a.M) {
#pragma unroll
                for (int i = 0; i < 16; ++i) xf[tt][i] = 0u;
            } else if (a.x) {
                float v[32];
                const long long at = m * a.ldx + block * MX_BLOCK;
                if (a.x_f32) mx_load_block<true>(static_cast<const float *>(a.x) + at, v);
                else mx_load_block<false>(static_cast<const uint16_t *>(a.x) + at, v);
                if (a.rotate) mx_rotate(v);
                quantized_fragments<XB>(v, xf[tt]);
            } else {
                const long long at = (long long)m * a.K + block * MX_BLOCK;
                stored_fragments<XB>(a.xq + at * XB / 8, __ldg(a.sx + mx_scale_at(m, block, a.tiles)), xf[tt]);
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const uint32_t s0 = mx_scale_bf16x2(ws[r][0]), s1 = mx_scale_bf16x2(ws[r][1]);
            const uint32_t u0[4] = {w[r][0].x, w[r][0].y, w[r][0].z, w[r][0].w}, u1[4] = {w[r][1].x, w[r][1].y, w[r][1].z, w[r][1].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t lo[4] = {unpack_e2m1<0>(u0[q], s0), unpack_e2m1<0>(u1[q], s1), unpack_e2m1<1>(u0[q], s0), unpack_e2m1<1>(u1[q], s1)};
                const uint32_t hi[4] = {unpack_e2m1<2>(u0[q], s0), unpack_e2m1<2>(u1[q], s1), unpack_e2m1<3>(u0[q], s0), unpack_e2m1<3>(u1[q], s1)};
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) {
                    mma_bf16(acc[r][tt], lo, &xf[tt][4 * q]);
                    mma_bf16(acc[r][tt], hi, &xf[tt][4 * q + 2]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int c = 0; c < 4; ++c) part[warp][8 * tt + 2 * t + (c & 1)][16 * r + 8 * (c >> 1) + g] = acc[r][tt][c];
    __syncthreads();
    for (int i = threadIdx.x; i < TT * 8 * RT * 16; i += 32 * WARPS) {
        const int m = i / (RT * 16), c = i - m * (RT * 16), n = n0 + c;
        if (m >= a.M || n >= a.N) continue;
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) s += part[k][m][c];
        if (a.y_f32) static_cast<float *>(a.y)[m * a.ldy + n] = s;
        else static_cast<__nv_bfloat16 *>(a.y)[m * a.ldy + n] = __float2bfloat16_rn(s);
    }
}

template <int XB, int TT>
cudaError_t launch_tokens(const FewArgs &a, int rt, cudaStream_t st) {
    const auto go = [&](auto kernel) { return launch_pdl(kernel, dim3((unsigned)((a.N + 16 * rt - 1) / (16 * rt))), dim3(32 * WARPS), 0, st, 1, a); };
    return rt == 1 ? go(mx_few_rows_kernel<XB, TT, 1>) : rt == 2 ? go(mx_few_rows_kernel<XB, TT, 2>) : go(mx_few_rows_kernel<XB, TT, 3>);
}
template <int XB>
cudaError_t launch_bits(const FewArgs &a, int rt, cudaStream_t st) {
    return a.M <= 8 ? launch_tokens<XB, 1>(a, rt, st) : a.M <= 16 ? launch_tokens<XB, 2>(a, rt, st) : a.M <= 24 ? launch_tokens<XB, 3>(a, rt, st) : launch_tokens<XB, 4>(a, rt, st);
}

}  // namespace

int launch_mx_few_rows(const void *x, int x_dtype, int64_t ldx, const uint8_t *xq, const uint8_t *sx, int bits_x, int had_block,
                       const uint8_t *wq, const uint8_t *sw, int64_t M, int64_t N, int64_t K, void *y, int y_dtype, int64_t ldy,
                       cudaStream_t st) {
    const FewArgs a = {x, xq, sx, (long long)ldx, wq, sw, (int)M, (int)N, (int)K, (int)((K + 127) / 128), y, (long long)ldy,
                       x_dtype == QUEST_F32, had_block == 32, y_dtype == QUEST_F32};
    const int64_t room = 2 * (int64_t)num_sms();
    const int rt = N <= 16 * room ? 1 : N <= 32 * room ? 2 : 3;
    const cudaError_t e = bits_x == 4 ? launch_bits<4>(a, rt, st) : launch_bits<8>(a, rt, st);
    return e == cudaSuccess ? QUEST_OK : cuda_fail(e);
}

}  // namespace quest
