// Microscaled tensors: quantisation, reading back, and the entry points of the microscaled layer.
//
//   scale byte s = clamp(floor(log2 max|v|) - emax, -127, 127) + 127     emax = 2 (E2M1) or 8 (E4M3), v a block of 32
//   code         = RN_sat(v 2^(127 - s))                                  ties to even
//
// with v the elements as they are, or their orthonormal Walsh-Hadamard transform (binary32, a fixed order of sums).  The
// product of two tensors that were rotated alike needs no inverse transform.
#include <algorithm>

#include "quest_mx.cuh"

namespace quest {
namespace {

struct MxQuantArgs {
    MxJob job[2];
    long long first_block1;         // CTAs from this one on work on the second tensor
    int cols, rows_per_cta, tiles;  // tiles of four blocks in a row, the last one possibly part empty
    uint32_t magic;                 // ceil(2^32 / (4 tiles))
};

// A thread owns one block: 64 (bfloat16) or 128 bytes in, 16 or 32 bytes of codes and one scale byte out, nothing is
// exchanged.  A CTA takes whole rows of whole tiles, so that the scale bytes that fill up a tile are written too (zero).
// Bound by memory: 16384 x 4096 bfloat16 to 8 bits 32.8 us (6.2 TB/s), to 4 bits 29.3; rotated 37 and 35, where the sums,
// conversions and maxima of a block (344 instructions) take 61 % of the issue slots between the waits for loads.  Tried without
// gain (bfloat16): blocks requested one ahead (two, four, eight to a thread: 34.5 .. 36.8), more threads to an SM (41 .. 47, registers),
// maxima of three at once and 1 / sqrt(32) folded into the scale (35.2).  binary32 is as near to memory, rotated too: 55 to 8 bits, 51 to 4.
template <bool F32, bool ROTATE>
__global__ void __launch_bounds__(256)
mx_quantize_kernel(const __grid_constant__ MxQuantArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const bool second = blockIdx.x >= a.first_block1;
    const MxJob &t = a.job[second ? 1 : 0];
    const long long row0 = (blockIdx.x - (second ? a.first_block1 : 0)) * (long long)a.rows_per_cta;
    const int per_row = 4 * a.tiles;
    const long long rows_padded = (t.rows + 127) / 128 * 128;
    const int n = (int)min((long long)a.rows_per_cta, rows_padded - row0) * per_row;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int r = (int)__umulhi((uint32_t)i, a.magic);
        const int block = i - r * per_row;
        const long long row = row0 + r;
        uint32_t s = 0;
        if (row < t.rows && block * MX_BLOCK < a.cols) {
            float v[32];
            mx_load_block<F32>(static_cast<const uint8_t *>(t.x) + (row * t.ld + block * MX_BLOCK) * (F32 ? 4 : 2), v);
            if constexpr (ROTATE) mx_rotate(v);
            uint32_t w[8];
            if (t.bits == 4) {
                s = mx_round_block<4>(v, w);
                *reinterpret_cast<uint4 *>(t.codes + (row * a.cols + block * MX_BLOCK) / 2) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                s = mx_round_block<8>(v, w);
                store_words<8>(t.codes + row * a.cols + block * MX_BLOCK, w);
            }
        }
        t.scales[mx_scale_at((int)row, block, a.tiles)] = (uint8_t)s;
    }
}

struct MxDequantArgs {
    MxDequantJob job[2];
    long long first_block1;
    int cols, rows_per_cta, tiles;
    uint32_t magic;                 // ceil(2^32 / (cols / 32)); 0 for rows of one block
};

// A thread reads one block and its scale byte and writes 64 or 128 bytes.  Bound by the writes: 16384 x 4096 from 8 bits to
// bfloat16 34 us (5.9 TB/s).
template <bool F32>
__global__ void __launch_bounds__(256)
mx_dequantize_kernel(const __grid_constant__ MxDequantArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const bool second = blockIdx.x >= a.first_block1;
    const MxDequantJob &t = a.job[second ? 1 : 0];
    const long long row0 = (blockIdx.x - (second ? a.first_block1 : 0)) * (long long)a.rows_per_cta;
    const int per_row = a.cols / MX_BLOCK;
    const int n = (int)min((long long)a.rows_per_cta, t.rows - row0) * per_row;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int r = a.magic ? (int)__umulhi((uint32_t)i, a.magic) : i;
        const int block = i - r * per_row;
        const long long row = row0 + r, at = row * a.cols + block * MX_BLOCK;
        const float sc = mx_scale_f32(__ldg(t.scales + mx_scale_at((int)row, block, a.tiles)));
        const float2 sc2 = make_float2(sc, sc);
        float2 v[16];
        if (t.bits == 4) {
            const uint4 q = __ldg(reinterpret_cast<const uint4 *>(t.codes + at / 2));
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = __fmul2_rn(mx_values_e2m1(w[j >> 2] >> (8 * (j & 3))), sc2);
        } else {
            uint32_t w[8];
            load_words<8>(t.codes + at, w);
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = __fmul2_rn(mx_values_e4m3(w[j >> 1] >> (16 * (j & 1))), sc2);
        }
        if constexpr (F32) {
            uint32_t o[32];
#pragma unroll
            for (int j = 0; j < 16; ++j) { o[2 * j] = __float_as_uint(v[j].x); o[2 * j + 1] = __float_as_uint(v[j].y); }
            store_words<32>(static_cast<float *>(t.out) + at, o);
        } else {
            uint32_t o[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[j].x, v[j].y);
                o[j] = *reinterpret_cast<const uint32_t *>(&h);
            }
            store_words<16>(static_cast<uint16_t *>(t.out) + at, o);
        }
        if (t.ones) reinterpret_cast<uint32_t *>(t.ones)[at / 32] = 0xFFFFFFFFu;
    }
}

bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Rows per CTA and threads for rows of `per_row` blocks: about 256 threads with a block each.
void row_split(int per_row, int &rows_per_cta, int &threads) {
    rows_per_cta = std::max(1, 256 / per_row);
    threads = std::min(256, (rows_per_cta * per_row + 31) / 32 * 32);
}

int check_rows(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld) {
    if (!x && rows != 0) return QUEST_ERR_NULL;
    if (dtype != QUEST_F32 && dtype != QUEST_BF16) return QUEST_ERR_DTYPE;
    if (!mx_rows_ok(rows) || !mx_cols_ok(cols) || ld < cols) return QUEST_ERR_SHAPE;
    if (!aligned(x, 16) || (rows > 1 && ld * (dtype == QUEST_F32 ? 4 : 2) % 16 != 0)) return QUEST_ERR_ALIGN;
    return QUEST_OK;
}

// What both products ask of codes, scales and y.
int check_product(const uint8_t *wq, const uint8_t *sw, int bits_x, int64_t M, int64_t N, int64_t K, const void *y, int y_dtype,
                  int64_t ldy) {
    if (!mx_bits_ok(bits_x)) return QUEST_ERR_BITS;
    if (!mx_rows_ok(M) || !mx_rows_ok(N) || !mx_cols_ok(K) || (bits_x == 8 && K % 128 != 0)) return QUEST_ERR_SHAPE;
    if (y_dtype != QUEST_F32 && y_dtype != QUEST_BF16) return QUEST_ERR_DTYPE;
    if (M == 0 || N == 0) return QUEST_OK;
    if (!wq || !sw || !y) return QUEST_ERR_NULL;
    if (ldy < N) return QUEST_ERR_SHAPE;
    // 4-bit rows that meet 8-bit ones are spread to bytes by the copy engine, which takes them from 32-byte boundaries
    if (!aligned(wq, bits_x == 8 ? 32 : 16) || !aligned(sw, 16) || !aligned(y, y_dtype == QUEST_F32 ? 4 : 2)) return QUEST_ERR_ALIGN;
    return QUEST_OK;
}
int product_of_codes(const uint8_t *xq, const uint8_t *sx, int bits_x, const uint8_t *wq, const uint8_t *sw, int64_t M, int64_t N, int64_t K,
                     void *y, int y_dtype, int64_t ldy, cudaStream_t st) {
    switch (mx_product(M, N, K, bits_x)) {
        case MxProduct::few: return launch_mx_few_rows(nullptr, 0, 0, xq, sx, bits_x, 1, wq, sw, M, N, K, y, y_dtype, ldy, st);
        case MxProduct::thin: return launch_mx_thin(xq, sx, bits_x, wq, sw, M, N, K, y, y_dtype, ldy, st);
        default: return launch_mx_gemm(xq, sx, bits_x, wq, sw, M, N, K, y, y_dtype, ldy, st);
    }
}

}  // namespace

int launch_mx_quantize(const MxJob *jobs, int njobs, int dtype, int64_t cols, int had_block, cudaStream_t st) {
    MxQuantArgs a = {};
    int threads;
    a.cols = (int)cols;
    a.tiles = (int)((cols + 127) / 128);
    row_split(4 * a.tiles, a.rows_per_cta, threads);
    a.magic = (uint32_t)((((uint64_t)1 << 32) + 4 * a.tiles - 1) / (4 * a.tiles));
    long long ctas = 0;
    for (int j = 0; j < 2; ++j) {
        a.job[j] = jobs[j < njobs ? j : 0];
        if (j == 1) a.first_block1 = ctas;
        if (j < njobs) ctas += ((a.job[j].rows + 127) / 128 * 128 + a.rows_per_cta - 1) / a.rows_per_cta;
    }
    if (ctas == 0) return QUEST_OK;
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3((unsigned)ctas), dim3((unsigned)threads), 0, st, 1, a); };
    const bool rotate = had_block == 32;
    const cudaError_t e = dtype == QUEST_F32 ? (rotate ? go(mx_quantize_kernel<true, true>) : go(mx_quantize_kernel<true, false>))
                                             : (rotate ? go(mx_quantize_kernel<false, true>) : go(mx_quantize_kernel<false, false>));
    return e == cudaSuccess ? QUEST_OK : cuda_fail(e);
}

int launch_mx_dequantize(const MxDequantJob *jobs, int njobs, int dtype, int64_t cols, cudaStream_t st) {
    MxDequantArgs a = {};
    int threads;
    a.cols = (int)cols;
    a.tiles = (int)((cols + 127) / 128);
    const int per_row = (int)(cols / MX_BLOCK);
    row_split(per_row, a.rows_per_cta, threads);
    a.magic = per_row == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + per_row - 1) / per_row);
    long long ctas = 0;
    for (int j = 0; j < 2; ++j) {
        a.job[j] = jobs[j < njobs ? j : 0];
        if (j == 1) a.first_block1 = ctas;
        if (j < njobs) ctas += (a.job[j].rows + a.rows_per_cta - 1) / a.rows_per_cta;
    }
    if (ctas == 0) return QUEST_OK;
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3((unsigned)ctas), dim3((unsigned)threads), 0, st, 1, a); };
    const cudaError_t e = dtype == QUEST_F32 ? go(mx_dequantize_kernel<true>) : go(mx_dequantize_kernel<false>);
    return e == cudaSuccess ? QUEST_OK : cuda_fail(e);
}

}  // namespace quest

using namespace quest;

extern "C" {

size_t quest_mx_scales_bytes(int64_t rows, int64_t cols) {
    return mx_rows_ok(rows) && mx_cols_ok(cols) ? mx_scales_bytes(rows, cols) : 0;
}

int quest_quantize_mx(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld_elems, int bits, int had_block,
                      uint8_t *codes, uint8_t *scales, void *stream) {
    int s;
    if (!mx_bits_ok(bits)) return QUEST_ERR_BITS;
    if ((s = check_rows(x, dtype, rows, cols, ld_elems))) return s;
    if (!mx_had_ok(had_block)) return QUEST_ERR_HAD_BLOCK;
    if (rows == 0) return QUEST_OK;
    if (!codes || !scales) return QUEST_ERR_NULL;
    if (!aligned(codes, 16)) return QUEST_ERR_ALIGN;
    if ((s = check_device())) return s;
    const MxJob job = {x, rows, ld_elems, codes, scales, bits};
    void *h = stage_begin(QUEST_STAGE_QUANT_X, reinterpret_cast<cudaStream_t>(stream));
    s = launch_mx_quantize(&job, 1, dtype, cols, had_block, reinterpret_cast<cudaStream_t>(stream));
    stage_end(h);
    return s;
}

int quest_dequantize_mx(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, int bits, void *out, int out_dtype,
                        void *stream) {
    if (!mx_bits_ok(bits)) return QUEST_ERR_BITS;
    if (out_dtype != QUEST_F32 && out_dtype != QUEST_BF16) return QUEST_ERR_DTYPE;
    if (!mx_rows_ok(rows) || !mx_cols_ok(cols)) return QUEST_ERR_SHAPE;
    if (rows == 0) return QUEST_OK;
    if (!codes || !scales || !out) return QUEST_ERR_NULL;
    if (!aligned(codes, 16) || !aligned(out, 16)) return QUEST_ERR_ALIGN;
    const int s = check_device();
    if (s) return s;
    const MxDequantJob job = {codes, scales, rows, out, nullptr, bits};
    return launch_mx_dequantize(&job, 1, out_dtype, cols, reinterpret_cast<cudaStream_t>(stream));
}

int quest_gemm_mx(const uint8_t *xq, const uint8_t *sx, int bits_x, const uint8_t *wq, const uint8_t *sw, int64_t M, int64_t N,
                  int64_t K, void *y, int y_dtype, int64_t ldy_elems, void *stream) {
    int s = check_product(wq, sw, bits_x, M, N, K, y, y_dtype, ldy_elems);
    if (s) return s;
    if (M == 0 || N == 0) return QUEST_OK;
    if (!xq || !sx) return QUEST_ERR_NULL;
    if (!aligned(xq, 16) || !aligned(sx, 16)) return QUEST_ERR_ALIGN;
    if ((s = check_device())) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    void *h = stage_begin(QUEST_STAGE_GEMM, st);
    s = product_of_codes(xq, sx, bits_x, wq, sw, M, N, K, y, y_dtype, ldy_elems, st);
    stage_end(h);
    return s;
}

int quest_mx_codes_optional(int64_t M, int64_t N, int64_t K) {
    return mx_rows_ok(M) && mx_rows_ok(N) && mx_cols_ok(K) && mx_fuses_quantizer(M, N, K);
}

int quest_linear_fwd_mx(const void *x, int x_dtype, int64_t ldx, const void *w, int w_dtype, int64_t ldw, int64_t M, int64_t N,
                        int64_t K, int bits_x, int had_block, void *y, int y_dtype, int64_t ldy_elems, uint8_t *xq, uint8_t *sx,
                        uint8_t *wq, uint8_t *sw, int w_is_cached, void *stream) {
    int s = check_product(wq, sw, bits_x, M, N, K, y, y_dtype, ldy_elems);
    if (s) return s;
    if (w_is_cached != 0 && w_is_cached != 1) return QUEST_ERR_SHAPE;
    if ((s = check_rows(x, x_dtype, M, K, ldx))) return s;
    if (!w_is_cached && (s = check_rows(w, w_dtype, N, K, ldw))) return s;
    if (!mx_had_ok(had_block)) return QUEST_ERR_HAD_BLOCK;
    // an empty product still quantizes the operand that there is
    const bool keep = M > 0 && (xq || sx), quantize_w = N > 0 && !w_is_cached;
    if (quantize_w && (!wq || !sw)) return QUEST_ERR_NULL;
    if ((keep || (M > 0 && N > 0 && !mx_fuses_quantizer(M, N, K))) && (!xq || !sx)) return QUEST_ERR_NULL;
    if ((keep && (!aligned(xq, 16) || !aligned(sx, 16))) || (quantize_w && !aligned(wq, 16))) return QUEST_ERR_ALIGN;
    if ((M == 0 || N == 0) && !keep && !quantize_w) return QUEST_OK;
    if ((s = check_device())) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    {
        MxJob jobs[2];
        int n = 0;
        if (keep) jobs[n++] = {x, M, ldx, xq, sx, bits_x};
        if (quantize_w) jobs[n++] = {w, N, ldw, wq, sw, 4};
        if (n) {
            void *h = stage_begin(keep ? QUEST_STAGE_QUANT_X : QUEST_STAGE_QUANT_W, st);
            if (n == 2 && x_dtype != w_dtype) {
                s = launch_mx_quantize(&jobs[0], 1, x_dtype, K, had_block, st);
                if (!s) s = launch_mx_quantize(&jobs[1], 1, w_dtype, K, had_block, st);
            } else {
                s = launch_mx_quantize(jobs, n, keep ? x_dtype : w_dtype, K, had_block, st);
            }
            stage_end(h);
            if (s) return s;
        }
    }
    if (M == 0 || N == 0) return QUEST_OK;
    void *h = stage_begin(QUEST_STAGE_GEMM, st);
    if (keep) s = product_of_codes(xq, sx, bits_x, wq, sw, M, N, K, y, y_dtype, ldy_elems, st);
    else s = launch_mx_few_rows(x, x_dtype, ldx, nullptr, nullptr, bits_x, had_block, wq, sw, M, N, K, y, y_dtype, ldy_elems, st);
    stage_end(h);
    return s;
}

}  // extern "C"
