// Root-mean-square norm with the residual stream's addition, forward and backward.  All three kernels are bound by memory: a row
// is read once, stays in registers over its reduction, and every output is written once.
//
//   forward    h = x + residual;  rstd = (mean h^2 + eps)^(-1/2);  y = (h rstd) w, as it is or as MX codes and scales
//   backward   n = h rstd, g = dy w;  dx = dres + rstd (g - n mean(g n));  dw = sum over rows of dy n
#include <math.h>

#include <algorithm>

#include "quest_mx.cuh"

namespace quest {
namespace {

__device__ __forceinline__ float element(const void *p, long long i, bool f32) {
    if (f32) return __ldg(static_cast<const float *>(p) + i);
    return __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t *>(p) + i) << 16);
}
// V consecutive elements: eight from a 16-byte boundary, or one.
template <bool F32, int V>
__device__ __forceinline__ void load_chunk(const void *p, long long i, float *v) {
    if constexpr (V == 1) {
        v[0] = element(p, i, F32);
    } else if constexpr (F32) {
        const float4 *q = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i);
        const float4 a = __ldg(q), b = __ldg(q + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 q = __ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + i));
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(w[k] << 16);
            v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
    }
}
template <bool F32, int V>
__device__ __forceinline__ void store_chunk(void *p, long long i, const float *v) {
    if constexpr (F32) {
        float *o = static_cast<float *>(p) + i;
        if constexpr (V == 1) {
            o[0] = v[0];
        } else {
            reinterpret_cast<float4 *>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
        __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(p) + i;
        if constexpr (V == 1) {
            o[0] = __float2bfloat16_rn(v[0]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
                w[k] = *reinterpret_cast<const uint32_t *>(&b);
            }
            *reinterpret_cast<uint4 *>(o) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}
template <int V>
__device__ __forceinline__ void load_weight(const void *p, long long i, bool f32, float *v) {
    if (f32) load_chunk<true, V>(p, i, v);
    else load_chunk<false, V>(p, i, v);
}
__device__ __forceinline__ float warp_sum(float s) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

struct NormArgs {
    const void *x, *residual, *weight;
    long long ldx, ldr;
    long long rows;
    int cols, w_f32, y_f32;
    float eps;
    void *h, *y;
    float *rstd;
    uint8_t *yq, *sy;
    int tiles, rotate;
};

// V elements to an access, VPT accesses to a thread; a row belongs to a warp (ROW_WARP, four rows to a CTA) or to the CTA.
// MX: 0, or the bits of the output: four neighbouring lanes hold a block of 32.
template <bool F32, int V, int VPT, bool ROW_WARP, int MX>
__global__ void __launch_bounds__(ROW_WARP ? 128 : 256)
rmsnorm_kernel(const __grid_constant__ NormArgs a) {
    static_assert(MX == 0 || V == 8, "MX output: eight elements to a lane");
    __shared__ float part[8];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int threads = ROW_WARP ? 32 : (int)blockDim.x;
    const int tr = ROW_WARP ? lane : (int)threadIdx.x;
    const long long row = ROW_WARP ? blockIdx.x * 4ll + warp : blockIdx.x;
    const bool live = row < a.rows;                  // MX: rows behind the last one only fill up a tile of scales
    if (!MX && !live) return;                        // the whole warp
    const int chunks = a.cols / V;
    float h[VPT][V];
    float ss = 0.0f;
    if (live) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = tr + threads * j;
            if (c < chunks) load_chunk<F32, V>(a.x, row * a.ldx + (long long)c * V, h[j]);
        }
        if (a.residual) {
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = tr + threads * j;
                if (c < chunks) {
                    float r[V];
                    load_chunk<F32, V>(a.residual, row * a.ldr + (long long)c * V, r);
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        h[j][k] += r[k];
                        // the stream is stored in its own type; what is normalised (and what a backward pass reads) is that
                        if (!F32) h[j][k] = __bfloat162float(__float2bfloat16_rn(h[j][k]));
                    }
                    store_chunk<F32, V>(a.h, row * a.cols + (long long)c * V, h[j]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < VPT; ++j)
            if (tr + threads * j < chunks) {
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < V; ++k) s = __fmaf_rn(h[j][k], h[j][k], s);
                ss += s;
            }
    }
    ss = warp_sum(ss);
    if constexpr (!ROW_WARP) {
        if (lane == 0) part[warp] = ss;
        __syncthreads();
        ss = 0.0f;
        for (int k = 0; k < (int)blockDim.x / 32; ++k) ss += part[k];
    }
    const float rstd = __frsqrt_rn(__fdiv_rn(ss, (float)a.cols) + a.eps);
    if (live && tr == 0 && a.rstd) a.rstd[row] = rstd;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = tr + threads * j;
        const bool in = live && c < chunks;
        float y[V];
#pragma unroll
        for (int k = 0; k < V; ++k) y[k] = 0.0f;
        if (in) {
            float w[V];
            load_weight<V>(a.weight, (long long)c * V, a.w_f32, w);
#pragma unroll
            for (int k = 0; k < V; ++k) y[k] = (h[j][k] * rstd) * w[k];
        }
        if constexpr (MX == 0) {
            if (in) {
                if (a.y_f32) store_chunk<true, V>(a.y, row * a.cols + (long long)c * V, y);
                else store_chunk<false, V>(a.y, row * a.cols + (long long)c * V, y);
            }
        } else {
            if (a.rotate) {
                // strides 16 and 8 of the block's transform are between lanes, 4, 2 and 1 inside
#pragma unroll
                for (int o = 2; o >= 1; o >>= 1)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float p = __shfl_xor_sync(0xffffffffu, y[k], o);
                        y[k] = (lane & o) ? __fsub_rn(p, y[k]) : __fadd_rn(y[k], p);
                    }
#pragma unroll
                for (int o = 4; o >= 1; o >>= 1)
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if ((k & o) == 0) {
                            const float p = y[k], q = y[k + o];
                            y[k] = __fadd_rn(p, q);
                            y[k + o] = __fsub_rn(p, q);
                        }
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = __fmul_rn(y[k], 0.17677669529663687f);
            }
            float m = mx_max_nan(mx_max_nan(mx_max_nan(y[0], y[1]), mx_max_nan(y[2], y[3])),
                                 mx_max_nan(mx_max_nan(y[4], y[5]), mx_max_nan(y[6], y[7])));
            m = mx_max_nan(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = mx_max_nan(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const uint32_t s = in ? mx_scale_byte<MX>(m) : 0u;
            if (in) {
                const float inv = mx_inverse_scale(s);
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = __fmul_rn(y[k], inv);
                const long long at = row * a.cols + (long long)c * 8;
                if constexpr (MX == 4) {
                    *reinterpret_cast<uint32_t *>(a.yq + at / 2) = s == 255u ? 0u : mx_e2m1x8(y);
                } else {
                    const uint2 q = make_uint2(mx_e4m3x4(y), mx_e4m3x4(y + 4));
                    *reinterpret_cast<uint2 *>(a.yq + at) = s == 255u ? make_uint2(0u, 0u) : q;
                }
            }
            if ((lane & 3) == 0 && c < 16 * a.tiles) a.sy[mx_scale_at(row, c >> 2, a.tiles)] = (uint8_t)s;
        }
    }
}

struct NormBwdArgs {
    const void *dy, *h, *dres, *weight;
    const float *rstd;
    long long lddy, ldh, lddr, rows;
    int cols, w_f32;
    void *dx;
    float *dw_part;                 // [gridDim.x x cols], or NULL
};

// A CTA takes RB rows at a time, a thread the same VPT chunks of each of them, so that its share of dw stays in registers over
// all of the CTA's rows; RB rows share one barrier and their loads are in flight together.
template <bool F32, int V, int VPT, int RB>
__global__ void __launch_bounds__(512)
rmsnorm_bwd_kernel(const __grid_constant__ NormBwdArgs a) {
    __shared__ float part[2][RB][16];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int chunks = a.cols / V;
    float w[VPT][V], dw[VPT][V] = {};
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = threadIdx.x + blockDim.x * j;
        if (c < chunks) load_weight<V>(a.weight, (long long)c * V, a.w_f32, w[j]);
    }
    int turn = 0;
    for (long long row0 = blockIdx.x * (long long)RB; row0 < a.rows; row0 += gridDim.x * (long long)RB, turn ^= 1) {
        float n[RB][VPT][V], g[RB][VPT][V], rstd[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            rstd[b] = row0 + b < a.rows ? __ldg(a.rstd + row0 + b) : 0.0f;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = threadIdx.x + blockDim.x * j;
                if (c < chunks && row0 + b < a.rows) {
                    load_chunk<F32, V>(a.h, (row0 + b) * a.ldh + (long long)c * V, n[b][j]);
                    load_chunk<F32, V>(a.dy, (row0 + b) * a.lddy + (long long)c * V, g[b][j]);
                } else {
#pragma unroll
                    for (int k = 0; k < V; ++k) n[b][j][k] = g[b][j][k] = 0.0f;
                }
            }
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < VPT; ++j)
                if ((int)(threadIdx.x + blockDim.x * j) < chunks) {
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        n[b][j][k] *= rstd[b];
                        dw[j][k] = __fmaf_rn(g[b][j][k], n[b][j][k], dw[j][k]);
                        g[b][j][k] *= w[j][k];
                        s = __fmaf_rn(g[b][j][k], n[b][j][k], s);
                    }
                }
            s = warp_sum(s);
            if (lane == 0) part[turn][b][warp] = s;
        }
        __syncthreads();
        if (a.dx) {
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                if (row0 + b >= a.rows) break;
                float s = 0.0f;
                for (int k = 0; k < warps; ++k) s += part[turn][b][k];
                const float mean = __fdiv_rn(s, (float)a.cols);
#pragma unroll
                for (int j = 0; j < VPT; ++j) {
                    const int c = threadIdx.x + blockDim.x * j;
                    if (c < chunks) {
                        float o[V];
#pragma unroll
                        for (int k = 0; k < V; ++k) o[k] = rstd[b] * __fmaf_rn(-n[b][j][k], mean, g[b][j][k]);
                        if (a.dres) {
                            float r[V];
                            load_chunk<F32, V>(a.dres, (row0 + b) * a.lddr + (long long)c * V, r);
#pragma unroll
                            for (int k = 0; k < V; ++k) o[k] += r[k];
                        }
                        store_chunk<F32, V>(a.dx, (row0 + b) * a.cols + (long long)c * V, o);
                    }
                }
            }
        }
    }
    if (a.dw_part) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = threadIdx.x + blockDim.x * j;
            if (c < chunks) store_chunk<true, V>(a.dw_part, (long long)blockIdx.x * a.cols + (long long)c * V, dw[j]);
        }
    }
}

// dw[c] = sum of `parts` rows of binary32 in a fixed order: 32 columns to a CTA, its warps take the parts in turn.
__global__ void __launch_bounds__(1024)
column_sum_kernel(const float *__restrict__ in, int parts, int cols, float *__restrict__ out) {
    __shared__ float s[32][33];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (int p = warp; p < parts; p += 32) v += __ldg(in + (long long)p * cols + c);
    }
    s[warp][lane] = v;
    __syncthreads();
    v = warp_sum(s[lane][warp]);
    const int o = blockIdx.x * 32 + warp;
    if (lane == 0 && o < cols) out[o] = v;
}

bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool shape_ok(int64_t rows, int64_t cols) { return mx_rows_ok(rows) && cols >= 1 && cols <= 16384; }

// Most CTAs of the backward kernel, hence rows of partial sums.
constexpr int64_t MAX_PARTS = 512;
int64_t bwd_parts(int64_t rows) { return std::min(rows, MAX_PARTS); }

template <bool F32, int V, int VPT, int RB>
cudaError_t launch_bwd(const NormBwdArgs &a, int &parts, cudaStream_t st) {
    const int chunks = a.cols / V;
    const int threads = std::min(512, ((chunks + VPT - 1) / VPT + 31) / 32 * 32);
    // CTAs that the chip holds at once, by threads (1024 to an SM keep enough loads in flight)
    const int64_t room = std::min<int64_t>((int64_t)num_sms() * std::max(1, 1024 / threads), MAX_PARTS);
    parts = (int)std::min<int64_t>((a.rows + RB - 1) / RB, room);
    return launch_pdl(rmsnorm_bwd_kernel<F32, V, VPT, RB>, dim3((unsigned)parts), dim3((unsigned)threads), 0, st, 1, a);
}
template <bool F32>
cudaError_t launch_bwd_type(const NormBwdArgs &a, bool vec, int &parts, cudaStream_t st) {
    if (vec) {
        const int chunks = a.cols / 8;
        return chunks <= 512 ? launch_bwd<F32, 8, 1, 4>(a, parts, st) : chunks <= 1024 ? launch_bwd<F32, 8, 2, 2>(a, parts, st)
                                                                                       : launch_bwd<F32, 8, 4, 1>(a, parts, st);
    }
    return a.cols <= 2048 ? launch_bwd<F32, 1, 4, 4>(a, parts, st) : a.cols <= 8192 ? launch_bwd<F32, 1, 16, 1>(a, parts, st)
                                                                                    : launch_bwd<F32, 1, 32, 1>(a, parts, st);
}

template <bool F32, int V, int VPT, int MX>
cudaError_t launch_row_cta(const NormArgs &a, int64_t rows, cudaStream_t st) {
    const int chunks = MX ? 16 * a.tiles : (a.cols + V - 1) / V;
    const int threads = std::min(256, ((chunks + VPT - 1) / VPT + 31) / 32 * 32);
    return launch_pdl(rmsnorm_kernel<F32, V, VPT, false, MX>, dim3((unsigned)rows), dim3((unsigned)threads), 0, st, 1, a);
}
template <bool F32, int V, int VPT, int MX>
cudaError_t launch_row_warp(const NormArgs &a, int64_t rows, cudaStream_t st) {
    return launch_pdl(rmsnorm_kernel<F32, V, VPT, true, MX>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, 1, a);
}
template <bool F32, int MX>
cudaError_t launch_fwd(const NormArgs &a, bool vec, cudaStream_t st) {
    const int64_t rows = MX ? (a.rows + 127) / 128 * 128 : a.rows;
    if constexpr (MX == 0) {
        if (!vec) {
            if (a.cols <= 1024) return launch_row_cta<F32, 1, 4, 0>(a, rows, st);
            if (a.cols <= 4096) return launch_row_cta<F32, 1, 16, 0>(a, rows, st);
            return launch_row_cta<F32, 1, 64, 0>(a, rows, st);
        }
    }
    const int chunks = MX ? 16 * a.tiles : a.cols / 8;
    if (chunks <= 256 && a.rows >= 2048)
        return chunks <= 64 ? launch_row_warp<F32, 8, 2, MX>(a, rows, st) : chunks <= 128 ? launch_row_warp<F32, 8, 4, MX>(a, rows, st)
                                                                                          : launch_row_warp<F32, 8, 8, MX>(a, rows, st);
    return chunks <= 256 ? launch_row_cta<F32, 8, 1, MX>(a, rows, st) : chunks <= 512 ? launch_row_cta<F32, 8, 2, MX>(a, rows, st)
         : chunks <= 1024 ? launch_row_cta<F32, 8, 4, MX>(a, rows, st) : launch_row_cta<F32, 8, 8, MX>(a, rows, st);
}

}  // namespace
}  // namespace quest

using namespace quest;

extern "C" {

int quest_rmsnorm_fwd(const void *x, const void *residual, int dtype, int64_t ldx, int64_t ldr, const void *weight, int w_dtype,
                      int64_t rows, int64_t cols, float eps, void *h, float *rstd, void *y, int y_dtype, int mx_bits, int had_block,
                      uint8_t *yq, uint8_t *sy, void *stream) {
    if ((dtype != QUEST_F32 && dtype != QUEST_BF16) || (w_dtype != QUEST_F32 && w_dtype != QUEST_BF16)) return QUEST_ERR_DTYPE;
    if (mx_bits != 0 && !mx_bits_ok(mx_bits)) return QUEST_ERR_BITS;
    if (!mx_bits && y_dtype != QUEST_F32 && y_dtype != QUEST_BF16) return QUEST_ERR_DTYPE;
    if (!shape_ok(rows, cols) || (mx_bits && !mx_cols_ok(cols)) || ldx < cols || (residual && ldr < cols)) return QUEST_ERR_SHAPE;
    if (mx_bits && !mx_had_ok(had_block)) return QUEST_ERR_HAD_BLOCK;
    if (!(eps >= 0.0f) || isinf(eps)) return QUEST_ERR_EPS;
    if (rows == 0) return QUEST_OK;
    if (!x || !weight || (residual && !h) || (mx_bits ? !yq || !sy : !y)) return QUEST_ERR_NULL;
    const size_t es = dtype == QUEST_F32 ? 4 : 2, ws = w_dtype == QUEST_F32 ? 4 : 2, ys = y_dtype == QUEST_F32 ? 4 : 2;
    if (!aligned(x, es) || !aligned(weight, ws) || (residual && (!aligned(residual, es) || !aligned(h, es))) || (rstd && !aligned(rstd, 4)) ||
        (!mx_bits && !aligned(y, ys)))
        return QUEST_ERR_ALIGN;
    const bool vec = cols % 8 == 0 && aligned(x, 16) && ldx * es % 16 == 0 && aligned(weight, 16) &&
                     (!residual || (aligned(residual, 16) && ldr * es % 16 == 0 && aligned(h, 16))) && (mx_bits ? aligned(yq, 16) : aligned(y, 16));
    if (mx_bits && !vec) return QUEST_ERR_ALIGN;
    const int s = check_device();
    if (s) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const NormArgs a = {x, residual, weight, (long long)ldx, (long long)ldr, (long long)rows, (int)cols, w_dtype == QUEST_F32,
                        y_dtype == QUEST_F32, eps, h, y, rstd, yq, sy, (int)((cols + 127) / 128), had_block == 32};
    const cudaError_t e = dtype == QUEST_F32
                              ? (mx_bits == 4 ? launch_fwd<true, 4>(a, vec, st) : mx_bits == 8 ? launch_fwd<true, 8>(a, vec, st) : launch_fwd<true, 0>(a, vec, st))
                              : (mx_bits == 4 ? launch_fwd<false, 4>(a, vec, st) : mx_bits == 8 ? launch_fwd<false, 8>(a, vec, st) : launch_fwd<false, 0>(a, vec, st));
    return e == cudaSuccess ? QUEST_OK : cuda_fail(e);
}

size_t quest_rmsnorm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
    if (!shape_ok(rows, cols)) return 0;
    return align_up((size_t)std::max<int64_t>(bwd_parts(rows), 1) * (size_t)cols * 4, 256);
}

int quest_rmsnorm_bwd(const void *dy, const void *h, const void *dres, int dtype, int64_t lddy, int64_t ldh, int64_t lddr,
                      const void *weight, int w_dtype, const float *rstd, int64_t rows, int64_t cols, void *dx, float *dw,
                      void *workspace, size_t workspace_bytes, void *stream) {
    if ((dtype != QUEST_F32 && dtype != QUEST_BF16) || (w_dtype != QUEST_F32 && w_dtype != QUEST_BF16)) return QUEST_ERR_DTYPE;
    if (!shape_ok(rows, cols) || lddy < cols || ldh < cols || (dres && lddr < cols)) return QUEST_ERR_SHAPE;
    if (!dx && !dw) return QUEST_ERR_NULL;
    const size_t es = dtype == QUEST_F32 ? 4 : 2, ws = w_dtype == QUEST_F32 ? 4 : 2;
    if (rows != 0 && (!dy || !h || !weight || !rstd)) return QUEST_ERR_NULL;
    if (!aligned(dy, es) || !aligned(h, es) || !aligned(dres, es) || !aligned(weight, ws) || !aligned(rstd, 4) || !aligned(dx, es) ||
        !aligned(dw, 4))
        return QUEST_ERR_ALIGN;
    if (dw && (!workspace || !aligned(workspace, 256) || workspace_bytes < quest_rmsnorm_bwd_workspace_bytes(rows, cols)))
        return QUEST_ERR_WORKSPACE;
    const int s = check_device();
    if (s) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    int parts = 0;
    cudaError_t e;
    if (rows != 0) {
        const NormBwdArgs a = {dy, h, dres, weight, rstd, (long long)lddy, (long long)ldh, (long long)lddr, (long long)rows, (int)cols,
                               w_dtype == QUEST_F32, dx, dw ? static_cast<float *>(workspace) : nullptr};
        const bool vec = cols % 8 == 0 && aligned(dy, 16) && aligned(h, 16) && aligned(dres, 16) && aligned(dx, 16) && aligned(weight, 16) &&
                         lddy * es % 16 == 0 && ldh * es % 16 == 0 && (!dres || lddr * es % 16 == 0);
        e = dtype == QUEST_F32 ? launch_bwd_type<true>(a, vec, parts, st) : launch_bwd_type<false>(a, vec, parts, st);
        if (e != cudaSuccess) return cuda_fail(e);
    }
    if (dw) {
        e = launch_pdl(column_sum_kernel, dim3((unsigned)((cols + 31) / 32)), dim3(1024), 0, st, 1, static_cast<const float *>(workspace), parts,
                       (int)cols, dw);
        if (e != cudaSuccess) return cuda_fail(e);
    }
    return QUEST_OK;
}

}  // extern "C"
