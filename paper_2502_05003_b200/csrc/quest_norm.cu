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

// A chunk is what a thread moves at once: 16 bytes (eight bfloat16 or four binary32), or one element where rows do not start
// on 16-byte boundaries.  It stays in its storage type until it is used: half the registers, twice the loads in flight.
template <bool F32, bool VEC>
struct Chunk {
    static constexpr int V = VEC ? (F32 ? 4 : 8) : 1;
    uint32_t w[VEC ? 4 : 1];
    // volatile: requested where it stands, not where the compiler would use it (a row ahead, behind a barrier).  Not as read-only
    // data: an output may take an input's place
    __device__ __forceinline__ void load(const void *p, long long i) {
        const uint8_t *at = static_cast<const uint8_t *>(p) + i * (F32 ? 4 : 2);
        if constexpr (VEC) {
            asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(at));
        } else if constexpr (F32) {
            asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(at));
        } else {
            uint16_t v;
            asm volatile("ld.global.b16 %0, [%1];" : "=h"(v) : "l"(at));
            w[0] = v;
        }
    }
    __device__ __forceinline__ void store(void *p, long long i) const {
        if constexpr (VEC) *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p) + i * (F32 ? 4 : 2)) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (F32) static_cast<uint32_t *>(p)[i] = w[0];
        else static_cast<uint16_t *>(p)[i] = (uint16_t)w[0];
    }
    __device__ __forceinline__ void get(float *v) const {
        if constexpr (F32) {
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = __uint_as_float(w[k]);
        } else if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[2 * k] = __uint_as_float(w[k] << 16);
                v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
            }
        } else {
            v[0] = __uint_as_float(w[0] << 16);
        }
    }
    __device__ __forceinline__ void set(const float *v) {                 // rounds to the storage type
        if constexpr (F32) {
#pragma unroll
            for (int k = 0; k < V; ++k) w[k] = __float_as_uint(v[k]);
        } else if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
                w[k] = *reinterpret_cast<const uint32_t *>(&h);
            }
        } else {
            const __nv_bfloat16 h = __float2bfloat16_rn(v[0]);
            w[0] = *reinterpret_cast<const uint16_t *>(&h);
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int k = 0; k < (VEC ? 4 : 1); ++k) w[k] = 0u;
    }
};
// V elements (8, 4 or 1) of the other tensors' types.
template <int V>
__device__ __forceinline__ void load_elements(const void *p, long long i, bool f32, float *v) {
    if constexpr (V == 1) {
        if (f32) v[0] = __ldg(static_cast<const float *>(p) + i);
        else v[0] = __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t *>(p) + i) << 16);
    } else if (f32) {
#pragma unroll
        for (int k = 0; k < V; k += 4) {
            const float4 q = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i + k));
            v[k] = q.x; v[k + 1] = q.y; v[k + 2] = q.z; v[k + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; k += 4) {
            const uint2 q = __ldg(reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + i + k));
            v[k] = __uint_as_float(q.x << 16); v[k + 1] = __uint_as_float(q.x & 0xFFFF0000u);
            v[k + 2] = __uint_as_float(q.y << 16); v[k + 3] = __uint_as_float(q.y & 0xFFFF0000u);
        }
    }
}
template <int V>
__device__ __forceinline__ void store_elements(void *p, long long i, bool f32, const float *v) {
    if constexpr (V == 1) {
        if (f32) static_cast<float *>(p)[i] = v[0];
        else static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v[0]);
    } else if (f32) {
#pragma unroll
        for (int k = 0; k < V; k += 4)
            *reinterpret_cast<float4 *>(static_cast<float *>(p) + i + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
    } else {
        uint32_t w[V / 2];
#pragma unroll
        for (int k = 0; k < V / 2; ++k) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
            w[k] = *reinterpret_cast<const uint32_t *>(&h);
        }
        if constexpr (V == 8) *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + i) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p) + i) = make_uint2(w[0], w[1]);
    }
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

// Most threads of a CTA that takes a row: few chunks each, or single elements, up to 1024 of them; many, 512 (their registers).
constexpr int row_threads(int vpt) { return vpt <= 1 ? 256 : vpt <= 4 || vpt == 16 ? 1024 : 512; }

// VPT chunks to a thread; a row belongs to a warp (ROW_WARP, four rows to a CTA) or to the CTA.  MX: 0, or the bits of the
// output: the 32 / V neighbouring lanes that hold a block agree on its scale.  8192 x 2048 with residual: bfloat16 22.1 us (6.1
// TB/s), MX out in 8 or 4 bits 22.9, rotated 27 (there the ALU pipe is busy two thirds of the time); binary32 41.5 (6.5 TB/s), MX out 35, rotated
// 39.  Rows that no 16-byte access divides, an element at a time: 8192 x 2047 52 in both types.
template <bool F32, bool VEC, int VPT, bool ROW_WARP, int MX>
__global__ void __launch_bounds__(ROW_WARP ? 128 : row_threads(VPT))
rmsnorm_kernel(const __grid_constant__ NormArgs a) {
    using C = Chunk<F32, VEC>;
    constexpr int V = C::V, LANES = 32 / V;
    static_assert(MX == 0 || VEC, "MX output: whole chunks");
    __shared__ float part[32];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int threads = ROW_WARP ? 32 : (int)blockDim.x;
    const int tr = ROW_WARP ? lane : (int)threadIdx.x;
    const long long row = ROW_WARP ? blockIdx.x * 4ll + warp : blockIdx.x;
    const bool live = row < a.rows;                  // MX: rows behind the last one only fill up a tile of scales
    if (!MX && !live) return;                        // the whole warp
    const int chunks = live ? a.cols / V : 0;
    C h[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j)
        if (tr + threads * j < chunks) h[j].load(a.x, row * a.ldx + (long long)(tr + threads * j) * V);
    if (a.residual) {
        C r[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j)
            if (tr + threads * j < chunks) r[j].load(a.residual, row * a.ldr + (long long)(tr + threads * j) * V);
#pragma unroll
        for (int j = 0; j < VPT; ++j)
            if (tr + threads * j < chunks) {
                float u[V], v[V];
                h[j].get(u);
                r[j].get(v);
#pragma unroll
                for (int k = 0; k < V; ++k) u[k] += v[k];
                // the stream is stored in its own type; what is normalised (and what a backward pass reads) is that
                h[j].set(u);
                h[j].store(a.h, row * a.cols + (long long)(tr + threads * j) * V);
            }
    }
    float ss = 0.0f;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
        if (tr + threads * j < chunks) {
            float u[V], s = 0.0f;
            h[j].get(u);
#pragma unroll
            for (int k = 0; k < V; ++k) s = __fmaf_rn(u[k], u[k], s);
            ss += s;
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
        const bool in = c < chunks;
        float y[V];
#pragma unroll
        for (int k = 0; k < V; ++k) y[k] = 0.0f;
        if (in) {
            float w[V];
            load_elements<V>(a.weight, (long long)c * V, a.w_f32, w);
            h[j].get(y);
#pragma unroll
            for (int k = 0; k < V; ++k) y[k] = (y[k] * rstd) * w[k];
        }
        if constexpr (MX == 0) {
            if (in) store_elements<V>(a.y, row * a.cols + (long long)c * V, a.y_f32, y);
        } else {
            if (a.rotate) {
                // the wider strides of the block's transform are between lanes, the others inside
#pragma unroll
                for (int o = LANES / 2; o >= 1; o >>= 1)
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const float p = __shfl_xor_sync(0xffffffffu, y[k], o);
                        y[k] = (lane & o) ? __fsub_rn(p, y[k]) : __fadd_rn(y[k], p);
                    }
#pragma unroll
                for (int o = V / 2; o >= 1; o >>= 1)
#pragma unroll
                    for (int k = 0; k < V; ++k)
                        if ((k & o) == 0) {
                            const float p = y[k], q = y[k + o];
                            y[k] = __fadd_rn(p, q);
                            y[k + o] = __fsub_rn(p, q);
                        }
#pragma unroll
                for (int k = 0; k < V; ++k) y[k] = __fmul_rn(y[k], 0.17677669529663687f);
            }
            float m = mx_max_nan(mx_max_nan(y[0], y[1]), mx_max_nan(y[2], y[3]));
            if constexpr (V == 8) m = mx_max_nan(m, mx_max_nan(mx_max_nan(y[4], y[5]), mx_max_nan(y[6], y[7])));
#pragma unroll
            for (int o = 1; o < LANES; o <<= 1) m = mx_max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
            const uint32_t s = in ? mx_scale_byte<MX>(m) : 0u;
            if (in) {
                const float inv = mx_inverse_scale(s);
#pragma unroll
                for (int k = 0; k < V; ++k) y[k] = __fmul_rn(y[k], inv);
                const long long at = row * a.cols + (long long)c * V;
                if constexpr (MX == 4) {
                    float t[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) t[k] = y[k % V];
                    const uint32_t q = s == 255u ? 0u : mx_e2m1x8(t);
                    if constexpr (V == 8) *reinterpret_cast<uint32_t *>(a.yq + at / 2) = q;
                    else *reinterpret_cast<uint16_t *>(a.yq + at / 2) = (uint16_t)q;
                } else {
#pragma unroll
                    for (int k = 0; k < V; k += 4) *reinterpret_cast<uint32_t *>(a.yq + at + k) = s == 255u ? 0u : mx_e4m3x4(y + k);
                }
            }
            const int block = c / LANES;
            if (lane % LANES == 0 && block < 4 * a.tiles) a.sy[mx_scale_at((int)row, block, a.tiles)] = (uint8_t)s;
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

// A CTA takes a row at a time (ROW_WARP: a warp does, four to a CTA), a thread the same VPT chunks of each of them, so that its
// share of dw stays in registers over all of the rows.  AHEAD: the next row is requested before the present one is reduced,
// which keeps loads in flight over the barrier.  Bound by memory; 8192 x 2048 bfloat16 with dres: 24.1 us and 3.1 for the sum of
// dw's parts, 4.9 TB/s together (four rows to a barrier without AHEAD: 32 us; half or all of the chunks in a thread: 28 .. 33).
// The weight stays in registers where the chunks are few.  binary32 46; an element at a time, 8192 x 2047 87 (bfloat16) and 85.
template <bool F32, bool VEC, int VPT, int THREADS, int CTAS, bool AHEAD, bool ROW_WARP>
__global__ void __launch_bounds__(THREADS, CTAS)
rmsnorm_bwd_kernel(const __grid_constant__ NormBwdArgs a) {
    using C = Chunk<F32, VEC>;
    constexpr int V = C::V;
    constexpr bool KEEP_W = VPT <= 2;
    constexpr int WARPS = (THREADS / 32 + 3) / 4 * 4;           // read four at a time
    __shared__ __align__(16) float part[2][WARPS];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int threads = ROW_WARP ? 32 : (int)blockDim.x, tr = ROW_WARP ? lane : (int)threadIdx.x;
    const int chunks = a.cols / V;
    const float inv_cols = __fdiv_rn(1.0f, (float)a.cols);
    if constexpr (!ROW_WARP) {
        for (int i = threadIdx.x; i < 2 * WARPS; i += blockDim.x) (&part[0][0])[i] = 0.0f;      // warps that there are not
        __syncthreads();
    }
    float dw[VPT][V] = {}, wk[KEEP_W ? VPT : 1][V];
    if constexpr (KEEP_W) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = tr + threads * j;
            if (c < chunks) load_elements<V>(a.weight, (long long)c * V, a.w_f32, wk[j]);
        }
    }
    const auto weight = [&](int j, int c, float *w) {
        if constexpr (KEEP_W) {
#pragma unroll
            for (int k = 0; k < V; ++k) w[k] = wk[j][k];
        } else {
            load_elements<V>(a.weight, (long long)c * V, a.w_f32, w);
        }
    };
    struct Row {
        C h[VPT], g[VPT], r[VPT];
        float rstd;
    };
    const auto fetch = [&](Row &t, long long row) {
        const bool in = row < a.rows;
        t.rstd = in ? __ldg(a.rstd + row) : 0.0f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = tr + threads * j;
            t.r[j].clear();
            if (in && c < chunks) {
                t.h[j].load(a.h, row * a.ldh + (long long)c * V);
                t.g[j].load(a.dy, row * a.lddy + (long long)c * V);
                if (a.dres && a.dx) t.r[j].load(a.dres, row * a.lddr + (long long)c * V);
            } else {
                t.h[j].clear();
                t.g[j].clear();
            }
        }
    };
    int turn = 0;
    const int per_cta = ROW_WARP ? THREADS / 32 : 1;
    const long long first = blockIdx.x * (long long)per_cta + (ROW_WARP ? warp : 0), step = gridDim.x * (long long)per_cta;
    Row next;
    if constexpr (AHEAD) fetch(next, first);
    for (long long row = first; row < a.rows; row += step, turn ^= 1) {
        Row now;
        if constexpr (AHEAD) {
            now = next;
            fetch(next, row + step);
        } else {
            fetch(now, row);
        }
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = tr + threads * j;
            if (c < chunks) {
                float n[V], d[V], w[V];
                now.h[j].get(n);
                now.g[j].get(d);
                weight(j, c, w);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    n[k] *= now.rstd;
                    dw[j][k] = __fmaf_rn(d[k], n[k], dw[j][k]);
                    s = __fmaf_rn(d[k] * w[k], n[k], s);
                }
            }
        }
        s = warp_sum(s);
        if constexpr (!ROW_WARP) {
            // the row after the next overwrites these sums, behind the barrier of the next one
            if (lane == 0) part[turn][warp] = s;
            __syncthreads();
            s = 0.0f;
#pragma unroll
            for (int k = 0; k < WARPS; k += 4) {
                const float4 q = *reinterpret_cast<const float4 *>(&part[turn][k]);
                s += (q.x + q.y) + (q.z + q.w);
            }
        }
        if (a.dx) {
            const float mean = s * inv_cols;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int c = tr + threads * j;
                if (c < chunks) {
                    float n[V], d[V], w[V], o[V];
                    now.h[j].get(n);
                    now.g[j].get(d);
                    now.r[j].get(o);
                    weight(j, c, w);
#pragma unroll
                    for (int k = 0; k < V; ++k) o[k] = __fmaf_rn(now.rstd, __fmaf_rn(-(n[k] * now.rstd), mean, d[k] * w[k]), o[k]);
                    C out;
                    out.set(o);
                    out.store(a.dx, row * a.cols + (long long)c * V);
                }
            }
        }
    }
    if (!a.dw_part) return;
    float *dst = a.dw_part + (long long)blockIdx.x * a.cols;
    if constexpr (ROW_WARP) {
        // the warps' shares, added in order
        __shared__ float sum[THREADS / 32][32 * VPT * V];
#pragma unroll
        for (int j = 0; j < VPT; ++j)
#pragma unroll
            for (int k = 0; k < V; ++k) sum[warp][(lane + 32 * j) * V + k] = dw[j][k];
        __syncthreads();
        for (int c = threadIdx.x; c < a.cols; c += THREADS) {
            float v = sum[0][c];
#pragma unroll
            for (int k = 1; k < THREADS / 32; ++k) v += sum[k][c];
            dst[c] = v;
        }
    } else {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = tr + threads * j;
            if (c < chunks) store_elements<V>(dst, (long long)c * V, true, dw[j]);
        }
    }
}

// dw[c] = sum of `parts` rows of binary32 in a fixed order: 16 columns to a CTA, SLOTS groups of 16 threads take the parts in turn.
template <int SLOTS>
__global__ void __launch_bounds__(16 * SLOTS)
column_sum_kernel(const float *__restrict__ in, int parts, int cols, float *__restrict__ out) {
    __shared__ float s[16][SLOTS + 1];
    pdl_launch_dependents();
    pdl_wait();
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), slot = threadIdx.x >> 4;
    float v = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (int p = slot; p < parts; p += SLOTS) v += __ldg(in + (long long)p * cols + c);
    }
    s[threadIdx.x & 15][slot] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    for (int i = threadIdx.x >> 5; i < 16; i += SLOTS / 2) {
        v = 0.0f;
#pragma unroll
        for (int k = 0; k < (SLOTS + 31) / 32; ++k)
            if (lane + 32 * k < SLOTS) v += s[i][lane + 32 * k];
        v = warp_sum(v);
        if (lane == 0 && blockIdx.x * 16 + i < cols) out[blockIdx.x * 16 + i] = v;
    }
}

bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
bool pitch_ok(int64_t rows, int64_t bytes) { return rows == 1 || bytes % 16 == 0; }       // a lone row has no next one
bool shape_ok(int64_t rows, int64_t cols) { return mx_rows_ok(rows) && cols >= 1 && cols <= 16384; }

// Most CTAs of the backward kernel, hence rows of partial sums.
int64_t most_parts(int64_t cols) { return cols <= 512 ? 1024 : 512; }

template <bool F32, bool VEC, int VPT, int THREADS, int CTAS, bool AHEAD, bool ROW_WARP = false>
cudaError_t launch_bwd(const NormBwdArgs &a, int &parts, cudaStream_t st) {
    const int chunks = a.cols / Chunk<F32, VEC>::V;
    const int threads = ROW_WARP ? THREADS : std::min(THREADS, ((chunks + VPT - 1) / VPT + 31) / 32 * 32);
    // as many CTAs as the chip holds at once: with fewer threads each, more of them
    const int64_t room = std::min<int64_t>((int64_t)num_sms() * std::min(32, CTAS * THREADS / threads), most_parts(a.cols));
    const int64_t rows = ROW_WARP ? THREADS / 32 : 1;
    parts = (int)std::min<int64_t>((a.rows + rows - 1) / rows, room);
    return launch_pdl(rmsnorm_bwd_kernel<F32, VEC, VPT, THREADS, CTAS, AHEAD, ROW_WARP>, dim3((unsigned)parts), dim3((unsigned)threads), 0, st, 1, a);
}
// Threads to a row and chunks to a thread, measured over bfloat16 and binary32 rows of 512 to 5504 (see the kernel).
template <bool F32>
cudaError_t launch_bwd_type(const NormBwdArgs &a, bool vec, int &parts, cudaStream_t st) {
    if (vec) {
        const int chunks = a.cols / Chunk<F32, true>::V;
        // short rows, many of them: a warp each (16384 x 512 bfloat16 16 us, a CTA each 22)
        if (chunks <= 64 && a.rows >= 1024)
            return chunks <= 32 ? launch_bwd<F32, true, 1, 128, 4, true, true>(a, parts, st) : launch_bwd<F32, true, 2, 128, 4, true, true>(a, parts, st);
        if constexpr (F32) {                     // rows of up to 16384 columns: bfloat16 has at most 2048 chunks
            if (chunks > 2048) return launch_bwd<F32, true, 8, 512, 1, false>(a, parts, st);
        }
        return chunks <= 256 ? launch_bwd<F32, true, 2, 128, 4, true>(a, parts, st) : chunks <= 512 ? launch_bwd<F32, true, 2, 256, 2, true>(a, parts, st)
             : chunks <= 1024 ? launch_bwd<F32, true, 2, 512, 1, true>(a, parts, st) : chunks <= 1536 ? launch_bwd<F32, true, 3, 512, 1, true>(a, parts, st)
             : launch_bwd<F32, true, 4, 512, 1, false>(a, parts, st);
    }
    return a.cols <= 1024 ? launch_bwd<F32, false, 4, 256, 2, true>(a, parts, st) : a.cols <= 4096 ? launch_bwd<F32, false, 4, 1024, 1, true>(a, parts, st)
         : a.cols <= 8192 ? launch_bwd<F32, false, 8, 1024, 1, false>(a, parts, st) : launch_bwd<F32, false, 16, 1024, 1, false>(a, parts, st);
}

template <bool F32, bool VEC, int VPT, int MX>
cudaError_t launch_row_cta(const NormArgs &a, int64_t rows, int chunks, cudaStream_t st) {
    const int threads = std::min(row_threads(VPT), ((chunks + VPT - 1) / VPT + 31) / 32 * 32);
    return launch_pdl(rmsnorm_kernel<F32, VEC, VPT, false, MX>, dim3((unsigned)rows), dim3((unsigned)threads), 0, st, 1, a);
}
template <bool F32, bool VEC, int VPT, int MX>
cudaError_t launch_row_warp(const NormArgs &a, int64_t rows, cudaStream_t st) {
    return launch_pdl(rmsnorm_kernel<F32, VEC, VPT, true, MX>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, 1, a);
}
template <bool F32, int MX>
cudaError_t launch_fwd(const NormArgs &a, bool vec, cudaStream_t st) {
    const int64_t rows = MX ? (a.rows + 127) / 128 * 128 : a.rows;
    if constexpr (MX == 0) {
        if (!vec) {
            return a.cols <= 4096 ? launch_row_cta<F32, false, 4, 0>(a, rows, a.cols, st) : launch_row_cta<F32, false, 16, 0>(a, rows, a.cols, st);
        }
    }
    constexpr int V = Chunk<F32, true>::V;
    const int chunks = MX ? a.tiles * (128 / V) : a.cols / V;      // MX: whole tiles of scales
    // short rows, many of them: a warp each (16384 x 512 bfloat16 12.4 us, a CTA each 18).  Longer ones: two chunks to a thread
    // (8192 x 2048: 22.3 us; one chunk 23.2, four 23.1, a warp to a row 24.7), one where the rows do not fill the chip anyway
    if (chunks <= 128 && a.rows >= 2048)
        return chunks <= 32 ? launch_row_warp<F32, true, 1, MX>(a, rows, st) : chunks <= 64 ? launch_row_warp<F32, true, 2, MX>(a, rows, st)
                                                                                            : launch_row_warp<F32, true, 4, MX>(a, rows, st);
    if (chunks <= 256 && a.rows <= 2 * num_sms()) return launch_row_cta<F32, true, 1, MX>(a, rows, chunks, st);
    if constexpr (F32) {                         // (bfloat16: at most 2048 chunks)
        if (chunks > 2048) return launch_row_cta<F32, true, 8, MX>(a, rows, chunks, st);
    }
    return chunks <= 512 ? launch_row_cta<F32, true, 2, MX>(a, rows, chunks, st) : launch_row_cta<F32, true, 4, MX>(a, rows, chunks, st);
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
    const bool vec = cols % 8 == 0 && aligned(x, 16) && pitch_ok(rows, ldx * es) && aligned(weight, 16) &&
                     (!residual || (aligned(residual, 16) && pitch_ok(rows, ldr * es) && aligned(h, 16))) && (mx_bits ? aligned(yq, 16) : aligned(y, 16));
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
    return align_up((size_t)std::max<int64_t>(std::min(rows, most_parts(cols)), 1) * (size_t)cols * 4, 256);
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
                         pitch_ok(rows, lddy * es) && pitch_ok(rows, ldh * es) && (!dres || pitch_ok(rows, lddr * es));
        e = dtype == QUEST_F32 ? launch_bwd_type<true>(a, vec, parts, st) : launch_bwd_type<false>(a, vec, parts, st);
        if (e != cudaSuccess) return cuda_fail(e);
    }
    if (dw) {
        const auto sum = [&](auto kernel, int slots) {
            return launch_pdl(kernel, dim3((unsigned)((cols + 15) / 16)), dim3((unsigned)(16 * slots)), 0, st, 1, static_cast<const float *>(workspace),
                              parts, (int)cols, dw);
        };
        e = parts <= 256 ? sum(column_sum_kernel<32>, 32) : sum(column_sum_kernel<64>, 64);
        if (e != cudaSuccess) return cuda_fail(e);
    }
    return QUEST_OK;
}

}  // extern "C"
