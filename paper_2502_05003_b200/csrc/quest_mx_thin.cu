// Product of two microscaled tensors for few rows of x and many of w, on the tensor cores:
//
//   y[m][n] = sum over blocks of 32 of 2^(sx + sw - 254) sum_k qx[m][k] qw[n][k]     binary32 accumulators
//
// The sides trade places: 128 rows of w fill the tensor cores' long side, x is a tile of BN columns.  Bound by reading w, so every SM has
// to take part: where the tiles leave SMs idle, clusters of up to eight CTAs share the k-blocks of one.  Each leaves the sums of its
// part in its shared memory and owns a share of the rows of x, for which it reads all parts and adds them in their order: no
// atomics, the same result every time.
//   warp 0      copies, 128 bytes of K a stage (256 elements of E2M1 against E2M1, 128 otherwise)
//   warp 1      scales to tensor memory, then up to four MMAs a stage
//   warps 2..9  epilogue: lanes hold neighbouring columns of y, so that its rows are written in whole lines
// Every wait is bounded.
//
// Back to back, weights out of L2, codes of x given: 24 x 5504 x 2048 5.7 us in 8 bits and 4.4 in 4 (floor 0.9), 24 x 32000 x 4096 16.3
// and 14.6 (floor 10.5), 64 x 4096 x 4096 7.2 and 6.4, 128 x 2048 x 5504 7.8 and 6.9.  Small ones are one latency after another (launch, first
// copies, last products, sums of the parts, stores), with DRAM at 7 % (24 x 5504 x 2048).  Above that an SM takes in 54 bytes of
// operands a cycle (0.17 us a stage of 17 KB with all products left out), spread nibbles counted as bytes: that is why 8-bit x, which
// needs w spread, takes longer than 4-bit x.  Of a launch after the quantizer of x, fetching the first five k-blocks into L2 ahead saves
// 0.3 us; sixteen cost the largest 10 %.  Tried: sums of the parts written to their owners (24 x 5504 x 2048 in thirds 7.1 us with remote
// stores, 7.8 with bulk copies, 5.9 with remote reads); pairs of CTAs on 256 rows of w, unsplit (6.3); w fetched ahead by rows (no gain).
#include <algorithm>

#include "quest_mx_tcgen05.cuh"

namespace quest {
namespace {

constexpr int BM = 128;
constexpr int BK = 128;                          // bytes of a stage's rows in shared memory
constexpr int EPI_WARPS = 8;
constexpr int NUM_THREADS = 64 + 32 * EPI_WARPS;
constexpr int MAX_STAGES = 10;
constexpr int MAX_SPLITS = 8;
constexpr int SMEM_OPTIN_MAX = 232448;
constexpr int PREFETCH = 5;                      // k-blocks on their way before x is there

struct ThinArgs {
    int rows_w, rows_x, K;
    void *y;
    int y_f32;
    long long ldy;
    int *status;
};

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *tm, int c0, int c1, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(tm)), "r"(bar), "r"(c0), "r"(c1)
                 : "memory");
}
__device__ __forceinline__ void tma_prefetch_2d(const CUtensorMap *tm, int c0, int c1) {
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(tm)), "r"(c0), "r"(c1)
                 : "memory");
}
template <int XB>
__device__ __forceinline__ void umma_mx(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate,
                                        uint32_t sfa_tmem, uint32_t sfb_tmem) {
    if constexpr (XB == 4)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(sfa_tmem), "r"(sfb_tmem)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(sfa_tmem), "r"(sfb_tmem)
            : "memory");
}
__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ float4 load_from_cta(uint32_t addr, int rank) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(mapa_shared(addr, (uint32_t)rank))
                 : "memory");
    return v;
}
__device__ __forceinline__ void umma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Shared memory from a 1024-byte-aligned base: barriers, then the ring, whose place the partial sums of a split
// product take when its last stage has been read.
template <int BN, int XB>
struct Thin {
    static constexpr int GROUPS = XB == 4 ? 2 : 1;                   // scale tiles (four blocks) of a row in a stage
    static constexpr int A_BYTES = BM * BK, B_BYTES = BN * BK, SF_BYTES = GROUPS * 512;
    // bytes that arrive: nibbles that are spread in shared memory count as the bytes they were
    static constexpr int LOAD_BYTES = (XB == 4 ? A_BYTES : A_BYTES / 2) + B_BYTES + 2 * SF_BYTES;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + 1024 * ((2 * SF_BYTES + 1023) / 1024);
    static constexpr int RING_OFFSET = 1024;
    static_assert(BN * BM * 4 <= 2 * STAGE_BYTES, "partial sums");
    // tensor memory: the accumulators, then the scales of a few stages in turn
    static constexpr int SF_SLOT = 8 * GROUPS, SF_SLOTS = 4;
    static constexpr int TMEM_COLS = BN <= 64 ? 128 : 256;
    static_assert(BN + SF_SLOTS * SF_SLOT <= TMEM_COLS, "tensor memory");
};

// 16 columns of this warp's 32 lanes of tensor memory, as tmem_ld32_issue.
__device__ __forceinline__ void tmem_ld16_issue(uint32_t taddr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}

template <int BN, int XB>
__global__ void __launch_bounds__(NUM_THREADS, 1)
mx_thin_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmSW,
               const __grid_constant__ CUtensorMap tmSX, int splits, int stages, ThinArgs p) {
    using L = Thin<BN, XB>;
    constexpr int KB = XB == 4 ? 256 : 128;      // elements of K per stage
    constexpr int KI = KB / 4;                   // and per instruction
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem);
    uint64_t *full_bar = bars, *empty_bar = bars + MAX_STAGES, *tfull_bar = bars + 2 * MAX_STAGES;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * MAX_STAGES + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    uint8_t *ring = smem + L::RING_OFFSET;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int split = splits == 1 ? 0 : (int)cluster_ctarank();
    const int tiles_w = (p.rows_w + BM - 1) / BM, unit = (int)blockIdx.x / splits;
    const int tile = unit % tiles_w, n0 = tile * BM;                 // rows of w
    const int m0 = unit / tiles_w * BN, live = min(p.rows_x - m0, BN);             // rows of x
    const int num_kb = (p.K + KB - 1) / KB;
    const int kb0 = (int)((long long)num_kb * split / splits), kb1 = (int)((long long)num_kb * (split + 1) / splits);
    pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), 1);
        }
        mbar_init(smem_u32(tfull_bar), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmX)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmSW)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmSX)) : "memory");
        // w on its way into L2 while the kernel before this one still writes x; a line that it changes is changed there
        for (int kb = kb0; kb < kb1 && kb < kb0 + PREFETCH; ++kb) tma_prefetch_2d(&tmW, kb * BK, n0);
    }
    __syncwarp();
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(L::TMEM_COLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();

    if (warp == 0) {
        if (elect_one()) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int kb = kb0; kb < kb1; ++kb) {
                ok = mbar_wait(smem_u32(&empty_bar[stage]), phase ^ 1u, abort_flag, p.status, ST_PRODUCER);
                if (!ok) break;
                const uint32_t fb = smem_u32(&full_bar[stage]), sa = smem_u32(ring + stage * L::STAGE_BYTES);
                mbar_expect_tx(fb, L::LOAD_BYTES);
                // packed rows of w: bytes; spread to bytes: elements.  Both 128 a stage
                tma_load_2d(sa, &tmW, kb * BK, n0, fb);
                tma_load_2d(sa + L::A_BYTES, &tmX, kb * BK, m0, fb);
                // scale words: 128 to a tile of 128 rows x 4 blocks, the tiles of a band in a row
                tma_load_2d(sa + L::A_BYTES + L::B_BYTES, &tmSW, kb * (128 * L::GROUPS), tile, fb);
                tma_load_2d(sa + L::A_BYTES + L::B_BYTES + L::SF_BYTES, &tmSX, kb * (128 * L::GROUPS), m0 >> 7, fb);
                if (++stage == stages) { stage = 0; phase ^= 1u; }
            }
            if (!ok) {
                // aborting: let copies that are still in flight land before the CTA retires
                for (int s = 0; s < stages; ++s) {
                    const long long t0 = clock64();
                    while (clock64() - t0 < 200000) { /* bounded drain window */ }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            constexpr uint32_t idesc = mx_idesc(XB == 4 ? 1 : 5, XB == 4 ? 1 : 0, BM, BN);
            int stage = 0, slot = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int kb = kb0; kb < kb1; ++kb) {
                ok = mbar_wait(smem_u32(&full_bar[stage]), phase, abort_flag, p.status, ST_MMA);
                if (!ok) break;
                tc_fence_after();
                const uint32_t sa = smem_u32(ring + stage * L::STAGE_BYTES), ss = sa + L::A_BYTES + L::B_BYTES;
                const uint32_t t_sfa = tmem_base + (uint32_t)(BN + slot * L::SF_SLOT), t_sfb = t_sfa + 4 * L::GROUPS;
#pragma unroll
                for (int g = 0; g < L::GROUPS; ++g) {
                    scales_to_tmem(t_sfa + 4 * g, make_scale_desc(ss + g * 512));
                    scales_to_tmem(t_sfb + 4 * g, make_scale_desc(ss + L::SF_BYTES + g * 512));
                }
                // instructions of the block: fewer than four in a last one that ends behind K, where the operands are zero, but nothing
                // says what the scale bytes of a group that no tile of the tensor has would hold
                const int instr = min(4, (p.K - kb * KB + KI - 1) / KI);
                const uint64_t a_desc = make_smem_desc(sa), b_desc = make_smem_desc(sa + L::A_BYTES);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    if (kk >= instr) break;
                    const int g = XB == 4 ? kk >> 1 : 0;
                    const uint32_t sf = XB == 4 ? (uint32_t)(kk & 1) * 2 : (uint32_t)kk;
                    umma_mx<XB>(tmem_base, a_desc + (uint64_t)(kk * 2), b_desc + (uint64_t)(kk * 2), idesc | (sf << 4) | (sf << 29),
                                kb == kb0 && kk == 0 ? 0u : 1u, t_sfa + 4 * g, t_sfb + 4 * g);
                }
                umma_commit(smem_u32(&empty_bar[stage]));
                slot = slot + 1 == L::SF_SLOTS ? 0 : slot + 1;
                if (++stage == stages) { stage = 0; phase ^= 1u; }
            }
            if (ok) umma_commit(smem_u32(tfull_bar));
        }
        __syncwarp();
    }
    if (warp >= 2) {
        // warp w reads tensor-memory lanes [32 (w & 3), +32), rows of w, and the column half (w - 2) / 4, rows of x
        constexpr int CW = BN / 2;
        const int row = (warp & 3) * 32 + lane, j0 = ((warp - 2) >> 2) * CW;
        bool ok = mbar_wait(smem_u32(tfull_bar), 0, abort_flag, p.status, ST_EPILOGUE);
        ok = __all_sync(0xffffffffu, ok);
        if (ok && j0 < live) {
            tc_fence_after();
            uint32_t r[CW];
            const uint32_t t_row = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)j0;
            if constexpr (CW == 16) {
                tmem_ld16_issue(t_row, r);
            } else {
#pragma unroll
                for (int c = 0; c < CW; c += 32) tmem_ld32_issue(t_row + c, &r[c]);
            }
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < CW; ++j) pin(r[j]);
            if (splits > 1) {
                float *part = reinterpret_cast<float *>(ring) + j0 * BM + row;       // [row of x][row of w]
#pragma unroll
                for (int j = 0; j < CW; ++j) part[j * BM] = __uint_as_float(r[j]);
            } else if (n0 + row < p.rows_w) {
                if (p.y_f32) {
                    float *dst = static_cast<float *>(p.y) + (m0 + j0) * p.ldy + n0 + row;
#pragma unroll
                    for (int j = 0; j < CW; ++j, dst += p.ldy)
                        if (j < live - j0) *dst = __uint_as_float(r[j]);
                } else {
                    __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(p.y) + (m0 + j0) * p.ldy + n0 + row;
#pragma unroll
                    for (int j = 0; j < CW; ++j, dst += p.ldy)
                        if (j < live - j0) *dst = __float2bfloat16_rn(__uint_as_float(r[j]));
                }
            }
        }
    }
    // tensor memory goes back before anybody waits for the cluster: another kernel's CTA may need it to let one of the cluster start
    tc_fence_before();
    __syncwarp();
    if (splits > 1) cluster_arrive();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(L::TMEM_COLS) : "memory");
    }
    if (splits > 1) {
        __syncwarp();
        cluster_wait();
        if (warp >= 2) {
            const int own = (live + splits - 1) / splits, first = split * own, last = min(first + own, live);
            const int n = n0 + 4 * lane;
            for (int j = first + warp - 2; j < last; j += EPI_WARPS) {
                const uint32_t at = smem_u32(ring) + (uint32_t)((j * BM + 4 * lane) * 4);
                float4 v[MAX_SPLITS];
#pragma unroll
                for (int q = 0; q < MAX_SPLITS; ++q) v[q] = q < splits ? load_from_cta(at, q) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                float4 s = v[0];
#pragma unroll
                for (int q = 1; q < MAX_SPLITS; ++q)
                    if (q < splits) { s.x += v[q].x; s.y += v[q].y; s.z += v[q].z; s.w += v[q].w; }
                const float f[4] = {s.x, s.y, s.z, s.w};
                const long long to = (m0 + j) * p.ldy + n;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (n + i < p.rows_w) {
                        if (p.y_f32) static_cast<float *>(p.y)[to + i] = f[i];
                        else static_cast<__nv_bfloat16 *>(p.y)[to + i] = __float2bfloat16_rn(f[i]);
                    }
            }
        }
        __syncwarp();
        cluster_arrive();                        // nobody leaves while others read its sums
        cluster_wait();
    }
}

template <int BN, int XB>
int launch_thin(const CUtensorMap *tm, const ThinArgs &p, int splits, int ctas_sm, cudaStream_t st) {
    using L = Thin<BN, XB>;
    static DynamicSmemOnce smem_attr;
    cudaError_t e = smem_attr.set(mx_thin_kernel<BN, XB>, SMEM_OPTIN_MAX);
    if (e != cudaSuccess) return cuda_fail(e);
    constexpr int fixed = 1024 + L::RING_OFFSET;
    const int room = (SMEM_OPTIN_MAX + 1024) / ctas_sm - 1024;
    const int stages = std::min(MAX_STAGES, (room - fixed) / L::STAGE_BYTES);
    const unsigned grid = (unsigned)((p.rows_w + BM - 1) / BM * ((p.rows_x + BN - 1) / BN) * splits);
    e = launch_pdl(mx_thin_kernel<BN, XB>, dim3(grid), dim3(NUM_THREADS), (size_t)(fixed + stages * L::STAGE_BYTES), st, splits, tm[0],
                   tm[1], tm[2], tm[3], splits, stages, p);
    return e == cudaSuccess ? QUEST_OK : cuda_fail(e);
}

}  // namespace

int launch_mx_thin(const uint8_t *xq, const uint8_t *sx, int bits_x, const uint8_t *wq, const uint8_t *sw, int64_t M, int64_t N,
                   int64_t K, void *y, int y_dtype, int64_t ldy, cudaStream_t st) {
    const ThinArgs p = {(int)N, (int)M, (int)K, y, y_dtype == QUEST_F32, (long long)ldy, device_status_word()};
    if (!p.status) return QUEST_ERR_CUDA;
    const bool x4 = bits_x == 4;
    const int groups = x4 ? 2 : 1, bn = M <= 32 ? 32 : M <= 64 ? 64 : 128;
    CUtensorMap tm[4];
    int s;
    if ((s = mx_weight_map(&tm[0], wq, N, K, !x4, BM)) || (s = make_map(&tm[1], {xq, K * bits_x / 8, M, K * bits_x / 8, BK, bn})) ||
        (s = mx_scale_map(&tm[2], sw, N, K, groups, 1)) || (s = mx_scale_map(&tm[3], sx, M, K, groups, 1)))
        return s;
    const int tiles = (int)((N + BM - 1) / BM * ((M + bn - 1) / bn)), kbs = (int)((K + (x4 ? 255 : 127)) / (x4 ? 256 : 128)), sms = num_sms();
    // Parts of K, in powers of two (clusters of three or six leave SMs of a pair idle: 384 x 2048 x 8192 in thirds takes 1.2 times the time
    // of the 256-row tiles, 512 x 2048 x 8192 in halves 0.9).  A part costs about a microsecond, more with more rows of x, so it has to
    // save more k-blocks; with up to 32 rows two CTAs share an SM.  164 products of 24 to 512 rows in 1, 2, 4 and 8 parts: with the
    // parts taken below 1.006 times the best of each on average, 1.12 at worst (48 x 1024 x 8192); all unsplit 1.21, 2.5 at worst.
    int splits = 1;
    if (bn == 32) {
        if ((kbs >= 32 && 8 * tiles <= sms) || (kbs >= 80 && 8 * tiles <= 2 * sms)) splits = 8;
        else if ((kbs >= 16 && 4 * tiles <= 2 * sms) || (kbs >= 8 && 4 * tiles <= sms)) splits = 4;
        else if (kbs >= 20 && tiles <= sms) splits = 2;
    } else {
        if (kbs >= 16 && 4 * tiles <= sms) splits = 4;
        else if (kbs >= 24 && 2 * tiles <= sms) splits = 2;
    }
    const int ctas_sm = tiles * splits > sms || splits > 4 ? 2 : 1;
    if (bn == 32) return x4 ? launch_thin<32, 4>(tm, p, splits, ctas_sm, st) : launch_thin<32, 8>(tm, p, splits, ctas_sm, st);
    if (bn == 64) return x4 ? launch_thin<64, 4>(tm, p, splits, ctas_sm, st) : launch_thin<64, 8>(tm, p, splits, ctas_sm, st);
    return x4 ? launch_thin<128, 4>(tm, p, splits, ctas_sm, st) : launch_thin<128, 8>(tm, p, splits, ctas_sm, st);
}

}  // namespace quest
