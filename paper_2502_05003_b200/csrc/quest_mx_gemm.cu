// Product of two microscaled tensors on the tensor cores:
//
//   y[m][n] = sum over blocks of 32 of 2^(sx + sw - 254) sum_k qx[m][k] qw[n][k]     binary32 accumulators
//
// tcgen05.mma kind::mxf4 where both operands are E2M1 (4 times the bfloat16 rate), kind::mxf8f6f4 where x is E4M3 (twice
// the rate).  The scales are applied by the tensor cores, which read them from tensor memory: a stage brings the scale bytes of its
// rows beside the operands, tcgen05.cp spreads them over the four lane quarters.  4-bit weights that meet 8-bit activations
// stay packed in memory: the copy engine spreads them to a byte each on the way to shared memory.
//
// Structure (as the contraction of the uniform grids): clusters of two CTAs on tiles of 256 x BN, each CTA stages its 128 rows of
// x and half of the tile's rows of w, but the scales of all BN rows of w, which both of the pair's tensor cores need.
//   warp 0      copies, 128 bytes of K a stage (256 elements of E2M1 against E2M1, 128 otherwise)
//   warp 1      scales to tensor memory, then up to four MMAs a stage
//   warps 2..9  epilogue: accumulators to registers, conversion, tile stores
// Every wait is bounded.
//
// 16384 x 4096 x 4096: 95 us in 4 bits (5.8 PFLOP/s), 180 in 8 bits against 4 (3.05), the tensor cores at work 71 and 83 % of the
// cycles (8192 x 4096 x 4096).  What bounds the first is L2: with a quarter of its products and everything else as it is it still takes
// 76 us (35.8 KB a k-block and CTA, 15 TB/s over the chip), without its stores 88; the scales' copies cost nothing measurable.
// Tensor memory has room for one 256-column accumulator beside the scales, so the products of a tile wait until the tile before
// has left for registers.  Few tiles: 768 x 2048 x 5504 takes 12 us, 43 k-blocks at 0.17 us and 4.5 us of launch, first loads and last epilogue.
#include <algorithm>

#include "quest_mx_tcgen05.cuh"

namespace quest {
namespace {

constexpr int BM = 128;
constexpr int BK = 128;                          // bytes of a stage's rows in shared memory
constexpr int EPI_WARPS = 8;
constexpr int NUM_THREADS = 64 + 32 * EPI_WARPS;
constexpr int MAX_STAGES = 6;
constexpr int SMEM_OPTIN_MAX = 232448;

struct MxGemmParams {
    int M, N, K;
    void *y;
    int y_dtype;
    long long ldy;
    int *status;
};

template <int XB>
__device__ __forceinline__ void umma_mx_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate,
                                             uint32_t sfa_tmem, uint32_t sfb_tmem) {
    if constexpr (XB == 4)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(sfa_tmem), "r"(sfb_tmem)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(sfa_tmem), "r"(sfb_tmem)
            : "memory");
}
// 512 scale bytes (128 rows x 4 blocks) of each CTA's shared memory -> four columns of its tensor memory, the same in all
// four lane quarters.
__device__ __forceinline__ void scales_to_tmem_pair(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// Shared memory from a 1024-byte-aligned base: output staging, barriers, then the ring.
template <int BN, int XB>
struct Layout {
    static constexpr int GROUPS = XB == 4 ? 2 : 1;                   // scale tiles (four blocks) of a row in a stage
    static constexpr int A_BYTES = BM * BK;
    static constexpr int B_ROWS = BN / 2;
    static constexpr int B_BYTES = B_ROWS * BK;
    static constexpr int SFA_BYTES = GROUPS * 512;
    static constexpr int SFB_BYTES = BN / 128 * GROUPS * 512;
    // bytes that arrive: nibbles that are spread in shared memory count as the bytes they were
    static constexpr int LOAD_BYTES = A_BYTES + (XB == 4 ? B_BYTES : B_BYTES / 2) + SFA_BYTES + SFB_BYTES;
    static constexpr int STAGE_BYTES = (A_BYTES + B_BYTES + SFA_BYTES + SFB_BYTES + 1023) / 1024 * 1024;
    static constexpr int SLABS = BN == 128 ? 2 : 1;
    static constexpr int STG_BYTES = EPI_WARPS * SLABS * 4096;
    static constexpr int BAR_OFFSET = STG_BYTES;
    static constexpr int RING_OFFSET = (BAR_OFFSET + 256 + 1023) / 1024 * 1024;
    static constexpr int WANTED = RING_OFFSET + MAX_STAGES * STAGE_BYTES + 1024;
    static constexpr int TOTAL = WANTED > SMEM_OPTIN_MAX ? SMEM_OPTIN_MAX : WANTED;
    // tensor memory: accumulators, then the scales of a few stages in turn
    static constexpr int NBUF = BN == 256 ? 1 : 2;
    static constexpr int SF_COL = 256;
    static constexpr int SF_SLOT = 4 * GROUPS * (1 + BN / 128);      // columns of one stage: A's, then B's
    static constexpr int SF_SLOTS = 4;
    static constexpr int TMEM_COLS = 512;
    static_assert(SF_COL + SF_SLOTS * SF_SLOT <= TMEM_COLS && NBUF * BN <= SF_COL, "tensor memory");
    static_assert(RING_OFFSET + 2 * STAGE_BYTES + 1024 <= TOTAL, "at least two stages must fit");
};

template <int BN, int XB, bool YT>
__global__ void __launch_bounds__(NUM_THREADS, 1)
mx_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmSA,
               const __grid_constant__ CUtensorMap tmSB, const __grid_constant__ CUtensorMap tmY, MxGemmParams p) {
    using L = Layout<BN, XB>;
    constexpr int TILE_M = 2 * BM;
    constexpr int KB = XB == 4 ? 256 : 128;      // elements of K per stage
    constexpr int KI = KB / 4;                   // and per instruction
    constexpr int CW = BN / 2;                   // columns per epilogue warp
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    int stages;
    {
        uint32_t dyn;
        asm volatile("mov.u32 %0, %%dynamic_smem_size;" : "=r"(dyn));
        stages = ((int)dyn - (int)(smem - smem_raw) - L::RING_OFFSET) / L::STAGE_BYTES;
        if (stages > MAX_STAGES) stages = MAX_STAGES;
        if (stages < 2) {                        // a launch with too little shared memory: refuse, touch nothing
            if (threadIdx.x == 0) atomicExch(p.status, ST_PRODUCER);
            return;
        }
    }
    uint8_t *ring = smem + L::RING_OFFSET;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + L::BAR_OFFSET);
    uint64_t *full_bar = bars, *empty_bar = bars + MAX_STAGES;
    uint64_t *tfull_bar = bars + 2 * MAX_STAGES, *tempty_bar = bars + 2 * MAX_STAGES + 2;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * MAX_STAGES + 4);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    pdl_launch_dependents();
    if (threadIdx.x == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmA)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmB)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmSA)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmSB)) : "memory");
        if constexpr (YT) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmY)) : "memory");
    }
    const int unit = (int)(blockIdx.x >> 1), num_units = (int)(gridDim.x >> 1);
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&tfull_bar[b]), 1);
            mbar_init(smem_u32(&tempty_bar[b]), 2 * EPI_WARPS);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    // every warp arrives at the cluster barrier as soon as it has nothing more to publish to the peer
    __syncwarp();
    cluster_arrive();
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                     "r"(L::TMEM_COLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_wait();                              // the peer's barriers are initialised before anything signals them
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();

    const int num_m = (p.M + TILE_M - 1) / TILE_M, num_n = (p.N + BN - 1) / BN;
    const int num_tiles = num_m * num_n;
    const int num_kb = (p.K + KB - 1) / KB;
    bool left = false;                           // this warp has arrived at the cluster barrier of the exit

    if (warp == 0) {
        if (elect_one()) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int tile = unit; tile < num_tiles && ok; tile += num_units) {
                int tm, tn;
                tile_coords(tile, num_m, num_n, tm, tn);
                const int m0 = tm * TILE_M + (int)rank * BM, n0 = tn * BN;
                for (int kb = 0; kb < num_kb; ++kb) {
                    ok = mbar_wait(smem_u32(&empty_bar[stage]), phase ^ 1u, abort_flag, p.status, ST_PRODUCER);
                    if (!ok) break;
                    const uint32_t fb = smem_u32(&full_bar[stage]), sa = smem_u32(ring + stage * L::STAGE_BYTES);
                    // both CTAs' loads complete on the leader's barrier, which expects the bytes of both
                    if (leader) mbar_expect_tx(fb, 2 * L::LOAD_BYTES);
                    const uint32_t lfb = mapa_shared(fb, 0);
                    tma_load_2d_pair(sa, &tmA, kb * BK, m0, lfb);
                    // packed weights against packed activations: bytes; spread to bytes: elements.  Both 128 a stage
                    tma_load_2d_pair(sa + L::A_BYTES, &tmB, kb * BK, n0 + (int)rank * L::B_ROWS, lfb);
                    // scale words: 128 to a tile of 128 rows x 4 blocks, the tiles of a band in a row
                    tma_load_2d_pair(sa + L::A_BYTES + L::B_BYTES, &tmSA, kb * (128 * L::GROUPS), m0 >> 7, lfb);
                    tma_load_2d_pair(sa + L::A_BYTES + L::B_BYTES + L::SFA_BYTES, &tmSB, kb * (128 * L::GROUPS), n0 >> 7, lfb);
                    if (++stage == stages) { stage = 0; phase ^= 1u; }
                }
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
        if (leader && elect_one()) {
            constexpr uint32_t idesc = mx_idesc(XB == 4 ? 1 : 0, XB == 4 ? 1 : 5, TILE_M, BN);
            const int num_whole = p.K / KB;
            int stage = 0, t = 0, slot = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int tile = unit; tile < num_tiles && ok; tile += num_units, ++t) {
                const int buf = L::NBUF == 2 ? (t & 1) : 0;
                const uint32_t bphase = (uint32_t)(L::NBUF == 2 ? (t >> 1) : t) & 1u;
                ok = mbar_wait(smem_u32(&tempty_bar[buf]), bphase ^ 1u, abort_flag, p.status, ST_MMA);
                if (!ok) break;
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + (uint32_t)(buf * BN);
                // one k-block: its scales, its products, the stage handed back.  instr: instructions of the block, fewer than four
                // in a last one that ends behind K: there the operands are zero, but nothing says what the scale bytes of a group
                // that no tile of the tensor has would hold
                const auto block = [&](bool first, int instr) {
                    ok = mbar_wait(smem_u32(&full_bar[stage]), phase, abort_flag, p.status, ST_MMA);
                    if (!ok) return;
                    tc_fence_after();
                    const uint32_t sa = smem_u32(ring + stage * L::STAGE_BYTES);
                    const uint32_t t_sfa = tmem_base + (uint32_t)(L::SF_COL + slot * L::SF_SLOT);
                    const uint32_t t_sfb = t_sfa + 4 * L::GROUPS;
                    // columns of B's scales: for each group of four blocks, four columns for each 128 rows
#pragma unroll
                    for (int g = 0; g < L::GROUPS; ++g) {
                        const uint64_t da = make_scale_desc(sa + L::A_BYTES + L::B_BYTES + g * 512);
                        scales_to_tmem_pair(t_sfa + 4 * g, da);
#pragma unroll
                        for (int b = 0; b < BN / 128; ++b) {
                            const uint64_t db = make_scale_desc(sa + L::A_BYTES + L::B_BYTES + L::SFA_BYTES + (b * L::GROUPS + g) * 512);
                            scales_to_tmem_pair(t_sfb + 4 * (g * (BN / 128) + b), db);
                        }
                    }
                    const uint64_t a_desc = make_smem_desc(sa), b_desc = make_smem_desc(sa + L::A_BYTES);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) {
                        if (kk >= instr) break;
                        const int g = XB == 4 ? kk >> 1 : 0;
                        const uint32_t sf = XB == 4 ? (uint32_t)(kk & 1) * 2 : (uint32_t)kk;
                        umma_mx_pair<XB>(d_tmem, a_desc + (uint64_t)(kk * 2), b_desc + (uint64_t)(kk * 2), idesc | (sf << 4) | (sf << 29),
                                         first && kk == 0 ? 0u : 1u, t_sfa + 4 * g, t_sfb + 4 * g * (BN / 128));
                    }
                    umma_commit_pair(smem_u32(&empty_bar[stage]));
                    slot = slot + 1 == L::SF_SLOTS ? 0 : slot + 1;
                    if (++stage == stages) { stage = 0; phase ^= 1u; }
                };
                for (int kb = 0; kb < num_whole && ok; ++kb) block(kb == 0, 4);
                if (ok && num_whole < num_kb) block(num_whole == 0, (p.K - num_whole * KB + KI - 1) / KI);
                if (!ok) break;
                umma_commit_pair(smem_u32(&tfull_bar[buf]));
            }
        }
        __syncwarp();
    } else {
        // warp w reads tensor-memory lanes [32 (w & 3), +32) = tile rows, and the column half (w - 2) / 4 of the tile
        const int quarter = warp & 3, cbase = ((warp - 2) >> 2) * CW;
        const bool y_f32 = p.y_dtype == QUEST_F32;
        uint8_t *slab_base = smem + (warp - 2) * (L::SLABS * 4096);
        int slab_count = 0, t = 0;
        for (int tile = unit; tile < num_tiles; tile += num_units, ++t) {
            int tm, tn;
            tile_coords(tile, num_m, num_n, tm, tn);
            const int m0 = tm * TILE_M + (int)rank * BM, n0 = tn * BN;
            const int buf = L::NBUF == 2 ? (t & 1) : 0;
            const uint32_t bphase = (uint32_t)(L::NBUF == 2 ? (t >> 1) : t) & 1u;
            bool ok = mbar_wait(smem_u32(&tfull_bar[buf]), bphase, abort_flag, p.status, ST_EPILOGUE);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const uint32_t t_row = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * BN);
            uint32_t r[CW];
#pragma unroll
            for (int c0 = 0; c0 < CW; c0 += 32)
                if (n0 + cbase + c0 < p.N) tmem_ld32_issue(t_row + (uint32_t)(cbase + c0), &r[c0]);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < CW; ++j) pin(r[j]);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(mapa_shared(smem_u32(&tempty_bar[buf]), 0));
            if (tile + num_units >= num_tiles) {       // this CTA's last tile: nothing more goes to the peer
                __syncwarp();
                cluster_arrive();
                left = true;
            }
            const int row = m0 + quarter * 32 + lane;
#pragma unroll
            for (int c0 = 0; c0 < CW; c0 += 32) {
                const int col0 = n0 + cbase + c0;
                if (col0 >= p.N) continue;             // uniform across the warp
                uint32_t *rc = &r[c0];
                if constexpr (YT) {
                    // 32 rows x 128 bytes in shared memory (128-byte swizzle), then one tile store, which clips at the edges
                    const int half = y_f32 ? 0 : ((c0 >> 5) & 1);
                    uint8_t *slab = slab_base + (L::SLABS == 2 ? (slab_count & 1) * 4096 : 0);
                    if (half == 0) {
                        if (lane == 0) {
                            if (L::SLABS == 2) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                            else asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                        }
                        __syncwarp();
                    }
                    uint8_t *rowp = slab + lane * 128;
                    const int sw7 = lane & 7;
                    if (y_f32) {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            *reinterpret_cast<uint4 *>(rowp + ((j ^ sw7) << 4)) = make_uint4(rc[4 * j], rc[4 * j + 1], rc[4 * j + 2], rc[4 * j + 3]);
                    } else {
                        uint32_t h[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(rc[2 * j]), __uint_as_float(rc[2 * j + 1]));
                            h[j] = *reinterpret_cast<const uint32_t *>(&b);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            *reinterpret_cast<uint4 *>(rowp + (((half * 4 + j) ^ sw7) << 4)) = make_uint4(h[4 * j], h[4 * j + 1], h[4 * j + 2], h[4 * j + 3]);
                    }
                    if (y_f32 || half == 1 || col0 + 32 >= p.N) {
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            const int xbytes = y_f32 ? col0 * 4 : (col0 - half * 32) * 2;
                            asm volatile(
                                "cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                                ::"l"(reinterpret_cast<uint64_t>(&tmY)), "r"(smem_u32(slab)), "r"(xbytes), "r"(m0 + quarter * 32)
                                : "memory");
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                        ++slab_count;
                    }
                } else if (row < p.M) {
                    // a base or pitch that no 16-byte access fits
                    if (y_f32) {
                        float *dst = reinterpret_cast<float *>(p.y) + (long long)row * p.ldy + col0;
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (col0 + j < p.N) dst[j] = __uint_as_float(rc[j]);
                    } else {
                        __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(p.y) + (long long)row * p.ldy + col0;
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (col0 + j < p.N) dst[j] = __float2bfloat16_rn(__uint_as_float(rc[j]));
                    }
                }
            }
        }
    }
    if constexpr (YT) {
        if (warp >= 2 && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    }
    tc_fence_before();
    __syncwarp();
    if (!left) cluster_arrive();
    cluster_wait();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(L::TMEM_COLS) : "memory");
    }
}

template <int BN, int XB, bool YT>
int launch_tiles(const CUtensorMap *tm, const MxGemmParams &p, cudaStream_t st) {
    using L = Layout<BN, XB>;
    static DynamicSmemOnce smem_attr;
    cudaError_t e = smem_attr.set(mx_gemm_kernel<BN, XB, YT>, L::TOTAL);
    if (e != cudaSuccess) return cuda_fail(e);
    const long long tiles = (long long)((p.M + 2 * BM - 1) / (2 * BM)) * ((p.N + BN - 1) / BN);
    const int pairs = (int)std::min<long long>(tiles, num_sms() / 2);
    e = launch_pdl(mx_gemm_kernel<BN, XB, YT>, dim3((unsigned)(2 * pairs)), dim3(NUM_THREADS), (size_t)L::TOTAL, st, 2, tm[0], tm[1],
                   tm[2], tm[3], tm[4], p);
    return e == cudaSuccess ? QUEST_OK : cuda_fail(e);
}

}  // namespace

int launch_mx_gemm(const uint8_t *xq, const uint8_t *sx, int bits_x, const uint8_t *wq, const uint8_t *sw, int64_t M, int64_t N,
                   int64_t K, void *y, int y_dtype, int64_t ldy, cudaStream_t st) {
    MxGemmParams p = {(int)M, (int)N, (int)K, y, y_dtype, (long long)ldy, device_status_word()};
    if (!p.status) return QUEST_ERR_CUDA;
    const bool x4 = bits_x == 4;
    const int64_t pairs = num_sms() / 2, tall = (M + 255) / 256;
    const int64_t rounds256 = (tall * ((N + 255) / 256) + pairs - 1) / pairs, rounds128 = (tall * ((N + 127) / 128) + pairs - 1) / pairs;
    // narrow tiles where they need no more than half again as many rounds: time with them over time with wide ones 0.64 .. 0.94 at equal
    // rounds, 0.92 .. 1.02 at three to two, 0.93 .. 1.07 at five to three, above that 1.0 .. 1.23 (70 shapes in both widths: within
    // 0.1 % of the better choice of each on average)
    const bool narrow = 2 * rounds128 <= 3 * rounds256;
    const int groups = x4 ? 2 : 1, bn = narrow ? 128 : 256;
    CUtensorMap tm[5];
    int s;
    if ((s = make_map(&tm[0], {xq, K * bits_x / 8, M, K * bits_x / 8, BK, BM})) || (s = mx_weight_map(&tm[1], wq, N, K, !x4, bn / 2)) ||
        (s = mx_scale_map(&tm[2], sx, M, K, groups, 1)) || (s = mx_scale_map(&tm[3], sw, N, K, groups, bn / 128)))
        return s;
    const size_t esz = y_dtype == QUEST_F32 ? 4 : 2;
    const bool yt = tile_stores(y, N, ldy, esz);
    tm[4] = tm[0];
    if (yt && (s = make_output_map(&tm[4], y, M, N * (int64_t)esz, ldy * (int64_t)esz))) return s;
    if (x4) {
        if (narrow) return yt ? launch_tiles<128, 4, true>(tm, p, st) : launch_tiles<128, 4, false>(tm, p, st);
        return yt ? launch_tiles<256, 4, true>(tm, p, st) : launch_tiles<256, 4, false>(tm, p, st);
    }
    if (narrow) return yt ? launch_tiles<128, 8, true>(tm, p, st) : launch_tiles<128, 8, false>(tm, p, st);
    return yt ? launch_tiles<256, 8, true>(tm, p, st) : launch_tiles<256, 8, false>(tm, p, st);
}

}  // namespace quest
