// Blackwell tensor-core plumbing shared by the contractions: barriers with bounded waits, descriptors, TMA loads of a CTA
// pair, tensor-memory reads, the tile order, and (host) cached tensor maps.
#pragma once
#include <cuda.h>

#include "quest_internal.cuh"

namespace quest {

constexpr long long WAIT_LIMIT_CYCLES = 4000000000LL;   // ~2 s at 2 GHz

enum { ST_OK = 0, ST_PRODUCER = 1, ST_MMA = 2, ST_EPILOGUE = 3 };

__device__ __forceinline__ uint32_t smem_u32(const void *p) {
    return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Bounded wait.  Returns false if the CTA is aborting or the limit expired (then it records
// `code` in the device status word and raises the CTA-wide abort flag).
static __device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity, volatile int *abort_flag,
                                            int *status, int code, long long limit_cycles) {
    const long long t0 = clock64();
    for (uint32_t it = 0; it < 0x7fffffffu; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 15u) == 15u) {
            if (*abort_flag) return false;
            if (clock64() - t0 > limit_cycles) break;
        }
    }
    *abort_flag = 1;
    atomicExch(status, code);
    return false;
}

__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, int *status, int code,
                                          long long limit_cycles = WAIT_LIMIT_CYCLES) {
    if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait_slow(bar, parity, abort_flag, status, code, limit_cycles);
}

// One thread of a converged warp.  The tensor-core and copy instructions take their operands from uniform registers;
// behind elect.sync the compiler knows that a single thread executes them, behind a test of the lane index it does not:
// then a k-block costs the issuing threads about 620 cycles whatever the tile, more than the 524 the tensor cores need
// for a 256 x 256 tile.  With it (and the inlined first try of the waits) the main loop runs at 516 cycles per k-block:
// 4096 x 2048 x 2048 17.4 -> 15.8 us, 8192 x 5504 x 2048 71.9 -> 65.6 us (with zeros for operands, which draw less power,
// 16.1 -> 14.0 and 65.5 -> 55.9 us).
__device__ __forceinline__ bool elect_one() {
    uint32_t is;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(is));
    return is != 0;
}

// Shared-memory matrix descriptor: K-major operand, 128-byte swizzle, rows of 128 bytes,
// 8-row groups 1024 bytes apart.
__device__ __forceinline__ uint64_t make_smem_desc(uint32_t smem_addr) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFF) >> 4);          // start address, bits [0,14)
    d |= (uint64_t)1 << 16;                                // leading byte offset (unused with swizzle), bits [16,30)
    d |= (uint64_t)(1024 >> 4) << 32;                      // stride byte offset, bits [32,46)
    d |= (uint64_t)1 << 46;                                // descriptor version (sm_100), bits [46,48)
    d |= (uint64_t)2 << 61;                                // layout: SWIZZLE_128B, bits [61,64)
    return d;
}
__device__ __forceinline__ uint32_t cluster_ctarank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// shared::cluster address of the same shared-memory offset in CTA `rank` of this cluster
__device__ __forceinline__ uint32_t mapa_shared(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The two halves of the cluster barrier on their own: a warp arrives as soon as it has nothing left to publish to
// the peer CTA and waits only where it needs the peer, so the barrier's latency overlaps the work between.
__device__ __forceinline__ void cluster_arrive() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// cta_group::2 forms: the load may signal an mbarrier of the peer CTA; the MMA spans both CTAs of
// the pair; the commit arrives on the same barrier offset in every CTA named by the mask.
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap *tm, int c0, int c1, uint32_t cluster_bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(cluster_bar), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void umma_commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3)
                 : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Tile order: m fastest inside bands of RASTER_M row tiles, bands one after another.  Concurrent CTAs
// then share one or two column tiles of B while the rows of A a band touches (RASTER_M x TILE_M x K
// bytes) stay in L2 for all of the band's column tiles; with a single band (up to RASTER_M row tiles)
// this is plain column-major order.
constexpr int RASTER_M = 16;
__device__ __forceinline__ void tile_coords(int tile, int num_m, int num_n, int &tm, int &tn) {
    const int band_tiles = RASTER_M * num_n;
    const int band = tile / band_tiles;
    const int t = tile - band * band_tiles;
    const int rows_here = min(RASTER_M, num_m - band * RASTER_M);
    tn = t / rows_here;
    tm = band * RASTER_M + (t - tn * rows_here);
}

// 32 columns of this warp's 32 TMEM lanes, issued without waiting: the registers are valid only
// after tmem_wait_ld() and pin() (an empty volatile asm that makes every later use depend on a
// statement ordered after the wait).
__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pin(uint32_t &v) { asm volatile("" : "+r"(v)::"memory"); }

// Tensor maps (host).  Encoding one is a driver call of a microsecond or two; each host thread keeps the last few.
struct MapSpec {
    const void *base;
    int64_t d0, d1, pitch;              // elements of a row, rows, bytes between rows
    int box0, box1;                     // elements, rows
    CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_UINT8;
    CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B;
    CUtensorMapL2promotion promo = CU_TENSOR_MAP_L2_PROMOTION_L2_256B;
    bool operator==(const MapSpec &o) const {
        return base == o.base && d0 == o.d0 && d1 == o.d1 && pitch == o.pitch && box0 == o.box0 && box1 == o.box1 &&
               type == o.type && swizzle == o.swizzle && promo == o.promo;
    }
};
int make_map(CUtensorMap *tm, const MapSpec &spec);
// int8 matrix [rows x K], K contiguous; box = 128 bytes of K x box_rows rows, 128-byte swizzle.
int make_operand_map(CUtensorMap *tm, const int8_t *base, int64_t rows, int64_t K, int box_rows);
// Whether y leaves by tile stores (make_output_map): base, pitch and the end of a row on 16-byte boundaries.  Tile stores write whole 16-byte pieces: of a
// row that ends inside one they would overwrite what stands behind it.
bool tile_stores(const void *y, int64_t N, int64_t ldy, size_t esz);
// y viewed as bytes: [rows x row_bytes], row pitch pitch_bytes; box = 128 bytes x 32 rows, 128-byte swizzle.
int make_output_map(CUtensorMap *tm, void *base, int64_t rows, int64_t row_bytes, int64_t pitch_bytes);

}  // namespace quest
