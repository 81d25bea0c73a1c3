// What the block-scaled tensor-core products share: instruction and scale descriptors, tensor maps of weights and scales.
#pragma once
#include "quest_mx.cuh"
#include "quest_tcgen05.cuh"

namespace quest {

// Instruction descriptor, block-scaled kinds: element types of A and B, UE8M0 scales, M, N; the scale byte of a
// 32-bit word that an instruction starts from (sf) goes into bits 4 (B) and 29 (A).
// kind::mxf4: E2M1 is type 1.  kind::mxf8f6f4: E4M3 is type 0, E2M1 type 5.
__host__ __device__ constexpr uint32_t mx_idesc(int type_a, int type_b, int m, int n) {
    return ((uint32_t)type_a << 7) | ((uint32_t)type_b << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 7) << 27);
}
// Descriptor of 512 scale bytes (128 rows x 4 blocks): no swizzle, groups of eight 16-byte rows 128 bytes apart.
__device__ __forceinline__ uint64_t make_scale_desc(uint32_t smem_addr) {
    return (uint64_t)((smem_addr & 0x3FFFF) >> 4) | (uint64_t)1 << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
// Scale bytes of `rows` rows as words: a box is `bands` bands of 128 rows and `groups` tiles of four blocks.
inline int mx_scale_map(CUtensorMap *m, const uint8_t *scales, int64_t rows, int64_t K, int groups, int bands) {
    const int64_t tiles = (K + 127) / 128;
    return make_map(m, {scales, 128 * tiles, (rows + 127) / 128, 512 * tiles, 128 * groups, bands, CU_TENSOR_MAP_DATA_TYPE_UINT32,
                        CU_TENSOR_MAP_SWIZZLE_NONE});
}
// Rows of 4-bit weights, 128 bytes a box in shared memory: packed, or elements that the copy engine spreads to bytes.
inline int mx_weight_map(CUtensorMap *m, const uint8_t *wq, int64_t N, int64_t K, bool spread, int box_rows) {
    if (!spread) return make_map(m, {wq, K / 2, N, K / 2, 128, box_rows});
    return make_map(m, {wq, K, N, K / 2, 128, box_rows, CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B});
}

}  // namespace quest
