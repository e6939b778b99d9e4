// Device helpers and tensor maps of the products' tile kernels (linear.cu, entropy.cu): operands by TMA, MMAs of one or
// two blocks, stores by TMA.
#pragma once

#include "ep_common.cuh"
#include "tc_device.cuh"

#include <algorithm>
#include <mutex>

namespace eptile {

using namespace eptc;

constexpr unsigned WHOLE_WARP = 0xffffffffu;

// Called by the whole warp; the elected lane (always the same one) issues.
__device__ __forceinline__ void tma_store_3d_elected(const CUtensorMap *map, const void *src, int x, int y, int z) {
    asm volatile("{\n.reg .pred pe;\nelect.sync _|pe, 0xffffffff;\n"
                 "@pe cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];\n"
                 "@pe cp.async.bulk.commit_group;\n}" ::"l"(map),
                 "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
// Until at most PENDING of the warp's stores still read shared memory; all lanes may then write there.  (Only the elected
// lane has any to wait for.)
template <int PENDING>
__device__ __forceinline__ void stores_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory");
    __syncwarp();
}
// What the lanes have written becomes visible to the stores that are issued next.
__device__ __forceinline__ void before_stores() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

// The four K-steps of one k-block.
#define EP_UMMA_KBLOCK(GROUP, KIND)                                                                                        \
    asm volatile("{\n.reg .pred pe, pa, pt;\n"                                                                             \
                 "elect.sync _|pe, 0xffffffff;\n"                                                                          \
                 "setp.ne.b32 pa, %10, 0;\nsetp.eq.b32 pt, 0, 0;\n"                                                        \
                 "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %5, %9, pa;\n"                             \
                 "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %2, %6, %9, pt;\n"                             \
                 "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %3, %7, %9, pt;\n"                             \
                 "@pe tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %4, %8, %9, pt;\n}" ::"r"(d_tmem),             \
                 "l"(adesc), "l"(a1), "l"(a2), "l"(a3), "l"(bdesc), "l"(b1), "l"(b2), "l"(b3), "r"(idesc),                 \
                 "r"(accumulate_first)                                                                                     \
                 : "memory")
// What the tensor core multiplies: 16-bit floats, e4m3, or 8-bit integers (whose sums are 32-bit integers).
enum Kind { HALF, E8, INT };
template <Kind KIND, bool PAIR>
__device__ __forceinline__ void umma_kblock_elected(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint64_t astep,
                                                    uint64_t bstep, uint32_t idesc, uint32_t accumulate_first) {
    const uint64_t a1 = adesc + astep, a2 = a1 + astep, a3 = a2 + astep;
    const uint64_t b1 = bdesc + bstep, b2 = b1 + bstep, b3 = b2 + bstep;
    if constexpr (KIND == INT && PAIR)
        EP_UMMA_KBLOCK("2", "i8");
    else if constexpr (KIND == INT)
        EP_UMMA_KBLOCK("1", "i8");
    else if constexpr (KIND == E8 && PAIR)
        EP_UMMA_KBLOCK("2", "f8f6f4");
    else if constexpr (KIND == E8)
        EP_UMMA_KBLOCK("1", "f8f6f4");
    else if constexpr (PAIR)
        EP_UMMA_KBLOCK("2", "f16");
    else
        EP_UMMA_KBLOCK("1", "f16");
}
#undef EP_UMMA_KBLOCK

// Forms for a pair of blocks.  The barrier's address may be the other block's (shared::cluster).
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// (relaxed: nothing but the reading of TMEM goes before it, which tcgen05's own fence and wait order; with release an
// arrival at the other block took 1500 clocks)
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void load_tile_elected(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    if constexpr (PAIR)
        asm volatile("{\n.reg .pred pe;\nelect.sync _|pe, 0xffffffff;\n"
                     "@pe cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], "
                     "[%1, {%2, %3, %4}], [%5];\n}" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                     : "memory");
    else
        asm volatile("{\n.reg .pred pe;\nelect.sync _|pe, 0xffffffff;\n"
                     "@pe cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], "
                     "[%1, {%2, %3, %4}], [%5];\n}" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                     : "memory");
}
// One arrival at the barrier, of both blocks where there are two, when all MMAs issued so far are done.
template <bool PAIR>
__device__ __forceinline__ void commit_elected(uint64_t *bar) {
    if constexpr (PAIR)
        asm volatile("{\n.reg .pred pe;\nelect.sync _|pe, 0xffffffff;\n"
                     "@pe tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}" ::"r"(
                         smem_u32(bar)),
                     "h"((uint16_t)3)
                     : "memory");
    else
        umma_commit_elected(bar);
}

// Shared-memory descriptor of an operand tile, 128-byte swizzle.  K-major: rows of 128 bytes along k, groups of 8 rows
// 1024 bytes apart; a K-step is 32 bytes further along the row.  MN-major: boxes of 64 columns x 64 k, 8192 bytes
// apart; inside a box rows of 128 bytes hold the 64 columns of one k, groups of 8 k are 1024 bytes apart, and a K-step
// of 16 k is two groups on.
__device__ __forceinline__ uint64_t operand_desc(uint32_t smem, bool mn) {
    const uint64_t lead = mn ? 8192 >> 4 : 1;
    return (uint64_t)((smem & 0x3FFFFu) >> 4) | (lead << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// ---------------------------------------------------------------------------------------------- host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiledFn encode_tiled_fn() {
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// A tile of the operand is 128 bytes of k (K-major) or 64 of its columns x 64 k (MN-major) by box_rows rows.
inline bool encode_operand(CUtensorMap *map, const ep::Operand &o, bool mn, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t size = (cuuint64_t)ep::type_size(o.type);
    const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.parts};
    const cuuint64_t strides[2] = {(cuuint64_t)o.ld * size, (cuuint64_t)(o.parts > 1 ? o.part_stride : o.ld * o.rows) * size};
    const cuuint32_t box[3] = {(cuuint32_t)(128 / size), (cuuint32_t)(mn ? 64 : box_rows), 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUtensorMapDataType type = o.type == EP_BF16  ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                     : o.type == EP_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                        : CU_TENSOR_MAP_DATA_TYPE_UINT8;
    return fn(map, type, 3, const_cast<void *>(o.base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A matrix [depth][rows][cols] as a warp of the tile kernel writes it: boxes of 32 rows of 128 bytes
// (64 bytes where a warp has only 32 columns of 16 bits).
inline bool encode_result(CUtensorMap *map, void *base, int type, int64_t depth, int64_t rows, int cols, int64_t ld, int bn) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t size = (cuuint64_t)ep::type_size(type);
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)depth};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * size, (cuuint64_t)(ld * rows) * size};
    const cuuint32_t width = (cuuint32_t)std::min<int64_t>(128 / (int64_t)size, bn == 256 ? 64 : 32);
    const cuuint32_t box[3] = {width, 32, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUtensorMapDataType t = type == EP_BF16  ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                  : type == EP_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                   : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    return fn(map, t, 3, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              width * size == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace eptile
