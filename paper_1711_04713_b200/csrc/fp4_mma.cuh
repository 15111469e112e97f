// Building blocks of the products of microscaled 4-bit operands: scale copies to TMEM, block-scaled MMA, outputs.
#pragma once

#include "fp4.cuh"
#include "tc_ptx.cuh"
#include "tensor_maps.cuh"

namespace adaption {
namespace {

constexpr int kRows = 128;                 // output channels of a CTA's tile
constexpr int kBlockBytes = 128;           // codes of a k-block and row
constexpr int kBlockElems = 256;
constexpr int kStepElems = 64;             // of one MMA
constexpr uint32_t kABytes = kRows * kBlockBytes;

__host__ __device__ constexpr int groups_of(int block) { return block == 32 ? 2 : 4; }    // scale tiles of a k-block and 128 rows

// Arrival on a barrier of any CTA of the cluster that orders this CTA's work only (TMEM reads, by the fence before it).
// With release at cluster scope it waited for the warp's stores to global memory: about 1000 cycles.
__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// Whether a phase has completed, without waiting for it (try_wait may suspend the thread for microseconds).
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// A box from shared memory to global memory, clipped at the tensor's ends; completion by groups of the issuing thread.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y)
               : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// at most N of the thread's last stores still read their shared memory
template <int N>
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void tma_store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ float4 ld_shared_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
// Arrival in the CTAs of `mask` once every instruction issued so far for the pair has retired.
__device__ __forceinline__ void commit_pair_if(uint32_t issue, uint32_t bar, uint16_t mask) {
  asm volatile(
      "{\n"
      ".reg .pred e;\n"
      "setp.ne.b32 e, %2, 0;\n"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n"
      "}\n" ::"r"(bar),
      "h"(mask), "r"(issue)
      : "memory");
}
// The issuing warp stays in uniform control flow and the lane with `issue` != 0 (elect_one, once) executes: operands live in
// uniform registers that way.  (In a branch of the elected lane, the sixteen instructions of a k-block of blocks of 16 took 700
// cycles to issue, more than the 512 that they run.)
//
// One scale tile (32 rows of 16 bytes) from shared memory to four TMEM columns, repeated in all lane quarters.  PAIR: in both
// CTAs, each from its own shared memory.
template <bool PAIR>
__device__ __forceinline__ void scales_to_tmem(uint32_t issue, uint32_t taddr, uint32_t desc_lo, uint32_t desc_hi) {
#define ADAPTION_SCALES(CG)                                       \
  asm volatile(                                                   \
      "{\n"                                                       \
      ".reg .pred e;\n"                                           \
      ".reg .b64 d;\n"                                            \
      "setp.ne.b32 e, %3, 0;\n"                                   \
      "mov.b64 d, {%1, %2};\n"                                    \
      "@e tcgen05.cp.cta_group::" CG ".32x128b.warpx4 [%0], d;\n" \
      "}\n" ::"r"(taddr),                                         \
      "r"(desc_lo), "r"(desc_hi), "r"(issue)                      \
      : "memory")
  if (PAIR)
    ADAPTION_SCALES("2");
  else
    ADAPTION_SCALES("1");
#undef ADAPTION_SCALES
}
template <int BLOCK, bool PAIR>
__device__ __forceinline__ void mma_fp4(uint32_t issue, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t desc_hi, uint32_t idesc,
                                        uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
#define ADAPTION_MMA_FP4(CG, KIND)                                                                 \
  asm volatile(                                                                                    \
      "{\n"                                                                                        \
      ".reg .pred p, e;\n"                                                                         \
      ".reg .b64 da, db;\n"                                                                        \
      "setp.ne.b32 e, %8, 0;\n"                                                                    \
      "setp.ne.b32 p, %5, 0;\n"                                                                    \
      "mov.b64 da, {%1, %3};\n"                                                                    \
      "mov.b64 db, {%2, %3};\n"                                                                    \
      "@e tcgen05.mma.cta_group::" CG "." KIND " [%0], da, db, %4, [%6], [%7], p;\n"               \
      "}\n" ::"r"(d),                                                                              \
      "r"(a_lo), "r"(b_lo), "r"(desc_hi), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb), "r"(issue) \
      : "memory")
  if (BLOCK == 32 && PAIR)
    ADAPTION_MMA_FP4("2", "kind::mxf4.block_scale.scale_vec::2X");
  else if (BLOCK == 32)
    ADAPTION_MMA_FP4("1", "kind::mxf4.block_scale.scale_vec::2X");
  else if (PAIR)
    ADAPTION_MMA_FP4("2", "kind::mxf4nvf4.block_scale.scale_vec::4X");
  else
    ADAPTION_MMA_FP4("1", "kind::mxf4nvf4.block_scale.scale_vec::4X");
#undef ADAPTION_MMA_FP4
}
// Instruction descriptor: E2M1 operands, both K-major, scales E8M0 (blocks of 32) or E4M3.
__device__ __forceinline__ uint32_t make_idesc_fp4(int block, int n, int m) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((block == 32 ? 1u : 0u) << 23) | ((uint32_t)(m >> 4) << 24);
}
// ... which two of the four scales of a TMEM word an instruction takes (blocks of 32): bytes 2 * half on
__device__ __forceinline__ uint32_t scale_half(uint32_t half) { return (half * 2u) << 4 | (half * 2u) << 29; }


// Codes: boxes of a k-block of `box_rows` rows.  A row ends with its last element's byte: what the box holds behind it arrives as zeros.
inline bool encode_fp4_codes(CUtensorMap* map, const adaption_fp4tensor& t, int64_t rows, int64_t inner, uint32_t box_rows, bool long_rows) {
  return encode_tiled_2d(map, t.codes, (uint64_t)(inner + 1) / 2, (uint64_t)rows, (uint64_t)t.c_stride / 2, kBlockBytes, box_rows,
                         CU_TENSOR_MAP_SWIZZLE_128B, long_rows);
}
// Scale planes: one row per row of scale tiles, in words of 8 bytes; boxes of a k-block of `box_tiles` rows of tiles.
inline bool encode_fp4_scales(CUtensorMap* map, const adaption_fp4tensor& t, int64_t rows, int64_t groups, uint32_t box_tiles) {
  const uint64_t dims[2] = {(uint64_t)groups * (kFp4TileBytes / 8), (uint64_t)((rows + kRows - 1) / kRows)};
  const uint64_t strides[1] = {(uint64_t)groups * kFp4TileBytes};
  const uint32_t box[2] = {(uint32_t)(groups_of(t.block) * (kFp4TileBytes / 8)), box_tiles};
  return encode_tiled_words(map, t.scales, 2, dims, strides, box);
}

}  // namespace
}  // namespace adaption
