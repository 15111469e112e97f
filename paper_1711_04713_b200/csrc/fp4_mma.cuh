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


// Scales to TMEM and MMAs of one k-block: `steps` instructions, `groups` scale tiles per 128 rows.  Scales of A go to the columns from
// ta on, of B from tb on, cols_b (4 or 8) per tile; in shared memory (from sf, in 16-byte units) those of A come first.
template <int BLOCK, bool PAIR>
__device__ __forceinline__ void issue_kblock(uint32_t issue, uint32_t d, uint32_t a, uint32_t b, uint32_t dhi, uint32_t id, uint32_t ta,
                                             uint32_t tb, uint32_t cols_b, uint32_t sf, uint32_t shi, uint32_t more, int steps, int groups) {
  constexpr int kGroups = groups_of(BLOCK);
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    if (g < groups) {
      scales_to_tmem<PAIR>(issue, ta + 4u * g, sf + 32u * g, shi);
      scales_to_tmem<PAIR>(issue, tb + cols_b * g, sf + 32u * (kGroups + g), shi);
      if (PAIR && cols_b == 8u) scales_to_tmem<PAIR>(issue, tb + cols_b * g + 4u, sf + 32u * (2 * kGroups + g), shi);
    }
  }
#pragma unroll
  for (int k = 0; k < kBlockElems / kStepElems; ++k) {
    const uint32_t g = BLOCK == 32 ? (uint32_t)k >> 1 : (uint32_t)k;
    if (k < steps)
      mma_fp4<BLOCK, PAIR>(issue, d, a + 2u * k, b + 2u * k, dhi, BLOCK == 32 ? id | scale_half(k & 1) : id, ta + 4u * g, tb + cols_b * g,
                           k > 0 ? 1u : more);
  }
}

// Outputs stored as 0 of one lane: pairs of 16-bit outputs are compared and counted together, in their own type (exact up to 256 pairs).
template <int DT>
struct ZeroCount {
  uint32_t n = 0;
  __half2 h = __floats2half2_rn(0.f, 0.f);
  __nv_bfloat162 b = __floats2bfloat162_rn(0.f, 0.f);
  __device__ __forceinline__ void pair(uint32_t w) {
    if (DT == ADAPTION_F16) h = __hadd2(h, __heq2(*reinterpret_cast<__half2*>(&w), __floats2half2_rn(0.f, 0.f)));
    else b = __hadd2(b, __heq2(*reinterpret_cast<__nv_bfloat162*>(&w), __floats2bfloat162_rn(0.f, 0.f)));
  }
  __device__ __forceinline__ uint32_t total() const {
    if (DT == ADAPTION_F32) return n;
    const float2 f = DT == ADAPTION_F16 ? __half22float2(h) : __bfloat1622float2(b);
    return n + (uint32_t)(f.x + f.y);
  }
};
template <int DT>
__device__ __forceinline__ uint32_t relu2(uint32_t w) {       // (a NaN stays one)
  if (DT == ADAPTION_F16) {
    const __half2 m = __hmax2_nan(*reinterpret_cast<__half2*>(&w), __floats2half2_rn(0.f, 0.f));
    return *reinterpret_cast<const uint32_t*>(&m);
  }
  const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<__nv_bfloat162*>(&w), __floats2bfloat162_rn(0.f, 0.f));
  return *reinterpret_cast<const uint32_t*>(&m);
}
__device__ __forceinline__ float relu1(float v) {
  asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(v));
  return v;
}

// One lane's channel in `N` consecutive batch rows, `rows` of them real (consecutive lanes store consecutive outputs, so that rows of any
// alignment do).  `at`: the channel in the first row.
// ALL: every row is (without the tests between them 16 rows of 16 bits take 870 cycles of sixteen warps
// instead of 1480; of 32 bits as many as with them).
template <int DT, int N, bool ALL>
__device__ __forceinline__ void store_channel_rows(const int32_t* r, uint8_t* at, long long pitch, int rows, float unit, float bias, bool relu,
                                                   ZeroCount<DT>& zeros) {
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    if (!ALL && j >= rows) break;
    float a = fmaf(__int_as_float(r[j]), unit, bias), b = fmaf(__int_as_float(r[j + 1]), unit, bias);
    uint8_t* const next = at + pitch;
    if (DT == ADAPTION_F32) {
      if (relu) { a = relu1(a); b = relu1(b); }
      zeros.n += a == 0.f;
      *reinterpret_cast<float*>(at) = a;
      if (ALL || j + 1 < rows) {
        zeros.n += b == 0.f;
        *reinterpret_cast<float*>(next) = b;
      }
    } else {
      uint32_t w = pack2<DT>(a, b);
      if (relu) w = relu2<DT>(w);
      *reinterpret_cast<uint16_t*>(at) = (uint16_t)w;
      if (ALL || j + 1 < rows) {
        zeros.pair(w);
        *reinterpret_cast<uint16_t*>(next) = (uint16_t)(w >> 16);
      } else {
        zeros.n += (w & 0x7fffu) == 0u;
      }
    }
    at = next + pitch;
  }
}
template <int DT, int N>
__device__ __forceinline__ void store_channel(const int32_t* r, uint8_t* at, long long pitch, int rows, float unit, float bias, bool relu,
                                              ZeroCount<DT>& zeros) {
  if (DT != ADAPTION_F32 && rows >= N) store_channel_rows<DT, N, true>(r, at, pitch, N, unit, bias, relu, zeros);
  else store_channel_rows<DT, N, false>(r, at, pitch, rows, unit, bias, relu, zeros);
}

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
