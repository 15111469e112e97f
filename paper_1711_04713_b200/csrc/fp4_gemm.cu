// Inner product of microscaled 4-bit operands (adaption_fp4_ip_fwd) on the tensor cores.
//
//   y[b][o] = act(2^(ex + ew) sum over blocks of sx sw (sum of code products) + bias[o])
//
// tcgen05.mma with block scales (kind mxf4 for blocks of 32, mxf4nvf4 for blocks of 16) takes 64 elements of K per
// instruction, multiplies each block's sum by the two scales and adds in 32-bit floating point.  The weights are the 128-row
// operand A and the batch is the column operand B, so that one row of activations costs 16 columns instead of 128
// rows; an accumulator lane is then one output channel, and consecutive lanes store consecutive outputs, whatever the
// alignment of y's rows.
//
// A k-block is 128 bytes of codes per row (256 elements), copied by TMA with the 128-byte swizzle, and the scale tiles of the same
// elements (two of 512 bytes per 128 rows for blocks of 32, four for blocks of 16), which lie one after the other in memory and are copied as one
// run.  The issuing thread moves them to TMEM (tcgen05.cp, 32 rows x 16 bytes repeated in the four lane quarters: what
// the MMA reads) into columns that belong to the ring's stage: they are written again only after the MMAs that read
// them have released the stage.
#include <cuda.h>

#include <cstring>

#include "fp4_mma.cuh"
#include "knobs.cuh"
#include "tensor_maps.cuh"

namespace adaption {

int num_sms();

namespace {

constexpr int kMaxStages = 10;
constexpr int kThreads = 256;              // warp 0: copies; 1: MMA; all of them: the epilogue

struct FpParams {
  int O, B;                     // output channels, batch rows
  int S;                        // CTAs per tile (cluster size)
  int tiles_o;
  int BN;                       // columns of a tile: multiple of 16, of 128 where there are several column tiles
  int chunks_b;                 // scale tiles that cover them
  int num_kb, kb_per_split;
  int steps_last;               // MMAs of the last k-block
  int groups_last;              // scale tiles of the last k-block and 128 rows
  int64_t groups;               // ... of all
  int scale_tiles_b;            // rows of scale tiles of the batch
  int stages;
  uint32_t b_bytes, stage_bytes, tmem_cols, sf_col;
  const uint8_t* sfa;
  const uint8_t* sfb;
  float unit;                   // 2^(sum of the operands' exponents)
  const float* bias;
  int relu;
  void* y;
  long long y_stride;
  int dtype;
  adaption_stats* stats;
  unsigned long long timeout_ns;
  int stall_at;                 // test aid, see adaption_debug_set
};

struct FpCtrl {
  unsigned long long full[kMaxStages];
  unsigned long long empty[kMaxStages];
  unsigned long long done;
  uint32_t tmem_base;
  volatile uint32_t abort;
};

__device__ __noinline__ bool fp_wait_slow(uint32_t bar, uint32_t parity, FpCtrl* ctrl, const FpParams& p) {
  const unsigned long long t0 = global_ns();
  while (!mbar_try_wait_suspend(bar, parity, 1000u)) {
    if (ctrl->abort) return false;
    if (global_ns() - t0 > p.timeout_ns) {
      ctrl->abort = 1;
      atomicExch(&p.stats->status, (int)ADAPTION_ERR_TIMEOUT);
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool fp_wait(uint32_t bar, uint32_t parity, FpCtrl* ctrl, const FpParams& p) {
  if (mbar_try_wait(bar, parity)) return true;
  return fp_wait_slow(bar, parity, ctrl, p);
}

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

// `n` (at most 4) consecutive outputs; returns how many are stored as 0
__device__ __forceinline__ uint32_t store_outputs(const FpParams& p, long long at, const float (&v)[4], int n) {
  uint32_t zeros = 0;
  if (p.dtype == ADAPTION_F32) {
    float* y = reinterpret_cast<float*>(p.y) + at;
#pragma unroll
    for (int k = 0; k < 4; ++k) zeros += k < n && v[k] == 0.f;
    if (n == 4 && (reinterpret_cast<uintptr_t>(y) & 15) == 0) {
      *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < n) y[k] = v[k];
    }
    return zeros;
  }
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) w[k] = p.dtype == ADAPTION_F16 ? pack2<ADAPTION_F16>(v[2 * k], v[2 * k + 1]) : pack2<ADAPTION_BF16>(v[2 * k], v[2 * k + 1]);
  uint16_t* y = reinterpret_cast<uint16_t*>(p.y) + at;
#pragma unroll
  for (int k = 0; k < 4; ++k) zeros += k < n && ((w[k >> 1] >> (16 * (k & 1))) & 0x7fffu) == 0u;
  if (n == 4 && (reinterpret_cast<uintptr_t>(y) & 7) == 0) {
    *reinterpret_cast<uint2*>(y) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < n) y[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
  }
  return zeros;
}

// One cluster of S CTAs per tile of 128 channels x BN batch rows: each CTA reduces its share of the k-blocks, leaves
// its partial sums in its shared memory, and finishes the columns that fall to it from all CTAs' sums in rank order.
template <int BLOCK>
__global__ void __launch_bounds__(kThreads, 1)
fp4_cluster_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const FpParams p) {
  constexpr int kGroups = groups_of(BLOCK);
  extern __shared__ uint8_t smem_raw[];
  __shared__ FpCtrl ctrl;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t rank = p.S > 1 ? cluster_ctarank() : 0u;
  const int tile = (int)blockIdx.x / p.S;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&ctrl.full[s]), 1);
      mbar_init(smem_u32(&ctrl.empty[s]), 1);
    }
    mbar_init(smem_u32(&ctrl.done), 1);
    ctrl.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc<false>(smem_u32(&ctrl.tmem_base), p.tmem_cols);
    tmem_relinquish<false>();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctrl.tmem_base;

  const int to = tile % p.tiles_o, tb = tile / p.tiles_o;
  const int o0 = to * kRows, b0 = tb * p.BN;
  const int kb_begin = (int)rank * p.kb_per_split;
  const int kb_end = min(p.num_kb, kb_begin + p.kb_per_split);

  pdl_wait();
  pdl_launch_dependents();

  bool ok = true;
  if (warp == 0) {
    const int chunks = min(p.chunks_b, p.scale_tiles_b - b0 / kRows);      // scale tiles that exist
    const uint8_t* const sfa = p.sfa + (int64_t)to * p.groups * kFp4TileBytes;
    const uint8_t* const sfb = p.sfb + (int64_t)(b0 / kRows) * p.groups * kFp4TileBytes;
    int s = 0, issued = 0;
    uint32_t ph = 0;
    for (int kb = kb_begin; kb < kb_end; ++kb) {
      if (issued == p.stall_at) break;
      ok = __all_sync(0xffffffffu, fp_wait(smem_u32(&ctrl.empty[s]), ph ^ 1u, &ctrl, p));
      if (!ok) break;
      if (elect_one()) {
        const uint32_t full = smem_u32(&ctrl.full[s]), dst = ring + (uint32_t)s * p.stage_bytes;
        const uint32_t sf = (uint32_t)(kb == p.num_kb - 1 ? p.groups_last : kGroups) * kFp4TileBytes;
        mbar_expect_tx(full, kABytes + p.b_bytes + sf * (uint32_t)(1 + chunks));
        tma_load_2d<false>(dst, &map_a, full, kb * kBlockBytes, o0);
        tma_load_2d<false>(dst + kABytes, &map_b, full, kb * kBlockBytes, b0);
        const uint32_t at = dst + kABytes + p.b_bytes;
        const int64_t src = (int64_t)kb * kGroups * kFp4TileBytes;
        bulk_load(at, sfa + src, sf, full);
        for (int c = 0; c < chunks; ++c)
          bulk_load(at + (uint32_t)(1 + c) * (kGroups * kFp4TileBytes), sfb + (int64_t)c * p.groups * kFp4TileBytes + src, sf, full);
      }
      __syncwarp();
      ++issued;
      if (++s == p.stages) { s = 0; ph ^= 1u; }
    }
    // the ring is given another use only once the MMAs (or the issuing warp, giving up) are through with it
    if (!fp_wait(smem_u32(&ctrl.done), 0, &ctrl, p)) ok = false;
    if ((!ok || ctrl.abort) && lane == 0) {
      // gave up: let the copies in flight land
      const int n = issued < p.stages ? issued : p.stages;
      for (int j = issued - n; j < issued; ++j) {
        const unsigned long long t0 = global_ns();
        while (!mbar_try_wait(smem_u32(&ctrl.full[j % p.stages]), (uint32_t)(j / p.stages) & 1u) &&
               global_ns() - t0 < 5000000ull) {
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t issue = elect_one() ? 1u : 0u;
    const uint32_t id = make_idesc_fp4(BLOCK, p.BN, kRows);
    const uint32_t dhi = smem_desc_hi(8u * kBlockBytes, 2u);          // 128-byte swizzle
    const uint32_t shi = smem_desc_hi(128u, 0u);                       // scale tiles: rows of 16 bytes, groups of 8 rows
    const uint32_t cols_b = 4u * (uint32_t)p.chunks_b;
    const uint32_t slot = (uint32_t)kGroups * (4u + cols_b);
    int s = 0;
    uint32_t ph = 0;
    for (int kb = kb_begin; kb < kb_end; ++kb) {
      ok = __all_sync(0xffffffffu, fp_wait(smem_u32(&ctrl.full[s]), ph, &ctrl, p));
      if (!ok) break;
      tc_fence_after();
      const bool last = kb == p.num_kb - 1;
      const int steps = last ? p.steps_last : kBlockElems / kStepElems, groups = last ? p.groups_last : kGroups;
      const uint32_t a = smem_desc_lo(ring) + (uint32_t)s * (p.stage_bytes >> 4), b = a + (kABytes >> 4);
      const uint32_t sf = ((ring + (uint32_t)s * p.stage_bytes + kABytes + p.b_bytes) >> 4) & 0x3FFFu;
      const uint32_t ta = tmem + p.sf_col + (uint32_t)s * slot, tbx = ta + 4u * kGroups;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        if (g < groups) {
          scales_to_tmem<false>(issue, ta + 4u * g, sf + 32u * g, shi);
          scales_to_tmem<false>(issue, tbx + cols_b * g, sf + 32u * (uint32_t)(kGroups + g), shi);
          if (p.chunks_b > 1) scales_to_tmem<false>(issue, tbx + cols_b * g + 4u, sf + 32u * (uint32_t)(2 * kGroups + g), shi);
        }
      }
#pragma unroll
      for (int k = 0; k < kBlockElems / kStepElems; ++k) {
        const uint32_t g = BLOCK == 32 ? (uint32_t)k >> 1 : (uint32_t)k;
        if (k < steps)
          mma_fp4<BLOCK, false>(issue, tmem, a + 2u * k, b + 2u * k, dhi, BLOCK == 32 ? id | scale_half(k & 1) : id, ta + 4u * g,
                                tbx + cols_b * g, (kb > kb_begin || k > 0) ? 1u : 0u);
      }
      tc_commit_if<false>(issue, smem_u32(&ctrl.empty[s]));
      if (++s == p.stages) { s = 0; ph ^= 1u; }
    }
    if (elect_one()) tc_commit<false>(smem_u32(&ctrl.done));
    __syncwarp();
    if (!ok || ctrl.abort) {
      // no MMA may still read shared memory when the ring is given another use
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(smem_u32(&ctrl.done), 0) && global_ns() - t0 < 50000000ull) {
      }
    }
  }
  __syncwarp();
  __syncthreads();
  const int cols = min(p.BN, p.B - b0);
  // partial sums to shared memory: [column][128 channels]
  float* const part = reinterpret_cast<float*>(smem_raw + (ring - smem_u32(smem_raw)));
  {
    tc_fence_after();
    const int quarter = warp & 3, row = quarter * 32 + lane;
    for (int c = 8 * (warp >> 2); c < cols; c += 8 * (kThreads / 128)) {
      int32_t a[8];
      tmem_ld8(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)c, a);
      tmem_ld_wait();
      pin_after_wait(a);
      // (a CTA without k-blocks has no sums: its accumulator was never written)
#pragma unroll
      for (int j = 0; j < 8; ++j) part[(c + j) * kRows + row] = kb_begin < kb_end ? __int_as_float(a[j]) : 0.f;
    }
    tc_fence_before();
  }
  if (p.S > 1) cluster_sync_all();
  else __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc<false>(tmem, p.tmem_cols);
  }
  uint32_t zeros = 0;
  if (!ctrl.abort) {
    const uint32_t base = smem_u32(part);
    for (int c = (int)rank + p.S * warp; c < cols; c += p.S * (kThreads / 32)) {
      const uint32_t at = base + (uint32_t)(c * kRows + 4 * lane) * 4u;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      for (int r = 0; r < p.S; ++r) {
        const float4 t = p.S > 1 ? ld_cluster_f4(mapa_rank(at, (uint32_t)r))
                                 : *reinterpret_cast<const float4*>(part + c * kRows + 4 * lane);
        v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
      }
      const int o = o0 + 4 * lane, n = min(4, p.O - o);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = fmaf(v[k], p.unit, p.bias != nullptr && k < n ? __ldg(p.bias + o + k) : 0.f);
        if (p.relu) v[k] = v[k] < 0.f ? 0.f : v[k];
      }
      if (n > 0) zeros += store_outputs(p, (long long)(b0 + c) * p.y_stride + o, v, n);
    }
  }
  __syncwarp();
  zeros = __reduce_add_sync(0xffffffffu, zeros);
  if (lane == 0 && zeros) atomicAdd((unsigned long long*)&p.stats->zeros, (unsigned long long)zeros);
  if (p.S > 1) cluster_sync_all();        // (peers may still read this CTA's sums)
}

constexpr size_t kSmemLimit = 227 * 1024 - 512;      // less the control block

template <int BLOCK>
int launch_cluster_fp4(const CUtensorMap& ma, const CUtensorMap& mb, const FpParams& p, int grid, size_t smem, cudaStream_t stream) {
  static std::atomic<uint64_t> prepared{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_failure(e, "fp4_cluster_kernel device");
  if (dev >= 64 || !((prepared.load(std::memory_order_acquire) >> dev) & 1)) {
    e = cudaFuncSetAttribute(fp4_cluster_kernel<BLOCK>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemLimit);
    if (e != cudaSuccess) return cuda_failure(e, "fp4_cluster_kernel attribute");
    if (dev < 64) prepared.fetch_or((uint64_t)1 << dev, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (p.S > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)p.S;
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (pdl_enabled()) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = n ? attr : nullptr;
  cfg.numAttrs = (unsigned)n;
  count_launch();
  e = cudaLaunchKernelEx(&cfg, fp4_cluster_kernel<BLOCK>, ma, mb, p);
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return cuda_failure(e, "fp4_cluster_kernel launch");
  }
  return ADAPTION_OK;
}

}  // namespace

static int launch_fp4_cluster(const Fp4Problem& g) {
  const int block = g.w.block, kgroups = groups_of(block);
  FpParams p;
  std::memset(&p, 0, sizeof(p));
  p.O = (int)g.O;
  p.B = (int)g.B;
  p.tiles_o = (p.O + kRows - 1) / kRows;
  p.BN = p.B <= 256 ? (p.B + 15) / 16 * 16 : 256;
  const int tiles_b = (p.B + p.BN - 1) / p.BN;
  p.chunks_b = (p.BN + kRows - 1) / kRows;
  p.num_kb = (int)((g.K + kBlockElems - 1) / kBlockElems);
  const int k_last = (int)(g.K - (int64_t)(p.num_kb - 1) * kBlockElems);
  p.steps_last = (k_last + kStepElems - 1) / kStepElems;
  p.groups = fp4_groups(g.K, block);
  p.groups_last = (int)(p.groups - (int64_t)(p.num_kb - 1) * kgroups);
  p.scale_tiles_b = (p.B + kRows - 1) / kRows;
  const int64_t tiles = (int64_t)p.tiles_o * tiles_b;
  p.S = 1;
  while (p.S < 8 && tiles * p.S * 2 <= num_sms() && p.num_kb >= p.S * 2) p.S *= 2;
  p.kb_per_split = (p.num_kb + p.S - 1) / p.S;
  if (tiles * p.S > 0x7fffffff) return ADAPTION_ERR_UNSUPPORTED;
  p.b_bytes = (uint32_t)p.BN * kBlockBytes;
  p.stage_bytes = kABytes + p.b_bytes + (uint32_t)(kgroups * kFp4TileBytes * (1 + p.chunks_b));
  const size_t sums = (size_t)p.BN * kRows * sizeof(float);
  int stages = (int)((kSmemLimit - 1024) / p.stage_bytes);
  if (stages > kMaxStages) stages = kMaxStages;
  if (stages > p.kb_per_split) stages = p.kb_per_split;
  p.sf_col = (uint32_t)(p.BN + 31) / 32 * 32;
  const uint32_t slot = (uint32_t)kgroups * 4u * (uint32_t)(1 + p.chunks_b);
  while (stages > 1 && p.sf_col + (uint32_t)stages * slot > 512u) --stages;
  p.stages = stages;
  p.tmem_cols = 32;
  while (p.tmem_cols < p.sf_col + (uint32_t)stages * slot) p.tmem_cols *= 2;
  size_t smem = (size_t)stages * p.stage_bytes;
  if (smem < sums) smem = sums;
  smem += 1024;
  p.sfa = (const uint8_t*)g.w.scales;
  p.sfb = (const uint8_t*)g.x.scales;
  p.unit = pow2_float(g.x.exp + g.w.exp);
  p.bias = g.bias;
  p.relu = g.relu ? 1 : 0;
  p.y = g.y.data;
  p.y_stride = g.y.stride;
  p.dtype = g.y.dtype;
  p.stats = g.stats;
  p.timeout_ns = wait_limit_ns();
  p.stall_at = knob(kStallAt);
  if (!load_tensor_map_encoders()) return ADAPTION_ERR_CUDA;
  CUtensorMap ma, mb;
  const uint64_t bytes = (uint64_t)(g.K + 1) / 2;
  if (!encode_tiled_2d(&ma, g.w.codes, bytes, (uint64_t)p.O, (uint64_t)g.w.c_stride / 2, kBlockBytes, kRows,
                       CU_TENSOR_MAP_SWIZZLE_128B, true) ||
      !encode_tiled_2d(&mb, g.x.codes, bytes, (uint64_t)p.B, (uint64_t)g.x.c_stride / 2, kBlockBytes, (uint32_t)p.BN,
                       CU_TENSOR_MAP_SWIZZLE_128B))
    return ADAPTION_ERR_CUDA;
  const int grid = (int)(tiles * p.S);
  return block == 32 ? launch_cluster_fp4<32>(ma, mb, p, grid, smem, g.stream)
                     : launch_cluster_fp4<16>(ma, mb, p, grid, smem, g.stream);
}

int fp4_ip_impl(const Fp4Problem& g) {
  return fp4_pair_preferred(g) ? launch_fp4_pair(g) : launch_fp4_cluster(g);
}

}  // namespace adaption
