// Inner product of microscaled 4-bit operands with many rows (adaption_fp4_ip_fwd): a persistent kernel, one pair of
// CTAs on two SMs per tile of 256 output channels x 256 batch rows.
//
// The product is fp4_gemm.cu's; what differs is what bounds it.  A pair instruction (cta_group::2) computes 256 x 256 x 64 from
// each CTA's own 128 rows of weights and half of the batch rows, so a k-block of 256 elements costs each SM 32 KB of codes
// (and 3 or 6 KB of scales) for 512 cycles of the tensor core, at most 76 bytes a cycle; 128 x 256 tiles of single CTAs
// need 54 KB.
//
// TMEM: an accumulator has 256 columns, two have all 512, and the scales of two k-blocks take 48 (blocks of 32) or 96.  So the second
// accumulator begins in the last 48 or 96 columns of the first.  The epilogue empties the shared columns of a tile first and hands
// them back; the next tile's MMAs start then, while it works through the others.
//
// Scales are copied to TMEM two k-blocks ahead at most: the issuing warp waits until the MMAs of the k-block before the last
// have retired (their release of the ring's stage says so) before it overwrites the columns they read.
#include <cuda.h>

#include <cstring>

#include "fp4_mma.cuh"
#include "knobs.cuh"
#include "tensor_maps.cuh"

namespace adaption {

int num_sms();

namespace {

constexpr int kTile = 256;                 // channels and rows of a pair's tile
constexpr int kMaxStages = 6;
constexpr int kThreads = 384;              // warp 0: copies; 1: MMA (leader); 4-11: epilogue
constexpr int kFirstEpiWarp = 4, kEpiWarps = 8;
constexpr uint32_t kTmemCols = 512;

// shared columns of the two accumulators = columns of the scales of two k-blocks
__host__ __device__ constexpr int scale_columns(int block) { return groups_of(block) * 4 * 3; }
__host__ __device__ constexpr int shared_columns(int block) { return 2 * scale_columns(block); }
__host__ __device__ constexpr uint32_t sf_bytes(int block) { return (uint32_t)groups_of(block) * kFp4TileBytes; }
__host__ __device__ constexpr uint32_t stage_bytes(int block) { return 2 * kABytes + 3 * sf_bytes(block); }

struct PairParams {
  int O, B;
  int tiles_o, tiles;
  int num_kb, steps_last, groups_last;
  int stages;
  float unit_x, unit_w;
  const float* bias;
  int relu;
  void* y;
  long long y_stride;
  adaption_stats* stats;
  unsigned long long timeout_ns;
  int stall_at;
};

struct PairCtrl {
  unsigned long long full[kMaxStages];     // the leader's: bytes of both CTAs
  unsigned long long empty[kMaxStages];    // in both CTAs
  unsigned long long acc_full[2];          // in both CTAs: a tile's sums are complete
  unsigned long long acc_free;             // the leader's: the shared columns of a tile have been read
  unsigned long long drain;
  uint32_t tmem_base;
  volatile uint32_t abort;
};

__device__ __noinline__ bool pair_wait_slow(uint32_t bar, uint32_t parity, PairCtrl* ctrl, const PairParams& p) {
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
__device__ __forceinline__ bool pair_wait(uint32_t bar, uint32_t parity, PairCtrl* ctrl, const PairParams& p) {
  if (mbar_try_wait(bar, parity)) return true;
  return pair_wait_slow(bar, parity, ctrl, p);
}

// 8 * N consecutive columns
template <int N>
__device__ __forceinline__ void load_columns(uint32_t taddr, int32_t (&r)[N][8]) {
#pragma unroll
  for (int i = 0; i < N; ++i) tmem_ld8(taddr + 8u * i, r[i]);
  tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < N; ++i) pin_after_wait(r[i]);
}
// ... finished and stored: column j is batch row b + j, this lane is channel o
template <int DT, int N>
__device__ __forceinline__ void store_columns(const PairParams& p, const int32_t (&r)[N][8], int b, int o, float bias,
                                              uint32_t& zeros) {
  if (o >= p.O) return;
  const int n = min(8 * N, p.B - b);
  long long at = (long long)b * p.y_stride + o;
#pragma unroll
  for (int j = 0; j < 8 * N; ++j) {
    if (j >= n) break;
    float v = fmaf(__int_as_float(r[j >> 3][j & 7]) * p.unit_x, p.unit_w, bias);
    if (p.relu) v = v < 0.f ? 0.f : v;
    zeros += v == 0.f;
    store_output<DT>(p.y, at, v);
    at += p.y_stride;
  }
}
template <int DT, int N>
__device__ __forceinline__ void finish_columns(const PairParams& p, uint32_t taddr, int b, int o, float bias, uint32_t& zeros) {
  int32_t r[N][8];
  load_columns<N>(taddr, r);
  store_columns<DT, N>(p, r, b, o, bias, zeros);
}

template <int BLOCK, int DT>
__global__ void __launch_bounds__(kThreads, 1)
fp4_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_sfa, const __grid_constant__ CUtensorMap map_sfb, const PairParams p) {
  constexpr int kGroups = groups_of(BLOCK);
  constexpr int kShared = shared_columns(BLOCK);                 // 48 or 96
  constexpr uint32_t kSecond = kTile - kShared;                  // first column of the second accumulator
  constexpr uint32_t kScales = kTmemCols - kShared;              // ... of the scales
  constexpr uint32_t kStage = stage_bytes(BLOCK);
  extern __shared__ uint8_t smem_raw[];
  __shared__ PairCtrl ctrl;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int worker = (int)(blockIdx.x >> 1), workers = (int)(gridDim.x >> 1);

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&ctrl.full[s]), 1);
      mbar_init(smem_u32(&ctrl.empty[s]), 1);
    }
    mbar_init(smem_u32(&ctrl.acc_full[0]), 1);
    mbar_init(smem_u32(&ctrl.acc_full[1]), 1);
    mbar_init(smem_u32(&ctrl.acc_free), 2 * kEpiWarps);
    mbar_init(smem_u32(&ctrl.drain), 1);
    ctrl.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    tmem_alloc<true>(smem_u32(&ctrl.tmem_base), kTmemCols);
    tmem_relinquish<true>();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();          // the peer's barriers exist before anything signals them
  tc_fence_after();
  const uint32_t tmem = ctrl.tmem_base;

  pdl_wait();
  pdl_launch_dependents();

  bool ok = true;
  if (warp == 0) {
    // ---- copies: this CTA's 128 channels and its half of the batch rows, their scales; reported to the leader's barrier
    uint32_t it = 0, ph = 0;
    int s = 0;
    for (int t = worker; ok && t < p.tiles; t += workers) {
      const int to = t % p.tiles_o, tb = t / p.tiles_o;
      for (int kb = 0; kb < p.num_kb; ++kb) {
        if ((int)it == p.stall_at) { ok = false; break; }
        ok = __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.empty[s]), ph ^ 1u, &ctrl, p));
        if (!ok) break;
        if (elect_one()) {
          const uint32_t own = smem_u32(&ctrl.full[s]), dst = ring + (uint32_t)s * kStage;
          if (rank == 0) mbar_expect_tx(own, 2u * kStage);
          const uint32_t full = mapa_rank(own, 0);
          const int words = kb * kGroups * (kFp4TileBytes / 8);
          tma_load_2d<true>(dst, &map_a, full, kb * kBlockBytes, to * kTile + (int)rank * kRows);
          tma_load_2d<true>(dst + kABytes, &map_b, full, kb * kBlockBytes, tb * kTile + (int)rank * kRows);
          tma_load_2d<true>(dst + 2 * kABytes, &map_sfa, full, words, to * 2 + (int)rank);
          tma_load_2d<true>(dst + 2 * kABytes + sf_bytes(BLOCK), &map_sfb, full, words, tb * 2);
        }
        __syncwarp();
        ++it;
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
    }
    if ((!ok || ctrl.abort) && lane == 0) {
      // gave up: let the copies in flight land.  (Their bytes are counted on the leader's barriers, so the follower just waits.)
      const uint32_t n = it < (uint32_t)p.stages ? it : (uint32_t)p.stages;
      const unsigned long long t0 = global_ns();
      for (uint32_t j = it - n; j < it; ++j) {
        while (global_ns() - t0 < 5000000ull &&
               (rank != 0 || !mbar_try_wait(smem_u32(&ctrl.full[j % (uint32_t)p.stages]), (j / (uint32_t)p.stages) & 1u))) {
        }
      }
    }
    __syncwarp();
  } else if (warp == 1 && rank == 0) {
    // ---- MMA issue
    const uint32_t id = make_idesc_fp4(BLOCK, kTile, kTile);
    const uint32_t dhi = smem_desc_hi(8u * kBlockBytes, 2u);          // 128-byte swizzle
    const uint32_t shi = smem_desc_hi(128u, 0u);                       // scale tiles: rows of 16 bytes, groups of 8 rows
    uint32_t it = 0, ph = 0, prev_ph = 0;
    int s = 0, prev = -1, prev2 = -1;                                  // stages of the last two k-blocks
    uint32_t prev2_ph = 0;
    int local = 0;
    for (int t = worker; ok && t < p.tiles; t += workers, ++local) {
      if (local > 0) {
        ok = __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.acc_free), (uint32_t)(local - 1) & 1u, &ctrl, p));
        if (!ok) break;
        tc_fence_after();
      }
      const uint32_t d = tmem + ((local & 1) ? kSecond : 0u);
      for (int kb = 0; kb < p.num_kb; ++kb) {
        ok = __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.full[s]), ph, &ctrl, p));
        if (ok && prev2 >= 0)
          ok = __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.empty[prev2]), prev2_ph, &ctrl, p));
        if (!ok) break;
        tc_fence_after();
        const uint32_t a = smem_desc_lo(ring) + (uint32_t)s * (kStage >> 4), b = a + (kABytes >> 4);
        const uint32_t sf = ((ring + (uint32_t)s * kStage + 2 * kABytes) >> 4) & 0x3FFFu;
        const uint32_t ta = tmem + kScales + (it & 1u) * (uint32_t)scale_columns(BLOCK), tb = ta + 4u * kGroups;
        const bool last = kb == p.num_kb - 1;
        const int steps = last ? p.steps_last : kBlockElems / kStepElems, groups = last ? p.groups_last : kGroups;
        if (elect_one()) {
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            if (g < groups) {
              scales_to_tmem<true>(ta + 4u * g, sf + 32u * g, shi);
              scales_to_tmem<true>(tb + 8u * g, sf + 32u * (kGroups + g), shi);
              scales_to_tmem<true>(tb + 8u * g + 4u, sf + 32u * (2 * kGroups + g), shi);
            }
          }
#pragma unroll
          for (int k = 0; k < kBlockElems / kStepElems; ++k) {
            const uint32_t g = BLOCK == 32 ? (uint32_t)k >> 1 : (uint32_t)k;
            if (k < steps)
              mma_fp4<BLOCK, true>(d, a + 2u * k, b + 2u * k, dhi, BLOCK == 32 ? id | scale_half(k & 1) : id, ta + 4u * g,
                                   tb + 8u * g, (kb > 0 || k > 0) ? 1u : 0u);
          }
          tc_commit<true>(smem_u32(&ctrl.empty[s]));
        }
        __syncwarp();
        prev2 = prev; prev2_ph = prev_ph;
        prev = s; prev_ph = ph;
        ++it;
        if (++s == p.stages) { s = 0; ph ^= 1u; }
      }
      if (ok && elect_one()) tc_commit<true>(smem_u32(&ctrl.acc_full[local & 1]));
      __syncwarp();
    }
    if ((!ok || ctrl.abort) && lane == 0) {
      // no MMA may still read shared memory or write TMEM when the CTAs tear down
      tc_commit<true>(smem_u32(&ctrl.drain));
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(smem_u32(&ctrl.drain), 0) && global_ns() - t0 < 50000000ull) {
      }
    }
    __syncwarp();
  } else if (warp >= kFirstEpiWarp) {
    // ---- epilogue: two warps per lane quarter, each half of the columns
    const int quarter = warp & 3, half = (warp - kFirstEpiWarp) >> 2;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    uint32_t zeros = 0;
    int local = 0;
    for (int t = worker; t < p.tiles; t += workers, ++local) {
      const int o = (t % p.tiles_o) * kTile + (int)rank * kRows + quarter * 32 + lane, b0 = (t / p.tiles_o) * kTile;
      const float bias = p.bias != nullptr && o < p.O ? __ldg(p.bias + o) : 0.f;
      ok = __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.acc_full[local & 1]), (uint32_t)(local >> 1) & 1u, &ctrl, p));
      if (!ok) break;
      tc_fence_after();
      // the columns that the next tile's accumulator shares first: the last ones of the first accumulator, the first ones
      // of the second
      constexpr int kMine = kShared / 2, kRest = (kTile - kShared) / 2;          // 24 or 48; 104 or 80
      const uint32_t acc = lanes + ((local & 1) ? kSecond : 0u);
      const int first = (local & 1) ? 0 : (int)kSecond, rest = (local & 1) ? kShared : 0;
      {
        int32_t r[kMine / 8][8];
        const int c = first + half * kMine;
        load_columns<kMine / 8>(acc + (uint32_t)c, r);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(mapa_rank(smem_u32(&ctrl.acc_free), 0));
        store_columns<DT, kMine / 8>(p, r, b0 + c, o, bias, zeros);
      }
      int c = rest + half * kRest;
      if (BLOCK == 32) {
        finish_columns<DT, 5>(p, acc + (uint32_t)c, b0 + c, o, bias, zeros);
        finish_columns<DT, 4>(p, acc + (uint32_t)(c + 40), b0 + c + 40, o, bias, zeros);
        finish_columns<DT, 4>(p, acc + (uint32_t)(c + 72), b0 + c + 72, o, bias, zeros);
      } else {
        finish_columns<DT, 5>(p, acc + (uint32_t)c, b0 + c, o, bias, zeros);
        finish_columns<DT, 5>(p, acc + (uint32_t)(c + 40), b0 + c + 40, o, bias, zeros);
      }
    }
    __syncwarp();
    zeros = __reduce_add_sync(0xffffffffu, zeros);
    if (lane == 0 && zeros) atomicAdd((unsigned long long*)&p.stats->zeros, (unsigned long long)zeros);
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync_all();          // neither CTA leaves (or frees TMEM) while the other may still signal it
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc<true>(tmem, kTmemCols);
  }
}

template <int BLOCK, int DT>
int launch_pair(const CUtensorMap* maps, const PairParams& p, int grid, cudaStream_t stream) {
  const size_t smem = (size_t)p.stages * stage_bytes(BLOCK) + 1024;
  static std::atomic<uint64_t> prepared{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_failure(e, "fp4_pair_kernel device");
  if (dev >= 64 || !((prepared.load(std::memory_order_acquire) >> dev) & 1)) {
    e = cudaFuncSetAttribute(fp4_pair_kernel<BLOCK, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)(kMaxStages * stage_bytes(BLOCK) + 1024 < 226 * 1024 ? kMaxStages * stage_bytes(BLOCK) + 1024 : 226 * 1024));
    if (e != cudaSuccess) return cuda_failure(e, "fp4_pair_kernel attribute");
    if (dev < 64) prepared.fetch_or((uint64_t)1 << dev, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  count_launch();
  e = cudaLaunchKernelEx(&cfg, fp4_pair_kernel<BLOCK, DT>, maps[0], maps[1], maps[2], maps[3], p);
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return cuda_failure(e, "fp4_pair_kernel launch");
  }
  return ADAPTION_OK;
}

template <int BLOCK>
int launch_pair(const CUtensorMap* maps, const PairParams& p, int dtype, int grid, cudaStream_t stream) {
  if (dtype == ADAPTION_F32) return launch_pair<BLOCK, ADAPTION_F32>(maps, p, grid, stream);
  if (dtype == ADAPTION_F16) return launch_pair<BLOCK, ADAPTION_F16>(maps, p, grid, stream);
  return launch_pair<BLOCK, ADAPTION_BF16>(maps, p, grid, stream);
}

}  // namespace

bool fp4_pair_preferred(const Fp4Problem& g) {
  const int mode = knob(kPair);
  if (mode >= 0) return mode != 0;
  const int64_t tiles = ((g.O + kTile - 1) / kTile) * ((g.B + kTile - 1) / kTile);
  return g.B > 128 && tiles >= num_sms() / 2;
}

int launch_fp4_pair(const Fp4Problem& g) {
  const int block = g.w.block;
  PairParams p;
  std::memset(&p, 0, sizeof(p));
  p.O = (int)g.O;
  p.B = (int)g.B;
  p.tiles_o = (p.O + kTile - 1) / kTile;
  const int64_t tiles = (int64_t)p.tiles_o * ((p.B + kTile - 1) / kTile);
  if (tiles > 0x3fffffff) return ADAPTION_ERR_UNSUPPORTED;
  p.tiles = (int)tiles;
  p.num_kb = (int)((g.K + kBlockElems - 1) / kBlockElems);
  const int64_t groups = fp4_groups(g.K, block);
  const int k_last = (int)(g.K - (int64_t)(p.num_kb - 1) * kBlockElems);
  p.steps_last = (k_last + kStepElems - 1) / kStepElems;
  p.groups_last = (int)(groups - (int64_t)(p.num_kb - 1) * groups_of(block));
  p.stages = (int)((226 * 1024 - 1024) / stage_bytes(block));
  if (p.stages > kMaxStages) p.stages = kMaxStages;
  p.unit_x = pow2_float(g.x.exp);
  p.unit_w = pow2_float(g.w.exp);
  p.bias = g.bias;
  p.relu = g.relu ? 1 : 0;
  p.y = g.y.data;
  p.y_stride = g.y.stride;
  p.stats = g.stats;
  p.timeout_ns = wait_limit_ns();
  p.stall_at = knob(kStallAt);
  if (!load_tensor_map_encoders()) return ADAPTION_ERR_CUDA;
  CUtensorMap maps[4];
  const uint64_t bytes = (uint64_t)(g.K + 1) / 2;
  bool ok = encode_tiled_2d(&maps[0], g.w.codes, bytes, (uint64_t)p.O, (uint64_t)g.w.c_stride / 2, kBlockBytes, kRows,
                            CU_TENSOR_MAP_SWIZZLE_128B) &&
            encode_tiled_2d(&maps[1], g.x.codes, bytes, (uint64_t)p.B, (uint64_t)g.x.c_stride / 2, kBlockBytes, kRows,
                            CU_TENSOR_MAP_SWIZZLE_128B);
  // scale planes: one row per row of tiles, in words of 8 bytes; what lies behind the last tile arrives as zeros
  for (int i = 0; ok && i < 2; ++i) {
    const uint64_t dims[2] = {(uint64_t)groups * (kFp4TileBytes / 8), (uint64_t)(((i ? p.B : p.O) + kRows - 1) / kRows)};
    const uint64_t strides[1] = {(uint64_t)groups * kFp4TileBytes};
    const uint32_t box[2] = {(uint32_t)(groups_of(block) * (kFp4TileBytes / 8)), i ? 2u : 1u};
    ok = encode_tiled_words(&maps[2 + i], i ? g.x.scales : g.w.scales, 2, dims, strides, box);
  }
  if (!ok) return ADAPTION_ERR_CUDA;
  int pairs = num_sms() / 2;
  if (pairs > p.tiles) pairs = p.tiles;
  return block == 32 ? launch_pair<32>(maps, p, g.y.dtype, 2 * pairs, g.stream) : launch_pair<16>(maps, p, g.y.dtype, 2 * pairs, g.stream);
}

}  // namespace adaption
