// Inner product of microscaled 4-bit operands with many rows (adaption_fp4_ip_fwd): a persistent kernel, one pair of
// CTAs on two SMs per tile of 256 output channels x 256 batch rows.
//
// The product is fp4_gemm.cu's; what differs is what bounds it.  A pair instruction (cta_group::2) computes 256 x 256 x 64 from
// each CTA's own 128 rows of weights and half of the batch rows, so a k-block of 256 elements costs each SM 32 KB of codes
// (and 3 or 6 KB of scales) for 512 cycles of the tensor core, at most 76 bytes a cycle; 128 x 256 tiles of single CTAs
// need 54 KB.
//
// TMEM: the accumulator has 256 of the 512 columns, the scales of the k-blocks in the ring have the others, a slot per stage of the
// ring, so that no scale is overwritten before the MMAs that read it have released the stage.  (With slots for two k-blocks the wait
// for that, about 1000 cycles from the last MMA to the first one of the k-block after next, held a k-block at 870 cycles
// instead of 512.)  All sixteen warps of the epilogue load a tile's sums at once, 64 columns each, and hand the accumulator
// back before they work on them: about 700 cycles from a tile's last MMA to the next one's first.  A second accumulator that shares
// half or more of the columns with the first saves none of it.
//
// Outputs leave by bulk-tensor stores from shared memory where their rows are aligned, one block of 4 KB after the other with
// three under way.  The 64 KB of a tile take 3500 cycles of the SM's share of L2's writes in any case; stored by the lanes
// themselves they held up the issuing warp's barrier tests and MMAs for that long (1100 cycles a k-block), as stores issued
// all at once they held up the copies.
//
// Measured: 8192 x 8192 x 8192, blocks of 16, to bf16 190 us (5.8 PFLOP/s) while the GPU is cool, 217 (5.1) when it runs at its power limit,
// where clocks fall to 1.6 GHz; an estimate of MMAs alone is 150 at 1.92 GHz.  Blocks of 32: 181.
#include <cuda.h>

#include <cstring>

#include "fp4_mma.cuh"
#include "knobs.cuh"

namespace adaption {

int num_sms();

namespace {

constexpr int kTile = 256;                 // channels and rows of a pair's tile
constexpr int kStages = 4;
constexpr int kThreads = 640;              // warp 0: copies; 1: MMA (leader); 3: stores; 4-19: epilogue
constexpr int kFirstEpiWarp = 4, kEpiWarps = 16;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kScales = kTile;        // first TMEM column of the scales
constexpr int kWarpCols = kTile / 4;       // columns of an epilogue warp
constexpr uint32_t kStagingBytes = 32 * 128;   // of an epilogue warp: 32 rows of 128 bytes

// TMEM columns of the scales of a k-block
__host__ __device__ constexpr int scale_columns(int block) { return groups_of(block) * 4 * 3; }
__host__ __device__ constexpr uint32_t sf_bytes(int block) { return (uint32_t)groups_of(block) * kFp4TileBytes; }
__host__ __device__ constexpr uint32_t stage_bytes(int block) { return 2 * kABytes + 3 * sf_bytes(block); }
__host__ __device__ constexpr uint32_t smem_bytes(int block) { return kStages * stage_bytes(block) + kEpiWarps * kStagingBytes + 1024; }
static_assert(kScales + kStages * scale_columns(16) <= kTmemCols, "a slot of scales for every stage");
static_assert(smem_bytes(16) <= 225 * 1024, "227 KB, less barriers and biases");

struct PairParams {
  int O, B;
  int tiles_a, tiles;           // tiles along A; all
  int num_kb, steps_last, groups_last;
  float unit;                   // 2^(sum of the operands' exponents)
  const float* bias;
  int relu;
  uint8_t* y;
  long long y_pitch;            // bytes
  int cols16;                   // channels before the last 16-byte boundary of a row
  adaption_stats* stats;
  unsigned long long timeout_ns;
  int stall_at;
};

struct PairCtrl {
  unsigned long long full[kStages];     // the leader's: bytes of both CTAs
  unsigned long long empty[kStages];    // in both CTAs
  unsigned long long acc_full;             // in both CTAs: a tile's sums are complete
  unsigned long long acc_free;             // the leader's: they are in registers
  unsigned long long staged[kEpiWarps];    // an epilogue warp has filled its staging block
  unsigned long long stored[kEpiWarps];    // the block has been read by its store
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

// Lanes are batch rows, columns are channels: 32 of them from channel `c` on, as half a row (16-bit types: half 0 or 1) or a
// whole row of the warp's staging block, in the order of the 128-byte swizzle.  The stores from there end on the row's last 16-byte
// boundary (a store clips at such boundaries only); outputs behind it go to the row `y` at once.
template <int DT>
__device__ __forceinline__ void stage_row(const PairParams& p, const int32_t (&r)[32], uint32_t staging, int half, int lane, int c,
                                          bool real, uint8_t* y, const float* bias, ZeroCount<DT>& zeros) {
  const int n = real ? p.O - c : 0;                    // channels that exist (what does not is clipped by the store)
  const uint32_t row = staging + (uint32_t)lane * 128u, key = (uint32_t)lane & 7u;
#pragma unroll
  for (int i = 0; i < 32; i += 8) {                    // eight channels
    const float4 b0 = *reinterpret_cast<const float4*>(bias + i), b1 = *reinterpret_cast<const float4*>(bias + i + 4);
    float v[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = fmaf(__int_as_float(r[i + j]), p.unit, v[j]);
    if constexpr (DT == ADAPTION_F32) {
      if (p.relu) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = relu1(v[j]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) zeros.n += v[j] == 0.f && i + j < n;
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        st_shared_v4(row + ((((uint32_t)(i + j) >> 2) ^ key) << 4), __float_as_uint(v[j]), __float_as_uint(v[j + 1]),
                     __float_as_uint(v[j + 2]), __float_as_uint(v[j + 3]));
        const int tail = n - i - j;
        if (tail > 0 && tail < 4) {
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (e < tail) reinterpret_cast<float*>(y)[c + i + j + e] = v[j + e];
        }
      }
    } else {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = pack2<DT>(v[2 * j], v[2 * j + 1]);
      if (p.relu) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = relu2<DT>(w[j]);
      }
      if (n >= 32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) zeros.pair(w[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) zeros.n += i + j < n && ((w[j >> 1] >> (16 * (j & 1))) & 0x7fffu) == 0u;
      }
      st_shared_v4(row + (((uint32_t)(4 * half + (i >> 3)) ^ key) << 4), w[0], w[1], w[2], w[3]);
      const int tail = n - i;
      if (tail > 0 && tail < 8) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (e < tail) reinterpret_cast<uint16_t*>(y)[c + i + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

// ROWS: the 128-row operand A is the batch (lanes of the accumulators are batch rows) and the columns are channels; otherwise
// A is the weights.  map_a, map_sfa and so on are of the operand in that place.
template <int BLOCK, int DT, bool ROWS>
__global__ void __launch_bounds__(kThreads, 1)
fp4_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_sfa, const __grid_constant__ CUtensorMap map_sfb,
                const __grid_constant__ CUtensorMap map_y, const PairParams p) {
  constexpr int kGroups = groups_of(BLOCK);
  constexpr uint32_t kStage = stage_bytes(BLOCK);
  extern __shared__ uint8_t smem_raw[];
  __shared__ PairCtrl ctrl;
  __shared__ __align__(16) float bias_tile[ROWS ? kTile : 4];
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int worker = (int)(blockIdx.x >> 1), workers = (int)(gridDim.x >> 1);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(smem_u32(&ctrl.full[s]), 1);
      mbar_init(smem_u32(&ctrl.empty[s]), 1);
    }
    mbar_init(smem_u32(&ctrl.acc_full), 1);
    mbar_init(smem_u32(&ctrl.acc_free), 2 * kEpiWarps);
    for (int w = 0; w < kEpiWarps; ++w) {
      mbar_init(smem_u32(&ctrl.staged[w]), 1);
      mbar_init(smem_u32(&ctrl.stored[w]), 1);
    }
    mbar_init(smem_u32(&ctrl.drain), 1);
    ctrl.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0 && lane < 4) prefetch_map(lane == 0 ? &map_a : (lane == 1 ? &map_b : (lane == 2 ? &map_sfa : &map_sfb)));
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
    // ---- copies: this CTA's 128 rows of A, its half of the rows of B, the scales of both; reported to the leader's barrier
    uint32_t it = 0, ph = 0;
    int s = 0;
    for (int t = worker; ok && t < p.tiles; t += workers) {
      const int ta = t % p.tiles_a, tb = t / p.tiles_a;
      for (int kb = 0; kb < p.num_kb; ++kb) {
        if ((int)it == p.stall_at) { ok = false; break; }
        ok = __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.empty[s]), ph ^ 1u, &ctrl, p));
        if (!ok) break;
        if (elect_one()) {
          const uint32_t own = smem_u32(&ctrl.full[s]), dst = ring + (uint32_t)s * kStage;
          if (rank == 0) mbar_expect_tx(own, 2u * kStage);
          const uint32_t full = mapa_rank(own, 0);
          const int words = kb * kGroups * (kFp4TileBytes / 8);
          tma_load_2d<true>(dst, &map_a, full, kb * kBlockBytes, ta * kTile + (int)rank * kRows);
          tma_load_2d<true>(dst + kABytes, &map_b, full, kb * kBlockBytes, tb * kTile + (int)rank * kRows);
          tma_load_2d<true>(dst + 2 * kABytes, &map_sfa, full, words, ta * 2 + (int)rank);
          tma_load_2d<true>(dst + 2 * kABytes + sf_bytes(BLOCK), &map_sfb, full, words, tb * 2);
        }
        __syncwarp();
        ++it;
        if (++s == kStages) { s = 0; ph ^= 1u; }
      }
    }
    if ((!ok || ctrl.abort) && lane == 0) {
      // gave up: let the copies in flight land.  (Their bytes are counted on the leader's barriers, so the follower just waits.)
      const uint32_t n = it < kStages ? it : kStages;
      const unsigned long long t0 = global_ns();
      for (uint32_t j = it - n; j < it; ++j) {
        while (global_ns() - t0 < 5000000ull &&
               (rank != 0 || !mbar_try_wait(smem_u32(&ctrl.full[j % kStages]), (j / kStages) & 1u))) {
        }
      }
    }
    __syncwarp();
  } else if (warp == 1 && rank == 0) {
    // ---- MMA issue
    const uint32_t issue = elect_one() ? 1u : 0u;
    const uint32_t id = make_idesc_fp4(BLOCK, kTile, kTile);
    const uint32_t dhi = smem_desc_hi(8u * kBlockBytes, 2u);          // 128-byte swizzle
    const uint32_t shi = smem_desc_hi(128u, 0u);                       // scale tiles: rows of 16 bytes, groups of 8 rows
    uint32_t ph = 0;
    int s = 0, local = 0;
    bool full_next = false;
    for (int t = worker; ok && t < p.tiles; t += workers, ++local) {
      if (local > 0) {
        ok = __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.acc_free), (uint32_t)(local - 1) & 1u, &ctrl, p));
        if (!ok) break;
        tc_fence_after();
      }
      for (int kb = 0; kb < p.num_kb; ++kb) {
        // (looked at while the k-block before was issued)
        if (!full_next) ok = __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.full[s]), ph, &ctrl, p));
        if (!ok) break;
        const int next_s = s + 1 == kStages ? 0 : s + 1;
        const uint32_t next_ph = next_s == 0 ? ph ^ 1u : ph;
        full_next = __all_sync(0xffffffffu, mbar_test(smem_u32(&ctrl.full[next_s]), next_ph));
        tc_fence_after();
        const uint32_t a = smem_desc_lo(ring) + (uint32_t)s * (kStage >> 4), b = a + (kABytes >> 4);
        const uint32_t sf = ((ring + (uint32_t)s * kStage + 2 * kABytes) >> 4) & 0x3FFFu;
        const uint32_t ta = tmem + kScales + (uint32_t)s * (uint32_t)scale_columns(BLOCK), tb = ta + 4u * kGroups;
        const bool last = kb == p.num_kb - 1;
        const uint32_t more = kb > 0 ? 1u : 0u;
        if (!last) {
          issue_kblock<BLOCK, true>(issue, tmem, a, b, dhi, id, ta, tb, 8u, sf, shi, more, kBlockElems / kStepElems, kGroups);
        } else {
          issue_kblock<BLOCK, true>(issue, tmem, a, b, dhi, id, ta, tb, 8u, sf, shi, more, p.steps_last, p.groups_last);
        }
        tc_commit_if<true>(issue, smem_u32(&ctrl.empty[s]));
        s = next_s;
        ph = next_ph;
      }
      if (ok) tc_commit_if<true>(issue, smem_u32(&ctrl.acc_full));
    }
    if ((!ok || ctrl.abort) && lane == 0) {
      // no MMA may still read shared memory or write TMEM when the CTAs tear down
      tc_commit<true>(smem_u32(&ctrl.drain));
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(smem_u32(&ctrl.drain), 0) && global_ns() - t0 < 50000000ull) {
      }
    }
    __syncwarp();
  } else if (warp == 3 && ROWS) {
    // ---- stores, one staging block after the other with at most three under way, so that copies are never far behind them
    constexpr int kPasses = DT == ADAPTION_F32 ? 2 : 1, kUnderWay = 2;
    int n = 0;                               // stores so far
    for (int t = worker; ok && t < p.tiles; t += workers) {
      const int row0 = (t % p.tiles_a) * kTile + (int)rank * kRows, col0 = (t / p.tiles_a) * kTile;
      for (int i = 0; ok && i < kPasses * kEpiWarps; ++i, ++n) {
        const int w = i % kEpiWarps;
        ok = __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.staged[w]), (uint32_t)(n / kEpiWarps) & 1u, &ctrl, p));
        if (!ok) break;
        const int row = row0 + (w & 3) * 32, col = col0 + (w >> 2) * kWarpCols + (i / kEpiWarps) * 32;
        if (lane == 0) {
          if (row < p.B && col < p.cols16)
            tma_store_2d(&map_y, ring + kStages * kStage + (uint32_t)w * kStagingBytes, col * (DT == ADAPTION_F32 ? 4 : 2), row);
          tma_store_commit();
          tma_store_wait_read<kUnderWay>();
          if (n >= kUnderWay) mbar_arrive(smem_u32(&ctrl.stored[(n - kUnderWay) % kEpiWarps]));
        }
        __syncwarp();
      }
    }
    if (lane == 0) tma_store_wait();
    __syncwarp();
  } else if (warp >= kFirstEpiWarp) {
    // ---- epilogue: four warps per lane quarter, 64 columns each
    const int quarter = warp & 3, part = (warp - kFirstEpiWarp) >> 2;
    const uint32_t acc = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(part * kWarpCols);
    const int self = warp - kFirstEpiWarp;
    const uint32_t staging = ring + kStages * kStage + (uint32_t)self * kStagingBytes;
    int blocks = 0;                          // staging blocks filled so far
    uint32_t counted = 0;
    int local = 0;
    for (int t = worker; t < p.tiles; t += workers, ++local) {
      const int ta = t % p.tiles_a, tb = t / p.tiles_a;
      const int at0 = ta * kTile + (int)rank * kRows + quarter * 32, at = at0 + lane;    // this warp's first row of A, this lane's
      const int col = tb * kTile + part * kWarpCols;                                      // its first row of B
      const bool real = at < (ROWS ? p.B : p.O);
      float bias = 0.f;
      if (ROWS) {
        // the channels' biases; every warp has left the last tile's behind when all come here
        const int i = (int)threadIdx.x - 32 * kFirstEpiWarp, o = tb * kTile + i;
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kEpiWarps) : "memory");
        if (i < kTile) bias_tile[i] = p.bias != nullptr && o < p.O ? __ldg(p.bias + o) : 0.f;
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kEpiWarps) : "memory");
      } else if (p.bias != nullptr && real) {
        bias = __ldg(p.bias + at);
      }
      // (a wait that ran out in one warp is seen by the others at their next one)
      ok = ok && __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.acc_full), (uint32_t)local & 1u, &ctrl, p));
      if (!ok) {
        if (ROWS) continue;              // (the others still meet at the barriers)
        break;
      }
      tc_fence_after();
      int32_t r[2][32];
      tmem_ld32(acc, r[0]);
      tmem_ld32(acc + 32u, r[1]);
      tmem_ld_wait();
      pin_after_wait32(r[0]);
      pin_after_wait32(r[1]);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(mapa_rank(smem_u32(&ctrl.acc_free), 0));
      ZeroCount<DT> zeros;
      if (ROWS) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (h == 0 || DT == ADAPTION_F32) {
            // the block is free once the last store has read it
            if (blocks > 0) ok = ok && __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.stored[self]), (uint32_t)(blocks - 1) & 1u, &ctrl, p));
            ++blocks;
          }
          if (!ok) break;
          stage_row<DT>(p, r[h], staging, h, lane, col + 32 * h, real, p.y + (long long)at * p.y_pitch, bias_tile + part * kWarpCols + 32 * h,
                        zeros);
          if (h == 1 || DT == ADAPTION_F32) {
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctrl.staged[self]));
          }
        }
      } else if (real) {
        uint8_t* const y = p.y + (long long)col * p.y_pitch + (long long)at * (DT == ADAPTION_F32 ? 4 : 2);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          store_channel<DT, 16>(&r[i >> 1][16 * (i & 1)], y + (long long)(16 * i) * p.y_pitch, p.y_pitch, p.B - col - 16 * i, p.unit, bias,
                                p.relu != 0, zeros);
      }
      counted += zeros.total();
    }
    __syncwarp();
    counted = __reduce_add_sync(0xffffffffu, counted);
    if (lane == 0 && counted) atomicAdd((unsigned long long*)&p.stats->zeros, (unsigned long long)counted);
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync_all();          // neither CTA leaves (or frees TMEM) while the other may still signal it
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc<true>(tmem, kTmemCols);
  }
}

template <int BLOCK, int DT, bool ROWS>
int launch_pair(const CUtensorMap* maps, const PairParams& p, int grid, cudaStream_t stream) {
  constexpr size_t smem = smem_bytes(BLOCK);
  static std::atomic<uint64_t> prepared{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_failure(e, "fp4_pair_kernel device");
  if (dev >= 64 || !((prepared.load(std::memory_order_acquire) >> dev) & 1)) {
    e = cudaFuncSetAttribute(fp4_pair_kernel<BLOCK, DT, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)smem);
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
  e = cudaLaunchKernelEx(&cfg, fp4_pair_kernel<BLOCK, DT, ROWS>, maps[0], maps[1], maps[2], maps[3], maps[4], p);
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return cuda_failure(e, "fp4_pair_kernel launch");
  }
  return ADAPTION_OK;
}

template <int BLOCK, bool ROWS>
int launch_pair(const CUtensorMap* maps, const PairParams& p, int dtype, int grid, cudaStream_t stream) {
  if (dtype == ADAPTION_F32) return launch_pair<BLOCK, ADAPTION_F32, ROWS>(maps, p, grid, stream);
  if (dtype == ADAPTION_F16) return launch_pair<BLOCK, ADAPTION_F16, ROWS>(maps, p, grid, stream);
  return launch_pair<BLOCK, ADAPTION_BF16, ROWS>(maps, p, grid, stream);
}

}  // namespace

int launch_fp4_pair(const Fp4Problem& g) {
  const int block = g.w.block;
  PairParams p;
  std::memset(&p, 0, sizeof(p));
  p.O = (int)g.O;
  p.B = (int)g.B;
  const int size = dtype_size(g.y.dtype);
  p.y = (uint8_t*)g.y.data;
  p.y_pitch = g.y.stride * size;
  // (a store's coordinates are bytes, below 2^31)
  const bool rows = aligned16(g.y.data) && (p.y_pitch & 15) == 0 && (int64_t)p.O * size >= 16 && (int64_t)p.O * size < (int64_t)1 << 31;
  p.cols16 = (int)(((int64_t)p.O * size & ~(int64_t)15) / size);
  const adaption_fp4tensor &ta = rows ? g.x : g.w, &tb = rows ? g.w : g.x;
  const int na = rows ? p.B : p.O, nb = rows ? p.O : p.B;
  p.tiles_a = (na + kTile - 1) / kTile;
  const int64_t tiles = (int64_t)p.tiles_a * ((nb + kTile - 1) / kTile);
  if (tiles > 0x3fffffff) return ADAPTION_ERR_UNSUPPORTED;
  p.tiles = (int)tiles;
  p.num_kb = (int)((g.K + kBlockElems - 1) / kBlockElems);
  const int64_t groups = fp4_groups(g.K, block);
  const int k_last = (int)(g.K - (int64_t)(p.num_kb - 1) * kBlockElems);
  p.steps_last = (k_last + kStepElems - 1) / kStepElems;
  p.groups_last = (int)(groups - (int64_t)(p.num_kb - 1) * groups_of(block));
  p.unit = pow2_float(g.x.exp + g.w.exp);
  p.bias = g.bias;
  p.relu = g.relu ? 1 : 0;
  p.stats = g.stats;
  p.timeout_ns = wait_limit_ns();
  p.stall_at = knob(kStallAt);
  if (!load_tensor_map_encoders()) return ADAPTION_ERR_CUDA;
  CUtensorMap maps[5];
  std::memset(&maps[4], 0, sizeof(maps[4]));
  bool ok = encode_fp4_codes(&maps[0], ta, na, g.K, kRows, false) && encode_fp4_codes(&maps[1], tb, nb, g.K, kRows, false) &&
            encode_fp4_scales(&maps[2], ta, na, groups, 1) && encode_fp4_scales(&maps[3], tb, nb, groups, 2);
  // rows of y: boxes of 128 bytes x 32 rows
  if (ok && rows)
    ok = encode_tiled_2d(&maps[4], p.y, (uint64_t)p.O * (uint64_t)size & ~(uint64_t)15, (uint64_t)p.B, (uint64_t)p.y_pitch, 128u, 32u, CU_TENSOR_MAP_SWIZZLE_128B);
  if (!ok) return ADAPTION_ERR_CUDA;
  int pairs = num_sms() / 2;
  if (pairs > p.tiles) pairs = p.tiles;
  if (block == 32)
    return rows ? launch_pair<32, true>(maps, p, g.y.dtype, 2 * pairs, g.stream) : launch_pair<32, false>(maps, p, g.y.dtype, 2 * pairs, g.stream);
  return rows ? launch_pair<16, true>(maps, p, g.y.dtype, 2 * pairs, g.stream) : launch_pair<16, false>(maps, p, g.y.dtype, 2 * pairs, g.stream);
}

}  // namespace adaption
