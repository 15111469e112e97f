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
constexpr size_t kSmemLimit = 225 * 1024;  // of 227 KB, less barriers and biases

// shared columns of the two accumulators = columns of the scales of two k-blocks
__host__ __device__ constexpr int scale_columns(int block) { return groups_of(block) * 4 * 3; }
__host__ __device__ constexpr int shared_columns(int block) { return 2 * scale_columns(block); }
__host__ __device__ constexpr uint32_t sf_bytes(int block) { return (uint32_t)groups_of(block) * kFp4TileBytes; }
__host__ __device__ constexpr uint32_t stage_bytes(int block) { return 2 * kABytes + 3 * sf_bytes(block); }

struct PairParams {
  int O, B;
  int tiles_a, tiles;           // tiles along A; all
  int num_kb, steps_last, groups_last;
  int stages;
  float unit;                   // 2^(sum of the operands' exponents)
  const float* bias;
  int relu;
  uint8_t* y;
  long long y_pitch;            // bytes
  int aligned32;                // rows of y lie on 32-byte boundaries
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

// 16 * N consecutive columns of the accumulator
template <int N>
__device__ __forceinline__ void load_columns(uint32_t taddr, int32_t (&r)[2 * N][8]) {
#pragma unroll
  for (int i = 0; i < N; ++i) tmem_ld16(taddr + 16u * i, r[2 * i], r[2 * i + 1]);
  tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < 2 * N; ++i) pin_after_wait(r[i]);
}

// Outputs stored as 0 of one lane and tile: pairs of 16-bit outputs are compared and counted together, in their own type (a
// lane has at most 128 of them, all counts are exact).
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

// Lanes are batch rows, columns are channels: 16 of them from channel `c` on become one or two 32-byte pieces of this lane's row.
template <int DT>
__device__ __forceinline__ void finish_row(const PairParams& p, const int32_t* r, uint8_t* row, int c, const float* bias,
                                           ZeroCount<DT>& zeros) {
  const int n = p.O - c;                               // channels that exist
  float v[16];
#pragma unroll
  for (int j = 0; j < 16; j += 4) {
    const float4 b = *reinterpret_cast<const float4*>(bias + j);
    v[j] = fmaf(__int_as_float(r[j]), p.unit, b.x);
    v[j + 1] = fmaf(__int_as_float(r[j + 1]), p.unit, b.y);
    v[j + 2] = fmaf(__int_as_float(r[j + 2]), p.unit, b.z);
    v[j + 3] = fmaf(__int_as_float(r[j + 3]), p.unit, b.w);
  }
  if constexpr (DT == ADAPTION_F32) {
    if (p.relu) {
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = relu1(v[j]);
    }
    float* const y = reinterpret_cast<float*>(row) + c;
    if (n >= 16) {
#pragma unroll
      for (int j = 0; j < 16; ++j) zeros.n += v[j] == 0.f;
#pragma unroll
      for (int j = 0; j < 16; j += 4) reinterpret_cast<float4*>(y)[j / 4] = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        if (j >= n) break;
        zeros.n += v[j] == 0.f;
        y[j] = v[j];
      }
    }
    return;
  }
  uint32_t w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = pack2<DT>(v[2 * j], v[2 * j + 1]);
  if (p.relu) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = relu2<DT>(w[j]);
  }
  uint16_t* const y = reinterpret_cast<uint16_t*>(row) + c;
  if (n >= 16) {
#pragma unroll
    for (int j = 0; j < 8; ++j) zeros.pair(w[j]);
    if (p.aligned32) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(y), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                   "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                   : "memory");
    } else {
      reinterpret_cast<uint4*>(y)[0] = make_uint4(w[0], w[1], w[2], w[3]);
      reinterpret_cast<uint4*>(y)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if (j >= n) break;
      const uint16_t h = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
      zeros.n += (h & 0x7fffu) == 0u;
      y[j] = h;
    }
  }
}

// Lanes are channels, columns are batch rows: 16 rows from `row` on, this lane's channel of each (consecutive lanes store
// consecutive outputs, so rows of any alignment do).
template <int DT>
__device__ __forceinline__ void finish_channel(const PairParams& p, const int32_t* r, uint8_t* at, int rows, float bias,
                                               ZeroCount<DT>& zeros) {
#pragma unroll
  for (int j = 0; j < 16; j += 2) {
    if (j >= rows) break;
    float a = fmaf(__int_as_float(r[j]), p.unit, bias), b = fmaf(__int_as_float(r[j + 1]), p.unit, bias);
    uint8_t* const next = at + p.y_pitch;
    if (DT == ADAPTION_F32) {
      if (p.relu) { a = relu1(a); b = relu1(b); }
      zeros.n += a == 0.f;
      *reinterpret_cast<float*>(at) = a;
      if (j + 1 < rows) {
        zeros.n += b == 0.f;
        *reinterpret_cast<float*>(next) = b;
      }
    } else {
      uint32_t w = pack2<DT>(a, b);
      if (p.relu) w = relu2<DT>(w);
      *reinterpret_cast<uint16_t*>(at) = (uint16_t)w;
      if (j + 1 < rows) {
        zeros.pair(w);
        *reinterpret_cast<uint16_t*>(next) = (uint16_t)(w >> 16);
      } else {
        zeros.n += (w & 0x7fffu) == 0u;
      }
    }
    at = next + p.y_pitch;
  }
}

// What a lane of the epilogue knows about its tile.
struct TileLane {
  uint8_t* y;          // ROWS: start of this lane's row; else this lane's channel in the tile's first row
  int first;           // first channel (ROWS) or batch row of the tile
  float bias;          // of this lane's channel
  const float* biases; // ROWS: of the tile's channels
  bool real;           // the lane's row or channel exists
};
template <int DT, bool ROWS, int N>
__device__ __forceinline__ void finish_columns(const PairParams& p, const int32_t (&r)[2 * N][8], const TileLane& t, int c,
                                               ZeroCount<DT>& zeros) {
  if (!t.real) return;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = c + 16 * i;
    if (ROWS)
      finish_row<DT>(p, &r[2 * i][0], t.y, t.first + at, t.biases + at, zeros);
    else
      finish_channel<DT>(p, &r[2 * i][0], t.y + (long long)at * p.y_pitch, p.B - t.first - at, t.bias, zeros);
  }
}
template <int DT, bool ROWS, int N>
__device__ __forceinline__ void finish_rest(const PairParams& p, uint32_t acc, const TileLane& t, int c, ZeroCount<DT>& zeros) {
  int32_t r[2 * N][8];
  load_columns<N>(acc + (uint32_t)c, r);
  finish_columns<DT, ROWS, N>(p, r, t, c, zeros);
}
// The shared columns: handed back as soon as they are in registers.
template <int DT, bool ROWS, int N>
__device__ __forceinline__ void finish_shared(const PairParams& p, uint32_t acc, const TileLane& t, int c, PairCtrl* ctrl, int lane,
                                              ZeroCount<DT>& zeros) {
  int32_t r[2 * N][8];
  load_columns<N>(acc + (uint32_t)c, r);
  tc_fence_before();
  __syncwarp();
  if (lane == 0) mbar_arrive_cluster(mapa_rank(smem_u32(&ctrl->acc_free), 0));
  finish_columns<DT, ROWS, N>(p, r, t, c, zeros);
}

// ROWS: the 128-row operand A is the batch (lanes of the accumulators are batch rows) and the columns are channels; otherwise
// A is the weights.  map_a, map_sfa and so on are of the operand in that place.
template <int BLOCK, int DT, bool ROWS>
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
  __shared__ __align__(16) float bias_tile[ROWS ? kTile : 4];
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
    uint32_t counted = 0;
    int local = 0;
    for (int t = worker; t < p.tiles; t += workers, ++local) {
      const int ta = t % p.tiles_a, tb = t / p.tiles_a;
      const int at = ta * kTile + (int)rank * kRows + quarter * 32 + lane;          // this lane's row of A
      TileLane tile;
      tile.first = tb * kTile;
      tile.real = at < (ROWS ? p.B : p.O);
      tile.bias = 0.f;
      tile.biases = bias_tile;
      if (ROWS) {
        tile.y = p.y + (long long)at * p.y_pitch;
        // the channels' biases; every warp has left the last tile's behind when all come here
        const int i = (int)threadIdx.x - 32 * kFirstEpiWarp, o = tile.first + i;
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kEpiWarps) : "memory");
        bias_tile[i] = p.bias != nullptr && o < p.O ? __ldg(p.bias + o) : 0.f;
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kEpiWarps) : "memory");
      } else {
        tile.y = p.y + (long long)tile.first * p.y_pitch + (long long)at * (DT == ADAPTION_F32 ? 4 : 2);
        if (p.bias != nullptr && tile.real) tile.bias = __ldg(p.bias + at);
      }
      // (a wait that ran out in one warp is seen by the others at their next one)
      ok = ok && __all_sync(0xffffffffu, pair_wait(smem_u32(&ctrl.acc_full[local & 1]), (uint32_t)(local >> 1) & 1u, &ctrl, p));
      if (!ok) {
        if (ROWS) continue;              // (the others still meet at the barriers)
        break;
      }
      tc_fence_after();
      ZeroCount<DT> zeros;
      // the columns that the next tile's accumulator shares first: the last ones of the first accumulator, the first ones
      // of the second; in runs of 16
      const uint32_t acc = lanes + ((local & 1) ? kSecond : 0u);
      const int first = (local & 1) ? 0 : (int)kSecond, rest = (local & 1) ? kShared : 0;
      if (BLOCK == 32) {
        if (half == 0) {
          finish_shared<DT, ROWS, 2>(p, acc, tile, first, &ctrl, lane, zeros);
          finish_rest<DT, ROWS, 3>(p, acc, tile, rest, zeros);
          finish_rest<DT, ROWS, 3>(p, acc, tile, rest + 48, zeros);
        } else {
          finish_shared<DT, ROWS, 1>(p, acc, tile, first + 32, &ctrl, lane, zeros);
          finish_rest<DT, ROWS, 3>(p, acc, tile, rest + 96, zeros);
          finish_rest<DT, ROWS, 2>(p, acc, tile, rest + 144, zeros);
          finish_rest<DT, ROWS, 2>(p, acc, tile, rest + 176, zeros);
        }
      } else {
        finish_shared<DT, ROWS, 3>(p, acc, tile, first + 48 * half, &ctrl, lane, zeros);
        finish_rest<DT, ROWS, 3>(p, acc, tile, rest + 80 * half, zeros);
        finish_rest<DT, ROWS, 2>(p, acc, tile, rest + 80 * half + 48, zeros);
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
  const size_t smem = (size_t)p.stages * stage_bytes(BLOCK) + 1024;
  static std::atomic<uint64_t> prepared{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_failure(e, "fp4_pair_kernel device");
  if (dev >= 64 || !((prepared.load(std::memory_order_acquire) >> dev) & 1)) {
    e = cudaFuncSetAttribute(fp4_pair_kernel<BLOCK, DT, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)kSmemLimit);
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
  e = cudaLaunchKernelEx(&cfg, fp4_pair_kernel<BLOCK, DT, ROWS>, maps[0], maps[1], maps[2], maps[3], p);
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
  const int size = dtype_size(g.y.dtype);
  p.y = (uint8_t*)g.y.data;
  p.y_pitch = g.y.stride * size;
  const bool rows = aligned16(g.y.data) && (p.y_pitch & 15) == 0;
  p.aligned32 = ((reinterpret_cast<uintptr_t>(g.y.data) | (uintptr_t)p.y_pitch) & 31u) == 0;
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
  p.stages = (int)((kSmemLimit - 1024) / stage_bytes(block));
  if (p.stages > kMaxStages) p.stages = kMaxStages;
  p.unit = pow2_float(g.x.exp + g.w.exp);
  p.bias = g.bias;
  p.relu = g.relu ? 1 : 0;
  p.stats = g.stats;
  p.timeout_ns = wait_limit_ns();
  p.stall_at = knob(kStallAt);
  if (!load_tensor_map_encoders()) return ADAPTION_ERR_CUDA;
  CUtensorMap maps[4];
  const uint64_t bytes = (uint64_t)(g.K + 1) / 2;
  bool ok = encode_tiled_2d(&maps[0], ta.codes, bytes, (uint64_t)na, (uint64_t)ta.c_stride / 2, kBlockBytes, kRows,
                            CU_TENSOR_MAP_SWIZZLE_128B) &&
            encode_tiled_2d(&maps[1], tb.codes, bytes, (uint64_t)nb, (uint64_t)tb.c_stride / 2, kBlockBytes, kRows,
                            CU_TENSOR_MAP_SWIZZLE_128B);
  // scale planes: one row per row of tiles, in words of 8 bytes; what lies behind the last tile arrives as zeros
  for (int i = 0; ok && i < 2; ++i) {
    const uint64_t dims[2] = {(uint64_t)groups * (kFp4TileBytes / 8), (uint64_t)(((i ? nb : na) + kRows - 1) / kRows)};
    const uint64_t strides[1] = {(uint64_t)groups * kFp4TileBytes};
    const uint32_t box[2] = {(uint32_t)(groups_of(block) * (kFp4TileBytes / 8)), i ? 2u : 1u};
    ok = encode_tiled_words(&maps[2 + i], i ? tb.scales : ta.scales, 2, dims, strides, box);
  }
  if (!ok) return ADAPTION_ERR_CUDA;
  int pairs = num_sms() / 2;
  if (pairs > p.tiles) pairs = p.tiles;
  if (block == 32)
    return rows ? launch_pair<32, true>(maps, p, g.y.dtype, 2 * pairs, g.stream) : launch_pair<32, false>(maps, p, g.y.dtype, 2 * pairs, g.stream);
  return rows ? launch_pair<16, true>(maps, p, g.y.dtype, 2 * pairs, g.stream) : launch_pair<16, false>(maps, p, g.y.dtype, 2 * pairs, g.stream);
}

}  // namespace adaption
