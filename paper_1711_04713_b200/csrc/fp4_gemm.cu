// Inner product of microscaled 4-bit operands (adaption_fp4_ip_fwd) on the tensor cores, for problems with few output tiles: one
// thread-block cluster per tile, which shares the reduction.
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
// elements (two of 512 bytes per 128 rows for blocks of 32, four for blocks of 16), which lie one after the other in memory.
// The issuing thread moves them to TMEM (tcgen05.cp, 32 rows x 16 bytes repeated in the four lane quarters: what
// the MMA reads) into columns that belong to the ring's stage: they are written again only after the MMAs that read
// them have released the stage.
//
// Activations that are still real numbers are quantized into the ring by the warps that are idle in the main loop (FUSED), if they are few:
// a warp takes a row's 256 elements of a k-block, and the full barrier of a stage counts the rows beside the copies' bytes.
// That saves a launch; every tile of channels quantizes them anew.
//
// Two forms: single CTAs on tiles of 128 channels x up to 128 rows, and pairs of CTAs (cta_group::2) on 256 x 256, which need two
// thirds of the copied bytes per product.  The S CTAs (pairs) of a cluster take shares of the k-blocks; at the end each owns
// a range of columns (runs of four), sends its partial sums of the others' columns to their shared memory, and adds what it
// receives to its own.  Few columns are sent by the lanes (st.async, counted by an mbarrier at the owner); as that mbarrier counts
// every 16 bytes apart, 5000 cycles for 256 columns, more than 32 go through shared memory and leave as a bulk copy per run.
//
// What bounds it (replays of a graph over weights that do not fit L2 together): the weights' bytes from HBM where rows are few, 4.9 TB/s over a
// launch of 11.8 us (25088 -> 4096, one row: 58 MB; about 2 us pass before the first k-block and 2 after the last; 15.1 us where the row is
// quantized here); with more rows an SM's share of L2's reads, 64 bytes a cycle (the same on 256 rows: 128 CTAs copy 171 MB in 10.5 of
// 17.9 us); for small matrices the launch's chain of copies, MMAs, exchange and stores (4096 -> 4096, one row: 4.8 us, 3.9 with the weights in L2).
#include <cuda.h>

#include <cstring>

#include "fp4_mma.cuh"
#include "fp4_quant.cuh"
#include "knobs.cuh"
#include "remember.cuh"
#include "tensor_maps.cuh"

namespace adaption {

int num_sms();

namespace {

constexpr int kMaxStages = 10;
__host__ __device__ constexpr int threads_of(bool pair, bool fused) { return pair || fused ? 512 : 256; }    // warp 0: copies; 1: MMA; all: the epilogue
constexpr size_t kSmemLimit = 226 * 1024;  // of 227 KB, less the control block

struct FpParams {
  int O, B;                     // output channels, batch rows
  int S;                        // shares of the reduction
  int tiles_o;
  int BN;                       // columns of a tile: a multiple of 16
  int chunks_b;                 // scale tiles that cover them
  int num_kb, kb_per_split;
  int steps_last;               // MMAs of the last k-block
  int groups_last;              // scale tiles of the last k-block and 128 rows
  int stages;
  uint32_t b_bytes, stage_bytes, tmem_cols, sf_col;
  uint32_t recv_offset;         // of the received sums, in bytes from the ring's start
  int bulk;                     // sums leave by bulk copies from where the ring was, and are received behind that
  // FUSED: real activations
  const uint8_t* x;
  long long x_pitch;            // bytes
  int x_aligned, K;             // rows of x lie on 16-byte boundaries
  float inv_unit, step_unit;    // 2^-exp, 2^exp of their 4-bit form
  int early;                    // the weights may be read before the kernel in front has ended
  int max_runs;                 // runs of four columns that a share owns (the last ones fewer)
  uint32_t owners;              // without bulk copies: the owner of each of up to eight runs, four bits each
  float unit;                   // 2^(sum of the operands' exponents)
  const float* bias;
  int relu;
  uint8_t* y;
  long long y_pitch;            // bytes
  int y_dtype;
  adaption_stats* stats;
  unsigned long long timeout_ns;
  int stall_at;                 // test aid, see adaption_debug_set
};

struct FpCtrl {
  unsigned long long full[kMaxStages];     // PAIR: the leader's, bytes of both CTAs
  unsigned long long empty[kMaxStages];
  unsigned long long done;
  unsigned long long recv;                 // the other shares' partial sums have arrived
  uint32_t tmem_base;
  volatile uint32_t abort;
};

__device__ __noinline__ bool fp_wait_slow(uint32_t bar, uint32_t parity, FpCtrl* ctrl, const FpParams& p, unsigned long long limit,
                                          bool heed_abort) {
  const unsigned long long t0 = global_ns();
  while (!mbar_try_wait_suspend(bar, parity, 1000u)) {
    if (heed_abort && ctrl->abort) return false;
    if (global_ns() - t0 > limit) {
      ctrl->abort = 1;
      atomicExch(&p.stats->status, (int)ADAPTION_ERR_TIMEOUT);
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool fp_wait(uint32_t bar, uint32_t parity, FpCtrl* ctrl, const FpParams& p) {
  if (mbar_try_wait(bar, parity)) return true;
  return fp_wait_slow(bar, parity, ctrl, p, p.timeout_ns, true);
}

constexpr uint32_t kRunBytes = kRows * 16;

// shared memory of this CTA -> shared memory of a CTA of the cluster, reported to a barrier there
__device__ __forceinline__ void bulk_copy_to_peer(uint32_t dst_cluster, uint32_t src, uint32_t bytes, uint32_t bar_cluster) {
  asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst_cluster),
               "r"(src), "r"(bytes), "r"(bar_cluster)
               : "memory");
}
// (without the release that would wait for the stores of this thread: the barrier orders uses of shared memory that have ended)
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
// four floats to the shared memory of a CTA of the cluster, counted by a barrier there
__device__ __forceinline__ void st_async_v4(uint32_t addr, uint32_t bar, int32_t a, int32_t b, int32_t c, int32_t d) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(addr), "r"(a), "r"(b),
               "r"(c), "r"(d), "r"(bar)
               : "memory");
}

template <int DT, int N>
__device__ __forceinline__ void store_columns(const FpParams& p, const int32_t* r, uint8_t* at, int rows, float bias, uint32_t& zeros) {
  if (DT >= 0) {
    ZeroCount<DT> z;
    store_channel<DT, N>(r, at, p.y_pitch, rows, p.unit, bias, p.relu != 0, z);
    zeros += z.total();
  } else if (p.y_dtype == ADAPTION_F32) {
    store_columns<ADAPTION_F32, N>(p, r, at, rows, bias, zeros);
  } else if (p.y_dtype == ADAPTION_F16) {
    store_columns<ADAPTION_F16, N>(p, r, at, rows, bias, zeros);
  } else {
    store_columns<ADAPTION_BF16, N>(p, r, at, rows, bias, zeros);
  }
}

// Eight elements of a row from element `col` on: as raw words, and as numbers (0 behind the row's end).
template <int SRC>
__device__ __forceinline__ void load_eight(const FpParams& p, const uint8_t* row, int col, uint32_t (&w)[8]) {
  constexpr int kSize = SRC == ADAPTION_F32 ? 4 : 2;
  const uint8_t* at = row + (long long)col * kSize;
  if (p.x_aligned && p.K - col >= 8) {
    const uint4 a = __ldg(reinterpret_cast<const uint4*>(at));
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    if (SRC == ADAPTION_F32) {
      const uint4 b = __ldg(reinterpret_cast<const uint4*>(at) + 1);
      w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
  } else {
    load_shifted(at, min(p.K - col, 8) * kSize, w);
  }
}
template <int SRC>
__device__ __forceinline__ float numbers_of(int n, const uint32_t (&w)[8], float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (SRC == ADAPTION_F32) v[k] = __uint_as_float(w[k]);
    else if (SRC == ADAPTION_F16) v[k] = __half2float(__ushort_as_half((unsigned short)(w[k >> 1] >> (16 * (k & 1)))));
    else v[k] = __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
  }
  if (n < 8) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k >= n) v[k] = 0.f;
  }
  uint32_t top = 0u;
#pragma unroll
  for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);    // (magnitudes in order, NaN above them all)
  return __uint_as_float(top);
}

// Quantizes the rows b0 .. b0 + rows - 1 of this CTA's k-blocks into the ring's stages; a warp's next item is loaded while it works on
// one.  No more warps than stages * rows take part: a warp's items are then at most a round of the ring apart, and the wait that it
// passed for one says that the phase before the one that it waits for next is over (a barrier tells phases apart modulo two only).
template <int BLOCK, int SRC>
__device__ __forceinline__ void quantize_into_ring(const FpParams& p, FpCtrl* ctrl, uint32_t ring, int kb_begin, int kb_end, int b0, int rows,
                                                   int first, int warps, int lane) {
  constexpr int kLanes = BLOCK / 8;
  const int blocks = kb_end - kb_begin;
  if (warps > p.stages * rows) warps = p.stages * rows;
  if (first >= warps) return;
  int kb = first / rows, row = first % rows;              // (of this warp's items: first, first + warps, ...)
  uint32_t w[8];
  if (kb < blocks) load_eight<SRC>(p, p.x + (long long)(b0 + row) * p.x_pitch, (kb_begin + kb) * kBlockElems + 8 * lane, w);
  int s = kb, round = 0;                                  // (kb < stages)
  while (kb < blocks) {
    const int this_kb = kb, this_row = row, this_s = s, this_round = round;
    float v[8];
    const int col = (kb_begin + this_kb) * kBlockElems + 8 * lane;
    float top = numbers_of<SRC>(p.K - col, w, v);
    row += warps;
    while (row >= rows) {
      row -= rows;
      ++kb;
      if (++s == p.stages) { s = 0; ++round; }
    }
    if (kb < blocks) load_eight<SRC>(p, p.x + (long long)(b0 + row) * p.x_pitch, (kb_begin + kb) * kBlockElems + 8 * lane, w);
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1)
      top = __uint_as_float(max(__float_as_uint(top), __shfl_xor_sync(0xffffffffu, __float_as_uint(top), o)));
    fp4_finite<BLOCK, 8>(v, top);
    uint32_t code[1];
    const uint32_t byte = fp4_encode<BLOCK, 8, SRC != ADAPTION_F32>(v, top, p.inv_unit, p.step_unit, code);
    __syncwarp();
    if (this_round > 0 && !__all_sync(0xffffffffu, fp_wait(smem_u32(&ctrl->empty[this_s]), (uint32_t)(this_round - 1) & 1u, ctrl, p))) return;
    const uint32_t b = ring + (uint32_t)this_s * p.stage_bytes + kABytes;
    // four bytes of the row, in the order of the 128-byte swizzle
    const uint32_t at = b + (uint32_t)this_row * 128u + ((((uint32_t)lane >> 2) ^ ((uint32_t)this_row & 7u)) << 4) + ((uint32_t)lane & 3u) * 4u;
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(code[0]) : "memory");
    if ((lane & (kLanes - 1)) == 0) {
      const uint32_t j = (uint32_t)lane / kLanes, r = (uint32_t)this_row;
      const uint32_t sf = b + p.b_bytes + (uint32_t)groups_of(BLOCK) * kFp4TileBytes + (j >> 2) * kFp4TileBytes + (r & 31u) * 16u + (r >> 5) * 4u + (j & 3u);
      asm volatile("st.shared.b8 [%0], %1;" ::"r"(sf), "r"(byte) : "memory");
    }
    fence_async_shared();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&ctrl->full[this_s]));
  }
}

// DT: type of y (-1: p.y_dtype).  FUSED: type of the activations that the kernel quantizes itself, -1 where they are 4-bit already.
template <int BLOCK, bool PAIR, int DT, int FUSED>
__global__ void __launch_bounds__(threads_of(PAIR, FUSED >= 0), 1)
fp4_cluster_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const __grid_constant__ CUtensorMap map_sfa, const __grid_constant__ CUtensorMap map_sfb, const FpParams p) {
  constexpr int kGroups = groups_of(BLOCK), kThreads = threads_of(PAIR, FUSED >= 0);
  constexpr uint32_t kSf = (uint32_t)kGroups * kFp4TileBytes;          // scales of a k-block and 128 rows
  extern __shared__ uint8_t smem_raw[];
  __shared__ FpCtrl ctrl;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const int ctas = PAIR ? 2 * p.S : p.S;
  const uint32_t rank = ctas > 1 ? cluster_ctarank() : 0u;
  const int share = (int)(PAIR ? rank >> 1 : rank);                    // of the reduction
  const uint32_t half = PAIR ? rank & 1u : 0u, leader = rank - half;   // place in the pair
  const int tile = (int)blockIdx.x / ctas, to = tile % p.tiles_o, tb = tile / p.tiles_o;
  const int o0 = (PAIR ? to * 2 + (int)half : to) * kRows, b0 = tb * p.BN;
  const int cols = min(p.BN, p.B - b0), col4 = (cols + 3) / 4;         // real columns, in runs of four

  // (each of these steps takes 500 cycles: warps of their own, and a lane per barrier)
  if (warp == 0) {
    if (lane < p.stages) {
      mbar_init(smem_u32(&ctrl.full[lane]), FUSED >= 0 ? 1 + cols : 1);
      mbar_init(smem_u32(&ctrl.empty[lane]), 1);
    } else if (lane == kMaxStages) {
      mbar_init(smem_u32(&ctrl.done), 1);
    } else if (lane == kMaxStages + 1) {
      mbar_init(smem_u32(&ctrl.recv), 1);
      ctrl.abort = 0;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2 && lane < 4) prefetch_map(lane == 0 ? &map_a : (lane == 1 ? &map_b : (lane == 2 ? &map_sfa : &map_sfb)));
  if (warp == 1) {
    tmem_alloc<PAIR>(smem_u32(&ctrl.tmem_base), p.tmem_cols);
    tmem_relinquish<PAIR>();
  }
  tc_fence_before();
  __syncthreads();
  // the barriers exist before another CTA signals them: a pair's at once, others when sums are sent.  (The fence behind their
  // initialisation is the release that this needs; another one waits 800 cycles.)
  if (ctas > 1) cluster_arrive_relaxed();
  if (PAIR) cluster_wait();
  tc_fence_after();
  const uint32_t tmem = ctrl.tmem_base;

  const int first_run = share * p.max_runs, runs = max(0, min(p.max_runs, col4 - first_run));     // that this CTA finishes
  const int kb_begin = share * p.kb_per_split;
  const int kb_end = min(p.num_kb, kb_begin + p.kb_per_split);

  // Copies of one k-block: operand A (the weights) and operand B, reported to the same barrier.
  const auto copy_a = [&](int kb, int s) {
    const uint32_t own = smem_u32(&ctrl.full[s]), dst = ring + (uint32_t)s * p.stage_bytes;
    if (half == 0u) mbar_expect_tx(own, FUSED >= 0 ? kABytes + kSf : (PAIR ? 2u : 1u) * p.stage_bytes);
    const uint32_t full = PAIR ? mapa_rank(own, leader) : own;
    tma_load_2d<PAIR>(dst, &map_a, full, kb * kBlockBytes, o0);
    tma_load_2d<PAIR>(dst + kABytes + p.b_bytes, &map_sfa, full, kb * kGroups * (kFp4TileBytes / 8), o0 / kRows);
  };
  const auto copy_b = [&](int kb, int s) {
    const uint32_t own = smem_u32(&ctrl.full[s]), dst = ring + (uint32_t)s * p.stage_bytes;
    const uint32_t full = PAIR ? mapa_rank(own, leader) : own;
    tma_load_2d<PAIR>(dst + kABytes, &map_b, full, kb * kBlockBytes, PAIR ? b0 + (int)half * (p.BN / 2) : b0);
    tma_load_2d<PAIR>(dst + kABytes + p.b_bytes + kSf, &map_sfb, full, kb * kGroups * (kFp4TileBytes / 8), b0 / kRows);
  };
  // With activations that the kernel before this one quantized, the weights need not wait for it: what wrote them ended before that
  // kernel passed its own wait, and this one was launched behind that.
  const int early = p.early ? max(0, min(kb_end - kb_begin, p.stages)) : 0;
  if (warp == 0 && early > 0 && p.stall_at < 0 && elect_one()) {
    for (int s = 0; s < early; ++s) copy_a(kb_begin + s, s);
  }
  __syncwarp();

  pdl_wait();
  pdl_launch_dependents();

  // this thread's channel in the epilogue
  const int o = o0 + ((int)threadIdx.x & (kRows - 1));
  const float bias = p.bias != nullptr && o < p.O ? __ldg(p.bias + o) : 0.f;

  bool ok = true;
  if (warp == 0) {
    int s = 0, issued = 0;
    uint32_t ph = 0;
    const uint32_t issue = elect_one() ? 1u : 0u;
    for (int kb = kb_begin; kb < kb_end; ++kb) {
      if (issued == p.stall_at) break;
      if (issued >= p.stages) {
        ok = __all_sync(0xffffffffu, fp_wait(smem_u32(&ctrl.empty[s]), ph ^ 1u, &ctrl, p));
        if (!ok) break;
      }
      if (issue) {
        if (issued >= early || p.stall_at >= 0) copy_a(kb, s);
        if (FUSED < 0) copy_b(kb, s);
      }
      __syncwarp();
      ++issued;
      if (++s == p.stages) { s = 0; ph ^= 1u; }
    }
    // the ring is given another use only once the MMAs (or the issuing warp, giving up) are through with it
    if (!fp_wait(smem_u32(&ctrl.done), 0, &ctrl, p)) ok = false;
    if ((!ok || ctrl.abort) && lane == 0) {
      // gave up: let the copies in flight land.  (A pair's bytes are counted on the leader's barriers: the follower just waits.)
      const int n = issued < p.stages ? issued : p.stages;
      const unsigned long long t0 = global_ns();
      for (int j = issued - n; j < issued; ++j) {
        while (global_ns() - t0 < 5000000ull &&
               (half != 0u || !mbar_try_wait(smem_u32(&ctrl.full[j % p.stages]), (uint32_t)(j / p.stages) & 1u))) {
        }
      }
    }
    __syncwarp();
  } else if (warp == 1 && half == 0u) {
    const uint32_t issue = elect_one() ? 1u : 0u;
    const uint32_t id = make_idesc_fp4(BLOCK, p.BN, PAIR ? 2 * kRows : kRows);
    const uint32_t dhi = smem_desc_hi(8u * kBlockBytes, 2u);          // 128-byte swizzle
    const uint32_t shi = smem_desc_hi(128u, 0u);                       // scale tiles: rows of 16 bytes, groups of 8 rows
    const uint32_t cols_b = 4u * (uint32_t)p.chunks_b, slot = (uint32_t)kGroups * (4u + cols_b);
    const uint16_t mask = (uint16_t)(3u << leader);
    int s = 0;
    uint32_t ph = 0;
    bool full_next = false;
    for (int kb = kb_begin; kb < kb_end; ++kb) {
      // (looked at while the k-block before was issued)
      if (!full_next) ok = __all_sync(0xffffffffu, fp_wait(smem_u32(&ctrl.full[s]), ph, &ctrl, p));
      if (!ok) break;
      const int next_s = s + 1 == p.stages ? 0 : s + 1;
      const uint32_t next_ph = next_s == 0 ? ph ^ 1u : ph;
      full_next = __all_sync(0xffffffffu, mbar_test(smem_u32(&ctrl.full[next_s]), next_ph));
      tc_fence_after();
      const uint32_t a = smem_desc_lo(ring) + (uint32_t)s * (p.stage_bytes >> 4), b = a + (kABytes >> 4);
      const uint32_t sf = ((ring + (uint32_t)s * p.stage_bytes + kABytes + p.b_bytes) >> 4) & 0x3FFFu;
      const uint32_t ta = tmem + p.sf_col + (uint32_t)s * slot, tb0 = ta + 4u * kGroups;
      const uint32_t more = kb > kb_begin ? 1u : 0u;
      if (kb < p.num_kb - 1) {
        issue_kblock<BLOCK, PAIR>(issue, tmem, a, b, dhi, id, ta, tb0, cols_b, sf, shi, more, kBlockElems / kStepElems, kGroups);
      } else {
        issue_kblock<BLOCK, PAIR>(issue, tmem, a, b, dhi, id, ta, tb0, cols_b, sf, shi, more, p.steps_last, p.groups_last);
      }
      if (PAIR) commit_pair_if(issue, smem_u32(&ctrl.empty[s]), mask);
      else tc_commit_if<false>(issue, smem_u32(&ctrl.empty[s]));
      s = next_s;
      ph = next_ph;
    }
    if (PAIR) commit_pair_if(issue, smem_u32(&ctrl.done), mask);
    else tc_commit_if<false>(issue, smem_u32(&ctrl.done));
    __syncwarp();
    if (!ok || ctrl.abort) {
      // no MMA may still read shared memory when the ring is given another use
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(smem_u32(&ctrl.done), 0) && global_ns() - t0 < 50000000ull) {
      }
    }
  }
  if (FUSED >= 0 && warp >= 2) quantize_into_ring<BLOCK, FUSED < 0 ? 0 : FUSED>(p, &ctrl, ring, kb_begin, kb_end, b0, cols, warp - 2, kThreads / 32 - 2, lane);
  __syncwarp();

  const int size = DT < 0 ? (p.y_dtype == ADAPTION_F32 ? 4 : 2) : (DT == ADAPTION_F32 ? 4 : 2);
  constexpr int kParts = kThreads / 128;     // warps per lane quarter: each takes runs of columns in turn
  const int quarter = warp & 3, part = warp >> 2, row = quarter * 32 + lane;
  const uint32_t acc = tmem + ((uint32_t)(quarter * 32) << 16);
  const bool empty = kb_begin >= kb_end;              // (no k-blocks: the accumulator was never written)
  uint32_t zeros = 0;
  // (warps 2.. wait here for the MMAs, and in a pair the follower's for the leader's)
  ok = fp_wait(smem_u32(&ctrl.done), 0, &ctrl, p) && ok;
  __syncthreads();
  tc_fence_after();
  if (p.S == 1) {
    // ---- the whole reduction is here: bias, ReLU, store
    if (!ctrl.abort) {
      uint8_t* const y = p.y + (long long)b0 * p.y_pitch + (long long)o * size;
      for (int c = 16 * part; c < cols; c += 16 * kParts) {
        int32_t r[16];
        tmem_ld16(acc + (uint32_t)c, reinterpret_cast<int32_t(&)[8]>(r[0]), reinterpret_cast<int32_t(&)[8]>(r[8]));
        tmem_ld_wait();
        pin_after_wait(reinterpret_cast<int32_t(&)[8]>(r[0]));
        pin_after_wait(reinterpret_cast<int32_t(&)[8]>(r[8]));
        if (o < p.O) store_columns<DT, 16>(p, r, y + (long long)c * p.y_pitch, cols - c, bias, zeros);
      }
    }
  } else {
    // ---- partial sums to their owners, as runs of four columns: [run][128 channels] of 16 bytes.  Sums of all columns, or of this
    // CTA's own, lie where the ring was or in the first block of recv; the other shares' blocks follow.
    if (threadIdx.x == 0 && runs > 0) mbar_expect_tx(smem_u32(&ctrl.recv), (uint32_t)(p.S - 1) * (uint32_t)runs * kRunBytes);
    if (!PAIR) cluster_wait();                        // (arrived at the start: long complete)
    if (p.bulk) cluster_arrive_relaxed();             // this CTA's ring has come to its end
    const uint32_t recv_bar = smem_u32(&ctrl.recv), block_bytes = (uint32_t)p.max_runs * kRunBytes;
    const uint32_t own = ring + (p.bulk ? (uint32_t)first_run * kRunBytes : p.recv_offset), recv = ring + p.recv_offset + (p.bulk ? 0u : block_bytes);
    // this CTA's block among another owner's
    const uint32_t below = recv + (uint32_t)share * block_bytes, above = below - block_bytes;
#pragma unroll 1
    for (int c = 16 * part; c < cols; c += 16 * kParts) {
      int32_t r[16];
      tmem_ld16(acc + (uint32_t)c, reinterpret_cast<int32_t(&)[8]>(r[0]), reinterpret_cast<int32_t(&)[8]>(r[8]));
      tmem_ld_wait();
      pin_after_wait(reinterpret_cast<int32_t(&)[8]>(r[0]));
      pin_after_wait(reinterpret_cast<int32_t(&)[8]>(r[8]));
      if (empty) {
#pragma unroll
        for (int j = 0; j < 16; ++j) r[j] = 0;
      }
      if (p.bulk) {
        // (columns behind the last real one are staged too, up to the tile's width, and never sent or read)
        const uint32_t at = ring + (uint32_t)(c >> 2) * kRunBytes + (uint32_t)row * 16u;
#pragma unroll
        for (int j = 0; j < 16; j += 4)
          st_shared_v4(at + (uint32_t)(j >> 2) * kRunBytes, (uint32_t)r[j], (uint32_t)r[j + 1], (uint32_t)r[j + 2], (uint32_t)r[j + 3]);
      } else {
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          const int run = (c + j) >> 2, owner = (int)(p.owners >> (4 * run)) & 15;
          if (c + j >= cols) break;
          const uint32_t at = (uint32_t)(run - owner * p.max_runs) * kRunBytes + (uint32_t)row * 16u;
          if (owner == share) {
            st_shared_v4(own + at, (uint32_t)r[j], (uint32_t)r[j + 1], (uint32_t)r[j + 2], (uint32_t)r[j + 3]);
          } else {
            const uint32_t to_rank = PAIR ? 2u * (uint32_t)owner + half : (uint32_t)owner;
            st_async_v4(mapa_rank((share > owner ? above : below) + at, to_rank), mapa_rank(recv_bar, to_rank), r[j], r[j + 1], r[j + 2], r[j + 3]);
          }
        }
      }
    }
    if (p.bulk) fence_async_shared();
    __syncthreads();
    if (p.bulk) {
      cluster_wait();                                 // ... and so have the others'
      // (a copy per run: one for all of an owner's moved 17 bytes a cycle)
      const int run = (int)threadIdx.x, to = run / p.max_runs;
      if (run < col4 && to != share) {
        const uint32_t to_rank = PAIR ? 2u * (uint32_t)to + half : (uint32_t)to;
        bulk_copy_to_peer(mapa_rank((share > to ? above : below) + (uint32_t)(run - to * p.max_runs) * kRunBytes, to_rank),
                          ring + (uint32_t)run * kRunBytes, kRunBytes, mapa_rank(recv_bar, to_rank));
      }
      __syncwarp();
    }
    // Every CTA of the cluster sends, also one that gave up (within its waits' limits), so this wait ends, and no CTA leaves while
    // sums for it are under way.
    if (runs > 0 && !mbar_try_wait(recv_bar, 0))
      ok = fp_wait_slow(recv_bar, 0, &ctrl, p, 4ull * p.timeout_ns + 1000000000ull, false) && ok;

    // ---- the runs this CTA owns: its own sums and the others' in the order of their shares, bias, ReLU, store
    if (ok && o < p.O && !ctrl.abort) {
      const uint8_t* const base = smem_raw - smem_u32(smem_raw);
      const uint32_t offset = (uint32_t)part * kRunBytes + (uint32_t)row * 16u;
      const uint8_t *mine = base + own + offset, *from = base + recv + offset;
      int c = 4 * (first_run + part);
      uint8_t* y = p.y + (long long)(b0 + c) * p.y_pitch + (long long)o * size;
#pragma unroll 2
      for (int i = part; i < runs; i += kParts) {
        float4 v = *reinterpret_cast<const float4*>(mine);
        const uint8_t* next = from;
#pragma unroll 1
        for (int k = 1; k < p.S; ++k, next += block_bytes) {
          const float4 t = *reinterpret_cast<const float4*>(next);
          v.x += t.x; v.y += t.y; v.z += t.z; v.w += t.w;
        }
        const int32_t r[4] = {__float_as_int(v.x), __float_as_int(v.y), __float_as_int(v.z), __float_as_int(v.w)};
        if (cols - c >= 4) store_columns<DT, 4>(p, r, y, 4, bias, zeros);
        else store_columns<DT, 4>(p, r, y, cols - c, bias, zeros);
        mine += kParts * kRunBytes;
        from += kParts * kRunBytes;
        c += 4 * kParts;
        y += (long long)(4 * kParts) * p.y_pitch;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc<PAIR>(tmem, p.tmem_cols);
  }
  const uint32_t counted = __reduce_add_sync(0xffffffffu, zeros);
  if (lane == 0 && counted) atomicAdd((unsigned long long*)&p.stats->zeros, (unsigned long long)counted);
  // (a pair frees TMEM together, and what a bulk copy reads stays until it has arrived)
  if (PAIR || (p.bulk && ctas > 1)) cluster_sync_all();
}

template <int BLOCK, bool PAIR, int DT, int FUSED>
int launch_cluster(const CUtensorMap* maps, const FpParams& p, int grid, size_t smem, cudaStream_t stream) {
  static std::atomic<uint64_t> prepared{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_failure(e, "fp4_cluster_kernel device");
  if (dev >= 64 || !((prepared.load(std::memory_order_acquire) >> dev) & 1)) {
    e = cudaFuncSetAttribute(fp4_cluster_kernel<BLOCK, PAIR, DT, FUSED>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemLimit);
    if (e != cudaSuccess) return cuda_failure(e, "fp4_cluster_kernel attribute");
    if (dev < 64) prepared.fetch_or((uint64_t)1 << dev, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(threads_of(PAIR, FUSED >= 0));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  int n = 0;
  const int ctas = PAIR ? 2 * p.S : p.S;
  if (ctas > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)ctas;
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
  e = cudaLaunchKernelEx(&cfg, fp4_cluster_kernel<BLOCK, PAIR, DT, FUSED>, maps[0], maps[1], maps[2], maps[3], p);
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    return cuda_failure(e, "fp4_cluster_kernel launch");
  }
  return ADAPTION_OK;
}

template <int BLOCK, bool PAIR>
int launch_cluster(const CUtensorMap* maps, const FpParams& p, int grid, size_t smem, cudaStream_t stream) {
  if (p.y_dtype == ADAPTION_F32) return launch_cluster<BLOCK, PAIR, ADAPTION_F32, -1>(maps, p, grid, smem, stream);
  if (p.y_dtype == ADAPTION_F16) return launch_cluster<BLOCK, PAIR, ADAPTION_F16, -1>(maps, p, grid, smem, stream);
  return launch_cluster<BLOCK, PAIR, ADAPTION_BF16, -1>(maps, p, grid, smem, stream);
}
template <int BLOCK>
int launch_fused(const CUtensorMap* maps, const FpParams& p, int x_dtype, int grid, size_t smem, cudaStream_t stream) {
  if (x_dtype == ADAPTION_F32) return launch_cluster<BLOCK, false, -1, ADAPTION_F32>(maps, p, grid, smem, stream);
  if (x_dtype == ADAPTION_F16) return launch_cluster<BLOCK, false, -1, ADAPTION_F16>(maps, p, grid, smem, stream);
  return launch_cluster<BLOCK, false, -1, ADAPTION_BF16>(maps, p, grid, smem, stream);
}

// Clusters of `ctas` blocks, one block per SM, that the current device runs at a time.  (A cluster stays inside one group of SMs, so
// there are fewer than SMs / ctas: 74 of 2, 33 of 4, 22 of 6, 15 of 8 on 148 SMs.)  Asked once per device and size; a guess where the
// device does not answer.
int max_clusters(int dev, int sms, int ctas) {
  constexpr int kMaxDevices = 64, kMaxCtas = 8;
  static std::atomic<int> known[kMaxDevices][kMaxCtas + 1];
  if (ctas == 1) return sms;
  std::atomic<int> nowhere{0};
  const int guess = sms / (ctas > 4 ? ctas + 1 : ctas);
  return remembered(dev < kMaxDevices ? known[dev][ctas] : nowhere, guess > 1 ? guess : 1, [ctas]() {
    int n = 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(threads_of(true, false));
    cfg.dynamicSmemBytes = kSmemLimit;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const auto kernel = fp4_cluster_kernel<16, true, ADAPTION_BF16, -1>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemLimit) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
      (void)cudaGetLastError();
      return 0;
    }
    return n;
  });
}

// Whether two single CTAs that wait for no other one fit on an SM, each with a ring of three stages or more: their ring's bytes.
constexpr int64_t kHalfRing = (int64_t)(kSmemLimit / 2) - 2048;
bool two_share_an_sm(int64_t stage_bytes) { return kHalfRing / stage_bytes >= 3; }

struct FpPlan {
  bool pair = false, persistent = false;
  int S = 1, BN = 16;
  double cycles = 1e300;
};

// Estimated cycles.  The form is that of the kernels: a k-block takes the time of its copies (an SM's share of L2's reads) or of its
// MMAs, all operand bytes come from HBM at 3950 bytes a cycle at most, or 100 per SM at work; then the sums of the columns are exchanged and
// stored.  The constants are fitted to 395 runs, every number of shares of every form at 65 sizes from 1 to 4096 rows: 11 % off on
// average, and the choice 1 % behind the best one, at most 13 % (in graphs, three sets of operands in turn: 256 x 25088 -> 4096 17.6 us, the best
// 17.6; 256 x 4096 -> 4096 6.5, the best 6.5; 777 x 1411 -> 2049 6.1, the best 6.1; 4096 x 1024 -> 1024 6.4, the best 5.7).
// quantizes: the activations may be quantized in single CTAs' rings, where a k-block takes 300 cycles and 65 a row at least (25088 -> 4096,
// one row, the same way: four shares 13.9 us, three 15.8; of 4-bit operands 12.3 and 12.5).
FpPlan make_plan(const Fp4Problem& g, int only_pair, bool quantizes) {
  constexpr double kStart = 3500;              // of a launch's or a wave's blocks, until their first k-block
  FpPlan best;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) dev = 64;
  const int sms = num_sms(), kb = (int)((g.K + kBlockElems - 1) / kBlockElems), sf = groups_of(g.w.block) * kFp4TileBytes;
  for (int form = 0; form < 3; ++form) {
    // single CTAs; pairs on up to 256 columns, and on 128 of more
    const bool pair = form > 0;
    if ((only_pair >= 0 && pair != (only_pair != 0)) || (form == 2 && g.B <= kRows) || (quantizes && pair)) continue;
    const int tile_o = pair ? 2 * kRows : kRows, per = pair ? 2 : 1, most = form == 1 ? 2 * kRows : kRows;
    const int64_t bn = g.B < most ? (g.B + 15) / 16 * 16 : most;
    const int64_t tiles = ((g.O + tile_o - 1) / tile_o) * ((g.B + bn - 1) / bn);
    const int64_t stage = kABytes + bn / per * kBlockBytes + sf * (1 + (bn + kRows - 1) / kRows);
    const double mma = quantizes ? 300.0 + 65.0 * (double)(g.B < bn ? g.B : bn) : 4.0 * (bn > 170 ? (double)bn / 2 : 85.0);
    const double block = (double)stage / 75 > mma ? (double)stage / 75 : mma;
    const double operands = (double)g.K * ((double)g.O + (double)g.B) * (0.5 + 1.0 / g.w.block);
    for (int S = 1; S * per <= 8 && S <= kb; ++S) {
      const int64_t at_once = max_clusters(dev, sms, S * per);
      const bool two = !pair && S == 1 && tiles > at_once && two_share_an_sm(stage);
      const double waves = two ? (double)((tiles + 2 * at_once - 1) / (2 * at_once)) : (double)((tiles + at_once - 1) / at_once);
      const double exchange = (double)bn * (S > 1 ? 0.5 + 100.0 * (S - 1) / S : (two ? 42.0 : 14.0)) + (pair ? 1950.0 : 0.0);
      const double ctas = (double)(tiles < at_once ? tiles : at_once) * S * per, all = operands / (ctas * 100.0 < 3950.0 ? ctas * 100.0 : 3950.0);
      const double main_loop = waves * (two ? 2.0 : 1.0) * (double)((kb + S - 1) / S) * block;
      const double cycles = (main_loop > all ? main_loop : all) + waves * (exchange + kStart);
      if (cycles < best.cycles) {
        best.pair = pair;
        best.S = S;
        best.BN = (int)bn;
        best.cycles = cycles;
      }
    }
  }
  if (only_pair < 0 && g.B > kRows && !quantizes) {
    // the persistent kernel: tiles of 256 x 256 in turn, the stores of all but the last behind the next one's main loop
    const int64_t tiles = ((g.O + 255) / 256) * ((g.B + 255) / 256), pairs = sms / 2;
    const double bytes = 2.0 * kABytes + 3.0 * sf, block = bytes / 65 > 512 ? bytes / 65 : 512;
    const double cycles = (double)((tiles + pairs - 1) / pairs) * (kb * block + 3400.0) + 5000.0 + kStart;
    if (cycles < best.cycles) {
      best.persistent = true;
      best.cycles = cycles;
    }
  }
  return best;
}

int launch_fp4_cluster(const Fp4Problem& g, const FpPlan& plan) {
  const bool pair = plan.pair, fused = g.x.codes == nullptr;
  const int block = g.w.block, kgroups = groups_of(block);
  FpParams p;
  std::memset(&p, 0, sizeof(p));
  p.O = (int)g.O;
  p.B = (int)g.B;
  const int tile_o = pair ? 2 * kRows : kRows;
  p.tiles_o = (p.O + tile_o - 1) / tile_o;
  // (several column tiles: whole scale tiles each; a pair's half of the columns is a multiple of 8)
  p.BN = plan.BN;
  const int64_t tiles = (int64_t)p.tiles_o * ((p.B + p.BN - 1) / p.BN);
  p.chunks_b = (p.BN + kRows - 1) / kRows;
  p.num_kb = (int)((g.K + kBlockElems - 1) / kBlockElems);
  const int k_last = (int)(g.K - (int64_t)(p.num_kb - 1) * kBlockElems);
  p.steps_last = (k_last + kStepElems - 1) / kStepElems;
  const int64_t groups = fp4_groups(g.K, block);
  p.groups_last = (int)(groups - (int64_t)(p.num_kb - 1) * kgroups);
  const int per = pair ? 2 : 1;
  p.S = plan.S;
  p.kb_per_split = (p.num_kb + p.S - 1) / p.S;
  if (tiles * per * p.S > 0x7fffffff) return ADAPTION_ERR_UNSUPPORTED;
  const int b_rows = pair ? p.BN / 2 : p.BN;
  p.b_bytes = (uint32_t)b_rows * kBlockBytes;
  p.stage_bytes = kABytes + p.b_bytes + (uint32_t)(kgroups * kFp4TileBytes * (1 + p.chunks_b));
  const int col4 = ((p.BN < p.B ? p.BN : p.B) + 3) / 4;
  p.early = g.x_follows ? 1 : 0;
  p.max_runs = (col4 + p.S - 1) / p.S;
  p.bulk = p.S > 1 && col4 > 8 ? 1 : 0;
  for (int r = 0; r < 8 && r < col4; ++r) p.owners |= (uint32_t)(r / p.max_runs) << (4 * r);
  // sums that a CTA receives, behind its own
  const size_t received = p.S > 1 ? (size_t)(p.bulk ? p.S - 1 : p.S) * p.max_runs * kRunBytes : 0;
  p.sf_col = (uint32_t)(p.BN + 31) / 32 * 32;
  const uint32_t slot = (uint32_t)kgroups * 4u * (uint32_t)(1 + p.chunks_b);
  int stages = (int)((kSmemLimit - 1024 - (p.bulk ? 0 : received)) / p.stage_bytes);
  // more blocks than SMs: two share one, if that leaves each a ring of three stages
  if (per * p.S == 1 && tiles > num_sms() && two_share_an_sm(p.stage_bytes) && p.sf_col + 3u * slot <= 256u) {
    stages = (int)(kHalfRing / p.stage_bytes);
    while (p.sf_col + (uint32_t)stages * slot > 256u) --stages;
  }
  if (stages > kMaxStages) stages = kMaxStages;
  if (stages > p.kb_per_split) stages = p.kb_per_split;
  while (stages > 1 && p.sf_col + (uint32_t)stages * slot > 512u) --stages;
  p.stages = stages;
  p.tmem_cols = 32;
  while (p.tmem_cols < p.sf_col + (uint32_t)stages * slot) p.tmem_cols *= 2;
  size_t smem = (size_t)stages * p.stage_bytes;
  if (p.bulk) {
    const size_t sums = (size_t)p.BN / 4 * kRunBytes;       // of all columns, where the ring was
    p.recv_offset = (uint32_t)sums;
    if (smem < sums + received) smem = sums + received;
  } else {
    p.recv_offset = (uint32_t)smem;
    smem += received;
  }
  smem += 1024;
  // CTAs that wait for one another take all of an SM's shared memory, so that no block with TMEM columns lies beside them: two clusters
  // (of two streams, say, one of them a layer's) that each hold columns which a CTA of the other one waits for would never end.  (Where
  // the next call's blocks could come beside them, 4096 -> 4096 of one row with two sets of weights in L2 took 3.6 us in a graph instead of 4.2; others the same.)
  if (per * p.S > 1) smem = kSmemLimit;
  p.unit = pow2_float(g.x.exp + g.w.exp);
  p.bias = g.bias;
  p.relu = g.relu ? 1 : 0;
  p.y = (uint8_t*)g.y.data;
  p.y_pitch = g.y.stride * dtype_size(g.y.dtype);
  p.y_dtype = g.y.dtype;
  p.stats = g.stats;
  p.timeout_ns = wait_limit_ns();
  p.stall_at = knob(kStallAt);
  if (!load_tensor_map_encoders()) return ADAPTION_ERR_CUDA;
  CUtensorMap maps[4];
  bool ok = encode_fp4_codes(&maps[0], g.w, p.O, g.K, kRows, true) && encode_fp4_scales(&maps[2], g.w, p.O, groups, 1);
  if (fused) {
    maps[1] = maps[0];          // (not used)
    maps[3] = maps[2];
    p.x = (const uint8_t*)g.x_real.data;
    p.x_pitch = g.x_real.stride * dtype_size(g.x_real.dtype);
    p.x_aligned = aligned16(p.x) && (p.x_pitch & 15) == 0;
    p.K = (int)g.K;
    p.inv_unit = pow2_float(-g.x.exp);
    p.step_unit = pow2_float(g.x.exp);
  } else {
    ok = ok && encode_fp4_codes(&maps[1], g.x, p.B, g.K, (uint32_t)b_rows, false) && encode_fp4_scales(&maps[3], g.x, p.B, groups, (uint32_t)p.chunks_b);
  }
  if (!ok) return ADAPTION_ERR_CUDA;
  const int grid = (int)(tiles * per * p.S);
  if (fused)
    return block == 32 ? launch_fused<32>(maps, p, g.x_real.dtype, grid, smem, g.stream) : launch_fused<16>(maps, p, g.x_real.dtype, grid, smem, g.stream);
  if (pair) return block == 32 ? launch_cluster<32, true>(maps, p, grid, smem, g.stream) : launch_cluster<16, true>(maps, p, grid, smem, g.stream);
  return block == 32 ? launch_cluster<32, false>(maps, p, grid, smem, g.stream) : launch_cluster<16, false>(maps, p, grid, smem, g.stream);
}

}  // namespace

// Whether the product quantizes the activations itself.  To 4096 channels, one call after the other, against a launch of its own: 4096
// elements, one row 6.5 us against 9.3, eight 6.0 against 7.0, sixteen 6.9 against 6.9 (in a graph 6.8 against 5.6); 25088 elements, one row
// 14.0 against 14.6, four 14.8 against 15.2, eight 16.1 against 15.4, sixteen 23 against 15.4; 12800, four 9.2 against 10.6, eight 9.8 against 8.9.
// To more channels, where more tiles quantize the same rows, the rule is up to 13 % behind the better form (weights not in L2): eight
// rows of 4096 to 11008 channels 12.1 against 10.7, to 28672 17.0 against 16.5, of 2048 to 57344 18.9 against 17.0; one of 4096 to 28672 14.2
// against 15.6.
static bool few_rows(const Fp4Problem& g) { return g.B <= (g.K <= 8192 ? 8 : 4); }

// The plan goes by the sizes (and the device) alone, not by where the activations are quantized: with few rows the product of 4-bit operands takes the
// plan of the one that quantizes, so that both give the same bits.
static FpPlan choose_plan(const Fp4Problem& g) {
  // (tests: one cluster per tile of single CTAs or of pairs, or the persistent kernel, wherever the call would run)
  const int pair = knob(kPair);
  FpPlan plan;
  if (pair == 1 && knob(kCluster) != 2) {
    plan.persistent = true;
    return plan;
  }
  plan = make_plan(g, pair, few_rows(g) && pair != 1);
  const int shares = knob(kClusterSize) / (plan.pair ? 2 : 1), most = plan.pair ? 4 : 8;
  if (shares > 0) plan.S = shares < most ? shares : most;
  if (knob(kClusterBN) == 128 && plan.pair && g.B > kRows) plan.BN = kRows;
  if (knob(kClusterBN) == 256 && plan.pair && g.B > kRows) plan.BN = g.B < 2 * kRows ? (int)(g.B + 15) / 16 * 16 : 2 * kRows;
  return plan;
}

static int run_plan(const Fp4Problem& g, const FpPlan& plan) {
  return plan.persistent ? launch_fp4_pair(g) : launch_fp4_cluster(g, plan);
}

int fp4_ip_impl(const Fp4Problem& g) { return run_plan(g, choose_plan(g)); }

int fp4_act_ip_impl(Fp4Problem& g, const adaption_fp4tensor& workspace) {
  const int mode = knob(kFused);
  const FpPlan plan = choose_plan(g);
  if ((mode == 2 || (mode == 1 && few_rows(g))) && !plan.persistent && !plan.pair) {
    g.x = workspace;
    g.x.codes = nullptr;
    return launch_fp4_cluster(g, plan);
  }
  g.x = workspace;
  g.x_follows = true;
  const int rc = fp4_quantize_impl(g.x_real, nullptr, (size_t)g.B, (size_t)g.K, 0, g.x, nullptr, g.stream);
  return rc != ADAPTION_OK ? rc : run_plan(g, plan);
}

}  // namespace adaption
