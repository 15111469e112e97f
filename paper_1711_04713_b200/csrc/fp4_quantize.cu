// Microscaled 4-bit floating point: the quantizer and its inverse (adaption_fp4_quantize, adaption_fp4_dequantize).
//
// Both are one pass over memory.  A lane takes a chunk of 32 bytes of a row's real values (8 or 16 elements); the lanes of a
// block, at most four, find its maximum with shuffles, so that the values are read once and stay in registers.
//
// Bound by HBM (in graphs; call after call 0.5 us more): 200704 x 256 fp32 into blocks of 32 34.0 us (6.85 TB/s), its values 36.9 (6.3 TB/s; to bf16
// 6.5).  16-bit sources into blocks of 16 by instructions as well: 4096 x 25088 bf16 45.8 us (5.75 TB/s, 11 instructions an element, issue slots 73 % busy).
#include "fp4_quant.cuh"

namespace adaption {

int check_fp4(const adaption_fp4tensor& t, int64_t inner) {
  if (t.block != 16 && t.block != 32) return ADAPTION_ERR_INVALID_ARG;
  if (t.block == 32 ? t.exp != 0 : (t.exp < -63 || t.exp > 63)) return ADAPTION_ERR_INVALID_ARG;
  if (t.codes == nullptr || t.scales == nullptr) return ADAPTION_ERR_INVALID_ARG;
  if (t.c_stride < inner || (t.c_stride & 31) != 0) return ADAPTION_ERR_INVALID_ARG;
  if (t.c_stride > 2 * kFp4MaxInner) return ADAPTION_ERR_UNSUPPORTED;
  if (!aligned16(t.codes) || !aligned16(t.scales)) return ADAPTION_ERR_ALIGNMENT;
  return ADAPTION_OK;
}

int check_matrix(const adaption_matrix& m, int64_t inner) {
  if (m.dtype != ADAPTION_F32 && m.dtype != ADAPTION_F16 && m.dtype != ADAPTION_BF16) return ADAPTION_ERR_INVALID_ARG;
  if (m.data == nullptr || m.stride < inner) return ADAPTION_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(m.data) & (uintptr_t)(dtype_size(m.dtype) - 1)) != 0) return ADAPTION_ERR_ALIGNMENT;
  return ADAPTION_OK;
}

namespace {

constexpr int kThreads = 128;        // of the quantizer (with 256 and 62 % of the warps 200704 x 256 fp32 took 38.2 us, before other changes, instead of 35.3)
constexpr int kValueThreads = 256;
constexpr int kAhead = 2;            // chunks of a thread whose loads are in flight together, where rows are aligned

enum Source { kF32 = ADAPTION_F32, kF16 = ADAPTION_F16, kBF16 = ADAPTION_BF16, kPlanes = 3 };

// Elements of a chunk: what a lane takes at once, 32 bytes of x or of y.
__host__ __device__ constexpr int chunk_of(int source) { return source == kF32 ? 8 : 16; }

// Division of numbers below 2^30 by a fixed one below 2^30.
struct Divider {
  uint32_t d, mul, shift;
};
Divider make_divider(uint32_t d) {
  // floor(n / d) = (2 n * mul) >> (32 + shift) with mul = ceil(2^(31 + shift) / d), shift = floor(log2 d): mul * d exceeds 2^(31 + shift) by
  // e < d < 2^(shift + 1), so the product is n / d + (n e / 2^(31 + shift)) / d, less than 1 / d too large
  uint32_t shift = 0;
  while ((d >> (shift + 1)) != 0) ++shift;
  const uint64_t p = (uint64_t)1 << (31 + shift);
  return Divider{d, (uint32_t)((p + d - 1) / d), shift};
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const Divider& v) { return __umulhi(n + n, v.mul) >> v.shift; }

// Bytes of `a` by selector; one with bit 3 set is eight times the byte's sign.
__device__ __forceinline__ uint32_t with_signs(uint32_t a, uint32_t selector) {
  uint32_t r;
  asm("prmt.b32 %0, %1, 0, %2;" : "=r"(r) : "r"(a), "r"(selector));
  return r;
}

struct QuantParams {
  const uint8_t* x;             // real values, or the low plane
  const uint8_t* hi;            // high plane or null
  int64_t pitch;                // of a row of x (of a plane), in bytes
  float unit;                   // 2^-frac_bits of a fixed-point tensor
  int aligned32;
  uint8_t* codes;
  uint8_t* scales;
  uint32_t row_bytes;           // of the codes
  int groups;
  uint32_t total;               // chunks of all rows
  Divider chunks;               // ... of one row
  int inner, c_stride, blocks4; // blocks4: blocks of a row, filled up to whole scale tiles
  float inv_unit, step_unit;    // 2^-exp, 2^exp
  int relu;
  adaption_stats* stats;
};

// The first n elements of a chunk as raw words (what lies behind them is undefined).
template <int SRC, bool ALIGNED>
__device__ __forceinline__ void load_chunk(const QuantParams& p, uint32_t row, int col, int n, uint32_t (&w)[8]) {
  constexpr int kVec = chunk_of(SRC), kSize = SRC == kF32 ? 4 : 2;
  if (SRC == kPlanes) {
    // (planes are 16-byte aligned, pitches a multiple of 16, and cover their padding)
    uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
    if (n > 0) {
      lo = __ldcs(reinterpret_cast<const uint4*>(p.x + (int64_t)row * p.pitch + col));
      if (p.hi != nullptr) hi = __ldcs(reinterpret_cast<const uint4*>(p.hi + (int64_t)row * p.pitch + col));
    }
    w[0] = lo.x; w[1] = lo.y; w[2] = lo.z; w[3] = lo.w;
    w[4] = hi.x; w[5] = hi.y; w[6] = hi.z; w[7] = hi.w;
    return;
  }
  const uint8_t* at = p.x + (int64_t)row * p.pitch + (int64_t)col * kSize;
  if (ALIGNED && n >= kVec)
    load_words(at, p.aligned32 != 0, w);
  else
    load_shifted(at, min(n, kVec) * kSize, w);
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// max(a, |b|) of two pairs of 16-bit numbers, a >= 0; a NaN stays one.
template <bool HALF>
__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {
  uint32_t r;
  if (HALF) asm("{\n.reg .b32 t;\nabs.f16x2 t, %2;\nmax.NaN.f16x2 %0, %1, t;\n}\n" : "=r"(r) : "r"(a), "r"(b));
  else asm("{\n.reg .b32 t;\nabs.bf16x2 t, %2;\nmax.NaN.bf16x2 %0, %1, t;\n}\n" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Quantizes one chunk; every lane of the warp comes along (n = 0: nothing to quantize, but codes and scales of the padding).
template <int SRC, int BLOCK>
__device__ __forceinline__ void quantize_chunk(const QuantParams& p, bool real, uint32_t row, int col, int n, uint32_t (&w)[8],
                                               Counts& cnt) {
  constexpr int kVec = chunk_of(SRC);
  float v[kVec];
  float top = 0.f;
  if (SRC == kPlanes) {
    // pairs of 16-bit integers from the planes' bytes (the sign repeated where there is one plane), their range, and each as
    // a float: q + 2^15 behind the exponent of 2^23, less 2^23 + 2^15
    uint32_t q[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t lo = w[k >> 1], hi = w[4 + (k >> 1)];
      q[k] = p.hi != nullptr ? __byte_perm(lo, hi, k & 1 ? 0x7362 : 0x5140) : with_signs(lo, k & 1 ? 0xb3a2u : 0x9180u);
    }
    if (n < kVec) {
#pragma unroll
      for (int k = 0; k < 8; ++k) q[k] &= 2 * k + 1 < n ? 0xffffffffu : (2 * k < n ? 0xffffu : 0u);
    }
    uint32_t most = 0u, least = 0u;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (p.relu) q[k] = __vmaxs2(q[k], 0u);
      most = __vmaxs2(most, q[k]);
      least = __vmins2(least, q[k]);
      q[k] ^= 0x80008000u;
    }
    int m = max(max((int)(int16_t)(most & 0xffffu), (int)most >> 16), -min((int)(int16_t)(least & 0xffffu), (int)least >> 16));
#pragma unroll
    for (int o = 1; o < BLOCK / kVec; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    top = (float)m * p.unit;
    const float less = -8421376.f * p.unit;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[2 * k] = fmaf(__uint_as_float(__byte_perm(q[k], 0x4b000000u, 0x7610)), p.unit, less);
      v[2 * k + 1] = fmaf(__uint_as_float(__byte_perm(q[k], 0x4b000000u, 0x7632)), p.unit, less);
    }
  } else if (SRC == kF32) {
    if (n < kVec) {
#pragma unroll
      for (int k = 0; k < kVec; ++k)
        if (k >= n) w[k] = 0u;
    }
    // (relu: what has a sign is negative as a whole number too; a NaN stays one in the maximum)
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      if (p.relu) w[k] = (uint32_t)max((int32_t)w[k], 0);
      v[k] = __uint_as_float(w[k]);
      top = max_nan(top, fabsf(v[k]));
    }
#pragma unroll
    for (int o = 1; o < BLOCK / kVec; o <<= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  } else {
    // two at a time; magnitudes are in order as 16-bit numbers, NaN above them all; relu: what has a sign is negative as a 16-bit number too
    uint32_t m = 0u;
    if (n < kVec) {
#pragma unroll
      for (int k = 0; k < kVec / 2; ++k) w[k] &= 2 * k + 1 < n ? 0xffffffffu : (2 * k < n ? 0xffffu : 0u);
    }
#pragma unroll
    for (int k = 0; k < kVec / 2; ++k) {
      if (p.relu) w[k] = __vmaxs2(w[k], 0u);
      m = max_abs2<SRC == kF16>(m, w[k]);
    }
    m = max(m & 0xffffu, m >> 16);
#pragma unroll
    for (int o = 1; o < BLOCK / kVec; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
    for (int k = 0; k < kVec / 2; ++k) {
      if (SRC == kF16) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
        v[2 * k] = f.x;
        v[2 * k + 1] = f.y;
      } else {
        v[2 * k] = __uint_as_float(w[k] << 16);
        v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
      }
    }
    top = SRC == kF16 ? __half2float(__ushort_as_half((unsigned short)m)) : __uint_as_float(m << 16);
  }
  if (SRC != kPlanes) fp4_finite<BLOCK, kVec>(v, top);      // (a NaN fails its comparison)
  uint32_t code[kVec / 8];
  const uint32_t byte = fp4_encode<BLOCK, kVec, SRC != kF32>(v, top, p.inv_unit, p.step_unit, code);
  if (p.stats != nullptr) {
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      if (k < n) {
        cnt.zeros += ((code[k >> 3] >> (4 * (k & 7))) & 7u) == 0u;
        cnt.sat_pos += v[k] >= 7.f;
        cnt.sat_neg += v[k] <= -7.f;
      }
    }
  }
  if (real) {
    uint8_t* to = p.codes + (row * p.row_bytes + (uint32_t)(col >> 1));
    if (kVec == 16) *reinterpret_cast<uint2*>(to) = make_uint2(code[0], code[kVec / 8 - 1]);
    else *reinterpret_cast<uint32_t*>(to) = code[0];
  }
  const int j = col / BLOCK;
  if (real && (col & (BLOCK - 1)) == 0 && j < p.blocks4) {
    uint8_t* const to = p.scales + fp4_scale_offset(row, j, p.groups);
    *to = (uint8_t)byte;
    // the last block of the pitch: zeros in the rest of the scale tile
    if (col + BLOCK >= p.c_stride)
      for (int k = 1; j + k < p.blocks4; ++k) to[k] = 0;
  }
}

template <int SRC, int BLOCK, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, SRC == kF32 ? 12 : 10) fp4_quantize_kernel(const QuantParams p) {
  pdl_prologue();
  constexpr int kVec = chunk_of(SRC), kChunks = ALIGNED ? kAhead : 1;
  Counts cnt;
  uint32_t w[kChunks][8], row[kChunks];
  int col[kChunks];
  bool real[kChunks];
  const uint32_t base = blockIdx.x * (kThreads * kChunks) + threadIdx.x;
#pragma unroll
  for (int u = 0; u < kChunks; ++u) {
    const uint32_t t = base + u * kThreads;
    real[u] = t < p.total;
    row[u] = real[u] ? divide(t, p.chunks) : 0u;
    col[u] = real[u] ? (int)(t - row[u] * p.chunks.d) * kVec : 0;
    load_chunk<SRC, ALIGNED>(p, row[u], col[u], real[u] ? p.inner - col[u] : 0, w[u]);
  }
#pragma unroll
  for (int u = 0; u < kChunks; ++u)
    quantize_chunk<SRC, BLOCK>(p, real[u], row[u], col[u], real[u] ? p.inner - col[u] : 0, w[u], cnt);
  if (p.stats != nullptr) flush_counts_block(cnt, p.stats);
}

struct ValueParams {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t row_bytes;
  int groups;
  uint32_t total;
  Divider chunks;
  int inner;
  float unit;                   // 2^exp
  int aligned32;
  uint8_t* y;
  int64_t pitch;                // of a row of y, in bytes
};

__device__ __forceinline__ void store_words(void* to, bool aligned32, const uint32_t (&w)[8]) {
  if (aligned32) {
    asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    __stcs(reinterpret_cast<uint4*>(to), make_uint4(w[0], w[1], w[2], w[3]));
    __stcs(reinterpret_cast<uint4*>(to) + 1, make_uint4(w[4], w[5], w[6], w[7]));
  }
}
template <int BLOCK>
__device__ __forceinline__ float step_of(const ValueParams& p, uint32_t byte) {
  if (BLOCK == 32) return e8m0_value(byte);
  return (byte & 127u) == 127u ? __uint_as_float(0x7fc00000u) : e4m3_value(byte & 127u) * p.unit;
}

// Rows of y on 16-byte boundaries: a lane takes a chunk of codes, which lies in one block.
template <int DT, int BLOCK>
__global__ void __launch_bounds__(kValueThreads) fp4_values_kernel(const ValueParams p) {
  pdl_prologue();
  constexpr int kVec = chunk_of(DT);
  uint32_t code[kAhead][kVec / 8], byte[kAhead], row[kAhead];
  int col[kAhead];
  const uint32_t base = blockIdx.x * (kValueThreads * kAhead) + threadIdx.x;
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const uint32_t t = base + u * kValueThreads;
    row[u] = t < p.total ? divide(t, p.chunks) : 0u;
    col[u] = t < p.total ? (int)(t - row[u] * p.chunks.d) * kVec : p.inner;
    if (col[u] < p.inner) {
      const uint8_t* at = p.codes + (int64_t)row[u] * p.row_bytes + (col[u] >> 1);
      if (kVec == 16) {
        const uint2 c = __ldg(reinterpret_cast<const uint2*>(at));
        code[u][0] = c.x;
        code[u][kVec / 8 - 1] = c.y;
      } else {
        code[u][0] = __ldg(reinterpret_cast<const uint32_t*>(at));
      }
      byte[u] = __ldg(p.scales + fp4_scale_offset(row[u], col[u] / BLOCK, p.groups));
    }
  }
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int n = p.inner - col[u];
    if (n <= 0) continue;
    const float s = step_of<BLOCK>(p, byte[u]);
    uint32_t w[8];
#pragma unroll
    for (int k = 0; k < kVec / 2; ++k) {
      const float2 f = __half22float2(fp4_unpack2((code[u][k >> 2] >> (8 * (k & 3))) & 255u));
      if (DT == kF32) {
        w[2 * k & 7] = __float_as_uint(f.x * s);
        w[(2 * k + 1) & 7] = __float_as_uint(f.y * s);
      } else {
        w[k] = pack2<DT>(f.x * s, f.y * s);
      }
    }
    uint8_t* to = p.y + (int64_t)row[u] * p.pitch + (int64_t)col[u] * (DT == kF32 ? 4 : 2);
    if (n >= kVec) {
      store_words(to, p.aligned32 != 0, w);
    } else {
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        if (k >= n) break;
        if (DT == kF32) reinterpret_cast<uint32_t*>(to)[k] = w[k & 7];
        else reinterpret_cast<uint16_t*>(to)[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
      }
    }
  }
}

// Rows of y anywhere: a lane takes an aligned 32-byte piece of y, whose elements start anywhere in a byte of codes and in a
// block.  `chunks` counts the pieces that a row can touch.  (One piece a lane: two in flight took 18.3 us for 4093 x 4099 fp32
// instead of 16.8.)
template <int DT, int BLOCK>
__global__ void __launch_bounds__(kValueThreads) fp4_values_shifted_kernel(const ValueParams p) {
  pdl_prologue();
  constexpr int kVec = chunk_of(DT), kSize = 32 / kVec, kWords = kVec / 8;
  const uint32_t t = blockIdx.x * kValueThreads + threadIdx.x;
  if (t >= p.total) return;
  const uint32_t row = divide(t, p.chunks);
  uint8_t* const y = p.y + (int64_t)row * p.pitch;
  const int off = (int)(reinterpret_cast<uintptr_t>(y) & 31u) / kSize;
  const int col = (int)(t - row * p.chunks.d) * kVec - off;         // negative: the piece begins before the row
  const int c0 = max(col, 0), c1 = min(col + kVec, p.inner) - 1;    // first and last element of the piece that exist
  if (c0 > c1) return;
  const uint32_t* const codes = reinterpret_cast<const uint32_t*>(p.codes + (int64_t)row * p.row_bytes) + (c0 >> 3);
  const int more = (c1 >> 3) - (c0 >> 3);
  uint32_t code[kWords + 1];
#pragma unroll
  for (int i = 0; i <= kWords; ++i) code[i] = i <= more ? __ldg(codes + i) : 0u;
  const int j0 = c0 / BLOCK, j1 = c1 / BLOCK;
  const uint32_t byte0 = __ldg(p.scales + fp4_scale_offset(row, j0, p.groups));
  const uint32_t byte1 = j1 == j0 ? byte0 : __ldg(p.scales + fp4_scale_offset(row, j1, p.groups));
  const float s0 = step_of<BLOCK>(p, byte0), s1 = step_of<BLOCK>(p, byte1);
  const int border = j1 * BLOCK - c0;                               // elements from here on lie in the second block
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    const uint32_t eight = __funnelshift_r(code[i], code[i + 1], 4 * (c0 & 7));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = 8 * i + 2 * k;
      const float2 f = __half22float2(fp4_unpack2((eight >> (8 * k)) & 255u));
      const float a = f.x * (e < border ? s0 : s1), b = f.y * (e + 1 < border ? s0 : s1);
      if (DT == kF32) {
        w[e & 7] = __float_as_uint(a);
        w[(e + 1) & 7] = __float_as_uint(b);
      } else {
        w[e >> 1] = pack2<DT>(a, b);
      }
    }
  }
  uint8_t* const to = y + (int64_t)c0 * kSize;
  const int n = c1 - c0 + 1;
  if (n == kVec) {
    store_words(to, true, w);
  } else {
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      if (k >= n) break;
      if (DT == kF32) reinterpret_cast<uint32_t*>(to)[k] = w[k & 7];
      else reinterpret_cast<uint16_t*>(to)[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
    }
  }
}

unsigned blocks_of(uint32_t total, int per_block) { return (total + (uint32_t)per_block - 1) / (uint32_t)per_block; }

template <int SRC, int BLOCK, bool ALIGNED>
int launch_quantize(const QuantParams& p, cudaStream_t stream) {
  const dim3 grid(blocks_of(p.total, kThreads * (ALIGNED ? kAhead : 1))), block(kThreads);
  return cuda_status(launch_after_predecessor(fp4_quantize_kernel<SRC, BLOCK, ALIGNED>, grid, block, stream, p), "fp4_quantize_kernel launch");
}
// (planes always lie on 16-byte boundaries)
template <int SRC, int BLOCK>
int launch_quantize(const QuantParams& p, bool aligned, cudaStream_t stream) {
  if constexpr (SRC != kPlanes) {
    if (!aligned) return launch_quantize<SRC, BLOCK, false>(p, stream);
  }
  return launch_quantize<SRC, BLOCK, true>(p, stream);
}
template <int SRC>
int launch_quantize(const QuantParams& p, int block, bool aligned, cudaStream_t stream) {
  return block == 32 ? launch_quantize<SRC, 32>(p, aligned, stream) : launch_quantize<SRC, 16>(p, aligned, stream);
}

template <int DT, int BLOCK>
int launch_values(const ValueParams& p, bool aligned, cudaStream_t stream) {
  const dim3 grid(blocks_of(p.total, kValueThreads * (aligned ? kAhead : 1))), block(kValueThreads);
  return cuda_status(aligned ? launch_after_predecessor(fp4_values_kernel<DT, BLOCK>, grid, block, stream, p)
                             : launch_after_predecessor(fp4_values_shifted_kernel<DT, BLOCK>, grid, block, stream, p),
                     "fp4_values_kernel launch");
}
template <int DT>
int launch_values(const ValueParams& p, int block, bool aligned, cudaStream_t stream) {
  return block == 32 ? launch_values<DT, 32>(p, aligned, stream) : launch_values<DT, 16>(p, aligned, stream);
}

// Rows per launch: chunks are counted below 2^27, so that offsets in codes and scales stay below 2^32.  A multiple of a scale tile's rows.
int64_t rows_per_launch(int64_t chunks) {
  const int64_t rows = (((int64_t)1 << 27) / chunks) & ~(int64_t)(kFp4TileRows - 1);
  return rows > kFp4TileRows ? rows : kFp4TileRows;
}

}  // namespace

int fp4_quantize_impl(const adaption_matrix& x, const adaption_qtensor* q, size_t outer, size_t inner, int32_t relu,
                      const adaption_fp4tensor& out, adaption_stats* stats, cudaStream_t stream) {
  if (outer == 0 || inner == 0) return ADAPTION_OK;
  if ((x.data == nullptr) == (q == nullptr)) return ADAPTION_ERR_INVALID_ARG;
  if (inner > (size_t)kFp4MaxInner || outer > (size_t)1 << 40) return ADAPTION_ERR_UNSUPPORTED;
  int rc = check_fp4(out, (int64_t)inner);
  if (rc != ADAPTION_OK) return rc;
  rc = q != nullptr ? check_qtensor_in(*q, (int64_t)inner) : check_matrix(x, (int64_t)inner);
  if (rc != ADAPTION_OK) return rc;
  if (!aligned_stats(stats)) return ADAPTION_ERR_ALIGNMENT;
  QuantParams p{};
  p.inner = (int)inner;
  p.c_stride = (int)out.c_stride;
  p.row_bytes = (uint32_t)(out.c_stride / 2);
  p.groups = (int)fp4_groups((int64_t)inner, out.block);
  p.blocks4 = p.groups * 4;
  p.inv_unit = pow2_float(-out.exp);
  p.step_unit = pow2_float(out.exp);
  p.relu = relu ? 1 : 0;
  p.stats = stats;
  const int vec = chunk_of(q != nullptr ? (int)kPlanes : x.dtype);
  p.chunks = make_divider((uint32_t)(out.c_stride / vec));
  bool aligned = true;
  if (q != nullptr) {
    p.x = (const uint8_t*)q->lo;
    p.hi = q->fmt.n_bits > 8 ? (const uint8_t*)q->hi : nullptr;
    p.pitch = q->c_stride;
    p.unit = pow2_float(-q->fmt.frac_bits);
  } else {
    p.x = (const uint8_t*)x.data;
    p.pitch = x.stride * dtype_size(x.dtype);
    aligned = aligned16(x.data) && (p.pitch & 15) == 0;
    p.aligned32 = ((reinterpret_cast<uintptr_t>(x.data) | (uintptr_t)p.pitch) & 31u) == 0;
  }
  p.codes = (uint8_t*)out.codes;
  p.scales = (uint8_t*)out.scales;
  const int64_t rows = rows_per_launch(p.chunks.d);
  for (int64_t r = 0; r < (int64_t)outer; r += rows) {
    const int64_t n = (int64_t)outer - r < rows ? (int64_t)outer - r : rows;
    p.total = (uint32_t)(n * p.chunks.d);
    if (q != nullptr) rc = launch_quantize<kPlanes>(p, out.block, aligned, stream);
    else if (x.dtype == ADAPTION_F32) rc = launch_quantize<kF32>(p, out.block, aligned, stream);
    else if (x.dtype == ADAPTION_F16) rc = launch_quantize<kF16>(p, out.block, aligned, stream);
    else rc = launch_quantize<kBF16>(p, out.block, aligned, stream);
    if (rc != ADAPTION_OK) return rc;
    p.x += n * p.pitch;
    if (p.hi != nullptr) p.hi += n * p.pitch;
    p.codes += n * p.row_bytes;
    p.scales += n / kFp4TileRows * (int64_t)p.groups * kFp4TileBytes;
  }
  return ADAPTION_OK;
}

int fp4_dequantize_impl(const adaption_fp4tensor& x, size_t outer, size_t inner, const adaption_matrix& y,
                        cudaStream_t stream) {
  if (outer == 0 || inner == 0) return ADAPTION_OK;
  if (inner > (size_t)kFp4MaxInner || outer > (size_t)1 << 40) return ADAPTION_ERR_UNSUPPORTED;
  int rc = check_fp4(x, (int64_t)inner);
  if (rc != ADAPTION_OK) return rc;
  rc = check_matrix(y, (int64_t)inner);
  if (rc != ADAPTION_OK) return rc;
  ValueParams p{};
  p.inner = (int)inner;
  p.row_bytes = x.c_stride / 2;
  p.groups = (int)fp4_groups((int64_t)inner, x.block);
  p.unit = pow2_float(x.exp);
  p.codes = (const uint8_t*)x.codes;
  p.scales = (const uint8_t*)x.scales;
  p.y = (uint8_t*)y.data;
  p.pitch = y.stride * dtype_size(y.dtype);
  const bool aligned = aligned16(y.data) && (p.pitch & 15) == 0;
  p.aligned32 = ((reinterpret_cast<uintptr_t>(y.data) | (uintptr_t)p.pitch) & 31u) == 0;
  const int64_t vec = chunk_of(y.dtype);
  // (a row off the boundary can touch one piece more)
  p.chunks = make_divider((uint32_t)(((int64_t)inner + vec - 1) / vec + (aligned ? 0 : 1)));
  const int64_t rows = rows_per_launch(p.chunks.d);
  for (int64_t r = 0; r < (int64_t)outer; r += rows) {
    const int64_t n = (int64_t)outer - r < rows ? (int64_t)outer - r : rows;
    p.total = (uint32_t)(n * p.chunks.d);
    if (y.dtype == ADAPTION_F32) rc = launch_values<kF32>(p, x.block, aligned, stream);
    else if (y.dtype == ADAPTION_F16) rc = launch_values<kF16>(p, x.block, aligned, stream);
    else rc = launch_values<kBF16>(p, x.block, aligned, stream);
    if (rc != ADAPTION_OK) return rc;
    p.codes += n * p.row_bytes;
    p.scales += n / kFp4TileRows * (int64_t)p.groups * kFp4TileBytes;
    p.y += n * p.pitch;
  }
  return ADAPTION_OK;
}

}  // namespace adaption
