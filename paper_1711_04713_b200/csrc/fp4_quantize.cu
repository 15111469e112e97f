// Microscaled 4-bit floating point: the quantizer and its inverse (adaption_fp4_quantize, adaption_fp4_dequantize).
//
// Both are one pass over memory.  A lane takes eight consecutive elements of a row (16 bytes of a 16-bit type, 4 bytes of
// codes); the two or four lanes of a block find its maximum with shuffles, so that the values are read once and stay in
// registers.
//
// Quantizer.  With amax the block's maximum:
//   block 32: step 2^(floor(log2 amax) - 2).  The scale byte is amax's exponent field less 2 (a denormal amax has field 0,
//     and every step below 2^-127 is clamped there), and x / step is a product by a power of two: exact.
//   block 16: step s 2^exp with s = E4M3(amax 2^-exp / 6), and x / step is needed to the last bit of the decision between
//     two codes.  The quotient is rounded to 32 bits before it is rounded to E2M1; that gives the nearest code
//     all the same: a border m between two codes and the step have 3 and 4 significant bits, so m * step is a float, an x
//     off that border is off by one unit in its last place at least, and that moves x / step by more than half a unit in m's last
//     place (the step's significand is at most 1.875).  The division itself is q = x r, q += (x - q step) r with r the rounded reciprocal (Markstein, IBM J.
//     Res. Dev. 34, 1990: the residual is exact in one fused multiply-add), three operations an element.  The same argument holds for
//     amax / 6 against the borders of E4M3.
#include "fp4.cuh"

namespace adaption {

int num_sms();

int check_fp4(const adaption_fp4tensor& t, int64_t inner) {
  if (t.block != 16 && t.block != 32) return ADAPTION_ERR_INVALID_ARG;
  if (t.block == 32 ? t.exp != 0 : (t.exp < -64 || t.exp > 63)) return ADAPTION_ERR_INVALID_ARG;
  if (t.codes == nullptr || t.scales == nullptr) return ADAPTION_ERR_INVALID_ARG;
  if (t.c_stride < inner || (t.c_stride & 31) != 0) return ADAPTION_ERR_INVALID_ARG;
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

constexpr int kVec = 8;              // elements of a lane
constexpr int kThreads = 256;

enum Source { kF32 = ADAPTION_F32, kF16 = ADAPTION_F16, kBF16 = ADAPTION_BF16, kPlanes = 3 };

// Division of numbers below 2^30 by a fixed one below 2^30.
struct Divider {
  uint32_t d, mul, shift;
};
Divider make_divider(uint32_t d) {
  // floor(n / d) = (n * mul) >> shift with mul = ceil(2^shift / d), shift = 31 + floor(log2 d): mul * d exceeds 2^shift by
  // e < d < 2^(shift - 30), so the product is n / d + (n e / 2^shift) / d, less than 1 / d too large
  uint32_t shift = 31;
  while ((d >> (shift - 30)) != 0) ++shift;
  const uint64_t p = (uint64_t)1 << shift;
  return Divider{d, (uint32_t)((p + d - 1) / d), shift};
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const Divider& v) {
  return (uint32_t)(((uint64_t)n * v.mul) >> v.shift);
}

struct QuantParams {
  const void* x;                // real values, or the low plane
  const int8_t* hi;             // high plane or null
  int64_t stride;               // of a row of x, in elements
  float unit;                   // 2^-frac_bits of a fixed-point tensor
  uint8_t* codes;
  uint8_t* scales;
  int64_t row_bytes;            // of the codes
  int64_t groups;
  uint32_t total;               // eight-element chunks of all rows
  Divider chunks;               // ... of one row
  int inner, c_stride, blocks4; // blocks4: blocks of a row, filled up to whole scale tiles
  int exp, relu;
  adaption_stats* stats;
};

template <int SRC>
__device__ __forceinline__ float load_one(const QuantParams& p, int64_t i) {
  if (SRC == kF32) return reinterpret_cast<const float*>(p.x)[i];
  if (SRC == kF16) return __half2float(reinterpret_cast<const __half*>(p.x)[i]);
  if (SRC == kBF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.x)[i]);
  return (float)load_q(p.hi, reinterpret_cast<const uint8_t*>(p.x), (size_t)i) * p.unit;
}

// eight elements from i on, as one vector (two for 32-bit elements)
template <int SRC>
__device__ __forceinline__ void load_vector(const QuantParams& p, int64_t i, float (&v)[kVec]) {
  if (SRC == kF32) {
    const float4* q = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.x) + i);
    const float4 a = __ldg(q), b = __ldg(q + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else if (SRC == kF16 || SRC == kBF16) {
    const uint4 a = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p.x) + i));
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (SRC == kF16) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
        v[2 * k] = f.x;
        v[2 * k + 1] = f.y;
      } else {
        v[2 * k] = __uint_as_float(w[k] << 16);
        v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
      }
    }
  } else {
    const uint2 lo = __ldg(reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(p.x) + i));
    if (p.hi != nullptr) {
      const uint2 hi = __ldg(reinterpret_cast<const uint2*>(p.hi + i));
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        const uint32_t l = ((k < 4 ? lo.x : lo.y) >> (8 * (k & 3))) & 255u;
        const int32_t h = (int32_t)((k < 4 ? hi.x : hi.y) << (24 - 8 * (k & 3))) >> 24;
        v[k] = (float)(h * 256 + (int32_t)l) * p.unit;
      }
    } else {
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[k] = (float)((int32_t)((k < 4 ? lo.x : lo.y) << (24 - 8 * (k & 3))) >> 24) * p.unit;
    }
  }
}

template <int SRC, int BLOCK, bool VEC>
__global__ void __launch_bounds__(kThreads) fp4_quantize_kernel(const QuantParams p) {
  pdl_prologue();
  Counts cnt;
  const uint32_t step = gridDim.x * kThreads;
  // (whole warps take part in the shuffles; lanes behind the last chunk work on zeros)
  for (uint32_t base = blockIdx.x * kThreads; base < p.total; base += step) {
    const uint32_t t = base + threadIdx.x;
    const bool real = t < p.total;
    const uint32_t row = real ? divide(t, p.chunks) : 0u;
    const int col = real ? (int)(t - row * p.chunks.d) * kVec : p.inner;
    float v[kVec];
    const int64_t at = (int64_t)row * p.stride + col;
    if (VEC && col + kVec <= p.inner) {
      load_vector<SRC>(p, at, v);
    } else {
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[k] = col + k < p.inner ? load_one<SRC>(p, at + k) : 0.f;
    }
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      if (SRC != kPlanes) {
        // NaN -> 0, infinities -> the largest finite number (fmaxf / fminf give the other operand for NaN)
        v[k] = v[k] == v[k] ? fminf(fmaxf(v[k], -3.402823466e38f), 3.402823466e38f) : 0.f;
      }
      if (p.relu) v[k] = v[k] > 0.f ? v[k] : 0.f;
      top = fmaxf(top, fabsf(v[k]));
    }
#pragma unroll
    for (int o = 1; o < BLOCK / kVec; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));

    uint32_t byte;
    if (BLOCK == 32) {
      const int field = (int)(__float_as_uint(top) >> 23);
      byte = (uint32_t)max(field - 2, 0);
      const float inv = __uint_as_float((254u - byte) << 23);
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[k] *= inv;
    } else {
      byte = e4m3_nearest(__fdiv_rn(fminf(top * pow2_float(-p.exp), 3e38f), 6.f));
      const float s = e4m3_value(byte) * pow2_float(p.exp);
      const float r = s > 0.f ? __frcp_rn(s) : 0.f;
      if (top > 8.f * s) {
        // the largest scale was too small, or the smallest too large: beyond 8 steps all is clipped
#pragma unroll
        for (int k = 0; k < kVec; ++k) v[k] = fminf(fmaxf(v[k], -8.f * s), 8.f * s);
      }
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        const float q = v[k] * r;
        v[k] = copysignf(fmaf(fmaf(-q, s, v[k]), r, q), v[k]);
      }
    }
    uint32_t code = 0;
#pragma unroll
    for (int k = 0; k < kVec / 2; ++k) code |= fp4_pack2(v[2 * k], v[2 * k + 1]) << (8 * k);
    if (p.stats != nullptr) {
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        if (col + k < p.inner) {
          cnt.zeros += ((code >> (4 * k)) & 7u) == 0u;
          cnt.sat_pos += v[k] >= 7.f;
          cnt.sat_neg += v[k] <= -7.f;
        }
      }
    }
    if (real && col < p.c_stride) *reinterpret_cast<uint32_t*>(p.codes + (int64_t)row * p.row_bytes + (col >> 1)) = code;
    const int j = col / BLOCK;
    if (real && (col & (BLOCK - 1)) == 0 && j < p.blocks4) p.scales[fp4_scale_offset(row, j, p.groups)] = (uint8_t)byte;
  }
  if (p.stats != nullptr) flush_counts_block(cnt, p.stats);
}

struct ValueParams {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t row_bytes, groups;
  uint32_t total;
  Divider chunks;
  int inner;
  float unit;                   // 2^exp
  void* y;
  int64_t stride;
};

template <int DT>
__device__ __forceinline__ void store_one(void* y, int64_t i, float v) {
  if (DT == kF32) reinterpret_cast<float*>(y)[i] = v;
  else if (DT == kF16) reinterpret_cast<__half*>(y)[i] = __float2half_rn(v);
  else reinterpret_cast<__nv_bfloat16*>(y)[i] = __float2bfloat16_rn(v);
}

template <int DT, int BLOCK, bool VEC>
__global__ void __launch_bounds__(kThreads) fp4_values_kernel(const ValueParams p) {
  pdl_prologue();
  const uint32_t step = gridDim.x * kThreads;
  for (uint32_t t = blockIdx.x * kThreads + threadIdx.x; t < p.total; t += step) {
    const uint32_t row = divide(t, p.chunks);
    const int col = (int)(t - row * p.chunks.d) * kVec;
    const uint32_t code = __ldg(reinterpret_cast<const uint32_t*>(p.codes + (int64_t)row * p.row_bytes + (col >> 1)));
    const uint32_t byte = __ldg(p.scales + fp4_scale_offset(row, col / BLOCK, p.groups));
    const float s = BLOCK == 32 ? e8m0_value(byte) : e4m3_value(byte) * p.unit;
    float v[kVec];
#pragma unroll
    for (int k = 0; k < kVec / 2; ++k) {
      const float2 f = __half22float2(fp4_unpack2((code >> (8 * k)) & 255u));
      v[2 * k] = f.x * s;
      v[2 * k + 1] = f.y * s;
    }
    const int64_t at = (int64_t)row * p.stride + col;
    if (VEC && col + kVec <= p.inner) {
      if (DT == kF32) {
        float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(p.y) + at);
        q[0] = make_float4(v[0], v[1], v[2], v[3]);
        q[1] = make_float4(v[4], v[5], v[6], v[7]);
      } else {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (DT == kF16) {
            const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
            w[k] = *reinterpret_cast<const uint32_t*>(&h);
          } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
            w[k] = *reinterpret_cast<const uint32_t*>(&h);
          }
        }
        *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p.y) + at) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kVec; ++k)
        if (col + k < p.inner) store_one<DT>(p.y, at + k, v[k]);
    }
  }
}

int grid_for(uint32_t total) {
  const int64_t blocks = ((int64_t)total + kThreads - 1) / kThreads, most = (int64_t)num_sms() * 8;
  return (int)(blocks < most ? blocks : most);
}

template <int SRC, int BLOCK>
int launch_quantize(const QuantParams& p, bool vec, cudaStream_t stream) {
  const dim3 grid(grid_for(p.total));
  return cuda_status(vec ? launch_after_predecessor(fp4_quantize_kernel<SRC, BLOCK, true>, grid, dim3(kThreads), stream, p)
                         : launch_after_predecessor(fp4_quantize_kernel<SRC, BLOCK, false>, grid, dim3(kThreads), stream, p),
                     "fp4_quantize_kernel launch");
}
template <int SRC>
int launch_quantize(const QuantParams& p, int block, bool vec, cudaStream_t stream) {
  return block == 32 ? launch_quantize<SRC, 32>(p, vec, stream) : launch_quantize<SRC, 16>(p, vec, stream);
}

template <int DT>
int launch_values(const ValueParams& p, int block, bool vec, cudaStream_t stream) {
  const dim3 grid(grid_for(p.total));
  cudaError_t e;
  if (block == 32)
    e = vec ? launch_after_predecessor(fp4_values_kernel<DT, 32, true>, grid, dim3(kThreads), stream, p)
            : launch_after_predecessor(fp4_values_kernel<DT, 32, false>, grid, dim3(kThreads), stream, p);
  else
    e = vec ? launch_after_predecessor(fp4_values_kernel<DT, 16, true>, grid, dim3(kThreads), stream, p)
            : launch_after_predecessor(fp4_values_kernel<DT, 16, false>, grid, dim3(kThreads), stream, p);
  return cuda_status(e, "fp4_values_kernel launch");
}

// Rows per launch: chunks are counted below 2^29.  A multiple of a scale tile's rows.
int64_t rows_per_launch(int64_t chunks) {
  const int64_t rows = (((int64_t)1 << 29) / chunks) & ~(int64_t)(kFp4TileRows - 1);
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
  if (out.c_stride > 2 * kFp4MaxInner) return ADAPTION_ERR_UNSUPPORTED;
  rc = q != nullptr ? check_qtensor_in(*q, (int64_t)inner) : check_matrix(x, (int64_t)inner);
  if (rc != ADAPTION_OK) return rc;
  QuantParams p{};
  p.inner = (int)inner;
  p.c_stride = (int)out.c_stride;
  p.row_bytes = out.c_stride / 2;
  p.groups = fp4_groups((int64_t)inner, out.block);
  p.blocks4 = (int)p.groups * 4;
  p.exp = out.exp;
  p.relu = relu ? 1 : 0;
  p.stats = stats;
  const int64_t width = out.c_stride > (int64_t)p.blocks4 * out.block ? out.c_stride : (int64_t)p.blocks4 * out.block;
  p.chunks = make_divider((uint32_t)(width / kVec));
  bool vec = true;
  int64_t item = 1;
  if (q != nullptr) {
    p.x = q->lo;
    p.hi = q->fmt.n_bits > 8 ? (const int8_t*)q->hi : nullptr;
    p.stride = q->c_stride;
    p.unit = pow2_float(-q->fmt.frac_bits);
  } else {
    p.x = x.data;
    p.stride = x.stride;
    item = dtype_size(x.dtype);
    vec = aligned16(x.data) && ((x.stride * item) & 15) == 0;
  }
  p.codes = (uint8_t*)out.codes;
  p.scales = (uint8_t*)out.scales;
  const int64_t rows = rows_per_launch(p.chunks.d);
  for (int64_t r = 0; r < (int64_t)outer; r += rows) {
    const int64_t n = (int64_t)outer - r < rows ? (int64_t)outer - r : rows;
    p.total = (uint32_t)(n * p.chunks.d);
    if (q != nullptr) rc = launch_quantize<kPlanes>(p, out.block, vec, stream);
    else if (x.dtype == ADAPTION_F32) rc = launch_quantize<kF32>(p, out.block, vec, stream);
    else if (x.dtype == ADAPTION_F16) rc = launch_quantize<kF16>(p, out.block, vec, stream);
    else rc = launch_quantize<kBF16>(p, out.block, vec, stream);
    if (rc != ADAPTION_OK) return rc;
    p.x = (const uint8_t*)p.x + n * p.stride * item;
    if (p.hi != nullptr) p.hi += n * p.stride;
    p.codes += n * p.row_bytes;
    p.scales += n / kFp4TileRows * p.groups * kFp4TileBytes;
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
  p.groups = fp4_groups((int64_t)inner, x.block);
  p.chunks = make_divider((uint32_t)((inner + kVec - 1) / kVec));
  p.unit = pow2_float(x.exp);
  p.codes = (const uint8_t*)x.codes;
  p.scales = (const uint8_t*)x.scales;
  p.y = y.data;
  p.stride = y.stride;
  const int64_t item = dtype_size(y.dtype);
  const bool vec = aligned16(y.data) && ((y.stride * item) & 15) == 0;
  const int64_t rows = rows_per_launch(p.chunks.d);
  for (int64_t r = 0; r < (int64_t)outer; r += rows) {
    const int64_t n = (int64_t)outer - r < rows ? (int64_t)outer - r : rows;
    p.total = (uint32_t)(n * p.chunks.d);
    if (y.dtype == ADAPTION_F32) rc = launch_values<kF32>(p, x.block, vec, stream);
    else if (y.dtype == ADAPTION_F16) rc = launch_values<kF16>(p, x.block, vec, stream);
    else rc = launch_values<kBF16>(p, x.block, vec, stream);
    if (rc != ADAPTION_OK) return rc;
    p.codes += n * p.row_bytes;
    p.scales += n / kFp4TileRows * p.groups * kFp4TileBytes;
    p.y = (uint8_t*)p.y + n * p.stride * item;
  }
  return ADAPTION_OK;
}

}  // namespace adaption
