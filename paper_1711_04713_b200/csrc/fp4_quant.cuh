// Microscaled 4-bit floating point: from real values in registers to codes and a scale, shared by the quantizer and the product that
// quantizes its activations itself.
//
// With amax the block's maximum:
//   block 32: step 2^(floor(log2 amax) - 2).  The scale byte is amax's exponent field less 2 (a denormal amax has field 0,
//     and every step below 2^-127 is clamped there), and x / step is a product by a power of two: exact.
//   block 16: step s 2^exp with s = E4M3(amax 2^-exp / 6), and x / step is needed to the last bit of the decision between
//     two codes.  The quotient is rounded to 32 bits before it is rounded to E2M1; that gives the nearest code
//     all the same: a border m between two codes and the step have 3 and 4 significant bits, so m * step is a float, an x
//     off that border is off by one unit in its last place at least, and that moves x / step by more than half a unit in m's last
//     place (the step's significand is at most 1.875).  The division itself is q = x r, q -= (q step - x) r with r the reciprocal
//     to one unit in the last place (Markstein, IBM J. Res. Dev. 34, 1990): the residual is exact in one fused multiply-add, the
//     correction leaves an error of 2^-44 before the last rounding, and an element costs three operations.  The same holds
//     for amax / 6 against the borders of E4M3.
//     Sources of 16 bits need two: an x off a border is off by 2^-16 of it at least.  With r raised by four units in the last place
//     the product lies above x / step by 2^-24 to 2^-20 of it; cut to 20 bits it is m on the border m, and stays on its side
//     of every other.  (4096 x 25088 bf16 in blocks of 16: 46.1 us instead of 46.8; with maxima two at a time 45.0.)
#pragma once

#include "fp4.cuh"

namespace adaption {
namespace {

// 32 bytes, read once
__device__ __forceinline__ void load_words(const void* at, bool aligned32, uint32_t (&w)[8]) {
  if (aligned32) {
    asm volatile("ld.global.cs.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(at));
  } else {
    const uint4 a = __ldcs(reinterpret_cast<const uint4*>(at)), b = __ldcs(reinterpret_cast<const uint4*>(at) + 1);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  }
}
// The first `bytes` (at most 32) of what lies at an address of any alignment, from the aligned 16-byte words that hold
// them: none of another word is touched.  What lies behind them is undefined.  (Element by element, rows off a 16-byte
// boundary were read at a fifth of the speed.)
__device__ __forceinline__ void load_shifted(const void* at, int bytes, uint32_t (&w)[8]) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(at);
  const uint32_t sh = (uint32_t)a & 15u;
  const uint4* q = reinterpret_cast<const uint4*>(a - sh);
  uint32_t g[12];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    uint4 t = make_uint4(0u, 0u, 0u, 0u);
    if (bytes > 0 && 16 * k < (int)sh + bytes) t = __ldg(q + k);
    g[4 * k] = t.x; g[4 * k + 1] = t.y; g[4 * k + 2] = t.z; g[4 * k + 3] = t.w;
  }
  if (sh & 8u) {
#pragma unroll
    for (int k = 0; k < 10; ++k) g[k] = g[k + 2];
  }
  if (sh & 4u) {
#pragma unroll
    for (int k = 0; k < 9; ++k) g[k] = g[k + 1];
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = sh & 2u ? __funnelshift_r(g[k], g[k + 1], 16) : g[k];
}

// NaN -> 0 and infinities -> the largest finite number, where a block's maximum says that it holds one.  (The lanes of a block agree on
// that and come here together; those of another block need not.)
template <int BLOCK, int kVec>
__device__ __forceinline__ void fp4_finite(float (&v)[kVec], float& top) {
  if (top < __uint_as_float(0x7f800000u)) return;
  constexpr int kLanes = BLOCK / kVec;
  const uint32_t lanes = ((1u << kLanes) - 1u) << (threadIdx.x & 31u & ~(uint32_t)(kLanes - 1));
  top = 0.f;
#pragma unroll
  for (int k = 0; k < kVec; ++k) {
    v[k] = v[k] == v[k] ? fminf(fmaxf(v[k], -3.402823466e38f), 3.402823466e38f) : 0.f;
    top = fmaxf(top, fabsf(v[k]));
  }
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) top = fmaxf(top, __shfl_xor_sync(lanes, top, o));
}

// This lane's part of a block whose maximum is `top` (finite): returns the block's scale byte, puts the codes, eight a word, into `code`
// and leaves the quotients x / step in `v`.  inv_unit, step_unit: 2^-exp and 2^exp of a tensor with blocks of 16.  SHORT: no element has
// more than 16 significant bits.
template <int BLOCK, int kVec, bool SHORT>
__device__ __forceinline__ uint32_t fp4_encode(float (&v)[kVec], float top, float inv_unit, float step_unit, uint32_t (&code)[kVec / 8]) {
  uint32_t byte;
  if (BLOCK == 32) {
    byte = (uint32_t)max((int)(__float_as_uint(top) >> 23) - 2, 0);
    const float inv = __uint_as_float((254u - byte) << 23);
#pragma unroll
    for (int k = 0; k < kVec; ++k) v[k] *= inv;
  } else {
    const float t = fminf(top * inv_unit, 3e38f), sixth = 1.f / 6.f, t6 = t * sixth;
    byte = e4m3_nearest(fmaf(fmaf(t6, 6.f, -t), -sixth, t6));
    const float s = e4m3_value(byte) * step_unit;
    const float r = s > 0.f ? __uint_as_float(__float_as_uint(reciprocal(s)) + (SHORT ? 4u : 0u)) : 0.f;
    if (top > 8.f * s) {
      // the largest scale was too small, or the smallest too large: beyond 8 steps all is clipped
#pragma unroll
      for (int k = 0; k < kVec; ++k) v[k] = fminf(fmaxf(v[k], -8.f * s), 8.f * s);
    }
    // (in both forms a zero keeps its sign)
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const float q = v[k] * r;
      v[k] = SHORT ? __uint_as_float(__float_as_uint(q) & 0xfffffff0u) : fmaf(fmaf(q, s, -v[k]), -r, q);
    }
  }
#pragma unroll
  for (int i = 0; i < kVec / 8; ++i) code[i] = fp4_pack8(v + 8 * i);
  return byte;
}

}  // namespace
}  // namespace adaption
