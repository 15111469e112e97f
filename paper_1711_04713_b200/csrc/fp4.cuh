// Microscaled 4-bit floating point: checks of descriptors, the scale tiles and the conversions shared by the kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace adaption {

constexpr int kFp4TileRows = 128;      // rows of a scale tile
constexpr int kFp4TileBytes = 512;     // 128 rows x 4 blocks
constexpr int64_t kFp4MaxInner = (int64_t)1 << 24;   // longest row: the codes of 128 of them (pitches up to twice that) are 2^31 bytes

inline int64_t fp4_blocks(int64_t inner, int block) { return (inner + block - 1) / block; }
// scale tiles of one row of tiles
inline int64_t fp4_groups(int64_t inner, int block) { return (fp4_blocks(inner, block) + 3) / 4; }

// Offset of the scale byte of row r and block j; `groups` scale tiles per row of tiles.  (Below 2^32: kernels get a part of the rows.)
__device__ __forceinline__ uint32_t fp4_scale_offset(uint32_t r, int j, int groups) {
  const uint32_t tile = (r >> 7) * (uint32_t)groups + ((uint32_t)j >> 2);
  return tile * kFp4TileBytes + (r & 31u) * 16u + ((r >> 5) & 3u) * 4u + ((uint32_t)j & 3u);
}

int check_fp4(const adaption_fp4tensor& t, int64_t inner);
int check_matrix(const adaption_matrix& m, int64_t inner);
// (64-bit counters, added to by atomics)
inline bool aligned_stats(const adaption_stats* s) { return (reinterpret_cast<uintptr_t>(s) & 7u) == 0; }

int fp4_quantize_impl(const adaption_matrix& x, const adaption_qtensor* q, size_t outer, size_t inner, int32_t relu,
                      const adaption_fp4tensor& out, adaption_stats* stats, cudaStream_t stream);
int fp4_dequantize_impl(const adaption_fp4tensor& x, size_t outer, size_t inner, const adaption_matrix& y,
                        cudaStream_t stream);

// y[B][O] = act(x [B][K] w [O][K]^T + bias); arguments checked by the caller
struct Fp4Problem {
  int64_t B = 0, K = 0, O = 0;
  adaption_fp4tensor x{}, w{};   // x.codes null: the kernel quantizes x_real itself
  adaption_matrix x_real{};
  bool x_follows = false;        // x comes from fp4_quantize_impl, the launch right before on the same stream
  const float* bias = nullptr;
  int32_t relu = 0;
  adaption_matrix y{};
  adaption_stats* stats = nullptr;
  cudaStream_t stream = nullptr;
};
int fp4_ip_impl(const Fp4Problem& p);
// The same on real activations p.x_real; `workspace` describes the place of their 4-bit form.
int fp4_act_ip_impl(Fp4Problem& p, const adaption_fp4tensor& workspace);
// The persistent kernel over tiles of 256 channels x 256 rows (csrc/fp4_pair.cu).
int launch_fp4_pair(const Fp4Problem& p);

inline int dtype_size(int32_t dtype) { return dtype == ADAPTION_F32 ? 4 : 2; }

// Eight numbers to E2M1 (nearest, ties to even, at most 6 in magnitude), the first in bits 0-3.
__device__ __forceinline__ uint32_t fp4_pack8(const float* v) {
  uint32_t r;
  asm("{\n"
      ".reg .b8 a, b, c, d;\n"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
      "mov.b32 %0, {a, b, c, d};\n"
      "}\n"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// The two E2M1 numbers of a byte, bits 0-3 in the low half.
__device__ __forceinline__ __half2 fp4_unpack2(uint32_t byte) {
  uint32_t r;
  asm("{\n"
      ".reg .b8 b;\n"
      "cvt.u8.u32 b, %1;\n"
      "cvt.rn.f16x2.e2m1x2 %0, b;\n"
      "}\n"
      : "=r"(r)
      : "r"(byte));
  return *reinterpret_cast<__half2*>(&r);
}
// 1 / v to one unit in the last place, for normal numbers
__device__ __forceinline__ float reciprocal(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// E4M3: the nearest of a number >= 0 (ties to even, at most 448), and the value of a byte.
__device__ __forceinline__ uint32_t e4m3_nearest(float v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(v));
  return r & 0xffu;
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
  // exponent and mantissa in their places of a float are 2^-120 of the value, a denormal one too
  return __uint_as_float(byte << 20) * 1.329227995784916e36f;
}
// E8M0: 2^(byte - 127); 2^-127 is a denormal float, 255 is NaN
__device__ __forceinline__ float e8m0_value(uint32_t byte) {
  return __uint_as_float(byte == 0u ? 0x00400000u : (byte == 255u ? 0x7fc00000u : byte << 23));
}
// Two numbers rounded to a 16-bit type, as one word.
template <int DT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if (DT == ADAPTION_F16) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// 2^e for e in [-126, 127]
__host__ __device__ __forceinline__ float pow2_float(int e) {
  const uint32_t b = (uint32_t)(e + 127) << 23;
#ifdef __CUDA_ARCH__
  return __uint_as_float(b);
#else
  float f;
  __builtin_memcpy(&f, &b, 4);
  return f;
#endif
}

}  // namespace adaption
