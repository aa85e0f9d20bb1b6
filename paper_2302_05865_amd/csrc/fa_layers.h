// Internal interface between the entry points of the workers' backward pass (fa_layers_api.hip) and
// its kernels (fa_layer_norm.hip, fa_linear_grad.hip).  Not installed; include/fa.h is public.
#ifndef FA_LAYERS_H_
#define FA_LAYERS_H_

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "fa.h"

// Whose rows are whose: worker w has rows [row0[w], row0[w + 1]).  Handed to the kernels by value (64 workers are
// 520 bytes of kernel arguments): nothing is copied to the device, so a call can be captured in a graph.
struct fa_row_blocks {
  int64_t row0[FA_P_MAX + 1];
  int p;
};

// A checkpoint's storage: rows of codes (whole blocks of 32) and rows of exponent bytes (multiples of four).
static inline __host__ __device__ int64_t fa_code_pitch(int features) { return ((int64_t)features + 31) / 32 * 32; }
static inline __host__ __device__ int64_t fa_exponent_pitch(int features) { return ((int64_t)features + 127) / 128 * 4; }

struct fa_norm_args {
  const void *x, *gamma, *beta;   // gamma, beta may be null
  void* y;
  float *mean, *rstd;             // may be null
  int8_t* codes;                  // null: no checkpoint
  uint8_t* exponents;
  int64_t ldx, ldy, rows;
  int features, param_bf16;
  float eps;
};

struct fa_norm_grad_args {
  const void *dy, *x, *gamma, *residual;   // x null: from the checkpoint; gamma, residual may be null
  const float *mean, *rstd;
  const int8_t* codes;
  const uint8_t* exponents;
  void *dx, *dgamma, *dbeta;               // dgamma, dbeta may be null
  float* partials;
  int64_t lddy, ldx, ldr, lddx, lddgamma, lddbeta, rows;
  int features, param_bf16, grad_bf16;
  fa_row_blocks blocks;
};

struct fa_linear_grad_args {
  const void *dy, *gamma, *beta;           // gamma and beta: both or neither
  const int8_t* codes;
  const uint8_t* exponents;
  void *dweight, *dbias;                   // dbias may be null
  float* partials;
  int64_t lddy, lddweight, lddbias;
  int features, outputs, param_bf16, grad_bf16;
  int splits;                              // parts that a worker's rows are cut into
  fa_row_blocks blocks;
};

hipError_t fa_launch_checkpoint_pack(const void* x, int64_t ldx, int64_t rows, int features, int dtype, int8_t* codes,
                                     uint8_t* exponents, hipStream_t st);
hipError_t fa_launch_checkpoint_unpack(const int8_t* codes, const uint8_t* exponents, int64_t rows, int features, int dtype,
                                       void* x, int64_t ldx, hipStream_t st);
hipError_t fa_launch_layer_norm(const fa_norm_args& a, int dtype, hipStream_t st);
size_t fa_layer_norm_partials(const fa_row_blocks& b, int64_t rows, int features);
hipError_t fa_launch_layer_norm_backward(const fa_norm_grad_args& a, int dtype, hipStream_t st);
size_t fa_linear_grad_partials(const fa_row_blocks& b, int features, int outputs, int dtype);
hipError_t fa_launch_linear_grad(fa_linear_grad_args a, int dtype, hipStream_t st);   // (a.splits is the launcher's)

#ifdef __HIPCC__
// ---- eight consecutive elements, at any alignment that the element type has (global memory takes 16-byte accesses
// at any address), as float -------------------------------------------------------------------------------------------
typedef uint32_t fa_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t fa_u32x2 __attribute__((ext_vector_type(2)));
typedef fa_u32x4 fa_u32x4_2 __attribute__((aligned(2)));
typedef fa_u32x4 fa_u32x4_4 __attribute__((aligned(4)));
typedef float fa_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 fa_bf16x2 __attribute__((ext_vector_type(2)));

struct fa_bf16 { uint16_t bits; };   // storage only

__device__ __forceinline__ uint32_t fa_pack_bf16(float a, float b) {   // round to nearest even; low half = a
  const fa_f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, fa_bf16x2));
}
__device__ __forceinline__ float fa_load1(const float* p) { return *p; }
__device__ __forceinline__ float fa_load1(const fa_bf16* p) { return __uint_as_float((uint32_t)p->bits << 16); }
__device__ __forceinline__ void fa_store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void fa_store1(fa_bf16* p, float v) { p->bits = (uint16_t)fa_pack_bf16(v, 0.f); }

__device__ __forceinline__ void fa_load8_whole(const fa_bf16* p, float v[8]) {
  const fa_u32x4 u = *reinterpret_cast<const fa_u32x4_2*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = __uint_as_float(u[e] << 16);
    v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void fa_load8_whole(const float* p, float v[8]) {
  const fa_u32x4 a = *reinterpret_cast<const fa_u32x4_4*>(p);
  const fa_u32x4 b = *reinterpret_cast<const fa_u32x4_4*>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = __uint_as_float(a[e]);
    v[4 + e] = __uint_as_float(b[e]);
  }
}
// the first `valid` of the eight elements at p, zeros behind them; nothing behind them is read
template <typename T>
__device__ __forceinline__ void fa_load8(const T* p, int valid, float v[8]) {
  if (valid >= 8) {
    fa_load8_whole(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < valid ? fa_load1(p + e) : 0.f;
  }
}
__device__ __forceinline__ void fa_store8_whole(fa_bf16* p, const float v[8]) {
  fa_u32x4 u;
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = fa_pack_bf16(v[2 * e], v[2 * e + 1]);
  *reinterpret_cast<fa_u32x4_2*>(p) = u;
}
__device__ __forceinline__ void fa_store8_whole(float* p, const float v[8]) {
  fa_u32x4 a, b;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    a[e] = __float_as_uint(v[e]);
    b[e] = __float_as_uint(v[4 + e]);
  }
  *reinterpret_cast<fa_u32x4_4*>(p) = a;
  *reinterpret_cast<fa_u32x4_4*>(p + 4) = b;
}
template <typename T>
__device__ __forceinline__ void fa_store8(T* p, int valid, const float v[8]) {
  if (valid >= 8) {
    fa_store8_whole(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < valid) fa_store1(p + e, v[e]);
  }
}
// eight parameters (gamma, beta) in either type, zeros behind the valid ones
__device__ __forceinline__ void fa_load8_param(const void* p, int bf16, int at, int valid, float v[8]) {
  if (bf16) fa_load8(static_cast<const fa_bf16*>(p) + at, valid, v);
  else fa_load8(static_cast<const float*>(p) + at, valid, v);
}

// ---- the 8-bit checkpoint ---------------------------------------------------------------------------------------------
// A block of 32 consecutive features of a row holds codes c and one byte e, and stands for c 2^(e - 127).  From the
// largest |v| of the block, of binary exponent E: e - 127 = max(E - 6, -126), so |v| 2^(127 - e) is below 128 and exact,
// c = that rounded to the nearest whole number (ties to even), at most 127 in size.  The value is off by at most half of
// 2^(e - 127), by less than all of it where the code was held at 127; it has seven significant bits: exact in bf16.  A block
// with an infinity or a NaN has e = 255 and codes 0, whose value, 0 times infinity, is NaN.
__device__ __forceinline__ uint32_t fa_block_exponent(uint32_t most_bits) {   // bits of the largest |v|
  const uint32_t biased = most_bits >> 23;
  if (biased == 255u) return 255u;
  return biased > 7u ? biased - 6u : 1u;
}
__device__ __forceinline__ float fa_block_scale(uint32_t e) { return __uint_as_float(e << 23); }
// the lanes 4k..4k+3 of a wavefront hold the 32 values of one block, eight each
__device__ __forceinline__ uint32_t fa_quad_most(const float v[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, true));   // lanes 1 0 3 2 of every four
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, true));   // lanes 2 3 0 1
  return m;
}
__device__ __forceinline__ uint2 fa_codes8(const float v[8], uint32_t e) {
  const float inverse = __uint_as_float((254u - e) << 23);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = (int)fminf(fmaxf(rintf(v[k] * inverse), -127.f), 127.f);
    w[k >> 2] |= ((uint32_t)c & 255u) << (8 * (k & 3));
  }
  return e == 255u ? make_uint2(0u, 0u) : make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void fa_values8(uint2 codes, float scale, float v[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    v[k] = (float)(int8_t)((k < 4 ? codes.x : codes.y) >> (8 * (k & 3))) * scale;
}
#endif  // __HIPCC__

#endif
