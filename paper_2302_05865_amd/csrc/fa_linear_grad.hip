// Weight and bias gradients of a linear layer, worker by worker, from the 8-bit checkpoint of its input.
//
//   P_w[o, i] = sum over the rows t of worker w of dY[t, o] v[t, i],    b_w[o] = the same sum of dY[t, o],
//   dW_w = gamma_i P_w + beta_i b_w[o]  (the layer's input was v gamma + beta)   or   dW_w = P_w,    db_w = b_w,
//
// where v are the checkpoint's values.  They have seven significant bits, so they are exact in bf16; dY is bf16, or fp32
// cut exactly into three pieces of eight bits.  Every product on the bf16 matrix core is exact, sums are fp32.  The rows are
// the contracted index of both operands and lie far apart in memory: the tiles go to LDS as they lie and are read through
// the transposing LDS load.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fa.h"
#include "fa_layers.h"

namespace {

constexpr int kThreads = 256;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// x = h + m + l exactly, each with eight significant bits, h and m cut off (h of the largest finite value stays finite).
// An infinity or a NaN is h, with nothing left over.
__device__ __forceinline__ void split3(float x, uint32_t* h, uint32_t* m, uint32_t* l) {
  const uint32_t u = __float_as_uint(x);
  const bool finite = (u & 0x7f800000u) != 0x7f800000u;
  const uint32_t hu = (u & 0xffff0000u) | ((u & 0x7fffffffu) > 0x7f800000u ? 0x00400000u : 0u);
  const float r = finite ? x - __uint_as_float(hu) : 0.f;
  const uint32_t mu = __float_as_uint(r) & 0xffff0000u;
  *h = hu;
  *m = mu;
  *l = __float_as_uint(r - __uint_as_float(mu));
}
// the upper halves of two words: low half of the result from a
__device__ __forceinline__ uint32_t upper_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

}  // namespace

// A workgroup makes a tile of BM outputs x BN features of one worker (of one split of its rows); its four wavefronts a
// quarter each, 32 x 32 results at a time.  T: storage of dY.
template <typename T, int BM, int BN, int BK>
__global__ __launch_bounds__(kThreads) void fa_linear_grad_kernel(fa_linear_grad_args a) {
  constexpr int PLANES = sizeof(T) == 4 ? 3 : 1;
  constexpr int AP = BM * 2 + 32, BP = BN * 2 + 32;       // LDS bytes of a row (+32: rows of one read on their own banks)
  constexpr int FM = BM / 64, FN = BN / 64;               // 32 x 32 results of a wavefront in either direction
  __shared__ __attribute__((aligned(16))) unsigned char la[PLANES][BK * AP];
  __shared__ __attribute__((aligned(16))) unsigned char lb[BK * BP];
  __shared__ float bias[BM];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tiles_o = (a.outputs + BM - 1) / BM, tiles_i = (a.features + BN - 1) / BN;
  int64_t k = blockIdx.x;
  const int ti = (int)(k % tiles_i);
  k /= tiles_i;
  const int to = (int)(k % tiles_o);
  k /= tiles_o;
  const int split = (int)(k % a.splits), w = (int)(k / a.splits);
  const int o0 = to * BM, i0 = ti * BN;
  // this split's rows: whole steps of BK rows
  const int64_t all = a.blocks.row0[w + 1] - a.blocks.row0[w];
  const int64_t steps = (all + BK - 1) / BK, per = (steps + a.splits - 1) / a.splits;
  const int64_t begin = a.blocks.row0[w] + min(all, (int64_t)split * per * BK);
  const int64_t end = a.blocks.row0[w] + min(all, ((int64_t)split + 1) * per * BK);
  const int64_t pitch = fa_code_pitch(a.features), epitch = fa_exponent_pitch(a.features);

  // what a thread brings in: pieces of 8 outputs of dY, pieces of 16 codes
  constexpr int A_PER_ROW = BM / 8, A_ROWS = kThreads / A_PER_ROW, A_N = BK / A_ROWS;
  constexpr int B_PER_ROW = BN / 16, B_ROWS = kThreads / B_PER_ROW, B_N = BK / B_ROWS;
  static_assert(A_N * A_ROWS == BK && B_N * B_ROWS == BK, "whole rounds of loads");
  const int ac = (tid % A_PER_ROW) * 8, ar = tid / A_PER_ROW;
  const int bc = (tid % B_PER_ROW) * 16, br = tid / B_PER_ROW;
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
  f32x16 acc[FM][FN];
#pragma unroll
  for (int m = 0; m < FM; ++m)
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.f;
  const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
  // a lane's place in a transposing read: of every 16 lanes, lane s names row s / 4 and columns 4 (s % 4).. and gets
  // column s of the four rows
  const int tr_row = (lane >> 5) * 8 + ((lane & 15) >> 2), tr_col = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;

  for (int64_t t0 = begin; t0 < end; t0 += BK) {
    __syncthreads();
#pragma unroll
    for (int n = 0; n < A_N; ++n) {
      const int64_t t = t0 + ar + n * A_ROWS;
      float v[8];
      fa_load8(static_cast<const T*>(a.dy) + t * a.lddy + o0 + ac, t < end ? a.outputs - o0 - ac : 0, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += v[e];
      unsigned char* at = &la[0][(ar + n * A_ROWS) * AP + ac * 2];
      if constexpr (PLANES == 1) {
        uint4 u;
        u.x = upper_halves(__float_as_uint(v[0]), __float_as_uint(v[1]));
        u.y = upper_halves(__float_as_uint(v[2]), __float_as_uint(v[3]));
        u.z = upper_halves(__float_as_uint(v[4]), __float_as_uint(v[5]));
        u.w = upper_halves(__float_as_uint(v[6]), __float_as_uint(v[7]));
        *reinterpret_cast<uint4*>(at) = u;
      } else {
        uint32_t piece[3][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) split3(v[e], &piece[0][e], &piece[1][e], &piece[2][e]);
#pragma unroll
        for (int q = 0; q < 3; ++q)
          *reinterpret_cast<uint4*>(at + q * (BK * AP)) =
              make_uint4(upper_halves(piece[q][0], piece[q][1]), upper_halves(piece[q][2], piece[q][3]),
                         upper_halves(piece[q][4], piece[q][5]), upper_halves(piece[q][6], piece[q][7]));
      }
    }
#pragma unroll
    for (int n = 0; n < B_N; ++n) {
      const int64_t t = t0 + br + n * B_ROWS;
      uint4 codes = make_uint4(0u, 0u, 0u, 0u);
      float scale = 0.f;
      if (t < end && i0 + bc < pitch) {
        codes = *reinterpret_cast<const uint4*>(a.codes + t * pitch + i0 + bc);
        scale = fa_block_scale(a.exponents[t * epitch + ((i0 + bc) >> 5)]);
      }
      float v[16];
      fa_values8(make_uint2(codes.x, codes.y), scale, v);
      fa_values8(make_uint2(codes.z, codes.w), scale, v + 8);
      uint32_t u[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = upper_halves(__float_as_uint(v[2 * e]), __float_as_uint(v[2 * e + 1]));
      uint4* at = reinterpret_cast<uint4*>(&lb[(br + n * B_ROWS) * BP + bc * 2]);
      at[0] = make_uint4(u[0], u[1], u[2], u[3]);
      at[1] = make_uint4(u[4], u[5], u[6], u[7]);
    }
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < BK; kk += 16) {
      bf16x8 fb[FN];
#pragma unroll
      for (int n = 0; n < FN; ++n) {
        const unsigned char* at = &lb[(kk + tr_row) * BP + (wn + 32 * n + tr_col) * 2];
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * BP));
        fb[n] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
#pragma unroll
      for (int q = PLANES - 1; q >= 0; --q)
#pragma unroll
        for (int m = 0; m < FM; ++m) {
          const unsigned char* at = &la[q][(kk + tr_row) * AP + (wm + 32 * m + tr_col) * 2];
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * AP));
          const bf16x8 fa = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int n = 0; n < FN; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa, fb[n], acc[m][n], 0, 0, 0);
        }
    }
  }
  // b_w: the threads that brought in the same outputs, in their order
  __syncthreads();
  float* part = reinterpret_cast<float*>(lb);
  static_assert(A_ROWS * BM * 4 <= BK * BP, "the column sums fit");
#pragma unroll
  for (int e = 0; e < 8; ++e) part[ar * BM + ac + e] = sum[e];
  __syncthreads();
  if (tid < BM) {
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < A_ROWS; ++r) s += part[r * BM + tid];
    bias[tid] = s;
  }
  __syncthreads();
  const int64_t OI = (int64_t)a.outputs * a.features;
  if (a.splits > 1) {
    float* out = a.partials + ((int64_t)w * a.splits + split) * (OI + a.outputs);
    if (ti == 0 && tid < BM && o0 + tid < a.outputs) out[OI + o0 + tid] = bias[tid];
#pragma unroll
    for (int n = 0; n < FN; ++n) {
      const int i = i0 + wn + 32 * n + (lane & 31);
#pragma unroll
      for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int o = o0 + wm + 32 * m + (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5);
          if (i < a.features && o < a.outputs) out[(int64_t)o * a.features + i] = acc[m][n][r];
        }
    }
    return;
  }
  if (a.dbias && ti == 0 && tid < BM && o0 + tid < a.outputs) {
    const int64_t at = w * a.lddbias + o0 + tid;
    if (a.grad_bf16) fa_store1(static_cast<fa_bf16*>(a.dbias) + at, bias[tid]);
    else fa_store1(static_cast<float*>(a.dbias) + at, bias[tid]);
  }
#pragma unroll
  for (int n = 0; n < FN; ++n) {
    const int i = i0 + wn + 32 * n + (lane & 31);
    float gamma = 1.f, beta = 0.f;
    if (a.gamma && i < a.features) {
      gamma = a.param_bf16 ? fa_load1(static_cast<const fa_bf16*>(a.gamma) + i) : static_cast<const float*>(a.gamma)[i];
      beta = a.param_bf16 ? fa_load1(static_cast<const fa_bf16*>(a.beta) + i) : static_cast<const float*>(a.beta)[i];
    }
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int ol = wm + 32 * m + (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5);
        if (i < a.features && o0 + ol < a.outputs) {
          const float v = a.gamma ? gamma * acc[m][n][r] + beta * bias[ol] : acc[m][n][r];
          const int64_t at = w * a.lddweight + (int64_t)(o0 + ol) * a.features + i;
          if (a.grad_bf16) fa_store1(static_cast<fa_bf16*>(a.dweight) + at, v);
          else fa_store1(static_cast<float*>(a.dweight) + at, v);
        }
      }
  }
}

// The splits of a worker's rows added up in their order, then as above.
__global__ __launch_bounds__(kThreads) void fa_linear_grad_join_kernel(fa_linear_grad_args a) {
  const int64_t OI = (int64_t)a.outputs * a.features, all = OI + a.outputs;
  const int w = blockIdx.y;
  const float* part = a.partials + (int64_t)w * a.splits * all;
  for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < all; k += (int64_t)gridDim.x * kThreads) {
    float s = 0.f;
    for (int q = 0; q < a.splits; ++q) s += part[q * all + k];
    if (k >= OI) {
      if (!a.dbias) continue;
      const int64_t at = w * a.lddbias + (k - OI);
      if (a.grad_bf16) fa_store1(static_cast<fa_bf16*>(a.dbias) + at, s);
      else fa_store1(static_cast<float*>(a.dbias) + at, s);
      continue;
    }
    if (a.gamma) {
      const int64_t o = k / a.features;
      const int i = (int)(k - o * a.features);
      float b = 0.f;
      for (int q = 0; q < a.splits; ++q) b += part[q * all + OI + o];
      const float gamma = a.param_bf16 ? fa_load1(static_cast<const fa_bf16*>(a.gamma) + i) : static_cast<const float*>(a.gamma)[i];
      const float beta = a.param_bf16 ? fa_load1(static_cast<const fa_bf16*>(a.beta) + i) : static_cast<const float*>(a.beta)[i];
      s = gamma * s + beta * b;
    }
    const int64_t at = w * a.lddweight + k;
    if (a.grad_bf16) fa_store1(static_cast<fa_bf16*>(a.dweight) + at, s);
    else fa_store1(static_cast<float*>(a.dweight) + at, s);
  }
}

namespace {
constexpr int kBM = 128, kBN = 128, kBK = 32;
}

int fa_linear_grad_splits(const fa_row_blocks& b, int features, int outputs, int dtype) {
  (void)dtype;
  int64_t most = 0;
  for (int w = 0; w < b.p; ++w) most = b.row0[w + 1] - b.row0[w] > most ? b.row0[w + 1] - b.row0[w] : most;
  const int64_t tiles = (int64_t)b.p * ((outputs + kBM - 1) / kBM) * ((features + kBN - 1) / kBN);
  int64_t s = 512 / tiles;
  if (s > most / 256) s = most / 256;
  return s < 1 ? 1 : (int)s;
}

size_t fa_linear_grad_partials(const fa_row_blocks& b, int features, int outputs, int splits) {
  return splits > 1 ? sizeof(float) * (size_t)b.p * splits * ((size_t)outputs * features + outputs) : 0;
}

hipError_t fa_launch_linear_grad(const fa_linear_grad_args& a, int dtype, hipStream_t st) {
  const int64_t tiles = (int64_t)((a.outputs + kBM - 1) / kBM) * ((a.features + kBN - 1) / kBN);
  const dim3 grid((unsigned)(tiles * a.blocks.p * a.splits));
  if (dtype == FA_F32)
    hipLaunchKernelGGL((fa_linear_grad_kernel<float, kBM, kBN, kBK>), grid, dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL((fa_linear_grad_kernel<fa_bf16, kBM, kBN, kBK>), grid, dim3(kThreads), 0, st, a);
  if (a.splits > 1) {
    int64_t blocks = ((int64_t)a.outputs * a.features + a.outputs + kThreads - 1) / kThreads;
    if (blocks > 2048) blocks = 2048;
    hipLaunchKernelGGL(fa_linear_grad_join_kernel, dim3((unsigned)blocks, (unsigned)a.blocks.p), dim3(kThreads), 0, st, a);
  }
  return hipGetLastError();
}
