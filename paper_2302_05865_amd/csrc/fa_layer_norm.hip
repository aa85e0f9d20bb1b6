// Layer norm over the rows of p workers, its backward pass, and the 8-bit checkpoint between the two.
//
//   mu = sum_j x_j / D,  var = sum_j (x_j - mu)^2 / D,  r = 1 / sqrt(var + eps),  xhat = (x - mu) r,  y = xhat gamma + beta
//   h = dy gamma,  a = sum_j h_j / D,  b = sum_j h_j xhat_j / D,  dx = r (h - a - xhat b) [+ residual]
//   dgamma_w = sum over the rows of worker w of dy xhat,  dbeta_w = the same of dy
//
// Bound by memory: forward reads x and writes y and the checkpoint, backward reads dy and xhat and writes dx, every element
// once.  A row is held in registers by a team of lanes, eight consecutive features a lane and piece, so the variance is that
// of the centred values, and four neighbouring lanes hold one block of a checkpoint.  The next row is on its way while this
// one is worked on.  Statistics and sums are fp32.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "fa.h"
#include "fa_layers.h"

namespace {

constexpr int kThreads = 256;

// sum over a team of L lanes (a power of two of one wavefront)
template <int L>
__device__ __forceinline__ float team_sum(float v) {
#pragma unroll
  for (int d = 1; d < L; d *= 2) v += __shfl_xor(v, d);
  return v;
}

typedef unsigned int vec_u32x4 __attribute__((__vector_size__(16)));
typedef unsigned int vec_u32x2 __attribute__((__vector_size__(8)));

// Eight consecutive elements as they lie in memory.
template <typename T>
struct raw8 {
  fa_u32x4 u[sizeof(T) / 2];
};
__device__ __forceinline__ raw8<fa_bf16> load_whole(const fa_bf16* p) {
  return {{*reinterpret_cast<const fa_u32x4_2*>(p)}};
}
__device__ __forceinline__ raw8<float> load_whole(const float* p) {
  return {{*reinterpret_cast<const fa_u32x4_4*>(p), *reinterpret_cast<const fa_u32x4_4*>(p + 4)}};
}
// One row of D elements, read and written in pieces of eight from `at`; what is past its end reads as zero and is not
// written.  A row of a whole wavefront or more (WIDE: its address is the same for every lane) is a buffer, and the memory
// unit looks after its end, in steps of four bytes: no branch stands between a load and the next.  The last element of an
// odd row of bf16 comes alone, in the upper half of a word.  (The waits between two rows count the loads and stores that
// may still be on their way: those are the same for every row, and none of them is in a branch.)
template <bool WIDE, typename T>
struct row_in;
template <typename T>
struct row_in<true, T> {
  __amdgpu_buffer_rsrc_t r, whole;
  int at_last;
  // (no row, p null: zeros)
  __device__ __forceinline__ row_in(const T* p, int D)
      : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(p), 0, p ? D * (int)sizeof(T) & ~3 : 0, 0x00020000)),
        whole(__builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(p), 0, p ? D * (int)sizeof(T) : 0, 0x00020000)),
        at_last(D * (int)sizeof(T) - 4) {}
  __device__ __forceinline__ raw8<T> load(int at, int) const {
    raw8<T> v;
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k)
      v.u[k] = __builtin_bit_cast(fa_u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at * (int)sizeof(T) + 16 * k, 0, 0));
    return v;
  }
  __device__ __forceinline__ uint32_t last() const {
    return sizeof(T) == 2 ? __builtin_amdgcn_raw_buffer_load_b32(whole, at_last, 0, 0) : 0u;
  }
};
// A row of fewer lanes: the piece that the row ends in is loaded element by element.
template <typename T>
struct row_in<false, T> {
  const T* p;
  __device__ __forceinline__ row_in(const T* row, int) : p(row) {}
  __device__ __forceinline__ raw8<T> load(int at, int D) const {
    if (at + 8 <= D) return load_whole(p + at);
    raw8<T> r = {};
    float v[8];
    fa_load8(p + at, D - at, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (sizeof(T) == 4) r.u[e >> 2][e & 3] = __float_as_uint(v[e]);
      else r.u[0][e >> 1] |= (__float_as_uint(v[e]) >> 16) << (16 * (e & 1));
    }
    return r;
  }
  __device__ __forceinline__ uint32_t last() const { return 0u; }
};
// as floats; `last` belongs into the row's last piece
template <bool WIDE, bool LAST, typename T>
__device__ __forceinline__ void values(raw8<T> r, uint32_t last, int at, int D, float v[8]) {
  // (held back to here: the compiler would convert a row where it arrives, and wait for it there)
  asm("" : "+v"(r.u[0]));
  if constexpr (sizeof(T) == 4) asm("" : "+v"(r.u[1]));
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (sizeof(T) == 4) v[e] = __uint_as_float(r.u[e >> 2][e & 3]);
    else v[e] = __uint_as_float(e & 1 ? r.u[0][e >> 1] & 0xffff0000u : r.u[0][e >> 1] << 16);
  }
  if constexpr (WIDE && LAST && sizeof(T) == 2) {
    if (D & 1) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) v[e] = at + e == D - 1 ? __uint_as_float(last & 0xffff0000u) : v[e];
    }
  }
}
// *p = v by the one lane that is `here`; p may be null
template <bool WIDE>
__device__ __forceinline__ void store_float(float* p, int64_t at, bool here, float v) {
  if constexpr (WIDE) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(p + at, 0, p ? 4 : 0, 0x00020000);
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, here ? 0 : 4, 0, 0);
  } else if (here && p) {
    p[at] = v;
  }
}
// the codes and exponents of a piece of a row (LAST: it may be past the end), the exponent by every fourth lane
template <bool WIDE, bool LAST>
__device__ __forceinline__ void store_codes(int8_t* codes, uint8_t* exponents, int64_t pitch, int at, uint2 u, uint32_t e) {
  if constexpr (WIDE) {
    const __amdgpu_buffer_rsrc_t c = __builtin_amdgcn_make_buffer_rsrc(codes, 0, (int)pitch, 0x00020000);
    const __amdgpu_buffer_rsrc_t x = __builtin_amdgcn_make_buffer_rsrc(exponents, 0, (int)pitch / 32, 0x00020000);
    __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(vec_u32x2, u), c, at, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b8((uint8_t)e, x, (at & 31) == 0 ? at >> 5 : (int)pitch, 0, 0);
  } else if (!LAST || at < pitch) {
    *reinterpret_cast<uint2*>(codes + at) = u;
    if ((at & 31) == 0) exponents[at >> 5] = (uint8_t)e;
  }
}
template <bool WIDE, bool LAST, typename T>
__device__ __forceinline__ void store_piece(T* row, int at, int D, const float v[8]) {
  if constexpr (!LAST) {
    fa_store8_whole(row + at, v);
  } else if constexpr (!WIDE) {
    fa_store8(row + at, D - at, v);
  } else {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(row, 0, D * (int)sizeof(T) & ~3, 0x00020000);
    fa_u32x4 u[2];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4) {
        u[0][k] = __float_as_uint(v[k]);
        u[1][k] = __float_as_uint(v[4 + k]);
      } else {
        u[0][k] = fa_pack_bf16(v[2 * k], v[2 * k + 1]);
      }
    }
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k)
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(vec_u32x4, u[k]), r, at * (int)sizeof(T) + 16 * k, 0, 0);
    if constexpr (sizeof(T) == 2) {
      if (D & 1) {
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          if (at + e == D - 1) fa_store1(row + D - 1, v[e]);
      }
    }
  }
}
// calls f(c, last) for the pieces 0..NC - 1, `last` a constant type of its call
template <int NC, typename F>
__device__ __forceinline__ void each_piece(F f) {
  if constexpr (NC > 1) each_piece<NC - 1>([&](auto c, auto) __attribute__((always_inline)) {
    f(c, std::integral_constant<bool, false>());
  });
  f(std::integral_constant<int, NC - 1>(), std::integral_constant<bool, true>());
}

}  // namespace

// T: storage of x and y; KEEP: with a checkpoint.  A row's team is L lanes of a wavefront (W = 1) or W whole wavefronts,
// with NC pieces of eight features a lane: 8 L W (NC - 1) < D <= 8 L W NC (or NC = 1).
//
// Bound by memory from some thousand rows on.  A row lies in registers from its one read to its one write, so the centred
// sum of squares costs no second pass; the next row's loads stand ahead of this one's reductions, and nothing a wavefront
// waits for is behind a branch (the waits would be for everything in flight).
// Rows of more than 256 features are read and written as buffers of their own length, in which lanes past the end do nothing.
// Measured: 65536 x 4096 bf16 220 us = 4.9 TB/s (a copy: 5.13), 32768 x 4096 fp32 194 us = 5.5 TB/s, 15360 x 768 bf16 with a
// checkpoint 14.3 us = 4.2 TB/s, one row of 768 2.7 us, which is a launch and one turn to memory and back.
template <typename T, bool KEEP, int L, int NC, int W>
__global__ __launch_bounds__(W > 1 ? 64 * W : kThreads) void fa_layer_norm_kernel(fa_norm_args a) {
  static_assert(W == 1 || L == 64, "a team of several wavefronts uses all their lanes");
  constexpr int TL = L * W;                                    // lanes of a team
  constexpr int TEAMS = W > 1 ? 1 : kThreads / L;
  __shared__ float red[2][W];
  const int lane = threadIdx.x % TL, D = a.features;
  const float width = (float)D;
  const int64_t pitch = fa_code_pitch(D), epitch = fa_exponent_pitch(D);
  constexpr bool WIDE = L == 64;
  const T* x = static_cast<const T*>(a.x);
  int team = threadIdx.x / TL;
  if constexpr (WIDE) team = __builtin_amdgcn_readfirstlane(team);
  int64_t row = (int64_t)blockIdx.x * TEAMS + team;
  const int64_t step = (int64_t)gridDim.x * TEAMS;
  if (W == 1 && row >= a.rows) return;
  raw8<T> next[NC];
  uint32_t next_last = 0;
  auto load = [&](int64_t r) __attribute__((always_inline)) {
    const row_in<WIDE, T> in(x + r * a.ldx, D);
#pragma unroll
    for (int c = 0; c < NC; ++c) next[c] = in.load(8 * (lane + TL * c), D);
    next_last = in.last();
  };
  load(row);
  float gamma[NC][8], beta[NC][8];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int at = 8 * (lane + TL * c);
    if (a.gamma) fa_load8_param(a.gamma, a.param_bf16, at, D - at, gamma[c]);
    if (a.beta) fa_load8_param(a.beta, a.param_bf16, at, D - at, beta[c]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (!a.gamma) gamma[c][e] = 1.f;
      if (!a.beta) beta[c][e] = 0.f;
    }
  }
  for (; row < a.rows; row += step) {
    float v[NC][8];
    float s = 0.f;
    each_piece<NC>([&](auto c, auto last) __attribute__((always_inline)) {
      values<WIDE, last>(next[c], next_last, 8 * (lane + TL * c), D, v[c]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[c][e];
    });
    load(row + step < a.rows ? row + step : row);       // (the last row comes again: a load that nothing waits for)
    __builtin_amdgcn_sched_barrier(0);
    s = team_sum<L>(s);
    if constexpr (W > 1) {
      if (threadIdx.x % 64 == 0) red[0][threadIdx.x / 64] = s;
      __syncthreads();
      s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += red[0][w];
    }
    const float mean = s / width;
    float q = 0.f;
    each_piece<NC>([&](auto c, auto last) __attribute__((always_inline)) {
      const int valid = D - 8 * (lane + TL * c);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[c][e] = !last || e < valid ? v[c][e] - mean : 0.f;
        q += v[c][e] * v[c][e];
      }
    });
    q = team_sum<L>(q);
    if constexpr (W > 1) {
      if (threadIdx.x % 64 == 0) red[1][threadIdx.x / 64] = q;
      __syncthreads();
      q = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) q += red[1][w];
    }
    const float rstd = 1.f / sqrtf(q / width + a.eps);
    store_float<WIDE>(a.mean, row, lane == 0, mean);
    store_float<WIDE>(a.rstd, row, lane == 0, rstd);
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    each_piece<NC>([&](auto c, auto last) __attribute__((always_inline)) {
      const int at = 8 * (lane + TL * c);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] *= rstd;
      if constexpr (KEEP) {
        // (past the end of a row of an infinite or NaN rstd there is no 0 but NaN: its block has that anyway)
        const uint32_t e = fa_block_exponent(fa_quad_most(v[c]));
        store_codes<WIDE, last>(a.codes + row * pitch, a.exponents + row * epitch, pitch, at, fa_codes8(v[c], e), e);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] = v[c][e] * gamma[c][e] + beta[c][e];
      store_piece<WIDE, last>(y, at, D, v[c]);
    });
  }
}

namespace {

// Rows that one workgroup of the backward pass takes: a share of one worker's.  There are no more chunks than workgroups
// have registers for at one time, three for every compute unit: a few that wait for a second turn would double the time
// (65536 x 4096 of 32 workers of uneven sizes: 355 us with chunks of one length and some more of them, 289 so).
constexpr int kNormBlocks = 768;

struct norm_chunks {
  int first[FA_P_MAX + 1];   // worker w has the chunks [first[w], first[w + 1])
};

norm_chunks cut(const fa_row_blocks& b, int64_t rows) {
  norm_chunks c;
  int64_t share = (rows + kNormBlocks - 1) / kNormBlocks;
  if (share < 4) share = 4;
  for (;; share += share / 16 + 1) {
    int64_t chunks = 0;
    c.first[0] = 0;
    for (int w = 0; w < FA_P_MAX; ++w) {
      if (w < b.p) chunks += (b.row0[w + 1] - b.row0[w] + share - 1) / share;
      c.first[w + 1] = (int)chunks;
    }
    if (chunks <= kNormBlocks) return c;      // (at the latest with one chunk a worker)
  }
}

// the worker that chunk k belongs to: as many workers end at or before it as come ahead of it
__device__ __forceinline__ int worker_of(const int* first, int p, int k) {
  int w = 0;
  for (int j = 1; j < p; ++j) w += first[j] <= k ? 1 : 0;
  return w;
}

}  // namespace

// T: storage of dy, x, dx; KEPT: xhat from the checkpoint.  One workgroup takes one chunk of rows of one worker and leaves
// its share of dgamma and dbeta in partials[chunk][2][D].  Teams and pieces as above.
//
// Bound by memory as well: dy and xhat are read once, dx is written once, and the sums over rows stay in the registers of
// the lane that has the feature, all its rows long.  That costs registers (two sums and gamma for every feature of a lane),
// so wide rows are spread over more wavefronts than in the forward pass.  Both sums over features go through one reduction
// and one barrier; no atomics: the sums come out the same at every call.  Measured: 65536 x 4096 bf16 from the checkpoint
// 280 us = 4.8 TB/s (eight features a lane in eight wavefronts 440, gamma in LDS 421), from x 334 us = 4.8 TB/s, 32768 x 4096
// fp32 from x 311 us = 5.2 TB/s, 15360 x 768 bf16 with residual 18.4 us = 4.5 TB/s, 1001 x 257 fp32 5.2 us.
template <typename T, bool KEPT, int L, int NC, int W>
__global__ __launch_bounds__(W > 1 ? 64 * W : kThreads) void fa_layer_norm_backward_kernel(fa_norm_grad_args a, norm_chunks ch) {
  constexpr int TL = L * W;
  constexpr int THREADS = W > 1 ? 64 * W : kThreads;
  constexpr int TEAMS = THREADS / TL;
  constexpr int WAVES = THREADS / 64;
  __shared__ float2 red[2][WAVES];
  __shared__ float join[W > 1 ? 1 : WAVES * 2 * L * NC * 8];
  const int lane = threadIdx.x % TL, D = a.features;
  const float width = (float)D;
  const int64_t pitch = fa_code_pitch(D), epitch = fa_exponent_pitch(D);
  const int w = worker_of(ch.first, a.blocks.p, blockIdx.x);
  // (a worker's chunks take its rows in turn: rows that are read at one time lie together, and not one chunk apart, which
  // for many widths would be the same few channels of the memory)
  const int64_t begin = a.blocks.row0[w] + (int64_t)(blockIdx.x - ch.first[w]) * TEAMS, end = a.blocks.row0[w + 1];
  const int64_t step = (int64_t)(ch.first[w + 1] - ch.first[w]) * TEAMS;
  constexpr bool WIDE = L == 64;
  const T* dy = static_cast<const T*>(a.dy);
  const T* x = static_cast<const T*>(a.x);
  const T* residual = static_cast<const T*>(a.residual);
  raw8<T> next_dy[NC], next_x[KEPT ? 1 : NC];
  uint2 next_codes[KEPT ? NC : 1];
  uint32_t next_e[KEPT ? NC : 1];
  uint32_t last_dy = 0, last_x = 0;
  float next_mean = 0.f, next_rstd = 0.f;
  auto load = [&](int64_t row) __attribute__((always_inline)) {
    next_rstd = a.rstd[row];
    const row_in<WIDE, T> in(dy + row * a.lddy, D);
#pragma unroll
    for (int c = 0; c < NC; ++c) next_dy[c] = in.load(8 * (lane + TL * c), D);
    last_dy = in.last();
    if constexpr (KEPT) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int at = 8 * (lane + TL * c);
        if constexpr (WIDE) {
          const __amdgpu_buffer_rsrc_t codes =
              __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(a.codes) + row * pitch, 0, (int)pitch, 0x00020000);
          const __amdgpu_buffer_rsrc_t exponents =
              __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.exponents) + row * epitch, 0, (int)epitch, 0x00020000);
          next_codes[c] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(codes, at, 0, 0));
          next_e[c] = __builtin_amdgcn_raw_buffer_load_b32(exponents, at >> 5 & ~3, 0, 0);
        } else {
          next_codes[c] = make_uint2(0u, 0u);
          next_e[c] = 0u;
          if (at < pitch) {
            next_codes[c] = *reinterpret_cast<const uint2*>(a.codes + row * pitch + at);
            next_e[c] = a.exponents[row * epitch + (at >> 5)];
          }
        }
      }
    } else {
      next_mean = a.mean[row];
      const row_in<WIDE, T> from(x + row * a.ldx, D);
#pragma unroll
      for (int c = 0; c < NC; ++c) next_x[c] = from.load(8 * (lane + TL * c), D);
      last_x = from.last();
    }
  };
  int team = threadIdx.x / TL;
  if constexpr (WIDE) team = __builtin_amdgcn_readfirstlane(team);
  int64_t row = begin + team;
  if (row < end) load(row);
  float gamma[NC][8], dg[NC][8], db[NC][8];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int at = 8 * (lane + TL * c);
    if (a.gamma) fa_load8_param(a.gamma, a.param_bf16, at, D - at, gamma[c]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dg[c][e] = db[c][e] = 0.f;
      if (!a.gamma) gamma[c][e] = 1.f;
    }
  }
  int turn = 0;
  for (; row < end; row += step, turn ^= 1) {
    // (copied here and not where the next one arrives, which would be a wait for it)
    float rstd;
    asm volatile("v_mov_b32 %0, %1" : "=v"(rstd) : "v"(next_rstd));
    const float mean = next_mean;
    float xh[NC][8], h[NC][8];
    raw8<T> res[NC];
    uint32_t last_res = 0;
    // the residual is wanted at the end of the row: this one's
    if (WIDE || residual) {
      const row_in<WIDE, T> more(residual ? residual + row * a.ldr : nullptr, D);
#pragma unroll
      for (int c = 0; c < NC; ++c) res[c] = more.load(8 * (lane + TL * c), D);
      last_res = more.last();
    }
    // (what lies past the end of the row is zero in h, and so adds nothing)
    each_piece<NC>([&](auto c, auto last) __attribute__((always_inline)) {
      const int at = 8 * (lane + TL * c);
      values<WIDE, last>(next_dy[c], last_dy, at, D, h[c]);
      if constexpr (KEPT) {
        asm("" : "+v"(next_codes[c].x), "+v"(next_codes[c].y), "+v"(next_e[c]));
        uint32_t e = next_e[c];
        if constexpr (WIDE) {            // the byte of the word; what is past the last block is not written there
          e = e >> (at >> 2 & 24) & 255u;
          if constexpr (last) e = at < pitch ? e : 0u;
        }
        fa_values8(next_codes[c], fa_block_scale(e), xh[c]);
      } else {
        values<WIDE, last>(next_x[c], last_x, at, D, xh[c]);
#pragma unroll
        for (int e = 0; e < 8; ++e) xh[c][e] = (xh[c][e] - mean) * rstd;
      }
    });
    load(row + step < end ? row + step : row);
    __builtin_amdgcn_sched_barrier(0);
    float s = 0.f, q = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        db[c][e] += h[c][e];
        dg[c][e] += h[c][e] * xh[c][e];
        h[c][e] *= gamma[c][e];
        s += h[c][e];
        q += h[c][e] * xh[c][e];
      }
    s = team_sum<L>(s);
    q = team_sum<L>(q);
    if constexpr (W > 1) {
      // (two slots in turn: a wavefront is past the next row's barrier before anyone writes this slot again)
      if (threadIdx.x % 64 == 0) red[turn][threadIdx.x / 64] = make_float2(s, q);
      __syncthreads();
      s = q = 0.f;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        s += red[turn][k].x;
        q += red[turn][k].y;
      }
    }
    s /= width;
    q /= width;
    T* dx = static_cast<T*>(a.dx) + row * a.lddx;
    each_piece<NC>([&](auto c, auto last) __attribute__((always_inline)) {
      const int at = 8 * (lane + TL * c);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[c][e] = rstd * (h[c][e] - s - xh[c][e] * q);
      if (WIDE || residual) {
        float r[8];
        values<WIDE, last>(res[c], last_res, at, D, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] += r[e];
      }
      store_piece<WIDE, last>(dx, at, D, h[c]);
    });
  }
  if (!a.dgamma && !a.dbeta) return;
  float* part = a.partials + (int64_t)blockIdx.x * 2 * D;
  if constexpr (W > 1) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int at = 8 * (lane + TL * c);
      fa_store8(part + at, D - at, dg[c]);
      fa_store8(part + D + at, D - at, db[c]);
    }
  } else {
    // the teams of a wavefront by shuffles, then the wavefronts through LDS, in their order
    constexpr int SPAN = L * NC * 8;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int d = L; d < 64; d *= 2) {
          dg[c][e] += __shfl_xor(dg[c][e], d);
          db[c][e] += __shfl_xor(db[c][e], d);
        }
    if (threadIdx.x % 64 < L) {
      float* mine = join + (threadIdx.x / 64) * 2 * SPAN;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          mine[8 * (lane + L * c) + e] = dg[c][e];
          mine[SPAN + 8 * (lane + L * c) + e] = db[c][e];
        }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 2 * D; k += THREADS) {
      const int at = k < D ? k : SPAN + k - D;
      float s = 0.f;
#pragma unroll
      for (int v = 0; v < WAVES; ++v) s += join[v * 2 * SPAN + at];
      part[k] = s;
    }
  }
}

// dgamma (blockIdx.z = 0) and dbeta (1) of one worker: its chunks' shares in eight interleaved sums, these in their order.
// Latency: a thread has eight loads in flight.  768 chunks of 4096 features (25 MB, from the cache) 7.2 us, of 768 3.9 us.
__global__ __launch_bounds__(kThreads) void fa_layer_norm_grads_kernel(fa_norm_grad_args a, norm_chunks ch) {
  constexpr int GROUPS = 8, COLUMNS = kThreads / GROUPS, DEEP = 8;
  __shared__ float red[GROUPS][COLUMNS];
  const int w = blockIdx.y, which = blockIdx.z, D = a.features;
  void* out = which ? a.dbeta : a.dgamma;
  if (!out) return;
  const int j = blockIdx.x * COLUMNS + threadIdx.x % COLUMNS, group = threadIdx.x / COLUMNS;
  float s = 0.f;
  if (j < D)
    for (int k = ch.first[w] + group; k < ch.first[w + 1]; k += GROUPS * DEEP) {
      float v[DEEP];
#pragma unroll
      for (int n = 0; n < DEEP; ++n) {
        const int at = k + GROUPS * n;
        v[n] = at < ch.first[w + 1] ? a.partials[((int64_t)at * 2 + which) * D + j] : 0.f;
      }
#pragma unroll
      for (int n = 0; n < DEEP; ++n) s += v[n];
    }
  red[group][threadIdx.x % COLUMNS] = s;
  __syncthreads();
  if (group == 0 && j < D) {
    s = 0.f;
#pragma unroll
    for (int n = 0; n < GROUPS; ++n) s += red[n][threadIdx.x];
    const int64_t at = (int64_t)w * (which ? a.lddbeta : a.lddgamma) + j;
    if (a.grad_bf16) fa_store1(static_cast<fa_bf16*>(out) + at, s);
    else fa_store1(static_cast<float*>(out) + at, s);
  }
}

// Any activation to a checkpoint: one pass bound by memory, every element read once.  9999 x 1111 fp32 10.1 us = 5.5 TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void fa_checkpoint_pack_kernel(const T* x, int64_t ldx, int64_t rows, int D, int8_t* codes,
                                                                      uint8_t* exponents) {
  // a thread for every eight codes of a padded row: four of them are one block, whichever row they are in
  const int64_t pitch = fa_code_pitch(D), epitch = fa_exponent_pitch(D);
  const int64_t per_row = pitch / 8, total = rows * per_row;
  const int64_t whole = (total + 63) / 64 * 64;   // (all lanes of a wavefront stay for the exchange between lanes)
  for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < whole; k += (int64_t)gridDim.x * kThreads) {
    const int64_t row = k / per_row;
    const int at = 8 * (int)(k - row * per_row);
    float v[8];
    fa_load8(x + row * ldx + at, k < total ? D - at : 0, v);
    const uint32_t e = fa_block_exponent(fa_quad_most(v));
    if (k < total) {
      *reinterpret_cast<uint2*>(codes + row * pitch + at) = fa_codes8(v, e);
      if ((k & 3) == 0) exponents[row * epitch + (at >> 5)] = (uint8_t)e;
    }
  }
}

// And back, a thread for every eight codes: bound by its writes.  65536 x 4096 to bf16 155 us = 5.2 TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void fa_checkpoint_unpack_kernel(const int8_t* codes, const uint8_t* exponents, int64_t rows,
                                                                        int D, T* x, int64_t ldx) {
  const int64_t pitch = fa_code_pitch(D), epitch = fa_exponent_pitch(D);
  const int64_t per_row = pitch / 8, total = rows * per_row;
  for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < total; k += (int64_t)gridDim.x * kThreads) {
    const int64_t row = k / per_row;
    const int at = 8 * (int)(k - row * per_row);
    float v[8];
    fa_values8(*reinterpret_cast<const uint2*>(codes + row * pitch + at), fa_block_scale(exponents[row * epitch + (at >> 5)]), v);
    fa_store8(x + row * ldx + at, D - at, v);
  }
}

namespace {

int grid_for(int64_t threads) {
  const int64_t blocks = (threads + kThreads - 1) / kThreads;
  return (int)(blocks < 1 ? 1 : blocks > 8192 ? 8192 : blocks);
}

// A team for the widths LOW < D <= HIGH: all its pieces but the last are whole, which the kernels take for granted.
template <int LOW, int HIGH, int L_, int NC_, int W_>
struct team_of {
  static constexpr int L = L_, NC = NC_, W = W_;
  static_assert(HIGH <= 8 * L * W * NC && LOW >= 8 * L * W * (NC - 1), "the pieces of a row");
};

template <typename T, typename TEAM>
void norm(const fa_norm_args& a, hipStream_t st) {
  constexpr int L = TEAM::L, NC = TEAM::NC, W = TEAM::W;
  const int teams = W > 1 ? 1 : kThreads / L;
  int64_t blocks = (a.rows + teams - 1) / teams;
  if (blocks > 2048) blocks = 2048;
  const dim3 grid((unsigned)blocks), block(W > 1 ? 64 * W : kThreads);
  if (a.codes) hipLaunchKernelGGL((fa_layer_norm_kernel<T, true, L, NC, W>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((fa_layer_norm_kernel<T, false, L, NC, W>), grid, block, 0, st, a);
}

// The team of a width: no more lanes than the row has work for, all pieces but the last whole.
template <typename T>
hipError_t norm_of(const fa_norm_args& a, hipStream_t st) {
  const int D = a.features;
  if (D <= 32) norm<T, team_of<0, 32, 4, 1, 1>>(a, st);
  else if (D <= 128) norm<T, team_of<32, 128, 16, 1, 1>>(a, st);
  else if (D <= 256) norm<T, team_of<128, 256, 32, 1, 1>>(a, st);
  else if (D <= 512) norm<T, team_of<256, 512, 64, 1, 1>>(a, st);
  else if (D <= 1024) norm<T, team_of<512, 1024, 64, 2, 1>>(a, st);
  else if (D <= 1536) norm<T, team_of<1024, 1536, 64, 3, 1>>(a, st);
  else if (D <= 2048) norm<T, team_of<1536, 2048, 64, 4, 1>>(a, st);
  else if (D <= 4096) norm<T, team_of<2048, 4096, 64, 2, 4>>(a, st);
  else if (D <= 6144) norm<T, team_of<4096, 6144, 64, 3, 4>>(a, st);
  else if (D <= 8192) norm<T, team_of<6144, 8192, 64, 4, 4>>(a, st);
  else if (D <= 12288) norm<T, team_of<8192, 12288, 64, 3, 8>>(a, st);
  else norm<T, team_of<12288, FA_NORM_FEATURES_MAX, 64, 4, 8>>(a, st);
  return hipGetLastError();
}

template <typename T, bool KEPT, typename TEAM>
void norm_backward(const fa_norm_grad_args& a, const norm_chunks& ch, hipStream_t st) {
  constexpr int L = TEAM::L, NC = TEAM::NC, W = TEAM::W;
  hipLaunchKernelGGL((fa_layer_norm_backward_kernel<T, KEPT, L, NC, W>), dim3((unsigned)ch.first[FA_P_MAX]),
                     dim3(W > 1 ? 64 * W : kThreads), 0, st, a, ch);
}

template <typename T, bool KEPT>
void norm_backward_of(const fa_norm_grad_args& a, const norm_chunks& ch, hipStream_t st) {
  const int D = a.features;
  if (D <= 32) norm_backward<T, KEPT, team_of<0, 32, 4, 1, 1>>(a, ch, st);
  else if (D <= 128) norm_backward<T, KEPT, team_of<32, 128, 16, 1, 1>>(a, ch, st);
  else if (D <= 256) norm_backward<T, KEPT, team_of<128, 256, 32, 1, 1>>(a, ch, st);
  else if (D <= 512) norm_backward<T, KEPT, team_of<256, 512, 64, 1, 1>>(a, ch, st);
  else if (D <= 1024) norm_backward<T, KEPT, team_of<512, 1024, 64, 2, 1>>(a, ch, st);
  else if (D <= 2048) norm_backward<T, KEPT, team_of<1024, 2048, 64, 1, 4>>(a, ch, st);
  else if (D <= 4096) norm_backward<T, KEPT, team_of<2048, 4096, 64, 2, 4>>(a, ch, st);
  else if (D <= 8192) norm_backward<T, KEPT, team_of<4096, 8192, 64, 2, 8>>(a, ch, st);
  else if (D <= 12288) norm_backward<T, KEPT, team_of<8192, 12288, 64, 3, 8>>(a, ch, st);
  else norm_backward<T, KEPT, team_of<12288, FA_NORM_FEATURES_MAX, 64, 4, 8>>(a, ch, st);
}

}  // namespace

hipError_t fa_launch_checkpoint_pack(const void* x, int64_t ldx, int64_t rows, int features, int dtype, int8_t* codes,
                                     uint8_t* exponents, hipStream_t st) {
  const dim3 grid(grid_for(rows * (fa_code_pitch(features) / 8))), block(kThreads);
  if (dtype == FA_F32)
    hipLaunchKernelGGL(fa_checkpoint_pack_kernel<float>, grid, block, 0, st, static_cast<const float*>(x), ldx, rows, features,
                       codes, exponents);
  else
    hipLaunchKernelGGL(fa_checkpoint_pack_kernel<fa_bf16>, grid, block, 0, st, static_cast<const fa_bf16*>(x), ldx, rows, features,
                       codes, exponents);
  return hipGetLastError();
}

hipError_t fa_launch_checkpoint_unpack(const int8_t* codes, const uint8_t* exponents, int64_t rows, int features, int dtype,
                                       void* x, int64_t ldx, hipStream_t st) {
  const dim3 grid(grid_for(rows * (fa_code_pitch(features) / 8))), block(kThreads);
  if (dtype == FA_F32)
    hipLaunchKernelGGL(fa_checkpoint_unpack_kernel<float>, grid, block, 0, st, codes, exponents, rows, features,
                       static_cast<float*>(x), ldx);
  else
    hipLaunchKernelGGL(fa_checkpoint_unpack_kernel<fa_bf16>, grid, block, 0, st, codes, exponents, rows, features,
                       static_cast<fa_bf16*>(x), ldx);
  return hipGetLastError();
}

hipError_t fa_launch_layer_norm(const fa_norm_args& a, int dtype, hipStream_t st) {
  return dtype == FA_F32 ? norm_of<float>(a, st) : norm_of<fa_bf16>(a, st);
}

size_t fa_layer_norm_partials(const fa_row_blocks& b, int64_t rows, int features) {
  return sizeof(float) * 2 * (size_t)cut(b, rows).first[FA_P_MAX] * (size_t)features;
}

hipError_t fa_launch_layer_norm_backward(const fa_norm_grad_args& a, int dtype, hipStream_t st) {
  const norm_chunks ch = cut(a.blocks, a.rows);
  if (a.rows > 0) {
    const bool kept = a.x == nullptr;
    if (dtype == FA_F32) {
      if (kept) norm_backward_of<float, true>(a, ch, st);
      else norm_backward_of<float, false>(a, ch, st);
    } else {
      if (kept) norm_backward_of<fa_bf16, true>(a, ch, st);
      else norm_backward_of<fa_bf16, false>(a, ch, st);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dgamma || a.dbeta)
    hipLaunchKernelGGL(fa_layer_norm_grads_kernel, dim3((unsigned)((a.features + 31) / 32), (unsigned)a.blocks.p, 2),
                       dim3(kThreads), 0, st, a, ch);
  return hipGetLastError();
}
