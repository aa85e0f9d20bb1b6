// Weight and bias gradients of a linear layer, worker by worker, from the 8-bit checkpoint of its input.
//
//   P_w[o, i] = sum over the rows t of worker w of dY[t, o] v[t, i],    b_w[o] = the same sum of dY[t, o],
//   dW_w = gamma_i P_w + beta_i b_w[o]  (the layer's input was v gamma + beta)   or   dW_w = P_w,    db_w = b_w,
//
// where v are the checkpoint's values.  They have seven significant bits, so they are exact in bf16; dY is bf16, or fp32
// cut into three pieces of eight bits: exactly, but below 2^-110, where the lowest piece is cut off at 2^-133, the last place
// of bf16.  Every product on the bf16 matrix core is exact, subnormal ones too, sums are fp32.  The rows are
// the contracted index of both operands and lie far apart in memory; a lane of the matrix instruction takes eight
// consecutive ones of a column, so tiles are turned on their way to LDS.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fa.h"
#include "fa_layers.h"
#include "fa_linear_plan.h"

namespace {

constexpr int kThreads = 256;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// x = h + m + l, each with eight significant bits (l to 2^-133 at the lowest), h and m cut off (h of the largest finite value
// stays finite).  An infinity is h, with nothing left over; of a NaN, whatever h is, m is one.
__device__ __forceinline__ void split3(float x, uint32_t* h, uint32_t* m, uint32_t* l) {
  const uint32_t hu = __float_as_uint(x) & 0xffff0000u;
  const float left = x - __uint_as_float(hu), r = __builtin_amdgcn_classf(x, 0x204) ? 0.f : left;
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
//
// Rows come in steps of BK.  While the matrix core works on one step in LDS, the next one, already in registers, is made
// into the other half of LDS and the one after it is on its way from memory: one barrier a step, no wait on memory.  A
// thread brings in 8 rows of a few outputs of dY and 8 rows of a few codes, and turns them on the way: LDS holds, for
// every output (feature), the BK values of the contracted index in pieces of 8, which is what a lane of the matrix
// instruction takes with one 16-byte read.  Piece c of column j lies at place c ^ swizzle(j): 16 lanes that read one
// piece of 16 neighbouring columns, and 8 that write one piece of every second, fourth or eighth column (as wide as a
// thread's unit is), meet no bank twice (65536 x 4096 x 4096: 4.2e6 cycles of conflicts to 2.9e8 in which LDS works, all of
// them in the reads of finished results; with column / 8 in place of column / 16 in swizzle() 1.39e8).
namespace {

template <typename T, int BM, int BN, int BK>
struct tile {
  static constexpr int PLANES = sizeof(T) == 4 ? 3 : 1;
  static constexpr int ROW = BK * 2;                           // LDS bytes of a column
  static constexpr int A_BYTES = BM * ROW * PLANES, B_BYTES = BN * ROW;   // of one step; LDS: dY, dY, codes, codes
  static constexpr int PIECES = BK / 8;
  // a thread's unit of dY is 8 rows of AC outputs, its unit of codes 8 rows of BC features
  static constexpr int AC = BM * PIECES / kThreads, BC = BN * PIECES / kThreads;
  static constexpr int AW = AC * (int)sizeof(T) / 4, BW = BC / 4;           // dwords of a row of it
  static_assert((AW == 2 || AW == 4) && (BW == 1 || BW == 2), "loads of 8 or 16, and of 4 or 8 bytes");
  static_assert(BK == 64 && PIECES == 8, "swizzle() is for eight pieces");
};

__device__ __forceinline__ int swizzle(int column) { return ((column >> 1) ^ (column >> 4)) & 7; }

__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");   // (loads from memory stay in flight)
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The tile of workgroup b of n.  Workgroups go to the eight dies in turn, and every die has its own L2: each gets one run of
// consecutive tiles, in which bands of four rows of tiles are walked column by column, so that the 32 workgroups of a die
// share four strips of dY and eight of codes.
struct place {
  int group, to, ti;   // which worker and split, which tile
};
__device__ __forceinline__ place place_of(uint32_t b, uint32_t n, int tiles_o, int tiles_i) {
  const uint32_t die = b % 8, whole = n / 8, more = n % 8;
  const uint32_t id = die * whole + min(die, more) + b / 8;
  const uint32_t per_group = (uint32_t)tiles_o * tiles_i, in = id % per_group;
  const uint32_t band = in / (4 * tiles_i), rest = in - band * 4 * tiles_i;
  const uint32_t rows = min(4u, tiles_o - 4 * band);
  return {(int)(id / per_group), (int)(4 * band + rest % rows), (int)(rest / rows)};
}

template <int N>
using words = uint32_t __attribute__((ext_vector_type(N)));

template <int N>
__device__ __forceinline__ words<N> load_words(const unsigned char* p) {   // at any address
  words<N> u;
  __builtin_memcpy(&u, p, sizeof(u));
  return u;
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const unsigned char* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(p), 0, bytes, 0x00020000);
}
template <int N>
__device__ __forceinline__ words<N> buffer_words(__amdgpu_buffer_rsrc_t r, uint32_t lane, int row) {
  if constexpr (N == 4) return __builtin_bit_cast(words<4>, __builtin_amdgcn_raw_buffer_load_b128(r, lane, row, 0));
  else if constexpr (N == 2) return __builtin_bit_cast(words<2>, __builtin_amdgcn_raw_buffer_load_b64(r, lane, row, 0));
  else return __builtin_bit_cast(words<1>, __builtin_amdgcn_raw_buffer_load_b32(r, lane, row, 0));
}
// a unit's row of dY of which the first `valid` elements exist, zeros behind them
template <int N>
__device__ __forceinline__ words<N> load_some(const fa_bf16* p, int valid) {
  words<N> u = {};
  if (valid >= 2 * N) return load_words<N>(reinterpret_cast<const unsigned char*>(p));
#pragma unroll
  for (int e = 0; e < 2 * N; ++e)
    if (e < valid) u[e >> 1] |= (uint32_t)p[e].bits << (16 * (e & 1));
  return u;
}
template <int N>
__device__ __forceinline__ words<N> load_some(const float* p, int valid) {
  words<N> u = {};
  if (valid >= N) return load_words<N>(reinterpret_cast<const unsigned char*>(p));
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < valid) u[e] = __float_as_uint(p[e]);
  return u;
}

// A wavefront issues in order: what is not a product goes between the products, a few instructions behind each, and costs
// nothing there.  PRODUCTS matrix instructions, READS and WRITES of LDS and the vector instructions of a region.
// (READS first, two behind a product, then the writes: nothing tells the compiler that those go to the other half.  Of the
// WRITES, the LATE last ones are of dY in three pieces, and wait for most of the vector instructions.)
template <int PRODUCTS, int READS, int WRITES, int LATE, int VECTOR, int I = 0>
__device__ __forceinline__ void interleave() {
  if constexpr (I < PRODUCTS) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                        // a product
    if constexpr (2 * I < READS) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    __builtin_amdgcn_sched_group_barrier(0x020, 2, 0);                                        // loads from memory
    constexpr int V = VECTOR * (I + 1) / PRODUCTS - VECTOR * I / PRODUCTS;
    if constexpr (V > 0) __builtin_amdgcn_sched_group_barrier(0x002, V, 0);
    constexpr int FROM = READS / 2, EARLY = WRITES - LATE, LAST = LATE > 0 ? PRODUCTS / 2 : PRODUCTS;
    constexpr int OVER = LAST - FROM > 0 ? LAST - FROM : 1, J = I - FROM < OVER ? I - FROM : OVER - 1;
    constexpr int W = J < 0 || I >= LAST ? 0 : EARLY * (J + 1) / OVER - EARLY * J / OVER;
    constexpr int W_LATE = LATE == 0 ? 0 : I == PRODUCTS - 1 ? LATE - LATE / 2 : I == PRODUCTS - 2 ? LATE / 2 : 0;
    if constexpr (W + W_LATE > 0) __builtin_amdgcn_sched_group_barrier(0x200, W + W_LATE, 0);
    interleave<PRODUCTS, READS, WRITES, LATE, VECTOR, I + 1>();
  }
}

// s + the sum of eight bf16 values, in fp32
__device__ __forceinline__ float add8(bf16x8 v, float s) {
  const fa_bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
  const fa_u32x4 u = __builtin_bit_cast(fa_u32x4, v);
#pragma unroll
  for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(fa_bf16x2, (uint32_t)u[e]), one, s, false);
  return s;
}

}  // namespace

// What bounds it: in long workers, issue and what it waits for.  A SIMD has one wavefront (its results take half of the
// registers), which issues 4.2 vector, 0.8 LDS and 1.1 other instructions for every product, in order: the matrix core is busy
// 51 % of the cycles (at 2.0 GHz), the wavefront waits in 42 %.  A wavefront makes 128 x 128 results, 16 products for 8 reads
// of LDS: 65536 x 4096 x 4096 in 2.04 to 2.11 ms = 1.04 to 1.08 PFLOP/s, as long as one plain product per worker in a
// library (2.08 ms); with 128 x 64 and two wavefronts a SIMD 2.20 ms, with 64 x 128 (tiles of 128 x 256) 2.59, with 64 x 64
// (128 x 128, two workgroups a compute unit) 2.93.  At 2.16 ms it took 1.57 without turning tiles and writing them, 1.69
// without loads, 2.07 without column sums.
// Few steps: 15 x 1024 rows of 768 -> 2304, bf16 to fp32, 86 us = 0.63 PFLOP/s, in 405 tiles for 256 compute units; the results
// are 106 MB that are written at one time at the end of a tile (65 us without it).  fp32 dY, three products for one: 60
// uneven workers, 30011 rows of 1001 -> 509, 133 us = 0.23 PFLOP/s, 0.69 with the pieces.  7 x 32 rows of 48 -> 64: 7.4 us.  (Kernels
// alone, on a card that has been at work for some milliseconds.)
template <typename T, int BM, int BN, int BK>
__global__ __launch_bounds__(kThreads, 1) void fa_linear_grad_kernel(fa_linear_grad_args a) {
  using S = tile<T, BM, BN, BK>;
  constexpr int FM = BM / 64, FN = BN / 64;               // 32 x 32 results of a wavefront in either direction
  constexpr int HM = FM > 1 ? FM / 2 : 1;                 // of the FM, those whose column sums a wavefront makes
  constexpr int AC = S::AC, KK = BK / 16;
  __shared__ __attribute__((aligned(16))) unsigned char lds[2 * (S::A_BYTES + S::B_BYTES)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tiles_o = (a.outputs + BM - 1) / BM, tiles_i = (a.features + BN - 1) / BN;
  const place at = place_of(blockIdx.x, gridDim.x, tiles_o, tiles_i);
  const int split = at.group % a.splits, w = at.group / a.splits;
  const int o0 = at.to * BM, i0 = at.ti * BN;
  // this split's rows: whole steps of BK rows
  const int64_t all = a.blocks.row0[w + 1] - a.blocks.row0[w];
  const int64_t steps_all = (all + BK - 1) / BK, per = (steps_all + a.splits - 1) / a.splits;
  const int64_t begin = a.blocks.row0[w] + min(all, (int64_t)split * per * BK);
  const int64_t end = a.blocks.row0[w] + min(all, ((int64_t)split + 1) * per * BK);
  const int64_t pitch = fa_code_pitch(a.features), epitch = fa_exponent_pitch(a.features);

  // The unit of dY and the unit of codes that this thread brings in: rows 8 piece.., columns.  Columns past the matrix
  // take part like any other and are not written at the end: what is read for them is the tile's first unit, or, where
  // the last column is inside the unit, the next row's beginning.  A step is a buffer that ends with the last element of its
  // last row: rows past the end come as zeros, and so does what would lie behind the matrix.  The end is kept in words of
  // four bytes, in which the last column of an odd number of bf16 would be lost: there the last step is taken element by
  // element behind the others.
  const int a_col = tid % (BM / AC) * AC, a_piece = tid / (BM / AC);
  const int b_col = tid % (BN / S::BC) * S::BC, b_piece = tid / (BN / S::BC);
  const int64_t steps = (end - begin + BK - 1) / BK;
  const bool odd = sizeof(T) == 2 && (a.outputs & 1);
  const bool near = a.lddy < (1 << 22);                   // the bytes of a step, and one row more, fit in 31 bits
  const int64_t fast = !near || steps == 0 ? 0 : odd ? steps - 1 : steps;
  const uint32_t a_off = (uint32_t)((int64_t)a_piece * 8 * a.lddy + (o0 + a_col < a.outputs ? a_col : 0)) * (uint32_t)sizeof(T);
  const int b_safe = i0 + b_col < pitch ? b_col : 0;
  const uint32_t b_off = (uint32_t)(b_piece * 8 * (int)pitch + b_safe);
  const uint32_t e_off = (uint32_t)(b_piece * 8 * (int)epitch + (b_safe >> 5));
  using AR = words<S::AW>;
  using BR = words<S::BW>;
  AR raw_a[2][8];
  BR raw_b[2][8];
  uint32_t raw_e[2][8];
  float sum[HM];
#pragma unroll
  for (int m = 0; m < HM; ++m) sum[m] = 0.f;
  f32x16 acc[FM][FN];
#pragma unroll
  for (int m = 0; m < FM; ++m)
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.f;

  // One of the fast steps from memory into registers, and on to the next.  (Buffer loads: a lane's place in the step, a row's
  // distance and the step's own address are three operands of the instruction, none of them is added up for a load.)
  const unsigned char* at_dy = static_cast<const unsigned char*>(a.dy) + (begin * a.lddy + o0) * (int64_t)sizeof(T);
  const unsigned char* at_codes = reinterpret_cast<const unsigned char*>(a.codes) + begin * pitch + i0;
  const unsigned char* at_exponents = a.exponents + begin * epitch + (i0 >> 5);
  const int row_dy = near ? (int)a.lddy * (int)sizeof(T) : 0, row_codes = (int)pitch, row_exponents = (int)epitch;
  // (ends of a step's buffers: of the last one's rows, of one row more than a step has where there is one more)
  const int rows_last = (int)(end - begin - (steps - 1) * BK), wide_dy = (a.outputs - o0) * (int)sizeof(T);
  const int last_dy = (rows_last - 1) * row_dy + wide_dy, full_dy = BK * row_dy + wide_dy;
  const int last_codes = rows_last * row_codes - i0, full_codes = BK * row_codes;
  const int last_exponents = rows_last * row_exponents - (i0 >> 5), full_exponents = BK * row_exponents;
  const uint32_t step_dy = BK * row_dy, step_codes = BK * row_codes, step_exponents = BK * row_exponents;
  int todo = (int)steps;                                  // steps from the one that is loaded next
  // (part 0 and 1, half of the rows each; a step's own address goes on behind part 1, the last step comes again and again)
  auto load = [&](int part, AR (&ra)[8], BR (&rb)[8], uint32_t (&re)[8]) __attribute__((always_inline)) {
    const bool more = todo > 1;
    const __amdgpu_buffer_rsrc_t dy = buffer(at_dy, more ? full_dy : last_dy),
                                 codes = buffer(at_codes, more ? full_codes : last_codes),
                                 exponents = buffer(at_exponents, more ? full_exponents : last_exponents);
#pragma unroll
    for (int j = 4 * part; j < 4 * part + 4; ++j) {
      ra[j] = buffer_words<S::AW>(dy, a_off, j * row_dy);
      rb[j] = buffer_words<S::BW>(codes, b_off, j * row_codes);
      re[j] = __builtin_amdgcn_raw_buffer_load_b8(exponents, e_off, j * row_exponents, 0);
    }
    if (part == 1) {
      at_dy += more ? step_dy : 0u;
      at_codes += more ? step_codes : 0u;
      at_exponents += more ? step_exponents : 0u;
      todo -= more ? 1 : 0;
    }
  };
  // any step; rows past the end are zero, and nothing that is not there is read
  auto load_edge = [&](int64_t k, AR (&ra)[8], BR (&rb)[8], uint32_t (&re)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t ta = begin + k * BK + a_piece * 8 + j, tb = begin + k * BK + b_piece * 8 + j;
      ra[j] = load_some<S::AW>(static_cast<const T*>(a.dy) + ta * a.lddy + o0 + a_col, ta < end ? a.outputs - o0 - a_col : 0);
      rb[j] = BR{};
      re[j] = 0u;
      if (tb < end) {
        rb[j] = *reinterpret_cast<const BR*>(a.codes + tb * pitch + i0 + b_safe);
        re[j] = a.exponents[tb * epitch + ((i0 + b_safe) >> 5)];
      }
    }
  };
  // Places in LDS as a few addresses of the lane and constants.  With column j = 8 g + r, swizzle(j) = swizzle(8 g) ^ (r / 2):
  // a unit's column 8 g + r is written at put[r / 2] + r ROW.  With j = j0 + 32 m in a run of 32, 64 or 128 columns that
  // begins at a multiple of its length, j0 in its first 32, swizzle(j) = swizzle(j0) ^ 2 m: piece 2 kk + lane / 32 of it is
  // read at get[kk ^ m] + 32 m ROW.  Of the two wavefronts that share their outputs, each adds up one half of them, the
  // half that it takes first: its results are in the order turned by `turn`.
  uint32_t put_a[4], put_b[4], get_first[4], get_last[4], get_b[4];
  const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
  const int turn = FM > 1 ? (wave & 1) * HM : 0;
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    put_a[y] = a_col * S::ROW + ((a_piece ^ swizzle(a_col) ^ y) << 4);
    put_b[y] = 2 * S::A_BYTES + b_col * S::ROW + ((b_piece ^ swizzle(b_col) ^ y) << 4);
    const int jf = wm + 32 * turn + (lane & 31), jl = wm + 32 * (HM - turn) + (lane & 31), jb = wn + (lane & 31);
    const int piece = (lane >> 5) ^ (2 * y);
    get_first[y] = jf * S::ROW + ((piece ^ swizzle(jf)) << 4);
    get_last[y] = jl * S::ROW + ((piece ^ swizzle(jl)) << 4);
    get_b[y] = 2 * S::A_BYTES + jb * S::ROW + ((piece ^ swizzle(jb)) << 4);
  }
  // a quarter (of four) of a step's registers into LDS
  auto stage_dy = [&](int quarter, int half, const AR (&ra)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int c = quarter * AC / 4; c < (quarter + 1) * AC / 4; ++c) {
      unsigned char* at = lds + put_a[c >> 1] + (half * S::A_BYTES + c * S::ROW);
      fa_u32x4 u[3];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (S::PLANES == 1) {
          u[0][e] = __builtin_amdgcn_perm(ra[2 * e + 1][c >> 1], ra[2 * e][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
        } else {
          uint32_t h0, m0, l0, h1, m1, l1;
          split3(__uint_as_float(ra[2 * e][c]), &h0, &m0, &l0);
          split3(__uint_as_float(ra[2 * e + 1][c]), &h1, &m1, &l1);
          u[0][e] = upper_halves(h0, h1);
          u[1][e] = upper_halves(m0, m1);
          u[2][e] = upper_halves(l0, l1);
        }
      }
#pragma unroll
      for (int q = 0; q < S::PLANES; ++q) *reinterpret_cast<fa_u32x4*>(at + q * (BM * S::ROW)) = u[q];
    }
  };
  auto stage_codes = [&](int quarter, int half, const BR (&rb)[8], const uint32_t (&re)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int c = quarter * S::BC / 4; c < (quarter + 1) * S::BC / 4; ++c) {
      fa_u32x4 u;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v0 = (float)(int8_t)(rb[2 * e][c >> 2] >> (8 * (c & 3))) * fa_block_scale(re[2 * e]);
        const float v1 = (float)(int8_t)(rb[2 * e + 1][c >> 2] >> (8 * (c & 3))) * fa_block_scale(re[2 * e + 1]);
        u[e] = upper_halves(__float_as_uint(v0), __float_as_uint(v1));
      }
      *reinterpret_cast<fa_u32x4*>(lds + put_b[c >> 1] + (half * S::B_BYTES + c * S::ROW)) = u;
    }
  };
  auto stage = [&](int quarter, int half, const AR (&ra)[8], const BR (&rb)[8],
                   const uint32_t (&re)[8]) __attribute__((always_inline)) {
    if constexpr (S::PLANES == 1) stage_dy(quarter, half, ra);      // (fp32 pieces take long: last)
    stage_codes(quarter, half, rb, re);
    if constexpr (S::PLANES == 3) stage_dy(quarter, half, ra);
  };
  // the operands of 16 rows of a step, and their products
  auto fetch = [&](int half, int kk, bf16x8 (&fa)[S::PLANES][FM], bf16x8 (&fb)[FN]) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < FN; ++n)
      fb[n] = *reinterpret_cast<const bf16x8*>(lds + get_b[kk ^ n] + (half * S::B_BYTES + 32 * n * S::ROW));
#pragma unroll
    for (int q = 0; q < S::PLANES; ++q)
#pragma unroll
      for (int m = 0; m < FM; ++m) {
        const int mm = m < HM ? m : m - HM;
        const uint32_t at = m < HM ? get_first[kk ^ mm] : get_last[kk ^ mm];
        fa[q][m] = *reinterpret_cast<const bf16x8*>(lds + at + (half * S::A_BYTES + 32 * mm * S::ROW + q * (BM * S::ROW)));
      }
  };
  auto multiply = [&](const bf16x8 (&fa)[S::PLANES][FM], const bf16x8 (&fb)[FN]) __attribute__((always_inline)) {
#pragma unroll
    for (int q = S::PLANES - 1; q >= 0; --q)
#pragma unroll
      for (int m = 0; m < FM; ++m) {
        if (m < HM) sum[m] = add8(fa[q][m], sum[m]);
#pragma unroll
        for (int n = 0; n < FN; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[q][m], fb[n], acc[m][n], 0, 0, 0);
      }
  };
  // the registers of a step are what they were loaded as until here (the compiler would convert them where they arrive,
  // a step early, and has no registers for that)
  auto here = [&](AR (&ra)[8], BR (&rb)[8], uint32_t (&re)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      asm("" : "+v"(ra[j]), "+v"(re[j]));
      if constexpr (S::BW == 1) {
        uint32_t u = rb[j][0];
        asm("" : "+v"(u));
        rb[j][0] = u;
      } else {
        asm("" : "+v"(rb[j]));
      }
    }
  };
  // vector instructions of a quarter: 20 for a column of codes, 4 or 60 for one of dY, 4 for each column sum
  constexpr int kVector = S::BC / 4 * 20 + S::AC * (S::PLANES == 1 ? 4 : 60) / 4 + S::PLANES * HM * 4;
  bf16x8 fa[2][S::PLANES][FM], fb[2][FN];
  if (fast > 0) {
    // A step k in half k % 2 of LDS takes four regions of 16 rows.  In the first three the last quarters of step k + 1 are
    // put down; behind the barrier everyone is done reading step k and step k + 1 is complete, so that the fourth region
    // fetches the first operands of step k + 1, puts down the first quarter of step k + 2 where step k was, and sends
    // for step k + 3.  (Past the last fast step the last one comes again, and nobody uses it.)
    load(0, raw_a[0], raw_b[0], raw_e[0]);
    load(1, raw_a[0], raw_b[0], raw_e[0]);
    load(0, raw_a[1], raw_b[1], raw_e[1]);
    load(1, raw_a[1], raw_b[1], raw_e[1]);
#pragma unroll
    for (int q = 0; q < 4; ++q) stage(q, 0, raw_a[0], raw_b[0], raw_e[0]);
    load(0, raw_a[0], raw_b[0], raw_e[0]);
    lds_barrier();
    fetch(0, 0, fa[0], fb[0]);
    stage(0, 1, raw_a[1], raw_b[1], raw_e[1]);
    int64_t k = 0;
    for (; k + 1 < fast; k += 2) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          if (kk + 1 < KK) {
            fetch(half, kk + 1, fa[(kk + 1) & 1], fb[(kk + 1) & 1]);
            if (kk == 0) load(1, raw_a[half], raw_b[half], raw_e[half]);
          } else {
            lds_barrier();
            fetch(1 - half, 0, fa[0], fb[0]);
            load(0, raw_a[1 - half], raw_b[1 - half], raw_e[1 - half]);
            here(raw_a[half], raw_b[half], raw_e[half]);
          }
          multiply(fa[kk & 1], fb[kk & 1]);
          if (kk + 1 < KK) stage(kk + 1, 1 - half, raw_a[1 - half], raw_b[1 - half], raw_e[1 - half]);
          else stage(0, half, raw_a[half], raw_b[half], raw_e[half]);
          interleave<S::PLANES * FM * FN, S::PLANES * FM + FN, (S::PLANES * S::AC + S::BC) / 4,
                     S::PLANES == 3 ? S::PLANES * S::AC / 4 : 0, kVector>();
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if (k < fast) {
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        fetch(0, kk, fa[0], fb[0]);
        multiply(fa[0], fb[0]);
      }
    }
    lds_barrier();
  }
  for (int64_t k = fast; k < steps; ++k) {
    load_edge(k, raw_a[0], raw_b[0], raw_e[0]);
#pragma unroll
    for (int q = 0; q < 4; ++q) stage(q, 0, raw_a[0], raw_b[0], raw_e[0]);
    lds_barrier();
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      fetch(0, kk, fa[0], fb[0]);
      multiply(fa[0], fb[0]);
    }
    lds_barrier();
  }
  // b_w: the lanes l and l + 32 have the two halves of every eight rows
  float* bias = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int m = 0; m < HM; ++m) {
    sum[m] += __shfl_xor(sum[m], 32);
    if (lane < 32 && (FM > 1 || wn == 0)) bias[wm + 32 * (m + turn) + lane] = sum[m];
  }
  __syncthreads();
  const int64_t OI = (int64_t)a.outputs * a.features;
  float* part = a.splits > 1 ? a.partials + ((int64_t)w * a.splits + split) * (OI + a.outputs) : nullptr;
  if (at.ti == 0 && tid < BM && o0 + tid < a.outputs) {
    if (part) part[OI + o0 + tid] = bias[tid];
    else if (a.dbias && a.grad_bf16) fa_store1(static_cast<fa_bf16*>(a.dbias) + w * a.lddbias + o0 + tid, bias[tid]);
    else if (a.dbias) static_cast<float*>(a.dbias)[w * a.lddbias + o0 + tid] = bias[tid];
  }
  // A lane of a result block has single features of eight outputs; through LDS it gets eight features of one, and the
  // gradient is written 16 bytes or more a lane.  (Rows of a block are 32 bytes apart from whole banks: the two rows
  // that one store puts down, four apart, meet on no bank.)
  constexpr int PITCH = BN / 2 + 8, LANES = BN / 16, ROWS = 64 / LANES;
  static_assert(BM * 4 + 4 * 32 * PITCH * 4 <= (int)sizeof(lds), "a block of every wavefront fits");
  float* block = bias + BM + wave * 32 * PITCH;
  const int i = i0 + wn + lane % LANES * 8, valid = a.features - i;
  float gamma[8], beta[8];
  const bool affine = a.gamma && !part && all > 0;        // (a worker without rows: zeros, also where beta is infinite)
  if (affine) {
    fa_load8_param(a.gamma, a.param_bf16, i, valid, gamma);
    fa_load8_param(a.beta, a.param_bf16, i, valid, beta);
  }
#pragma unroll
  for (int m = 0; m < FM; ++m) {
    const int o_block = wm + 32 * (m < HM ? m + turn : m - turn);
    wave_fence();
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        block[((r & 3) + 8 * (r >> 2) + 4 * (lane >> 5)) * PITCH + 32 * n + (lane & 31)] = acc[m][n][r];
    wave_fence();
#pragma unroll
    for (int row = 0; row < 32; row += ROWS) {
      const int in = row + lane / LANES, o = o0 + o_block + in;
      float v[8];
      fa_load8_whole(block + in * PITCH + lane % LANES * 8, v);
      if (o < a.outputs) {
        const int64_t to = (int64_t)o * a.features + i;
        if (affine) {
          const float b = bias[o_block + in];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = gamma[e] * v[e] + beta[e] * b;
        }
        if (part) fa_store8(part + to, valid, v);
        else if (a.grad_bf16) fa_store8(static_cast<fa_bf16*>(a.dweight) + w * a.lddweight + to, valid, v);
        else fa_store8(static_cast<float*>(a.dweight) + w * a.lddweight + to, valid, v);
      }
    }
  }
}

// n values `apart` from each other added up in their order, eight at a time on their way
__device__ __forceinline__ float add_up(const float* p, int64_t apart, int n) {
  float s = 0.f;
  for (int q = 0; q < n; q += 8) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = q + e < n ? p[(q + e) * apart] : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[e];
  }
  return s;
}

// The splits of a worker's rows added up in their order, then as above.  Bound by memory (its parts are read once); eight
// loads a thread in flight.
__global__ __launch_bounds__(kThreads) void fa_linear_grad_join_kernel(fa_linear_grad_args a) {
  const int64_t OI = (int64_t)a.outputs * a.features, all = OI + a.outputs;
  const int w = blockIdx.y;
  const float* part = a.partials + (int64_t)w * a.splits * all;
  const bool affine = a.gamma && a.blocks.row0[w + 1] > a.blocks.row0[w];
  for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < all; k += (int64_t)gridDim.x * kThreads) {
    float s = add_up(part + k, all, a.splits);
    if (k >= OI) {
      if (!a.dbias) continue;
      const int64_t at = w * a.lddbias + (k - OI);
      if (a.grad_bf16) fa_store1(static_cast<fa_bf16*>(a.dbias) + at, s);
      else fa_store1(static_cast<float*>(a.dbias) + at, s);
      continue;
    }
    if (affine) {
      const int64_t o = k / a.features;
      const int i = (int)(k - o * a.features);
      const float b = add_up(part + OI + o, all, a.splits);
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

fa_linear_plan plan_of(const fa_row_blocks& b, int features, int outputs, int dtype) {
  return fa_plan_linear_grad(b.row0[b.p], b.p, features, outputs, dtype == FA_BF16);
}

}  // namespace

size_t fa_linear_grad_partials(const fa_row_blocks& b, int features, int outputs, int dtype) {
  const int splits = plan_of(b, features, outputs, dtype).splits;
  return splits > 1 ? sizeof(float) * (size_t)b.p * splits * ((size_t)outputs * features + outputs) : 0;
}

hipError_t fa_launch_linear_grad(fa_linear_grad_args a, int dtype, hipStream_t st) {
  const fa_linear_plan c = plan_of(a.blocks, a.features, a.outputs, dtype);
  a.splits = c.splits;
  const dim3 grid((unsigned)(c.tiles * a.blocks.p * c.splits));
  if (dtype == FA_F32) {
    if (c.wide) hipLaunchKernelGGL((fa_linear_grad_kernel<float, 128, 256, 64>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((fa_linear_grad_kernel<float, 64, 128, 64>), grid, dim3(kThreads), 0, st, a);
  } else {
    if (c.wide) hipLaunchKernelGGL((fa_linear_grad_kernel<fa_bf16, 256, 256, 64>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((fa_linear_grad_kernel<fa_bf16, 128, 128, 64>), grid, dim3(kThreads), 0, st, a);
  }
  if (a.splits > 1) {
    int64_t blocks = ((int64_t)a.outputs * a.features + a.outputs + kThreads - 1) / kThreads;
    if (blocks > 2048) blocks = 2048;
    hipLaunchKernelGGL(fa_linear_grad_join_kernel, dim3((unsigned)blocks, (unsigned)a.blocks.p), dim3(kThreads), 0, st, a);
  }
  return hipGetLastError();
}
