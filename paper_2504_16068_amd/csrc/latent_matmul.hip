// MI355X (gfx950) kernels and C ABI of the products per type over ragged groups
// of rows (include/allegro_latent.h): forward, both gradients, and 8-bit operands.
//
//   product_kernel            Y[r] = act(X[r]) W[g], or with W transposed dX[r] =
//                             (dY[r] W[g]^T) act'(X[r]): 128 rows of one group by TN columns
//   product_stream_kernel     the same in fp32 for many rows: past weights kept in LDS
//   weight_kernel             dW[g] = act(X)^T dY over a range of a group's rows
//   weight_sum_kernel         sums the ranges of the groups that have several, in order
//   product_f8_kernel         the 8-bit product in tiles
//   product_f8_stream_kernel  the 8-bit product past weights kept in LDS
//
// Measured: one launch alone, under a kernel trace; the smallest and the median of 30
// where there are two figures.
//
// Ragged groups.  The offsets are on the device, so the host launches an upper
// bound of tiles, M / rows + G + 1, and a workgroup finds its tile by itself: group
// g's tiles of `rows` rows are numbered from offsets[g] / rows + g on.  Rounding down
// loses less than one tile per group and + g gives one back, so a group's tiles
// never reach the next one's number.  No sums over groups and no launch go before;
// rows without a type are one more group, of zeros.
//
// Operands.  Every tensor is read 16 bytes at a time along its memory rows.  Where
// the contraction runs along them (X and, transposed, W) a tile lies in LDS as it
// is multiplied (Along); where it runs across them (W, and both operands of dW)
// the transposing LDS loads turn it (Across).  The matrix instructions take the
// result's columns as their rows: lane l then holds 4 consecutive columns of row
// l % 16 per 16 x 16 product and stores them straight from registers; with 16-bit
// results two products' columns are interleaved (column_of) to 8 consecutive ones.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device_common.hpp"
#include "latent_common.hpp"

namespace {

using namespace latent;
using allegro_dev::lds_sync;
using allegro_dev::static_for;

constexpr int kThreads = 256;
constexpr int kTileRows = 128;  // rows of a tile

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// SiLU a sigma(a) and its derivative sigma(a) + a sigma(a) (1 - sigma(a)), from the
// hardware's exponential and reciprocal (1 ulp each; the library's correctly
// rounded division costs ten more operations per element).
//
// fp32: exp(-m) = 2^t exp(r) with t = -m log2(e), rounded, and r = -m - t ln 2 what the
// rounding lost, at most 2^-17; exp(r) = 1 + r to 2^-35.  ln 2 itself is rounded, which
// leaves m / 21 units of 2^-24.  With it SiLU is within (7 + |a| / 21) 2^-24 of its value,
// the derivative within (16 + |a| / 21) 2^-24 of its terms' magnitudes.  m is limited so
// that infinities leave r finite; of NaN a itself keeps one.  Measured, product and both
// gradients of 523,599 rows, 128 x 64: 366 us, 359 without r, which is off by 60 units
// at a = -80.
constexpr float kLog2e = 0x1.715476p+0f, kLn2 = 0x1.62e43p-1f;
__device__ __forceinline__ float silu(float a) {
  const float m = __builtin_amdgcn_fmed3f(a, -128.0f, 128.0f);
  const float t = -kLog2e * m, r = __builtin_fmaf(-kLn2, t, -m);
  // exp(-a) is infinite below -88.7, hence the factor 1 + r above 0
  return a * __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_amdgcn_exp2f(t), 1.0f + r, 1.0f));
}
// From e = exp(-|a|): sigma is 1 / (1 + e) or e / (1 + e) by the sign of a and 1 - sigma
// the other one, so nothing is a difference.  e is zero for |a| above 87.3: what is lost
// for negative a is below 2^-119.
__device__ __forceinline__ float silu_grad(float a) {
  const float m = fminf(fabsf(a), 128.0f);
  const float t = -kLog2e * m, r = __builtin_fmaf(-kLn2, t, -m);
  const float e0 = __builtin_amdgcn_exp2f(t), e = __builtin_fmaf(e0, r, e0);
  const float d = __builtin_amdgcn_rcpf(1.0f + e), ed = e * d;
  return __builtin_fmaf(a, ed * d, a < 0.0f ? ed : d);
}
// bf16 operands and results (half a unit is 2^-9) take the shorter form, off by up to
// 2^-20 of the value at a = -20 and 2^-18 at -80: the exponent's rounding.
__device__ __forceinline__ float sigmoid_bf16(float a) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * a));
}
__device__ __forceinline__ float silu_bf16(float a) { return a * sigmoid_bf16(a); }
__device__ __forceinline__ float silu_grad_bf16(float a) {
  const float s = sigmoid_bf16(a);
  return s * (1.0f + a * (1.0f - s));
}

// ------------------------------------------------------ group of a tile
struct Tile {
  int g;                   // group, G for the rows without a type
  int64_t begin, m0, end;  // list positions: the group, the tile's first row; nothing to do if m0 >= end
};

__device__ __forceinline__ Tile find_tile(const int64_t *__restrict__ offsets, int G, int64_t M, uint32_t rows,
                                          int64_t t, int lane) {
  auto clamped = [&](int i) {
    const int64_t o = offsets[i];
    return o < 0 ? int64_t(0) : o > M ? M : o;
  };
  int below = 0;
  for (int i = lane; i <= G; i += kWave) below += uint32_t(clamped(i)) / rows + int64_t(i) <= t;
  for (int m = kWave / 2; m; m >>= 1) below += __shfl_xor(below, m);
  const int g = __builtin_amdgcn_readfirstlane(below > 0 ? below - 1 : 0);
  const int64_t begin = clamped(g), end = g < G ? clamped(g + 1) : M;
  const int64_t k = t - (uint32_t(begin) / rows + int64_t(g));
  return {g, begin, k < 0 ? end : begin + k * rows, end};
}

// The group at `unit` of a line on which group g starts at offsets[g] + cost * g.
__device__ __forceinline__ Tile find_group(const int64_t *__restrict__ offsets, int G, int64_t M, int64_t unit,
                                           int64_t cost, int lane) {
  auto clamped = [&](int i) {
    const int64_t o = offsets[i];
    return o < 0 ? int64_t(0) : o > M ? M : o;
  };
  int below = 0;
  for (int i = lane; i <= G; i += kWave) below += clamped(i) + cost * i <= unit;
  for (int m = kWave / 2; m; m >>= 1) below += __shfl_xor(below, m);
  const int g = __builtin_amdgcn_readfirstlane(below > 0 ? below - 1 : 0);
  const int64_t begin = clamped(g), end = g < G ? clamped(g + 1) : M;
  return {g, begin, begin, end > begin ? end : begin};
}

__host__ __device__ inline int64_t tile_bound(int64_t M, int G, int rows) { return M / rows + G + 1; }

// Workgroups go round the 8 XCDs: give each XCD consecutive tiles, so that the
// tiles that share rows or weights share an L2.
__device__ __forceinline__ int64_t xcd_order(int64_t b, int64_t n) {
  const int64_t per = n >> 3, rest = n & 7, x = b & 7, i = b >> 3;
  return x * per + (x < rest ? x : rest) + i;
}

// --------------------------------------------------- operands in LDS
// fp32 operands are split into three bf16 parts each, x = h + m + l (8 bits of
// the significand in each, all exact), and of the nine products of the parts the
// six with h, and m m, are summed; the dropped ones are below 2^-24 of the product
// (|m| is at most 2^-8 of x and |l| 2^-17).  kScale keeps the parts of small values
// above bf16's subnormals, which hold fewer bits.  The matrix instructions round
// their sums down, hence every step's sum starts from zero and is added to the
// running one by the vector units, and every other row (or step) enters negated,
// so that what is left of the bias cancels over rows.  A sum that
// is not finite (infinities, NaN, values beyond the scale) is formed again with
// the fp32 matrix instructions.
constexpr float kScale = 0x1p24f, kUnscale = 0x1p-48f;

template <class T>
struct Kind;
template <>
struct Kind<float> {
  static constexpr int P = 3, KS = 32, PE = 4;  // planes, contraction step, elements of 16 bytes
};
template <>
struct Kind<uint16_t> {
  static constexpr int P = 1, KS = 64, PE = 8;
};

// Result column of row i of the matrix instructions' 16 x 16 product j: with 16-bit
// results (WIDE) two products share 32 columns so that lane l, which gets rows
// 4 (l / 16) .. + 3 of each, holds 8 consecutive columns of the two.
template <bool WIDE>
__device__ __forceinline__ int column_of(int j, int i) {
  return WIDE ? 32 * (j / 2) + 8 * (i / 4) + 4 * (j % 2) + i % 4 : 16 * j + i;
}

__device__ __forceinline__ void split2(float a, float b, uint32_t &h, uint32_t &m, uint32_t &l) {
  h = bf16_pair(a, b);
  const float ra = a - __builtin_bit_cast(float, h << 16), rb = b - __builtin_bit_cast(float, h & 0xffff0000u);
  m = bf16_pair(ra, rb);
  l = bf16_pair(ra - __builtin_bit_cast(float, m << 16), rb - __builtin_bit_cast(float, m & 0xffff0000u));
}

// One 16-byte piece of fp32 values, through SiLU or not, as the three planes' parts.
__device__ __forceinline__ void split_piece(u32x4 v, bool act, float scale, u32x2 (&o)[3]) {
  float x[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t bits = v[e];  // a bit cast of the vector's element itself gives element 0
    x[e] = __builtin_bit_cast(float, bits);
  }
  if (act) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = silu(x[e]);
  }
  uint32_t h[2], m[2], l[2];
  split2(scale * x[0], scale * x[1], h[0], m[0], l[0]);
  split2(scale * x[2], scale * x[3], h[1], m[1], l[1]);
  o[0] = u32x2{h[0], h[1]};
  o[1] = u32x2{m[0], m[1]};
  o[2] = u32x2{l[0], l[1]};
}
// The same of bf16 values.  SiLU is rounded to bf16 again, the type that the matrix
// instructions take: with K = 1024 the product is then off by 2.4e-3 of the 64-bit one
// (2-norm), by 1.7e-3 without, which is the output's rounding; two parts would
// double the products.
__device__ __forceinline__ u32x4 act_piece(u32x4 v, bool act) {
  if (act) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      v[e] = bf16_pair(silu_bf16(__builtin_bit_cast(float, v[e] << 16)),
                       silu_bf16(__builtin_bit_cast(float, v[e] & 0xffff0000u)));
  }
  return v;
}

// Pieces of the elements k .. of rows of n (k below n or not), row(i) pointing to
// row i's first one.  The loads are issued without a condition: where a piece
// crosses the row's end the row's last PE elements are loaded, and shifted down
// by shift_of when they are used.  SHORT: rows may have fewer than PE.
template <class T, bool SHORT, int NP, class Row>
__device__ __forceinline__ void load_pieces(u32x4 (&v)[NP], Row row, int k, int n) {
  constexpr int PE = Kind<T>::PE;
  if (!SHORT || n >= PE) {
    const unsigned at = unsigned(k < n - PE ? k : n - PE);
#pragma unroll
    for (int i = 0; i < NP; ++i) v[i] = *reinterpret_cast<const u32x4_any *>(row(i) + at);
    return;
  }
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    v[i] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < PE - 1; ++e)
      if (k == 0 && e < n) {
        if constexpr (sizeof(T) == 4)
          v[i][e] = __builtin_bit_cast(uint32_t, row(i)[e]);
        else
          v[i][e / 2] |= uint32_t(row(i)[e]) << (16 * (e % 2));
      }
  }
}
template <class T>
__device__ __forceinline__ int shift_of(int k, int n) {
  constexpr int PE = Kind<T>::PE;
  return n < PE || k < n - PE ? 0 : k - (n - PE);
}
// Drops the first `by` elements; zeros follow the last.
template <class T>
__device__ __forceinline__ u32x4 shifted(u32x4 a, int by) {
  if constexpr (sizeof(T) == 2) {
    if (by & 1) a = u32x4{a[0] >> 16 | a[1] << 16, a[1] >> 16 | a[2] << 16, a[2] >> 16 | a[3] << 16, a[3] >> 16};
  }
  constexpr int E = 4 / int(sizeof(T));
  if (by & E) a = u32x4{a[1], a[2], a[3], 0};
  if (by & (2 * E)) a = u32x4{a[2], a[3], 0, 0};
  if (by >= Kind<T>::PE) a = u32x4{0, 0, 0, 0};
  return a;
}

// 16-byte chunk c of row r of rows of 4 or 8 chunks (64 or 128 bytes).  One chunk
// of the rows that 8 or 16 consecutive lanes read lies in distinct banks: of
// consecutive rows, or (WIDE) of those that column_of<true> picks.
template <int C, bool WIDE>
__device__ __forceinline__ int swizzled(int r, int c) {
  const int f = C == 4 ? ((r >> 1) & 3) ^ ((r >> 3) & 1)
                : WIDE ? ((r & 3) | (r >> 1 & 4)) ^ ((r >> 4) & 1)
                       : (r & 7) ^ ((r >> 3) & 1);
  return r * C + (c ^ f);
}

// A tile of `ROWS` rows (of X, or columns of the result) whose contraction runs
// along memory.  In LDS: rows of KS 16-bit values, in 16-byte chunks swizzled by
// row so that 8 and 16 lanes reading one chunk of consecutive rows hit distinct
// banks.  NT threads move pieces tid % 8 of rows tid / 8 + RP i.  SHORT as in
// load_pieces: without it every row must have PE elements.
template <class T, int ROWS, bool WIDE, int NT, bool SHORT>
struct Along {
  static constexpr int P = Kind<T>::P, KS = Kind<T>::KS, PE = Kind<T>::PE, RP = NT / 8, NP = ROWS / RP, C = KS / 8;
  static constexpr int SIZE = P * ROWS * C;  // 16-byte units
  u32x4 v[NP];
  static __device__ __forceinline__ int row(int i, int tid) { return tid / 8 + RP * i; }
  // row(i): pointer to the first element of row row(i, tid); n elements to a row
  template <class Row>
  __device__ __forceinline__ void load(Row row, int k0, int n, int tid) {
    load_pieces<T, SHORT>(v, row, k0 + PE * (tid % 8), n);
  }
  __device__ __forceinline__ void put(u32x4 *lds, bool act, float scale, int k0, int n, int tid) {
    if (k0 + KS > n) {  // the last step: nothing from n on
#pragma unroll
      for (int i = 0; i < NP; ++i) v[i] = shifted<T>(v[i], shift_of<T>(k0 + PE * (tid % 8), n));
    }
    // rows RP apart are swizzled alike
    const int at =
        P == 3 ? 2 * swizzled<C, WIDE>(tid / 8, tid % 8 / 2) + tid % 2 : swizzled<C, WIDE>(tid / 8, tid % 8);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if constexpr (P == 3) {
        u32x2 o[3];
        split_piece(v[i], act, scale, o);
#pragma unroll
        for (int p = 0; p < 3; ++p) reinterpret_cast<u32x2 *>(lds)[at + 2 * C * (p * ROWS + RP * i)] = o[p];
      } else {
        lds[at + C * RP * i] = act_piece(v[i], act);
      }
    }
  }
  // Operands of a wave from product j0 on (a whole number of 32 columns if WIDE):
  // lane l has row l % 16 of product j0 + j and k = 32 kk + 8 (l / 16) ...  The
  // lane's part of the address is the same for all j up to the product's parity,
  // and kk flips one of its bits.
  struct Reader {
    int base[WIDE ? 2 : 1];
    __device__ __forceinline__ Reader(int j0, int l) {
#pragma unroll
      for (int h = 0; h < (WIDE ? 2 : 1); ++h) base[h] = swizzled<C, WIDE>(column_of<WIDE>(j0 + h, l % 16), l / 16);
    }
    __device__ __forceinline__ bf16x8 get(const u32x4 *lds, int p, int j, int kk) const {
      const int row = p * ROWS + (WIDE ? 32 * (j / 2) : 16 * j);
      return __builtin_bit_cast(bf16x8, lds[(base[WIDE ? j % 2 : 0] ^ (4 * kk)) + C * row]);
    }
  };
};

// A tile of COLS columns whose contraction runs across memory rows.  In LDS: KS
// rows of COLS 16-bit values as they come; operands are read with the transposing
// LDS load, by which 16 lanes turn 4 rows of 16 columns into 4 rows of one column
// each.  A wave's load touches 4 columns' quads of 16 rows; chunks (and their
// halves) are swizzled by row so that those 512 bytes lie in all banks twice.
template <class T, int COLS, bool WIDE, int NT, bool SHORT>
struct Across {
  static constexpr int P = Kind<T>::P, KS = Kind<T>::KS, PE = Kind<T>::PE;
  static constexpr int PR = COLS / PE, RP = NT / PR, NP = KS / RP;  // pieces to a row, rows to a pass
  static constexpr int SIZE = P * KS * COLS / 8;                          // 16-byte units
  u32x4 v[NP];
  static __device__ __forceinline__ int quad_at(int k, int c4) {  // in 8-byte units
    const int f = COLS >= 128 ? (k & 3) << 2 | ((k >> 3) & 1) << 1 : ((k >> 1) & 1) << 2 | ((k >> 3) & 1) << 1;
    return k * (COLS / 4) + ((((c4 >> 1) ^ f) << 1) | ((c4 & 1) ^ ((k >> 3) & 1)));
  }
  static __device__ __forceinline__ int step(int i, int tid) { return tid / PR + i * RP; }
  static __device__ __forceinline__ int col(int tid) { return tid % PR * PE; }
  // row(i): pointer to the first element of the row of step step(i, tid); the tile's
  // columns start at c0 of n
  template <class Row>
  __device__ __forceinline__ void load(Row row, int c0, int n, int tid) {
    load_pieces<T, SHORT>(v, row, c0 + col(tid), n);
  }
  // missing: bit i is set if step(i, tid) does not exist and becomes zero
  __device__ __forceinline__ void put(u32x4 *lds, bool act, float scale, int c0, int n, int missing, int tid) {
    if (n - c0 < COLS) {
#pragma unroll
      for (int i = 0; i < NP; ++i) v[i] = shifted<T>(v[i], shift_of<T>(c0 + col(tid), n));
    }
    if (__any(missing)) {
#pragma unroll
      for (int i = 0; i < NP; ++i) v[i] = missing >> i & 1 ? u32x4{0, 0, 0, 0} : v[i];
    }
    // rows of one pass are RP apart: RP = 8 flips the bits of k / 8, 16 and 32 none
    const int at = quad_at(step(0, tid), tid % PR * (PE / 4));
    const bool swap = P == 1 && (step(0, tid) >> 3 & 1);  // the halves' order in a 16-byte chunk
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int flip = RP == 8 && i % 2 ? 5 : 0, row = i * RP * (COLS / 4);
      if constexpr (P == 3) {
        u32x2 o[3];
        split_piece(v[i], act, scale, o);
#pragma unroll
        for (int p = 0; p < 3; ++p) reinterpret_cast<u32x2 *>(lds)[(at ^ flip) + row + p * KS * (COLS / 4)] = o[p];
      } else {
        const u32x4 a = act_piece(v[i], act);
        lds[(at + row) / 2] = swap ? u32x4{a[2], a[3], a[0], a[1]} : a;
      }
    }
  }
  // Operands of a wave from product j0 on, as Along::Reader.  Columns 4 j flip bits
  // of the lane's address; the swizzle repeats every 4 rows of 8 and every 16.
  struct Reader {
    int base;
    __device__ __forceinline__ Reader(int j0, int l) {
      base = quad_at(8 * (l / 16) + l % 16 / 4, l % 4 * (WIDE ? 2 : 1)) ^ (4 * j0);
    }
    __device__ __forceinline__ bf16x8 get(const u32x4 *lds, int p, int j, int kk) const {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
      const u32x2 *q = reinterpret_cast<const u32x2 *>(lds) + (base ^ (WIDE ? 8 * (j / 2) + j % 2 : 4 * j)) +
                       (p * KS + 32 * kk) * (COLS / 4);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)q);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(q + COLS));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
};

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// One contraction step of a wave: MI x NI products of 16 x 16 of the tiles ML (the
// instructions' columns) and NL (their rows).  fp32 sums are added with the factor
// `sign`.
template <class T, class ML, class NL, bool TIGHT, int MI, int NI>
__device__ __forceinline__ void multiply(const u32x4 *m_lds, const u32x4 *n_lds, const typename ML::Reader &m_read,
                                         const typename NL::Reader &n_read, float sign, f32x4 (&acc)[MI][NI]) {
  constexpr int P = Kind<T>::P;
#pragma unroll
  for (int kk = 0; kk < Kind<T>::KS / 32; ++kk) {
    if constexpr (TIGHT) __builtin_amdgcn_sched_barrier(0);  // operands of one half at a time
    bf16x8 b[MI][P];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int p = 0; p < P; ++p) b[i][p] = m_read.get(m_lds, p, i, kk);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      bf16x8 a[P];
#pragma unroll
      for (int p = 0; p < P; ++p) a[p] = n_read.get(n_lds, p, j, kk);
      if constexpr (P == 1) {
#pragma unroll
        for (int i = 0; i < MI; ++i) acc[i][j] = mfma16(a[0], b[i][0], acc[i][j]);
      } else {
        // the small products first; MI sums at a time hide each other's latency
        constexpr int PA[6] = {2, 0, 1, 1, 0, 0}, PB[6] = {0, 2, 1, 0, 1, 0};
        f32x4 s[MI];
#pragma unroll
        for (int i = 0; i < MI; ++i) s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 6; ++q)
#pragma unroll
          for (int i = 0; i < MI; ++i) s[i] = mfma16(a[PA[q]], b[i][PB[q]], s[i]);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(sign, s[i][e], acc[i][j][e]);
      }
    }
  }
}

template <int MI, int NI>
__device__ __forceinline__ bool any_not_finite(const f32x4 (&acc)[MI][NI]) {
  float bad = 0.f;
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) bad = __builtin_fmaf(acc[i][j][e], 0.f, bad);
  return __any(bad != bad);
}

// The same sums with the fp32 matrix instructions, from memory: m_elem(i, k) and
// n_elem(j, k) are the operands of this lane's row of product (i, j).
template <int MI, int NI, class ME, class NE>
__device__ __forceinline__ void multiply_again(f32x4 (&acc)[MI][NI], int64_t K, int l, ME m_elem, NE n_elem) {
  static_for<0, MI>([&](auto i) {
    static_for<0, NI>([&](auto j) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int64_t k = 0; k < K; k += 4) {
        const int64_t kl = k + l / 16;
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(kl < K ? n_elem(j(), kl) : 0.f, kl < K ? m_elem(i(), kl) : 0.f, s, 0,
                                                 0, 0);
      }
      acc[i()][j()] = s;
    });
  });
}

// Loads or stores the 4 (or, of two products, 8) consecutive values that a lane
// holds of a row; `left` columns exist from the first on.
template <int W>
__device__ __forceinline__ void store_row(float *p, const float *v, int left) {
  if (left >= W) {
    *reinterpret_cast<u32x4_any *>(p) = __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < left) p[i] = v[i];
  }
}
template <int W>
__device__ __forceinline__ void store_row(uint16_t *p, const float *v, int left) {
  if (left >= W) {
    if constexpr (W == 8)
      *reinterpret_cast<u32x4_any *>(p) =
          u32x4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    else
      *reinterpret_cast<u32x2_any *>(p) = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < left) p[i] = bf16_bits(v[i]);
  }
}
__device__ __forceinline__ void store_bits(uint16_t *p, u32x4 v, int left) {
  if (left >= 8) {
    *reinterpret_cast<u32x4_any *>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < left) p[i] = uint16_t(v[i / 2] >> (16 * (i % 2)));
  }
}
template <int W, class T>  // 16 bytes in both types
__device__ __forceinline__ u32x4 load_bits(const T *p, int left) {
  if (left >= W) return *reinterpret_cast<const u32x4_any *>(p);
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < W - 1; ++i)
    if (i < left) {
      if constexpr (sizeof(T) == 4)
        v[i] = __builtin_bit_cast(uint32_t, p[i]);
      else
        v[i / 2] |= uint32_t(p[i]) << (16 * (i % 2));
    }
  return v;
}
template <class T>
__device__ __forceinline__ float value_of(u32x4 v, int e) {
  if constexpr (sizeof(T) == 4) {
    const uint32_t bits = v[e];
    return __builtin_bit_cast(float, bits);
  } else {
    const uint32_t bits = e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16;
    return __builtin_bit_cast(float, bits);
  }
}

// Lanes 4 a + b (b < 4) hold, in v[0 .. 3], 16 bytes of each of four columns' parts
// of a row of their own; afterwards lane b holds part b of the four rows, v[s]
// that of lane 4 a + s.
__device__ __forceinline__ void quad_transpose(u32x4 (&v)[4], int l) {
  auto swap = [&](u32x4 &lo, u32x4 &hi, auto perm, bool upper) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t a = lo[e], b = hi[e];
      const uint32_t got = uint32_t(__builtin_amdgcn_mov_dpp(int(upper ? a : b), perm(), 0xf, 0xf, true));
      lo[e] = upper ? got : a;
      hi[e] = upper ? b : got;
    }
  };
  const std::integral_constant<int, 0xb1> by1;  // lanes 1, 0, 3, 2 of every four
  const std::integral_constant<int, 0x4e> by2;  // lanes 2, 3, 0, 1
  swap(v[0], v[1], by1, l & 1);
  swap(v[2], v[3], by1, l & 1);
  swap(v[0], v[2], by2, l & 2);
  swap(v[1], v[3], by2, l & 2);
}

// Row list of a tile: srow[i] = row of list position m0 + i, -1 past the end or
// out of range.
__device__ __forceinline__ void list_rows(int *srow, const int32_t *rows, const Tile &t, int64_t M, int tid) {
  if (tid < kTileRows) {
    int64_t r = -1;
    if (t.m0 + tid < t.end) {
      r = rows ? int64_t(rows[t.m0 + tid]) : t.m0 + tid;
      if (r < 0 || r >= M) r = -1;
    }
    srow[tid] = int(r);
  }
}

// Zeros for the rows of a tile, columns n0 .. n0 + n - 1.
template <class T>
__device__ __forceinline__ void zero_rows(const int *srow, T *y, int64_t ldy, int n0, int n, int tid) {
  for (int i = tid; i < kTileRows * n; i += int(blockDim.x)) {
    const int r = srow[i / n];
    if (r >= 0) y[int64_t(r) * ldy + n0 + i % n] = T(0);
  }
}

// -------------------------------------------------------------- products
struct ProductArgs {
  int64_t M;
  int K, N, G;  // contraction and columns of the result
  const int64_t *offsets;
  const int32_t *rows;
  const void *x;  // [M][K]
  int64_t ldx;
  const void *w;  // [G][K][N], transposed [G][N][K]
  void *y;        // [M][N]
  int64_t ldy;
  const void *pre;  // transposed: y is multiplied with SiLU'(pre), if given ([M][N])
  int64_t ldp;
  int act;     // SiLU on x (not transposed)
  int nt;      // column tiles
  int64_t mt;  // upper bound of the row tiles
  int64_t first;  // the launch's first tile
};

// Threads of a tile TN columns wide: four waves, eight of a wide one.
constexpr int tile_threads(int TN) { return TN == 256 ? 2 * kThreads : kThreads; }
// Whether K or N may be less than a 16-byte piece: tiles of 256 columns are launched
// with K > 64 and N > 128 only.
constexpr bool tile_short(int TN) { return TN != 256; }

// A contraction step is loaded into registers, put into LDS as operands and
// multiplied.  BUFS == 1: one step in LDS and two meetings of the waves a step;
// several workgroups on a compute unit overlap each other's phases.  BUFS == 2, for
// grids with a tile or two to a compute unit: eight waves and two steps in LDS, so
// that the waves meet once a step and half of them put the next one while the others
// multiply.
//
// Measured (bf16, 100,003 rows of 100 types, K = 1024, N = 512 with SiLU, 105 GFLOP): forward
// 176 to 186 us, 564 TFLOP/s, and the gradient of X 220 to 227 us.  A wave's 64 x 64 of the result reads
// 16 KB from LDS a step for 32 matrix instructions: of eight waves as many cycles (1,024)
// as the instructions take, and with one buffer the step's stores come on top.  And of the
// gradient, contracting 2048 instead of 512 columns runs at 855 TFLOP/s: 8 steps are too
// few to hide a tile's start and its epilogue (512 MB of dY, X and dX, 107 us at the copy
// rate).  The forward computes each SiLU twice (two tiles of 256 columns).  Few tiles are bound by
// the latency of a step: 1.2 us in fp32 (load, split, store to LDS, meet, read,
// multiply), 1.6 us with one buffer and four waves.
template <class T, int TN, bool WT, int BUFS>
__global__ __launch_bounds__(BUFS == 2 ? 512 : tile_threads(TN), TN == 256 && BUFS == 1 ? 4 : 2) void product_kernel(
    ProductArgs g) {
  constexpr int KS = Kind<T>::KS;
  constexpr bool F32 = sizeof(T) == 4;
  // waves along the tile's rows; products of a wave
  constexpr int NT = BUFS == 2 ? 512 : tile_threads(TN), WM = NT == 512 && TN == 64 ? 4 : 2;
  constexpr int MI = 8 / WM, NI = TN / 16 / (NT / kWave / WM);
  constexpr bool TIGHT = TN == 256 && BUFS == 1;  // 128 registers, for two workgroups of eight waves
  using XTile = Along<T, kTileRows, false, NT, tile_short(TN)>;
  using WTile = std::conditional_t<WT, Along<T, TN, !F32, NT, tile_short(TN)>,
                                   Across<T, TN, !F32, NT, tile_short(TN)>>;
  __shared__ u32x4 x_lds[BUFS * XTile::SIZE], w_lds[BUFS * WTile::SIZE];
  __shared__ int srow[kTileRows];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), l = tid % kWave;
  const int64_t b = g.first + xcd_order(blockIdx.x, gridDim.x);
  const Tile t = find_tile(g.offsets, g.G, g.M, kTileRows, b / g.nt, l);
  if (t.m0 >= t.end) return;
  const int n0 = int(b % g.nt) * TN, K = g.K, N = g.N;
  T *y = static_cast<T *>(g.y);
  list_rows(srow, g.rows, t, g.M, tid);
  __syncthreads();
  if (t.g == g.G) {
    zero_rows(srow, y, g.ldy, n0, N - n0 < TN ? N - n0 : TN, tid);
    return;
  }
  const T *x = static_cast<const T *>(g.x), *w = static_cast<const T *>(g.w) + int64_t(t.g) * K * N;
  int xr[XTile::NP];
#pragma unroll
  for (int i = 0; i < XTile::NP; ++i) {
    const int r = srow[XTile::row(i, tid)];
    xr[i] = r < 0 ? 0 : r;  // rows past the end are multiplied but not stored
  }
  XTile a;
  WTile bw;
  auto load = [&](int k0) {
    int t = tid;
    if constexpr (TIGHT) asm volatile("" : "+v"(t));  // addresses are formed anew
    a.load([&](int i) { return x + int64_t(xr[i]) * g.ldx; }, k0, K, t);
    if constexpr (WT) {
      bw.load(
          [&](int i) {
            const int n = WTile::row(i, t);  // columns past the last read it, and reach no output
            return w + int64_t(n0) * K + (n < N - n0 ? n : N - n0 - 1) * K;
          },
          k0, K, t);
    } else {
      bw.load(
          [&](int i) {
            const int k = WTile::step(i, t), left = K - k0;
            return w + int64_t(k0) * N + (k < left ? k : left - 1) * N;
          },
          n0, N, t);
    }
  };
  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int wm = 16 * MI * (wave % WM), wn = 16 * NI * (wave / WM);
  const typename XTile::Reader x_read(wm / 16, l);
  const typename WTile::Reader w_read(wn / 16, l);
  const float xs = (tid / 8) % 2 ? -kScale : kScale;  // odd rows negated
  auto put = [&](int buf, int k0) {
    a.put(x_lds + buf * XTile::SIZE, !WT && g.act, xs, k0, K, tid);
    u32x4 *w_at = w_lds + buf * WTile::SIZE;
    if constexpr (WT) {
      bw.put(w_at, false, kScale, k0, K, tid);
    } else {
      int missing = 0;
      if (k0 + KS > K) {
#pragma unroll
        for (int i = 0; i < WTile::NP; ++i) missing |= (k0 + WTile::step(i, tid) >= K) << i;
      }
      bw.put(w_at, false, kScale, n0, N, missing, tid);
    }
  };
  load(0);
  if constexpr (BUFS == 1) {
    for (int k0 = 0; k0 < K; k0 += KS) {
      lds_sync<NT / kWave>();  // the previous step has been read
      put(0, k0);
      lds_sync<NT / kWave>();
      if (k0 + KS < K) load(k0 + KS);
      multiply<T, XTile, WTile, TIGHT>(x_lds, w_lds, x_read, w_read, 1.f, acc);
    }
  } else {
    put(0, 0);
    if (KS < K) load(KS);
    for (int k0 = 0, buf = 0; k0 < K; k0 += KS, buf ^= 1) {
      lds_sync<NT / kWave>();  // this step is in LDS, and the one before has been read
      auto next = [&] {
        if (k0 + KS < K) put(buf ^ 1, k0 + KS);
        if (k0 + 2 * KS < K) load(k0 + 2 * KS);
      };
      if (wave < NT / kWave / 2) next();
      multiply<T, XTile, WTile, TIGHT>(x_lds + buf * XTile::SIZE, w_lds + buf * WTile::SIZE, x_read, w_read, 1.f, acc);
      if (wave >= NT / kWave / 2) next();
    }
  }
  if constexpr (F32) {
    if (any_not_finite(acc)) {
      multiply_again(
          acc, K, l,
          [&](int i, int64_t k) {
            const int r = srow[wm + 16 * i + l % 16];
            const float v = r < 0 ? 0.f : x[int64_t(r) * g.ldx + k];
            return g.act ? silu(v) : v;
          },
          [&](int j, int64_t k) {
            const int n = n0 + wn + 16 * j + l % 16;  // fp32: columns in order
            return n >= N ? 0.f : WT ? w[int64_t(n) * K + k] : w[k * N + n];
          });
    } else {
      const float u = l % 2 ? -kUnscale : kUnscale;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] *= u;
    }
  }
  // lane l: row l % 16 of each row product
  constexpr int W = F32 ? 4 : 8, JW = W / 4;
  const T *pre = static_cast<const T *>(g.pre);
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = srow[wm + 16 * i + l % 16];
    if (r < 0) continue;
#pragma unroll
    for (int j = 0; j < NI; j += JW) {
      const int n = n0 + wn + 16 * j + W * (l / 16);
      float v[W];
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] = acc[i][j + e / 4][e % 4];
      if (WT && pre) {
        const u32x4 p = load_bits<W>(pre + int64_t(r) * g.ldp + n, N - n);
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] *= F32 ? silu_grad(value_of<T>(p, e)) : silu_grad_bf16(value_of<T>(p, e));
      }
      store_row<W>(y + int64_t(r) * g.ldy + n, v, N - n);
    }
  }
}

// The fp32 products where the weights of a group fit the LDS and there are many
// rows: a workgroup of 8 waves holds the split form of one group's W (TN columns)
// and streams rows past it.  X goes from memory straight to the matrix
// instructions' operand registers (lane l has row l % 16 and 8 consecutive values
// from 8 (l / 16) on), so each value is read and split once, and waves meet at no
// barrier but when the group changes.  A wave goes through (32 rows, step) pairs
// with loads two steps ahead, also from one 32 rows to the next.
//
// Measured: 1,048,820 rows of 16 types, K = 192, N = 128 350 us (1.34 GB, 3.8 TB/s; the six
// bf16 products of each fp32 one at 0.88 PFLOP/s, close to the rate of a large library
// product); 523,599 rows, K = 128, N = 64 with SiLU 97 to 113 us (402 MB, 4.1 TB/s) and its
// gradient of X 146 to 158 us (0.67 GB, 4.6 TB/s), both bound by memory.  In tiles the first took 411 us.
constexpr int kStreamThreads = 512, kStreamWaves = kStreamThreads / kWave, kStreamLds = 147456;
constexpr int kStreamGroups = 256;  // workgroups: one on every compute unit

template <int TN>
constexpr int stream_k() {  // the longest contraction whose weights fit: whole pairs of steps
  return kStreamLds / (Kind<float>::P * TN * 128) * 64;
}

// Goes through share `share` of `shares` of equal cost: a group costs its rows and
// what it takes to load its weights and to fill the waves, as much as RB rows for
// each wave.  Calls group(g, chunks, list) for its part of each group, g == G for
// the rows without a type; list(c) gives lane i row i of the RB rows of chunk c, -1
// past the end or out of range.  Every wave of the workgroup makes the same calls.
template <int RB, class Group>
__device__ __forceinline__ void stream_share(const int64_t *__restrict__ offsets, const int32_t *__restrict__ rows, int G,
                                             int64_t M, int64_t share, int64_t shares, int l, Group group) {
  // cost units of group g lie at its rows from offsets[g] + kGroupRows (g + 1) on
  constexpr int64_t kGroupRows = kStreamWaves * RB;
  const int64_t units = M + kGroupRows * (G + 1), stop = units * (share + 1) / shares;
  for (int64_t unit = units * share / shares; unit < stop;) {
    int lg = l;
    asm volatile("" : "+v"(lg));  // addresses of a group are formed in its turn
    const Tile t = offsets ? find_group(offsets, G, M, unit, kGroupRows, lg) : Tile{0, 0, 0, M};
    const int64_t first = t.begin + kGroupRows * (t.g + 1);  // the unit of the group's first row
    const int64_t lo = t.begin + (unit > first ? unit - first : 0);
    const int64_t hi = t.end < t.begin + stop - first ? t.end : t.begin + stop - first;
    const int64_t next_group = first + (t.end - t.begin);
    if (next_group <= unit) break;  // offsets out of order, or no more groups
    unit = next_group;
    if (lo >= hi) continue;
    group(t.g, int((hi - lo + RB - 1) / RB), [=](int c) -> int {
      const int64_t at = lo + int64_t(c) * RB + lg % RB, in = at < hi ? at : hi - 1;
      const int r = rows ? rows[in] : int(in);
      return at < hi && r >= 0 && r < M ? r : -1;
    });
  }
}

// Zeros for columns n0 .. n1 - 1 of the wave's share of the rows without a type.
template <int RB, class T, class List>
__device__ __forceinline__ void stream_zeros(int chunks, List list, T *y, int64_t ldy, int n0, int n1, int wave, int l) {
  for (int c = wave; c < chunks; c += kStreamWaves) {
    const int rows = list(c);
    for (int i = 0; i < RB; ++i) {
      const int r = __builtin_amdgcn_readlane(rows, i);
      if (r < 0) continue;
      for (int n = n0 + l; n < n1; n += kWave) y[int64_t(r) * ldy + n] = T(0);
    }
  }
}

template <int TN, bool WT>
__global__ __launch_bounds__(kStreamThreads, 2) void product_stream_kernel(ProductArgs g) {
  constexpr int KS = Kind<float>::KS, PE = Kind<float>::PE, XP = 8 / PE, MT = 2, NI = TN / 16, RB = 16 * MT;
  using WTile = std::conditional_t<WT, Along<float, TN, false, kThreads, true>, Across<float, TN, false, kThreads, true>>;
  __shared__ u32x4 w_lds[kStreamLds / 16];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), l = tid % kWave;
  const int64_t b = xcd_order(blockIdx.x, g.mt * g.nt);
  const int n0 = int(b % g.nt) * TN, K = g.K, N = g.N, steps = (K + 2 * KS - 1) / (2 * KS) * 2;  // an even number
  const float *x = static_cast<const float *>(g.x);
  float *y = static_cast<float *>(g.y);
  const float *pre = static_cast<const float *>(g.pre);
  const float xs = l % 2 ? -kScale : kScale;  // odd rows negated
  const typename WTile::Reader w_read(0, l);
  stream_share<RB>(g.offsets, g.rows, g.G, g.M, b / g.nt, g.mt, l, [&](int group, int chunks, auto list) {
    if (group == g.G) {
      stream_zeros<RB>(chunks, list, y, g.ldy, n0, n0 + TN < N ? n0 + TN : N, wave, l);
      return;
    }
    auto row_of = [&](int rows, int i) { return __shfl(rows, 16 * i + l % 16); };
    int lg = l;
    asm volatile("" : "+v"(lg));
    const float *w = static_cast<const float *>(g.w) + int64_t(group) * K * N;
    __syncthreads();  // the group before has been multiplied
    // each half of the workgroup fills every other tile
    const int ft = wave % 4 * kWave + lg;
    const int half = tid / kThreads;
    auto fill_load = [&](WTile &f, int tile) {
      const int k0 = tile * KS;
      if constexpr (WT) {
        f.load(
            [&](int i) {
              const int n = ft / 8 + 32 * i;  // columns past the last read it, and reach no output
              return w + int64_t(n0) * K + (n < N - n0 ? n : N - n0 - 1) * K;
            },
            k0, K, ft);
      } else {
        f.load(
            [&](int i) {
              const int k = WTile::step(i, ft), left = K - k0;
              return w + int64_t(k0) * N + (k < left ? k : left - 1) * N;
            },
            n0, N, ft);
      }
    };
    auto fill_put = [&](WTile &f, int tile) {
      const int k0 = tile * KS;
      if constexpr (WT) {
        f.put(w_lds + tile * WTile::SIZE, false, kScale, k0, K, ft);
      } else {
        int missing = 0;
#pragma unroll
        for (int i = 0; i < WTile::NP; ++i) missing |= (k0 + WTile::step(i, ft) >= K) << i;
        f.put(w_lds + tile * WTile::SIZE, false, kScale, n0, N, missing, ft);
      }
    };
#pragma unroll 1
    for (int tile = half; tile < steps; tile += 2) {
      WTile f;
      fill_load(f, tile);
      fill_put(f, tile);
    }
    __syncthreads();
    if (wave < chunks) {
      // the loads' side: chunk lc, step lk; next: the rows of the chunk after lc
      int lc = wave, lk = 0, next = list(lc);
      const float *xp[MT];
      auto point = [&]() {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const int r = row_of(next, i);
          xp[i] = x + (r < 0 ? 0 : int64_t(r) * g.ldx);
        }
        next = list(lc + kStreamWaves);
      };
      point();
      auto load = [&](u32x4 (&v)[MT][XP]) {
        const int k = lk * 32 + 8 * (l / 16);
#pragma unroll
        for (int q = 0; q < XP; ++q) {
          const unsigned at = unsigned(k + PE * q < K - PE ? k + PE * q : K - PE);
#pragma unroll
          for (int i = 0; i < MT; ++i) v[i][q] = *reinterpret_cast<const u32x4_any *>(xp[i] + at);
        }
        if (++lk == steps) {
          lk = 0;
          lc += kStreamWaves;
          point();
        }
      };
      f32x4 acc[MT][NI];
      auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      };
      clear();
      int cc = wave, ck = 0, rows = list(cc);  // the products' side
      auto step = [&](u32x4 (&v)[MT][XP]) {
        bf16x8 xf[MT][3];
        const int k = ck * 32 + 8 * (l / 16);
        if (ck * 32 + 32 > K) {
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int q = 0; q < XP; ++q) v[i][q] = shifted<float>(v[i][q], shift_of<float>(k + PE * q, K));
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          u32x2 o[2][3];
          split_piece(v[i][0], !WT && g.act, xs, o[0]);
          split_piece(v[i][1], !WT && g.act, xs, o[1]);
#pragma unroll
          for (int p = 0; p < 3; ++p)
            xf[i][p] = __builtin_bit_cast(bf16x8, u32x4{o[0][p][0], o[0][p][1], o[1][p][0], o[1][p][1]});
        }
        load(v);
        const u32x4 *d = w_lds + ck * WTile::SIZE;
        typename WTile::Reader read = w_read;
        if constexpr (!WT) asm volatile("" : "+v"(read.base));  // one register, not one for each j
        auto frag = [&](int p, int j) { return read.get(d, p, j, 0); };
        constexpr int PA[6] = {2, 0, 1, 1, 0, 0}, PB[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          if (j % 2 == 0) __builtin_amdgcn_sched_barrier(0);  // operands of two products at a time
          bf16x8 a[3];
          f32x4 sum[MT];
#pragma unroll
          for (int p = 0; p < 3; ++p) a[p] = frag(p, j);
#pragma unroll
          for (int i = 0; i < MT; ++i) sum[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int q = 0; q < 6; ++q)
#pragma unroll
            for (int i = 0; i < MT; ++i) sum[i] = mfma16(a[PA[q]], xf[i][PB[q]], sum[i]);
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[i][j] += sum[i];
        }
        ++ck;
      };
      // writes the rows of a chunk
      auto finish = [&]() {
        int lane = l;
        asm volatile("" : "+v"(lane));  // keeps the addresses formed here out of the loop's registers
        if (any_not_finite(acc)) {
          int row[MT];
#pragma unroll
          for (int i = 0; i < MT; ++i) row[i] = row_of(rows, i);
          multiply_again(
              acc, K, lane,
              [&](int i, int64_t k) {
                const float a = row[i] < 0 ? 0.f : x[int64_t(row[i]) * g.ldx + k];
                return !WT && g.act ? silu(a) : a;
              },
              [&](int j, int64_t k) {
                const int n = n0 + 16 * j + lane % 16;
                return n >= N ? 0.f : WT ? w[int64_t(n) * K + k] : w[k * N + n];
              });
        } else {
          const float u = l % 2 ? -kUnscale : kUnscale;
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] *= u;
        }
        constexpr int W = 4;
        int row[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) row[i] = row_of(rows, i);
        const int n = n0 + W * (lane / 16);
        if (WT && pre) {
          const bool whole = N - n0 >= TN;
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const float *p = pre + int64_t(row[i] < 0 ? 0 : row[i]) * g.ldp + n;
            __builtin_amdgcn_sched_barrier(0);  // one row's values at a time
            u32x4 v[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) v[j] = load_bits<W>(p + 16 * j, whole ? W : N - n - 16 * j);
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][j][e] *= silu_grad(value_of<float>(v[j], e));
          }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          if (row[i] < 0) continue;
          float *o = y + int64_t(row[i]) * g.ldy + n;
#pragma unroll
          for (int j = 0; j < NI; ++j) {
            const float v[W] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            store_row<W>(o + 16 * j, v, N - n - 16 * j);
          }
        }
        clear();
        ck = 0;
        cc += kStreamWaves;
        rows = list(cc);
      };
      u32x4 v0[MT][XP], v1[MT][XP];
      load(v0);
      load(v1);
      while (cc < chunks) {
        for (int k = 0; k < steps; k += 2) {
          step(v0);
          step(v1);
        }
        finish();
      }
    }
  });
}

// ------------------------------------------------------- weight gradient
struct WeightArgs {
  int64_t M;
  int K, N, G, act, range;  // rows of a range
  const int64_t *offsets;
  const int32_t *rows;
  const void *x;  // [M][K]
  int64_t ldx;
  const void *dy;  // [M][N]
  int64_t lddy;
  void *dw;     // [G][K][N]
  float *part;  // [2 (M / range) + 1][slot]
  int64_t slot;
  int kt, nt;
  int64_t ranges;  // upper bound
};

// Range k of a group of several goes to slot 2 (offsets[g] / range) + k: such a
// group has more than `range` rows, so the next one's slots start behind it.  BUFS as
// in product_kernel.
//
// Measured: 523,599 rows of 16 types, K = 128, N = 64 fp32 with SiLU 114 to 130 us (402 MB,
// 3.5 TB/s: three workgroups a compute unit have one step of 24 KB each in flight); bf16,
// 100,003 x 1024 x 512 of 100 types 222 to 233 us of 105 GFLOP: both operands' transposing
// reads fill the LDS, and 100 groups of uneven length leave the last of three rounds half
// empty (one type: a fifth less).
template <class T, int TK, int TN, int BUFS>
__global__ __launch_bounds__(BUFS == 2 ? 512 : tile_threads(TN), TN == 256 ? 4 : 2) void weight_kernel(
    WeightArgs g) {
  constexpr int KS = Kind<T>::KS;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int NT = BUFS == 2 ? 512 : tile_threads(TN), MI = TK / 32, NI = TN / 16 / (NT / 128);
  using XTile = Across<T, TK, false, NT, tile_short(TN)>;
  using YTile = Across<T, TN, false, NT, tile_short(TN)>;
  __shared__ u32x4 x_lds[BUFS * XTile::SIZE], y_lds[BUFS * YTile::SIZE];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), l = tid % kWave;
  const int tiles = g.kt * g.nt;
  // in plain order over the XCDs: groups differ in length, and a range's tiles
  // take the same time
  const int64_t b = blockIdx.x;
  const Tile t = find_tile(g.offsets, g.G, g.M, g.range, b / tiles, l);
  if (t.g == g.G) return;
  const int64_t begin = t.begin;
  const bool only = t.end - begin <= g.range;  // the group's only range, if it has rows at all
  if (t.m0 >= t.end && !(t.m0 == begin && t.end == begin)) return;
  const int64_t end = t.m0 + g.range < t.end ? t.m0 + g.range : t.end;
  const int k0 = int(b % tiles) / g.nt * TK, n0 = int(b % tiles) % g.nt * TN, K = g.K, N = g.N;
  const T *x = static_cast<const T *>(g.x), *dy = static_cast<const T *>(g.dy);
  auto row_of = [&](int64_t i) -> int {
    const int64_t in = i < end ? i : end - 1;
    const int r = g.rows ? g.rows[in] : int(in);
    return i < end && r >= 0 && r < g.M ? r : -1;
  };
  XTile xa;
  YTile ya;
  // rows: lane i has the list's entry i of the next step, loaded a step ahead; bit i
  // of xm and ym: the step at hand has no row step(i, tid)
  int rows = 0, xm = 0, ym = 0;
  auto load = [&]() {
    int t = tid;
    if constexpr (TN == 256) asm volatile("" : "+v"(t));  // addresses are formed anew: 128 registers
    int xr[XTile::NP], yr[YTile::NP];
    xm = ym = 0;
#pragma unroll
    for (int i = 0; i < XTile::NP; ++i) {
      xr[i] = __shfl(rows, XTile::step(i, t));
      xm |= int(xr[i] < 0) << i;
    }
#pragma unroll
    for (int i = 0; i < YTile::NP; ++i) {
      yr[i] = __shfl(rows, YTile::step(i, t));
      ym |= int(yr[i] < 0) << i;
    }
    xa.load([&](int i) { return x + (xr[i] < 0 ? 0 : int64_t(xr[i]) * g.ldx); }, k0, K, t);
    ya.load([&](int i) { return dy + (yr[i] < 0 ? 0 : int64_t(yr[i]) * g.lddy); }, n0, N, t);
  };
  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int wk = 16 * MI * (wave % 2), wn = 16 * NI * (wave / 2);
  const typename XTile::Reader x_read(wk / 16, l);
  const typename YTile::Reader y_read(wn / 16, l);
  float sign = 1.f;
  if (t.m0 < end) {
    rows = row_of(t.m0 + l % KS);
    load();
    rows = row_of(t.m0 + KS + l % KS);
  }
  auto put = [&](int buf, float sign) {
    xa.put(x_lds + buf * XTile::SIZE, g.act, sign * kScale, k0, K, xm, tid);
    ya.put(y_lds + buf * YTile::SIZE, false, kScale, n0, N, ym, tid);
  };
  if constexpr (BUFS == 1) {
    for (int64_t m = t.m0; m < end; m += KS) {
      lds_sync<NT / kWave>();
      put(0, sign);
      lds_sync<NT / kWave>();
      if (m + KS < end) {
        load();
        rows = row_of(m + 2 * KS + l % KS);
      }
      multiply<T, XTile, YTile, TN == 256>(x_lds, y_lds, x_read, y_read, sign, acc);
      sign = -sign;
    }
  } else if (t.m0 < end) {
    put(0, sign);
    if (t.m0 + KS < end) {
      load();
      rows = row_of(t.m0 + 2 * KS + l % KS);
    }
    int buf = 0;
    for (int64_t m = t.m0; m < end; m += KS) {
      lds_sync<NT / kWave>();
      auto next = [&] {
        if (m + KS < end) put(buf ^ 1, -sign);
        if (m + 2 * KS < end) {
          load();
          rows = row_of(m + 3 * KS + l % KS);
        }
      };
      if (wave < NT / kWave / 2) next();
      multiply<T, XTile, YTile, TN == 256>(x_lds + buf * XTile::SIZE, y_lds + buf * YTile::SIZE, x_read, y_read, sign, acc);
      if (wave >= NT / kWave / 2) next();
      sign = -sign;
      buf ^= 1;
    }
  }
  if constexpr (F32) {
    if (any_not_finite(acc)) {
      multiply_again(
          acc, end - t.m0, l,
          [&](int i, int64_t m) {
            const int r = row_of(t.m0 + m);
            const int k = k0 + wk + 16 * i + l % 16;
            const float v = r < 0 || k >= K ? 0.f : x[int64_t(r) * g.ldx + k];
            return g.act ? silu(v) : v;
          },
          [&](int j, int64_t m) {
            const int r = row_of(t.m0 + m);
            const int n = n0 + wn + 16 * j + l % 16;
            return r < 0 || n >= N ? 0.f : dy[int64_t(r) * g.lddy + n];
          });
    } else {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] *= kUnscale;
    }
  }
  const int k_first = uint32_t(t.m0 - begin) / uint32_t(g.range);
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int k = k0 + wk + 16 * i + l % 16;
    if (k >= K) continue;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int n = n0 + wn + 16 * j + 4 * (l / 16);
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e];
      if (only)
        store_row<4>(static_cast<T *>(g.dw) + (int64_t(t.g) * K + k) * N + n, v, N - n);
      else
        store_row<4>(g.part + (2 * int64_t(uint32_t(begin) / uint32_t(g.range)) + k_first) * g.slot + int64_t(k) * N + n, v, N - n);
    }
  }
}

// Workgroup (e, y): elements of the y-th group that has several ranges.  SPLIT: 256
// elements, whose ranges the waves share; else 256 for every wave, which adds all
// ranges: where there are that many elements (1024 x 512 of 24 ranges: 54 us
// with SPLIT, 13 without).  Bound by reading the partial sums once.
constexpr int kSumThreads = 512, kSumWaves = kSumThreads / kWave;
template <class T, bool SPLIT>
__global__ __launch_bounds__(kSumThreads) void weight_sum_kernel(WeightArgs g) {
  __shared__ f32x4 sums[SPLIT ? kSumWaves : 1][kWave];
  const int tid = threadIdx.x, l = tid % kWave, wave = tid / kWave;
  auto clamped = [&](int i) {
    const int64_t o = g.offsets[i];
    return o < 0 ? int64_t(0) : o > g.M ? g.M : o;
  };
  int left = blockIdx.y, found = -1;
  for (int i0 = 0; i0 < g.G && found < 0; i0 += kWave) {
    const int i = i0 + l;
    const uint64_t several = __ballot(i < g.G && clamped(i + 1) - clamped(i) > g.range);
    const int n = __popcll(several);
    if (left < n) {
      uint64_t rest = several;
      for (int k = 0; k < left; ++k) rest &= rest - 1;
      found = i0 + __builtin_ctzll(rest);
    } else {
      left -= n;
    }
  }
  if (found < 0) return;
  const int64_t begin = clamped(found), rows = clamped(found + 1) - begin, KN = int64_t(g.K) * g.N;
  const int ranges = int((rows + g.range - 1) / g.range);
  const int64_t e = (SPLIT ? int64_t(blockIdx.x) : int64_t(blockIdx.x) * kSumWaves + wave) * 256 + 4 * l;
  const int first = SPLIT ? wave : 0, step = SPLIT ? kSumWaves : 1;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (e < KN) {
    const float *p = g.part + 2 * (begin / g.range) * g.slot + e;  // slots are padded to whole vectors
#pragma unroll 8
    for (int k = first; k < ranges; k += step) s += *reinterpret_cast<const f32x4 *>(p + k * g.slot);
  }
  if constexpr (SPLIT) {
    sums[wave][l] = s;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int k = 1; k < kSumWaves; ++k) s += sums[k][l];
  }
  if (e >= KN) return;
  T *o = static_cast<T *>(g.dw) + int64_t(found) * KN + e;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (e + i < KN) o[i] = from_f32<T>(s[i]);
}

template <class T>
__global__ void fill_zero_kernel(int64_t n, T *p) {
  for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < n; i += int64_t(gridDim.x) * blockDim.x)
    p[i] = T(0);
}

// --------------------------------------------------------- 8-bit product
struct ProductF8Args {
  int64_t M;
  int K, N, G;
  const int64_t *offsets;  // null, and then rows too: one group of all rows
  const int32_t *rows;
  const uint8_t *x;  // [M][K]
  int64_t ldx;
  const float *xs;   // [M][kb]
  const uint8_t *w;  // [G][N][K]
  const float *ws;   // [G][nb][kb]
  uint16_t *y;       // [M][N] bf16
  int64_t ldy;
  int nt;
  int64_t mt;
  int64_t first;
};

// Drops the first `by` bytes of 16; zeros follow the last.
__device__ __forceinline__ u32x4 cut_bytes(u32x4 a, int by) {
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_alignbit(i < 3 ? a[i + 1] : 0u, a[i], 8 * (by % 4));
  if (by & 4) o = u32x4{o[1], o[2], o[3], 0};
  if (by & 8) o = u32x4{o[2], o[3], 0, 0};
  if (by >= 16) o = u32x4{0, 0, 0, 0};
  return o;
}

__device__ __forceinline__ i32x8 operand_f8(u32x4 lo, u32x4 hi) {
  return i32x8{int(lo[0]), int(lo[1]), int(lo[2]), int(lo[3]), int(hi[0]), int(hi[1]), int(hi[2]), int(hi[3])};
}

// The sums of one block of 128; both block scales of the instruction are 2^(127 - 127).
__device__ __forceinline__ f32x4 block_sum_f8(i32x8 w, i32x8 x) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0x7f7f7f7f, 0,
                                                          0x7f7f7f7f);
}

// A step is one block of 128 along K: one matrix instruction (16 x 16 x 128) forms
// the block's sums, which the vector units add with the two scales' product.  The
// instruction aligns each 8 products to the largest of them and drops what is
// below 2^-13 of it (measured; the 16 x 16 x 32 one does the same at half the
// rate), 2e-6 of the terms' magnitudes for normally distributed operands: far
// below the bf16 output's 2^-8, and the reason that there is no fp32 output.
template <int TN>
__global__ __launch_bounds__(kThreads, 2) void product_f8_kernel(ProductF8Args g) {
  constexpr int KS = 128, MI = 4, NI = TN / 32;
  __shared__ u32x4 x_lds[kTileRows * KS / 16], w_lds[TN * KS / 16];
  __shared__ int srow[kTileRows];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), l = tid % kWave;
  const int64_t b = g.first + xcd_order(blockIdx.x, gridDim.x);
  Tile t;
  if (g.offsets)
    t = find_tile(g.offsets, g.G, g.M, kTileRows, b / g.nt, l);
  else
    t = {0, 0, (b / g.nt) * kTileRows, g.M};
  if (t.m0 >= t.end) return;
  const int n0 = int(b % g.nt) * TN, K = g.K, N = g.N;
  uint16_t *y = g.y;
  list_rows(srow, g.rows, t, g.M, tid);
  __syncthreads();
  if (t.g == g.G) {
    zero_rows(srow, y, g.ldy, n0, N - n0 < TN ? N - n0 : TN, tid);
    return;
  }
  const int kb = (K + KS - 1) / KS, nb = (N + KS - 1) / KS;
  const uint8_t *w = g.w + int64_t(t.g) * N * K;
  // TN divides 128, so a tile's columns share their scales
  const float *ws = g.ws + (int64_t(t.g) * nb + n0 / KS) * kb;
  const int wm = 64 * (wave % 2), wn = TN / 2 * (wave / 2);
  const uint8_t *xr[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = srow[tid / 8 + 32 * i];
    xr[i] = g.x + (r < 0 ? 0 : int64_t(r) * g.ldx);
  }
  int mrow[MI];
#pragma unroll
  for (int i = 0; i < MI; ++i) mrow[i] = srow[wm + 16 * i + l % 16];
  // 16 bytes from k on, as Along does: pieces that cross the row's end are loaded
  // before it and shifted when they are used
  const int at_last = K - 16;
  auto load16 = [&](const uint8_t *p, int k) {
    u32x4 v = {0, 0, 0, 0};
    if (at_last >= 0) {
      v = *reinterpret_cast<const u32x4_any8 *>(p + unsigned(k < at_last ? k : at_last));
    } else {
#pragma unroll
      for (int e = 0; e < 15; ++e)
        if (k == 0 && e < K) v[e / 4] |= uint32_t(p[e]) << (8 * (e % 4));
    }
    return v;
  };
  auto cut = [&](u32x4 a, int k) { return at_last < 0 ? a : cut_bytes(a, k < at_last ? 0 : k - at_last); };
  constexpr int NW = TN / 32;
  u32x4 a[4], bw[NW];
  float sx[MI], sw = 0.f;
  auto load = [&](int k0) {
    const int k = k0 + 16 * (tid % 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = load16(xr[i], k);
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const int n = n0 + tid / 8 + 32 * i;
      bw[i] = load16(w + int64_t(n < N ? n : N - 1) * K, k);
    }
    sw = ws[k0 / KS];
#pragma unroll
    for (int i = 0; i < MI; ++i) sx[i] = g.xs[int64_t(mrow[i] < 0 ? 0 : mrow[i]) * kb + k0 / KS];
  };
  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  load(0);
  for (int k0 = 0; k0 < K; k0 += KS) {
    lds_sync<4>();
    if (k0 + KS > K) {
      const int k = k0 + 16 * (tid % 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = cut(a[i], k);
#pragma unroll
      for (int i = 0; i < NW; ++i) bw[i] = cut(bw[i], k);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x_lds[swizzled<8, false>(tid / 8 + 32 * i, tid % 8)] = a[i];
#pragma unroll
    for (int i = 0; i < NW; ++i) w_lds[swizzled<8, true>(tid / 8 + 32 * i, tid % 8)] = bw[i];
    lds_sync<4>();
    float sc[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) sc[i] = sx[i] * sw;
    if (k0 + KS < K) load(k0 + KS);
    // lane l takes chunks l / 16 and l / 16 + 4 of both operands
    i32x8 xf[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int r = wm + 16 * i + l % 16;
      xf[i] = operand_f8(x_lds[swizzled<8, false>(r, l / 16)], x_lds[swizzled<8, false>(r, l / 16 + 4)]);
    }
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int n = wn + column_of<true>(j, l % 16);
      const i32x8 wf = operand_f8(w_lds[swizzled<8, true>(n, l / 16)], w_lds[swizzled<8, true>(n, l / 16 + 4)]);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const f32x4 s = block_sum_f8(wf, xf[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(sc[i], s[e], acc[i][j][e]);
      }
    }
  }
  constexpr int W = 8, JW = 2;
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    if (mrow[i] < 0) continue;
#pragma unroll
    for (int j = 0; j < NI; j += JW) {
      const int n = n0 + wn + 16 * j + W * (l / 16);
      float v[W];
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] = acc[i][j + e / 4][e % 4];
      store_row<W>(y + int64_t(mrow[i]) * g.ldy + n, v, N - n);
    }
  }
}

// The same past weights that stay in LDS (see product_stream_kernel): rows of up to
// 1152 values for 128 columns.  A wave has 48 rows in flight, its loads a block
// ahead; a block's sums are scaled as above.
//
// Measured: 262,144 rows of 16 types, K = N = 1024 385 us, 1.43 PFLOP/s, bound by its loads: with
// them alone it takes 302 us, without loads and stores 213.  X is read by 8 workgroups, one for
// each 128 columns (2.1 GB through L2), and a block's 24 products of a wave do not cover a
// load's latency.  Stores
// of 64 bytes a row took 460.
constexpr int kStreamF8K = kStreamLds / 128;  // longest contraction

__global__ __launch_bounds__(kStreamThreads, 2) void product_f8_stream_kernel(ProductF8Args g) {
  constexpr int KS = 128, TN = 128, C = KS / 16, MT = 3, NI = TN / 16, RB = 16 * MT;
  __shared__ u32x4 w_lds[kStreamLds / 16];  // per block of K: TN rows of 128 bytes
  constexpr int KB = kStreamF8K / KS;
  __shared__ float ws_lds[KB], xs_lds[kStreamWaves][RB * KB];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), l = tid % kWave;
  const int64_t b = xcd_order(blockIdx.x, g.mt * g.nt);
  const int n0 = int(b % g.nt) * TN, K = g.K, N = g.N, kb = (K + KS - 1) / KS, nb = (N + KS - 1) / KS;
  const int at_last = K - 16;
  uint16_t *y = g.y;
  // rows column_of<true>(j, l % 16), chunks l / 16 and l / 16 + 4, of an even and an odd j
  const int base[2] = {swizzled<C, true>(column_of<true>(0, l % 16), l / 16),
                       swizzled<C, true>(column_of<true>(1, l % 16), l / 16)};
  stream_share<RB>(g.offsets, g.rows, g.G, g.M, b / g.nt, g.mt, l, [&](int group, int chunks, auto list) {
    if (group == g.G) {
      stream_zeros<RB>(chunks, list, y, g.ldy, n0, n0 + TN < N ? n0 + TN : N, wave, l);
      return;
    }
    auto row_of = [&](int rows, int i) { return __shfl(rows, 16 * i + l % 16); };
    const uint8_t *w = g.w + int64_t(group) * N * K;
    int ft = tid;
    asm volatile("" : "+v"(ft));
    __syncthreads();  // the group before has been multiplied
    if (ft < kb) ws_lds[ft] = g.ws[(int64_t(group) * nb + n0 / KS) * kb + ft];
#pragma unroll 1
    for (int k0 = 0; k0 < K; k0 += KS) {
      u32x4 v[2];
      const int k = k0 + 16 * (ft % 8);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int n = n0 + ft / 8 + 64 * i;  // columns past the last read it, and reach no output
        v[i] = *reinterpret_cast<const u32x4_any8 *>(w + int64_t(n < N ? n : N - 1) * K + (k < at_last ? k : at_last));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
        w_lds[k0 / KS * (TN * C) + swizzled<C, true>(ft / 8 + 64 * i, ft % 8)] = cut_bytes(v[i], k < at_last ? 0 : k - at_last);
    }
    __syncthreads();
    if (wave >= chunks) return;
    // the loads' side: chunk lc, block lk; next: the rows of the chunk after lc
    int lc = wave, lk = 0, next = list(lc), lrow[MT];
    auto point = [&]() {
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int r = row_of(next, i);
        lrow[i] = r < 0 ? 0 : r;
      }
      next = list(lc + kStreamWaves);
    };
    point();
    // The rows' scales, kb to a row, pass through LDS: lane i loads those of row i a
    // chunk ahead.  (Loaded where they are used, 16 rows' lines at a time, they took
    // as long as a fifth of the kernel.)
    float *scales = xs_lds[wave];
    float ahead[KB];
    auto load_scales = [&](int rows) {
      const float *p = g.xs + int64_t(rows < 0 ? 0 : rows) * kb;
#pragma unroll
      for (int i = 0; i < KB; ++i) ahead[i] = p[i < kb ? i : kb - 1];
    };
    auto keep_scales = [&]() {
      if (l < RB) {
#pragma unroll
        for (int i = 0; i < KB; ++i) scales[l * KB + i] = ahead[i];
      }
      lds_sync<1>();
    };
    struct Rows {
      u32x4 lo[MT], hi[MT];
    };
    auto load = [&](Rows &v) {
      const int k = lk * KS + 16 * (l / 16), k2 = k + 64;
      const unsigned at = unsigned(k < at_last ? k : at_last), at2 = unsigned(k2 < at_last ? k2 : at_last);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const uint8_t *p = g.x + int64_t(lrow[i]) * g.ldx;
        v.lo[i] = *reinterpret_cast<const u32x4_any8 *>(p + at);
        v.hi[i] = *reinterpret_cast<const u32x4_any8 *>(p + at2);
      }
      if (++lk == kb) {
        lk = 0;
        lc += kStreamWaves;
        point();
      }
    };
    f32x4 acc[MT][NI];
    auto clear = [&]() {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    clear();
    int cc = wave, ck = 0, rows = list(cc);  // the products' side
    auto step = [&](Rows &v) {
      if (ck * KS + KS > K) {
        const int k = ck * KS + 16 * (l / 16);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          v.lo[i] = cut_bytes(v.lo[i], k < at_last ? 0 : k - at_last);
          v.hi[i] = cut_bytes(v.hi[i], k + 64 < at_last ? 0 : k + 64 - at_last);
        }
      }
      i32x8 xf[MT];
      float sc[MT];
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        xf[i] = operand_f8(v.lo[i], v.hi[i]);
        sc[i] = scales[(16 * i + l % 16) * KB + ck] * ws_lds[ck];
      }
      load(v);
      const u32x4 *d = w_lds + ck * (TN * C);
      auto operand = [&](int j) {
        const u32x4 *p = d + 32 * (j / 2) * C;
        return operand_f8(p[base[j % 2]], p[base[j % 2] ^ 4]);
      };
      // the sums of a product are added under the next one's instructions
      f32x4 s[MT];
      i32x8 wf = operand(0);
#pragma unroll
      for (int i = 0; i < MT; ++i) s[i] = block_sum_f8(wf, xf[i]);
      wf = operand(1);
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        f32x4 u[MT];
        i32x8 wn = wf;
        if (j + 2 < NI) wn = operand(j + 2);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          if (j + 1 < NI) u[i] = block_sum_f8(wf, xf[i]);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(sc[i], s[i][e], acc[i][j][e]);
        }
        wf = wn;
#pragma unroll
        for (int i = 0; i < MT; ++i) s[i] = u[i];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
        }
      }
      if (++ck < kb) return;
      int lane = l;
      asm volatile("" : "+v"(lane));  // keeps the addresses formed here out of the loop's registers
      // four columns' parts of four rows change lanes, so that a store covers whole
      // rows of the tile: 256 bytes of four instead of 64 of sixteen
      const int n = n0 + 32 * (lane % 4) + 8 * (lane / 16);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        u32x4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[q][e] = bf16_pair(acc[i][2 * q + e / 2][2 * (e % 2)], acc[i][2 * q + e / 2][2 * (e % 2) + 1]);
        quad_transpose(v, lane);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int r = __shfl(rows, 16 * i + (lane % 16 & 12) + q);
          if (r >= 0) store_bits(y + int64_t(r) * g.ldy + n, v[q], N - n);
        }
      }
      clear();
      ck = 0;
      cc += kStreamWaves;
      rows = list(cc);
      keep_scales();
      load_scales(list(cc + kStreamWaves));
    };
    Rows v;
    load(v);
    load_scales(rows);
    keep_scales();
    load_scales(list(cc + kStreamWaves));
    while (cc < chunks) step(v);
  });
}

// ------------------------------------------------------------- launches
// A workgroup for every tile, in as many launches as that takes.
template <class Args>
void launch_tiles(void (*kernel)(Args), Args g, int64_t tiles, int threads, hipStream_t s) {
  for (g.first = 0; g.first < tiles; g.first += kMaxGrid)
    hipLaunchKernelGGL(kernel, dim3(unsigned(std::min(tiles - g.first, kMaxGrid))), dim3(threads), 0, s, g);
}

template <class T, bool WT>
void launch_product(ProductArgs g, hipStream_t s) {
  const bool narrow = g.N <= 64;
  g.nt = narrow ? 1 : int(cdiv(g.N, 128));
  if constexpr (sizeof(T) == 4) {
    // Rows past stationary weights, or tiles.  Tiles against this, us, forward, 1 and
    // 100 types: M = 32,000 K = 128 N = 128 18 against 21 and 22 against 24;
    // M = 128,000 44 against 38 and 52 against 43; M = 500,000 168 against 138 and
    // 178 against 140 (K = 192: 220 against 183); with few rows to a type the
    // weights' loads tell: M = 8,000 and 100 types 17 against 37.
    const int fits = narrow ? stream_k<64>() : stream_k<128>();
    if (g.K >= Kind<T>::PE && g.K <= fits && g.M >= 65536 && g.M >= 512 * int64_t(g.G)) {
      g.mt = std::max(1, kStreamGroups / g.nt);
      const dim3 grid(unsigned(g.mt * g.nt)), block(kStreamThreads);
      if (narrow)
        hipLaunchKernelGGL((product_stream_kernel<64, WT>), grid, block, 0, s, g);
      else
        hipLaunchKernelGGL((product_stream_kernel<128, WT>), grid, block, 0, s, g);
      return;
    }
  }
  g.mt = tile_bound(g.M, g.G, kTileRows);
  if constexpr (sizeof(T) == 2 && !WT) {
    // 256 columns at a time, so that a row's SiLU is computed half as often: against
    // 128, K = 512, N = 512, 1 and 100 types: M = 32,000 38 against 29 and 50 against
    // 46, M = 400,000 394 against 352 and 415 against 358; against 64, M = 3,700 and 100
    // types 28 against 19.  Without SiLU and for the gradient of X both are within 5%.
    // Two buffers up to a tile per compute unit: 204 tiles, K = 1024 35 against 28;
    // 254, K = 512 22 against 18; 259, K = 1024 46 against 50.
    const int nt = int(cdiv(g.N, 256));
    const int64_t tiles = g.mt * nt;
    if (g.act && g.N > 128 && g.K >= 256 && tiles > 128) {
      g.nt = nt;
      if (tiles <= 256)
        launch_tiles(product_kernel<T, 256, false, 2>, g, tiles, 2 * kThreads, s);
      else
        launch_tiles(product_kernel<T, 256, false, 1>, g, tiles, 2 * kThreads, s);
      return;
    }
  }
  // 64 columns at a time where 128 would leave compute units without a tile, or a
  // quarter of the columns empty: 128 against 64, forward of fp32 512 x 512: 164 tiles
  // (of 128 columns) 39 against 31, 316 53 against 51, 424 55 against 62; bf16 17 against
  // 15 and 17.5 against 17.9 at 316 and 424.  The gradient of X gains with more tiles:
  // fp32 K = 256, N = 256 530 tiles 55 against 44, K = 768, N = 128 636 tiles 41 against
  // 32, 512 x 512 756 tiles 90 and 90; bf16 474 tiles 12.6 against 11.5, 530 17.6
  // against 18.2.  Two buffers against one, forward: fp32 M = 5,000 K = 768, N = 128 41
  // against 29, M = 50,000 256 x 64 28 against 25; bf16 M = 3,700 1024 x 256 22.3
  // against 20.0, but with 1,564 tiles of 64 x 64 13.8 against 16.4.
  constexpr bool F32 = sizeof(T) == 4;
  const int64_t tiles = g.mt * g.nt;
  if (narrow || tiles <= (!WT ? 320 : F32 ? 640 : 512) || 4 * g.N <= 3 * 128 * g.nt) {
    g.nt = int(cdiv(g.N, 64));
    if (F32 || g.mt * g.nt <= 256) {
      launch_tiles(product_kernel<T, 64, WT, 2>, g, g.mt * g.nt, 2 * kThreads, s);
      return;
    }
    if constexpr (!F32) launch_tiles(product_kernel<T, 64, WT, 1>, g, g.mt * g.nt, kThreads, s);
  } else {
    launch_tiles(product_kernel<T, 128, WT, 1>, g, tiles, kThreads, s);
  }
}

// Of dW's sums: tiles, rows of a range, slots of partial sums.
//
// As many workgroups as stay on the chip together (`all`) and not one more, since a few
// left over would take as long again: with n = G tiles workgroups, ranges of R rows are at
// most M tiles / R + n of them.  Where the groups' ends, half a range each, would leave a
// sixteenth of the chip idle, twice as many; where the groups alone fill half of it, ranges only
// even out their lengths.  No more than 2 `all` tiles of partial sums in any case.  fp32
// against ranges of a power of two, 2/3 to 4/3 of 768 workgroups, us: M = 523,599 K = 128
// N = 64 of 16 types 146 against 116, M = 300,000 192 x 128 257 against 178, M = 1,000,000
// 256 x 100 574 against 570, and 935 with ranges 2% too short.
struct WeightShape {
  int range, kt, nt;
  bool wide, few;
  int64_t slot, slots;
};
WeightShape weight_shape(int dtype, int64_t M, int K, int N, int G) {
  WeightShape z;
  z.kt = int(K <= 64 ? 1 : cdiv(K, 128));
  z.nt = int(N <= 64 ? 1 : cdiv(N, 128));
  z.wide = dtype == ALLEGRO_BF16 && K > 64 && N > 128 && M * z.kt * z.nt >= 1 << 20;
  if (z.wide) z.nt = int(cdiv(N, 256));
  const int on_unit = z.wide || (dtype == ALLEGRO_F32 && K > 64 && N > 64) ? 2 : 3;
  const int64_t tiles = int64_t(z.kt) * z.nt, n = G * tiles, all = 256 * on_unit;
  const int64_t rows = cdiv(M * tiles, n <= all / 8 ? all - n : n <= all / 2 ? 2 * all - n : all);
  z.range = int(cdiv(std::min<int64_t>(std::max<int64_t>(rows, 256), 1 << 30), 64) * 64);
  // Up to a workgroup per compute unit: tiles of 64 x 64 instead, through two buffers, and
  // while their ranges are few, shorter ones (from 1024 rows on, below which they would
  // add the launch of their sums).  fp32, us, against 128 columns and two buffers: M =
  // 1,640 192 x 103 25.6 against 17.5, and 14.7 with ranges of 128; 3,700 rows of 16 types
  // 128 x 64 19.4, 16.1, 15.3; 20,000 128 x 128 28.6, 24.1 (22.5 with the ranges that are too
  // many by the rule); 12,000 96 x 200 29.1, 24.3 (26.5); bf16 gains up to 3 us.
  z.few = (M / z.range) * tiles + n <= 256;
  if (z.few) {
    z.kt = int(cdiv(K, 64));
    z.nt = int(cdiv(N, 64));
    if (M >= 1024 && (M / 128) * z.kt * z.nt <= 256) z.range = 128;
  }
  z.slot = cdiv(int64_t(K) * N, 4) * 4;
  z.slots = M > z.range ? 2 * (M / z.range) + 1 : 0;
  return z;
}

template <class T>
void launch_weight(WeightArgs g, const WeightShape &z, hipStream_t s) {
  g.range = z.range;
  g.kt = z.kt;
  g.nt = z.nt;
  g.slot = z.slot;
  g.ranges = tile_bound(g.M, g.G, z.range);
  const dim3 grid(unsigned(g.ranges * g.kt * g.nt));
  if constexpr (sizeof(T) == 2) {
    // 256 columns of dW at a time against 128, us, 1 and 100 types: K = 128, N = 256
    // M = 32,000 22.5 against 26.7 and 26 against 28, 100,000 39 against 39 and 43 against 44;
    // K = 512, N = 512 M = 32,000 59 against 59 and 70 against 78, 400,000 476 against 403
    // and 482 against 439; M = 100,003 1024 x 512 of 100 types 245 against 230
    if (z.wide) hipLaunchKernelGGL((weight_kernel<T, 128, 256, 1>), grid, dim3(tile_threads(256)), 0, s, g);
  }
  if (!z.wide) {
    if (z.few)
      hipLaunchKernelGGL((weight_kernel<T, 64, 64, 2>), grid, dim3(2 * kThreads), 0, s, g);
    else if (g.K <= 64 && g.N <= 64)
      hipLaunchKernelGGL((weight_kernel<T, 64, 64, 1>), grid, dim3(kThreads), 0, s, g);
    else if (g.K <= 64)
      hipLaunchKernelGGL((weight_kernel<T, 64, 128, 1>), grid, dim3(kThreads), 0, s, g);
    else if (g.N <= 64)
      hipLaunchKernelGGL((weight_kernel<T, 128, 64, 1>), grid, dim3(kThreads), 0, s, g);
    else
      hipLaunchKernelGGL((weight_kernel<T, 128, 128, 1>), grid, dim3(kThreads), 0, s, g);
  }
  if (z.slots) {
    const unsigned several = unsigned(std::min<int64_t>(g.G, g.M / z.range));
    const int64_t parts = cdiv(int64_t(g.K) * g.N, 256);
    if (parts * several < 4096)
      hipLaunchKernelGGL((weight_sum_kernel<T, true>), dim3(unsigned(parts), several), dim3(kSumThreads), 0, s, g);
    else
      hipLaunchKernelGGL((weight_sum_kernel<T, false>), dim3(unsigned(cdiv(parts, kSumWaves)), several),
                         dim3(kSumThreads), 0, s, g);
  }
}

int check_product(int dtype, int act, int64_t M, int K, int N, int G) {
  int rc;
  if ((rc = check_dtype(dtype))) return rc;
  if (act != ALLEGRO_ACT_NONE && act != ALLEGRO_ACT_SILU) return fail(ALLEGRO_E_INVALID, "unknown act %d", act);
  if ((rc = check_m(M)) || (rc = check_width(K, "K")) || (rc = check_width(N, "N")) || (rc = check_g(G))) return rc;
  // one workgroup per tile of 128 rows and 64 columns or more, at most 2^31 - 1 of them
  if (cdiv(std::max(K, N), 64) * tile_bound(M, G, kTileRows) > kMaxRows)
    return fail(ALLEGRO_E_UNSUPPORTED, "M=%lld rows of %d columns are more than 2^31 - 1 tiles", (long long)M,
                std::max(K, N));
  return ALLEGRO_OK;
}

}  // namespace

extern "C" {

int allegro_grouped_matmul(int dtype, int act, int64_t M, int K, int N, int G, const int64_t *offsets,
                           const int32_t *rows, const void *X, int64_t ldx, const void *W, void *Y, int64_t ldy,
                           void *stream) {
  int rc;
  if ((rc = check_product(dtype, act, M, K, N, G))) return rc;
  if (M == 0) return ALLEGRO_OK;
  const int e = dtype == ALLEGRO_F32 ? 4 : 2;
  if ((rc = check_ptr(offsets, "offsets", 8)) || (rows && (rc = check_ptr(rows, "rows", 4))) ||
      (rc = check_rows(X, "X", ldx, K, e)) || (rc = check_ptr(W, "W", e)) || (rc = check_rows(Y, "Y", ldy, N, e)) ||
      (rc = check_apart(Y, "Y", {X, W})))
    return rc;
  const ProductArgs g{M, K, N, G, offsets, rows, X, ldx, W, Y, ldy, nullptr, 0, act, 0, 0, 0};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == ALLEGRO_F32)
    launch_product<float, false>(g, s);
  else
    launch_product<uint16_t, false>(g, s);
  return after("allegro_grouped_matmul");
}

int allegro_grouped_matmul_workspace(int64_t M, int K, int N, int G, size_t *bytes) {
  int rc;
  if ((rc = check_product(ALLEGRO_F32, ALLEGRO_ACT_NONE, M, K, N, G))) return rc;
  if (!bytes) return fail(ALLEGRO_E_INVALID, "bytes is NULL");
  const WeightShape a = weight_shape(ALLEGRO_F32, M, K, N, G), b = weight_shape(ALLEGRO_BF16, M, K, N, G);
  *bytes = size_t(std::max(a.slots, b.slots)) * size_t(a.slot) * sizeof(float);
  return ALLEGRO_OK;
}

int allegro_grouped_matmul_backward(int dtype, int act, int64_t M, int K, int N, int G, const int64_t *offsets,
                                    const int32_t *rows, const void *X, int64_t ldx, const void *W, const void *dY,
                                    int64_t lddy, void *dX, int64_t lddx, void *dW, void *workspace,
                                    size_t workspace_bytes, void *stream) {
  int rc;
  if ((rc = check_product(dtype, act, M, K, N, G))) return rc;
  const int e = dtype == ALLEGRO_F32 ? 4 : 2;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dW && (rc = check_ptr(dW, "dW", e))) return rc;
  if (M == 0) {
    if (!dW) return ALLEGRO_OK;
    const int64_t n = int64_t(G) * K * N;
    const dim3 grid(unsigned(std::min<int64_t>(cdiv(n, kThreads), 4096)));
    if (dtype == ALLEGRO_F32)
      hipLaunchKernelGGL(fill_zero_kernel<float>, grid, dim3(kThreads), 0, s, n, static_cast<float *>(dW));
    else
      hipLaunchKernelGGL(fill_zero_kernel<uint16_t>, grid, dim3(kThreads), 0, s, n, static_cast<uint16_t *>(dW));
    return after("allegro_grouped_matmul_backward");
  }
  if ((rc = check_ptr(offsets, "offsets", 8)) || (rows && (rc = check_ptr(rows, "rows", 4))) ||
      (rc = check_rows(dY, "dY", lddy, N, e)))
    return rc;
  const bool need_x = dW || act != ALLEGRO_ACT_NONE;
  if (need_x && (rc = check_rows(X, "X", ldx, K, e))) return rc;
  if (dX && ((rc = check_ptr(W, "W", e)) || (rc = check_rows(dX, "dX", lddx, K, e)))) return rc;
  WeightShape z{};
  if (dW) {
    z = weight_shape(dtype, M, K, N, G);
    if ((rc = check_workspace(workspace, workspace_bytes, size_t(z.slots) * size_t(z.slot) * sizeof(float)))) return rc;
  }
  // dX is written before dW reads X
  if ((rc = check_apart(dX, "dX", {dY, W, dW ? X : nullptr})) || (rc = check_apart(dW, "dW", {X, dY}))) return rc;
  if (dX) {
    // the same product with W transposed: the contraction runs along dY's columns
    const ProductArgs g{M, N, K, G, offsets, rows, dY, lddy, W, dX, lddx, act ? X : nullptr, ldx, 0, 0, 0, 0};
    if (dtype == ALLEGRO_F32)
      launch_product<float, true>(g, s);
    else
      launch_product<uint16_t, true>(g, s);
  }
  if (dW) {
    const WeightArgs g{M,  K,    N,  G,    act, 0, offsets, rows, X, ldx, dY, lddy, dW, static_cast<float *>(workspace),
                       0, 0, 0, 0};
    if (dtype == ALLEGRO_F32)
      launch_weight<float>(g, z, s);
    else
      launch_weight<uint16_t>(g, z, s);
  }
  return after("allegro_grouped_matmul_backward");
}

int allegro_grouped_matmul_fp8(int64_t M, int K, int N, int G, const int64_t *offsets, const int32_t *rows,
                               const void *X, int64_t ldx, const float *xs, const void *W, const float *ws, void *Y,
                               int64_t ldy, void *stream) {
  int rc;
  if ((rc = check_product(ALLEGRO_BF16, ALLEGRO_ACT_NONE, M, K, N, G))) return rc;
  if (!offsets && G != 1) return fail(ALLEGRO_E_INVALID, "offsets is NULL with G=%d groups", G);
  if (M == 0) return ALLEGRO_OK;
  if ((offsets && (rc = check_ptr(offsets, "offsets", 8))) || (rows && (rc = check_ptr(rows, "rows", 4))) ||
      (rc = check_rows(X, "X", ldx, K, 1)) || (rc = check_ptr(xs, "xs", 4)) || (rc = check_ptr(W, "W", 1)) ||
      (rc = check_ptr(ws, "ws", 4)) || (rc = check_rows(Y, "Y", ldy, N, 2)) || (rc = check_apart(Y, "Y", {X, xs, W, ws})))
    return rc;
  if (!offsets) rows = nullptr;  // one group, of all rows in their own order
  ProductF8Args g{M,  K,
                        N,  G,
                        offsets, rows,
                        static_cast<const uint8_t *>(X), ldx,
                        xs, static_cast<const uint8_t *>(W),
                        ws, static_cast<uint16_t *>(Y),
                        ldy, int(cdiv(N, N <= 64 ? 64 : 128)),
                        tile_bound(M, G, kTileRows), 0};
  hipStream_t s = static_cast<hipStream_t>(stream);
  // Tiles against rows past stationary weights, us, 1 and 64 types: K = 512, N = 512 M =
  // 32,000 23 against 28 and 28 against 29 (16 types), 64,000 41 against 39 and 48 against
  // 48, 128,000 76 against 60 and 83 against 69; 1024 x 1024 M = 32,000 66 against 56,
  // 128,000 295 against 191 and 309 against 225, and 349 against 321 with 225; 128,000 1024 x
  // 128 39 against 41 and 48 against 44, 256 x 128 19 against 21.5 and 24 against 23.
  const int64_t nt = cdiv(N, 128);
  if (N > 64 && K >= 16 && K <= kStreamF8K && M * nt >= 131072 && M >= 1024 * int64_t(G)) {
    g.nt = int(cdiv(N, 128));
    g.mt = std::max(1, kStreamGroups / g.nt);
    hipLaunchKernelGGL(product_f8_stream_kernel, dim3(unsigned(g.mt * g.nt)), dim3(kStreamThreads), 0, s, g);
    return after("allegro_grouped_matmul_fp8");
  }
  if (N <= 64)
    launch_tiles(product_f8_kernel<64>, g, g.mt * g.nt, kThreads, s);
  else
    launch_tiles(product_f8_kernel<128>, g, g.mt * g.nt, kThreads, s);
  return after("allegro_grouped_matmul_fp8");
}

}  // extern "C"
