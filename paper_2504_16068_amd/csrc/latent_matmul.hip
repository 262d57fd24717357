// MI355X (gfx950) kernels and C ABI of the products per type over ragged groups
// of rows (include/allegro_latent.h): forward, both gradients, and 8-bit operands.
//
//   product_kernel     Y[r] = act(X[r]) W[g], or with W transposed dX[r] =
//                      (dY[r] W[g]^T) act'(X[r]): 128 rows of one group by TN columns
//   weight_kernel      dW[g] = act(X)^T dY over a range of a group's rows
//   weight_sum_kernel  sums the ranges of the groups that have several, in order
//   product_f8_kernel  the 8-bit product
//
// Ragged groups.  The offsets are on the device, so the host launches an upper
// bound of tiles: group g's tiles start at index (offsets[g] >> shift) + g.  A
// group of n rows needs at most (n >> shift) + 2 tiles less whatever the next
// group's start rounds off, which is what that index leaves room for, so every
// workgroup finds its group by comparing its index with those of all groups,
// with no sums over groups and no launch before.  Rows without a type are one
// more group, of zeros.
//
// Operand layout.  Tiles lie in LDS as rows of 16-bit (or 8-bit) values along
// the contraction, 16-byte chunks XOR-swizzled by row so that 8 and 16 lanes on
// consecutive rows hit distinct banks.  The matrix instructions take W's columns
// as their rows: lane l then holds 4 consecutive columns of Y's row l % 16 per
// 16 x 16 product and stores them straight from registers; with 16-bit results
// two products' columns are interleaved (slot_of) to 8 consecutive ones.
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
constexpr int kTileRows = 128, kTileShift = 7;  // rows of a tile

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// SiLU and its derivative.  The hardware's exponential and reciprocal (1 ulp
// each) leave about 2e-7 of the value; the library's correctly rounded division
// costs ten more operations per element.
__device__ __forceinline__ float sigmoid(float a) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * a));
}
__device__ __forceinline__ float silu(float a) { return a * sigmoid(a); }
__device__ __forceinline__ float silu_grad(float a) {
  const float s = sigmoid(a);
  return s * (1.0f + a * (1.0f - s));
}

// ------------------------------------------------------ group of a tile
struct Tile {
  int g;                   // group, G for the rows without a type
  int64_t begin, m0, end;  // list positions: the group, the tile's first row; nothing to do if m0 >= end
};

__device__ __forceinline__ Tile find_tile(const int64_t *__restrict__ offsets, int G, int64_t M, int shift, int64_t t,
                                          int lane) {
  auto clamped = [&](int i) {
    const int64_t o = offsets[i];
    return o < 0 ? int64_t(0) : o > M ? M : o;
  };
  int below = 0;
  for (int i = lane; i <= G; i += kWave) below += (clamped(i) >> shift) + i <= t;
  for (int m = kWave / 2; m; m >>= 1) below += __shfl_xor(below, m);
  const int g = __builtin_amdgcn_readfirstlane(below > 0 ? below - 1 : 0);
  const int64_t begin = clamped(g), end = g < G ? clamped(g + 1) : M;
  const int64_t k = t - ((begin >> shift) + g);
  return {g, begin, k < 0 ? end : begin + (k << shift), end};
}

__host__ __device__ inline int64_t tile_bound(int64_t M, int G, int shift) { return (M >> shift) + G + 1; }

// Workgroups go round the 8 XCDs: give each XCD consecutive tiles, so that the
// tiles that share rows or weights share an L2.
__device__ __forceinline__ int64_t xcd_order(int64_t b, int64_t n) {
  const int64_t per = n >> 3, rest = n & 7, x = b & 7, i = b >> 3;
  return x * per + (x < rest ? x : rest) + i;
}

// --------------------------------------------------- operands in LDS
// fp32 operands are split into three bf16 parts each, x = h + m + l (8 bits of
// the significand in each, all exact), and of the nine products of the parts the
// six of weight 2^-16 and more are summed; the dropped ones are below 2^-26 of
// the product.  The bf16 matrix instructions take subnormals as zero, hence
// kScale, and round their sums down, hence every step's sum starts from zero and
// is added to the running one by the vector units, and every other row (or step)
// enters negated, so that what is left of the bias cancels over rows.  A sum that
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

// 16-byte chunk c of row r of plane p of a tile of R rows with C chunks to a row.
template <int C, int R>
__device__ __forceinline__ int chunk_at(int p, int r, int c) {
  const int f = C == 4 ? ((r >> 1) & 3) ^ ((r >> 3) & 1) : (r & 7) ^ ((r >> 3) & 1);
  return (p * R + r) * C + (c ^ f);
}

// LDS row of result column n: with 16-bit results, columns 8 q + 4 h + i of 32
// (i < 4, h < 2) lie at row 16 h + 4 q + i.
template <bool WIDE>
__device__ __forceinline__ int slot_of(int n) {
  return WIDE ? (n & ~31) | ((n >> 2) & 1) << 4 | ((n >> 3) & 3) << 2 | (n & 3) : n;
}

__device__ __forceinline__ void split2(float a, float b, uint32_t &h, uint32_t &m, uint32_t &l) {
  h = bf16_pair(a, b);
  const float ra = a - __builtin_bit_cast(float, h << 16), rb = b - __builtin_bit_cast(float, h & 0xffff0000u);
  m = bf16_pair(ra, rb);
  l = bf16_pair(ra - __builtin_bit_cast(float, m << 16), rb - __builtin_bit_cast(float, m & 0xffff0000u));
}

// Writes 8 consecutive contraction values of LDS row r (chunk c).
template <class T, int R>
__device__ __forceinline__ void put8(u32x4 *lds, int r, int c, const float (&v)[8], float scale) {
  constexpr int C = Kind<T>::KS / 8;
  if constexpr (sizeof(T) == 4) {
    u32x4 h, m, l;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t a, b, d;
      split2(scale * v[2 * i], scale * v[2 * i + 1], a, b, d);
      h[i] = a; m[i] = b; l[i] = d;
    }
    lds[chunk_at<C, R>(0, r, c)] = h;
    lds[chunk_at<C, R>(1, r, c)] = m;
    lds[chunk_at<C, R>(2, r, c)] = l;
  } else {
    u32x4 h;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    lds[chunk_at<C, R>(0, r, c)] = h;
  }
}

// A thread's share of the rows of a tile whose contraction runs along memory:
// 16-byte pieces tid % 8 of rows tid / 8 + 32 i.  Every load is issued, without a
// condition: a piece that crosses the end of its row (n elements) is loaded from
// n - PE on and shifted down in put(), in the last step alone.
template <class T, int ROWS>
struct Along {
  static constexpr int NP = ROWS / 32, PE = Kind<T>::PE, KS = Kind<T>::KS;
  u32x4 v[NP];
  // row(i): pointer to the first element of row tid / 8 + 32 i
  template <class Row>
  __device__ __forceinline__ void load(Row row, int k0, int n, int tid) {
    const int k = k0 + PE * (tid % 8);
    if (n >= PE) {
      const unsigned at = unsigned(k < n - PE ? k : n - PE);
#pragma unroll
      for (int i = 0; i < NP; ++i) v[i] = *reinterpret_cast<const u32x4_any *>(row(i) + at);
    } else {
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
  }
  // the elements from n on become zero
  __device__ __forceinline__ void cut(int k0, int n, int tid) {
    const int k = k0 + PE * (tid % 8), by = k < n - PE ? 0 : k - (n - PE);
    if (n < PE) return;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      u32x4 a = v[i];
      if constexpr (sizeof(T) == 2) {
        if (by & 1) a = u32x4{a[0] >> 16 | a[1] << 16, a[1] >> 16 | a[2] << 16, a[2] >> 16 | a[3] << 16, a[3] >> 16};
      }
      constexpr int E = 4 / int(sizeof(T));
      if (by & E) a = u32x4{a[1], a[2], a[3], 0};
      if (by & (2 * E)) a = u32x4{a[2], a[3], 0, 0};
      if (by >= PE) a = u32x4{0, 0, 0, 0};
      v[i] = a;
    }
  }
  // into LDS rows base + slot(tid / 8 + 32 i)
  template <int R, bool WIDE>
  __device__ __forceinline__ void put(u32x4 *lds, int base, bool act, float scale, int k0, int n, int tid) {
    constexpr int C = KS / 8;
    if (k0 + KS > n) cut(k0, n, tid);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = base + slot_of<WIDE>(tid / 8 + 32 * i);
      if constexpr (sizeof(T) == 4) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t bits = v[i][e];  // a bit cast of the vector's element itself gives element 0
          x[e] = __builtin_bit_cast(float, bits);
        }
        if (act) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = silu(x[e]);
        }
        uint32_t h[2], m[2], l[2];
        split2(scale * x[0], scale * x[1], h[0], m[0], l[0]);
        split2(scale * x[2], scale * x[3], h[1], m[1], l[1]);
        u32x2 *d = reinterpret_cast<u32x2 *>(lds) + tid % 2;
        d[2 * chunk_at<C, R>(0, r, tid % 8 / 2)] = u32x2{h[0], h[1]};
        d[2 * chunk_at<C, R>(1, r, tid % 8 / 2)] = u32x2{m[0], m[1]};
        d[2 * chunk_at<C, R>(2, r, tid % 8 / 2)] = u32x2{l[0], l[1]};
      } else {
        u32x4 o = v[i];
        if (act) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            o[e] = bf16_pair(silu(__builtin_bit_cast(float, o[e] << 16)),
                             silu(__builtin_bit_cast(float, o[e] & 0xffff0000u)));
        }
        lds[chunk_at<C, R>(0, r, tid % 8)] = o;
      }
    }
  }
};

// A thread's share of a tile whose contraction runs across memory rows: EPT
// consecutive steps of one column, or of 16-bit tiles 128 wide of two neighbouring
// ones.  The memory rows are the same for a whole wave, so their addresses are
// scalar.  Columns past the last one read the last: they reach no output.
template <class T, int COLS>
struct Across {
  static constexpr bool PAIR = sizeof(T) == 2 && COLS == 128;
  static constexpr int LANES = PAIR ? COLS / 2 : COLS, EPT = Kind<T>::KS * LANES / kThreads;
  static_assert(EPT % 8 == 0 && LANES % kWave == 0, "whole chunks, one part to a wave");
  static __device__ __forceinline__ int part(int tid) { return __builtin_amdgcn_readfirstlane(tid / LANES); }
  static __device__ __forceinline__ int col(int tid) { return tid % LANES * (PAIR ? 2 : 1); }
  uint32_t v[EPT];
  // row(i): pointer to element 0 of step part * EPT + i, the same for all lanes; c: the column, n of them
  template <class Row>
  __device__ __forceinline__ void load(Row row, int c, int n) {
    if (PAIR && n > 1) {
      const unsigned at = unsigned(c < n - 2 ? c : n - 2);
#pragma unroll
      for (int i = 0; i < EPT; ++i) v[i] = *reinterpret_cast<const u32_any *>(row(i) + at);
      if (n & 1) {  // the last column's pair holds it in its upper half
#pragma unroll
        for (int i = 0; i < EPT; ++i) v[i] = c == n - 1 ? v[i] >> 16 : v[i];
      }
    } else {
      const unsigned at = unsigned(c < n ? c : n - 1);
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        if constexpr (sizeof(T) == 4)
          v[i] = __builtin_bit_cast(uint32_t, row(i)[at]);
        else
          v[i] = row(i)[at];
      }
    }
  }
  // valid: bit i is set if step part * EPT + i exists; the others become zero
  template <int R, bool WIDE>
  __device__ __forceinline__ void put(u32x4 *lds, int base, bool act, float scale, uint32_t valid, int tid) {
    if (valid != (EPT == 32 ? ~0u : (1u << EPT) - 1)) {
#pragma unroll
      for (int i = 0; i < EPT; ++i) v[i] = valid >> i & 1 ? v[i] : 0u;
    }
    const int c0 = part(tid) * (EPT / 8);
#pragma unroll
    for (int q = 0; q < EPT / 8; ++q) {
#pragma unroll
      for (int s = 0; s < (PAIR ? 2 : 1); ++s) {
        const int r = base + slot_of<WIDE>(col(tid) + s);
        if constexpr (sizeof(T) == 2) {
          // 16-bit values are moved as they are, or through SiLU
          u32x4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t a = v[8 * q + 2 * e], b = v[8 * q + 2 * e + 1];
            o[e] = s ? __builtin_amdgcn_perm(b, a, 0x07060302) : __builtin_amdgcn_perm(b, a, 0x05040100);
          }
          if (act) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              o[e] = bf16_pair(silu(__builtin_bit_cast(float, o[e] << 16)),
                               silu(__builtin_bit_cast(float, o[e] & 0xffff0000u)));
          }
          lds[chunk_at<Kind<T>::KS / 8, R>(0, r, c0 + q)] = o;
        } else {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = __builtin_bit_cast(float, v[8 * q + e]);
          if (act) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = silu(x[e]);
          }
          put8<T, R>(lds, r, c0 + q, x, scale);
        }
      }
    }
  }
};

// Bits i < n of the steps first + i that are below end.
__device__ __forceinline__ uint32_t steps_below(int64_t first, int64_t end, int n) {
  const int64_t left = end - first;
  const uint32_t all = n == 32 ? ~0u : (1u << n) - 1;
  return left >= n ? all : left <= 0 ? 0u : (1u << left) - 1;
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// One contraction step of a wave: MI x NI products of 16 x 16.  The matrix
// instructions' rows are LDS rows row_n + 16 j + l % 16, their columns LDS rows
// row_m + 16 i + l % 16.  fp32 sums are added with the factor `sign`.
template <class T, int R, int MI, int NI>
__device__ __forceinline__ void multiply(const u32x4 *lds, int row_m, int row_n, float sign, f32x4 (&acc)[MI][NI],
                                         int l) {
  constexpr int P = Kind<T>::P, C = Kind<T>::KS / 8;
  auto frag = [&](int p, int r, int c) { return __builtin_bit_cast(bf16x8, lds[chunk_at<C, R>(p, r, c)]); };
#pragma unroll
  for (int kk = 0; kk < C / 4; ++kk) {
    const int c = 4 * kk + l / 16;
    bf16x8 b[MI][P];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int p = 0; p < P; ++p) b[i][p] = frag(p, row_m + 16 * i + l % 16, c);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      bf16x8 a[P];
#pragma unroll
      for (int p = 0; p < P; ++p) a[p] = frag(p, row_n + 16 * j + l % 16, c);
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
template <int W, class T>
__device__ __forceinline__ void load_row(const T *p, float *v, int left) {
  if (left >= W) {
    const u32x4 a = *reinterpret_cast<const u32x4_any *>(p);  // 16 bytes in both types
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t bits = a[i];
      if constexpr (sizeof(T) == 4) {
        v[i] = __builtin_bit_cast(float, bits);
      } else {
        v[2 * i] = __builtin_bit_cast(float, bits << 16);
        v[2 * i + 1] = __builtin_bit_cast(float, bits & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = i < left ? to_f32(p[i]) : 0.f;
  }
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
  for (int i = tid; i < kTileRows * n; i += kThreads) {
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
  const void *pre;  // y is multiplied with SiLU'(pre), if given ([M][N])
  int64_t ldp;
  int act;     // SiLU on x
  int nt;      // column tiles
  int64_t mt;  // upper bound of the row tiles
};

template <class T, int TN, bool WT>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(ProductArgs g) {
  constexpr int P = Kind<T>::P, KS = Kind<T>::KS, R = kTileRows + TN, C = KS / 8;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int MI = 4, NI = TN / 32;
  __shared__ u32x4 lds[P * R * C];
  __shared__ int srow[kTileRows];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), l = tid % kWave;
  const int64_t b = xcd_order(blockIdx.x, g.mt * g.nt);
  const Tile t = find_tile(g.offsets, g.G, g.M, kTileShift, b / g.nt, l);
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
  const T *xr[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = srow[tid / 8 + 32 * i];
    xr[i] = x + (r < 0 ? 0 : int64_t(r) * g.ldx);  // rows past the end are multiplied but not stored
  }
  using WLoad = std::conditional_t<WT, Along<T, TN>, Across<T, TN>>;
  Along<T, kTileRows> a;
  WLoad bw;
  int wr[TN / 32];  // W transposed: the rows' offsets from column n0's
  if constexpr (WT) {
    w += int64_t(n0) * K;
#pragma unroll
    for (int i = 0; i < TN / 32; ++i) {
      const int n = tid / 8 + 32 * i;
      wr[i] = (n < N - n0 ? n : N - n0 - 1) * K;
    }
  }
  auto load = [&](int k0) {
    a.load([&](int i) { return xr[i]; }, k0, K, tid);
    if constexpr (WT) {
      bw.load([&](int i) { return w + wr[i]; }, k0, K, tid);
    } else {
      const int kp = k0 + WLoad::part(tid) * WLoad::EPT;
      bw.load([&](int i) { return w + int64_t(kp + i < K ? kp + i : K - 1) * N + n0; }, WLoad::col(tid), N - n0);
    }
  };
  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int wm = 64 * (wave % 2), wn = TN / 2 * (wave / 2);
  const float xs = (tid / 8) % 2 ? -kScale : kScale;  // odd rows negated
  load(0);
  for (int k0 = 0; k0 < K; k0 += KS) {
    lds_sync<4>();  // the previous step has been read
    a.template put<R, false>(lds, 0, g.act, xs, k0, K, tid);
    if constexpr (WT)
      bw.template put<R, !F32>(lds, kTileRows, false, kScale, k0, K, tid);
    else
      bw.template put<R, !F32>(lds, kTileRows, false, kScale,
                               steps_below(k0 + WLoad::part(tid) * WLoad::EPT, K, WLoad::EPT), tid);
    lds_sync<4>();
    if (k0 + KS < K) load(k0 + KS);
    multiply<T, R, MI, NI>(lds, wm, kTileRows + wn, 1.f, acc, l);
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
            const int n = n0 + wn + 16 * j + l % 16;
            return n >= N ? 0.f : WT ? w[int64_t(n - n0) * K + k] : w[k * N + n];
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
      if (pre) {
        float p[W];
        load_row<W>(pre + int64_t(r) * g.ldp + n, p, N - n);
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] *= silu_grad(p[e]);
      }
      store_row<W>(y + int64_t(r) * g.ldy + n, v, N - n);
    }
  }
}

// ------------------------------------------------------- weight gradient
struct WeightArgs {
  int64_t M;
  int K, N, G, act, shift;  // ranges of 1 << shift rows
  const int64_t *offsets;
  const int32_t *rows;
  const void *x;  // [M][K]
  int64_t ldx;
  const void *dy;  // [M][N]
  int64_t lddy;
  void *dw;     // [G][K][N]
  float *part;  // [2 (M >> shift) + 1][slot]
  int64_t slot;
  int kt, nt;
  int64_t ranges;  // upper bound
};

// Range k of a group of several goes to slot 2 (offsets[g] >> shift) + k: such a
// group has more than 1 << shift rows, so the next one's slots start behind it.
template <class T, int TK, int TN>
__global__ __launch_bounds__(kThreads, 2) void weight_kernel(WeightArgs g) {
  constexpr int P = Kind<T>::P, KS = Kind<T>::KS, R = TK + TN, C = KS / 8;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int MI = TK / 32, NI = TN / 32;
  __shared__ u32x4 lds[P * R * C];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), l = tid % kWave;
  const int tiles = g.kt * g.nt;
  const int64_t b = xcd_order(blockIdx.x, g.ranges * tiles);
  const Tile t = find_tile(g.offsets, g.G, g.M, g.shift, b / tiles, l);
  if (t.g == g.G) return;
  const int64_t begin = t.begin;
  const bool only = t.end - begin <= (int64_t(1) << g.shift);  // the group's only range, if it has rows at all
  if (t.m0 >= t.end && !(t.m0 == begin && t.end == begin)) return;
  const int64_t end = t.m0 + (int64_t(1) << g.shift) < t.end ? t.m0 + (int64_t(1) << g.shift) : t.end;
  const int k0 = int(b % tiles) / g.nt * TK, n0 = int(b % tiles) % g.nt * TN, K = g.K, N = g.N;
  const T *x = static_cast<const T *>(g.x), *dy = static_cast<const T *>(g.dy);
  using XLoad = Across<T, TK>;
  using YLoad = Across<T, TN>;
  XLoad xa;
  YLoad ya;
  auto row_of = [&](int64_t i) -> int {
    if (i >= end) return -1;
    const int64_t r = g.rows ? int64_t(g.rows[i]) : i;
    return r < 0 || r >= g.M ? -1 : int(r);
  };
  // the rows of a step are the same for all lanes: lane i loads row i of the step
  // two ahead, the addresses are formed with its value in a scalar register
  const int xpart = XLoad::part(tid) * XLoad::EPT, ypart = YLoad::part(tid) * YLoad::EPT;
  auto load = [&](int rows) {
    const int r = rows < 0 ? 0 : rows;
    xa.load([&](int i) { return x + int64_t(__builtin_amdgcn_readlane(r, xpart + i)) * g.ldx + k0; }, XLoad::col(tid),
            K - k0);
    ya.load([&](int i) { return dy + int64_t(__builtin_amdgcn_readlane(r, ypart + i)) * g.lddy + n0; },
            YLoad::col(tid), N - n0);
  };
  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int wk = TK / 2 * (wave % 2), wn = TN / 2 * (wave / 2);
  float sign = 1.f;
  const int lk = l % KS;
  int rows = row_of(t.m0 + lk);
  uint64_t valid = __ballot(rows >= 0);
  if (t.m0 < end) load(rows);
  rows = row_of(t.m0 + KS + lk);
  for (int64_t m = t.m0; m < end; m += KS) {
    lds_sync<4>();
    xa.template put<R, false>(lds, 0, g.act, sign * kScale, uint32_t(valid >> xpart) & steps_below(0, KS, XLoad::EPT), tid);
    ya.template put<R, false>(lds, TK, false, kScale, uint32_t(valid >> ypart) & steps_below(0, KS, YLoad::EPT), tid);
    lds_sync<4>();
    valid = __ballot(rows >= 0);
    if (m + KS < end) {
      load(rows);
      rows = row_of(m + 2 * KS + lk);
    }
    multiply<T, R, MI, NI>(lds, wk, TK + wn, sign, acc, l);
    sign = -sign;
  }
  if constexpr (F32) {
    if (any_not_finite(acc)) {
      multiply_again(
          acc, end - t.m0, l,
          [&](int i, int64_t m) {
            const int64_t r = row_of(t.m0 + m);
            const int k = k0 + wk + 16 * i + l % 16;
            const float v = r < 0 || k >= K ? 0.f : x[r * g.ldx + k];
            return g.act ? silu(v) : v;
          },
          [&](int j, int64_t m) {
            const int64_t r = row_of(t.m0 + m);
            const int n = n0 + wn + 16 * j + l % 16;
            return r < 0 || n >= N ? 0.f : dy[r * g.lddy + n];
          });
    } else {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] *= kUnscale;
    }
  }
  const int64_t k_first = (t.m0 - begin) >> g.shift;
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
        store_row<4>(g.part + (2 * (begin >> g.shift) + k_first) * g.slot + int64_t(k) * N + n, v, N - n);
    }
  }
}

// Workgroup (e, y): elements 256 e .. of the y-th group that has several ranges.
constexpr int kSumThreads = 512;
template <class T>
__global__ __launch_bounds__(kSumThreads) void weight_sum_kernel(WeightArgs g) {
  __shared__ f32x4 sums[kSumThreads / kWave][kWave];
  const int tid = threadIdx.x, l = tid % kWave, wave = tid / kWave;
  auto clamped = [&](int i) {
    const int64_t o = g.offsets[i];
    return o < 0 ? int64_t(0) : o > g.M ? g.M : o;
  };
  int left = blockIdx.y, found = -1;
  for (int i0 = 0; i0 < g.G && found < 0; i0 += kWave) {
    const int i = i0 + l;
    const uint64_t several = __ballot(i < g.G && clamped(i + 1) - clamped(i) > (int64_t(1) << g.shift));
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
  const int ranges = int((rows + (int64_t(1) << g.shift) - 1) >> g.shift);
  const int64_t e = int64_t(blockIdx.x) * 256 + 4 * l;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (e < KN) {
    const float *p = g.part + 2 * (begin >> g.shift) * g.slot + e;  // slots are padded to whole vectors
#pragma unroll 4
    for (int k = wave; k < ranges; k += kSumThreads / kWave) s += *reinterpret_cast<const f32x4 *>(p + k * g.slot);
  }
  sums[wave][l] = s;
  __syncthreads();
  if (wave || e >= KN) return;
#pragma unroll
  for (int k = 1; k < kSumThreads / kWave; ++k) s += sums[k][l];
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
  const int64_t *offsets;  // null: one group of all rows
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
};

// A step is one block of 128 along K: one matrix instruction (16 x 16 x 128) forms
// the block's sums, which the vector units add with the two scales' product.  The
// instruction aligns each 8 products to the largest of them and drops what is
// below 2^-13 of it (measured; the 16 x 16 x 32 one does the same at half the
// rate), 2e-6 of the terms' magnitudes for normally distributed operands: far
// below the bf16 output's 2^-8, and the reason that there is no fp32 output.
template <int TN>
__global__ __launch_bounds__(kThreads, 2) void product_f8_kernel(ProductF8Args g) {
  constexpr int KS = 128, C = KS / 16, R = kTileRows + TN, MI = 4, NI = TN / 32;
  __shared__ u32x4 lds[R * C];
  __shared__ int srow[kTileRows];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), l = tid % kWave;
  const int64_t b = xcd_order(blockIdx.x, g.mt * g.nt);
  Tile t;
  if (g.offsets)
    t = find_tile(g.offsets, g.G, g.M, kTileShift, b / g.nt, l);
  else
    t = {0, 0, (b / g.nt) << kTileShift, g.M};
  if (t.m0 >= t.end) return;
  const int n0 = int(b % g.nt) * TN, K = g.K, N = g.N;
  uint16_t *y = g.y;
  list_rows(srow, g.offsets ? g.rows : nullptr, t, g.M, tid);
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
  auto cut = [&](u32x4 a, int k) {
    const int by = k < at_last ? 0 : k - at_last, bits = 8 * (by % 4);
    if (at_last < 0) return a;
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_alignbit(i < 3 ? a[i + 1] : 0u, a[i], bits);
    if (by & 4) o = u32x4{o[1], o[2], o[3], 0};
    if (by & 8) o = u32x4{o[2], o[3], 0, 0};
    if (by >= 16) o = u32x4{0, 0, 0, 0};
    return o;
  };
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
    for (int i = 0; i < 4; ++i) lds[chunk_at<C, R>(0, tid / 8 + 32 * i, tid % 8)] = a[i];
#pragma unroll
    for (int i = 0; i < NW; ++i) lds[chunk_at<C, R>(0, kTileRows + slot_of<true>(tid / 8 + 32 * i), tid % 8)] = bw[i];
    lds_sync<4>();
    float sc[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) sc[i] = sx[i] * sw;
    if (k0 + KS < K) load(k0 + KS);
    // lane l takes chunks l / 16 and l / 16 + 4 of both operands
    auto frag = [&](int r) {
      const u32x4 lo = lds[chunk_at<C, R>(0, r, l / 16)], hi = lds[chunk_at<C, R>(0, r, l / 16 + 4)];
      return i32x8{int(lo[0]), int(lo[1]), int(lo[2]), int(lo[3]), int(hi[0]), int(hi[1]), int(hi[2]), int(hi[3])};
    };
    i32x8 xf[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) xf[i] = frag(wm + 16 * i + l % 16);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const i32x8 wf = frag(kTileRows + wn + 16 * j + l % 16);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        // both block scales of the instruction are 2^(127 - 127)
        const f32x4 s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, xf[i], zero, 0, 0, 0, 0x7f7f7f7f, 0,
                                                                         0x7f7f7f7f);
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

// ------------------------------------------------------------- launches
template <class T, bool WT>
void launch_product(ProductArgs g, hipStream_t s) {
  const bool narrow = g.N <= 64;
  g.nt = narrow ? 1 : int(cdiv(g.N, 128));
  g.mt = tile_bound(g.M, g.G, kTileShift);
  const dim3 grid(unsigned(g.mt * g.nt)), block(kThreads);
  if (narrow)
    hipLaunchKernelGGL((product_kernel<T, 64, WT>), grid, block, 0, s, g);
  else
    hipLaunchKernelGGL((product_kernel<T, 128, WT>), grid, block, 0, s, g);
}

struct WeightShape {
  int shift, kt, nt;
  int64_t slot, slots;
};
WeightShape weight_shape(int64_t M, int K, int N) {
  WeightShape z;
  z.kt = int(K <= 64 ? 1 : cdiv(K, 128));
  z.nt = int(N <= 64 ? 1 : cdiv(N, 128));
  // about 768 workgroups, ranges of at least 256 rows
  const int64_t rows = M * z.kt * z.nt / 768;
  z.shift = 8;
  while ((int64_t(1) << z.shift) < rows && z.shift < 30) ++z.shift;
  z.slot = cdiv(int64_t(K) * N, 4) * 4;
  z.slots = M > (int64_t(1) << z.shift) ? 2 * (M >> z.shift) + 1 : 0;
  return z;
}

template <class T>
void launch_weight(WeightArgs g, const WeightShape &z, hipStream_t s) {
  g.shift = z.shift;
  g.kt = z.kt;
  g.nt = z.nt;
  g.slot = z.slot;
  g.ranges = tile_bound(g.M, g.G, z.shift);
  const dim3 grid(unsigned(g.ranges * g.kt * g.nt)), block(kThreads);
  if (g.K <= 64 && g.N <= 64)
    hipLaunchKernelGGL((weight_kernel<T, 64, 64>), grid, block, 0, s, g);
  else if (g.K <= 64)
    hipLaunchKernelGGL((weight_kernel<T, 64, 128>), grid, block, 0, s, g);
  else if (g.N <= 64)
    hipLaunchKernelGGL((weight_kernel<T, 128, 64>), grid, block, 0, s, g);
  else
    hipLaunchKernelGGL((weight_kernel<T, 128, 128>), grid, block, 0, s, g);
  if (z.slots) {
    const unsigned several = unsigned(std::min<int64_t>(g.G, g.M >> z.shift));
    hipLaunchKernelGGL((weight_sum_kernel<T>), dim3(unsigned(cdiv(int64_t(g.K) * g.N, 256)), several),
                       dim3(kSumThreads), 0, s, g);
  }
}

int check_product(int dtype, int act, int64_t M, int K, int N, int G) {
  int rc;
  if ((rc = check_dtype(dtype))) return rc;
  if (act != ALLEGRO_ACT_NONE && act != ALLEGRO_ACT_SILU) return fail(ALLEGRO_E_INVALID, "unknown act %d", act);
  if ((rc = check_m(M)) || (rc = check_width(K, "K")) || (rc = check_width(N, "N")) || (rc = check_g(G))) return rc;
  // one workgroup per 128 x 128 tile, at most 2^31 - 1 of them
  if (cdiv(std::max(K, N), 64) * tile_bound(M, G, kTileShift) > kMaxRows)
    return fail(ALLEGRO_E_UNSUPPORTED, "M=%lld rows of %d columns are more tiles than one launch takes", (long long)M,
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
      (rc = check_rows(X, "X", ldx, K, e)) || (rc = check_ptr(W, "W", e)) || (rc = check_rows(Y, "Y", ldy, N, e)))
    return rc;
  const ProductArgs g{M, K, N, G, offsets, rows, X, ldx, W, Y, ldy, nullptr, 0, act, 0, 0};
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
  const WeightShape z = weight_shape(M, K, N);
  *bytes = size_t(z.slots) * size_t(z.slot) * sizeof(float);
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
    z = weight_shape(M, K, N);
    if ((rc = check_workspace(workspace, workspace_bytes, size_t(z.slots) * size_t(z.slot) * sizeof(float)))) return rc;
  }
  if (dX) {
    // the same product with W transposed: the contraction runs along dY's columns
    const ProductArgs g{M, N, K, G, offsets, rows, dY, lddy, W, dX, lddx, act ? X : nullptr, ldx, 0, 0, 0};
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
      (rc = check_ptr(ws, "ws", 4)) || (rc = check_rows(Y, "Y", ldy, N, 2)))
    return rc;
  const ProductF8Args g{M,  K,
                        N,  G,
                        offsets, rows,
                        static_cast<const uint8_t *>(X), ldx,
                        xs, static_cast<const uint8_t *>(W),
                        ws, static_cast<uint16_t *>(Y),
                        ldy, int(cdiv(N, N <= 64 ? 64 : 128)),
                        tile_bound(M, G, kTileShift)};
  const dim3 grid(unsigned(g.mt * g.nt)), block(kThreads);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (N <= 64)
    hipLaunchKernelGGL((product_f8_kernel<64>), grid, block, 0, s, g);
  else
    hipLaunchKernelGGL((product_f8_kernel<128>), grid, block, 0, s, g);
  return after("allegro_grouped_matmul_fp8");
}

}  // extern "C"
