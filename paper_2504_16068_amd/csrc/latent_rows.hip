// MI355X (gfx950) kernels and C ABI of the latent track's row operators
// (include/allegro_latent.h): rows grouped by type, and the root-mean-square
// norm with the residual's addition, forward, in 8 bits and backward.
//
//   group_one_kernel      rows of one chunk: histogram, scan and placement in LDS
//   group_count_kernel    per chunk of rows, how many of each type
//   group_scan_kernel     per type, the exclusive sums of those counts over chunks
//   group_place_kernel    offsets, and every row at its place
//   norm_forward_kernel   rows in registers, 1 .. 64 lanes to a row
//   norm_backward_kernel  the same, with the columns' sums of dw kept in registers
//   norm_wide_*_kernel    one workgroup per row, any width
//   column_sum_kernel     fixed-order sum of the workgroups' dw
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "device_common.hpp"
#include "latent_common.hpp"

namespace {

using namespace latent;

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// ------------------------------------------------------------- grouping
// A stable counting sort in chunks of rows.  Every wave owns a consecutive part
// of its workgroup's chunk; a row's place is the sum of the rows of smaller
// types, those of its type in earlier chunks, in earlier waves of the chunk, in
// earlier steps of the wave, and in lower lanes of its step.  Nothing depends on
// an order of arrival.
//
// 8 bytes a row (1.05M rows: 8.4 MB, 1.8 us at the copy rate) in three dependent
// launches, two for few chunks, one for a single one.  Measured, 1,048,820 rows of
// 225 types: 3.5 us for the counts and 4.5 for their sums, both latency, and 10.9 for
// the places: 8 waves a compute unit, whose lanes store 4 bytes each to runs of 9
// rows.  Chunks of 4096 or 8192 rows with as many more waves, and neighbouring
// chunks on one XCD, took as long or longer.
constexpr int kOneChunk = 4096;  // rows that one workgroup takes alone

__host__ __device__ inline int64_t chunk_rows(int64_t M) {  // at most 1024 chunks
  const int64_t c = (M + 1023) / 1024;
  return c <= 2048 ? 2048 : (c + 2047) / 2048 * 2048;
}

__device__ __forceinline__ int key_of(const int32_t *type, int64_t r, int G) {
  const int t = type[r];
  return unsigned(t) < unsigned(G) ? t : G;  // no type: after all groups
}

// Lanes of the wave (among `active`) whose key equals this lane's, over the
// `bits` low bits of the keys.
__device__ __forceinline__ uint64_t same_key(int key, int bits, uint64_t active) {
  uint64_t peers = active;
  for (int b = 0; b < bits; ++b) {
    const bool set = (key >> b) & 1;
    const uint64_t m = __ballot(set);
    peers &= set ? m : ~m;
  }
  return peers;
}

// Adds the keys of rows lo .. hi - 1 to count (the wave's own LDS counters).
__device__ __forceinline__ void count_rows(const int32_t *type, int64_t lo, int64_t hi, int G, int *count, int lane) {
  for (int64_t r = lo + lane; r < hi; r += kWave) atomicAdd(&count[key_of(type, r, G)], 1);
}

// Writes rows lo .. hi - 1 (the wave's part) to their places; next[key] is the
// next free place of each key, advanced in the order of the rows.
__device__ __forceinline__ void place_rows(const int32_t *type, int64_t lo, int64_t hi, int G, int bits, int *next,
                                           int32_t *rows, int lane) {
  for (int64_t r0 = lo; r0 < hi; r0 += kWave) {
    const int64_t r = r0 + lane;
    const bool on = r < hi;
    const int key = on ? key_of(type, r, G) : 0;
    const uint64_t peers = same_key(key, bits, __ballot(on));
    const int before = __popcll(peers & ((uint64_t(1) << lane) - 1));
    const int base = on ? next[key] : 0;
    allegro_dev::lds_sync<1>();  // every lane has read its counter
    if (on) {
      if (before == 0) next[key] = base + __popcll(peers);
      rows[base + before] = int32_t(r);
    }
    allegro_dev::lds_sync<1>();
  }
}

// Exclusive sum over the workgroup's threads of one value each; total gets the sum.
__device__ __forceinline__ int block_exclusive(int v, int *tmp, int &total, int tid) {
  const int lane = tid % kWave, wave = tid / kWave;
  int inc = v;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int o = __shfl_up(inc, d);
    if (lane >= d) inc += o;
  }
  if (lane == kWave - 1) tmp[wave] = inc;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += tmp[w];
    total += tmp[w];
  }
  __syncthreads();
  return before + inc - v;
}

__device__ __forceinline__ void part_of(int64_t n, int wave, int64_t &lo, int64_t &hi) {
  const int64_t per = ((n + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
  lo = per * wave < n ? per * wave : n;
  hi = lo + per < n ? lo + per : n;
}

// All rows in one workgroup (M <= kOneChunk).
__global__ __launch_bounds__(kThreads) void group_one_kernel(int M, int G, int bits, const int32_t *__restrict__ type,
                                                             int64_t *__restrict__ offsets,
                                                             int32_t *__restrict__ rows) {
  __shared__ int count[kWaves][kMaxGroups + 1];
  __shared__ int tmp[kWaves];
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  for (int i = tid; i < kWaves * (kMaxGroups + 1); i += kThreads) (&count[0][0])[i] = 0;
  __syncthreads();
  int64_t lo, hi;
  part_of(M, wave, lo, hi);
  count_rows(type, lo, hi, G, count[wave], lane);
  __syncthreads();
  int base = 0;
  for (int g0 = 0; g0 <= G; g0 += kThreads) {
    const int g = g0 + tid;
    int sum = 0, total;
    if (g <= G)
      for (int w = 0; w < kWaves; ++w) sum += count[w][g];
    int at = base + block_exclusive(sum, tmp, total, tid);
    if (g <= G) {
      offsets[g] = at;  // g == G: the rows that have a type
      for (int w = 0; w < kWaves; ++w) {
        const int c = count[w][g];
        count[w][g] = at;
        at += c;
      }
    }
    base += total;
  }
  __syncthreads();
  place_rows(type, lo, hi, G, bits, count[wave], rows, lane);
}

__global__ __launch_bounds__(kThreads) void group_count_kernel(int64_t M, int G, int64_t chunk,
                                                               const int32_t *__restrict__ type,
                                                               int *__restrict__ hist) {
  __shared__ int count[kMaxGroups + 1];
  const int tid = threadIdx.x;
  for (int i = tid; i <= G; i += kThreads) count[i] = 0;
  __syncthreads();
  const int64_t lo = chunk * blockIdx.x, hi = lo + chunk < M ? lo + chunk : M;
  for (int64_t r = lo + tid; r < hi; r += kThreads) atomicAdd(&count[key_of(type, r, G)], 1);
  __syncthreads();
  for (int i = tid; i <= G; i += kThreads) hist[int64_t(blockIdx.x) * (G + 1) + i] = count[i];
}

// A workgroup has 16 types; its 64 threads for each share the (at most 1024)
// chunks.  hist[.][g] becomes its exclusive sums over the chunks, total[g] the whole.
constexpr int kScanTypes = 16, kScanParts = 64;
__global__ __launch_bounds__(kScanTypes *kScanParts) void group_scan_kernel(int chunks, int G, int *__restrict__ hist,
                                                                          int *__restrict__ total) {
  __shared__ int sums[kScanParts][kScanTypes];
  const int i = threadIdx.x % kScanTypes, part = threadIdx.x / kScanTypes, g = blockIdx.x * kScanTypes + i;
  constexpr int PER = 1024 / kScanParts;
  const int per = (chunks + kScanParts - 1) / kScanParts, lo = part * per;
  const int n = g > G || lo >= chunks ? 0 : lo + per < chunks ? per : chunks - lo;
  int v[PER], sum = 0;
#pragma unroll
  for (int c = 0; c < PER; ++c) v[c] = c < n ? hist[int64_t(lo + c) * (G + 1) + g] : 0;
#pragma unroll
  for (int c = 0; c < PER; ++c) sum += v[c];
  sums[part][i] = sum;
  __syncthreads();
  int at = 0;
#pragma unroll 8
  for (int p = 0; p < part; ++p) at += sums[p][i];
#pragma unroll
  for (int c = 0; c < PER; ++c) {
    if (c < n) hist[int64_t(lo + c) * (G + 1) + g] = at;
    at += v[c];
  }
  if (part == kScanParts - 1 && g <= G) total[g] = at;
}

// A chunk goes through in parts of kPart rows, each wave with consecutive rows: a
// row's rank among its wave's rows of its type, then the places of each wave's
// first row of each type, then the rows to their places.
// SUMS: hist holds the chunks' counts themselves, and every workgroup adds them up.
constexpr int kPart = 2048, kPartSteps = kPart / kThreads;
template <bool SUMS>
__global__ __launch_bounds__(kThreads) void group_place_kernel(int64_t M, int G, int bits, int64_t chunk,
                                                               const int32_t *__restrict__ type,
                                                               const int *__restrict__ hist,
                                                               const int *__restrict__ total,
                                                               int64_t *__restrict__ offsets,
                                                               int32_t *__restrict__ rows) {
  __shared__ int count[kWaves][kMaxGroups + 1], first[kMaxGroups + 1];
  __shared__ int tmp[kWaves];
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  const int64_t c0 = chunk * blockIdx.x, c1 = c0 + chunk < M ? c0 + chunk : M;
  int key[kPartSteps], rank[kPartSteps];
  auto load_keys = [&](int64_t part) {
    const int64_t r0 = part + wave * (kPart / kWaves) + lane;
#pragma unroll
    for (int s = 0; s < kPartSteps; ++s) key[s] = r0 + s * kWave < c1 ? key_of(type, r0 + s * kWave, G) : -1;
  };
  load_keys(c0);
  int sum = 0;
  for (int g0 = 0; g0 <= G; g0 += kThreads) {
    const int g = g0 + tid;
    int here = 0, whole = 0, all;  // rows of type g in earlier chunks, in all of them
    if (g <= G) {
      if constexpr (SUMS) {
#pragma unroll 16
        for (int c = 0; c < int(gridDim.x); ++c) {
          const int n = hist[int64_t(c) * (G + 1) + g];
          whole += n;
          here += c < int(blockIdx.x) ? n : 0;
        }
      } else {
        here = hist[int64_t(blockIdx.x) * (G + 1) + g];
        whole = total[g];
      }
    }
    const int at = sum + block_exclusive(whole, tmp, all, tid);
    if (g <= G) {
      if (blockIdx.x == 0) offsets[g] = at;
      first[g] = at + here;
    }
    sum += all;
  }
  for (int64_t part = c0; part < c1; part += kPart) {
    for (int w = 0; w < kWaves; ++w)
      for (int i = tid; i <= G; i += kThreads) count[w][i] = 0;
    __syncthreads();
    const int64_t r0 = part + wave * (kPart / kWaves) + lane;
    uint64_t peers[kPartSteps];
#pragma unroll
    for (int s = 0; s < kPartSteps; ++s) peers[s] = same_key(key[s], bits, __ballot(key[s] >= 0));
#pragma unroll
    for (int s = 0; s < kPartSteps; ++s) {
      const bool on = key[s] >= 0;
      const int before = __popcll(peers[s] & ((uint64_t(1) << lane) - 1));
      const int base = on ? count[wave][key[s]] : 0;
      allegro_dev::lds_sync<1>();  // every lane has read its counter
      if (on && before == 0) count[wave][key[s]] = base + __popcll(peers[s]);
      allegro_dev::lds_sync<1>();
      rank[s] = base + before;
    }
    __syncthreads();
    for (int g = tid; g <= G; g += kThreads) {
      int at = first[g];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const int n = count[w][g];
        count[w][g] = at;
        at += n;
      }
      first[g] = at;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kPartSteps; ++s)
      if (key[s] >= 0) rows[count[wave][key[s]] + rank[s]] = int32_t(r0 + s * kWave);
    if (part + kPart < c1) load_keys(part + kPart);
    __syncthreads();
  }
}

__global__ void zero_kernel(int64_t n, float *p) {
  const int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

// ----------------------------------------------------------------- norm
// A row lies in the registers of `lanes` lanes (a power of two, 1 .. 64): lane t of
// them holds vector j * lanes + t, j < NV, of VW elements each.  VW is 16 bytes'
// worth, at any alignment of the rows, or 1 for rows shorter than that.  The last
// vector of a row may cross its end: it is loaded from C - VW on and shifted.
template <class T, int VW>
struct Vec {
  u32x4 bits;
  // elements c .. of a row of C (c below C)
  __device__ __forceinline__ void load(const T *row, int c, int C) {
    if constexpr (VW == 1) {
      if constexpr (sizeof(T) == 4)
        bits[0] = __builtin_bit_cast(uint32_t, row[c]);
      else
        bits[0] = row[c];
    } else {
      const u32x4_any *p = reinterpret_cast<const u32x4_any *>(row + (c < C - VW ? c : C - VW));
      bits = __builtin_nontemporal_load(p);
    }
  }
  // their values, zero from C on
  __device__ __forceinline__ void values(int c, int C, float (&v)[VW]) const {
    if constexpr (VW == 1) {
      const uint32_t b = bits[0];
      v[0] = __builtin_bit_cast(float, sizeof(T) == 4 ? b : b << 16);
    } else {
      u32x4 a = bits;
      if (C % VW) {
        const int by = c < C - VW ? 0 : c - (C - VW);
        if constexpr (sizeof(T) == 2) {
          if (by & 1) a = u32x4{a[0] >> 16 | a[1] << 16, a[1] >> 16 | a[2] << 16, a[2] >> 16 | a[3] << 16, a[3] >> 16};
        }
        constexpr int E = 4 / int(sizeof(T));
        if (by & E) a = u32x4{a[1], a[2], a[3], 0};
        if (by & (2 * E)) a = u32x4{a[2], a[3], 0, 0};
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t b = a[i];
        if constexpr (sizeof(T) == 4) {
          v[i] = __builtin_bit_cast(float, b);
        } else {
          v[2 * i] = __builtin_bit_cast(float, b << 16);
          v[2 * i + 1] = __builtin_bit_cast(float, b & 0xffff0000u);
        }
      }
    }
  }
  static __device__ __forceinline__ void store(T *row, int c, int C, const float (&v)[VW]) {
    if (VW == 1 || c + VW > C) {
#pragma unroll
      for (int i = 0; i < VW; ++i)
        if (c + i < C) row[c + i] = from_f32<T>(v[i]);
    } else if constexpr (VW > 1) {
      u32x4 a;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4)
          a[i] = __builtin_bit_cast(uint32_t, v[i]);
        else
          a[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
      }
      __builtin_nontemporal_store(a, reinterpret_cast<u32x4_any *>(row + c));
    }
  }
};

constexpr int kBlock = 128;              // columns that share a scale
constexpr float kF8Max = 448.f, kF8MinScale = 0x1p-126f;

__device__ __forceinline__ uint32_t f8_pair(float a, float b) {  // low 16 bits
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false)) & 0xffffu;
}

// Elements c .. of y times inv as 8-bit values of a row of C.
template <int VW>
__device__ __forceinline__ void store_f8(uint8_t *row, int c, int C, const float (&y)[VW], float inv) {
  typedef uint32_t u32_byte __attribute__((aligned(1)));
  uint32_t w[VW == 1 ? 1 : VW / 4];
  if constexpr (VW == 1) {
    w[0] = f8_pair(y[0] * inv, 0.f);
  } else {
#pragma unroll
    for (int i = 0; i < VW / 4; ++i)
      w[i] = f8_pair(y[4 * i] * inv, y[4 * i + 1] * inv) | f8_pair(y[4 * i + 2] * inv, y[4 * i + 3] * inv) << 16;
  }
  if (VW == 1 || c + VW > C) {
#pragma unroll
    for (int i = 0; i < VW; ++i)
      if (c + i < C) row[c + i] = uint8_t(w[i / 4] >> (8 * (i % 4)));
  } else {
#pragma unroll
    for (int i = 0; i < VW / 4; ++i) *reinterpret_cast<u32_byte *>(row + c + 4 * i) = w[i];
  }
}

// The largest magnitude as bits: ordered as unsigned numbers, with NaN above infinity.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

__device__ __forceinline__ float f8_scale(uint32_t amax) {
  const float s = __builtin_bit_cast(float, amax) / kF8Max;
  return s < kF8MinScale ? kF8MinScale : s;  // NaN stays
}

template <class V>
__device__ __forceinline__ V lanes_sum(V v, int lanes) {
  for (int m = lanes / 2; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, int lanes) {
  for (int m = lanes / 2; m; m >>= 1) {
    const uint32_t o = __shfl_xor(v, m);
    v = o > v ? o : v;
  }
  return v;
}

struct NormArgs {
  int64_t M;
  int C, lanes;
  float eps;
  const void *x, *residual;
  const float *w;
  void *total, *y;  // y: dtype, or 8 bits
  float *rstd, *scale;
  int64_t ldx, ldr, ldt, ldy;
};

// One pass: a row's sum of squares is formed across the lanes that hold it, then the
// row is scaled, rounded and written from registers (so total may be x or residual).  Bound by memory (smallest and median of
// 30, under a kernel trace): 1,048,820 rows of 128 fp32 with residual and total 349 to 359 us
// (2.15 GB, 6.1 TB/s), 523,599 of 256 bf16 to 8 bits 168 to 179 us (0.95 GB, 5.6 TB/s), 20,001
// of 1031 bf16 43 us (165 MB, 3.8 TB/s: rows of odd width end within vectors, and 20,001
// rows are five rounds of a workgroup).

// Rows that a lane has in flight: as many as 16 floats (forward) hold.
template <int VW, int NV, int FLOATS>
constexpr int norm_rows() {
  return VW * NV * 4 <= FLOATS ? 4 : VW * NV * 2 <= FLOATS ? 2 : 1;
}

template <class T, int VW, int NV, bool F8>
__global__ __launch_bounds__(kThreads) void norm_forward_kernel(NormArgs g) {
  constexpr int R = norm_rows<VW, NV, 16>();
  const int lanes = g.lanes, tid = threadIdx.x, t = tid & (lanes - 1);
  const int per = kThreads / lanes;  // rows of a workgroup at a time, R times
  const int C = g.C;
  const T *x = static_cast<const T *>(g.x), *res = static_cast<const T *>(g.residual);
  T *total = static_cast<T *>(g.total);
  const float inv_c = 1.0f / float(C);
  float w[NV][VW];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * lanes + t) * VW;
#pragma unroll
    for (int i = 0; i < VW; ++i) w[j][i] = c + i < C ? g.w[c + i] : 0.f;
  }
  // every lane of a wave goes through the same rows' steps, so that the shuffles have all of them
  const int64_t step = int64_t(gridDim.x) * per * R;
  for (int64_t r0 = int64_t(blockIdx.x) * per * R; r0 < g.M; r0 += step) {
    float s[R][NV][VW], sq[R];
    Vec<T, VW> xv[R][NV], rv[R][NV];
    int64_t r[R];
    bool on[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      r[k] = r0 + k * per + tid / lanes;
      on[k] = r[k] < g.M;
      const T *row = x + (on[k] ? r[k] : 0) * g.ldx;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * lanes + t) * VW;
        xv[k][j].load(row, c < C ? c : 0, C);
      }
    }
    if (res) {
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const T *row = res + (on[k] ? r[k] : 0) * g.ldr;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int c = (j * lanes + t) * VW;
          rv[k][j].load(row, c < C ? c : 0, C);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * lanes + t) * VW;
        xv[k][j].values(c, C, s[k][j]);
        if (res) {
          float a[VW];
          rv[k][j].values(c, C, a);
#pragma unroll
          for (int i = 0; i < VW; ++i) s[k][j][i] += a[i];
        }
        if (!on[k] || c >= C) {
#pragma unroll
          for (int i = 0; i < VW; ++i) s[k][j][i] = 0.f;
        }
      }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      sq[k] = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VW; ++i) sq[k] = __builtin_fmaf(s[k][j][i], s[k][j][i], sq[k]);
    }
    for (int m = lanes / 2; m; m >>= 1)
#pragma unroll
      for (int k = 0; k < R; ++k) sq[k] += __shfl_xor(sq[k], m);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const float rstd = 1.0f / sqrtf(sq[k] * inv_c + g.eps);
      if (on[k] && g.rstd && t == 0) g.rstd[r[k]] = rstd;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * lanes + t) * VW;
        if (on[k] && c < C && total) Vec<T, VW>::store(total + r[k] * g.ldt, c, C, s[k][j]);
#pragma unroll
        for (int i = 0; i < VW; ++i) s[k][j][i] = s[k][j][i] * rstd * w[j][i];
        if constexpr (!F8) {
          if (on[k] && c < C) Vec<T, VW>::store(static_cast<T *>(g.y) + r[k] * g.ldy, c, C, s[k][j]);
        }
      }
      if constexpr (F8) {
        // a block of 128 columns is 128 / VW lanes of one vector, or the whole row
        const int bl = lanes < kBlock / VW ? lanes : kBlock / VW;
        const int blocks = (C + kBlock - 1) / kBlock;
        uint8_t *q = static_cast<uint8_t *>(g.y) + r[k] * g.ldy;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          uint32_t m = 0;
#pragma unroll
          for (int i = 0; i < VW; ++i) {
            const uint32_t b = abs_bits(s[k][j][i]);  // zero past the last column
            m = b > m ? b : m;
          }
          m = lanes_max(m, bl);
          const float sc = f8_scale(m), inv = 1.0f / sc;
          const int c = (j * lanes + t) * VW, b = c / kBlock;
          if (on[k] && (t & (bl - 1)) == 0 && b < blocks) g.scale[r[k] * blocks + b] = sc;
          if (on[k] && c < C) store_f8<VW>(q, c, C, s[k][j], inv);
        }
      }
    }
  }
}

__device__ __forceinline__ float block_sum(float v, float *tmp, int tid) {
  v = lanes_sum(v, kWave);
  __syncthreads();
  if (tid % kWave == 0) tmp[tid / kWave] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += tmp[w];
  return s;
}

// One workgroup per row, which it reads twice (the second time from the caches):
// widths that registers do not hold.  total is written in the second pass, by the
// thread that reads the element for the last time: it may be x or residual itself.
// Elements are read one to a lane: 20,000 rows of 8192 fp32 751 us (3.5 TB/s), bf16 560
// (2.3); backward 1,346 (1.9) and 1,205 (1.1).
template <class T, bool F8>
__global__ __launch_bounds__(kThreads) void norm_wide_forward_kernel(NormArgs g) {
  __shared__ float tmp[kWaves];
  const int tid = threadIdx.x, C = g.C;
  for (int64_t r = blockIdx.x; r < g.M; r += gridDim.x) {
    const T *x = static_cast<const T *>(g.x) + r * g.ldx;
    const T *res = g.residual ? static_cast<const T *>(g.residual) + r * g.ldr : nullptr;
    T *total = g.total ? static_cast<T *>(g.total) + r * g.ldt : nullptr;
    float sq = 0.f;
    for (int c = tid; c < C; c += kThreads) {
      const float s = to_f32(x[c]) + (res ? to_f32(res[c]) : 0.f);
      sq = __builtin_fmaf(s, s, sq);
    }
    const float rstd = 1.0f / sqrtf(block_sum(sq, tmp, tid) * (1.0f / float(C)) + g.eps);
    if (g.rstd && tid == 0) g.rstd[r] = rstd;
    if constexpr (!F8) {
      T *y = static_cast<T *>(g.y) + r * g.ldy;
      for (int c = tid; c < C; c += kThreads) {
        const float s = to_f32(x[c]) + (res ? to_f32(res[c]) : 0.f);
        if (total) total[c] = from_f32<T>(s);
        y[c] = from_f32<T>(s * rstd * g.w[c]);
      }
    } else {
      uint8_t *q = static_cast<uint8_t *>(g.y) + r * g.ldy;
      const int blocks = (C + kBlock - 1) / kBlock, lane = tid % kWave;
      for (int b = tid / kWave; b < blocks; b += kWaves) {  // a wave per block, two columns per lane
        float y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int c = b * kBlock + i * kWave + lane;
          y[i] = 0.f;
          if (c < C) {
            const float s = to_f32(x[c]) + (res ? to_f32(res[c]) : 0.f);
            if (total) total[c] = from_f32<T>(s);
            y[i] = s * rstd * g.w[c];
          }
        }
        const uint32_t m0 = abs_bits(y[0]), m1 = abs_bits(y[1]);
        const float sc = f8_scale(lanes_max(m0 > m1 ? m0 : m1, kWave)), inv = 1.0f / sc;
        if (lane == 0) g.scale[r * blocks + b] = sc;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int c = b * kBlock + i * kWave + lane;
          if (c < C) q[c] = uint8_t(f8_pair(y[i] * inv, 0.f));
        }
      }
    }
  }
}

struct NormBackArgs {
  int64_t M;
  int C, lanes;
  const void *total, *dy, *dtotal;
  const float *w, *rstd;
  void *dx;
  float *part;  // [gridDim.x][C]
  int64_t ldt, lddy, lddt, lddx;
};

// dx of a row and its terms of dw in one pass; a lane sums the dw terms of its
// columns over the rows it visits (a fixed stride), the row groups of a
// workgroup are then added in order, and the workgroups by column_sum_kernel.
// Bound by memory: 1,048,820 rows of 128 fp32 366 to 375 us (2.15 GB, 5.9 TB/s), 20,001 of
// 1031 bf16 38 us (165 MB, 4.3 TB/s); the sums 4 to 5 us.
template <class T, int VW, int NV>
__global__ __launch_bounds__(kThreads) void norm_backward_kernel(NormBackArgs g) {
  constexpr int kCols = kWave * NV * VW;  // at most: lanes * NV * VW
  constexpr int R = norm_rows<VW, NV, 8>();
  __shared__ float sums[kCols];
  const int lanes = g.lanes, tid = threadIdx.x, t = tid & (lanes - 1), per = kThreads / lanes, C = g.C;
  const T *total = static_cast<const T *>(g.total), *dy = static_cast<const T *>(g.dy);
  const T *dtotal = static_cast<const T *>(g.dtotal);
  T *dx = static_cast<T *>(g.dx);
  const float inv_c = 1.0f / float(C);
  float w[NV][VW], dw[NV][VW];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * lanes + t) * VW;
#pragma unroll
    for (int i = 0; i < VW; ++i) {
      w[j][i] = c + i < C ? g.w[c + i] : 0.f;
      dw[j][i] = 0.f;
    }
  }
  const int64_t step = int64_t(gridDim.x) * per * R;
  for (int64_t r0 = int64_t(blockIdx.x) * per * R; r0 < g.M; r0 += step) {
    float u[R][NV][VW], d[R][NV][VW], dot[R], rstd[R];
    Vec<T, VW> uv[R][NV], dv[R][NV], tv[R][NV];
    int64_t r[R];
    bool on[R];
    // dtotal early, where registers allow it
    constexpr bool EARLY = NV * VW <= 24;
    auto load_t = [&](int k) {
      const T *row = dtotal + (on[k] ? r[k] : 0) * g.lddt;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * lanes + t) * VW;
        tv[k][j].load(row, c < C ? c : 0, C);
      }
    };
#pragma unroll
    for (int k = 0; k < R; ++k) {
      r[k] = r0 + k * per + tid / lanes;
      on[k] = r[k] < g.M;
      const int64_t at = on[k] ? r[k] : 0;
      rstd[k] = g.rstd[at];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * lanes + t) * VW, in = c < C ? c : 0;
        uv[k][j].load(total + at * g.ldt, in, C);
        dv[k][j].load(dy + at * g.lddy, in, C);
      }
    }
    if (EARLY && dtotal) {
#pragma unroll
      for (int k = 0; k < R; ++k) load_t(k);
    }
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * lanes + t) * VW;
        uv[k][j].values(c, C, u[k][j]);
        dv[k][j].values(c, C, d[k][j]);
        if (!on[k] || c >= C) {
#pragma unroll
          for (int i = 0; i < VW; ++i) u[k][j][i] = d[k][j][i] = 0.f;
        }
      }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      dot[k] = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          u[k][j][i] *= rstd[k];
          dw[j][i] = __builtin_fmaf(d[k][j][i], u[k][j][i], dw[j][i]);
          d[k][j][i] *= w[j][i];
          dot[k] = __builtin_fmaf(d[k][j][i], u[k][j][i], dot[k]);
        }
    }
    for (int m = lanes / 2; m; m >>= 1)
#pragma unroll
      for (int k = 0; k < R; ++k) dot[k] += __shfl_xor(dot[k], m);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (!EARLY && dtotal) load_t(k);
      const float mean = dot[k] * inv_c;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * lanes + t) * VW;
        float v[VW];
        if (dtotal) {
          tv[k][j].values(c, C, v);
        } else {
#pragma unroll
          for (int i = 0; i < VW; ++i) v[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < VW; ++i) v[i] = __builtin_fmaf(rstd[k], d[k][j][i] - u[k][j][i] * mean, v[i]);
        if (on[k] && c < C) Vec<T, VW>::store(dx + r[k] * g.lddx, c, C, v);
      }
    }
  }
  // the wave's row groups by a butterfly, then the waves in turn
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VW; ++i)
      for (int m = lanes; m < kWave; m <<= 1) dw[j][i] += __shfl_xor(dw[j][i], m);
  for (int k = 0; k < kWaves; ++k) {
    if (tid / kWave == k && tid % kWave < lanes) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          const int c = (j * lanes + t) * VW + i;
          sums[c] = k == 0 ? dw[j][i] : sums[c] + dw[j][i];
        }
    }
    __syncthreads();
  }
  for (int c = tid; c < C; c += kThreads) g.part[int64_t(blockIdx.x) * C + c] = sums[c];
}

template <class T>
__global__ __launch_bounds__(kThreads) void norm_wide_backward_kernel(NormBackArgs g) {
  __shared__ float tmp[kWaves];
  const int tid = threadIdx.x, C = g.C;
  float *part = g.part + int64_t(blockIdx.x) * C;
  bool first = true;
  for (int64_t r = blockIdx.x; r < g.M; r += gridDim.x, first = false) {
    const T *total = static_cast<const T *>(g.total) + r * g.ldt, *dy = static_cast<const T *>(g.dy) + r * g.lddy;
    const T *dtotal = g.dtotal ? static_cast<const T *>(g.dtotal) + r * g.lddt : nullptr;
    T *dx = static_cast<T *>(g.dx) + r * g.lddx;
    const float rstd = g.rstd[r];
    float dot = 0.f;
    for (int c = tid; c < C; c += kThreads) {  // every thread has its own columns of part
      const float u = to_f32(total[c]) * rstd, d = to_f32(dy[c]);
      part[c] = first ? d * u : __builtin_fmaf(d, u, part[c]);
      dot = __builtin_fmaf(d * g.w[c], u, dot);
    }
    dot = block_sum(dot, tmp, tid) * (1.0f / float(C));
    for (int c = tid; c < C; c += kThreads) {
      const float u = to_f32(total[c]) * rstd, t = to_f32(dy[c]) * g.w[c];
      dx[c] = from_f32<T>(__builtin_fmaf(rstd, t - u * dot, dtotal ? to_f32(dtotal[c]) : 0.f));
    }
  }
}

// out[c] = sum of part[.][c] in a fixed order: a workgroup owns 16 columns and 64
// row groups, each thread sums every 64th row, then the groups are added in order.
constexpr int kSumCols = 16, kSumGroups = 64;
__global__ __launch_bounds__(kSumCols *kSumGroups) void column_sum_kernel(int R, int C, const float *__restrict__ part,
                                                                        float *__restrict__ out) {
  __shared__ float sums[kSumGroups][kSumCols];
  const int col = threadIdx.x % kSumCols, grp = threadIdx.x / kSumCols, c = blockIdx.x * kSumCols + col;
  float s = 0.f;
  if (c < C) {
#pragma unroll 4
    for (int r = grp; r < R; r += kSumGroups) s += part[int64_t(r) * C + c];
  }
  sums[grp][col] = s;
  __syncthreads();
  if (grp == 0 && c < C) {
    float a = 0.f;
#pragma unroll 8
    for (int k = 0; k < kSumGroups; ++k) a += sums[k][col];
    out[c] = a;
  }
}

// ------------------------------------------------------------- launches
constexpr int kMaxBackGroups = 1024;  // partial rows of dw
// of rows in registers: two to a compute unit, of which registers hold one at a time
// for the widest rows (1.05M rows of 128 fp32: 736 us with the forward, 766 with 1024
// workgroups; 20,001 of 1031 bf16: 87 and 92)
constexpr int kBackGroups = 512;

// Rows in registers up to 64 floats a lane, else one workgroup per row.
struct NormShape {
  int lanes, nv;  // nv == 0: wide
};
template <class T>
NormShape norm_shape(int C) {
  constexpr int W = 16 / sizeof(T);
  const int vw = C < W ? 1 : W, units = int(cdiv(C, vw));
  int lanes = 1;
  while (lanes < units && lanes < kWave) lanes *= 2;
  const int nv = int(cdiv(units, lanes));
  return {lanes, nv * vw <= 64 ? nv : 0};
}

// Calls f(VW, NV) as compile-time constants, NV the next of the compiled ones;
// false if no kernel in registers fits.
template <class T, class F>
bool with_shape(int C, int nv, F &&f) {
  constexpr int W = 16 / sizeof(T);
#define ALLEGRO_NORM_CASE(n)                                               \
  if (nv <= n && n * W <= 64) {                                            \
    f(std::integral_constant<int, W>{}, std::integral_constant<int, n>{}); \
    return true;                                                           \
  }
  if (nv == 0) return false;
  if (C < W) {
    f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
    return true;
  }
  ALLEGRO_NORM_CASE(1)
  ALLEGRO_NORM_CASE(2)
  ALLEGRO_NORM_CASE(3)
  ALLEGRO_NORM_CASE(4)
  ALLEGRO_NORM_CASE(6)
  ALLEGRO_NORM_CASE(8)
  if constexpr (W == 4) {
    ALLEGRO_NORM_CASE(12)
    ALLEGRO_NORM_CASE(16)
  }
#undef ALLEGRO_NORM_CASE
  return false;
}

template <class T, bool F8>
void norm_forward(NormArgs g, hipStream_t s) {
  const NormShape z = norm_shape<T>(g.C);
  g.lanes = z.lanes;
  if (with_shape<T>(g.C, z.nv, [&](auto vw, auto nv) {
        const int64_t rows = kThreads / z.lanes * norm_rows<vw(), nv(), 16>();
        // rows of one vector a lane: a workgroup for each few rows, in order of arrival
        // (1.05M rows of 128 fp32: 766 us with the backward, 793 with 2048 persistent
        // workgroups); longer ones: four workgroups to a compute unit (registers hold 1 to
        // 7 there), as each first loads its columns' w
        const unsigned grid = unsigned(std::min<int64_t>(cdiv(g.M, rows), nv() == 1 ? kMaxGrid : 1024));
        hipLaunchKernelGGL((norm_forward_kernel<T, vw(), nv(), F8>), dim3(grid), dim3(kThreads), 0, s, g);
      }))
    return;
  hipLaunchKernelGGL((norm_wide_forward_kernel<T, F8>), dim3(unsigned(std::min<int64_t>(g.M, 4096))), dim3(kThreads), 0,
                     s, g);
}

int64_t back_groups(int64_t M) { return std::min<int64_t>(M, kMaxBackGroups); }

template <class T>
void norm_backward(NormBackArgs g, float *dw, hipStream_t s) {
  const NormShape z = norm_shape<T>(g.C);
  g.lanes = z.lanes;
  int64_t grid = 0;
  if (!with_shape<T>(g.C, z.nv, [&](auto vw, auto nv) {
        grid = std::min<int64_t>(cdiv(g.M, kThreads / z.lanes * norm_rows<vw(), nv(), 8>()), kBackGroups);
        if (grid == 1) g.part = dw;  // few rows: no sums over workgroups
        hipLaunchKernelGGL((norm_backward_kernel<T, vw(), nv()>), dim3(unsigned(grid)), dim3(kThreads), 0, s, g);
      })) {
    grid = back_groups(g.M);
    if (grid == 1) g.part = dw;
    hipLaunchKernelGGL((norm_wide_backward_kernel<T>), dim3(unsigned(grid)), dim3(kThreads), 0, s, g);
  }
  if (grid == 1) return;
  hipLaunchKernelGGL(column_sum_kernel, dim3(unsigned(cdiv(g.C, kSumCols))), dim3(kSumCols * kSumGroups), 0, s,
                     int(grid), g.C, g.part, dw);
}

int key_bits(int G) {  // bits of the keys 0 .. G
  int b = 1;
  while ((1 << b) <= G) ++b;
  return b;
}

size_t group_bytes(int64_t M, int G) {
  if (M <= kOneChunk) return 0;
  return size_t(cdiv(M, chunk_rows(M)) + 1) * size_t(G + 1) * sizeof(int);
}

int check_norm(int dtype, int64_t M, int C, float eps) {
  int rc;
  if ((rc = check_dtype(dtype)) || (rc = check_m(M)) || (rc = check_width(C, "C"))) return rc;
  if (!(eps >= 0.f)) return fail(ALLEGRO_E_INVALID, "eps=%g is negative", double(eps));
  return ALLEGRO_OK;
}

int forward_call(const char *what, bool f8, int dtype, NormArgs g, hipStream_t s) {
  int rc;
  const int elem = dtype == ALLEGRO_F32 ? 4 : 2;
  if ((rc = check_norm(dtype, g.M, g.C, g.eps))) return rc;
  if (g.M == 0) return ALLEGRO_OK;
  if ((rc = check_rows(g.x, "x", g.ldx, g.C, elem)) || (rc = check_ptr(g.w, "w", 4)) ||
      (rc = check_rows(g.y, f8 ? "q" : "y", g.ldy, g.C, f8 ? 1 : elem)))
    return rc;
  if (g.residual && (rc = check_rows(g.residual, "residual", g.ldr, g.C, elem))) return rc;
  if (g.total && (rc = check_rows(g.total, "total", g.ldt, g.C, elem))) return rc;
  if (f8 && (rc = check_ptr(g.scale, "scale", 4))) return rc;
  if (g.rstd && (rc = check_ptr(g.rstd, "rstd", 4))) return rc;
  if (dtype == ALLEGRO_F32)
    f8 ? norm_forward<float, true>(g, s) : norm_forward<float, false>(g, s);
  else
    f8 ? norm_forward<uint16_t, true>(g, s) : norm_forward<uint16_t, false>(g, s);
  return after(what);
}

}  // namespace

extern "C" {

const char *allegro_latent_last_error(void) { return allegro_internal::last_error(); }

int allegro_group_rows_workspace(int64_t M, int G, size_t *bytes) {
  int rc;
  if ((rc = check_m(M)) || (rc = check_g(G))) return rc;
  if (!bytes) return fail(ALLEGRO_E_INVALID, "bytes is NULL");
  *bytes = group_bytes(M, G);
  return ALLEGRO_OK;
}

int allegro_group_rows(int64_t M, int G, const int32_t *type, int64_t *offsets, int32_t *rows, void *workspace,
                       size_t workspace_bytes, void *stream) {
  int rc;
  if ((rc = check_m(M)) || (rc = check_g(G)) || (rc = check_ptr(offsets, "offsets", 8))) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (M > 0 && ((rc = check_ptr(type, "type", 4)) || (rc = check_ptr(rows, "rows", 4)) ||
                (rc = check_workspace(workspace, workspace_bytes, group_bytes(M, G)))))
    return rc;
  const int bits = key_bits(G);
  if (M <= kOneChunk) {
    hipLaunchKernelGGL(group_one_kernel, dim3(1), dim3(kThreads), 0, s, int(M), G, bits, type, offsets, rows);
    return after("allegro_group_rows");
  }
  const int64_t chunk = chunk_rows(M);
  const int chunks = int(cdiv(M, chunk));
  int *hist = static_cast<int *>(workspace), *total = hist + int64_t(G + 1) * chunks;
  hipLaunchKernelGGL(group_count_kernel, dim3(chunks), dim3(kThreads), 0, s, M, G, chunk, type, hist);
  // Sums over few chunks cost less than a launch of their own, us, three launches against
  // two: 5,000 rows 16 against 13, 120,000 of 16 types 16 against 13 and of 225 16 against
  // 15, 250,000 of 225 16 against 17; 30,000 of 1000 (four rounds of the threads) 18
  // against 27.
  if (chunks <= 64 && G < kThreads) {
    hipLaunchKernelGGL(group_place_kernel<true>, dim3(chunks), dim3(kThreads), 0, s, M, G, bits, chunk, type, hist, total,
                       offsets, rows);
  } else {
    hipLaunchKernelGGL(group_scan_kernel, dim3(unsigned(cdiv(G + 1, kScanTypes))), dim3(kScanTypes * kScanParts), 0, s,
                       chunks, G, hist, total);
    hipLaunchKernelGGL(group_place_kernel<false>, dim3(chunks), dim3(kThreads), 0, s, M, G, bits, chunk, type, hist, total,
                       offsets, rows);
  }
  return after("allegro_group_rows");
}

int allegro_rms_norm_forward(int dtype, int64_t M, int C, float eps, const void *x, int64_t ldx, const void *residual,
                             int64_t ldr, const float *w, void *total, int64_t ldt, void *y, int64_t ldy, float *rstd,
                             void *stream) {
  return forward_call("allegro_rms_norm_forward", false, dtype,
                      {M, C, 0, eps, x, residual, w, total, y, rstd, nullptr, ldx, ldr, ldt, ldy},
                      static_cast<hipStream_t>(stream));
}

int allegro_rms_norm_fp8(int dtype, int64_t M, int C, float eps, const void *x, int64_t ldx, const void *residual,
                         int64_t ldr, const float *w, void *total, int64_t ldt, void *q, int64_t ldq, float *scale,
                         void *stream) {
  return forward_call("allegro_rms_norm_fp8", true, dtype,
                      {M, C, 0, eps, x, residual, w, total, q, nullptr, scale, ldx, ldr, ldt, ldq},
                      static_cast<hipStream_t>(stream));
}

int allegro_rms_norm_workspace(int64_t M, int C, size_t *bytes) {
  int rc;
  if ((rc = check_m(M)) || (rc = check_width(C, "C"))) return rc;
  if (!bytes) return fail(ALLEGRO_E_INVALID, "bytes is NULL");
  *bytes = size_t(back_groups(M)) * size_t(C) * sizeof(float);
  return ALLEGRO_OK;
}

int allegro_rms_norm_backward(int dtype, int64_t M, int C, const void *total, int64_t ldt, const float *w,
                              const float *rstd, const void *dy, int64_t lddy, const void *dtotal, int64_t lddt,
                              void *dx, int64_t lddx, float *dw, void *workspace, size_t workspace_bytes,
                              void *stream) {
  int rc;
  const int elem = dtype == ALLEGRO_F32 ? 4 : 2;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if ((rc = check_norm(dtype, M, C, 0.f)) || (rc = check_ptr(dw, "dw", 4))) return rc;
  if (M == 0) {
    hipLaunchKernelGGL(zero_kernel, dim3(unsigned(cdiv(C, kThreads))), dim3(kThreads), 0, s, int64_t(C), dw);
    return after("allegro_rms_norm_backward");
  }
  size_t need;
  if ((rc = check_rows(total, "total", ldt, C, elem)) || (rc = check_ptr(w, "w", 4)) ||
      (rc = check_ptr(rstd, "rstd", 4)) || (rc = check_rows(dy, "dy", lddy, C, elem)) ||
      (rc = check_rows(dx, "dx", lddx, C, elem)) || (rc = allegro_rms_norm_workspace(M, C, &need)) ||
      (rc = check_workspace(workspace, workspace_bytes, need)))
    return rc;
  if (dtotal && (rc = check_rows(dtotal, "dtotal", lddt, C, elem))) return rc;
  const NormBackArgs g{M, C, 0, total, dy, dtotal, w, rstd, dx, static_cast<float *>(workspace), ldt, lddy, lddt, lddx};
  if (dtype == ALLEGRO_F32)
    norm_backward<float>(g, dw, s);
  else
    norm_backward<uint16_t>(g, dw, s);
  return after("allegro_rms_norm_backward");
}

}  // extern "C"
