// What the kernels of the latent track share: element types, argument checks and the search of a
// tile's group (host and device side).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>

#include "allegro_latent.h"
#include "plan.hpp"

namespace latent {

using allegro_internal::fail;

constexpr int kWave = 64;
constexpr int kMaxWidth = 65536, kMaxGroups = 1024;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The same, and four floats, at any address that suits 16-bit (or 32-bit)
// elements: rows of odd widths and strides are read and written 16 bytes at a
// time too, which the memory path takes without a detour.
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_any8 __attribute__((ext_vector_type(4), aligned(1)));

// Elements of a row: fp32, or bf16 held as its 16 bits.
template <class T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32(uint16_t v) { return __builtin_bit_cast(float, uint32_t(v) << 16); }

__device__ __forceinline__ uint16_t bf16_bits(float v) { return __builtin_bit_cast(uint16_t, __bf16(v)); }  // to nearest
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32(float v) { return v; }
template <>
__device__ __forceinline__ uint16_t from_f32(float v) { return bf16_bits(v); }

// Workgroups of a launch, which takes fewer than 2^32 threads.  Where there are more
// tiles than this there are several launches; where a grid strides, it ends here.
constexpr int64_t kMaxGrid = int64_t(1) << 22;

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int after(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ALLEGRO_OK : fail(ALLEGRO_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Host checks.  A tensor of rows: pointer, element alignment, row stride.
inline int check_ptr(const void *p, const char *name, int elem) {
  if (!p) return fail(ALLEGRO_E_INVALID, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % unsigned(elem))
    return fail(ALLEGRO_E_INVALID, "%s is not %d-byte aligned", name, elem);
  return ALLEGRO_OK;
}
inline int check_rows(const void *p, const char *name, int64_t ld, int width, int elem) {
  if (ld < width)
    return fail(ALLEGRO_E_INVALID, "%s has row stride %lld, below its width %d", name, (long long)ld, width);
  if (ld > (int64_t(1) << 31)) return fail(ALLEGRO_E_INVALID, "%s has row stride %lld, over 2^31", name, (long long)ld);
  return check_ptr(p, name, elem);
}
// An output that is one of the inputs that are read while, or after, it is written.
inline int check_apart(const void *out, const char *name, std::initializer_list<const void *> inputs) {
  for (const void *in : inputs)
    if (out && out == in) return fail(ALLEGRO_E_INVALID, "%s is also an input", name);
  return ALLEGRO_OK;
}
inline int check_width(int v, const char *name) {
  if (v < 1 || v > kMaxWidth) return fail(ALLEGRO_E_INVALID, "%s=%d is not in 1 .. %d", name, v, kMaxWidth);
  return ALLEGRO_OK;
}
inline int check_m(int64_t M) {
  if (M < 0) return fail(ALLEGRO_E_INVALID, "negative size (M=%lld)", (long long)M);
  if (M > kMaxRows) return fail(ALLEGRO_E_INVALID, "M=%lld exceeds 2^31-1", (long long)M);
  return ALLEGRO_OK;
}
inline int check_g(int G) {
  if (G < 1 || G > kMaxGroups) return fail(ALLEGRO_E_INVALID, "G=%d is not in 1 .. %d", G, kMaxGroups);
  return ALLEGRO_OK;
}
inline int check_dtype(int dtype, const char *name = "dtype") {
  if (dtype != ALLEGRO_F32 && dtype != ALLEGRO_BF16) return fail(ALLEGRO_E_INVALID, "unknown %s %d", name, dtype);
  return ALLEGRO_OK;
}
inline int check_workspace(const void *p, size_t bytes, size_t need) {
  if (need == 0) return ALLEGRO_OK;
  if (!p) return fail(ALLEGRO_E_INVALID, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(p) & 15u) return fail(ALLEGRO_E_INVALID, "workspace is not 16-byte aligned");
  if (bytes < need)
    return fail(ALLEGRO_E_INVALID, "workspace of %zu bytes is smaller than the %zu required", bytes, need);
  return ALLEGRO_OK;
}

}  // namespace latent
