// Shared pieces of the full-rank operators (fullrank.hip, embed.hip): element access at any alignment, and the entry points' guard
// against C++ exceptions.
#pragma once
#include "../../include/lordo.h"
#include "common.h"

#include <cmath>
#include <cstdio>
#include <new>

namespace lordo {

// Four consecutive elements from any element on: the hardware takes 8- and 16-byte accesses at 2- and 4-byte addresses, so only the type has to
// say that it is aligned to an element.
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4a __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4a __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_value(uint32_t h) { return __uint_as_float(h << 16); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {      // the conversion instruction: two at once, nearest-even
  const f32x2 x = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

template <bool BF>
__device__ __forceinline__ float load_element(const void* p, int64_t i) {
  if constexpr (BF) return bf16_value(reinterpret_cast<const uint16_t*>(p)[i]);
  else return reinterpret_cast<const float*>(p)[i];
}
template <bool BF>
__device__ __forceinline__ void store_element(void* p, int64_t i, float x) {
  if constexpr (BF) reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)bf16_pair(x, 0.f);
  else reinterpret_cast<float*>(p)[i] = x;
}
// STREAM: touched once a call, by one workgroup: kept out of the caches' way
template <bool BF, bool STREAM>
__device__ __forceinline__ void load_quad(const void* p, int64_t i, float (&x)[4]) {
  if constexpr (BF) {
    const u32x2u* q = reinterpret_cast<const u32x2u*>(reinterpret_cast<const uint16_t*>(p) + i);
    u32x2u t;
    if constexpr (STREAM) t = __builtin_nontemporal_load(q);
    else t = *q;
    x[0] = __uint_as_float(t.x << 16); x[1] = __uint_as_float(t.x & 0xffff0000u);
    x[2] = __uint_as_float(t.y << 16); x[3] = __uint_as_float(t.y & 0xffff0000u);
  } else {
    const f32x4u* q = reinterpret_cast<const f32x4u*>(reinterpret_cast<const float*>(p) + i);
    f32x4u t;
    if constexpr (STREAM) t = __builtin_nontemporal_load(q);
    else t = *q;
    x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w;
  }
}
template <bool BF, bool STREAM>
__device__ __forceinline__ void store_quad(void* p, int64_t i, const float (&x)[4]) {
  if constexpr (BF) {
    const u32x2u t = {bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
    u32x2u* q = reinterpret_cast<u32x2u*>(reinterpret_cast<uint16_t*>(p) + i);
    if constexpr (STREAM) __builtin_nontemporal_store(t, q);
    else *q = t;
  } else {
    f32x4u t = {x[0], x[1], x[2], x[3]};
    f32x4u* q = reinterpret_cast<f32x4u*>(reinterpret_cast<float*>(p) + i);
    if constexpr (STREAM) __builtin_nontemporal_store(t, q);
    else *q = t;
  }
}

// VEC consecutive elements from any element on, as they are stored.
template <bool BF, int VEC>
struct Piece;
template <>
struct Piece<false, 4> {
  f32x4u v;
  __device__ __forceinline__ void clear() { v = f32x4u{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void load(const void* p, int64_t at) { v = *reinterpret_cast<const f32x4u*>(reinterpret_cast<const float*>(p) + at); }
  __device__ __forceinline__ float value(int e) const { return v[e]; }
};
template <>
struct Piece<true, 4> {
  u32x2u v;
  __device__ __forceinline__ void clear() { v = u32x2u{0, 0}; }
  __device__ __forceinline__ void load(const void* p, int64_t at) { v = *reinterpret_cast<const u32x2u*>(reinterpret_cast<const uint16_t*>(p) + at); }
  __device__ __forceinline__ float value(int e) const { return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16); }
};
template <>
struct Piece<true, 8> {
  u32x4u v;
  __device__ __forceinline__ void load(const void* p, int64_t at) { v = *reinterpret_cast<const u32x4u*>(reinterpret_cast<const uint16_t*>(p) + at); }
  __device__ __forceinline__ void clear() { v = u32x4u{0, 0, 0, 0}; }
  __device__ __forceinline__ float value(int e) const { return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16); }
};
template <>
struct Piece<false, 8> {
  Piece<false, 4> v[2];
  __device__ __forceinline__ void load(const void* p, int64_t at) { v[0].load(p, at); v[1].load(p, at + 4); }
  __device__ __forceinline__ void clear() { v[0].clear(); v[1].clear(); }
  __device__ __forceinline__ float value(int e) const { return v[e / 4].value(e & 3); }
};
template <bool BF>
struct Piece<BF, 1> {
  float v;
  __device__ __forceinline__ void load(const void* p, int64_t at) { v = load_element<BF>(p, at); }
  __device__ __forceinline__ void clear() { v = 0.f; }
  __device__ __forceinline__ float value(int) const { return v; }
};

// Elements skip ... VEC - 1 of a piece (what comes before them is the neighbour's).
template <bool BF, int VEC>
__device__ __forceinline__ void put_piece(void* p, int64_t at, const float (&x)[VEC], int skip) {
  if constexpr (VEC >= 4) {
    if (skip == 0) {
#pragma unroll
      for (int h = 0; h < VEC; h += 4) {
        const float y[4] = {x[h], x[h + 1], x[h + 2], x[h + 3]};
        store_quad<BF, false>(p, at + h, y);
      }
      return;
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e)
    if (e >= skip) store_element<BF>(p, at + e, x[e]);
}

// Which of up to 256 tensors chunk c belongs to: first[k] is the first chunk of tensor k (first[0] <= c).  Every lane compares its own entries, the
// bits are counted: one round of loads instead of a chain of them.
__device__ __forceinline__ int find_tensor(const int32_t* first, int count, int32_t c) {
  const int lane = threadIdx.x & 63;
  int32_t x[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) x[q] = first[64 * q + lane < count ? 64 * q + lane : 0];
  int k = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) k += __popcll(__ballot(64 * q + lane < count && x[q] <= c));
  return __builtin_amdgcn_readfirstlane(k - 1);
}

// A factor that reaches the kernels in fp32: neither infinite there nor NaN.
inline bool finite_in_fp32(double x) { return std::isfinite((float)x); }

// Nothing may leave a C entry point but a code.
template <class F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    fprintf(stderr, "lordo: out of host memory\n");
    return LORDO_ENOMEM;
  } catch (...) {
    return LORDO_EHIP;
  }
}
inline int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return LORDO_OK;
  fprintf(stderr, "lordo: %s failed: %s\n", what, hipGetErrorString(e));
  return LORDO_EHIP;
}

}  // namespace lordo
