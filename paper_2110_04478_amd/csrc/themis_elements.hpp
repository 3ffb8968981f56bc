// Elements of the gradient operators (gfx950 only): binary32, bfloat16 and binary16 in memory,
// binary32 in registers, eight at a time.
//
// A lane reads and writes eight adjacent elements with one or two 16-byte accesses, at any
// address that the element type itself may have: global memory takes such accesses at every
// byte address, so rows of odd lengths and tensors packed end to end need no path of their own.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "themis.h"

namespace themis {

constexpr int kVec = 8;  // elements of a lane's access

typedef float float8 __attribute__((ext_vector_type(8)));

template <typename T>
struct Packed;
template <>
struct Packed<float> {
  typedef float type __attribute__((ext_vector_type(8)));
  typedef float in_memory __attribute__((ext_vector_type(8), aligned(4)));
};
template <>
struct Packed<__bf16> {
  typedef __bf16 type __attribute__((ext_vector_type(8)));
  typedef __bf16 in_memory __attribute__((ext_vector_type(8), aligned(2)));
};
template <>
struct Packed<_Float16> {
  typedef _Float16 type __attribute__((ext_vector_type(8)));
  typedef _Float16 in_memory __attribute__((ext_vector_type(8), aligned(2)));
};

// As in memory (a load that is in flight), and as binary32.
template <typename T>
__device__ __forceinline__ typename Packed<T>::type load8(const T* p) {
  return *(const typename Packed<T>::in_memory*)p;
}
template <typename T>
__device__ __forceinline__ float8 widen8(typename Packed<T>::type v) {
  return __builtin_convertvector(v, float8);
}
// Rounded to nearest, ties to even; beyond the type's range infinite.
template <typename T>
__device__ __forceinline__ void store8(T* p, float8 v) {
  *(typename Packed<T>::in_memory*)p = __builtin_convertvector(v, typename Packed<T>::type);
}

// The first `count` (1..8) of eight.
template <typename T>
__device__ __forceinline__ typename Packed<T>::type load_some(const T* p, uint32_t count) {
  if (count == kVec) return load8(p);
  typename Packed<T>::type v = {};
#pragma unroll
  for (uint32_t k = 0; k < kVec - 1; ++k)
    if (k < count) v[k] = p[k];
  return v;
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, float8 v, uint32_t count) {
  if (count == kVec) return store8(p, v);
#pragma unroll
  for (uint32_t k = 0; k < kVec - 1; ++k)
    if (k < count) p[k] = (T)v[k];
}

__host__ __device__ constexpr bool is_float_type(int type) { return type >= THEMIS_F32 && type <= THEMIS_F16; }
__host__ __device__ constexpr bool is_index_type(int type) { return type == THEMIS_I32 || type == THEMIS_I64; }
__host__ __device__ constexpr uint32_t type_bytes(int type) {
  return type == THEMIS_I64 ? 8u : type == THEMIS_F32 || type == THEMIS_I32 ? 4u : 2u;
}

// Elements in front of row r (see themis_rows_t).  n, and so every row number, is below 2^31.
__device__ __forceinline__ int64_t row_offset(const themis_rows_t& rows, uint32_t r) {
  if (r < rows.inner) return (int64_t)r * rows.inner_stride;   // (one level, or the first of two)
  const uint32_t inner = (uint32_t)rows.inner, outer = r / inner;
  return (int64_t)outer * rows.outer_stride + (int64_t)(r - outer * inner) * rows.inner_stride;
}

// Token number t as a table row, or ~0u for one outside the table.
__device__ __forceinline__ uint32_t token_row(const themis_rows_t& ids, uint32_t t, uint32_t vocab) {
  const int64_t at = row_offset(ids, t);
  const int64_t id = ids.type == THEMIS_I64 ? ((const int64_t*)ids.data)[at] : (int64_t)((const int32_t*)ids.data)[at];
  return (uint64_t)id < vocab ? (uint32_t)id : ~0u;
}

// Calls f with a value of the element type that `type` names.
template <typename F>
inline void with_type(int type, F&& f) {
  if (type == THEMIS_F32) f(float{});
  else if (type == THEMIS_BF16) f(__bf16{});
  else f(_Float16{});
}

}  // namespace themis
