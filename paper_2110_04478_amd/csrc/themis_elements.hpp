// Elements of the gradient operators (gfx950 only): binary32, bfloat16 and binary16 in memory,
// binary32 in registers.
//
// A lane's access is 16 bytes of the wider type (kVec elements), lanes side by side, at any address
// that the element type itself may have: global memory takes such accesses at every byte address,
// so rows of odd lengths and tensors packed end to end need no path of their own.  What is read for
// the last time, or written for a later kernel, goes past the caches (`once`, `away`); that needs
// lines that one instruction covers, which eight binary32 elements of a lane would not.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "themis.h"

namespace themis {

typedef float float8 __attribute__((ext_vector_type(8)));

template <typename T, int N>
struct Packed {
  typedef T type __attribute__((ext_vector_type(N)));
  typedef T in_memory __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <int N>
using Floats = typename Packed<float, N>::type;

// Elements of an access where these types are read or written.
template <typename A, typename B = A>
constexpr int kVecOf = sizeof(A) == 4 || sizeof(B) == 4 ? 4 : 8;

// As in memory (a load that is in flight), and as binary32.
template <int N, typename T>
__device__ __forceinline__ typename Packed<T, N>::type load(const T* p) {
  return *(const typename Packed<T, N>::in_memory*)p;
}
template <int N, typename T>
__device__ __forceinline__ typename Packed<T, N>::type load_once(const T* p) {
  return __builtin_nontemporal_load((const typename Packed<T, N>::in_memory*)p);
}
template <int N, typename V>
__device__ __forceinline__ Floats<N> widen(V v) {
  return __builtin_convertvector(v, Floats<N>);
}
// Rounded to nearest, ties to even; beyond the type's range infinite.
template <int N, typename T>
__device__ __forceinline__ void store(T* p, Floats<N> v) {
  *(typename Packed<T, N>::in_memory*)p = __builtin_convertvector(v, typename Packed<T, N>::type);
}
template <int N, typename T>
__device__ __forceinline__ void store_away(T* p, Floats<N> v) {
  __builtin_nontemporal_store(__builtin_convertvector(v, typename Packed<T, N>::type),
                              (typename Packed<T, N>::in_memory*)p);
}

// The first `count` (0..N) elements.
template <int N, typename T>
__device__ __forceinline__ typename Packed<T, N>::type load_some(const T* p, uint32_t count) {
  if (count == N) return load<N>(p);
  typename Packed<T, N>::type v = {};
#pragma unroll
  for (uint32_t k = 0; k < N - 1; ++k)
    if (k < count) v[k] = p[k];
  return v;
}
template <int N, typename T>
__device__ __forceinline__ void store_some(T* p, Floats<N> v, uint32_t count) {
  if (count == N) return store<N>(p, v);
#pragma unroll
  for (uint32_t k = 0; k < N - 1; ++k)
    if (k < count) p[k] = (T)v[k];
}
template <int N, typename T>
__device__ __forceinline__ void store_some_away(T* p, Floats<N> v, uint32_t count) {
  if (count == N) return store_away<N>(p, v);
  store_some<N>(p, v, count);
}

// Eight elements of a row for every lane of a group of `lanes`, `first` being the group's first:
// adjacent ones (kVec = 8), or four and four, `lanes` accesses apart (kVec = 4).  Only the last ones
// of a row may be short of that: code that keeps loads in flight has a copy for full() lanes, whose
// accesses are whole, and in which no load depends on a count.
template <int kVec>
struct Slice;
template <>
struct Slice<8> {
  uint32_t at, count;
  __device__ __forceinline__ Slice(uint32_t first, uint32_t lane, uint32_t, uint32_t width) {
    at = first + lane * 8;
    count = at < width ? min(width - at, 8u) : 0u;
  }
  __device__ __forceinline__ bool any() const { return count != 0; }
  __device__ __forceinline__ bool full() const { return count == 8; }
  template <bool kFull, typename T>
  __device__ __forceinline__ typename Packed<T, 8>::type read(const T* row) const {
    return kFull ? load<8>(row + at) : load_some<8>(row + at, count);
  }
  template <bool kFull, typename T>
  __device__ __forceinline__ void write(T* row, float8 v) const {
    if (kFull) store<8>(row + at, v);
    else store_some<8>(row + at, v, count);
  }
  template <bool kFull, typename T>
  __device__ __forceinline__ void write_away(T* row, float8 v) const {
    if (kFull) store_away<8>(row + at, v);
    else store_some<8>(row + at, v, count);
  }
};
template <>
struct Slice<4> {
  uint32_t at, next, count, more;
  __device__ __forceinline__ Slice(uint32_t first, uint32_t lane, uint32_t lanes, uint32_t width) {
    at = first + lane * 4;
    next = at + lanes * 4;
    count = at < width ? min(width - at, 4u) : 0u;
    more = next < width ? min(width - next, 4u) : 0u;
    if (!more) next = at;   // (what is read there is not used)
  }
  __device__ __forceinline__ bool any() const { return count != 0; }
  __device__ __forceinline__ bool full() const { return count == 4 && (more & 3u) == 0; }
  template <bool kFull, typename T>
  __device__ __forceinline__ typename Packed<T, 8>::type read(const T* row) const {
    const auto a = kFull ? load<4>(row + at) : load_some<4>(row + at, count);
    const auto b = kFull ? load<4>(row + next) : load_some<4>(row + next, more);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  template <bool kFull, typename T>
  __device__ __forceinline__ void write(T* row, float8 v) const {
    if (kFull) {
      store<4>(row + at, v.lo);
      if (more) store<4>(row + next, v.hi);
    } else {
      store_some<4>(row + at, v.lo, count);
      store_some<4>(row + next, v.hi, more);
    }
  }
  template <bool kFull, typename T>
  __device__ __forceinline__ void write_away(T* row, float8 v) const {
    if (!kFull) return write<false>(row, v);
    store_away<4>(row + at, v.lo);
    if (more) store_away<4>(row + next, v.hi);
  }
};
constexpr uint32_t kLaneElements = 8;

__host__ __device__ constexpr bool is_float_type(int type) { return type >= THEMIS_F32 && type <= THEMIS_F16; }
__host__ __device__ constexpr bool is_index_type(int type) { return type == THEMIS_I32 || type == THEMIS_I64; }
__host__ __device__ constexpr uint32_t type_bytes(int type) {
  return type == THEMIS_I64 ? 8u : type == THEMIS_F32 || type == THEMIS_I32 ? 4u : 2u;
}

// themis_rows_t as the kernels take it: inner is 0 where one level is all that is used.  Row numbers
// are below 2^31.
struct Rows {
  char* data;
  int64_t outer_stride, inner_stride;
  uint32_t inner;
  int32_t type;
};
inline Rows rows_of(const themis_rows_t& r, uint64_t n) {
  return {(char*)r.data, r.outer_stride, r.inner_stride, r.inner < n ? (uint32_t)r.inner : 0u, r.type};
}
template <typename T>
__device__ __forceinline__ T* row_at(const Rows& rows, uint32_t r) {
  int64_t at = (int64_t)r * rows.inner_stride;
  if (rows.inner) {
    const uint32_t outer = r / rows.inner;
    at = (int64_t)outer * rows.outer_stride + (int64_t)(r - outer * rows.inner) * rows.inner_stride;
  }
  return (T*)rows.data + at;
}

// Token number t as a table row, or ~0u for one outside the table.
__device__ __forceinline__ uint32_t token_row(const Rows& ids, uint32_t t, uint32_t vocab) {
  const int64_t id = ids.type == THEMIS_I64 ? *row_at<const int64_t>(ids, t) : (int64_t)*row_at<const int32_t>(ids, t);
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
