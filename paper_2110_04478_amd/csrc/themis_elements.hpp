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
constexpr uint32_t kLaneElements = 8;

// A lane's access to elements `first`.. of a row: kVec of them.  The last access of a row is moved back
// so that it is whole as well, and its first `skip` elements are another lane's.  Rows of less than
// kLaneElements are read and written element by element: kWhole is false for them, and only for them.
// (All choices are made at compile time: of two stores to one place, one of which goes past the
// caches, the compiler makes one that does not.)
template <int kVec>
struct Access {
  uint32_t at, skip, count;   // count: elements of its own (0: none)
  __device__ __forceinline__ Access(uint32_t first, uint32_t width) {
    count = first < width ? min(width - first, (uint32_t)kVec) : 0u;
    // (a lane without elements of its own reads the last ones again)
    at = width >= kLaneElements ? min(first, width - kVec) : first;
    skip = count ? first - at : 0u;
  }
  template <bool kWhole, bool kOnce = false, typename T>
  __device__ __forceinline__ typename Packed<T, kVec>::type read(const T* row) const {
    return !kWhole ? load_some<kVec>(row + at, count) : kOnce ? load_once<kVec>(row + at) : load<kVec>(row + at);
  }
  template <bool kWhole, bool kAway = false, typename T>
  __device__ __forceinline__ void write(T* row, Floats<kVec> v) const {
    if (!kWhole) return store_some<kVec>(row + at, v, count);
    if (count == kVec) return kAway ? store_away<kVec>(row + at, v) : store<kVec>(row + at, v);
    if (!count) return;
#pragma unroll
    for (uint32_t k = 1; k < kVec; ++k)
      if (k >= skip) row[at + k] = (T)v[k];
  }
  // Zero in the places of other lanes' elements.
  template <bool kWhole>
  __device__ __forceinline__ Floats<kVec> own(Floats<kVec> v) const {
    if (count == kVec) return v;
#pragma unroll
    for (uint32_t k = 0; k < kVec; ++k)
      if (kWhole ? k < skip || !count : k >= count) v[k] = 0.0f;
    return v;
  }
  // Where lanes that share elements, or have none of their own, write what the owner writes.
  template <bool kWhole, bool kAway, typename T>
  __device__ __forceinline__ void write_over(T* row, Floats<kVec> v) const {
    if constexpr (!kWhole) {
      store_some<kVec>(row + at, v, count);
    } else if constexpr (kAway) {
      store_away<kVec>(row + at, v);
    } else {
      store<kVec>(row + at, v);
    }
  }
};

// Eight elements of a row for every lane of a group of `lanes`, `first` being the group's first:
// adjacent ones (kVec = 8), or four and four, `lanes` accesses apart (kVec = 4).
template <int kVec>
struct Slice;
template <>
struct Slice<8> {
  Access<8> a;
  __device__ __forceinline__ Slice(uint32_t first, uint32_t lane, uint32_t, uint32_t width) : a(first + lane * 8, width) {}
  __device__ __forceinline__ bool any() const { return a.count != 0; }
  __device__ __forceinline__ bool whole() const { return a.count == 8; }
  template <bool kWhole, bool kOnce = false, typename T>
  __device__ __forceinline__ typename Packed<T, 8>::type read(const T* row) const { return a.read<kWhole, kOnce>(row); }
  template <bool kWhole, typename T>
  __device__ __forceinline__ void write(T* row, float8 v) const { a.write<kWhole>(row, v); }
  template <bool kWhole>
  __device__ __forceinline__ float8 own(float8 v) const { return a.own<kWhole>(v); }
  template <bool kWhole, bool kAway, typename T>
  __device__ __forceinline__ void write_over(T* row, float8 v) const { a.write_over<kWhole, kAway>(row, v); }
};
template <>
struct Slice<4> {
  Access<4> a, b;
  __device__ __forceinline__ Slice(uint32_t first, uint32_t lane, uint32_t lanes, uint32_t width)
      : a(first + lane * 4, width), b(first + (lanes + lane) * 4, width) {}
  __device__ __forceinline__ bool any() const { return a.count != 0; }
  __device__ __forceinline__ bool whole() const { return a.count == 4 && b.count == 4; }
  template <bool kWhole, bool kOnce = false, typename T>
  __device__ __forceinline__ typename Packed<T, 8>::type read(const T* row) const {
    return __builtin_shufflevector(a.read<kWhole, kOnce>(row), b.read<kWhole, kOnce>(row), 0, 1, 2, 3, 4, 5, 6, 7);
  }
  template <bool kWhole, typename T>
  __device__ __forceinline__ void write(T* row, float8 v) const {
    a.write<kWhole>(row, v.lo);
    b.write<kWhole>(row, v.hi);
  }
  template <bool kWhole>
  __device__ __forceinline__ float8 own(float8 v) const {
    return __builtin_shufflevector(a.own<kWhole>(v.lo), b.own<kWhole>(v.hi), 0, 1, 2, 3, 4, 5, 6, 7);
  }
  template <bool kWhole, bool kAway, typename T>
  __device__ __forceinline__ void write_over(T* row, float8 v) const {
    a.write_over<kWhole, kAway>(row, v.lo);
    b.write_over<kWhole, kAway>(row, v.hi);
  }
};

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
__device__ __forceinline__ int64_t row_offset(const Rows& rows, uint32_t r) {
  if (!rows.inner) return (int64_t)r * rows.inner_stride;
  const uint32_t outer = r / rows.inner;
  return (int64_t)outer * rows.outer_stride + (int64_t)(r - outer * rows.inner) * rows.inner_stride;
}
template <typename T>
__device__ __forceinline__ T* row_at(const Rows& rows, uint32_t r) {
  return (T*)rows.data + row_offset(rows, r);
}

// Zeros in the rows of `empty` behind v0, by a workgroup: short rows side by side.  kAway: past the
// caches (beside sums that need them: 65,537 tokens of 1,000 108 us, through them 116; alone it is
// 200 MB in 52 us and 45).
template <bool kWhole, bool kAway, typename Out>
__device__ __forceinline__ void write_zeros(uint64_t empty, uint32_t v0, uint32_t width, const Rows& grad) {
  constexpr int kVec = kVecOf<Out>;
  const uint32_t vecs = (width + kVec - 1) / kVec;
  const uint32_t shift = vecs >= 256 ? 8u : vecs <= 1 ? 0u : 32u - (uint32_t)__builtin_clz(vecs - 1);
  for (uint32_t r = threadIdx.x >> shift; r < 64; r += 256u >> shift) {
    if (!((empty >> r) & 1u)) continue;
    Out* to = row_at<Out>(grad, v0 + r);
    for (uint32_t c = threadIdx.x & ((1u << shift) - 1u); c < vecs; c += 256)
      Access<kVec>(c * kVec, width).template write_over<kWhole, kAway>(to, Floats<kVec>(0.0f));
  }
}

// Rows spread over a grid lane by lane, whatever their length: a row's `lanes` follow the one before's,
// across wavefronts and workgroups.  Segments of rows (blockIdx.y) keep the count of lanes below 2^31.
struct Spread {
  uint32_t lanes, inverse, shift;   // of a row: at / lanes is (at * inverse) >> (32 + shift), of 1 at itself
  uint32_t rows, segments;
};
// Calls f(row, lane) for this lane of workgroup `block`, of n rows, once for every segment.
template <typename F>
__device__ __forceinline__ void spread_rows(const Spread& s, uint32_t block, uint32_t n, F&& f) {
  for (uint32_t segment = blockIdx.y; segment < s.segments; segment += gridDim.y) {
    const uint32_t first = segment * s.rows, rows = min(n - first, s.rows), at = block * 256u + threadIdx.x;
    const uint32_t row = s.lanes == 1 ? at : __umulhi(at, s.inverse) >> s.shift;
    if (row < rows) f(first + row, at - row * s.lanes);
  }
}

// Numbers of the tokens t[] as table rows, ~0u for those outside the table; the loads are in flight
// together.
template <int kTokens>
__device__ __forceinline__ void token_rows(const Rows& ids, const uint32_t (&t)[kTokens], uint32_t vocab,
                                           uint32_t (&row)[kTokens]) {
  int64_t at[kTokens], id[kTokens];
  if (!ids.inner) {
#pragma unroll
    for (int k = 0; k < kTokens; ++k) at[k] = (int64_t)t[k] * ids.inner_stride;
  } else {
#pragma unroll
    for (int k = 0; k < kTokens; ++k) at[k] = row_offset(ids, t[k]);
  }
  if (ids.type == THEMIS_I64) {
#pragma unroll
    for (int k = 0; k < kTokens; ++k) id[k] = ((const int64_t*)ids.data)[at[k]];
  } else {
#pragma unroll
    for (int k = 0; k < kTokens; ++k) id[k] = ((const int32_t*)ids.data)[at[k]];
  }
#pragma unroll
  for (int k = 0; k < kTokens; ++k) row[k] = (uint64_t)id[k] < vocab ? (uint32_t)id[k] : ~0u;
}
__device__ __forceinline__ uint32_t token_row(const Rows& ids, uint32_t t, uint32_t vocab) {
  const uint32_t one[1] = {t};
  uint32_t row[1];
  token_rows(ids, one, vocab, row);
  return row[0];
}

// Calls f with a value of the element type that `type` names.
template <typename F>
inline void with_type(int type, F&& f) {
  if (type == THEMIS_F32) f(float{});
  else if (type == THEMIS_BF16) f(__bf16{});
  else f(_Float16{});
}

}  // namespace themis
