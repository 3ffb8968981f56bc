// What the entry points on rows share: limits, checks of arguments, launches.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <tuple>
#include <utility>

#include "themis.h"
#include "themis_elements.hpp"

namespace themis {
namespace {

constexpr uint64_t kMost = 0x7fffffffu;   // of tokens, table rows and elements of a row

// Launches and keeps the first error that a launch of this call returns.
struct Launches {
  hipStream_t stream;
  hipError_t first = hipSuccess;
  explicit Launches(void* s) : stream((hipStream_t)s) {}
  template <typename... P, typename... A>
  void operator()(void (*kernel)(P...), dim3 grid, unsigned threads, A&&... a) {
    std::tuple<P...> params(std::forward<A>(a)...);
    launch(kernel, grid, threads, params, std::index_sequence_for<P...>{});
  }
  int status() const { return first == hipSuccess ? THEMIS_OK : THEMIS_ERR_DEVICE; }

 private:
  template <typename... P, size_t... I>
  void launch(void (*kernel)(P...), dim3 grid, unsigned threads, std::tuple<P...>& params, std::index_sequence<I...>) {
    if (first != hipSuccess) return;   // (what follows would work on what is not there)
    void* ptrs[sizeof...(P)] = {(void*)&std::get<I>(params)...};
    first = hipLaunchKernel((const void*)kernel, grid, dim3(threads), ptrs, 0, stream);
  }
};

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Rows that are only read.
bool rows_ok(const themis_rows_t* r, bool index) {
  return r && r->data && r->inner >= 1 && (index ? is_index_type(r->type) : is_float_type(r->type)) &&
         aligned(r->data, type_bytes(r->type));
}

// Whether n rows of `width` elements share no element: the level with the shorter steps steps over
// a row, the other over all of the shorter one's.
bool rows_apart(const themis_rows_t& r, uint64_t n, uint64_t width) {
  const uint64_t inner = std::min(r.inner, n), outer = (n + r.inner - 1) / r.inner;
  struct Level { uint64_t count; __int128 stride; } a{inner, r.inner_stride}, b{outer, r.outer_stride};
  if (a.stride < 0) a.stride = -a.stride;
  if (b.stride < 0) b.stride = -b.stride;
  if (a.count < 2) std::swap(a, b);
  if (a.count < 2) return true;                            // one row
  if (b.count < 2) return a.stride >= (__int128)width;
  if (a.stride > b.stride) std::swap(a, b);
  return a.stride >= (__int128)width && b.stride >= a.stride * (__int128)(a.count - 1) + (__int128)width;
}

uint32_t next_power(uint32_t x) {   // the smallest p with 2^p >= x
  uint32_t p = 0;
  while ((1u << p) < x) ++p;
  return p;
}

}  // namespace
}  // namespace themis
