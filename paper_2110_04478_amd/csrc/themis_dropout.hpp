// themis_dropout: elements kept or dropped by a counter-based generator; no mask is stored.
#pragma once

#include "themis_elements.hpp"

namespace themis {

// ---------------------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011): ten
// rounds of two 32 x 32 bit products on a counter of 128 bits under a key of 64.  A counter is (block of
// four columns, row, call), so what an element gets depends on its row and column alone: not on
// the row's length, on strides, or on how the work is split.
// ---------------------------------------------------------------------------
struct DropoutKey {
  uint32_t key[2], call[2];
  uint32_t least;   // words from here on keep their element
  bool none;        // no word does
  float scale;
};

__device__ __forceinline__ void philox(const DropoutKey& d, uint32_t block, uint32_t row, uint32_t* word) {
  uint32_t c0 = block, c1 = row, c2 = d.call[0], c3 = d.call[1], k0 = d.key[0], k1 = d.key[1];
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  word[0] = c0;
  word[1] = c1;
  word[2] = c2;
  word[3] = c3;
}

// x's elements of an access, those that are dropped 0 and the others scaled.
template <int kVec>
__device__ __forceinline__ Floats<kVec> drop(const DropoutKey& d, const Access<kVec>& a, uint32_t row, Floats<kVec> x) {
  uint32_t word[kVec];
#pragma unroll
  for (int b = 0; b < kVec / 4; ++b) philox(d, (a.at + a.skip) / 4 + b, row, word + 4 * b);
  for (uint32_t s = 0; s < a.skip; ++s)   // (an access that was moved back: its own elements are the last ones)
#pragma unroll
    for (int i = kVec - 1; i > 0; --i) word[i] = word[i - 1];
#pragma unroll
  for (int i = 0; i < kVec; ++i) x[i] = word[i] >= d.least && !d.none ? x[i] * d.scale : 0.0f;
  return x;
}

// 2^shift lanes take a row (a chunk of 256 accesses of a longer one: blockIdx.y).
template <bool kWhole, bool kAdd, typename In, typename Out>
__global__ void __launch_bounds__(256)
dropout_kernel(Rows x, uint32_t n, uint32_t width, DropoutKey d, const uint64_t* call_at, Rows add, Rows out,
               uint32_t shift) {
  constexpr int kVec = kVecOf<In, Out>;
  const uint32_t lanes = 1u << shift, groups = 256u >> shift;
  const Access<kVec> a((blockIdx.y * 256u + (threadIdx.x & (lanes - 1u))) * kVec, width);
  if (!a.count) return;
  if (call_at) {
    const uint64_t call = ((uint64_t)d.call[1] << 32 | d.call[0]) + *call_at;
    d.call[0] = (uint32_t)call;
    d.call[1] = (uint32_t)(call >> 32);
  }
  for (uint64_t r = (uint64_t)blockIdx.x * groups + (threadIdx.x >> shift); r < n; r += (uint64_t)gridDim.x * groups) {
    const uint32_t row = (uint32_t)r;
    Out* to = row_at<Out>(out, row);
    const auto v = a.template read<kWhole>(row_at<const In>(x, row));
    Floats<kVec> held = 0.0f;
    if constexpr (kAdd) held = widen<kVec>(a.template read<kWhole>(row_at<const Out>(add, row)));
    Floats<kVec> kept = drop<kVec>(d, a, row, widen<kVec>(v));
    if constexpr (kAdd) kept += held;
    a.template write<kWhole>(to, kept);
  }
}

}  // namespace themis
