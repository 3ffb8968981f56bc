// themis_dropout: elements kept or dropped by a counter-based generator; no mask is stored.
#pragma once

#include "themis_elements.hpp"

namespace themis {

// ---------------------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011): ten
// rounds of two 32 x 32 bit products on a counter of 128 bits under a key of 64.  A counter is (block of
// four columns, row, call), so what an element gets depends on its row and column alone: not on
// the row's length, on strides, or on how the work is split.  Bound by the products (five an element, of a quarter
// of the rate of others) and by memory, about alike: 268 M bf16 in 167 us, 6.4 TB/s.
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
    // (0x96: exclusive or of three, which the compiler makes two instructions)
    c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(b >> 32), c1, k0, 0x96);
    c1 = (uint32_t)b;
    c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(a >> 32), c3, k1, 0x96);
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

// kRows rows a lane, one under the other: the first two rounds' products of a column, and of a row, are made
// once.  kOnce: past the caches.
template <bool kWhole, bool kOnce, bool kAdd, int kRows, typename In, typename Out>
__global__ void __launch_bounds__(256)
dropout_kernel(Rows x, uint32_t n, uint32_t width, DropoutKey d, const uint64_t* call_at, Rows add, Rows out,
               Spread spread) {
  constexpr int kVec = kVecOf<In, Out>;
  if (call_at) {
    const uint64_t call = ((uint64_t)d.call[1] << 32 | d.call[0]) + *call_at;
    d.call[0] = (uint32_t)call;
    d.call[1] = (uint32_t)(call >> 32);
  }
  spread_rows(spread, blockIdx.x, (n + kRows - 1) / kRows, [&](uint32_t group, uint32_t lane) {
    const Access<kVec> a(lane * kVec, width);
    typename Packed<In, kVec>::type v[kRows];
    typename Packed<Out, kVec>::type held[kRows];
#pragma unroll
    for (uint32_t u = 0; u < kRows; ++u) {
      const uint32_t row = min(group * kRows + u, n - 1u);
      v[u] = a.template read<kWhole, kOnce>(row_at<const In>(x, row));
      if constexpr (kAdd) held[u] = a.template read<kWhole, kOnce>(row_at<const Out>(add, row));
    }
#pragma unroll
    for (uint32_t u = 0; u < kRows; ++u) {
      const uint32_t row = group * kRows + u;
      if (row >= n) break;
      Floats<kVec> kept = drop<kVec>(d, a, row, widen<kVec>(v[u]));
      if constexpr (kAdd) kept += widen<kVec>(held[u]);
      // (its own elements and no others: x or add may be where out is)
      a.template write<kWhole, kOnce>(row_at<Out>(out, row), kept);
    }
  });
}

}  // namespace themis
