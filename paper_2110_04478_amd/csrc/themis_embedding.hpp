// Rows of a token table and the table's gradient (themis_embedding_lookup, _grad).
#pragma once

#include "themis_elements.hpp"

namespace themis {

// ---------------------------------------------------------------------------
// themis_embedding_lookup: out[t] = scale * table[ids[t]].
//
// 2^shift lanes take a row (a chunk of 2,048 elements of a longer one: blockIdx.y), each eight
// elements; a workgroup of 256 lanes takes kRows rows per group of lanes at once, so that their
// loads are in flight together: the number, then the row, are two dependent trips to memory and
// all that there is to hide.
// ---------------------------------------------------------------------------
template <typename In, typename Out, int kRows>
__global__ void __launch_bounds__(256)
lookup_kernel(themis_rows_t table, uint32_t vocab, uint32_t width, themis_rows_t ids, uint32_t n, float scale,
              themis_rows_t out, uint32_t shift) {
  const uint32_t col = (blockIdx.y * 256u + (threadIdx.x & ((1u << shift) - 1u))) * kVec;
  if (col >= width) return;
  const uint32_t count = min(width - col, (uint32_t)kVec);
  const uint32_t groups = 256u >> shift;   // rows side by side
  const uint32_t step = groups * kRows;
  for (uint64_t first = (uint64_t)blockIdx.x * step; first < n; first += (uint64_t)gridDim.x * step) {
    const uint32_t t0 = (uint32_t)first + (threadIdx.x >> shift);
    uint32_t row[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const uint64_t t = (uint64_t)t0 + k * groups;
      row[k] = t < n ? token_row(ids, (uint32_t)t, vocab) : ~0u;
    }
    typename Packed<In>::type v[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (row[k] != ~0u) v[k] = load_some((const In*)table.data + row_offset(table, row[k]) + col, count);
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const uint64_t t = (uint64_t)t0 + k * groups;
      if (t >= n) break;
      const float8 nan = __builtin_nanf("");
      const float8 x = row[k] != ~0u ? widen8<In>(v[k]) * scale : nan;
      store_some((Out*)out.data + row_offset(out, (uint32_t)t) + col, x, count);
    }
  }
}

// ---------------------------------------------------------------------------
// themis_embedding_grad: grad[v] (+)= scale * sum of grad_out[t] over ids[t] == v.
//
// A wavefront per table row and 512 of its elements: it looks through all token numbers, 64 at a
// time, and adds the rows of those that are its own in ascending order.
// ---------------------------------------------------------------------------
template <typename In, typename Out>
__global__ void __launch_bounds__(64)
embedding_grad_kernel(themis_rows_t grad_out, uint32_t width, themis_rows_t ids, uint32_t n, float scale,
                      uint32_t ignored, bool accumulate, themis_rows_t grad, uint32_t vocab) {
  const uint32_t col = (blockIdx.y * 64u + threadIdx.x) * kVec;
  const uint32_t count = col < width ? min(width - col, (uint32_t)kVec) : 0u;
  for (uint32_t v = blockIdx.x; v < vocab; v += gridDim.x) {
    float8 sum = 0.0f;
    bool any = false;
    for (uint32_t t = 0; t < n; t += 64) {
      const uint32_t id = t + threadIdx.x < n ? token_row(ids, t + threadIdx.x, vocab) : ~0u;
      uint64_t mine = v == ignored ? 0ull : __ballot(id == v);
      any |= mine != 0;
      for (; mine; mine &= mine - 1) {
        const uint32_t at = t + (uint32_t)__builtin_ctzll(mine);
        if (count) sum += widen8<In>(load_some((const In*)grad_out.data + row_offset(grad_out, at) + col, count));
      }
    }
    if (!count || (accumulate && !any)) continue;
    Out* to = (Out*)grad.data + row_offset(grad, v) + col;
    float8 x = sum * scale;
    if (accumulate) x = widen8<Out>(load_some(to, count)) + x;
    store_some(to, x, count);
  }
}

}  // namespace themis
