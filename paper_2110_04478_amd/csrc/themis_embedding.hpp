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
// The tokens are sorted by their number, stable, so that a table row's tokens stand next to each
// other in ascending order; the sorted list is cut into tiles of one length, whatever the numbers
// are, so that a token that makes up half of the list costs no more than any other half.  A tile
// adds its rows one after the other and writes the sums that begin and end in it.  A sum that
// crosses tiles is left in parts, which are added in the order of the tiles.
//
// Sort: least significant digit first, up to ten bits a pass and two launches: every workgroup
// counts the digits of its part of the list, then every workgroup finds from all counts where its
// part's tokens go.  A token's key is its number, or `vocab` (behind all others) if it has no
// gradient.
// ---------------------------------------------------------------------------
constexpr uint32_t kMaxBins = 1024;
constexpr uint32_t kSortGroup = 1024, kSortWaves = kSortGroup / 64;

struct SortView {
  uint32_t n, part;      // tokens, tokens of a workgroup (a multiple of kSortGroup)
  uint32_t parts;        // workgroups
  uint32_t shift, bits;  // the pass's digit
  uint32_t* counts;      // [parts][1 << bits]
  const uint32_t* key_in;    // the pass before's, or none: the token numbers themselves
  const uint32_t* token_in;
  uint32_t* key_out;
  uint32_t* token_out;
};

__device__ __forceinline__ uint32_t sort_key(const SortView& s, const themis_rows_t& ids, uint32_t vocab,
                                             uint32_t ignored, uint32_t i) {
  if (s.key_in) return s.key_in[i];
  const uint32_t id = token_row(ids, i, vocab);
  return id == ~0u || id == ignored ? vocab : id;
}

__global__ void __launch_bounds__(kSortGroup)
sort_count_kernel(SortView s, themis_rows_t ids, uint32_t vocab, uint32_t ignored) {
  __shared__ uint32_t count[kMaxBins];
  const uint32_t bins = 1u << s.bits, first = blockIdx.x * s.part;
  const uint32_t last = min(first + s.part, s.n);
  for (uint32_t b = threadIdx.x; b < bins; b += kSortGroup) count[b] = 0;
  __syncthreads();
  for (uint32_t i = first + threadIdx.x; i < last; i += kSortGroup)
    atomicAdd(&count[(sort_key(s, ids, vocab, ignored, i) >> s.shift) & (bins - 1)], 1u);
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < bins; b += kSortGroup) s.counts[blockIdx.x * bins + b] = count[b];
}

__global__ void __launch_bounds__(kSortGroup)
sort_move_kernel(SortView s, themis_rows_t ids, uint32_t vocab, uint32_t ignored) {
  __shared__ uint32_t place[kSortWaves][kMaxBins];   // first a wavefront's counts, then where its next one goes
  __shared__ uint32_t wave_sums[kSortWaves];
  const uint32_t bins = 1u << s.bits, first = blockIdx.x * s.part;
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
  const uint32_t share = s.part / kSortWaves;   // a wavefront's tokens stand together (a multiple of 64)
  const uint32_t begin = min(first + wave * share, s.n), end = min(begin + share, s.n);
  const uint32_t b = threadIdx.x;               // a lane has one digit, or none
  if (b < bins)
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) place[w][b] = 0;
  __syncthreads();
  for (uint32_t i = begin + lane; i < end; i += 64)
    atomicAdd(&place[wave][(sort_key(s, ids, vocab, ignored, i) >> s.shift) & (bins - 1)], 1u);
  // Where a digit's tokens of this part go: behind all of smaller digits and those of the parts before.
  uint32_t before = 0, all = 0;
  if (b < bins) {
#pragma unroll 8
    for (uint32_t p = 0; p < s.parts; ++p) {
      const uint32_t c = s.counts[p * bins + b];
      before += p < blockIdx.x ? c : 0u;
      all += c;
    }
  }
  uint32_t upto = all;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(upto, d);
    if (lane >= (uint32_t)d) upto += y;
  }
  if (lane == 63) wave_sums[wave] = upto;
  __syncthreads();   // (the counts in LDS are complete as well)
  uint32_t at = upto - all + before;
#pragma unroll
  for (uint32_t w = 0; w < kSortWaves; ++w) at += w < wave ? wave_sums[w] : 0u;
  if (b < bins)
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) {
      const uint32_t c = place[w][b];
      place[w][b] = at;
      at += c;
    }
  __syncthreads();
  for (uint32_t i0 = begin; i0 < end; i0 += 64) {
    const uint32_t i = i0 + lane;
    const bool on = i < end;
    const uint32_t key = on ? sort_key(s, ids, vocab, ignored, i) : 0u;
    const uint32_t token = on ? (s.key_in ? s.token_in[i] : i) : 0u;
    const uint32_t digit = (key >> s.shift) & (bins - 1);
    uint64_t same = __ballot(on);   // lanes with this lane's digit
    for (uint32_t b = 0; b < s.bits; ++b) {
      const uint64_t ones = __ballot((digit >> b) & 1u);
      same &= (digit >> b) & 1u ? ones : ~ones;
    }
    const uint32_t rank = (uint32_t)__popcll(same & ((1ull << lane) - 1));
    // (all lanes have read before the first of a digit's adds: a wavefront's accesses to LDS are
    // served in the order of the program, and these are kept in it)
    const uint32_t at = (on ? __hip_atomic_load(&place[wave][digit], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) : 0u) + rank;
    if (on && rank == 0)
      __hip_atomic_store(&place[wave][digit], at + (uint32_t)__popcll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    if (on) {
      s.key_out[at] = key;
      s.token_out[at] = token;
    }
  }
}

// The sorted list in tiles, one for every group of lanes of a workgroup (a wavefront, less where the
// rows are short), and the tiles of a workgroup in blocks.
struct TileView {
  const uint32_t* key;     // [n], ascending, rounded up to a multiple of kTileStep
  const uint32_t* token;
  uint32_t n, tile;        // tokens, tokens of a tile (a multiple of kTileStep)
  uint32_t block;          // tokens of a block
  uint32_t blocks, slabs;  // slabs of 512 elements
  uint32_t shift;          // 2^shift lanes take a tile's slab
  uint32_t fill_rows;      // table rows of a workgroup that writes zeros, up to 64
  float* parts;            // [blocks][2][stride]: of a sum that began before, of one that goes on
  uint32_t stride;
};
constexpr uint32_t kTileStep = 8;    // rows in flight
constexpr uint32_t kLeastShift = 3;  // (up to 32 groups of lanes)

// Zeros in those of up to 64 table rows from `v0` on that no token has: a lane looks for its row.
template <typename Out>
__device__ __forceinline__ void fill_rows(const TileView& s, uint32_t v0, uint32_t width, const themis_rows_t& grad,
                                          uint32_t vocab) {
  const uint32_t lane = threadIdx.x & 63u, v = v0 + lane;
  const bool mine = lane < s.fill_rows && v < vocab;
  uint32_t lo = 0, hi = mine ? s.n : 0u;   // the first key that is not smaller
  while (__any(lo < hi)) {
    if (lo < hi) {
      const uint32_t mid = lo + ((hi - lo) >> 1);
      if (s.key[mid] < v) lo = mid + 1;
      else hi = mid;
    }
  }
  uint64_t empty = __ballot(mine && (lo >= s.n || s.key[lo] != v));
  const uint32_t vecs = (width + kVec - 1) / kVec;
  const float8 zero = 0.0f;
  for (; empty; empty &= empty - 1) {
    Out* to = (Out*)grad.data + row_offset(grad, v0 + (uint32_t)__builtin_ctzll(empty));
    for (uint32_t c = threadIdx.x; c < vecs; c += 256) store_some(to + c * kVec, zero, min(width - c * kVec, (uint32_t)kVec));
  }
}

template <typename Out>
__device__ __forceinline__ void write_sum(const themis_rows_t& grad, uint32_t v, uint32_t col, uint32_t count,
                                          float8 sum, float scale, bool accumulate) {
  Out* to = (Out*)grad.data + row_offset(grad, v) + col;
  float8 x = sum * scale;
  if (accumulate) x = widen8<Out>(load_some(to, count)) + x;
  store_some(to, x, count);
}

template <typename In, typename Out>
__global__ void __launch_bounds__(256)
tile_sum_kernel(TileView s, themis_rows_t grad_out, uint32_t width, float scale, bool accumulate, themis_rows_t grad,
                uint32_t vocab) {
  // A group's sums that its tile does not hold whole: of one that began before, of one that goes on.
  __shared__ float8 part[2][256];
  const uint32_t sums = s.blocks * s.slabs;
  if (blockIdx.x >= sums) {
    const uint64_t step = (uint64_t)(gridDim.x - sums) * s.fill_rows;
    for (uint64_t v = (uint64_t)(blockIdx.x - sums) * s.fill_rows; v < vocab; v += step)
      fill_rows<Out>(s, (uint32_t)v, width, grad, vocab);
    return;
  }
  const uint32_t block = blockIdx.x / s.slabs, slab = blockIdx.x - block * s.slabs;
  const uint32_t lanes = 1u << s.shift, group = threadIdx.x >> s.shift;
  const uint32_t col = (slab * 64u + (threadIdx.x & (lanes - 1u))) * kVec;
  const uint32_t count = col < width ? min(width - col, (uint32_t)kVec) : 0u;
  const uint32_t block_end = min(block * s.block + s.block, s.n);
  const uint32_t first = block * s.block + group * s.tile, last = min(first + s.tile, s.n);
  if (count && first < last) {
    bool head = first > 0 && s.key[first - 1] == s.key[first];
    float8 sum = 0.0f;
    for (uint32_t j = first; j < last; j += kTileStep) {
      uint32_t key[kTileStep + 1], token[kTileStep];
#pragma unroll
      for (uint32_t u = 0; u < kTileStep; ++u) {
        key[u] = s.key[j + u];
        token[u] = s.token[j + u];
      }
      key[kTileStep] = j + kTileStep < s.n ? s.key[j + kTileStep] : ~0u;
      if (key[0] >= vocab) break;
      typename Packed<In>::type v[kTileStep];
#pragma unroll
      for (uint32_t u = 0; u < kTileStep; ++u)
        if (j + u < last && key[u] < vocab)
          v[u] = load_some((const In*)grad_out.data + row_offset(grad_out, token[u]) + col, count);
#pragma unroll
      for (uint32_t u = 0; u < kTileStep; ++u) {
        if (j + u >= last || key[u] >= vocab) break;
        sum += widen8<In>(v[u]);
        const bool goes_on = j + u + 1 < s.n && key[u + 1] == key[u];
        if (goes_on && j + u + 1 < last) continue;
        if (head || goes_on) part[head ? 0 : 1][threadIdx.x] = sum;
        else write_sum<Out>(grad, key[u], col, count, sum, scale, accumulate);
        head = false;
        sum = 0.0f;
      }
    }
  }
  __syncthreads();
  if (group || !count) return;
  // The first group goes through the tiles and puts together what crosses them; what crosses the
  // block's ends is left to tile_join_kernel.
  float* out = s.parts + (uint64_t)block * 2 * s.stride + col;
  float8 sum = 0.0f;
  bool open = false, began_before = false;
  for (uint32_t g = 0, a = first; a < block_end; ++g, a += s.tile) {
    const uint32_t b = min(a + s.tile, block_end), k0 = s.key[a], k1 = s.key[b - 1];
    if (k0 >= vocab) break;
    const uint32_t mine = (g << s.shift) + threadIdx.x;
    const bool head = a > 0 && s.key[a - 1] == k0, goes_on = k1 < vocab && b < s.n && s.key[b] == k1;
    if (head) {
      if (g == 0) began_before = true;
      sum += part[0][mine];
      open = true;
      if (k0 == k1 && goes_on) continue;   // the whole tile
      if (began_before) store8(out, sum);
      else write_sum<Out>(grad, k0, col, count, sum, scale, accumulate);
      open = began_before = false;
      sum = 0.0f;
    }
    if (goes_on) {
      sum = part[1][mine];
      open = true;
    }
  }
  if (open) store8(out + (began_before ? 0 : s.stride), sum);
}

// Adds the parts of a sum that crosses blocks: a workgroup for every block in which one begins and
// does not end, its four wavefronts a quarter of the parts each.
template <typename Out>
__global__ void __launch_bounds__(256)
tile_join_kernel(TileView s, uint32_t width, float scale, bool accumulate, themis_rows_t grad, uint32_t vocab) {
  __shared__ float8 quarter[3][64];
  const uint32_t block = blockIdx.x, first = block * s.block, next = first + s.block;
  if (next >= s.n) return;
  const uint32_t v = s.key[next - 1];
  if (v >= vocab || s.key[next] != v) return;
  if (first > 0 && s.key[first - 1] == v) return;   // it began before
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
  // The blocks behind this one that it reaches into: those whose first key is v.  Every lane looks
  // at one of 64 places, which are nearer to each other each time.
  uint32_t lo = block + 1, hi = s.blocks;   // block lo is one, block hi (if there is one) is none
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo + 63) / 64;
    const uint64_t at = (uint64_t)lo + (uint64_t)lane * step;
    const uint64_t in = __ballot(at < hi && s.key[at * s.block] == v);   // (lane 0 is always in)
    const uint32_t reach = 64 - (uint32_t)__builtin_clzll(in);           // the first place that is not
    const uint32_t new_lo = lo + (reach - 1) * step;
    hi = min(hi, new_lo + step);
    lo = new_lo;
  }
  const uint32_t terms = lo - block + 1;
  const uint32_t col = (blockIdx.y * 64u + lane) * kVec;
  const bool on = col < width;
  const uint32_t each = (terms + 3) / 4, begin = min(wave * each, terms), end = min(begin + each, terms);
  float8 sum = 0.0f;
  if (on) {
#pragma unroll 8
    for (uint32_t p = begin; p < end; ++p)
      sum += load8(s.parts + ((uint64_t)(block + p) * 2 + (p == 0 ? 1 : 0)) * s.stride + col);
  }
  if (wave) quarter[wave - 1][lane] = sum;
  __syncthreads();
  if (wave || !on) return;
#pragma unroll
  for (int w = 0; w < 3; ++w) sum += quarter[w][lane];
  write_sum<Out>(grad, v, col, min(width - col, (uint32_t)kVec), sum, scale, accumulate);
}

}  // namespace themis
