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
// all that there is to hide.  Bound by memory: 65,536 rows of 4,096 bf16 (0.70 GB with each table row
// once) in 133 us, 5.3 TB/s, where a copy of 4 GiB makes 4.8 and one of 128 MiB 7.2; a few rows take
// the time of a launch.
// ---------------------------------------------------------------------------
template <bool kWhole, int kRows, typename In, typename Out, int kVec>
__device__ __forceinline__ void lookup_rows(const Slice<kVec>& slice, const Rows& table, uint32_t vocab, const Rows& ids,
                                            uint32_t n, float scale, const Rows& out, uint32_t t0, uint32_t groups) {
  uint32_t token[kRows], row[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) token[k] = min(t0 + k * groups, n - 1u);
  token_rows(ids, token, vocab, row);
  typename Packed<In, 8>::type v[kRows];
  if (vocab) {
#pragma unroll
    for (int k = 0; k < kRows; ++k)   // (row 0 in the place of none: its values are not used)
      v[k] = slice.template read<kWhole>(row_at<const In>(table, row[k] == ~0u ? 0u : row[k]));
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const uint32_t t = t0 + k * groups;
    if (t >= n) break;
    const float8 nan = __builtin_nanf("");
    const float8 x = row[k] != ~0u ? widen<8>(v[k]) * scale : nan;
    slice.template write_over<kWhole, (kRows > 1)>(row_at<Out>(out, t), x);
  }
}

template <bool kWhole, typename In, typename Out, int kRows>
__global__ void __launch_bounds__(256)
lookup_kernel(Rows table, uint32_t vocab, uint32_t width, Rows ids, uint32_t n, float scale, Rows out, uint32_t shift) {
  const uint32_t lanes = 1u << shift;
  const Slice<kVecOf<In, Out>> slice(blockIdx.y * 256u * kLaneElements, threadIdx.x & (lanes - 1u), lanes, width);
  if (!slice.any()) return;
  const uint32_t groups = 256u >> shift;   // rows side by side
  const uint32_t step = groups * kRows;
  for (uint64_t first = (uint64_t)blockIdx.x * step; first < n; first += (uint64_t)gridDim.x * step) {
    const uint32_t t0 = (uint32_t)first + (threadIdx.x >> shift);   // (below 2^32: n is below 2^31)
    lookup_rows<kWhole, kRows, In, Out>(slice, table, vocab, ids, n, scale, out, t0, groups);
  }
}

// ---------------------------------------------------------------------------
// themis_embedding_grad: grad[v] (+)= scale * sum of grad_out[t] over ids[t] == v.
//
// Up to kFewTokens tokens: one launch, no workspace.  A workgroup for every token finds all tokens
// of its number; the workgroups of one number share the row's elements (a token that occurs often
// has many), and the lanes of a workgroup the elements and the tokens: G groups of lanes take a
// G-th of the tokens each, in order, and their sums are added in order.  Bound by the waits one after
// the other (number, numbers, rows, what they are added to) and, towards kFewTokens, by every
// workgroup's look at all numbers: added to a binary32 table, rows of 1,024, 512 tokens 5.4 us, 2,048
// 10.9, 4,096 23.5, where the sort below takes 20, 23 and 26.
// ---------------------------------------------------------------------------
constexpr uint32_t kFewTokens = 4096;
constexpr uint32_t kRowsInFlight = 8;
constexpr uint32_t kMostGroups = 32;
constexpr uint32_t kScan = 4;   // token numbers of a lane in flight

template <bool kWhole, typename In, int kVec>
__device__ __forceinline__ float8 sum_listed(const Slice<kVec>& slice, const Rows& grad_out, const uint16_t* list,
                                             uint32_t begin, uint32_t end) {
  float8 sum = 0.0f;
  uint32_t i = begin;
  for (; i + kRowsInFlight <= end; i += kRowsInFlight) {
    typename Packed<In, 8>::type v[kRowsInFlight];
#pragma unroll
    for (uint32_t u = 0; u < kRowsInFlight; ++u)
      v[u] = slice.template read<kWhole>(row_at<const In>(grad_out, list[i + u]));
#pragma unroll
    for (uint32_t u = 0; u < kRowsInFlight; ++u) sum += widen<8>(v[u]);
  }
#pragma unroll 2
  for (; i < end; ++i) sum += widen<8>(slice.template read<kWhole>(row_at<const In>(grad_out, list[i])));
  return sum;
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

// Zeros in a whole table, before the sums.  One store a lane: workgroups that end at once follow each
// other through memory, and nothing is waited for (1 GiB: 7.1 TB/s; in loops over 16 KiB to 1 MiB, or
// behind a look at whether a row is needed, 4 to 6).
__global__ void __launch_bounds__(256) clear_kernel(char* table, uint64_t bytes) {
  const uint64_t head = min((uint64_t)(-(uintptr_t)table & 15u), bytes), body = (bytes - head) / 16;
  uint4* to = (uint4*)(table + head);
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < body; i += (uint64_t)gridDim.x * 256)
    to[i] = make_uint4(0, 0, 0, 0);
  if (blockIdx.x) return;   // what is not aligned to 16 bytes
  if (threadIdx.x < head) table[threadIdx.x] = 0;
  const uint64_t rest = head + body * 16 + threadIdx.x;
  if (rest < bytes) table[rest] = 0;
}
// The same, rows that do not follow each other: 2^shift lanes a row, or 4 KiB of one.
template <bool kWhole, typename Out>
__global__ void __launch_bounds__(256)
clear_rows_kernel(Rows table, uint32_t width, uint32_t vocab, uint32_t shift) {
  constexpr int kVec = kVecOf<Out>;
  for (uint64_t c = ((uint64_t)blockIdx.y * 256u + (threadIdx.x & ((1u << shift) - 1u))) * kVec; c < width;
       c += (uint64_t)gridDim.y * 256u * kVec)
    for (uint64_t v = (uint64_t)blockIdx.x * (256u >> shift) + (threadIdx.x >> shift); v < vocab;
         v += (uint64_t)gridDim.x * (256u >> shift))
      Access<kVec>((uint32_t)c, width)
          .template write_over<kWhole, false>(row_at<Out>(table, (uint32_t)v), Floats<kVec>(0.0f));
}

template <bool kWhole, int kVec, typename Out>
__device__ __forceinline__ void write_sum(const Rows& grad, uint32_t v, const Slice<kVec>& slice, float8 sum, float scale,
                                          bool accumulate) {
  Out* to = row_at<Out>(grad, v);
  float8 x = sum * scale;
  if (accumulate) x = widen<8>(slice.template read<kWhole>((const Out*)to)) + x;
  slice.template write<kWhole>(to, x);
}

// The last n workgroups: the tokens; the others write the zeros of up to 64 rows at a time.
template <bool kWhole, typename In, typename Out>
__global__ void __launch_bounds__(256)
few_tokens_kernel(uint32_t n, Rows grad_out, uint32_t width, Rows ids, float scale, uint32_t ignored, bool accumulate,
                  Rows grad, uint32_t vocab, uint32_t fill_rows) {
  __shared__ uint64_t masks[kFewTokens / 64];   // which tokens, 64 each
  __shared__ uint16_t list[kFewTokens];
  __shared__ float8 part[256];
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t chunks = (n + 63) / 64;
  const uint32_t fills = gridDim.x - n;
  // (the zeros before the tokens, which wait more than they write: 4,096 of 1,024 42 us, behind 49)
  const bool is_fill = blockIdx.x < fills;
  const uint32_t number = is_fill ? blockIdx.x : blockIdx.x - fills;
  if (is_fill) {
    if (blockIdx.y) return;
    const uint64_t step = (uint64_t)fills * fill_rows;
    for (uint64_t v = (uint64_t)number * fill_rows; v < vocab; v += step) {
      const uint32_t v0 = (uint32_t)v, rows = min(vocab - v0, fill_rows);
      __syncthreads();
      if (threadIdx.x == 0) masks[0] = 0;
      __syncthreads();
      for (uint32_t t = threadIdx.x; t < n; t += 256 * kScan) {
        uint32_t token[kScan], found[kScan];
#pragma unroll
        for (uint32_t k = 0; k < kScan; ++k) token[k] = min(t + k * 256, n - 1u);
        token_rows(ids, token, vocab, found);
#pragma unroll
        for (uint32_t k = 0; k < kScan; ++k) {
          const uint32_t at = found[k] - v0;
          if (t + k * 256 < n && found[k] >= v0 && at < rows && found[k] != ignored)
            atomicOr((unsigned long long*)&masks[0], 1ull << at);
        }
      }
      __syncthreads();
      const uint64_t all = rows == 64 ? ~0ull : (1ull << rows) - 1;
      write_zeros<kWhole, false, Out>(all & ~masks[0], v0, width, grad);
    }
    return;
  }
  const uint32_t t = number, id = token_row(ids, t, vocab);
  if (id == ~0u || id == ignored) return;
  for (uint32_t c = wave * kScan; c < chunks; c += 4 * kScan) {
    uint32_t at[kScan], found[kScan];
#pragma unroll
    for (uint32_t k = 0; k < kScan; ++k) at[k] = min((c + k) * 64 + lane, n - 1u);
    token_rows(ids, at, vocab, found);
#pragma unroll
    for (uint32_t k = 0; k < kScan; ++k) {
      const uint64_t mine = __ballot((c + k) * 64 + lane < n && found[k] == id);
      if (lane == 0 && c + k < chunks) masks[c + k] = mine;
    }
  }
  __syncthreads();
  const uint64_t mask = lane < chunks ? masks[lane] : 0ull;
  uint32_t upto = (uint32_t)__popcll(mask);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(upto, d);
    if (lane >= (uint32_t)d) upto += y;
  }
  const uint32_t before = upto - (uint32_t)__popcll(mask);
  const uint32_t count = __builtin_amdgcn_readlane(upto, 63);
  const uint32_t rank = __builtin_amdgcn_readlane(before, t / 64) +
                        (uint32_t)__popcll(masks[t / 64] & ((1ull << (t & 63u)) - 1));
  // Groups of lanes: as many as there are tokens, a power of two.
  const uint32_t more = 31 - (uint32_t)__builtin_clz(min(count, kMostGroups));
  const uint32_t groups = 1u << more, shift = 8 - more, lanes = 1u << shift;
  const uint32_t slices = (width + lanes * kLaneElements - 1) / (lanes * kLaneElements);
  if (rank + count * blockIdx.y >= slices) return;
  for (uint32_t c = wave; c < chunks; c += 4) {
    const uint64_t m = masks[c];
    const uint32_t at = __builtin_amdgcn_readlane(before, c);
    if ((m >> lane) & 1u) list[at + (uint32_t)__popcll(m & ((1ull << lane) - 1))] = (uint16_t)(c * 64 + lane);
  }
  __syncthreads();
  const uint32_t group = threadIdx.x >> shift, each = (count + groups - 1) / groups;
  const uint32_t begin = min(group * each, count), end = min(begin + each, count);
  for (uint32_t k = rank + count * blockIdx.y; k < slices; k += count * gridDim.y) {
    constexpr int kVec = kVecOf<In>;
    const Slice<kVec> slice(k * lanes * kLaneElements, threadIdx.x & (lanes - 1u), lanes, width);
    float8 sum = 0.0f;
    if (slice.any()) sum = sum_listed<kWhole, In>(slice, grad_out, list, begin, end);
    if (groups > 1) {
      part[threadIdx.x] = sum;
      __syncthreads();
      if (group == 0)
        for (uint32_t g = 1; g < groups; ++g) sum += part[(g << shift) + threadIdx.x];
    }
    if (group == 0 && slice.any()) write_sum<kWhole, kVec, Out>(grad, id, slice, sum, scale, accumulate);
    if (groups > 1) __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// More tokens: they are sorted by their number, stable, so that a table row's tokens stand next to
// each other in ascending order; the sorted list is cut into tiles of one length, whatever the
// numbers are, so that a token that makes up half of the list costs no more than any other half.  A
// tile adds its rows one after the other and writes the sums that begin and end in it.  A sum that
// crosses tiles is left in parts, which are added in the order of the tiles.
//
// Sort: least significant digit first, up to ten bits a pass and two launches: every workgroup
// counts the digits of its part of the list, then every workgroup finds from all counts where its
// part's tokens go.  A token's key is its number, or `vocab` (behind all others) if it has no
// gradient.  Bound by waits: of 16,384 tokens the four launches take 20 us, of 131,072 27 us.
//
// Sums: bound by memory and, a step of eight tokens after the other, by the waits for keys, then rows.
// 131,072 tokens of 2,048 bf16 added to 65,536 binary32 rows (0.96 GB) take 222 us without the sort,
// 4.3 TB/s, where a plain pass of three reads and a write makes 5.95; 16,384 tokens of 4,096 into a
// cleared table of 131,072 rows 61 (2.9 TB/s).
// A tile is 32 tokens: with 16 more sums cross tiles (65,537 tokens, half of them one number: 113 us,
// 107), with 64 the longest workgroups end late (131,072 tokens of 1,024 131 us, 122).
// ---------------------------------------------------------------------------
constexpr uint32_t kMaxBins = 1024;
constexpr uint32_t kSortGroup = 1024, kSortWaves = kSortGroup / 64;
constexpr uint32_t kSortAhead = 2;      // keys of a lane in flight
constexpr uint32_t kCountsAhead = 16;   // counts

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

// Keys of the places i[] of the list.
template <int kKeys>
__device__ __forceinline__ void sort_keys(const SortView& s, const Rows& ids, uint32_t vocab, uint32_t ignored,
                                          const uint32_t (&i)[kKeys], uint32_t (&key)[kKeys]) {
  if (s.key_in) {
#pragma unroll
    for (int k = 0; k < kKeys; ++k) key[k] = s.key_in[i[k]];
    return;
  }
  token_rows(ids, i, vocab, key);
#pragma unroll
  for (int k = 0; k < kKeys; ++k) key[k] = key[k] == ~0u || key[k] == ignored ? vocab : key[k];
}

// One more of `digit` in `bins`, for every lane that is on.  (Lanes with the first lane's digit go
// together: a token that makes up half of the list would be added one lane at a time.)
__device__ __forceinline__ void count_digit(uint32_t* bins, uint32_t digit, bool on) {
  const uint64_t all = __ballot(on);
  if (!all) return;
  const uint32_t first = __builtin_amdgcn_readlane(digit, (uint32_t)__builtin_ctzll(all));
  const uint64_t same = __ballot(on && digit == first);
  if ((threadIdx.x & 63u) == (uint32_t)__builtin_ctzll(all)) atomicAdd(&bins[first], (uint32_t)__popcll(same));
  if (on && digit != first) atomicAdd(&bins[digit], 1u);
}

__global__ void __launch_bounds__(kSortGroup)
sort_count_kernel(SortView s, Rows ids, uint32_t vocab, uint32_t ignored) {
  __shared__ uint32_t count[kMaxBins];
  const uint32_t bins = 1u << s.bits, first = blockIdx.x * s.part;
  const uint32_t last = min(first + s.part, s.n), lane = threadIdx.x & 63u;
  for (uint32_t b = threadIdx.x; b < bins; b += kSortGroup) count[b] = 0;
  __syncthreads();
  for (uint32_t i = first + threadIdx.x; i - lane < last; i += kSortAhead * kSortGroup) {
    uint32_t at[kSortAhead], key[kSortAhead];
#pragma unroll
    for (uint32_t k = 0; k < kSortAhead; ++k) at[k] = min(i + k * kSortGroup, last - 1u);
    sort_keys(s, ids, vocab, ignored, at, key);
#pragma unroll
    for (uint32_t k = 0; k < kSortAhead; ++k) {
      if (i - lane + k * kSortGroup >= last) break;   // (the wavefront's first)
      count_digit(count, (key[k] >> s.shift) & (bins - 1), i + k * kSortGroup < last);
    }
  }
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < bins; b += kSortGroup) s.counts[blockIdx.x * bins + b] = count[b];
}

__global__ void __launch_bounds__(kSortGroup)
sort_move_kernel(SortView s, Rows ids, uint32_t vocab, uint32_t ignored) {
  __shared__ uint32_t place[kSortWaves][kMaxBins];   // first a wavefront's counts, then where its next one goes
  __shared__ uint32_t wave_sums[kSortWaves];
  const uint32_t bins = 1u << s.bits, first = blockIdx.x * s.part;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
  const uint32_t share = s.part / kSortWaves;   // a wavefront's tokens stand together (a multiple of 64)
  const uint32_t begin = min(first + wave * share, s.n), end = min(begin + share, s.n);
  const uint32_t b = threadIdx.x;               // a lane has one digit, or none
  if (b < bins)
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) place[w][b] = 0;
  __syncthreads();
  for (uint32_t i = begin; i < end; i += kSortAhead * 64) {
    uint32_t at[kSortAhead], key[kSortAhead];
#pragma unroll
    for (uint32_t k = 0; k < kSortAhead; ++k) at[k] = min(i + k * 64 + lane, end - 1u);
    sort_keys(s, ids, vocab, ignored, at, key);
#pragma unroll
    for (uint32_t k = 0; k < kSortAhead; ++k) {
      if (i + k * 64 >= end) break;
      count_digit(place[wave], (key[k] >> s.shift) & (bins - 1), i + k * 64 + lane < end);
    }
  }
  // Where a digit's tokens of this part go: behind all of smaller digits and those of the parts before.
  uint32_t before = 0, all = 0;
  if (b < bins) {
    for (uint32_t p = 0; p < s.parts; p += kCountsAhead) {
      uint32_t c[kCountsAhead];
#pragma unroll
      for (uint32_t k = 0; k < kCountsAhead; ++k) c[k] = s.counts[min(p + k, s.parts - 1u) * bins + b];
#pragma unroll
      for (uint32_t k = 0; k < kCountsAhead; ++k) {
        before += p + k < blockIdx.x ? c[k] : 0u;
        all += p + k < s.parts ? c[k] : 0u;
      }
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
  for (uint32_t i0 = begin; i0 < end; i0 += kSortAhead * 64) {
    uint32_t from[kSortAhead], keys[kSortAhead], tokens[kSortAhead];
#pragma unroll
    for (uint32_t k = 0; k < kSortAhead; ++k) from[k] = min(i0 + k * 64 + lane, end - 1u);
    sort_keys(s, ids, vocab, ignored, from, keys);
#pragma unroll
    for (uint32_t k = 0; k < kSortAhead; ++k) tokens[k] = s.key_in ? s.token_in[from[k]] : from[k];
#pragma unroll
    for (uint32_t k = 0; k < kSortAhead; ++k) {
      if (i0 + k * 64 >= end) break;
      const bool on = i0 + k * 64 + lane < end;
      const uint32_t digit = (keys[k] >> s.shift) & (bins - 1);
      uint64_t same = __ballot(on);   // lanes with this lane's digit
      for (uint32_t b = 0; b < s.bits; ++b) {
        const uint64_t ones = __ballot((digit >> b) & 1u);
        same &= (digit >> b) & 1u ? ones : ~ones;
      }
      const uint32_t rank = (uint32_t)__popcll(same & ((1ull << lane) - 1));
      // (all lanes have read before the first of a digit's adds: a wavefront's accesses to LDS are
      // served in the order of the program, and these are kept in it)
      uint32_t* next = &place[wave][digit];
      const uint32_t to = (on ? __hip_atomic_load(next, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) : 0u) + rank;
      if (on && rank == 0)
        __hip_atomic_store(next, to + (uint32_t)__popcll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      if (on) {
        s.key_out[to] = keys[k];
        s.token_out[to] = tokens[k];
      }
    }
  }
}

// The sorted list in tiles, one for every group of lanes of a workgroup (a wavefront, less where the
// rows are short), and the tiles of a workgroup in blocks.
struct TileView {
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
enum : uint32_t { kHead = 1, kOneSum = 2, kGoesOn = 4 };

// Zeros in those of up to 64 table rows from `v0` on that no token has: a lane looks for its row.
template <bool kWhole, typename Out>
__device__ __forceinline__ void fill_rows(const TileView& s, const uint32_t* keys, uint32_t v0, uint32_t width,
                                          const Rows& grad, uint32_t vocab) {
  const uint32_t lane = threadIdx.x & 63u, v = v0 + lane;
  const bool mine = lane < s.fill_rows && v < vocab;
  uint32_t lo = 0, hi = mine ? s.n : 0u;   // the first key that is not smaller
  while (__any(lo < hi)) {
    if (lo < hi) {
      const uint32_t mid = lo + ((hi - lo) >> 1);
      if (keys[mid] < v) lo = mid + 1;
      else hi = mid;
    }
  }
  write_zeros<kWhole, true, Out>(__ballot(mine && (lo >= s.n || keys[lo] != v)), v0, width, grad);
}

// A tile's sums: those that begin and end in it to the table, the others to `head` (one that began
// before) and `tail`.
template <bool kWhole, typename In, typename Out, int kVec>
__device__ __forceinline__ void sum_tile(const TileView& s, const uint32_t* __restrict__ keys,
                                         const uint32_t* __restrict__ tokens, const Slice<kVec>& slice,
                                         const Rows& grad_out, float scale, bool accumulate, const Rows& grad,
                                         uint32_t vocab, uint32_t first, uint32_t last, float8& head, float8& tail) {
  bool before = first > 0 && keys[first - 1] == keys[first];
  float8 sum = 0.0f;
  for (uint32_t j = first; j < last; j += kTileStep) {
    // (the lists are longer than n by a step; what stands there is not used)
    const uint32_t *key_at = keys + j, *token_at = tokens + j;
    uint32_t key[kTileStep + 1], token[kTileStep];
#pragma unroll
    for (uint32_t u = 0; u < kTileStep; ++u) {
      key[u] = key_at[u];
      token[u] = token_at[u];
    }
    key[kTileStep] = j + kTileStep < s.n ? keys[j + kTileStep] : ~0u;
    uint32_t some = min(last - j, kTileStep);
    if (some == kTileStep && key[kTileStep - 1] < vocab) {
      typename Packed<In, 8>::type v[kTileStep];
#pragma unroll
      for (uint32_t u = 0; u < kTileStep; ++u) v[u] = slice.template read<kWhole>(row_at<const In>(grad_out, token[u]));
      // (what the sums that end here are added to is asked for at the same time: 131,072 tokens of
      // 1,024, spread evenly, added to 131,072 bf16 rows 171 -> 162 us)
      typename Packed<Out, 8>::type held[kTileStep];
      if (accumulate) {
#pragma unroll
        for (uint32_t u = 0; u < kTileStep; ++u)
          if (key[u + 1] != key[u]) held[u] = slice.template read<kWhole>(row_at<const Out>(grad, key[u]));
      }
#pragma unroll
      for (uint32_t u = 0; u < kTileStep; ++u) {
        sum += widen<8>(v[u]);
        const bool goes_on = key[u + 1] == key[u];
        if (goes_on && j + u + 1 < last) continue;
        if (before) {
          head = sum;
        } else if (goes_on) {
          tail = sum;
        } else {
          float8 x = sum * scale;
          if (accumulate) x = widen<8>(held[u]) + x;
          slice.template write<kWhole>(row_at<Out>(grad, key[u]), x);
        }
        before = false;
        sum = 0.0f;
      }
    } else {   // the list's end, or the first tokens without a gradient
      for (uint32_t u = 0; u < some; ++u) {
        const uint32_t k = keys[j + u];
        if (k >= vocab) return;
        sum += widen<8>(slice.template read<kWhole>(row_at<const In>(grad_out, tokens[j + u])));
        const bool goes_on = j + u + 1 < s.n && keys[j + u + 1] == k;
        if (goes_on && j + u + 1 < last) continue;
        if (before) head = sum;
        else if (goes_on) tail = sum;
        else write_sum<kWhole, kVec, Out>(grad, k, slice, sum, scale, accumulate);
        before = false;
        sum = 0.0f;
      }
    }
  }
}

// kWave: a wavefront for every tile, all of whose lanes go the same way.
template <bool kWhole, typename In, typename Out, bool kWave>
__global__ void __launch_bounds__(256)
tile_sum_kernel(TileView s, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ tokens, Rows grad_out,
                uint32_t width, float scale, bool accumulate, Rows grad, uint32_t vocab) {
  // A group's sums that its tile does not hold whole: of one that began before, of one that goes on.
  __shared__ float8 part[2][256];
  __shared__ uint32_t tile_key[32];     // a tile's first key
  __shared__ uint32_t tile_is[32];      // kHead | kOneSum | kGoesOn
  const uint32_t sums = s.blocks * s.slabs, fills = gridDim.x - sums;
  // (the zeros behind the sums: 65,537 tokens of 1,000 109 us, before them 120, among them 112)
  const bool is_fill = blockIdx.x >= sums;
  const uint32_t number = is_fill ? blockIdx.x - sums : blockIdx.x;
  if (is_fill) {
    const uint64_t step = (uint64_t)fills * s.fill_rows;
    for (uint64_t v = (uint64_t)number * s.fill_rows; v < vocab; v += step)
      fill_rows<kWhole, Out>(s, keys, (uint32_t)v, width, grad, vocab);
    return;
  }
  const uint32_t shift = kWave ? 6u : s.shift, lanes = 1u << shift;
  const uint32_t block = number / s.slabs, slab = number - block * s.slabs;
  const uint32_t group = kWave ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x >> shift;
  constexpr int kVec = kVecOf<In, Out>;
  const Slice<kVec> slice(slab * 512u, threadIdx.x & (lanes - 1u), lanes, width);
  const uint32_t block_end = min(block * s.block + s.block, s.n);
  const uint32_t first = block * s.block + group * s.tile, last = min(first + s.tile, s.n);
  if (slice.any() && first < last) {
    float8 head = 0.0f, tail = 0.0f;
    sum_tile<kWhole, In, Out>(s, keys, tokens, slice, grad_out, scale, accumulate, grad, vocab, first, last, head, tail);
    part[0][threadIdx.x] = head;
    part[1][threadIdx.x] = tail;
    if ((threadIdx.x & (lanes - 1u)) == 0) {
      const uint32_t k0 = keys[first], k1 = keys[last - 1];
      tile_key[group] = k0;
      tile_is[group] = (first > 0 && keys[first - 1] == k0 ? kHead : 0u) | (k0 == k1 ? kOneSum : 0u) |
                       (k1 < vocab && last < s.n && keys[last] == k1 ? kGoesOn : 0u);
    }
  }
  __syncthreads();
  if (!slice.any() || first >= last) return;
  // What crosses tiles is put together by the group in whose tile it ends; what crosses the block's
  // ends is left to tile_join_kernel.
  const uint32_t is = tile_is[group], own = threadIdx.x & (lanes - 1u);
  const bool ends = (is & kHead) && (is & (kOneSum | kGoesOn)) != (kOneSum | kGoesOn);
  const bool leaves = (is & kGoesOn) && last == block_end;
  if (tile_key[group] >= vocab || !(ends || leaves)) return;
  uint32_t from = group;   // the tile it begins in, or the block's first
  bool before = is & kHead;
  while (before && from > 0) before = (tile_is[--from] & (kHead | kOneSum)) == (kHead | kOneSum);
  float8 sum = 0.0f;
  if (is & kHead) {
    sum = part[before ? 0 : 1][(from << shift) + own];
    for (uint32_t g = from + 1; g <= group; ++g) sum += part[0][(g << shift) + own];
  }
  float* out = s.parts + (uint64_t)block * 2 * s.stride + (slab * 64u + own) * kLaneElements;
  if (ends) {
    if (before) store<8>(out, sum);
    else write_sum<kWhole, kVec, Out>(grad, tile_key[group], slice, sum, scale, accumulate);
  }
  if (leaves) {
    const bool own_tail = !(is & kHead) || ends;   // it began in this tile
    if (own_tail) sum = part[1][threadIdx.x];
    store<8>(out + (before && !own_tail ? 0 : s.stride), sum);
  }
}

// Adds the parts of a sum that crosses blocks: a workgroup for every block in which one begins and
// does not end, its wavefronts a share of the parts each, in order.  (Eight wavefronts, which wait for
// few parts each where one token has many; four where there are so many workgroups that these end one
// after the other: 65,537 tokens, half of them one number, 102 us with eight and 105 with four; the
// joins of 131,072 tokens of 4,096 37 us and 24.)
template <bool kWhole, int kVec, typename Out, int kWaves>
__global__ void __launch_bounds__(kWaves * 64)
tile_join_kernel(TileView s, const uint32_t* __restrict__ keys, uint32_t width, float scale, bool accumulate, Rows grad,
                 uint32_t vocab) {
  __shared__ float8 share[kWaves - 1][64];
  const uint32_t block = blockIdx.x, first = block * s.block, next = first + s.block;
  if (next >= s.n) return;
  const uint32_t after = min(next + s.block, s.n - 1u);   // (the block behind the next begins here, if there is one)
  const uint32_t v = keys[next - 1], v_next = keys[next], v_after = keys[after], v_before = keys[first > 0 ? first - 1 : 0];
  if (v >= vocab || v_next != v) return;
  if (first > 0 && v_before == v) return;   // it began before
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
  // The blocks behind this one that it reaches into, those whose first key is v: mostly one.  Where
  // there are more every lane looks at one of 64 places, which are nearer to each other each time.
  uint32_t lo = block + 1, hi = s.blocks;   // block lo is one, block hi (if there is one) is none
  if (v_after != v) hi = lo + 1;
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo + 63) / 64;
    const uint64_t at = (uint64_t)lo + (uint64_t)lane * step;
    const uint64_t in = __ballot(at < hi && keys[at * s.block] == v);   // (lane 0 is always in)
    const uint32_t reach = 64 - (uint32_t)__builtin_clzll(in);           // the first place that is not
    const uint32_t new_lo = lo + (reach - 1) * step;
    hi = min(hi, new_lo + step);
    lo = new_lo;
  }
  const uint32_t terms = lo - block + 1;
  const Slice<kVec> slice(blockIdx.y * 512u, lane & ((1u << s.shift) - 1u), 1u << s.shift, width);
  const bool on = lane >> s.shift == 0 && slice.any();
  const uint32_t each = (terms + kWaves - 1) / kWaves, begin = min(wave * each, terms), end = min(begin + each, terms);
  float8 sum = 0.0f;
  if (on) {
#pragma unroll 8
    for (uint32_t p = begin; p < end; ++p)
      sum += load<8>(s.parts + ((uint64_t)(block + p) * 2 + (p == 0 ? 1 : 0)) * s.stride +
                     (blockIdx.y * 64u + lane) * kLaneElements);
  }
  if (wave) share[wave - 1][lane] = sum;
  __syncthreads();
  if (wave || !on) return;
#pragma unroll
  for (uint32_t w = 0; w < kWaves - 1; ++w) sum += share[w][lane];
  write_sum<kWhole, kVec, Out>(grad, v, slice, sum, scale, accumulate);
}

}  // namespace themis
