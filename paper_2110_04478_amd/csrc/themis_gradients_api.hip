// C ABI of the gradient operators (see include/themis.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "themis.h"
#include "themis_elements.hpp"
#include "themis_embedding.hpp"
#include "themis_gradient.hpp"
#include "themis_launch.hpp"

namespace themis {
namespace {

constexpr uint64_t kMostTensors = 1u << 24;

// How a gradient of the table is worked out, and what is where in its workspace (bytes).
struct GradLayout {
  uint32_t passes, bits;           // of the sort
  uint32_t part, sort_parts;       // tokens of a workgroup, workgroups
  uint32_t tile, block, blocks, slabs, shift, stride;
  size_t key[2], token[2], counts, parts, bytes;
};

GradLayout grad_layout(uint32_t n, uint32_t width, uint32_t vocab) {
  GradLayout l = {};
  if (n <= kFewTokens) return l;
  const uint32_t bits = next_power(vocab + 1);   // keys 0 .. vocab
  l.passes = (bits + 9) / 10;
  l.bits = (bits + l.passes - 1) / l.passes;
  // A workgroup of the sort takes kSortGroup tokens in a turn, and reads the counts of all parts, 16 at
  // a time: up to 40 parts for every turn (131,072 tokens: 9.6 us a move; with 20 11.4, with 80 9.7).
  l.part = kSortGroup;
  while ((uint64_t)n > (uint64_t)l.part * (40 * (l.part / kSortGroup))) l.part *= 2;
  l.sort_parts = (n + l.part - 1) / l.part;
  const uint32_t vecs = (width + kLaneElements - 1) / kLaneElements;
  l.shift = std::max(std::min(next_power(vecs), 6u), kLeastShift);
  l.slabs = (vecs + 63) / 64;
  l.stride = l.slabs * 512;
  // Tiles: 32 tokens, fewer where that leaves less than four wavefronts for every SIMD.
  l.tile = 32;
  while (l.tile > 8 && (((uint64_t)n + l.tile - 1) / l.tile * l.slabs << l.shift) / 64 < 4096) l.tile /= 2;
  l.block = l.tile * (256u >> l.shift);
  l.blocks = (n + l.block - 1) / l.block;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  const size_t list = ((size_t)n + kTileStep) * sizeof(uint32_t);
  for (int k = 0; k < (l.passes > 1 ? 2 : 1); ++k) {
    l.key[k] = take(list);
    l.token[k] = take(list);
  }
  l.counts = take((size_t)l.sort_parts * (sizeof(uint32_t) << l.bits));
  l.parts = take((size_t)l.blocks * 2 * l.stride * sizeof(float));
  l.bytes = at;
  return l;
}

// What the grids of the sums and the joins hold: less than 2^32 lanes, 65,535 workgroups the other way.
bool grad_fits(const GradLayout& l) { return (uint64_t)l.blocks * l.slabs <= 1u << 23 && l.slabs <= 65535; }

void clear_table(Launches& go, const Rows& table, uint32_t width, uint32_t vocab) {
  if (table.inner == 0 && table.inner_stride == (int64_t)width) {
    const uint64_t bytes = (uint64_t)vocab * width * type_bytes(table.type);
    go(clear_kernel, dim3((uint32_t)std::min<uint64_t>((bytes + 4095) / 4096, (1u << 24) - 1)), 256, table.data, bytes);
    return;
  }
  const uint32_t vec = table.type == THEMIS_F32 ? 4 : 8, vecs = (width + vec - 1) / vec;
  const uint32_t shift = std::min(next_power(vecs), 8u), rows = 256u >> shift;
  with_type(table.type, [&](auto out) {
    const dim3 grid(std::min((vocab + rows - 1) / rows, (1u << 24) - 1), std::min((vecs + 255) / 256, 65535u));
    typedef decltype(out) Out;
    go(width < kLaneElements ? clear_rows_kernel<false, Out> : clear_rows_kernel<true, Out>, grid, 256, table, width,
       vocab, shift);
  });
}

// Whether zeros are written by a launch of their own before the sums, in all rows, or with the sums
// in those rows that no token has.  The first is the faster store, but writes the rows of the sums
// twice.  One token, 16 MiB: 9 us with the sums, 8 and another launch before; 128 MiB: 27 and 25;
// 1 GiB: 195 and 161.  16,384 tokens, 1 GiB in 131,072 rows: 246 and 235 us; 512 MiB in 65,536 rows:
// 145 and 162.  Rows that end inside a line share it with the next, whose zeros another workgroup
// writes: 16,384 tokens, 131 MB in 65,537 rows of 2,002 bytes 73 and 61 us, 65,536 tokens 89 and 107.
bool clears(uint64_t n, uint64_t vocab, uint64_t width, int type) {
  const uint64_t row = width * type_bytes(type), least = row % 128 ? 2 : 8;
  return n == 0 || (vocab * row > 64u << 20 && (n <= kFewTokens || vocab >= least * n));
}

}  // namespace
}  // namespace themis

using namespace themis;

extern "C" {

int themis_embedding_lookup(const themis_rows_t* table, uint64_t vocab, uint64_t width, const themis_rows_t* ids,
                            uint64_t n, float scale, const themis_rows_t* out, void* stream) {
  if (n == 0 || width == 0) return THEMIS_OK;
  if (!rows_ok(ids, true) || !rows_ok(out, false)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (!table || !is_float_type(table->type) || (vocab && !rows_ok(table, false))) return THEMIS_ERR_INVALID_ARGUMENT;
  if (n > kMost || width > kMost || vocab > kMost) return THEMIS_ERR_UNSUPPORTED;
  if (!rows_apart(*out, n, width)) return THEMIS_ERR_INVALID_ARGUMENT;
  const uint32_t vecs = (uint32_t)((width + kLaneElements - 1) / kLaneElements);
  const uint32_t shift = std::min(next_power(vecs), 8u), chunks = (vecs + 255) / 256;
  if (chunks > 65535) return THEMIS_ERR_UNSUPPORTED;
  Launches go(stream);
  auto run = [&](auto kernel, uint32_t rows) {
    const uint64_t step = (256u >> shift) * rows;
    const uint32_t blocks = (uint32_t)std::min<uint64_t>((n + step - 1) / step, 1u << 20);
    go(kernel, dim3(blocks, chunks), 256, rows_of(*table, vocab), (uint32_t)vocab, (uint32_t)width, rows_of(*ids, n),
       (uint32_t)n, scale, rows_of(*out, n), shift);
  };
  with_type(table->type, [&](auto in) {
    with_type(out->type, [&](auto to) {
      // Two rows a lane, written past the caches, where workgroups of one row would be sixteen for
      // every CU (65,536 rows of 4,096: with one 180 us, two 133, three 137, four 145).
      typedef decltype(in) In;
      typedef decltype(to) Out;
      if (width < kLaneElements) run(lookup_kernel<false, In, Out, 1>, 1);
      else if (n / (256u >> shift) * chunks >= 4096) run(lookup_kernel<true, In, Out, 2>, 2);
      else run(lookup_kernel<true, In, Out, 1>, 1);
    });
  });
  return go.status();
}

size_t themis_embedding_grad_workspace_bytes(uint64_t n, uint64_t width, uint64_t vocab) {
  if (n == 0 || width == 0 || vocab == 0 || n > kMost || width > kMost || vocab > kMost) return 0;
  const GradLayout l = grad_layout((uint32_t)n, (uint32_t)width, (uint32_t)vocab);
  return grad_fits(l) ? l.bytes : 0;
}

int themis_embedding_grad(const themis_rows_t* grad_out, uint64_t width, const themis_rows_t* ids, uint64_t n,
                          float scale, int64_t ignored, int accumulate, const themis_rows_t* grad, uint64_t vocab,
                          void* workspace, size_t workspace_bytes, void* stream) {
  if (width == 0 || vocab == 0 || (n == 0 && accumulate)) return THEMIS_OK;
  if (!rows_ok(grad, false)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (n && (!rows_ok(ids, true) || !rows_ok(grad_out, false))) return THEMIS_ERR_INVALID_ARGUMENT;
  if (n > kMost || width > kMost || vocab > kMost) return THEMIS_ERR_UNSUPPORTED;
  if (!rows_apart(*grad, vocab, width)) return THEMIS_ERR_INVALID_ARGUMENT;
  const GradLayout l = grad_layout((uint32_t)n, (uint32_t)width, (uint32_t)vocab);
  if (!grad_fits(l)) return THEMIS_ERR_UNSUPPORTED;
  if (l.bytes && (!workspace || workspace_bytes < l.bytes || !aligned(workspace, 16))) return THEMIS_ERR_WORKSPACE;
  const uint64_t sums = (uint64_t)l.blocks * l.slabs;
  const Rows g = n ? rows_of(*grad_out, n) : Rows{}, k = n ? rows_of(*ids, n) : Rows{}, to = rows_of(*grad, vocab);
  const uint32_t skip = ignored >= 0 && (uint64_t)ignored < vocab ? (uint32_t)ignored : ~0u;
  Launches go(stream);
  // (a workgroup's zeros: about 256 KiB, in up to 64 rows)
  const uint64_t row_bytes = width * type_bytes(to.type);
  const uint32_t fill_rows = (uint32_t)std::min<uint64_t>(64, std::max<uint64_t>(1, (256u << 10) / row_bytes));
  const bool clear = !accumulate && clears(n, vocab, width, to.type);
  const uint64_t fill = accumulate || clear ? 0 : std::min<uint64_t>((vocab + fill_rows - 1) / fill_rows, 1u << 20);
  if (clear) clear_table(go, to, (uint32_t)width, (uint32_t)vocab);
  if (n == 0) return go.status();
  if (n <= kFewTokens) {
    // (a row that one token has is 2,048 elements for a workgroup, of longer ones several while there are few)
    const uint32_t columns = (uint32_t)std::min<uint64_t>((width + 2047) / 2048, n < 1024 ? 1024 / n : 1);
    with_type(g.type, [&](auto in) {
      with_type(to.type, [&](auto out) {
        typedef decltype(in) In;
        typedef decltype(out) Out;
        go(width < kLaneElements ? few_tokens_kernel<false, In, Out> : few_tokens_kernel<true, In, Out>,
           dim3((uint32_t)(n + fill), columns), 256, (uint32_t)n, g, (uint32_t)width, k, scale, skip, accumulate != 0, to,
           (uint32_t)vocab, fill_rows);
      });
    });
    return go.status();
  }
  char* at = (char*)workspace;
  uint32_t *key[2] = {(uint32_t*)(at + l.key[0]), (uint32_t*)(at + l.key[1])};
  uint32_t *token[2] = {(uint32_t*)(at + l.token[0]), (uint32_t*)(at + l.token[1])};
  for (uint32_t pass = 0; pass < l.passes; ++pass) {
    SortView s;
    s.n = (uint32_t)n;
    s.part = l.part;
    s.parts = l.sort_parts;
    s.shift = pass * l.bits;
    s.bits = l.bits;
    s.counts = (uint32_t*)(at + l.counts);
    s.key_in = pass ? key[(pass - 1) & 1] : nullptr;
    s.token_in = pass ? token[(pass - 1) & 1] : nullptr;
    s.key_out = key[pass & 1];
    s.token_out = token[pass & 1];
    go(sort_count_kernel, dim3(s.parts), kSortGroup, s, k, (uint32_t)vocab, skip);
    go(sort_move_kernel, dim3(s.parts), kSortGroup, s, k, (uint32_t)vocab, skip);
  }
  TileView t;
  const uint32_t *keys = key[(l.passes - 1) & 1], *tokens = token[(l.passes - 1) & 1];
  t.n = (uint32_t)n;
  t.tile = l.tile;
  t.block = l.block;
  t.blocks = l.blocks;
  t.slabs = l.slabs;
  t.shift = l.shift;
  t.parts = (float*)(at + l.parts);
  t.stride = l.stride;
  t.fill_rows = fill_rows;
  with_type(g.type, [&](auto in) {
    with_type(to.type, [&](auto out) {
      typedef decltype(in) In;
      typedef decltype(out) Out;
      go(width < kLaneElements ? tile_sum_kernel<false, In, Out, false>
         : l.shift < 6         ? tile_sum_kernel<true, In, Out, false>
                               : tile_sum_kernel<true, In, Out, true>,
         dim3((uint32_t)(sums + fill)), 256, t, keys, tokens, g, (uint32_t)width, scale, accumulate != 0, to,
         (uint32_t)vocab);
      constexpr int kVec = kVecOf<In, Out>;
      auto join = [&](auto kernel, unsigned waves) {
        go(kernel, dim3(l.blocks - 1, l.slabs), waves * 64, t, keys, (uint32_t)width, scale, accumulate != 0, to,
           (uint32_t)vocab);
      };
      if (l.blocks < 2) return;
      if (width < kLaneElements) join(tile_join_kernel<false, kVec, Out, 8>, 8);
      else if (sums <= 2048) join(tile_join_kernel<true, kVec, Out, 8>, 8);
      else join(tile_join_kernel<true, kVec, Out, 4>, 4);
    });
  });
  return go.status();
}

int themis_gradient_plan(const themis_gradient_t* parts, uint64_t n_parts, uint64_t n_tensors,
                         themis_gradient_plan_t* plan, void* image, size_t image_bytes) {
  if (!plan || (n_parts && !parts)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (n_tensors > kMostTensors) return THEMIS_ERR_UNSUPPORTED;
  unsigned __int128 total = 0;
  uint64_t bytes = 0;
  bool has_out = true, strided = false;
  for (uint64_t i = 0; i < n_parts; ++i) {
    const themis_gradient_t& g = parts[i];
    if (g.tensor >= n_tensors || (i && g.tensor < parts[i - 1].tensor)) return THEMIS_ERR_INVALID_ARGUMENT;
    if (!is_float_type(g.in_type) || (g.out && !is_float_type(g.out_type))) return THEMIS_ERR_INVALID_ARGUMENT;
    const unsigned __int128 count = (unsigned __int128)g.rows * g.cols;
    if (!count) continue;
    if (!g.in || !aligned(g.in, type_bytes(g.in_type))) return THEMIS_ERR_INVALID_ARGUMENT;
    if (g.out && !aligned(g.out, type_bytes(g.out_type))) return THEMIS_ERR_INVALID_ARGUMENT;
    if (g.out == g.in && (g.in_type != g.out_type || g.in_row_stride != g.out_row_stride ||
                          g.in_col_stride != g.out_col_stride)) return THEMIS_ERR_INVALID_ARGUMENT;
    if (count >> 46) return THEMIS_ERR_UNSUPPORTED;
    if (g.out && !rows_apart({g.out, g.out_type, g.cols, g.out_row_stride, g.out_col_stride}, (uint64_t)count, 1))
      return THEMIS_ERR_INVALID_ARGUMENT;   // (an element written twice)
    has_out = has_out && g.out;
    total += count;
    bytes += (uint64_t)count * type_bytes(g.in_type);
  }
  if (total >> 46) return THEMIS_ERR_UNSUPPORTED;
  const uint64_t most = piece_elements((uint64_t)total);

  uint64_t n_pieces = 0;
  Piece* to = (Piece*)image;
  uint64_t room = 0;
  uint32_t* first = nullptr;
  auto walk = [&](bool write) {
    uint64_t at = 0, tensor = 0;
    for (uint64_t i = 0; i < n_parts; ++i) {
      const themis_gradient_t& g = parts[i];
      for (; write && tensor <= g.tensor; ++tensor) first[tensor] = (uint32_t)at;
      uint64_t rows = g.rows, cols = g.cols;
      if (!rows || !cols) continue;
      const bool in_run = rows == 1 || (g.in_row_stride == (int64_t)cols && g.in_col_stride == 1);
      const bool out_run = !g.out || rows == 1 || (g.out_row_stride == (int64_t)cols && g.out_col_stride == 1);
      if (in_run && out_run) { cols *= rows; rows = 1; }   // one row, each with its one stride
      strided = strided || rows > 1 || (cols > 1 && (g.in_col_stride != 1 || (g.out && g.out_col_stride != 1)));
      const uint64_t wide = std::min(cols, most), high = std::max<uint64_t>(most / wide, 1);
      for (uint64_t r = 0; r < rows; r += high)
        for (uint64_t c = 0; c < cols; c += wide, ++at) {
          if (!write) continue;
          Piece p;
          const uint64_t nr = std::min(high, rows - r), nc = std::min(wide, cols - c);
          const int64_t in_at = (int64_t)r * g.in_row_stride + (int64_t)c * g.in_col_stride;
          const int64_t out_at = (int64_t)r * g.out_row_stride + (int64_t)c * g.out_col_stride;
          p.in = (const char*)g.in + in_at * type_bytes(g.in_type);
          p.out = g.out ? (char*)g.out + out_at * type_bytes(g.out_type) : nullptr;
          p.count = (uint32_t)(nr * nc);
          p.cols = (uint32_t)nc;
          p.tensor = g.tensor;
          const bool one = nr == 1 || nc == cols;
          const bool in_dense = (g.in_col_stride == 1 || nc == 1) && (nr == 1 || (one && g.in_row_stride == (int64_t)nc));
          const bool out_dense = (g.out_col_stride == 1 || nc == 1) && (nr == 1 || (one && g.out_row_stride == (int64_t)nc));
          p.kind = (uint32_t)g.in_type | (uint32_t)(g.out ? g.out_type : 0) << 8 | (in_dense ? kInDense : 0) |
                   (out_dense ? kOutDense : 0) | (g.out == g.in ? kInPlace : 0);
          p.in_row = g.in_row_stride;
          p.in_col = g.in_col_stride;
          p.out_row = g.out_row_stride;
          p.out_col = g.out_col_stride;
          to[at] = p;
        }
    }
    for (; write && tensor <= n_tensors; ++tensor) first[tensor] = (uint32_t)at;
    n_pieces = at;
  };
  walk(false);
  if (n_pieces >= kMost) return THEMIS_ERR_UNSUPPORTED;
  room = n_pieces * sizeof(Piece) + (n_tensors + 1) * sizeof(uint32_t);
  plan->n_tensors = n_tensors;
  plan->n_pieces = n_pieces;
  plan->image_bytes = room;
  plan->workspace_bytes = (pass_groups(n_pieces, bytes) + n_pieces) * sizeof(double);
  plan->in_bytes = bytes;
  plan->has_out = has_out;
  plan->strided = strided;
  plan->image = nullptr;
  if (!image) return THEMIS_OK;
  if (image_bytes < room || !aligned(image, 8)) return THEMIS_ERR_WORKSPACE;
  first = (uint32_t*)(to + n_pieces);
  walk(true);
  return THEMIS_OK;
}

static int gradient_pass(const themis_gradient_plan_t* plan, double max_norm, bool clip, float* total, float* norms,
                         void* workspace, size_t workspace_bytes, void* stream) {
  if (!plan || !plan->image || !total || !aligned(plan->image, 16)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (plan->n_pieces >= kMost || plan->n_tensors > kMostTensors) return THEMIS_ERR_UNSUPPORTED;
  if (clip && (!(max_norm > 0.0) || !std::isfinite(max_norm) || !plan->has_out)) return THEMIS_ERR_INVALID_ARGUMENT;
  const uint32_t groups = pass_groups(plan->n_pieces, plan->in_bytes);
  const size_t need = (groups + plan->n_pieces) * sizeof(double);
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return THEMIS_ERR_WORKSPACE;
  const PlanView view = plan_view(*plan);
  double* group_sums = (double*)workspace;
  double* piece_sums = group_sums + groups;
  const uint32_t norm_blocks = norms ? (uint32_t)((plan->n_tensors + 3) / 4) : 0u;
  Launches go(stream);
  const uint32_t passed = plan->in_bytes <= kKeptBytes ? 0u
                          : (uint32_t)((double)plan->n_pieces * (1.0 - (double)kKeptBytes / (double)plan->in_bytes));
  if (groups) go(norm_kernel, dim3(groups), 256, view, passed, group_sums, piece_sums);
  if (clip) {
    const uint32_t scalers = std::max(groups, 1u);
    go(clip_kernel, dim3(scalers + norm_blocks), 256, view, groups, group_sums, piece_sums, max_norm, scalers, total,
       norms);
  } else {
    go(norm_finish_kernel, dim3(1 + norm_blocks), 256, view, groups, group_sums, piece_sums, total, norms);
  }
  return go.status();
}

int themis_gradient_norm(const themis_gradient_plan_t* plan, float* total, float* norms, void* workspace,
                         size_t workspace_bytes, void* stream) {
  return gradient_pass(plan, 1.0, false, total, norms, workspace, workspace_bytes, stream);
}

int themis_gradient_clip(const themis_gradient_plan_t* plan, double max_norm, float* total, float* norms,
                         void* workspace, size_t workspace_bytes, void* stream) {
  return gradient_pass(plan, max_norm, true, total, norms, workspace, workspace_bytes, stream);
}

}  // extern "C"
