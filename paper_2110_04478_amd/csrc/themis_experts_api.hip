// C ABI of the expert layer's operators and of dropout (see include/themis.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "themis.h"
#include "themis_dropout.hpp"
#include "themis_elements.hpp"
#include "themis_experts.hpp"
#include "themis_launch.hpp"

namespace themis {
namespace {

constexpr uint64_t kLastCache = 256u << 20;   // bytes of the last cache level
constexpr uint64_t kMostWidth = 1u << 25;

// Lanes of a token's logits: 2^shift of `own` each; where lists are kept, of `own` times eight.  (More than
// kMostListed chosen: nine experts at least.)
struct GateLayout { uint32_t own, shift; };
GateLayout gate_layout(uint32_t experts) {
  if (experts > 512) return {16, 6};
  if (experts > 64) return {8, next_power((experts + 7) / 8)};
  return {experts <= 16 ? 2u : experts <= 32 ? 4u : 8u, kGateLeastShift};
}
GateLayout list_layout(uint32_t experts) {
  const uint32_t chunks = experts <= 64 ? 1 : experts <= 128 ? 2 : 4;
  return {chunks, next_power((experts + 8 * chunks - 1) / (8 * chunks))};
}
// Calls f with `own` as a constant, one of kOwn.
template <int... kOwn, typename F>
void with_own(uint32_t own, F&& f) {
  ((own == kOwn ? f(std::integral_constant<int, kOwn>{}) : void()), ...);
}

uint32_t blocks_of(uint64_t n, uint64_t each) { return (uint32_t)std::min<uint64_t>((n + each - 1) / each, 1u << 20); }

// Pairs of a workgroup and workgroups of the sort.  Up to 8,192 pairs one workgroup, without a count
// before it (8,192: 10.9 us with the host's side, in parts 14.8; 16,384: 13.8 to 19.2 by the experts, and 14.8).
// Else four pairs a lane, more where the counts, all of which every workgroup reads, would outgrow what it
// sorts (1,048,576 pairs on 1,024 experts: 36.6 us with 4,096 pairs, 26.7 with 8,192, 29.5 with 16,384).
struct SortLayout { uint32_t part, parts; size_t bytes; };
SortLayout sort_layout(uint32_t pairs, uint32_t experts) {
  SortLayout l = {std::max(kPairGroup, std::min((pairs + kPairGroup - 1) / kPairGroup * kPairGroup, 8192u)), 1, 0};
  if (pairs > l.part) {
    l.part = kPairsAhead * kPairGroup;
    auto counts = [&] { return ((uint64_t)pairs + l.part - 1) / l.part * experts; };
    while (counts() > 32ull * l.part) l.part *= 2;
    l.parts = (pairs + l.part - 1) / l.part;
    l.bytes = counts() * sizeof(uint32_t);
  }
  return l;
}

// Sizes and addresses of an order; its view.
int order_status(const themis_expert_order_t* o, Order& view) {
  if (!o || o->n_experts == 0) return THEMIS_ERR_INVALID_ARGUMENT;
  if (o->n_experts > kMostExperts || o->n > kMost || o->k > kMost || o->capacity > kMost) return THEMIS_ERR_UNSUPPORTED;
  const uint64_t pairs = o->n * o->k, slots = o->capacity ? o->n_experts * o->capacity : pairs;
  if (pairs > kMost || slots > kMost) return THEMIS_ERR_UNSUPPORTED;
  view = {(uint32_t)o->n, (uint32_t)o->k, (uint32_t)pairs, (uint32_t)o->n_experts, (uint32_t)o->capacity, (uint32_t)slots,
          o->place, o->counts, o->starts, o->source};
  if ((pairs && (!o->place || !aligned(o->place, 4))) || (slots && (!o->source || !aligned(o->source, 4))))
    return THEMIS_ERR_INVALID_ARGUMENT;
  return THEMIS_OK;
}

// n rows of `width` elements over a grid, `vec` elements a lane.  (Lanes in powers of two for a row: 65 of 128 have
// work in rows of 520, whose sums of eight take 121 us in place of 97.)
Spread spread_of(uint64_t n, uint64_t width, uint32_t vec) {
  // (of numbers below 2^31 the quotient is exact: inverse exceeds 2^(31 + power) / lanes by less than one, and
  // lanes are at most 2^power)
  const uint32_t lanes = (uint32_t)((width + vec - 1) / vec), power = next_power(lanes);
  const uint32_t rows = (uint32_t)std::min<uint64_t>(n, (kMost - 256) / lanes);
  return {lanes, (uint32_t)(((1ull << (31 + power)) + lanes - 1) / lanes), power ? power - 1 : 0, rows,
          (uint32_t)((n + rows - 1) / rows)};
}
dim3 grid_of(const Spread& s, uint32_t more = 0) {
  return dim3(more + (uint32_t)(((uint64_t)s.rows * s.lanes + 255) / 256), std::min(s.segments, 65535u));
}

// Rows of experts that the last cache level cannot hold are read past it (1.07 GB: sums 242 us, through it
// 253; 537 MB of binary32 122, 145); the others may still be there (200 MB: 28 us, 24).
bool read_once(const Order& o, uint64_t width, int type) {
  return (uint64_t)std::min(o.slots, o.pairs) * width * type_bytes(type) >= kLastCache;
}

// Whether rows of `width` elements are whole lines of the caches.
bool whole_lines(const Rows& r, uint64_t width) { return width * type_bytes(r.type) % 128 == 0 && aligned(r.data, 128); }

// Slots of a workgroup that looks for those of no pair: about 256 KiB.
uint32_t slots_to_clear(uint64_t row_bytes) {
  return (uint32_t)std::min<uint64_t>(64, std::max<uint64_t>(1, (256u << 10) / row_bytes));
}

Rows rows_or_none(const themis_rows_t* r, uint64_t n) { return r ? rows_of(*r, n) : Rows{}; }

}  // namespace
}  // namespace themis

using namespace themis;

extern "C" {

int themis_expert_gate(const themis_rows_t* logits, uint64_t n_experts, uint64_t n, uint64_t k, int renormalize,
                       const themis_rows_t* weights, const themis_rows_t* experts, void* stream) {
  if (k > n_experts) return THEMIS_ERR_INVALID_ARGUMENT;
  if (n == 0 || k == 0) return THEMIS_OK;
  if (!rows_ok(logits, false) || !rows_ok(weights, false) || !rows_ok(experts, true)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (n > kMost || n_experts > kMostExperts || k > kMostChosen) return THEMIS_ERR_UNSUPPORTED;
  if (!rows_apart(*weights, n, k) || !rows_apart(*experts, n, k)) return THEMIS_ERR_INVALID_ARGUMENT;
  const GateLayout l = gate_layout((uint32_t)n_experts);
  Launches go(stream);
  if (k <= kMostListed) {
    const GateLayout m = list_layout((uint32_t)n_experts);
    auto run = [&](auto kernel) {
      go(kernel, dim3(blocks_of(n, 256u >> m.shift)), 256, rows_of(*logits, n), (uint32_t)n_experts, (uint32_t)n, (uint32_t)k,
         rows_of(*weights, n), rows_of(*experts, n), m.shift);
    };
    with_type(logits->type, [&](auto in) {
      typedef decltype(in) In;
      with_own<1, 2, 4>(m.own, [&](auto own) {
        constexpr int kChunks = decltype(own)::value;
        auto over = [&](auto all) {
          constexpr bool kAll = decltype(all)::value;
          if (k == 1) run(gate_list_kernel<In, kChunks, 1, kAll>);
          else if (k == 2) run(gate_list_kernel<In, kChunks, 2, kAll>);
          else if (k <= 4) run(gate_list_kernel<In, kChunks, 4, kAll>);
          else run(gate_list_kernel<In, kChunks, 8, kAll>);
        };
        if (renormalize) over(std::false_type{});
        else over(std::true_type{});
      });
    });
    return go.status();
  }
  with_type(logits->type, [&](auto in) {
    with_own<2, 4, 8, 16>(l.own, [&](auto own) {
      go(gate_kernel<decltype(in), decltype(own)::value>, dim3(blocks_of(n, 256u >> l.shift)), 256, rows_of(*logits, n),
         (uint32_t)n_experts, (uint32_t)n, (uint32_t)k, renormalize != 0, rows_of(*weights, n), rows_of(*experts, n),
         l.shift);
    });
  });
  return go.status();
}

int themis_expert_gate_grad(const themis_rows_t* grad_weights, const themis_rows_t* logits, uint64_t n_experts,
                            const themis_rows_t* experts, uint64_t n, uint64_t k, int renormalize,
                            const themis_rows_t* grad_logits, void* stream) {
  if (n == 0 || n_experts == 0) return THEMIS_OK;
  if (!rows_ok(logits, false) || !rows_ok(grad_logits, false)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (k && (!rows_ok(grad_weights, false) || !rows_ok(experts, true))) return THEMIS_ERR_INVALID_ARGUMENT;
  if (n > kMost || n_experts > kMostExperts || k > kMostChosen) return THEMIS_ERR_UNSUPPORTED;
  if (!rows_apart(*grad_logits, n, n_experts)) return THEMIS_ERR_INVALID_ARGUMENT;
  const GateLayout l = list_layout((uint32_t)n_experts);
  const Rows g = k ? rows_of(*grad_weights, n) : Rows{}, e = k ? rows_of(*experts, n) : Rows{};
  Launches go(stream);
  with_type(logits->type, [&](auto in) {
    with_type(grad_logits->type, [&](auto out) {
      with_own<1, 2, 4>(l.own, [&](auto own) {
        constexpr int kChunks = decltype(own)::value;
        typedef decltype(in) In;
        typedef decltype(out) Out;
        go(renormalize ? gate_grad_kernel<In, Out, kChunks, false> : gate_grad_kernel<In, Out, kChunks, true>,
           dim3(blocks_of(n, 256u >> l.shift)), 256, g, rows_of(*logits, n), (uint32_t)n_experts, e, (uint32_t)n, (uint32_t)k,
           rows_of(*grad_logits, n), l.shift);
      });
    });
  });
  return go.status();
}

size_t themis_expert_sort_workspace_bytes(uint64_t n, uint64_t k, uint64_t n_experts) {
  if (n > kMost || k > kMost || n * k > kMost || n_experts == 0 || n_experts > kMostExperts) return 0;
  return sort_layout((uint32_t)(n * k), (uint32_t)n_experts).bytes;
}

int themis_expert_sort(const themis_rows_t* experts, const themis_expert_order_t* order, void* workspace,
                       size_t workspace_bytes, void* stream) {
  Order o;
  if (const int status = order_status(order, o)) return status;
  if (o.pairs && !rows_ok(experts, true)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (!o.counts || !o.starts || !aligned(o.counts, 4) || !aligned(o.starts, 4)) return THEMIS_ERR_INVALID_ARGUMENT;
  const SortLayout l = sort_layout(o.pairs, o.experts);
  if (l.bytes && (!workspace || workspace_bytes < l.bytes || !aligned(workspace, 16))) return THEMIS_ERR_WORKSPACE;
  const Rows chosen = o.pairs ? rows_of(*experts, o.n) : Rows{};
  uint32_t* counts = (uint32_t*)workspace;
  Launches go(stream);
  if (l.parts > 1) go(expert_count_kernel, dim3(l.parts), kPairGroup, o, chosen, l.part, counts);
  go(expert_sort_kernel, dim3(l.parts), kPairGroup, o, chosen, l.part, l.parts, (const uint32_t*)counts,
     next_power(o.experts));
  return go.status();
}

int themis_expert_dispatch(const themis_expert_order_t* order, const themis_rows_t* x, uint64_t width,
                           const themis_rows_t* out, void* stream) {
  Order o;
  if (const int status = order_status(order, o)) return status;
  if (o.slots == 0 || width == 0) return THEMIS_OK;
  if ((o.n && !rows_ok(x, false)) || !rows_ok(out, false)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (width > kMostWidth) return THEMIS_ERR_UNSUPPORTED;
  if (!rows_apart(*out, o.slots, width)) return THEMIS_ERR_INVALID_ARGUMENT;
  const Spread spread = o.n ? spread_of(o.n, width, kLaneElements) : Spread{};
  const Rows from = o.n ? rows_of(*x, o.n) : Rows{0, 0, 0, 0, out->type}, to = rows_of(*out, o.slots);
  const uint32_t fill_rows = slots_to_clear(width * type_bytes(to.type)), fills = blocks_of(o.slots, fill_rows);
  Launches go(stream);
  with_type(from.type, [&](auto in) {
    with_type(to.type, [&](auto out) {
      typedef decltype(in) In;
      typedef decltype(out) Out;
      auto run = [&](auto kernel) {
        go(kernel, o.n ? grid_of(spread, fills) : dim3(fills), 256, o, from, (uint32_t)width, to, spread, fills, fill_rows);
      };
      // Whole lines go past the caches (65,536 rows of 2,048 bf16: 50 us, through them 58), others, which two rows
      // share, do not (100,000 rows of 1,001: 47 us, past them 57).
      auto places = [&](auto ahead) {
        constexpr int kAhead = decltype(ahead)::value;
        if (width < kLaneElements) run(dispatch_kernel<false, false, kAhead, In, Out>);
        else if (whole_lines(to, width)) run(dispatch_kernel<true, true, kAhead, In, Out>);
        else run(dispatch_kernel<true, false, kAhead, In, Out>);
      };
      // (one place a token, 65,536 rows of 512 bf16: 24.8 us, with eight looked up 25.7)
      if (o.k <= 2) places(std::integral_constant<int, 2>{});
      else places(std::integral_constant<int, 8>{});
    });
  });
  return go.status();
}

int themis_expert_combine(const themis_expert_order_t* order, const themis_rows_t* y, uint64_t width,
                          const themis_rows_t* weights, int accumulate, const themis_rows_t* out, void* stream) {
  Order o;
  if (const int status = order_status(order, o)) return status;
  if (o.n == 0 || width == 0 || (o.pairs == 0 && accumulate)) return THEMIS_OK;
  if (!rows_ok(out, false) || (o.slots && !rows_ok(y, false))) return THEMIS_ERR_INVALID_ARGUMENT;
  if (weights && o.k && !rows_ok(weights, false)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (width > kMostWidth) return THEMIS_ERR_UNSUPPORTED;
  if (!rows_apart(*out, o.n, width)) return THEMIS_ERR_INVALID_ARGUMENT;
  const Spread spread = spread_of(o.n, width, kLaneElements);
  const Rows from = o.slots ? rows_of(*y, o.slots) : Rows{0, 0, 0, 0, out->type}, to = rows_of(*out, o.n);
  const bool once = read_once(o, width, from.type);
  Launches go(stream);
  with_type(from.type, [&](auto in) {
    with_type(to.type, [&](auto out) {
      typedef decltype(in) In;
      typedef decltype(out) Out;
      auto run = [&](auto kernel) {
        go(kernel, grid_of(spread), 256, o, from, (uint32_t)width, rows_or_none(weights, o.n), accumulate != 0, to, spread);
      };
      auto turns_of = [&](auto ahead) {
        constexpr int kAhead = decltype(ahead)::value;
        if (width < kLaneElements) run(combine_kernel<false, false, kAhead, In, Out>);
        else if (once) run(combine_kernel<true, true, kAhead, In, Out>);
        else run(combine_kernel<true, false, kAhead, In, Out>);
      };
      // (20,480 tokens of 5,120 bf16, k = 2: 108 us, with four rows in flight 122)
      if (o.k <= 2) turns_of(std::integral_constant<int, 2>{});
      else turns_of(std::integral_constant<int, 4>{});
    });
  });
  return go.status();
}

int themis_expert_combine_grad(const themis_expert_order_t* order, const themis_rows_t* grad_out, uint64_t width,
                               const themis_rows_t* y, const themis_rows_t* weights, const themis_rows_t* grad_y,
                               const themis_rows_t* grad_weights, void* stream) {
  Order o;
  if (const int status = order_status(order, o)) return status;
  if ((grad_y && o.slots && width && !rows_ok(grad_y, false)) || (grad_weights && o.pairs && !rows_ok(grad_weights, false)))
    return THEMIS_ERR_INVALID_ARGUMENT;
  const bool rows = grad_y && o.slots && width, products = grad_weights && o.pairs;
  if (!rows && !products) return THEMIS_OK;
  if (o.pairs && ((width && !rows_ok(grad_out, false)) || !rows_ok(weights, false))) return THEMIS_ERR_INVALID_ARGUMENT;
  if (products && o.slots && width && !rows_ok(y, false)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (rows && products && y->type != grad_y->type) return THEMIS_ERR_INVALID_ARGUMENT;
  if (width > kMostWidth) return THEMIS_ERR_UNSUPPORTED;
  if ((rows && !rows_apart(*grad_y, o.slots, width)) || (products && !rows_apart(*grad_weights, o.n, o.k)))
    return THEMIS_ERR_INVALID_ARGUMENT;
  const Rows to = rows ? rows_of(*grad_y, o.slots) : Rows{};
  const Rows from = products && width ? rows_of(*y, o.slots) : Rows{0, 0, 0, 0, rows ? to.type : THEMIS_F32};
  const Rows g = o.pairs && width ? rows_of(*grad_out, o.n) : Rows{0, 0, 0, 0, from.type};
  const uint32_t fill_rows = rows ? slots_to_clear(width * type_bytes(to.type)) : 1u;
  const uint32_t fills = rows ? blocks_of(o.slots, fill_rows) : 0u;
  const uint32_t shift = std::min(next_power((uint32_t)((width + kLaneElements - 1) / kLaneElements)), 6u);
  const bool once = read_once(o, width, from.type);
  // (rows past the caches: 268 MB 110 us, through them 125; 410 MB 178 and 187; rows that share
  // lines take 7 to 10 % more that way)
  const bool away = rows && whole_lines(to, width) && (uint64_t)o.slots * width * type_bytes(to.type) >= kLastCache;
  Launches go(stream);
  with_type(g.type, [&](auto grad) {
    with_type(from.type, [&](auto row) {
      typedef decltype(grad) G;
      typedef decltype(row) Y;
      go(width < kLaneElements ? combine_grad_kernel<false, false, false, G, Y>
         : once && away        ? combine_grad_kernel<true, true, true, G, Y>
         : once                ? combine_grad_kernel<true, true, false, G, Y>
                               : combine_grad_kernel<true, false, false, G, Y>,
         dim3(fills + blocks_of((uint64_t)o.n * ((o.k + kGradPairs - 1) / kGradPairs), 256u >> shift)), 256, o, g,
         (uint32_t)width, from, o.pairs ? rows_of(*weights, o.n) : Rows{}, to,
         products ? rows_of(*grad_weights, o.n) : Rows{}, shift, fills, fill_rows);
    });
  });
  return go.status();
}

int themis_dropout(const themis_rows_t* x, uint64_t n, uint64_t width, double p, uint64_t seed, uint64_t call,
                   const uint64_t* call_at, const themis_rows_t* add, const themis_rows_t* out, void* stream) {
  if (!(p >= 0.0 && p <= 1.0) || !aligned(call_at, 8)) return THEMIS_ERR_INVALID_ARGUMENT;
  if (n == 0 || width == 0) return THEMIS_OK;
  if (!rows_ok(x, false) || !rows_ok(out, false) || (add && !rows_ok(add, false))) return THEMIS_ERR_INVALID_ARGUMENT;
  if (add && add->type != out->type) return THEMIS_ERR_INVALID_ARGUMENT;
  if (n > kMost || width > kMostWidth) return THEMIS_ERR_UNSUPPORTED;
  if (!rows_apart(*out, n, width)) return THEMIS_ERR_INVALID_ARGUMENT;
  const uint64_t least = (uint64_t)std::nearbyint(p * 4294967296.0);
  const DropoutKey d = {{(uint32_t)seed, (uint32_t)(seed >> 32)}, {(uint32_t)call, (uint32_t)(call >> 32)},
                        (uint32_t)least, least >> 32 != 0, p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.0f};
  Launches go(stream);
  with_type(x->type, [&](auto in) {
    with_type(out->type, [&](auto to) {
      typedef decltype(in) In;
      typedef decltype(to) Out;
      // What the last cache level cannot hold goes past it, and two rows of 16 bits a lane are in flight then
      // (268 M bf16: 169 us, otherwise 194; with a residual 256, 285; 50 M 19 and 18; binary32 with a residual, 134 M,
      // one row 269, two 286, through the caches 292).
      const bool once = n * width * (type_bytes(x->type) + type_bytes(out->type)) >= kLastCache;
      constexpr int kTwo = sizeof(In) == 2 && sizeof(Out) == 2 ? 2 : 1;
      auto run = [&](auto kernel, uint32_t rows) {
        const Spread spread = spread_of((n + rows - 1) / rows, width, kVecOf<In, Out>);
        go(kernel, grid_of(spread), 256, rows_of(*x, n), (uint32_t)n, (uint32_t)width, d, call_at, rows_or_none(add, n),
           rows_of(*out, n), spread);
      };
      auto adds = [&](auto is) {
        constexpr bool kAdd = decltype(is)::value;
        if (width < kLaneElements) run(dropout_kernel<false, false, kAdd, 1, In, Out>, 1);
        else if (once) run(dropout_kernel<true, true, kAdd, kTwo, In, Out>, kTwo);
        else run(dropout_kernel<true, false, kAdd, 1, In, Out>, 1);
      };
      if (add) adds(std::true_type{});
      else adds(std::false_type{});
    });
  });
  return go.status();
}

}  // extern "C"
