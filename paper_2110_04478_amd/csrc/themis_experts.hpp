// An expert layer's operators on the rank: the gate, the order of tokens by expert, rows into that
// order and back (themis_expert_*).
#pragma once

#include "themis_elements.hpp"

namespace themis {

// ---------------------------------------------------------------------------
// Over the 2^shift lanes of a group (aligned, up to a wavefront; all lanes are on): a sum, the same in
// every lane and every call, and the largest and smallest value.
// ---------------------------------------------------------------------------
template <typename F>
__device__ __forceinline__ uint32_t over_group(uint32_t x, uint32_t shift, F f) {
  if (shift > 0) x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));    // lane ^ 1
  if (shift > 1) x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));    // lane ^ 2
  if (shift > 2) x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, false));   // 7 - lane
  if (shift > 3) x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, false));   // 15 - lane
  if (shift > 4) {   // rows of 16 lanes, two and two, then the halves
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = f(r[0], r[1]);
  }
  if (shift > 5) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = f(r[0], r[1]);
  }
  return x;
}
__device__ __forceinline__ float group_sum(float x, uint32_t shift) {
  return __uint_as_float(over_group(__float_as_uint(x), shift, [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
__device__ __forceinline__ float group_max(float x, uint32_t shift) {
  return __uint_as_float(over_group(__float_as_uint(x), shift, [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}
__device__ __forceinline__ uint32_t group_max(uint32_t x, uint32_t shift) {
  return over_group(x, shift, [](uint32_t a, uint32_t b) { return max(a, b); });
}
__device__ __forceinline__ uint32_t group_min(uint32_t x, uint32_t shift) {
  return over_group(x, shift, [](uint32_t a, uint32_t b) { return min(a, b); });
}

// One element of a row of any type.
__device__ __forceinline__ float float_at(const Rows& rows, uint32_t r, uint32_t j) {
  const int64_t at = row_offset(rows, r) + j;
  if (rows.type == THEMIS_F32) return ((const float*)rows.data)[at];
  if (rows.type == THEMIS_BF16) return (float)((const __bf16*)rows.data)[at];
  return (float)((const _Float16*)rows.data)[at];
}
__device__ __forceinline__ void put_float(const Rows& rows, uint32_t r, uint32_t j, float x) {
  const int64_t at = row_offset(rows, r) + j;
  if (rows.type == THEMIS_F32) ((float*)rows.data)[at] = x;
  else if (rows.type == THEMIS_BF16) ((__bf16*)rows.data)[at] = (__bf16)x;
  else ((_Float16*)rows.data)[at] = (_Float16)x;
}
// A number of 0 .. most-1, or ~0u.
__device__ __forceinline__ uint32_t number_at(const Rows& rows, uint32_t r, uint32_t j, uint32_t most) {
  const int64_t at = row_offset(rows, r) + j;
  const int64_t x = rows.type == THEMIS_I64 ? ((const int64_t*)rows.data)[at] : ((const int32_t*)rows.data)[at];
  return (uint64_t)x < most ? (uint32_t)x : ~0u;
}
__device__ __forceinline__ void put_number(const Rows& rows, uint32_t r, uint32_t j, int32_t x) {
  const int64_t at = row_offset(rows, r) + j;
  if (rows.type == THEMIS_I64) ((int64_t*)rows.data)[at] = x;
  else ((int32_t*)rows.data)[at] = x;
}

// ---------------------------------------------------------------------------
// themis_expert_gate: the k largest logits of a token and their softmax.
//
// 2^shift lanes take a token, each kOwn adjacent logits in registers; k times the largest is found
// (over a lane's own, then over the lanes) and taken out.  Logits are compared as whole numbers
// that are ordered as the values are; those of 16 bits carry their index in the lower half, smaller ones
// first, so that one maximum gives both.  For more than eight experts.  Bound by its instructions, which leave no
// cycle free: 65,536 tokens on 256 experts, 16 of them (bf16), 45 us, 64 of them 129.
// ---------------------------------------------------------------------------
constexpr uint32_t kMostExperts = 1024;
constexpr uint32_t kMostChosen = 64;
constexpr uint32_t kGateLeastShift = 3;   // (32 tokens a workgroup at most: the results wait in LDS)

// A logit as a key: NaN above all, -0 as 0.  No element: 0.  first(): of what may be chosen.
template <typename T>
struct LogitKey {   // 16 bits
  static constexpr bool kIndexed = true;
  static __device__ __forceinline__ uint32_t of(T x, uint32_t index) {
    uint32_t b = __builtin_bit_cast(uint16_t, x);
    b = x != x ? 0x7FFFu : b == 0x8000u ? 0u : b;
    return (b & 0x8000u ? ~b & 0xFFFFu : b | 0x8000u) << 16 | (0xFFFFu - index);
  }
  static __device__ __forceinline__ float value(uint32_t key) {
    const uint32_t s = key >> 16, b = s & 0x8000u ? s & 0x7FFFu : ~s & 0xFFFFu;
    return (float)__builtin_bit_cast(T, (uint16_t)b);
  }
  static __device__ __forceinline__ uint32_t index(uint32_t key) { return 0xFFFFu - (key & 0xFFFFu); }
  static __device__ __forceinline__ uint32_t first() { return of(-(T)__builtin_inff(), 0) + 1; }
};
template <>
struct LogitKey<float> {
  static constexpr bool kIndexed = false;
  static __device__ __forceinline__ uint32_t of(float x, uint32_t) {
    uint32_t b = __float_as_uint(x);
    b = x != x ? 0x7FFFFFFFu : b == 0x80000000u ? 0u : b;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
  }
  static __device__ __forceinline__ float value(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
  }
  static __device__ __forceinline__ uint32_t first() { return of(-__builtin_inff(), 0) + 1; }
};

// A lane's kOwn logits from `first` on, `none` behind the last one.
template <int kOwn, typename T>
__device__ __forceinline__ typename Packed<T, kOwn>::type own_logits(const T* row, uint32_t first, uint32_t experts, T none) {
  if (first + kOwn <= experts) return load<kOwn>(row + first);
  typename Packed<T, kOwn>::type v = none;
#pragma unroll
  for (uint32_t i = 0; i + 1 < kOwn; ++i)
    if (first + i < experts) v[i] = row[first + i];
  return v;
}

template <typename T, int kOwn>
__global__ void __launch_bounds__(256)
gate_kernel(Rows logits, uint32_t experts, uint32_t n, uint32_t k, bool renormalize, Rows weights, Rows chosen,
            uint32_t shift) {
  typedef LogitKey<T> Key;
  __shared__ uint32_t best[(256 >> kGateLeastShift) * kMostChosen];
  __shared__ int32_t number[(256 >> kGateLeastShift) * kMostChosen];
  const uint32_t lanes = 1u << shift, lane = threadIdx.x & (lanes - 1u), group = threadIdx.x >> shift;
  const uint32_t groups = 256u >> shift, own = lane * kOwn;
  for (uint64_t at = (uint64_t)blockIdx.x * groups; at < n; at += (uint64_t)gridDim.x * groups) {
    const uint32_t t = (uint32_t)at + group;
    const T* row = row_at<const T>(logits, min(t, n - 1u));
    const auto v = own_logits<kOwn>(row, own, experts, (T)-__builtin_inff());
    uint32_t key[kOwn];
#pragma unroll
    for (uint32_t i = 0; i < kOwn; ++i) key[i] = own + i < experts ? Key::of(v[i], own + i) : 0u;
    float largest = -__builtin_inff();
    for (uint32_t j = 0; j < k; ++j) {
      uint32_t top = key[0];
#pragma unroll
      for (uint32_t i = 1; i < kOwn; ++i) top = max(top, key[i]);
      top = group_max(top, shift);
      uint32_t index;
      if constexpr (Key::kIndexed) {
        index = Key::index(top);
#pragma unroll
        for (uint32_t i = 0; i < kOwn; ++i) key[i] = key[i] == top ? 0u : key[i];
      } else {
        index = ~0u;
#pragma unroll
        for (uint32_t i = kOwn; i-- > 0;) index = key[i] == top ? own + i : index;
        index = group_min(index, shift);
#pragma unroll
        for (uint32_t i = 0; i < kOwn; ++i) key[i] = own + i == index ? 0u : key[i];
      }
      const bool any = top >= Key::first();
      if (j == 0 && any) largest = Key::value(top);
      if (lane == 0) {
        best[group * k + j] = top;
        number[group * k + j] = any ? (int32_t)index : -1;
      }
    }
    float sum = 0.0f;
    if (!renormalize) {
#pragma unroll
      for (uint32_t i = 0; i < kOwn; ++i) sum += own + i < experts ? expf((float)v[i] - largest) : 0.0f;
      sum = group_sum(sum, shift);
    }
    __syncthreads();
    if (renormalize) {
      for (uint32_t j = lane; j < k; j += lanes)
        if (number[group * k + j] >= 0) sum += expf(Key::value(best[group * k + j]) - largest);
      sum = group_sum(sum, shift);
    }
    if (t < n)
      for (uint32_t j = lane; j < k; j += lanes) {
        const int32_t e = number[group * k + j];
        put_number(chosen, t, j, e);
        put_float(weights, t, j, e < 0 ? 0.0f : expf(Key::value(best[group * k + j]) - largest) / sum);
      }
    __syncthreads();   // (the next tokens' results)
  }
}

// ---------------------------------------------------------------------------
// The same for up to kMostListed experts: every lane keeps the kList largest of its own, sorted, while it
// goes through them, and the lanes' lists are merged two and two: the larger of a list and the other one
// backwards are the largest of both, and a few exchanges sort them.
//
// An entry is a number that is ordered as (logit, index from the end) is: of logits of 16 bits
// a whole number, the logit as a signed one (so that -0 is 0) over its index, of binary32 a binary64
// number, the logit with its index in the last of the 29 bits that it leaves free.
// 65,536 tokens on 256 experts, eight of them (bf16): 11.7 us, of which the logits' bytes need 8, by k
// rounds of a maximum 33; over all 18.  Bound by instructions (on 86 % of the cycles, over all 97 %).
// ---------------------------------------------------------------------------
constexpr uint32_t kMostListed = 8;

__device__ __forceinline__ int32_t larger(int32_t a, int32_t b) { return max(a, b); }
__device__ __forceinline__ int32_t smaller(int32_t a, int32_t b) { return min(a, b); }
// (the instructions themselves: of fmax the compiler makes two, in case an argument is a signalling NaN;
// entries are none)
__device__ __forceinline__ double larger(double a, double b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ double smaller(double a, double b) {
  double r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}

// A place's new entry is the median of its own, the next larger one's and the new one.
template <int kList>
__device__ __forceinline__ void insert(int32_t (&list)[kList], int32_t x) {
#pragma unroll
  for (int i = kList - 1; i > 0; --i) {   // (in the form that is one instruction)
    const int32_t a = list[i - 1], b = list[i];
    list[i] = max(min(a, b), min(max(a, b), x));
  }
  list[0] = max(list[0], x);
}
template <int kList>
__device__ __forceinline__ void insert(double (&list)[kList], double x) {
#pragma unroll
  for (int i = 0; i < kList; ++i) {
    const double up = larger(list[i], x);
    if (i + 1 < kList) x = smaller(list[i], x);
    list[i] = up;
  }
}

// Between what assembly wrote and another lane's look at it: the compiler counts the wait states that this needs
// (two) from its own instructions only.
template <int kList>
__device__ __forceinline__ void settle(int32_t (&)[kList]) {}
template <int kList>
__device__ __forceinline__ void settle(double (&l)[kList]) {
  if constexpr (kList == 1) asm volatile("s_nop 1" : "+v"(l[0]));
  if constexpr (kList == 2) asm volatile("s_nop 1" : "+v"(l[0]), "+v"(l[1]));
  if constexpr (kList == 4) asm volatile("s_nop 1" : "+v"(l[0]), "+v"(l[1]), "+v"(l[2]), "+v"(l[3]));
  if constexpr (kList == 8)
    asm volatile("s_nop 1" : "+v"(l[0]), "+v"(l[1]), "+v"(l[2]), "+v"(l[3]), "+v"(l[4]), "+v"(l[5]), "+v"(l[6]), "+v"(l[7]));
}

// The largest of this lane's list and another's, sorted.
template <int kList, typename E, typename F>
__device__ __forceinline__ void merge_with(E (&list)[kList], F other) {
  settle(list);
  E both[kList];
#pragma unroll
  for (int i = 0; i < kList; ++i) both[i] = larger(list[i], other(list[kList - 1 - i]));
#pragma unroll
  for (int d = kList / 2; d > 0; d /= 2)
#pragma unroll
    for (int i = 0; i < kList; ++i)
      if ((i & d) == 0) {
        const E a = both[i], b = both[i + d];
        both[i] = larger(a, b);
        both[i + d] = smaller(a, b);
      }
#pragma unroll
  for (int i = 0; i < kList; ++i) list[i] = both[i];
}
template <int kControl>
__device__ __forceinline__ int32_t of_lane(int32_t x) {
  return __builtin_amdgcn_update_dpp(0, x, kControl, 0xF, 0xF, false);
}
template <int kControl>
__device__ __forceinline__ double of_lane(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)of_lane<kControl>((int32_t)b), hi = (uint32_t)of_lane<kControl>((int32_t)(b >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int kList, typename E>
__device__ __forceinline__ void merge_group(E (&list)[kList], uint32_t shift) {
  if (shift > 0) merge_with(list, [](E x) { return of_lane<0xB1>(x); });    // lane ^ 1
  if (shift > 1) merge_with(list, [](E x) { return of_lane<0x4E>(x); });    // lane ^ 2
  if (shift > 2) merge_with(list, [](E x) { return of_lane<0x141>(x); });   // 7 - lane
  if (shift > 3) merge_with(list, [](E x) { return of_lane<0x140>(x); });   // 15 - lane
  if (shift > 4) merge_with(list, [](E x) { return __shfl_xor(x, 16); });
}

template <typename T>
struct Listed {   // 16 bits
  typedef int32_t Entry;
  typedef int16_t Pair __attribute__((ext_vector_type(2)));
  struct Pairs { Pair two[4]; };
  static constexpr int16_t kInfinite = __is_same(T, __bf16) ? 0x7F80 : 0x7C00;
  static constexpr Entry kNone = INT32_MIN;

  Pair key[4];
  // The lane's eight logits; `begin` is the first one's index.
  __device__ __forceinline__ Listed(typename Packed<T, 8>::type v) {
    Pair most = 0;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const Pair x = __builtin_bit_cast(Pairs, v).two[i], sign = x >> 15, size = x & (int16_t)0x7FFF;
      most = __builtin_elementwise_max(most, size);
      key[i] = (size ^ sign) - sign;
    }
    if (most[0] > kInfinite || most[1] > kInfinite)   // a NaN: above all
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        const Pair size = __builtin_bit_cast(Pairs, v).two[i] & (int16_t)0x7FFF, one = 1;
        const Pair is = -__builtin_elementwise_min(__builtin_elementwise_max(size, (Pair)kInfinite) - (Pair)kInfinite, one);
        key[i] = (key[i] | is) & ~(is & (int16_t)0x8000);
      }
  }
  __device__ __forceinline__ Entry entry(uint32_t i, uint32_t begin) const {
    const uint32_t two = __builtin_bit_cast(uint32_t, key[i / 2]);
    return (Entry)((i & 1 ? two & 0xFFFF0000u : two << 16) | (0xFFFFu - begin - i));
  }
  static __device__ __forceinline__ bool any(Entry e) { return e >> 16 > -kInfinite; }
  static __device__ __forceinline__ int32_t index(Entry e) { return 0xFFFF - (e & 0xFFFF); }
  static __device__ __forceinline__ float value(Entry e) {
    const int32_t s = e >> 16;
    return (float)__builtin_bit_cast(T, (uint16_t)(s < 0 ? -s | 0x8000 : s));
  }
};
template <>
struct Listed<float> {
  typedef double Entry;
  static constexpr Entry kNone = -0x1p300, kMasked = -0x1p200;   // (behind all that binary32 holds)
  static constexpr uint32_t kIndex = kMostExperts - 1;

  double key[8];
  __device__ __forceinline__ Listed(typename Packed<float, 8>::type v) {
    float most = 0.0f;
    bool nan = false;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      most = fmaxf(most, v[i]);
      nan = nan || v[i] != v[i];
      key[i] = larger((double)(v[i] + 0.0f), kMasked);   // (-0 is 0)
    }
    if (nan || most == __builtin_inff())
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i)
        key[i] = v[i] != v[i] ? 0x1p300 : v[i] == __builtin_inff() ? 0x1p200 : key[i];
  }
  __device__ __forceinline__ Entry entry(uint32_t i, uint32_t begin) const {
    const uint64_t b = __builtin_bit_cast(uint64_t, key[i]);
    // (a negative number is the smaller the larger its bits are)
    const uint32_t last = (int64_t)b < 0 ? begin + i : kIndex - begin - i;
    return __builtin_bit_cast(double, b | last);
  }
  static __device__ __forceinline__ bool any(Entry e) { return e > kMasked * 0.5; }
  static __device__ __forceinline__ int32_t index(Entry e) {
    const uint64_t b = __builtin_bit_cast(uint64_t, e);
    return (int32_t)(((int64_t)b < 0 ? b : ~b) & kIndex);
  }
  static __device__ __forceinline__ float value(Entry e) {
    if (e >= 0x1p300) return __builtin_nanf("");
    return (float)__builtin_bit_cast(double, __builtin_bit_cast(uint64_t, e) & ~(uint64_t)kIndex);   // (2^200: infinite)
  }
};

template <typename T, int kChunks, int kList, bool kAll>
__global__ void __launch_bounds__(256)
gate_list_kernel(Rows logits, uint32_t experts, uint32_t n, uint32_t k, Rows weights, Rows chosen, uint32_t shift) {
  const uint32_t lanes = 1u << shift, lane = threadIdx.x & (lanes - 1u), group = threadIdx.x >> shift;
  const uint32_t groups = 256u >> shift;
  for (uint64_t at = (uint64_t)blockIdx.x * groups; at < n; at += (uint64_t)gridDim.x * groups) {
    const uint32_t t = (uint32_t)at + group;
    const T* row = row_at<const T>(logits, min(t, n - 1u));
    // Eight adjacent logits an access, an access of the lanes after the other; the row's last one is moved
    // back so that it is whole, and what it has of the one before is -inf.
    uint32_t begin[kChunks];
    typename Packed<T, 8>::type v[kChunks];
#pragma unroll
    for (uint32_t c = 0; c < kChunks; ++c) {
      const uint32_t first = (c * lanes + lane) * 8;
      begin[c] = kChunks == 1 && experts < 8 ? 0u : min(first, experts - 8);
      if (kChunks == 1 && experts < 8) v[c] = own_logits<8>(row, 0u, experts, (T)-__builtin_inff());
      else v[c] = load<8>(row + begin[c]);
    }
#pragma unroll
    for (uint32_t c = 0; c < kChunks; ++c) {
      uint32_t others = (c * lanes + lane) * 8 - begin[c];
      asm volatile("" : "+v"(others));   // (the comparisons, kept for all tokens, would take more masks than there are)
      if (others)
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) v[c][i] = i < others ? (T)-__builtin_inff() : v[c][i];
    }
    typedef Listed<T> L;
    typename L::Entry list[kList];
#pragma unroll
    for (uint32_t i = 0; i < kList; ++i) list[i] = L::kNone;
#pragma unroll
    for (uint32_t c = 0; c < kChunks; ++c) {
      const L mine(v[c]);
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) insert(list, mine.entry(i, begin[c]));
      __builtin_amdgcn_sched_barrier(0);   // (all entries at once would take the registers of other wavefronts)
    }
    merge_group(list, shift);
    const float largest = L::any(list[0]) ? L::value(list[0]) : 0.0f;
    float sum = 0.0f;
    if constexpr (kAll) {
#pragma unroll
      for (uint32_t c = 0; c < kChunks; ++c)
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
          sum += expf((float)v[c][i] - largest);
          if (i % 2) __builtin_amdgcn_sched_barrier(0);
        }
      sum = group_sum(sum, shift);
    }
    // Entry j of the list is lane j's; of few lanes several.
    auto entry = [&](uint32_t j) {
      typename L::Entry e = list[0];
#pragma unroll
      for (uint32_t i = 1; i < kList; ++i) {
        const typename L::Entry x = list[i];   // (a value: of two places the compiler would keep the list in memory)
        e = j == i ? x : e;
      }
      return e;
    };
    auto power = [&](typename L::Entry e) { return L::any(e) ? expf(L::value(e) - largest) : 0.0f; };
    const typename L::Entry first = entry(lane);
    const float mine = power(first);
    if constexpr (!kAll) {
      for (uint32_t j = lane; j < k; j += lanes) sum += j == lane ? mine : power(entry(j));
      sum = group_sum(sum, shift);
    }
    if (t < n)
      for (uint32_t j = lane; j < k; j += lanes) {
        const typename L::Entry e = j == lane ? first : entry(j);
        put_number(chosen, t, j, L::any(e) ? L::index(e) : -1);
        put_float(weights, t, j, L::any(e) ? (j == lane ? mine : power(e)) / sum : 0.0f);
      }
  }
}

// ---------------------------------------------------------------------------
// themis_expert_gate_grad.  With w the weights and p the softmax over all logits:
//   over the chosen:  dl[e] = sum over j with e_j == e of w_j (dw_j - sum_i w_i dw_i)
//   over all:         dl[e] = sum over j with e_j == e of w_j dw_j  -  p_e sum_i w_i dw_i
// The lanes of a token hold its logits in the gate's chunks (over the chosen none: those of the list are read
// by themselves), and a pair (expert, gradient) each, whose term goes to the expert's lane through LDS.
// 65,536 tokens on 256 experts, eight of them (bf16): 15.9 us over the chosen (their bytes need 8), 27 over all
// (15); with every pair compared with every register 37 and 42.  Bound by waits: over the chosen the terms' 32 KB of
// LDS leave room for five workgroups, which issue on 32 % of the cycles, over all 176 registers for two wavefronts a
// SIMD, which issue on 60 %; a third of the instructions are the exponentials'.
// ---------------------------------------------------------------------------
template <typename T, typename Out, int kChunks, bool kAll>
__global__ void __launch_bounds__(256)
gate_grad_kernel(Rows grad, Rows logits, uint32_t experts, Rows chosen, uint32_t n, uint32_t k, Rows out, uint32_t shift) {
  __shared__ float terms[256 * 8 * kChunks];
  const uint32_t lanes = 1u << shift, lane = threadIdx.x & (lanes - 1u), group = threadIdx.x >> shift;
  const uint32_t groups = 256u >> shift;
  const float none = -__builtin_inff();
  float* term = terms + group * (lanes * 8 * kChunks);   // a token's, by expert
  const bool short_row = kChunks == 1 && experts < 8;
  for (uint64_t at = (uint64_t)blockIdx.x * groups; at < n; at += (uint64_t)gridDim.x * groups) {
    const uint32_t t0 = (uint32_t)at + group, t = min(t0, n - 1u);
    const T* row = row_at<const T>(logits, t);
    uint32_t begin[kChunks];   // (the row's last access is moved back, as in the gate)
    typename Packed<T, 8>::type v[kChunks];
#pragma unroll
    for (uint32_t c = 0; c < kChunks; ++c) {
      begin[c] = short_row ? 0u : min((c * lanes + lane) * 8, experts - 8);
      if (kAll) v[c] = short_row ? own_logits<8>(row, 0u, experts, (T)none) : load<8>(row + begin[c]);
    }
    struct Pair { uint32_t expert; float logit, grad; };
    auto pair_of = [&](uint32_t j) {
      Pair p = {~0u, none, 0.0f};
      if (j < k) p.expert = number_at(chosen, t, j, experts);
      if (p.expert != ~0u) {
        p.logit = (float)row[p.expert];
        p.grad = float_at(grad, t, j);
      }
      return p;
    };
    const Pair first = pair_of(lane);
    float top = none;   // (of NaN the others; it comes back in the sum)
    if constexpr (kAll) {
#pragma unroll
      for (uint32_t c = 0; c < kChunks; ++c)
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) top = fmaxf(top, (float)v[c][i]);
    } else {
      for (uint32_t j = lane; j < k; j += lanes) top = fmaxf(top, j == lane ? first.logit : pair_of(j).logit);
    }
    top = group_max(top, shift);
    const float largest = top > none ? top : 0.0f;
    float sum = 0.0f, dot = 0.0f;
    typename Packed<float, 8>::type e[kChunks];
    if constexpr (kAll) {
#pragma unroll
      for (uint32_t c = 0; c < kChunks; ++c) {
        const uint32_t others = short_row ? 0u : (c * lanes + lane) * 8 - begin[c];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
          e[c][i] = expf((float)v[c][i] - largest);
          sum += i >= others ? e[c][i] : 0.0f;
          if (i % 2) __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    for (uint32_t j = lane; j < k; j += lanes) {
      const Pair p = j == lane ? first : pair_of(j);
      if (p.expert == ~0u) continue;
      const float w = expf(p.logit - largest);
      if (!kAll) sum += w;
      dot += w * p.grad;
    }
    sum = group_sum(sum, shift);
    const bool any = !(sum == 0.0f);   // (of anything but -inf the sum is 1 at least, or NaN)
    const float scale = any ? 1.0f / sum : 0.0f;
    dot = group_sum(dot, shift) * scale;
    const float pull = dot * scale;
    // The terms: all at once where no expert stands twice in the wavefront's lists, else one after the other.
    auto term_of = [&](const Pair& p) {
      return expf(p.logit - largest) * scale * (kAll ? p.grad : p.grad - dot);
    };
    bool again = k > lanes;
    if (first.expert != ~0u)
      __hip_atomic_store((uint32_t*)term + first.expert, lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    again = again || (first.expert != ~0u && __hip_atomic_load((uint32_t*)term + first.expert, __ATOMIC_RELAXED,
                                                               __HIP_MEMORY_SCOPE_WORKGROUP) != lane);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (uint32_t c = 0; c < kChunks; ++c) *(Floats<8>*)(term + (c * lanes + lane) * 8) = 0.0f;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (!__any(again)) {
      if (first.expert != ~0u) term[first.expert] = term_of(first);
    } else {
      for (uint32_t j0 = 0; j0 < k; j0 += lanes) {
        const Pair p = j0 == 0 ? first : pair_of(j0 + lane);
        const float mine = term_of(p);
        for (uint32_t j = 0; j < min(k - j0, lanes); ++j) {
          if (lane == j && p.expert != ~0u) term[p.expert] += mine;
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (t0 < n) {
      Out* to = row_at<Out>(out, t);
#pragma unroll
      for (uint32_t c = 0; c < kChunks; ++c) {
        Floats<8> x;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
          x[i] = term[begin[c] + i];
          if (kAll) x[i] -= e[c][i] * pull;
        }
        if (short_row) store_some<8>(to, x, experts);
        else if ((c * lanes + lane) * 8 < experts) store<8>(to + begin[c], x);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (the next token's terms)
  }
}

// ---------------------------------------------------------------------------
// themis_expert_sort: pairs (token, expert) by expert, stable.
//
// As the table gradient's sort, in one pass: the workgroups count the experts of their parts of the
// list, then every workgroup finds from all counts where its part's pairs go.  One workgroup does both
// where the list is short.  Bound by waits: of 1,048,576 pairs on 256 experts the count takes 3 us, the rest 15.7 (each by
// itself; the call 17.2): 4 to the first barrier, 4.5 for the counts of 256 parts, 4 for the ranks, 3 for numbers of
// pairs that are written in runs of 16.
// ---------------------------------------------------------------------------
struct Order {
  uint32_t n, k, pairs, experts, capacity, slots;   // capacity 0: packed
  int32_t *place, *counts, *starts, *source;
};

constexpr uint32_t kPairGroup = 1024, kPairWaves = kPairGroup / 64;
constexpr uint32_t kPairsAhead = 4;    // of a lane in flight
constexpr uint32_t kPartsAhead = 16;   // counts

// Experts of the pairs a[] (token * k + j), ~0u for none.
template <int kPairs>
__device__ __forceinline__ void experts_of(const Order& o, const Rows& chosen, const uint32_t (&a)[kPairs],
                                           uint32_t (&expert)[kPairs]) {
  if (!chosen.inner && chosen.inner_stride == (int64_t)o.k) {   // one run of numbers
    const Rows run = {chosen.data, 0, 1, 0, chosen.type};
    token_rows(run, a, o.experts, expert);
    return;
  }
#pragma unroll
  for (int i = 0; i < kPairs; ++i) expert[i] = number_at(chosen, a[i] / o.k, a[i] % o.k, o.experts);
}

__device__ __forceinline__ void count_expert(uint32_t* bins, uint32_t expert, bool on) {
  if (on) atomicAdd(&bins[expert], 1u);
}

__global__ void __launch_bounds__(kPairGroup)
expert_count_kernel(Order o, Rows chosen, uint32_t part, uint32_t* counts) {
  __shared__ uint32_t count[kMostExperts];
  const uint32_t first = blockIdx.x * part, last = min(first + part, o.pairs);
  for (uint32_t b = threadIdx.x; b < o.experts; b += kPairGroup) count[b] = 0;
  __syncthreads();
  for (uint32_t i = first + threadIdx.x; i < last; i += kPairsAhead * kPairGroup) {
    uint32_t at[kPairsAhead], expert[kPairsAhead];
#pragma unroll
    for (uint32_t k = 0; k < kPairsAhead; ++k) at[k] = min(i + k * kPairGroup, last - 1u);
    experts_of(o, chosen, at, expert);
#pragma unroll
    for (uint32_t k = 0; k < kPairsAhead; ++k)
      count_expert(count, expert[k], i + k * kPairGroup < last && expert[k] != ~0u);
  }
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < o.experts; b += kPairGroup) counts[blockIdx.x * o.experts + b] = count[b];
}

__global__ void __launch_bounds__(kPairGroup)
expert_sort_kernel(Order o, Rows chosen, uint32_t part, uint32_t parts, const uint32_t* counts, uint32_t bits) {
  __shared__ uint32_t next[kPairWaves][kMostExperts];   // first a wavefront's counts, then where its next one goes
  __shared__ uint32_t wave_sums[kPairWaves], shared_before[kPairGroup], shared_all[kPairGroup];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
  // Workgroups go round the eight XCDs; the parts of one XCD stand together, so that what they write side by side
  // meets in its cache (1,048,576 pairs: 15.7 us, with a part for every workgroup in turn 16.3).
  const uint32_t xcd = blockIdx.x % 8, mine = xcd * (parts / 8) + min(xcd, parts % 8) + blockIdx.x / 8;
  const uint32_t first = mine * part, share = part / kPairWaves;   // (a multiple of 64)
  const uint32_t begin = min(first + wave * share, o.pairs), end = min(begin + share, o.pairs);
  const uint32_t b = threadIdx.x;   // a lane has one expert, or none
  if (b < o.experts)
#pragma unroll
    for (uint32_t w = 0; w < kPairWaves; ++w) next[w][b] = 0;
  uint32_t expert[kPairsAhead];   // (of the first turn: read before the barrier, and kept where it is the only one)
  {
    uint32_t at[kPairsAhead];
#pragma unroll
    for (uint32_t k = 0; k < kPairsAhead; ++k) at[k] = min(begin + k * 64 + lane, o.pairs - 1u);
    if (begin < end) experts_of(o, chosen, at, expert);
  }
  __syncthreads();
  for (uint32_t i = begin; i < end; i += kPairsAhead * 64) {
    uint32_t at[kPairsAhead];
#pragma unroll
    for (uint32_t k = 0; k < kPairsAhead; ++k) at[k] = min(i + k * 64 + lane, end - 1u);
    if (i != begin) experts_of(o, chosen, at, expert);
#pragma unroll
    for (uint32_t k = 0; k < kPairsAhead; ++k)
      count_expert(next[wave], expert[k], i + k * 64 + lane < end && expert[k] != ~0u);
  }
  // Of every expert: pairs in the parts before, and in all.  The lanes of an expert take some parts each.
  uint32_t before = 0, all = 0;
  if (parts > 1) {
    const uint32_t e = threadIdx.x & ((1u << bits) - 1u), sharer = threadIdx.x >> bits;
    const uint32_t some = max((parts + (kPairGroup >> bits) - 1) / (kPairGroup >> bits), kPartsAhead);
    const uint32_t sharers = (parts + some - 1) / some, from = min(sharer * some, parts), to = min(from + some, parts);
    if (e < o.experts)
      for (uint32_t p = from; p < to; p += kPartsAhead) {
        uint32_t c[kPartsAhead];
#pragma unroll
        for (uint32_t k = 0; k < kPartsAhead; ++k) c[k] = counts[min(p + k, to - 1u) * o.experts + e];
#pragma unroll
        for (uint32_t k = 0; k < kPartsAhead; ++k) {
          before += p + k < min(to, mine) ? c[k] : 0u;
          all += p + k < to ? c[k] : 0u;
        }
      }
    shared_before[threadIdx.x] = before;
    shared_all[threadIdx.x] = all;
    __syncthreads();
    before = all = 0;
    if (b < o.experts)
      for (uint32_t q = 0; q < sharers; ++q) {
        before += shared_before[(q << bits) + b];
        all += shared_all[(q << bits) + b];
      }
  }
  __syncthreads();   // (the wavefronts' counts are complete)
  if (parts == 1 && b < o.experts)
#pragma unroll
    for (uint32_t w = 0; w < kPairWaves; ++w) all += next[w][b];
  uint32_t upto = all;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(upto, d);
    if (lane >= (uint32_t)d) upto += y;
  }
  if (lane == 63) wave_sums[wave] = upto;
  __syncthreads();
  uint32_t start = upto - all, total = 0;   // where the expert's pairs begin; how many pairs have an expert
#pragma unroll
  for (uint32_t w = 0; w < kPairWaves; ++w) {
    start += w < wave ? wave_sums[w] : 0u;
    total += wave_sums[w];
  }
  if (o.capacity) start = b * o.capacity;
  if (b < o.experts) {
    uint32_t at = before;   // (counted from the expert's first)
#pragma unroll
    for (uint32_t w = 0; w < kPairWaves; ++w) {
      const uint32_t c = next[w][b];
      next[w][b] = at;
      at += c;
    }
  }
  uint32_t* starts = shared_before;   // (read above for the last time before the last barrier)
  uint32_t* filled = shared_all;
  if (b < o.experts) {
    starts[b] = start;
    filled[b] = all;
  }
  if (blockIdx.x == 0) {
    if (b < o.experts) {
      o.counts[b] = (int32_t)all;
      o.starts[b] = (int32_t)start;
    }
    if (b == 0) o.starts[o.experts] = (int32_t)(o.capacity ? o.slots : total);
  }
  __syncthreads();
  for (uint32_t i0 = begin; i0 < end; i0 += kPairsAhead * 64) {
    uint32_t from[kPairsAhead];
#pragma unroll
    for (uint32_t k = 0; k < kPairsAhead; ++k) from[k] = min(i0 + k * 64 + lane, end - 1u);
    if (share > kPairsAhead * 64) experts_of(o, chosen, from, expert);
#pragma unroll
    for (uint32_t k = 0; k < kPairsAhead; ++k) {
      if (i0 + k * 64 >= end) break;
      const bool in = i0 + k * 64 + lane < end, on = in && expert[k] != ~0u;
      uint64_t same = __ballot(on);   // lanes with this lane's expert
      for (uint32_t x = 0; x < bits; ++x) {
        const uint64_t ones = __ballot((expert[k] >> x) & 1u);
        same &= (expert[k] >> x) & 1u ? ones : ~ones;
      }
      const uint32_t rank = (uint32_t)__popcll(same & ((1ull << lane) - 1));
      // (all lanes have read before the first of an expert's adds: a wavefront's accesses to LDS are
      // served in the order of the program, and these are kept in it)
      uint32_t* seat = &next[wave][on ? expert[k] : 0u];
      const uint32_t to = (on ? __hip_atomic_load(seat, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) : 0u) + rank;
      if (on && rank == 0)
        __hip_atomic_store(seat, to + (uint32_t)__popcll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      const bool kept = on && (!o.capacity || to < o.capacity);
      const uint32_t slot = kept ? starts[expert[k]] + to : ~0u;
      if (in) o.place[from[k]] = (int32_t)slot;
      if (kept) o.source[slot] = (int32_t)from[k];
    }
  }
  // Slots of no pair.
  if (!o.capacity) {
    for (uint64_t s = total + (uint64_t)blockIdx.x * kPairGroup + threadIdx.x; s < o.slots; s += (uint64_t)parts * kPairGroup)
      o.source[s] = -1;
    return;
  }
  for (uint64_t e = blockIdx.x * kPairWaves + wave; e < o.experts; e += (uint64_t)parts * kPairWaves)
    for (uint64_t s = (uint64_t)filled[e] + lane; s < o.capacity; s += 64) o.source[e * o.capacity + s] = -1;
}

// ---------------------------------------------------------------------------
// Rows into the order of the experts and back: eight elements a lane.  A place that is no slot (-1, or
// what a caller wrote there) is none.  What is written by slots goes by both directions: slot s is pair a's
// where place[a] is s and source[s] is a, and is cleared where that is so for no pair, so that in an order
// which a caller has changed, too, every slot is written, and once.  (The looks at the other direction: rows of
// 4,096 bf16 take as long as without, 100,000 tokens' rows of 64 to six places 23 us for 19.4.)
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t source_of(const Order& o, uint32_t s) {
  return s < o.slots ? (uint32_t)o.source[s] : ~0u;
}

// sum += x * w, each element rounded once.
__device__ __forceinline__ void add_product(float8& sum, float8 x, float w) {
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] = __builtin_fmaf(x[i], w, sum[i]);
}

// Zeros in the slots of no pair, by workgroup `block` of `blocks`.  kAway, here and below: past the caches.
template <bool kWhole, bool kAway, typename Out>
__device__ __forceinline__ void clear_empty_slots(const Order& o, uint32_t block, uint32_t blocks, uint32_t rows,
                                                  uint32_t width, const Rows& out) {
  const uint32_t lane = threadIdx.x & 63u;
  for (uint64_t s0 = (uint64_t)block * rows; s0 < o.slots; s0 += (uint64_t)blocks * rows) {
    const uint32_t s = (uint32_t)s0 + lane;
    bool empty = lane < rows && s < o.slots;
    if (empty) {
      const uint32_t pair = (uint32_t)o.source[s];
      empty = pair >= o.pairs || (uint32_t)o.place[pair] != s;
    }
    write_zeros<kWhole, kAway, Out>(__ballot(empty), (uint32_t)s0, width, out);
  }
}

// themis_expert_dispatch: a row is read once and written to its token's slots, kAhead places looked up in front of
// the writes; the first `fills` workgroups clear the slots of no pair.  Bound by memory: 131,072 rows of 4,096 bf16,
// eight of every row read, in 228 us, 5.3 TB/s, where a fill makes 6.8; slot by slot, in the order of the memory that
// is written, each row is read eight times from the caches and it takes 300.
constexpr int kOneWrite = 0x0F71;   // s_waitcnt: at most one access to memory is under way
template <bool kWhole, bool kAway, int kAhead, typename In, typename Out>
__global__ void __launch_bounds__(256)
dispatch_kernel(Order o, Rows x, uint32_t width, Rows out, Spread spread, uint32_t fills, uint32_t fill_rows) {
  if (blockIdx.x < fills) {
    if (blockIdx.y == 0) clear_empty_slots<kWhole, kAway, Out>(o, blockIdx.x, fills, fill_rows, width, out);
    return;
  }
  spread_rows(spread, blockIdx.x - fills, o.n, [&](uint32_t t, uint32_t lane) {
    const Slice<kVecOf<In, Out>> slice(0, lane, spread.lanes, width);
    const uint32_t first = t * o.k;
    const float8 v = widen<8>(slice.template read<kWhole>(row_at<const In>(x, t)));
    for (uint32_t j0 = 0; j0 < o.k; j0 += kAhead) {
      uint32_t s[kAhead], source[kAhead];
#pragma unroll
      for (uint32_t u = 0; u < kAhead; ++u) s[u] = j0 + u < o.k ? (uint32_t)o.place[first + j0 + u] : ~0u;
#pragma unroll
      for (uint32_t u = 0; u < kAhead; ++u) source[u] = source_of(o, s[u]);
#pragma unroll
      for (uint32_t u = 0; u < kAhead; ++u)
        if (source[u] == first + j0 + u) {
          slice.template write_over<kWhole, kAway>(row_at<Out>(out, s[u]), v);
          // (the memory takes the writes of many rows the better the fewer of them a wavefront has under way:
          // eight at once 244 us; two places, then two writes 238)
          if (kAhead > 2) __builtin_amdgcn_s_waitcnt(kOneWrite);
        }
    }
  });
}

// themis_expert_combine: out[t] (+)= sum over j of weights[t][j] * y[place[t][j]], kAhead rows in flight.
// Bound by the waits for places, then rows, which other wavefronts fill: few instructions and registers count
// (1.07 GB of rows added to 0.13 GB 238 us; products and sums by themselves, what is added to read last 250; the next
// token's places asked for in advance 273; eight rows in flight 301).  kOnce, here and below: y is read past the caches.
template <bool kWhole, bool kOnce, int kAhead, typename In, typename Out>
__global__ void __launch_bounds__(256)
combine_kernel(Order o, Rows y, uint32_t width, Rows weights, bool accumulate, Rows out, Spread spread) {
  spread_rows(spread, blockIdx.x, o.n, [&](uint32_t t, uint32_t lane) {
    const Slice<kVecOf<In, Out>> slice(0, lane, spread.lanes, width);
    const int32_t* place = o.place + (uint64_t)t * o.k;
    const int64_t weights_at = row_offset(weights, t);
    Out* to = row_at<Out>(out, t);
    float8 sum = 0.0f;
    if (accumulate) sum = widen<8>(slice.template read<kWhole>((const Out*)to));
    for (uint32_t j0 = 0; j0 < o.k; j0 += kAhead) {
      uint32_t s[kAhead];
      float w[kAhead];
      typename Packed<In, 8>::type v[kAhead];
#pragma unroll
      for (uint32_t u = 0; u < kAhead; ++u) s[u] = j0 + u < o.k ? (uint32_t)place[j0 + u] : ~0u;
#pragma unroll
      for (uint32_t u = 0; u < kAhead; ++u) {
        w[u] = 1.0f;
        if (weights.data && j0 + u < o.k)
          w[u] = weights.type == THEMIS_F32 ? ((const float*)weights.data)[weights_at + j0 + u] : float_at(weights, t, j0 + u);
      }
#pragma unroll
      for (uint32_t u = 0; u < kAhead; ++u) {
        v[u] = {};
        if (s[u] < o.slots) v[u] = slice.template read<kWhole, kOnce>(row_at<const In>(y, s[u]));
      }
#pragma unroll
      for (uint32_t u = 0; u < kAhead; ++u) add_product(sum, widen<8>(v[u]), s[u] < o.slots ? w[u] : 0.0f);
    }
    slice.template write<kWhole>(to, sum);
  });
}

// themis_expert_combine_grad: rows[s] = weights[a] * grad[t] and weights'[a] = <grad[t], y[s]> for the pair
// a = (t, j) in slot s.  2^shift lanes (up to a wavefront) take two of a token's pairs over the whole row, so
// that a product is summed where it is made.  Bound by memory and by its instructions: 268 MB of rows of 4,096 bf16
// read and 335 written 135 us (5.5 TB/s); one pair or four for a wavefront cost up to 29 % and 7 % more.
constexpr uint32_t kGradPairs = 2;
template <bool kWhole, bool kOnce, bool kAway, typename G, typename Y>
__global__ void __launch_bounds__(256)
combine_grad_kernel(Order o, Rows grad, uint32_t width, Rows y, Rows weights, Rows rows, Rows grad_weights, uint32_t shift,
                    uint32_t fills, uint32_t fill_rows) {
  if (blockIdx.x < fills) {
    clear_empty_slots<kWhole, kAway, Y>(o, blockIdx.x, fills, fill_rows, width, rows);
    return;
  }
  const uint32_t lanes = 1u << shift, lane = threadIdx.x & (lanes - 1u), each = (o.k + kGradPairs - 1) / kGradPairs;
  const uint32_t groups = 256u >> shift, block = blockIdx.x - fills, blocks = gridDim.x - fills;
  const uint32_t units = o.n * each;   // (no more than pairs)
  for (uint64_t u0 = (uint64_t)block * groups; u0 < units; u0 += (uint64_t)blocks * groups) {
    const uint32_t unit = (uint32_t)u0 + (threadIdx.x >> shift);
    const bool mine = unit < units;
    const uint32_t t = mine ? unit / each : 0u, j0 = mine ? unit % each * kGradPairs : 0u;
    uint32_t s[kGradPairs], source[kGradPairs];
    float w[kGradPairs], dot[kGradPairs];
#pragma unroll
    for (uint32_t u = 0; u < kGradPairs; ++u) {
      const uint32_t j = min(j0 + u, o.k - 1u);
      s[u] = mine && j0 + u < o.k ? (uint32_t)o.place[(uint64_t)t * o.k + j] : ~0u;
      w[u] = float_at(weights, t, j);
      dot[u] = 0.0f;
    }
#pragma unroll
    for (uint32_t u = 0; u < kGradPairs; ++u) source[u] = rows.data ? source_of(o, s[u]) : ~0u;
    for (uint32_t c = 0; c < width; c += lanes * kLaneElements) {
      const Slice<kVecOf<G, Y>> slice(c, lane, lanes, width);
      if (!slice.any()) continue;
      const float8 g = widen<8>(slice.template read<kWhole>(row_at<const G>(grad, t)));
      // (other lanes' elements: a choice for the wavefront, since most have none and instructions count)
      const bool whole = !__ballot(!slice.whole());
      typename Packed<Y, 8>::type v[kGradPairs];
#pragma unroll
      for (uint32_t u = 0; u < kGradPairs; ++u) {
        v[u] = {};
        if (grad_weights.data && s[u] < o.slots) v[u] = slice.template read<kWhole, kOnce>(row_at<const Y>(y, s[u]));
      }
#pragma unroll
      for (uint32_t u = 0; u < kGradPairs; ++u) {
        if (s[u] >= o.slots) continue;
        if (source[u] == t * o.k + j0 + u) slice.template write_over<kWhole, kAway>(row_at<Y>(rows, s[u]), g * w[u]);
        float8 a = widen<8>(v[u]), b = g;
        if (!whole) {
          a = slice.template own<kWhole>(a);
          b = slice.template own<kWhole>(b);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) dot[u] = __builtin_fmaf(a[i], b[i], dot[u]);
      }
    }
    if (!grad_weights.data) continue;
#pragma unroll
    for (uint32_t u = 0; u < kGradPairs; ++u) {
      const float sum = group_sum(dot[u], shift);
      if (mine && lane == 0 && j0 + u < o.k) put_float(grad_weights, t, j0 + u, sum);
    }
  }
}

}  // namespace themis
