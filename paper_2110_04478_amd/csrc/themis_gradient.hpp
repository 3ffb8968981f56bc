// Norms of a list of gradients and their clipped copies (themis_gradient_norm, _clip).
//
// The list is cut into pieces of at most kPieceMost elements once, on the host; a piece never
// spans two tensors.  A pass over the list is one launch in which every workgroup takes pieces at
// a fixed distance, so which workgroup adds what depends on the list alone.  The squares are
// binary64: a conversion and a fused multiply-add per element, a tenth of what the vector units
// can issue while the elements come from memory, and no scaling against overflow is needed.
//
// What is not one run of elements goes element by element, with a division each: three column slices
// of 4,096^2 bf16 take 83 us (dense 24), 162 when they are clipped (57).
//
// Clipping is a second launch, in which every workgroup adds the first one's sums again, in the same
// order (8 KiB), and takes the pieces from the last to the first.  Bound by memory: the norm of
// 1.74 G bf16 elements 499 us, 7.0 TB/s; 1.07 G binary32 elements into bf16 1,730 us, 6.2 TB/s of
// what is read twice and written once; 134 M bf16 elements 136 us; small lists by two launches.
#pragma once

#include "themis_elements.hpp"

namespace themis {

constexpr uint32_t kPieceLeast = 2048;   // one access of 256 lanes
constexpr uint32_t kPieceMost = 65536;
constexpr uint32_t kInFlight = 8;        // accesses of a lane

// Workgroups of a pass over the list: four for every CU, two where the list is long and each has
// many pieces (1.07 G binary32 elements clipped into bf16 1,727 us, with four 1,770; 16.8 M bf16
// 36 and 31 us).
inline uint32_t pass_groups(uint64_t n_pieces, uint64_t bytes) {
  const uint32_t most = bytes >= 1ull << 30 ? 512 : 1024;
  return n_pieces < most ? (uint32_t)n_pieces : most;
}
// Elements of a piece: one for every workgroup while that keeps its lanes' accesses in flight, then
// eight for every workgroup, so that they end together.
inline uint64_t piece_elements(uint64_t total) {
  const uint64_t one = total / 1024 < 16384 ? total / 1024 : 16384;
  const uint64_t eight = total / 8192 < kPieceMost ? total / 8192 : kPieceMost;
  const uint64_t some = one > eight ? one : eight;
  return some <= kPieceLeast ? kPieceLeast : (some + kPieceLeast - 1) / kPieceLeast * kPieceLeast;
}

// The last cache level holds 256 MiB: of a list that is longer, all but its last part is read past
// it in the first pass, so that the part the second pass begins with is still there (clip of 1.07 G
// binary32 elements 1,798 -> 1,773 us, of 134 M bf16 elements 144 -> 137 us; nothing past it:
// 1,873 and 138 us; the norm of 1.74 G bf16 elements 583 -> 514 us).
constexpr uint64_t kKeptBytes = 192ull << 20;

enum : uint32_t { kInDense = 1u << 16, kOutDense = 1u << 17, kInPlace = 1u << 18 };

struct Piece {
  const void* in;
  void* out;
  uint32_t count;   // elements
  uint32_t cols;    // element e is (e / cols, e % cols)
  uint32_t tensor;
  uint32_t kind;    // in type | out type << 8 | kInDense ..
  int64_t in_row, in_col, out_row, out_col;   // strides, elements
};
static_assert(sizeof(Piece) == 64, "an image's layout");

// The image: the pieces, then for every tensor the number of its first piece (and n_pieces).
struct PlanView {
  const Piece* pieces;
  const uint32_t* first;
  uint32_t n_pieces, n_tensors;
};
inline PlanView plan_view(const themis_gradient_plan_t& p) {
  return {(const Piece*)p.image, (const uint32_t*)((const char*)p.image + p.n_pieces * sizeof(Piece)),
          (uint32_t)p.n_pieces, (uint32_t)p.n_tensors};
}

// The workspace: the workgroups' sums of squares (pass_groups()), then the pieces'.

// ---------------------------------------------------------------------------
// Sums over a workgroup of 256 lanes, the same in every lane.
// ---------------------------------------------------------------------------
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ double group_sum(double x, double (&part)[4]) {
  x = wave_sum(x);
  __syncthreads();   // part may still be read from the sum before
  if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

template <int N>
__device__ __forceinline__ double squares(Floats<N> v, double sum) {
  double odd = 0.0;
#pragma unroll
  for (int k = 0; k < N; k += 2) {
    sum = fma((double)v[k], (double)v[k], sum);
    odd = fma((double)v[k + 1], (double)v[k + 1], odd);
  }
  return sum + odd;
}

// A lane's share of a piece's sum of squares; kOnce: read past the caches.
template <bool kOnce, typename T>
__device__ __forceinline__ double piece_squares(const Piece& p) {
  const T* in = (const T*)p.in;
  double sum = 0.0;
  if (p.kind & kInDense) {
    constexpr int kVec = kVecOf<T>;
    constexpr uint32_t kStep = 256 * kVec, kUnroll = kInFlight;
    uint32_t e = threadIdx.x * kVec;
    for (; e + (kUnroll - 1) * kStep + kVec <= p.count; e += kUnroll * kStep) {
      typename Packed<T, kVec>::type v[kUnroll];
#pragma unroll
      for (uint32_t k = 0; k < kUnroll; ++k)
        v[k] = kOnce ? load_once<kVec>(in + e + k * kStep) : load<kVec>(in + e + k * kStep);
#pragma unroll
      for (uint32_t k = 0; k < kUnroll; ++k) sum = squares<kVec>(widen<kVec>(v[k]), sum);
    }
    for (; e < p.count; e += kStep)
      sum = squares<kVec>(widen<kVec>(load_some<kVec>(in + e, min(p.count - e, (uint32_t)kVec))), sum);
  } else {
    for (uint32_t e = threadIdx.x; e < p.count; e += 256) {
      const uint32_t r = e / p.cols, c = e - r * p.cols;
      const double x = (double)(float)in[(int64_t)r * p.in_row + (int64_t)c * p.in_col];
      sum = fma(x, x, sum);
    }
  }
  return sum;
}

template <bool kOnce>
__device__ __forceinline__ double piece_squares_of(const Piece& p) {
  const uint32_t type = p.kind & 0xffu;
  return type == THEMIS_F32 ? piece_squares<kOnce, float>(p)
         : type == THEMIS_BF16 ? piece_squares<kOnce, __bf16>(p) : piece_squares<kOnce, _Float16>(p);
}

__global__ void __launch_bounds__(256)
norm_kernel(PlanView plan, uint32_t passed, double* __restrict__ group_sums, double* __restrict__ piece_sums) {
  __shared__ double part[4];
  double total = 0.0;
  for (uint32_t i = blockIdx.x; i < plan.n_pieces; i += gridDim.x) {
    const Piece& p = plan.pieces[i];
    double s = i < passed ? piece_squares_of<true>(p) : piece_squares_of<false>(p);
    s = group_sum(s, part);
    total += s;
    if (threadIdx.x == 0) piece_sums[i] = s;
  }
  if (threadIdx.x == 0) group_sums[blockIdx.x] = total;
}

// The sum of squares of the whole list, in every lane of every workgroup that asks.
__device__ __forceinline__ double list_squares(uint32_t groups, const double* __restrict__ group_sums,
                                               double (&part)[4]) {
  double x = 0.0;
  for (uint32_t w = threadIdx.x; w < groups; w += 256) x += group_sums[w];
  return group_sum(x, part);
}

// Norms of four tensors, one for every wavefront of workgroup `block`.
__device__ __forceinline__ void tensor_norms(const PlanView& plan, uint32_t block,
                                             const double* __restrict__ piece_sums, float* __restrict__ norms) {
  const uint32_t t = block * 4u + (threadIdx.x >> 6);
  if (t >= plan.n_tensors) return;
  const uint32_t end = plan.first[t + 1];
  double x = 0.0;
  for (uint32_t i = plan.first[t] + (threadIdx.x & 63u); i < end; i += 64 * kInFlight) {
    double s[kInFlight];
#pragma unroll
    for (uint32_t k = 0; k < kInFlight; ++k) s[k] = piece_sums[min(i + k * 64, end - 1u)];
#pragma unroll
    for (uint32_t k = 0; k < kInFlight; ++k) x += i + k * 64 < end ? s[k] : 0.0;
  }
  x = wave_sum(x);
  if ((threadIdx.x & 63u) == 0) norms[t] = (float)sqrt(x);
}

__global__ void __launch_bounds__(256)
norm_finish_kernel(PlanView plan, uint32_t groups, const double* __restrict__ group_sums,
                   const double* __restrict__ piece_sums, float* __restrict__ total, float* __restrict__ norms) {
  __shared__ double part[4];
  if (blockIdx.x) return tensor_norms(plan, blockIdx.x - 1, piece_sums, norms);
  const double x = list_squares(groups, group_sums, part);
  if (threadIdx.x == 0) total[0] = (float)sqrt(x);
}

template <typename In, typename Out>
__device__ __forceinline__ void scale_piece(const Piece& p, float factor) {
  const In* in = (const In*)p.in;
  Out* out = (Out*)p.out;
  if ((p.kind & (kInDense | kOutDense)) == (kInDense | kOutDense)) {
    constexpr int kVec = kVecOf<In, Out>;
    constexpr uint32_t kStep = 256 * kVec, kUnroll = kInFlight;
    uint32_t e = threadIdx.x * kVec;
    for (; e + (kUnroll - 1) * kStep + kVec <= p.count; e += kUnroll * kStep) {
      typename Packed<In, kVec>::type v[kUnroll];
#pragma unroll
      for (uint32_t k = 0; k < kUnroll; ++k) v[k] = load_once<kVec>(in + e + k * kStep);
#pragma unroll
      for (uint32_t k = 0; k < kUnroll; ++k) store_away<kVec>(out + e + k * kStep, widen<kVec>(v[k]) * factor);
    }
    for (; e < p.count; e += kStep) {
      const uint32_t some = min(p.count - e, (uint32_t)kVec);
      store_some<kVec>(out + e, widen<kVec>(load_some<kVec>(in + e, some)) * factor, some);
    }
  } else {
    for (uint32_t e = threadIdx.x; e < p.count; e += 256) {
      const uint32_t r = e / p.cols, c = e - r * p.cols;
      out[(int64_t)r * p.out_row + (int64_t)c * p.out_col] =
          (Out)((float)in[(int64_t)r * p.in_row + (int64_t)c * p.in_col] * factor);
    }
  }
}
template <typename In>
__device__ __forceinline__ void scale_piece_to(const Piece& p, float factor) {
  const uint32_t type = (p.kind >> 8) & 0xffu;
  if (type == THEMIS_F32) scale_piece<In, float>(p, factor);
  else if (type == THEMIS_BF16) scale_piece<In, __bf16>(p, factor);
  else scale_piece<In, _Float16>(p, factor);
}

// The first `scalers` workgroups scale, the others take the tensors' norms.
__global__ void __launch_bounds__(256)
clip_kernel(PlanView plan, uint32_t groups, const double* __restrict__ group_sums,
            const double* __restrict__ piece_sums, double max_norm, uint32_t scalers, float* __restrict__ total,
            float* __restrict__ norms) {
  __shared__ double part[4];
  if (blockIdx.x >= scalers) return tensor_norms(plan, blockIdx.x - scalers, piece_sums, norms);
  const double norm = sqrt(list_squares(groups, group_sums, part));
  const double ratio = norm <= max_norm ? 1.0 : max_norm / norm;   // (NaN stays NaN)
  const float factor = (float)ratio;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    total[0] = (float)norm;
    total[1] = factor;
  }
  for (uint32_t i = blockIdx.x; i < plan.n_pieces; i += scalers) {
    const Piece& p = plan.pieces[plan.n_pieces - 1 - i];
    if ((p.kind & kInPlace) && factor == 1.0f) continue;
    const uint32_t type = p.kind & 0xffu;
    if (type == THEMIS_F32) scale_piece_to<float>(p, factor);
    else if (type == THEMIS_BF16) scale_piece_to<__bf16>(p, factor);
    else scale_piece_to<_Float16>(p, factor);
  }
}

}  // namespace themis
