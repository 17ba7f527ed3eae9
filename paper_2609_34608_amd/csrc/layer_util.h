// What the layer operators without a handle share: wide loads and stores of rows at
// any alignment, and the checks of their arguments.
#pragma once

#include "fp8.h"
#include "wam_internal.h"

namespace wam {

// ------------------------------------------------------------- elements
// N consecutive elements at p, which needs only the alignment of an element:
// global memory takes wide loads and stores at any address.  Elements from n on
// are zero (not loaded) or left alone (not stored).
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
  T v[N];
};
template <int N, typename T>
__device__ __forceinline__ void load_n(float (&x)[N], const T* p, int n) {
  if (n >= N) {
    const Pack<T, N> w = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_f32(w.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}

template <int N, typename T>
__device__ __forceinline__ void store_n(T* p, const float (&x)[N], int n, bool stream) {
  Pack<T, N> w;
#pragma unroll
  for (int i = 0; i < N; ++i) w.v[i] = static_cast<T>(x[i]);
  if (n >= N) {
    put(p, w, stream);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = w.v[i];
  }
}

template <int N>
__device__ __forceinline__ uint32_t most_of(const float (&x)[N]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) most = max(most, abs_bits(x[i]));
  return most;
}

// ------------------------------------------------------------- argument checks
constexpr int64_t kMaxStride = (int64_t)1 << 40;  // a larger one is no buffer of this machine

// Elements of a strided result are distinct: by stride, each dimension of more
// than one index steps over the whole of the smaller ones (the last, contiguous
// one has `inner` elements).
inline bool distinct(const int64_t* stride, const int64_t* size, int n, int64_t inner) {
  bool used[3] = {false, false, false};
  int64_t extent = inner;
  for (int step = 0; step < n; ++step) {
    int at = -1;
    for (int i = 0; i < n; ++i)
      if (!used[i] && size[i] > 1 && (at < 0 || stride[i] < stride[at])) at = i;
    if (at < 0) return true;
    if (stride[at] < extent) return false;
    extent = stride[at] * (size[at] - 1) + extent;
    used[at] = true;
  }
  return true;
}
// strides of at most 2^40 elements, so that no offset or extent passes 64 bits
inline bool strides_ok(const int64_t* stride, int n) {
  for (int i = 0; i < n; ++i)
    if (stride[i] < 0 || stride[i] > kMaxStride) return false;
  return true;
}
inline bool same(const int64_t* a, const int64_t* b, int n) {
  for (int i = 0; i < n; ++i)
    if (a[i] != b[i]) return false;
  return true;
}
inline bool float_type(int t) { return t == WAM_FP32 || t == WAM_BF16; }
inline int64_t type_size(int t) { return t == WAM_FP32 ? 4 : t == WAM_BF16 ? 2 : 1; }
inline bool aligned_to(const void* p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)n == 0; }

// blocks of 256 threads along one dimension of a grid, whose threads count in 32 bits
constexpr int64_t kMaxGrid = (1 << 24) - 1;

}  // namespace wam
