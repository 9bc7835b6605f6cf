// lists.hpp -- eight values at a time, and lists of tensors brought to a kernel
// in its arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace pp {

// Consecutive values; the hardware loads and stores 16 bytes at any address of the
// element's own alignment.
template <class S>
using Eight = __attribute__((ext_vector_type(8), aligned(sizeof(S)))) S;
template <class S>
using Four = __attribute__((ext_vector_type(4), aligned(sizeof(S)))) S;

// ONCE: it is not used again soon, and takes no room in the caches
template <bool ONCE, class T>
__device__ __forceinline__ T fetch(const T* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  return *p;
}
template <bool ONCE, class T>
__device__ __forceinline__ void keep_at(T* p, T x) {
  if constexpr (ONCE)
    __builtin_nontemporal_store(x, p);
  else
    *p = x;
}

// The n values from p on, or as many as a vector has; 0 in the place of the others.
template <bool ONCE, class V, class S>
__device__ __forceinline__ V get(const S* p, int64_t n) {
  constexpr int N = sizeof(V) / sizeof(S);
  if (n >= N) return fetch<ONCE>(reinterpret_cast<const V*>(p));
  V x;
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = e < n ? p[e] : static_cast<S>(0.f);
  return x;
}
template <bool ONCE, class V, class S>
__device__ __forceinline__ void put(S* p, int64_t n, const V& x) {
  constexpr int N = sizeof(V) / sizeof(S);
  if (n >= N) {
    keep_at<ONCE>(reinterpret_cast<V*>(p), x);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) p[e] = x[e];
  }
}

// A lane's eight of the n values from p on: in a row, or (SPLIT) four, and four `far`
// values further on.  Lanes that lie 8, or 4, values apart then have 16 bytes in a row
// at each access, whole lines together.
template <class... S>
constexpr bool kSplit = ((sizeof(S) == 4) || ...);
template <bool SPLIT, bool ONCE = false, class S>
__device__ __forceinline__ Eight<S> get8(const S* p, int64_t n, int far) {
  if constexpr (SPLIT) {
    const Four<S> x = get<ONCE, Four<S>>(p, n), y = get<ONCE, Four<S>>(p + far, n - far);
    return {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  } else {
    return get<ONCE, Eight<S>>(p, n);
  }
}
template <bool SPLIT, bool ONCE = false, class S>
__device__ __forceinline__ void put8(S* p, int64_t n, int far, const Eight<S>& x) {
  if constexpr (SPLIT) {
    put<ONCE>(p, n, Four<S>{x[0], x[1], x[2], x[3]});
    put<ONCE>(p + far, n - far, Four<S>{x[4], x[5], x[6], x[7]});
  } else {
    put<ONCE>(p, n, x);
  }
}
// the same by way of fp32
template <bool SPLIT, bool ONCE = false, class S>
__device__ __forceinline__ void load8(const S* p, int64_t n, int far, float (&v)[8]) {
  const Eight<S> x = get8<SPLIT, ONCE>(p, n, far);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(x[e]);
}
template <bool SPLIT, bool ONCE = false, class S>
__device__ __forceinline__ void store8(S* p, int64_t n, int far, const float (&v)[8]) {
  Eight<S> x;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = static_cast<S>(v[e]);
  put8<SPLIT, ONCE>(p, n, far, x);
}

// A list's tensors in a kernel's arguments (which hold 4 KB), each with the
// first of its workgroups.
template <class Item, int N>
struct List {
  Item item[N];
  int32_t first[N];
  int32_t count;
};
// The tensor that workgroup `id` is of; *local: which of its workgroups it is.
template <class Item, int N>
__device__ __forceinline__ int find(const List<Item, N>& t, int id, int* local) {
  int at = -1;
#pragma unroll
  for (int i = 0; i < N; i += 64) {
    const int k = i + (threadIdx.x & 63);
    at += __popcll(__ballot(k < t.count && t.first[k < N ? k : 0] <= id));
  }
  at = __builtin_amdgcn_readfirstlane(at);
  *local = id - t.first[at];
  return at;
}

}  // namespace pp
