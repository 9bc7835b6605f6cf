// embed.hip -- pp_embed_fwd / pp_embed_bwd: rows of a table by id, and the
// table's gradient.
//
//   y[t] = scale w[ids[t]],   dw[j] = add[j] + scale sum over t, ids[t] = j, of dy[t]
//
// The gradient goes by tokens sorted by id (sort_kernel), so that each row of the
// table is summed in an order that the ids alone fix, without atomics: a row of up
// to `piece` tokens by one group of lanes, and a longer one by a workgroup for
// each `piece` places of the sorted list, whose sums a last kernel adds up.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "api_internal.hpp"
#include "lists.hpp"
#include "train.hpp"

namespace pp {
namespace {

using bf16 = __bf16;

// A row is read by 2^lanes lanes of a workgroup of 256, eight features each, and
// by as many columns of the grid as that needs.
struct Lanes {
  int32_t log, columns;
};
Lanes lanes_for(int64_t d) {
  int log = 0;
  while (log < 8 && (int64_t(8) << log) < d) ++log;
  return {log, static_cast<int32_t>(cdiv(d, int64_t(8) << log))};
}

struct Look {
  const int64_t* ids;
  const void* w;
  void* y;
  int64_t t, v, w_ld, y_ld, ignore;
  int32_t d, lanes;
  float scale;
};

constexpr int kLookRows = 4;    // rows of a group of lanes, read together
template <class W, class Y>
__global__ __launch_bounds__(256) void look_kernel(const Look a) {
  const int groups = 256 >> a.lanes, g = threadIdx.x >> a.lanes;
  const int c = ((blockIdx.y << a.lanes) + (threadIdx.x & ((1 << a.lanes) - 1))) * 8;
  const int cols = a.d - c;
  if (cols <= 0) return;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * groups * kLookRows + g;
  float x[kLookRows][8];
  int64_t id[kLookRows];
#pragma unroll
  for (int u = 0; u < kLookRows; ++u) {
    const int64_t t = first + u * groups;
    id[u] = t < a.t ? a.ids[t] : a.ignore;
  }
#pragma unroll
  for (int u = 0; u < kLookRows; ++u) {
    const bool in = static_cast<uint64_t>(id[u]) < static_cast<uint64_t>(a.v);
    if (in && id[u] != a.ignore) {
      load8(static_cast<const W*>(a.w) + id[u] * a.w_ld + c, cols, x[u]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[u][e] = id[u] == a.ignore ? 0.f : __builtin_nanf("");
    }
  }
#pragma unroll
  for (int u = 0; u < kLookRows; ++u) {
    const int64_t t = first + u * groups;
    if (t < a.t) {
      if (id[u] != a.ignore) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] *= a.scale;
      }
      store8(static_cast<Y*>(a.y) + t * a.y_ld + c, cols, x[u]);
    }
  }
}

// ---------------------------------------------------------------------------
// tokens in the order of their ids
// ---------------------------------------------------------------------------

constexpr int kSortWaves = 16, kSortRows = 1024, kOwn = 256;

struct Sort {
  const int64_t* ids;
  int32_t* start;               // [v + 1]: where each row's tokens begin
  int32_t* order;               // tokens, by row and then by token
  int64_t v, ignore;
  int32_t t, per;               // rows of the table a workgroup has: kSortRows at most
};

// A workgroup has `per` rows of the table and reads all ids: it counts those of
// rows before its own, which is where its part of the list begins, and puts its
// own tokens there, all in one launch and without a word from another workgroup.
// A wave has consecutive tokens; counts by row and wave, summed up, give each wave
// the places of its tokens of each row, which it then fills in order.
__global__ __launch_bounds__(kSortWaves * 64) void sort_kernel(const Sort a) {
  __shared__ uint32_t count[kSortWaves][kSortRows];
  __shared__ uint2 own[kSortWaves][kOwn];       // token, row: a wave's first ones
  __shared__ uint32_t sums[kSortWaves], belows[kSortWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t lo = static_cast<int64_t>(blockIdx.x) * a.per;
  const int per = static_cast<int>(a.v - lo < a.per ? a.v - lo : a.per);
  const uint64_t before = (uint64_t(1) << lane) - 1;
  const int64_t each = (a.t + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
  const int t0 = static_cast<int>(min(each * wave, static_cast<int64_t>(a.t)));
  const int t1 = static_cast<int>(min(each * (wave + 1), static_cast<int64_t>(a.t)));

  for (int i = threadIdx.x; i < kSortWaves * kSortRows; i += kSortWaves * 64) count[0][i] = 0;
  __syncthreads();

  // the row of an id among the workgroup's, or -1; *below: it is of a row before them
  auto row_of = [&](int64_t id, bool* below) {
    const bool live = static_cast<uint64_t>(id) < static_cast<uint64_t>(a.v) && id != a.ignore;
    *below = live && id < lo;
    return live && id >= lo && id < lo + per ? static_cast<int>(id - lo) : -1;
  };

  constexpr int kAtOnce = 4;
  uint32_t below = 0, mine = 0;
  for (int t = t0; t < t1; t += 64 * kAtOnce) {
    int64_t id[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) id[u] = t + 64 * u + lane < t1 ? a.ids[t + 64 * u + lane] : a.ignore;
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      bool under;
      const int r = row_of(id[u], &under);
      below += under;
      const uint64_t here = __ballot(r >= 0);
      if (here) {
        const uint32_t at = mine + __popcll(here & before);
        if (r >= 0) {
          atomicAdd(&count[wave][r], 1u);
          if (at < kOwn) own[wave][at] = {static_cast<uint32_t>(t + 64 * u + lane), static_cast<uint32_t>(r)};
        }
        mine += __popcll(here);
      }
    }
  }
  for (int d = 32; d; d >>= 1) below += __shfl_xor(below, d);
  if (lane == 0) belows[wave] = below;
  __syncthreads();

  // where each row's tokens begin, and in them each wave's: a thread a row
  const int row = threadIdx.x;
  uint32_t n = 0;
  if (row < per) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) n += count[w][row];
  }
  uint32_t at = n;              // inclusive sum over the wave
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t x = __shfl_up(at, d);
    if (lane >= d) at += x;
  }
  if (lane == 63) sums[wave] = at;
  __syncthreads();
  uint32_t all = 0;
  at -= n;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    at += belows[w] + (w < wave ? sums[w] : 0u);
    all += belows[w] + sums[w];
  }
  if (row < per) {
    a.start[lo + row] = static_cast<int32_t>(at);
    uint32_t place = at;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t x = count[w][row];
      count[w][row] = place;
      place += x;
    }
  }
  if (row == 0 && lo + per == a.v) a.start[a.v] = static_cast<int32_t>(all);
  __syncthreads();

  // a wave's tokens to their places, 64 at a time: a token's place among those of
  // its row is how many of the lanes before it have the same row
  const int bits = 32 - __clz(per - 1);
  volatile uint32_t* next = count[wave];
  auto place = [&](int r, uint32_t token) {
    uint64_t same = __ballot(r >= 0);
    for (int b = 0; b < bits; ++b) {
      const uint64_t set = __ballot(r >> b & 1);
      same &= r >> b & 1 ? set : ~set;
    }
    if (r >= 0) {
      const uint32_t base = next[r];
      a.order[base + __popcll(same & before)] = static_cast<int32_t>(token);
      if ((same & before) == 0) next[r] = base + __popcll(same);
    }
    __builtin_amdgcn_wave_barrier();
  };
  if (mine <= kOwn) {
    for (uint32_t i = 0; i < mine; i += 64) {
      const bool on = i + lane < mine;
      const uint2 x = own[wave][on ? i + lane : 0];
      place(on ? static_cast<int>(x.y) : -1, x.x);
    }
  } else {
    for (int t = t0; t < t1; t += 64) {
      bool under;
      const int r = row_of(t + lane < t1 ? a.ids[t + lane] : a.ignore, &under);
      if (__ballot(r >= 0)) place(r, static_cast<uint32_t>(t + lane));
    }
  }
}

// ---------------------------------------------------------------------------
// the sums
// ---------------------------------------------------------------------------

struct Sum {
  const int64_t* ids;
  const int32_t* start;
  const int32_t* order;
  const void* dy;
  const void* add;
  void* dw;
  float* part;                  // [pieces][2][part_ld]
  int64_t y_ld, w_ld;
  int32_t v, d, lanes, rows;    // rows: of a group of lanes
  int32_t piece, pieces, part_ld;
  float scale;
};

// Adds dy's rows order[i], i = i0, i0 + by, .. < i1.
template <class Y>
__device__ __forceinline__ void add_rows(const Sum& a, int i0, int i1, int by, int c, float (&acc)[8]) {
  constexpr int kAtOnce = 4;
  const int cols = a.d - c;
  const Y* dy = static_cast<const Y*>(a.dy) + c;
  for (int i = i0; i < i1; i += kAtOnce * by) {
    float x[kAtOnce][8];
    int32_t t[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) t[u] = a.order[min(i + u * by, i1 - 1)];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) load8(dy + t[u] * a.y_ld, cols, x[u]);
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
      if (i + u * by < i1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += x[u][e];
      }
  }
}

template <class W>
__device__ __forceinline__ void put_row(const Sum& a, int64_t row, int c, const float (&acc)[8]) {
  float x[8] = {};
  const int64_t at = row * a.w_ld + c;
  if (a.add) load8(static_cast<const W*>(a.add) + at, a.d - c, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] += a.scale * acc[e];
  store8(static_cast<W*>(a.dw) + at, a.d - c, x);
}

// The first `pieces` workgroups: each its places of the list, for rows of more than
// `piece` tokens (of which it can hold the end of one, or all, and the beginning of
// another).  The others: `rows` rows of the table for each group of lanes, but for
// those.
template <class Y, class W>
__global__ __launch_bounds__(256) void sum_kernel(const Sum a) {
  __shared__ float shared[256 * 8];
  const int groups = 256 >> a.lanes, g = threadIdx.x >> a.lanes, lane = threadIdx.x & ((1 << a.lanes) - 1);
  const int c = ((blockIdx.y << a.lanes) + lane) * 8;
  if (static_cast<int>(blockIdx.x) >= a.pieces) {
    if (c >= a.d) return;
    const int64_t first = (static_cast<int64_t>(blockIdx.x - a.pieces) * groups + g) * a.rows;
    const int64_t last = min(first + a.rows, static_cast<int64_t>(a.v));
    if (first >= last) return;
    int i0 = a.start[first];
    for (int64_t row = first; row < last; ++row) {
      const int i1 = a.start[row + 1], n = i1 - i0;
      if (n <= a.piece && (n > 0 || a.add != a.dw)) {
        float acc[8] = {};
        add_rows<Y>(a, i0, i1, 1, c, acc);
        put_row<W>(a, row, c, acc);
      }
      i0 = i1;
    }
    return;
  }
  const int total = a.start[a.v], i0 = static_cast<int>(blockIdx.x) * a.piece, i1 = min(i0 + a.piece, total);
  if (i0 >= i1) return;
#pragma unroll
  for (int slot = 0; slot < 2; ++slot) {
    const int64_t row = a.ids[a.order[slot ? i1 - 1 : i0]];
    const int b = a.start[row], e = a.start[row + 1];
    if (e - b <= a.piece || (slot && b <= i0)) continue;      // (all of these are the workgroup's)
    float acc[8] = {};
    if (c < a.d) add_rows<Y>(a, max(b, i0) + g, min(e, i1), groups, c, acc);
#pragma unroll
    for (int k = 0; k < 8; ++k) shared[threadIdx.x * 8 + k] = acc[k];
    __syncthreads();
    if (g == 0 && c < a.d) {
      for (int q = 1; q < groups; ++q)
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] += shared[((q << a.lanes) + lane) * 8 + k];
      store8(a.part + (static_cast<int64_t>(blockIdx.x) * 2 + slot) * a.part_ld + c, 8, acc);
    }
    __syncthreads();
  }
}

// Rows of more than `piece` tokens from their pieces' sums: a workgroup for each
// piece that such a row begins in, and 256 features.
constexpr int kJoinGroups = 16;
template <class W>
__global__ __launch_bounds__(kJoinGroups * 64) void join_kernel(const Sum a) {
  using F4 = __attribute__((ext_vector_type(4))) float;
  __shared__ F4 shared[kJoinGroups][64];
  const int total = a.start[a.v], i0 = static_cast<int>(blockIdx.x) * a.piece, i1 = min(i0 + a.piece, total);
  if (i0 >= i1) return;
  const int64_t row = a.ids[a.order[i1 - 1]];
  const int b = a.start[row], e = a.start[row + 1];
  if (e - b <= a.piece || b < i0) return;
  const int g = threadIdx.x >> 6, lane = threadIdx.x & 63, c = (static_cast<int>(blockIdx.y) * 64 + lane) * 4;
  const int p0 = blockIdx.x, p1 = (e - 1) / a.piece + 1;
  F4 acc = {0.f, 0.f, 0.f, 0.f};
  if (c < a.d)
    for (int p = p0 + g; p < p1; p += kJoinGroups)
      acc += *reinterpret_cast<const F4*>(a.part + (static_cast<int64_t>(p) * 2 + (p == p0 && b > i0)) * a.part_ld + c);
  shared[g][lane] = acc;
  __syncthreads();
  if (g > 0 || c >= a.d) return;
  for (int q = 1; q < kJoinGroups; ++q) acc += shared[q][lane];
  const int64_t at = row * a.w_ld + c;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (c + k < a.d) {
      const float x = a.add ? static_cast<float>(static_cast<const W*>(a.add)[at + k]) : 0.f;
      static_cast<W*>(a.dw)[at + k] = static_cast<W>(x + a.scale * acc[k]);
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

bool off(const void* p, size_t by) { return reinterpret_cast<uintptr_t>(p) % by != 0; }
size_t size_of(int32_t dtype) { return dtype == PP_BF16 ? 2 : 4; }

pp_status check(const pp_embed_desc* desc) {
  if (!desc) return fail(PP_EINVAL, "desc is NULL");
  const pp_embed_desc& d = *desc;
  for (int32_t t : {d.w_dtype, d.y_dtype})
    if (t != PP_F32 && t != PP_BF16) return fail(PP_EINVAL, "bad dtype");
  if (d.t < 0 || d.v < 1 || d.d < 1) return fail(PP_EINVAL, "bad size");
  if ((d.v > 1 && d.w_ld < d.d) || (d.t > 1 && d.y_ld < d.d)) return fail(PP_EINVAL, "rows closer than their length");
  if (d.t >= int64_t(1) << 30 || d.v >= int64_t(1) << 30) return fail(PP_EUNSUPPORTED, "tokens and rows must be fewer than 2^30");
  if (d.d >= 1 << 24) return fail(PP_EUNSUPPORTED, "rows must have fewer than 2^24 features");
  for (int64_t n : {d.w_ld, d.y_ld})
    if (n >= int64_t(1) << 32) return fail(PP_EUNSUPPORTED, "rows must be fewer than 2^32 elements apart");
  return PP_OK;
}

// Tokens of a piece: at least 32, and at most 1024 pieces.
struct Plan {
  int32_t piece = 0, pieces = 0, part_ld = 0;
  size_t order = 0, part = 0, total = 0;
};
Plan plan_of(const pp_embed_desc& d) {
  Plan p;
  p.piece = 32;
  while (static_cast<int64_t>(p.piece) * 1024 < d.t) p.piece *= 2;
  p.pieces = d.t > p.piece ? static_cast<int32_t>(cdiv(d.t, p.piece)) : 0;   // (no row can have more)
  p.part_ld = static_cast<int32_t>(cdiv(d.d, 8) * 8);
  auto take = [&](int64_t n) {
    const size_t at = p.total;
    p.total += static_cast<size_t>(cdiv(n, 256) * 256);
    return at;
  };
  take(4 * (d.v + 1));
  p.order = take(4 * d.t);
  p.part = take(static_cast<int64_t>(p.pieces) * 2 * p.part_ld * 4);
  return p;
}

template <class F>
void with_types(int32_t a, int32_t b, F&& f) {
  if (a == PP_BF16) b == PP_BF16 ? f(bf16(), bf16()) : f(bf16(), float());
  else b == PP_BF16 ? f(float(), bf16()) : f(float(), float());
}

pp_status look(const pp_embed_desc* desc, const int64_t* ids, const void* w, void* y, hipStream_t st) {
  const pp_status r = check(desc);
  if (r != PP_OK) return r;
  const pp_embed_desc& d = *desc;
  if (d.t == 0) return PP_OK;
  if (!ids || !w || !y) return fail(PP_EINVAL, "NULL pointer");
  if (off(ids, 8) || off(w, size_of(d.w_dtype)) || off(y, size_of(d.y_dtype))) return fail(PP_EINVAL, "misaligned pointer");
  const Lanes l = lanes_for(d.d);
  const Look a = {ids, w, y, d.t, d.v, d.w_ld, d.y_ld, d.ignore_index, static_cast<int32_t>(d.d), l.log, d.scale};
  const dim3 grid(static_cast<uint32_t>(cdiv(d.t, (256 >> l.log) * kLookRows)), static_cast<uint32_t>(l.columns));
  with_types(d.w_dtype, d.y_dtype, [&](auto wt, auto yt) {
    hipLaunchKernelGGL((look_kernel<decltype(wt), decltype(yt)>), grid, dim3(256), 0, st, a);
  });
  return launched();
}

pp_status grad(const pp_embed_desc* desc, const int64_t* ids, const void* dy, const void* add, void* dw, void* ws, size_t bytes,
               hipStream_t st) {
  const pp_status r = check(desc);
  if (r != PP_OK) return r;
  const pp_embed_desc& d = *desc;
  if (!dw || (d.t && (!ids || !dy))) return fail(PP_EINVAL, "NULL pointer");
  if (off(ids, 8) || off(dy, size_of(d.y_dtype)) || off(dw, size_of(d.w_dtype)) || off(add, size_of(d.w_dtype)))
    return fail(PP_EINVAL, "misaligned pointer");
  if (!ws || off(ws, 256)) return fail(PP_EINVAL, "the workspace must be 256-byte aligned");
  const Plan p = plan_of(d);
  if (bytes < p.total) return fail(PP_ESIZE, "workspace smaller than needed");
  uint8_t* base = static_cast<uint8_t*>(ws);
  int32_t* start = reinterpret_cast<int32_t*>(base);
  int32_t* order = reinterpret_cast<int32_t*>(base + p.order);

  // as many workgroups as CUs, or more where a workgroup's rows would be too many
  const int64_t per = std::min<int64_t>(kSortRows, cdiv(d.v, kCUs));
  const Sort s = {ids, start, order, d.v, d.ignore_index, static_cast<int32_t>(d.t), static_cast<int32_t>(per)};
  hipLaunchKernelGGL(sort_kernel, dim3(static_cast<uint32_t>(cdiv(d.v, per))), dim3(kSortWaves * 64), 0, st, s);

  const Lanes l = lanes_for(d.d);
  const int64_t groups = 256 >> l.log;
  const int64_t rows = std::min<int64_t>(8, std::max<int64_t>(1, d.v / (groups * 4096)));
  const Sum a = {ids,    start,  order, dy,      add,      dw,        reinterpret_cast<float*>(base + p.part), d.y_ld, d.w_ld, static_cast<int32_t>(d.v),
                 static_cast<int32_t>(d.d), l.log, static_cast<int32_t>(rows), p.piece, p.pieces, p.part_ld, d.scale};
  const dim3 grid(static_cast<uint32_t>(p.pieces + cdiv(d.v, groups * rows)), static_cast<uint32_t>(l.columns));
  const dim3 joins(static_cast<uint32_t>(p.pieces), static_cast<uint32_t>(cdiv(d.d, 256)));
  with_types(d.y_dtype, d.w_dtype, [&](auto yt, auto wt) {
    hipLaunchKernelGGL((sum_kernel<decltype(yt), decltype(wt)>), grid, dim3(256), 0, st, a);
    if (p.pieces) hipLaunchKernelGGL((join_kernel<decltype(wt)>), joins, dim3(kJoinGroups * 64), 0, st, a);
  });
  return launched();
}

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" pp_status pp_embed_fwd(const pp_embed_desc* desc, const int64_t* ids, const void* w, void* y, void* hip_stream) {
  return guarded([&] { return look(desc, ids, w, y, static_cast<hipStream_t>(hip_stream)); });
}

extern "C" pp_status pp_embed_workspace(const pp_embed_desc* desc, size_t* bytes) {
  return guarded([&]() -> pp_status {
    const pp_status s = check(desc);
    if (s != PP_OK) return s;
    if (!bytes) return fail(PP_EINVAL, "bytes is NULL");
    *bytes = plan_of(*desc).total;
    return PP_OK;
  });
}

extern "C" pp_status pp_embed_bwd(const pp_embed_desc* desc, const int64_t* ids, const void* dy, const void* add, void* dw,
                                  void* workspace, size_t ws_bytes, void* hip_stream) {
  return guarded([&] { return grad(desc, ids, dy, add, dw, workspace, ws_bytes, static_cast<hipStream_t>(hip_stream)); });
}
