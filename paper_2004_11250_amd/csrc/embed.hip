// embed.hip -- pp_embed_fwd / pp_embed_bwd: rows of a table by id, and the
// table's gradient.
//
//   y[t] = scale w[ids[t]],   dw[j] = add[j] + scale sum over t, ids[t] = j, of dy[t]
//
// The gradient goes by tokens sorted by id (sort_kernel, or count_kernel and
// place_kernel; few_kernel does all of a small call), so that each row of the table
// is summed in an order that the ids alone fix, without atomics, and all workgroups
// have equally many tokens, however many share a row: sum_kernel goes by pieces of
// the sorted list, and join_kernel adds up the sums of rows that lie in more than
// one.
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

// A row is read by 2^log lanes of a workgroup of 256, eight features each, and
// by as many columns of the grid as that needs.
struct Lanes {
  int32_t log, columns;
};
Lanes lanes_for(int64_t d) {
  int log = 0;
  while (log < 8 && (int64_t(8) << log) < d) ++log;
  return {log, static_cast<int32_t>(cdiv(d, int64_t(8) << log))};
}

// The first of a lane's features, and how far the second four are from it (SPLIT).
template <bool SPLIT>
__device__ __forceinline__ int first_of(int log) {
  const int lane = threadIdx.x & ((1 << log) - 1);
  return (static_cast<int>(blockIdx.y) << log) * 8 + lane * (SPLIT ? 4 : 8);
}
__device__ __forceinline__ int far_of(int log) { return 4 << log; }

struct Look {
  const int64_t* ids;
  const void* w;
  void* y;
  int64_t t, v, w_ld, y_ld, ignore;
  int32_t d, lanes;
  float scale;
};

// A group of lanes a token.  Bound by memory: 8192 tokens of 1024 bf16 features from a
// table of 50000 6.4 us (5.2 TB/s), 65536 39.6 (two, four and eight tokens of a group,
// read together: 6.6, 7.0 and 7.9, the last ones' waves leave the card too early);
// one token 1.8, the launch.  16384 tokens of 4096 fp32 features 86 us, 6.3 TB/s (a lane's
// eight in a row instead of two fours: 96; their gradient into 20000 rows 122 and 163).
template <class W, class Y>
__global__ __launch_bounds__(256) void look_kernel(const Look a) {
  constexpr bool SPLIT = kSplit<W, Y>;
  const int c = first_of<SPLIT>(a.lanes), cols = a.d - c, far = far_of(a.lanes);
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (256 >> a.lanes) + (threadIdx.x >> a.lanes);
  if (cols <= 0 || t >= a.t) return;
  const int64_t id = a.ids[t];
  float y[8];
  if (id != a.ignore && static_cast<uint64_t>(id) < static_cast<uint64_t>(a.v)) {
    load8<SPLIT>(static_cast<const W*>(a.w) + id * a.w_ld + c, cols, far, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= a.scale;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = id == a.ignore ? 0.f : __builtin_nanf("");
  }
  store8<SPLIT>(static_cast<Y*>(a.y) + t * a.y_ld + c, cols, far, y);
}

// ---------------------------------------------------------------------------
// tokens in the order of their ids
// ---------------------------------------------------------------------------

constexpr int kSortWaves = 16, kOwnBits = 10, kSortRows = 1 << kOwnBits, kSortWords = 2400;

struct Place {
  int32_t token, row;
};

// Rows are dealt to 2^log workgroups, 2^run consecutive ones at a time, so that
// rows that occur often, which tend to lie together, come to different ones.
struct Deal {
  int32_t log, run, per;        // per: rows of a workgroup, kSortRows at most
  __device__ __forceinline__ uint32_t group(uint32_t row) const { return row >> run & ((1u << log) - 1); }
  __device__ __forceinline__ uint32_t local(uint32_t row) const { return (row >> (run + log)) << run | (row & ((1u << run) - 1)); }
  __device__ __forceinline__ uint32_t row(uint32_t group, uint32_t local) const {
    return (local >> run) << (run + log) | group << run | (local & ((1u << run) - 1));
  }
  // where a row's entry of `start` is
  __device__ __forceinline__ int64_t at(uint32_t row) const { return static_cast<int64_t>(group(row)) * per + local(row); }
  __host__ __device__ int64_t entries() const { return (static_cast<int64_t>(per) << log) + 1; }
};

struct Sort {
  const int64_t* ids;
  int32_t* start;               // [deal.entries()]: where each row's tokens begin
  Place* order;                 // tokens, by row (in the order of `start`)
  uint32_t v, ignore;           // (ignore: v where it is no row)
  int32_t t;
  Deal deal;
};

// A workgroup has its rows of the table and reads all ids: it counts those of the
// workgroups before it, which is where its part of the list begins, and puts its
// own tokens there, all in one launch and without a word from another workgroup.
// A wave has consecutive tokens; counts by row and wave, summed up, give each wave
// the places of its tokens of each row, which it then fills in order.
// Bound by the instructions of the scan, some ten an id and workgroup, and by its fixed
// part: 777 tokens 5.5 us, 8192 7.3, 32768 10.4 with uniform ids; and by the workgroup of
// the most frequent row (32768 log-uniform ids 14).  (Rows dealt in consecutive ranges
// instead: 131072 log-uniform ids 130 us, now 57.)
__global__ __launch_bounds__(kSortWaves * 64) void sort_kernel(const Sort a) {
  // for each wave a count of each row's tokens, then a list of tokens:
  // (token - base) << kOwnBits | row
  __shared__ uint32_t words[kSortWaves * kSortWords];
  __shared__ uint32_t sums[kSortWaves], belows[kSortWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t me = blockIdx.x;
  const Deal deal = a.deal;
  const int per = deal.per;
  const uint64_t before = (uint64_t(1) << lane) - 1;
  const int64_t each = (a.t + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
  const int t0 = static_cast<int>(min(each * wave, static_cast<int64_t>(a.t)));
  const int t1 = static_cast<int>(min(each * (wave + 1), static_cast<int64_t>(a.t)));
  uint32_t* count = words;
  uint32_t* own = words + kSortWaves * per + wave * (kSortWords - per);
  const uint32_t most = kSortWords - per;
  for (int i = lane; i < per; i += 64) count[wave * per + i] = 0;   // (a wave's own until all have counted)

  // All of a wave's tokens: those of the workgroup's rows go on a list in LDS, of `mine`
  // entries that count tokens from `base` on, and `use` takes it when it is full (the
  // last list is left to the caller).
  constexpr int kAtOnce = 8, kStep = 64 * kAtOnce;
  uint32_t below = 0, mine = 0;
  int base = t0;
  bool whole = true;
  auto scan = [&](auto&& use, auto first) {
    mine = 0, base = t0;
    for (int t = t0; t < t1; t += kStep) {
      const uint2* p = reinterpret_cast<const uint2*>(a.ids) + t;   // (an id's upper half: y)
      uint2 id[kAtOnce];
      if (t + kStep <= t1) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) id[u] = p[64 * u + lane];
      } else {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) id[u] = t + 64 * u + lane < t1 ? p[64 * u + lane] : uint2{0u, 1u};
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const uint32_t i = id[u].x;
        const bool live = id[u].y == 0 && i < a.v && i != a.ignore;
        const uint32_t g = live ? deal.group(i) : ~0u;
        if constexpr (decltype(first)::value) below += __popcll(__ballot(g < me));
        const uint64_t here = __ballot(g == me);
        if (here) {
          if (g == me) own[mine + __popcll(here & before)] = static_cast<uint32_t>(t + 64 * u + lane - base) << kOwnBits | deal.local(i);
          mine += __popcll(here);
        }
      }
      if (mine > most - kStep || t + 2 * kStep - base > 1 << (32 - kOwnBits)) {
        use();
        mine = 0, base = t + kStep, whole = false;
      }
    }
  };
  // f(row, the token's bits of its entry, lanes of the same row) for 64 entries at a
  // time (a step's lanes add to each row once: additions to one address take turns)
  const int bits = 32 - __clz(per - 1);
  auto each_entry = [&](auto&& f) {
    __builtin_amdgcn_wave_barrier();   // (the list is the wave's own; LDS is done in order)
    for (uint32_t i = 0; i < mine; i += 64) {
      const bool on = i + lane < mine;
      const uint32_t x = own[on ? i + lane : 0], r = x & (kSortRows - 1);
      uint64_t same = __ballot(on);
      for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot(r >> b & 1);
        same &= r >> b & 1 ? set : ~set;
      }
      if (on) f(r, x >> kOwnBits, same);
      __builtin_amdgcn_wave_barrier();
    }
  };
  auto tally = [&] {
    each_entry([&](uint32_t r, uint32_t, uint64_t same) {
      if ((same & before) == 0) atomicAdd(&count[wave * per + r], static_cast<uint32_t>(__popcll(same)));
    });
  };
  scan(tally, std::true_type());
  tally();
  if (lane == 0) belows[wave] = below;
  __syncthreads();

  // where each row's tokens begin, and in them each wave's: a thread a row
  const int row = threadIdx.x;
  uint32_t n = 0;
  if (row < per) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) n += count[w * per + row];
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
    a.start[static_cast<int64_t>(me) * per + row] = static_cast<int32_t>(at);
    uint32_t place = at;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t x = count[w * per + row];
      count[w * per + row] = place;
      place += x;
    }
  }
  if (row == 0 && me + 1 == gridDim.x) a.start[deal.entries() - 1] = static_cast<int32_t>(all);
  __syncthreads();

  // a wave's tokens to their places, 64 at a time: a token's place among those of
  // its row is how many of the lanes before it have the same row
  volatile uint32_t* next = count + wave * per;
  auto place = [&] {
    each_entry([&](uint32_t r, uint32_t token, uint64_t same) {
      const uint32_t at = next[r];
      a.order[at + __popcll(same & before)] = {base + static_cast<int>(token), static_cast<int32_t>(deal.row(me, r))};
      if ((same & before) == 0) next[r] = at + __popcll(same);
    });
  };
  if (!whole) scan(place, std::false_type());
  place();
}

// The same by digits of the row's number, up to kOwnBits bits each, the lowest first,
// without a workgroup that has all tokens of a row.  A workgroup has `each` places of
// the list so far.  count_kernel counts its tokens of each digit; place_kernel adds up
// the counts, which gives each workgroup the places of its tokens of each digit, and
// puts them there, in their order.  32768 pixels 2.9 and 6.7 us: latency, of ids,
// counts, a scan and an exchange in turn.
constexpr int64_t kCounts = 128;                // workgroups at most
struct Digit {
  const int64_t* ids;           // the first digit's list
  const Place* in;              // the others', and its length
  const int32_t* in_total;
  int32_t* clear;               // [cleared] values that the first digit's count_kernel sets to 0
  int64_t cleared;
  int32_t groups;               // workgroups that count (others only clear)
  uint32_t* count;              // [workgroups][values]
  int32_t* start;               // [values + 1]: where each value's tokens begin
  Place* order;
  uint32_t v, ignore;
  int32_t t, each;              // each: a multiple of 1024
  int32_t shift, values;        // the digit: row >> shift & (2^bits - 1), below `values`
  int32_t bits;
};

// The places of a wave of the workgroup, a lane each: f(token, row, digit or -1).  The
// first ones are fetched at once, and kept.
template <bool FIRST>
struct WaveTokens {
  const uint2* p;
  int64_t t, left;
  int32_t part;
  uint2 first;
  __device__ __forceinline__ explicit WaveTokens(const Digit& a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    part = a.each / kSortWaves;
    t = static_cast<int64_t>(blockIdx.x) * a.each + wave * part + lane;
    p = (FIRST ? reinterpret_cast<const uint2*>(a.ids) : reinterpret_cast<const uint2*>(a.in)) + t;
    left = (FIRST ? a.t : *a.in_total) - t;
    first = fetch(0);
  }
  __device__ __forceinline__ uint2 fetch(int i) const { return i < left ? p[i] : uint2{0u, 1u}; }
  template <class F>
  __device__ __forceinline__ void each(const Digit& a, F&& f) const {
    for (int i = 0; i < part; i += 64) {
      const uint2 x = i ? fetch(i) : first;
      const uint32_t row = FIRST ? x.x : x.y;
      const bool live = FIRST ? x.y == 0 && row < a.v && row != a.ignore : i < left;
      f(FIRST ? static_cast<int>(t + i) : static_cast<int>(x.x), static_cast<int>(row),
        live ? static_cast<int>(row >> a.shift & ((1u << a.bits) - 1)) : -1);
    }
  }
};

template <bool FIRST>
__global__ __launch_bounds__(kSortWaves * 64) void count_kernel(const Digit a) {
  __shared__ uint32_t count[kSortRows];
  if constexpr (FIRST)
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kSortWaves * 64 + threadIdx.x; i < a.cleared; i += static_cast<int64_t>(gridDim.x) * kSortWaves * 64)
      a.clear[i] = 0;
  if (static_cast<int>(blockIdx.x) >= a.groups) return;
  const WaveTokens<FIRST> tokens(a);
  count[threadIdx.x] = 0;
  __syncthreads();
  tokens.each(a, [&](int, int, int k) {
    if (k >= 0) atomicAdd(&count[k], 1u);
  });
  __syncthreads();
  if (static_cast<int>(threadIdx.x) < a.values) a.count[static_cast<int64_t>(blockIdx.x) * a.values + threadIdx.x] = count[threadIdx.x];
}

template <bool FIRST>
__global__ __launch_bounds__(kSortWaves * 64) void place_kernel(const Digit a) {
  __shared__ uint32_t count[kSortWaves][kSortRows];
  __shared__ uint32_t sums[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint64_t before = (uint64_t(1) << lane) - 1;
  const WaveTokens<FIRST> tokens(a);
  // a thread a value: its tokens in all, and in the workgroups before this one
  constexpr int kAtOnce = 32;
  uint32_t n = 0, earlier = 0;
  if (tid < a.values) {
    const int groups = gridDim.x;
    for (int g = 0; g < groups; g += kAtOnce) {
      uint32_t x[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) x[u] = a.count[static_cast<int64_t>(min(g + u, groups - 1)) * a.values + tid];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        n += g + u < groups ? x[u] : 0u;
        earlier += g + u < static_cast<int>(blockIdx.x) ? x[u] : 0u;
      }
    }
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) count[w][tid] = 0;
  }
  uint32_t at = n;              // inclusive sum over the wave
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t x = __shfl_up(at, d);
    if (lane >= d) at += x;
  }
  if (lane == 63) sums[wave] = at;
  __syncthreads();

  // lanes with the same digit
  auto same_digit = [&](int k) {
    uint64_t same = __ballot(k >= 0);
    for (int b = 0; b < a.bits; ++b) {
      const uint64_t set = __ballot(k >> b & 1);
      same &= k >> b & 1 ? set : ~set;
    }
    return same;
  };
  tokens.each(a, [&](int, int, int k) {
    const uint64_t same = same_digit(k);
    if (k >= 0 && (same & before) == 0) atomicAdd(&count[wave][k], static_cast<uint32_t>(__popcll(same)));
  });
  __syncthreads();
  for (int w = 0; w < wave; ++w) at += sums[w];
  if (tid < a.values) {
    if (blockIdx.x == 0) {
      a.start[tid] = static_cast<int32_t>(at - n);
      if (tid + 1 == a.values) a.start[a.values] = static_cast<int32_t>(at);
    }
    uint32_t place = at - n + earlier;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t x = count[w][tid];
      count[w][tid] = place;
      place += x;
    }
  }
  __syncthreads();
  volatile uint32_t* next = count[wave];
  tokens.each(a, [&](int t, int row, int k) {
    const uint64_t same = same_digit(k);
    if (k >= 0) {
      const uint32_t place = next[k];
      a.order[place + __popcll(same & before)] = {t, row};
      if ((same & before) == 0) next[k] = place + __popcll(same);
    }
    __builtin_amdgcn_wave_barrier();
  });
}

// Where each row's tokens begin and end in a list sorted by several digits; rows without
// tokens have 0 and 0 already.
__global__ __launch_bounds__(256) void bounds_kernel(const Place* order, const int32_t* total, int32_t* begin, int32_t* end) {
  const int n = *total;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= n) return;
  const int32_t row = order[i].row;
  if (i == 0 || order[i - 1].row != row) begin[row] = static_cast<int32_t>(i);
  if (i + 1 == n || order[i + 1].row != row) end[row] = static_cast<int32_t>(i) + 1;
}

// ---------------------------------------------------------------------------
// the sums
// ---------------------------------------------------------------------------

struct Sum {
  const int32_t *begin, *end;   // of a row's tokens, at deal.at(row)
  const int32_t* total;         // of the list
  const Place* order;
  const void* dy;
  const void* add;
  void* dw;
  float* part;                  // [pieces][2][part_ld]
  int64_t y_ld, w_ld;
  int32_t t, v, d, lanes;
  Deal deal;
  int32_t pieces, batches, piece;       // of a group of lanes: batches of kBatch tokens; of a workgroup: tokens
  int32_t part_ld;
  float scale;
};

constexpr int kBatch = 8;

template <bool SPLIT, class W>
__device__ __forceinline__ void put_row(const Sum& a, int64_t row, int c, const float (&acc)[8]) {
  float x[8] = {};
  const int64_t at = row * a.w_ld + c;
  if (a.add) load8<SPLIT>(static_cast<const W*>(a.add) + at, a.d - c, far_of(a.lanes), x);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] += a.scale * acc[e];
  store8<SPLIT>(static_cast<W*>(a.dw) + at, a.d - c, far_of(a.lanes), x);
}

// Rows without a token, of kFillRows a group of lanes: what they are added to, or 0.
// They lie between the tokens' workgroups in one launch, which is bound by memory then:
// 8192 tokens into 50000 x 1024 bf16 21 us, 5.7 TB/s (in a launch before it, together
// with the sort: 22 + 9.5 in place of 7.5 + 21); added to another gradient, 32768 tokens,
// 47 us, 6 TB/s, 67 without the hint that what is copied is not read again.  (Rows of a
// group: 4; 8 and 16 take 49 and 54 us.)
constexpr int kFillRows = 4;
template <class W>
__device__ __forceinline__ void fill_rows(const Sum& a, int block) {
  constexpr bool SPLIT = kSplit<W>;
  const int groups = 256 >> a.lanes, g = threadIdx.x >> a.lanes;
  const int c = first_of<SPLIT>(a.lanes), cols = a.d - c, far = far_of(a.lanes);
  if (cols <= 0) return;
  const int64_t first = static_cast<int64_t>(block) * groups * kFillRows + g;
  int64_t at[kFillRows];
#pragma unroll
  for (int u = 0; u < kFillRows; ++u) {
    const int64_t row = first + u * groups, i = a.deal.at(static_cast<uint32_t>(min(row, static_cast<int64_t>(a.v - 1))));
    at[u] = a.begin[i] == a.end[i] && row < a.v ? row * a.w_ld + c : -1;
  }
  Eight<W> x[kFillRows] = {};
  if (a.add) {
#pragma unroll
    for (int u = 0; u < kFillRows; ++u)
      if (at[u] >= 0) x[u] = get8<SPLIT, true>(static_cast<const W*>(a.add) + at[u], cols, far);
  }
#pragma unroll
  for (int u = 0; u < kFillRows; ++u)
    if (at[u] >= 0) put8<SPLIT, true>(static_cast<W*>(a.dw) + at[u], cols, far, x[u]);
}

// A workgroup sums the piece p0 .. p1 of a list, a group of lanes a part of it, of
// `batches` batches of kBatch tokens; `at`: the group's first batch.  A run of one
// row's tokens that begins and ends inside a group's part is written by the group; a
// part's first and last run meet their neighbours' in the wave, by steps that double,
// and a wave's first and last run (where a group is a wave or more, a group's) meet
// theirs in LDS.  (All groups' in LDS, one after the other: 17102 tokens into 112 x 32
// bf16, three in ten ids the same, 27 us a call, now 18; 8192 into 1000 x 64 20 and 18.
// With rows of few tokens it was 0.8 to 1.8 us less: 8192 uniform ids into 1000 x 64 14.7
// and 15.9, 1200 into 313 x 256 fp32, two groups a wave, 14.3 and 15.8.)  What goes on past the piece's ends (row `prev` before it,
// `next` behind it, -1: none) goes to part: the sum of a run that goes on from the
// piece before to row 0, of one that begins here to row 1.  A batch's rows are in
// flight together, and a piece's time is that of its list, its rows and its neighbours
// in LDS one after the other: 32768 tokens into 313 x 256 bf16 7.9 us (batches of 4
// 7.1, but twice the pieces for join_kernel, of 16 23: too few waves).
template <class Y, class W, int THREADS>
__device__ __forceinline__ void sum_piece(const Sum& a, const Place* order, int p0, int p1, int batches, Place (&at)[kBatch],
                                          int32_t prev, int32_t next, float* part, float (*edge)[8], int32_t* edge_row) {
  constexpr bool SPLIT = kSplit<Y, W>;
  const int groups = THREADS >> a.lanes, g = threadIdx.x >> a.lanes, lane = threadIdx.x & ((1 << a.lanes) - 1);
  const int c = first_of<SPLIT>(a.lanes), cols = a.d - c, far = far_of(a.lanes);
  const Y* dy = static_cast<const Y*>(a.dy) + c;
  const int i0 = p0 + g * batches * kBatch, i1 = min(i0 + batches * kBatch, p1);

  float acc[8] = {};
  int cur = -1, head = -1;      // the row of acc, and of the group's first run where that is another
  // Units whose runs meet in LDS: groups, or waves of several.  A unit's first run has
  // its first slot, its last one, where that is another, its second.
  const int unit = a.lanes < 6 ? static_cast<int>(threadIdx.x) >> 6 : g;
  const int wide = max(a.lanes, 6);
  auto to_edge = [&](int slot, const float (&x)[8]) {     // (slot: of the unit, or 2 k: the wave's group k's)
#pragma unroll
    for (int e = 0; e < 8; ++e) edge[(unit << (wide + 1)) + (slot << a.lanes) + lane][e] = x[e];
  };
  auto from_edge = [&](int at, int slot, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = edge[(at << (wide + 1)) + (slot << a.lanes) + lane][e];
  };
  const int member = a.lanes < 6 ? g & ((64 >> a.lanes) - 1) : 0;
  for (int i = i0; i < i1; i += kBatch) {
    Eight<Y> x[kBatch];
    if (i > i0) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) at[u] = order[min(i + u, i1 - 1)];
    }
    if (cols > 0) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) x[u] = get8<SPLIT, true>(dy + (i + u < i1 ? at[u].token : at[0].token) * a.y_ld, cols, far);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (i + u >= i1) break;
      if (at[u].row != cur) {
        if (cur >= 0) {
          if (head < 0)
            to_edge(2 * member, acc), head = cur;
          else if (cols > 0)
            put_row<SPLIT, W>(a, cur, c, acc);
        }
        cur = at[u].row;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += static_cast<float>(x[u][e]);
    }
  }
  const int32_t last = head >= 0 ? cur : -1;      // the row of the last run, where it is another
  if (head < 0) head = cur;
  if (a.lanes < 6) {
    // in a wave: each group's first run with what follows of it (rows of a sorted list
    // are the same only where all between them are), then the last runs with the next
    // group's first
    const int in_wave = 64 >> a.lanes, step = 1 << a.lanes;
    float x[8];
    __builtin_amdgcn_wave_barrier();
    if (last >= 0) {
      from_edge(unit, 2 * member, x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = acc[e];
    }
    const int32_t end = last >= 0 ? last : head, prior = __shfl_up(end, step), follows = __shfl_down(head, step);
    const uint64_t some = __ballot(head >= 0);
    const int32_t row0 = __builtin_amdgcn_readlane(head, 0), row1 = __builtin_amdgcn_readlane(end, some ? 63 - __clzll(some) : 0);
    int32_t row = follows;
    for (int k = 1; k < in_wave; k *= 2) {
      if (k > 1) row = __shfl_down(head, k * step);
      const bool on = member + k < in_wave && row == head && row >= 0;
      if (!__ballot(on)) break;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = __shfl_down(x[e], k * step);
        x[e] += on ? y : 0.f;
      }
    }
    const bool more = member + 1 < in_wave && follows == last && last >= 0;
    if (__ballot(more)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = __shfl_down(x[e], step);
        acc[e] += more ? y : 0.f;
      }
    }
    __builtin_amdgcn_wave_barrier();
    if (head >= 0 && (member == 0 || prior != head)) {
      if (member == 0 || head == row1)
        to_edge(member == 0 ? 0 : 1, x);
      else if (cols > 0)
        put_row<SPLIT, W>(a, head, c, x);
    }
    if (last >= 0) {
      if (last == row1)
        to_edge(1, acc);
      else if (cols > 0)
        put_row<SPLIT, W>(a, last, c, acc);
    }
    if ((threadIdx.x & 63) == 0) edge_row[2 * unit] = row0, edge_row[2 * unit + 1] = row1 == row0 ? -1 : row1;
  } else {
    if (cur >= 0) to_edge(last >= 0 ? 1 : 0, acc);
    if (lane == 0) edge_row[2 * unit] = head, edge_row[2 * unit + 1] = last;
  }
  __syncthreads();
  if (cols <= 0 || member > 0) return;

  // the runs that begin at this unit's edges; units past the piece's end have none
  const int of_unit = (batches * kBatch) << (wide - a.lanes);
  const int slots = 2 * min(THREADS >> wide, (p1 - p0 + of_unit - 1) / of_unit);
  for (int s = 2 * unit; s < 2 * unit + 2; ++s) {
    const int32_t row = edge_row[s];
    if (row < 0) continue;
    const int32_t left = s == 0 ? -1 : edge_row[s - 1] >= 0 ? edge_row[s - 1] : s > 1 ? edge_row[s - 2] : -1;
    if (left == row) continue;
    from_edge(unit, s & 1, acc);
    bool ends = false;          // another run follows in this piece
    constexpr int kNear = 4;    // (read together, whether they belong to the run or not)
    for (int q = s + 1; q < slots && !ends; q += kNear) {
      int32_t r[kNear];
      float x[kNear][8];
#pragma unroll
      for (int u = 0; u < kNear; ++u) {
        const int k = min(q + u, slots - 1);
        r[u] = edge_row[k];
        from_edge(k >> 1, k & 1, x[u]);
      }
#pragma unroll
      for (int u = 0; u < kNear; ++u) {
        if (q + u >= slots || ends) break;
        if (r[u] == row) {
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] += x[u][e];
        } else if (r[u] >= 0) {
          ends = true;
        }
      }
    }
    const bool from = s == 0 && prev == row, on = !ends && next == row;
    if (from || on)
      store8<SPLIT>(part + static_cast<int64_t>(!from) * a.part_ld + c, a.part_ld - c, far, acc);
    else
      put_row<SPLIT, W>(a, row, c, acc);
  }
}

// The first `pieces` workgroups: a piece of the sorted list each.  The others: rows
// without a token.
template <class Y, class W>
__global__ __launch_bounds__(256) void sum_kernel(const Sum a) {
  __shared__ float edge[2 * 256][8];            // [2 group + (not the first run)][lane]
  __shared__ int32_t edge_row[2 * 256];
  if (static_cast<int>(blockIdx.x) >= a.pieces) {
    fill_rows<W>(a, static_cast<int>(blockIdx.x) - a.pieces);
    return;
  }
  const int total = *a.total;
  const int p0 = static_cast<int>(blockIdx.x) * a.piece, p1 = min(p0 + a.piece, total);
  // (the places do not wait for the total; behind it they hold nothing)
  Place at[kBatch];
#pragma unroll
  for (int u = 0; u < kBatch; ++u) at[u] = a.order[min(p0 + static_cast<int>(threadIdx.x >> a.lanes) * a.batches * kBatch + u, a.t - 1)];
  const int32_t prev = a.order[max(p0 - 1, 0)].row, next = a.order[min(p0 + a.piece, a.t - 1)].row;
  if (p0 >= p1) return;
  sum_piece<Y, W, 256>(a, a.order, p0, p1, a.batches, at, p0 > 0 ? prev : -1, p1 < total ? next : -1,
                       a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.part_ld, edge, edge_row);
}

// Up to kFewTokens tokens: a workgroup has its rows of the table, finds their tokens,
// a thread an id, sorts them in LDS, sums them, and fills its rows without a token,
// all in one launch.  777 tokens into 5003 x 203 fp32 8 us: ids, the order, rows of
// features and edges, one after the other; a table of 50000 x 1024 bf16 is filled in
// 20, 5 TB/s.
constexpr int kFewTokens = 1024, kFewRanks = 256;
template <class Y, class W>
__global__ __launch_bounds__(kFewTokens) void few_kernel(const Sort s, const Sum a) {
  __shared__ float edge[2 * kFewTokens][8];
  __shared__ int32_t edge_row[2 * kFewTokens];
  __shared__ uint32_t keys[kFewTokens];
  __shared__ Place order[kFewTokens];
  __shared__ bool found[kSortRows];
  __shared__ int32_t counts[kFewTokens / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t me = blockIdx.x;
  const uint2 id = tid < s.t ? reinterpret_cast<const uint2*>(s.ids)[tid] : uint2{0u, 1u};
  const bool own = id.y == 0 && id.x < s.v && id.x != s.ignore && s.deal.group(id.x) == me;
  const uint64_t here = __ballot(own);
  if (lane == 0) counts[wave] = __popcll(here);
  found[tid] = false;
  __syncthreads();
  int n = 0, at = __popcll(here & ((uint64_t(1) << lane) - 1));
  for (int w = 0; w < kFewTokens / 64; ++w) {
    at += w < wave ? counts[w] : 0;
    n += counts[w];
  }
  if (own) {
    keys[at] = s.deal.local(id.x) << kOwnBits | static_cast<uint32_t>(tid);   // (by row, then by token)
    found[s.deal.local(id.x)] = true;
  }
  if (tid >= n) keys[tid] = ~0u;
  __syncthreads();
  if (n) {
    const auto put = [&](int rank, uint32_t key) {
      order[rank] = {static_cast<int32_t>(key & (kFewTokens - 1)), static_cast<int32_t>(s.deal.row(me, key >> kOwnBits))};
    };
    if (n <= kFewRanks) {
      // a token's place is how many come before it
      if (tid < n) {
        const uint32_t mine = keys[tid];
        int rank = 0;
        for (int j = 0; j < n; j += 4)
#pragma unroll
          for (int k = 0; k < 4; ++k) rank += keys[j + k] < mine;
        put(rank, mine);
      }
    } else {
      // exchanges in runs that double (n^2 / 256 reads of LDS take longer from here on)
      for (int run = 2; run < 2 * n; run *= 2)
        for (int step = run / 2; step > 0; step /= 2) {
          const int other = tid ^ step;
          if (other > tid && tid < 2 * n) {
            const uint32_t x = keys[tid], y = keys[other];
            if ((x > y) == ((tid & run) == 0)) keys[tid] = y, keys[other] = x;
          }
          __syncthreads();
        }
      if (tid < n) put(tid, keys[tid]);
    }
    __syncthreads();
    const int groups = kFewTokens >> a.lanes, batches = (n + groups * kBatch - 1) / (groups * kBatch);
    Place first[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) first[u] = order[min((tid >> a.lanes) * batches * kBatch + u, n - 1)];
    sum_piece<Y, W, kFewTokens>(a, order, 0, n, batches, first, -1, -1, nullptr, edge, edge_row);
  }

  if (a.add == a.dw) return;
  constexpr int kRows = 4;
  constexpr bool SPLIT = kSplit<W>;
  const int groups = kFewTokens >> a.lanes, c = first_of<SPLIT>(a.lanes), cols = a.d - c, far = far_of(a.lanes);
  if (cols <= 0) return;
  for (int l = tid >> a.lanes; l < s.deal.per; l += kRows * groups) {
    Eight<W> x[kRows] = {};
    int64_t to[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int k = l + u * groups;
      const uint32_t row = s.deal.row(me, k);
      to[u] = k < s.deal.per && row < s.v && !found[k] ? row * a.w_ld + c : -1;
    }
    if (a.add) {
#pragma unroll
      for (int u = 0; u < kRows; ++u)
        if (to[u] >= 0) x[u] = get8<SPLIT, true>(static_cast<const W*>(a.add) + to[u], cols, far);
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u)
      if (to[u] >= 0) put8<SPLIT, true>(static_cast<W*>(a.dw) + to[u], cols, far, x[u]);
  }
}

// Rows whose tokens lie in more than one piece, from the pieces' sums: a workgroup
// for each piece that such a row may begin in, and 256 features.  Most end at once, so
// that its time is the workgroups' (1024 pieces of 1024 features 6.3 us with 4 waves
// each, 8.8 with 8) and the longest row's (313 rows of 256 features, 32768 pixels: 5.3,
// 4.1 with 8).
template <class W, int kJoinGroups>
__global__ __launch_bounds__(kJoinGroups * 64) void join_kernel(const Sum a) {
  using F4 = __attribute__((ext_vector_type(4))) float;
  __shared__ F4 shared[kJoinGroups][64];
  const int p0 = static_cast<int>(blockIdx.x) * a.piece, p1 = p0 + a.piece;
  if (p1 >= a.t) return;
  const int total = *a.total;
  const int64_t row = a.order[p1 - 1].row, next = a.order[p1].row;
  if (p1 >= total || next != row) return;
  const int64_t at_row = a.deal.at(static_cast<uint32_t>(row));
  const int b = a.begin[at_row], e = a.end[at_row];
  if (b < p0) return;
  const int g = threadIdx.x >> 6, lane = threadIdx.x & 63, c = (static_cast<int>(blockIdx.y) * 64 + lane) * 4;
  const int first = blockIdx.x, last = (e - 1) / a.piece;
  F4 acc = {0.f, 0.f, 0.f, 0.f};
  if (c < a.d) {
    constexpr int kAtOnce = 8;
    const float* part = a.part + c;
    for (int p = first + g; p <= last; p += kAtOnce * kJoinGroups) {
      F4 x[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int64_t q = min(p + u * kJoinGroups, last);
        x[u] = *reinterpret_cast<const F4*>(part + (2 * q + (q == first)) * a.part_ld);
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
        if (p + u * kJoinGroups <= last) acc += x[u];
    }
  }
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
  if (d.d >= 1 << 23) return fail(PP_EUNSUPPORTED, "rows must have fewer than 2^23 features");
  for (int64_t n : {d.w_ld, d.y_ld})
    if (n >= int64_t(1) << 32) return fail(PP_EUNSUPPORTED, "rows must be fewer than 2^32 elements apart");
  return PP_OK;
}

constexpr int64_t kPieces = 1024;            // of the sorted list, at most
constexpr int64_t kGrid = int64_t(1) << 24;  // (a launch has fewer than 2^32 threads)
// Whether a table's rows without a token are fewer workgroups than that.
pp_status check_rows(const pp_embed_desc& d) {
  if (cdiv(d.v, (256 >> lanes_for(d.d).log) * kFillRows) + kPieces >= kGrid) return fail(PP_EUNSUPPORTED, "a table of too many rows of this length");
  return PP_OK;
}

// Tokens of a group's part: kBatch, or as many times that as keep the pieces
// to kPieces.
struct Plan {
  Lanes lanes;
  Deal deal;
  bool few;                     // one launch
  int digits = 0;               // sorted by so many digits (0: by sort_kernel)
  int32_t values[3] = {}, bits[3] = {};
  int32_t batches = 1, piece = 0, pieces = 0, part_ld = 0, each = 0, counts = 0;
  size_t order = 0, part = 0, count = 0, starts[2] = {}, order2 = 0, total = 0;
};
Plan plan_of(const pp_embed_desc& d) {
  Plan p;
  p.lanes = lanes_for(d.d);
  // One launch instead of two or three, at the risk that one row has all tokens, whose
  // features one workgroup then reads (at 100 GB/s).  us a call, one launch / three:
  // 777 tokens into 5003 x 203 fp32 8 / 15, 128 tokens into 50000 x 1024 bf16 21 / 26;
  // all of one row: 777 tokens 26 / 15, 256 tokens, 1024 features, fp32 (1 MB) 25 / 15,
  // 1024 tokens (4 MB) 85 / 18.
  p.few = d.t <= kFewTokens && d.t * d.d * static_cast<int64_t>(size_of(d.y_dtype)) <= 1 << 20;
  // Workgroups of sort_kernel and few_kernel: as many as CUs, or more where one's rows
  // would be too many; of narrow rows some at a time, 256 bytes, so that whole lines of
  // memory are written by one.
  const int64_t bytes = d.d * static_cast<int64_t>(size_of(d.w_dtype));
  p.deal.run = 0, p.deal.log = 0;
  while (bytes << p.deal.run < 256) ++p.deal.run;
  const int64_t runs = cdiv(d.v, int64_t(1) << p.deal.run);
  while (int64_t(1) << p.deal.log < std::min<int64_t>(runs, kCUs) || cdiv(runs, int64_t(1) << p.deal.log) << p.deal.run > kSortRows)
    ++p.deal.log;
  p.deal.per = static_cast<int32_t>(cdiv(runs, int64_t(1) << p.deal.log) << p.deal.run);
  // The sort by digits: two launches (five for two digits), but no workgroup that reads
  // all ids or has all tokens of a row.  us a call, sort_kernel / digits: 313 rows of 256
  // bf16 features, three in ten ids the same, 16384 tokens 20 / 20, 32768 27 / 21, 2^20
  // 665 / 129; 50000 rows of 64 features, 32768 tokens: ids log-uniform 27 / 30, uniform
  // 22 / 30, three in ten the same 35 / 31; 65536: 38 / 33, 26 / 33, 56 / 35; 2^20: 571 /
  // 102, 179 / 96, 845 / 100; 200000 rows of 256, 16384 tokens: 33 / 44, 32 / 44, 40 / 46.
  // sort_kernel's workgroups come in rounds of kCUs, each of about 4.5 us and 0.2 for
  // 1000 tokens.
  const int64_t rounds = cdiv(int64_t(1) << p.deal.log, kCUs);
  int all = 0;
  while (int64_t(1) << all < d.v) ++all;
  if (!p.few && (d.v <= kSortRows ? d.t > 16384 : rounds * (d.t + 22500) >= 88000)) {
    p.digits = d.v <= kSortRows ? 1 : (all + kOwnBits - 1) / kOwnBits;
    p.deal.run = 0, p.deal.log = 0, p.deal.per = static_cast<int32_t>(d.v);
    p.each = static_cast<int32_t>(cdiv(d.t, kCounts * 1024) * 1024);
    p.counts = static_cast<int32_t>(cdiv(d.t, p.each));
    for (int k = 0, done = 0; k < p.digits; ++k) {
      p.bits[k] = (all - done) / (p.digits - k);
      p.values[k] = k + 1 < p.digits ? 1 << p.bits[k] : static_cast<int32_t>(cdiv(d.v, int64_t(1) << done));
      done += p.bits[k];
    }
  }
  const int64_t groups = 256 >> p.lanes.log;
  p.batches = static_cast<int32_t>(std::max<int64_t>(1, cdiv(d.t, groups * kBatch * kPieces)));
  p.piece = static_cast<int32_t>(groups) * kBatch * p.batches;
  p.pieces = static_cast<int32_t>(cdiv(d.t, p.piece));
  p.part_ld = static_cast<int32_t>(cdiv(d.d, 8) * 8);
  auto take = [&](int64_t n) {
    const size_t at = p.total;
    p.total += static_cast<size_t>(cdiv(n, 256) * 256);
    return at;
  };
  take(4 * (p.digits > 1 ? 2 * d.v : p.deal.entries()));
  p.order = take(static_cast<int64_t>(sizeof(Place)) * d.t);
  p.part = take(p.pieces > 1 ? static_cast<int64_t>(p.pieces) * 2 * p.part_ld * 4 : 0);
  if (p.digits) p.count = take(4 * static_cast<int64_t>(p.counts) * kSortRows);
  if (p.digits > 1) {
    for (size_t& at : p.starts) at = take(4 * (kSortRows + 1));
    p.order2 = take(static_cast<int64_t>(sizeof(Place)) * d.t);
  }
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
  const int64_t per = 256 >> l.log;        // tokens of a workgroup
  if (per == 1 && d.t >= kGrid) return fail(PP_EUNSUPPORTED, "too many tokens of this length");
  // (a launch of fewer than kGrid workgroups; nearly always one)
  const int64_t most = (kGrid - 1) * per;
  for (int64_t t0 = 0; t0 < d.t; t0 += most) {
    const int64_t t = std::min(most, d.t - t0);
    uint8_t* rows = static_cast<uint8_t*>(y) + t0 * d.y_ld * static_cast<int64_t>(size_of(d.y_dtype));
    const Look a = {ids + t0, w, rows, t, d.v, d.w_ld, d.y_ld, d.ignore_index, static_cast<int32_t>(d.d), l.log, d.scale};
    const dim3 grid(static_cast<uint32_t>(cdiv(t, per)), static_cast<uint32_t>(l.columns));
    with_types(d.w_dtype, d.y_dtype, [&](auto wt, auto yt) {
      hipLaunchKernelGGL((look_kernel<decltype(wt), decltype(yt)>), grid, dim3(256), 0, st, a);
    });
    const pp_status s = launched();
    if (s != PP_OK) return s;
  }
  return PP_OK;
}

pp_status grad(const pp_embed_desc* desc, const int64_t* ids, const void* dy, const void* add, void* dw, void* ws, size_t bytes,
               hipStream_t st) {
  pp_status r = check(desc);
  if (r == PP_OK) r = check_rows(*desc);
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
  Place* order = reinterpret_cast<Place*>(base + p.order);

  const bool row = d.ignore_index >= 0 && d.ignore_index < d.v;
  const Sort s = {ids, start, order, static_cast<uint32_t>(d.v), static_cast<uint32_t>(row ? d.ignore_index : d.v),
                  static_cast<int32_t>(d.t), p.deal};
  const bool several = p.digits > 1;
  auto start_of = [&](int k) { return several ? reinterpret_cast<int32_t*>(base + p.starts[k & 1]) : start; };   // of digit k
  const Sum a = {start, start + (several ? d.v : 1), p.digits ? start_of(p.digits - 1) + p.values[p.digits - 1] : start + p.deal.entries() - 1, order,
                 dy, add, dw, reinterpret_cast<float*>(base + p.part), d.y_ld, d.w_ld, static_cast<int32_t>(d.t), static_cast<int32_t>(d.v),
                 static_cast<int32_t>(d.d), p.lanes.log, p.deal, p.pieces, p.batches, p.piece, p.part_ld, d.scale};
  // (a gradient that is added to in place: rows without a token stay as they are)
  const int64_t fills = add == dw ? 0 : cdiv(d.v, (256 >> p.lanes.log) * kFillRows);
  const dim3 sums(static_cast<uint32_t>(p.pieces + fills), static_cast<uint32_t>(p.lanes.columns));
  const dim3 joins(static_cast<uint32_t>(p.pieces), static_cast<uint32_t>(cdiv(d.d, 256)));
  with_types(d.y_dtype, d.w_dtype, [&](auto yt, auto wt) {
    using Y = decltype(yt);
    using W = decltype(wt);
    if (p.few) {
      hipLaunchKernelGGL((few_kernel<Y, W>), dim3(1u << p.deal.log, static_cast<uint32_t>(p.lanes.columns)), dim3(kFewTokens), 0, st, s, a);
      return;
    }
    if (p.digits) {
      const dim3 block(kSortWaves * 64);
      Digit f = {};
      f.ids = ids, f.count = reinterpret_cast<uint32_t*>(base + p.count), f.v = s.v, f.ignore = s.ignore, f.t = s.t;
      f.each = p.each, f.groups = p.counts;
      if (several && fills) f.clear = start, f.cleared = 2 * d.v;   // (rows without a token are looked for by it)
      for (int k = 0; k < p.digits; ++k) {
        f.start = start_of(k), f.values = p.values[k], f.bits = p.bits[k];
        // (the last digit's list is `order`)
        f.order = (p.digits - k) % 2 ? order : reinterpret_cast<Place*>(base + p.order2);
        if (k == 0) {
          const int64_t clears = std::min<int64_t>(1024, cdiv(f.cleared, 16384));
          hipLaunchKernelGGL((count_kernel<true>), dim3(static_cast<uint32_t>(std::max<int64_t>(p.counts, clears))), block, 0, st, f);
          hipLaunchKernelGGL((place_kernel<true>), dim3(p.counts), block, 0, st, f);
        } else {
          hipLaunchKernelGGL((count_kernel<false>), dim3(p.counts), block, 0, st, f);
          hipLaunchKernelGGL((place_kernel<false>), dim3(p.counts), block, 0, st, f);
        }
        f.in = f.order, f.in_total = f.start + f.values, f.shift += f.bits;
      }
      if (several)
        hipLaunchKernelGGL(bounds_kernel, dim3(static_cast<uint32_t>(cdiv(d.t, 256))), dim3(256), 0, st, order, a.total, start, start + d.v);
    } else {
      hipLaunchKernelGGL(sort_kernel, dim3(1u << p.deal.log), dim3(kSortWaves * 64), 0, st, s);
    }
    if (sums.x) hipLaunchKernelGGL((sum_kernel<Y, W>), sums, dim3(256), 0, st, a);
    if (p.pieces < 2) return;
    if (joins.y == 1)
      hipLaunchKernelGGL((join_kernel<W, 8>), joins, dim3(8 * 64), 0, st, a);
    else
      hipLaunchKernelGGL((join_kernel<W, 4>), joins, dim3(4 * 64), 0, st, a);
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
    pp_status s = check(desc);
    if (s == PP_OK) s = check_rows(*desc);
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
