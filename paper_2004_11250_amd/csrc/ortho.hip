// ortho.hip -- pp_ortho / pp_muon_step: updates orthogonalised by
// Newton-Schulz products, and the weight step of (pruned) layers with them.
//
//   X = U / (|U|_F + eps), turned so that it has m <= n rows, then `steps` times
//   A = X X^T,  B = b A + c A^2,  X <- a X + B X
//
// so every singular value s of X goes to a s + b s^3 + c s^5, towards 1.
//
// Numbers.  Small singular values grow by about a factor a a step, and with
// them what was rounded off X, A and B: 16 bits a value would leave errors of
// a few per cent.  X, A and B are therefore kept as pairs of fp16 values
// (22 bits; the values' range is known, so a fixed power of two keeps them
// clear of fp16's ends), products are summed in fp32, and
//   fp32 updates   take three plane products each (all but rest x rest), and
//                  a is added to B's diagonal: X <- (a + B) X;
//   bf16 updates   take one: the upper values' product.  The rests enter where
//                  they cost nothing, in the epilogues: a X and b A use both
//                  values, and of A's and B's rests, whose largest part by far
//                  lies on the diagonal, the diagonal is multiplied in
//                  (A_h D + D A_h, D X).  The error of five steps is 1.0e-3 to
//                  1.7e-3 of the result beside the output's own rounding of
//                  1.7e-3 (2048 x 2048 and 70 x 90 of normal values; 1.2e-3
//                  with strong directions over them, 1e-4 to 1e-3 where rows or
//                  single directions dominate); without the diagonals it is 2
//                  to 4e-3.
//
// All matrices of a call go through each stage in one launch: a sum of
// squares, the scaling, and three products a step.  (Small ones are done whole by
// a workgroup each.)  A and B are symmetric:
// only the tiles on and below the diagonal are computed, and written twice.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <string>
#include <vector>

#include "api_internal.hpp"
#include "gemm_tile.hpp"
#include "train.hpp"

namespace pp {
namespace {

using half_t = _Float16;

// X, A and B are stored times these
constexpr float kSX = 8192.f, kSA = 4096.f, kSB = 1024.f;

enum { kStageNorm = 0, kStageFill, kStageGram, kStagePoly, kStageApply, kStages };

struct Mat {
  // the update (r, c), r < rows, c < cols
  const void* u;
  int64_t u_rs, u_cs;
  void* o;
  int64_t o_rs, o_cs;
  // the weight step (rows x cols contiguous); g null: only orthogonalise
  const void* g;
  const float* mom;
  const void* w;
  void* w_out;
  float* mom_out;
  const uint16_t* keep;
  float up;                     // lr times the layer's scale
  int32_t rows, cols;
  int32_t turned;               // X is the transpose: m = cols, n = rows
  int32_t m, n, mp, np;
  int32_t wide, o_wide;         // pieces of eight of a contiguous row are 16-byte aligned
  int32_t chunk, chunks;        // elements a workgroup of the sum of squares takes
  half_t* x[2];                 // [2 planes][m][np], two in turn
  half_t* a;                    // [2][m][mp]
  half_t* b;                    // [2][m][mp]
  float *da, *db;               // [m]: the diagonals' rests of A and B (bf16)
  double* part;                 // [chunks]
};

struct Step {
  float lr, momentum, decay;
  int32_t nesterov;
  float a, b, c, eps;
  int32_t steps;
};

constexpr int kSetup = 12;      // matrices a set-up launch brings (kernel arguments hold 4 KB)
struct Setup {
  Mat mat[kSetup];
  int32_t start[kStages][kSetup];
  int32_t first, count, all;
};

// The plan in device memory: all matrices, and for each stage the first tile
// of each.
struct Table {
  const Mat* mat;
  const int32_t* start;         // [kStages][all]
  int32_t all;
  Mat one;                      // the matrix, if there is only one
};

__global__ __launch_bounds__(256) void setup_kernel(Setup s, Mat* mat, int32_t* start) {
  const int words = s.count * static_cast<int>(sizeof(Mat) / 4);
  const uint32_t* from = reinterpret_cast<const uint32_t*>(s.mat);
  uint32_t* to = reinterpret_cast<uint32_t*>(mat + s.first);
  for (int i = threadIdx.x; i < words; i += 256) to[i] = from[i];
  for (int i = threadIdx.x; i < kStages * s.count; i += 256) {
    const int k = i / s.count, j = i - k * s.count;
    start[k * s.all + s.first + j] = s.start[k][j];
  }
}

// A matrix of the plan, by scalar loads (an earlier kernel wrote it: constant
// here).
__device__ __forceinline__ Mat get(const Table& t, int i) {
  if (t.all == 1) return t.one;
  struct Words {
    uint32_t w[sizeof(Mat) / 4];
  } x;
  const auto* p = (const __attribute__((address_space(4))) uint32_t*)reinterpret_cast<uintptr_t>(t.mat + i);
#pragma unroll
  for (int k = 0; k < static_cast<int>(sizeof(Mat) / 4); ++k) x.w[k] = p[k];
  return __builtin_bit_cast(Mat, x);
}

// A product stage's tiles over the workgroups: workgroups are dealt to the
// eight XCDs (each with an L2 of its own) in turn, so runs of `chunk`
// consecutive tiles, which share operands, go to one XCD each.
struct Spread {
  int32_t total, chunk;
};
__device__ __forceinline__ int spread(const Spread& s, int block) {
  const int slot = block >> 3;
  return (slot / s.chunk * 8 + (block & 7)) * s.chunk + slot % s.chunk;
}

// The matrix that tile `id` of a stage belongs to; *local: its tile there.
__device__ __forceinline__ int find(const Table& t, int stage, const int id, int* local) {
  if (t.all == 1) {
    *local = id;
    return 0;
  }
  const int32_t* st = t.start + stage * t.all;
  int at = -1;
  for (int i = 0; i < t.all; i += 64) {
    const int k = i + (threadIdx.x & 63);
    const bool below = k < t.all && st[k] <= id;
    at += __popcll(__ballot(below));
  }
  at = __builtin_amdgcn_readfirstlane(at);
  *local = id - __builtin_amdgcn_readfirstlane(st[at]);
  return at;
}

// Which of the elements e .. e + 7 of a layer are kept taps (bit by bit).
__device__ __forceinline__ uint32_t kept8(const Mat& m, uint32_t e, uint32_t all) {
  if (!m.keep) return 255u;
  const uint32_t k = e / 9u;
  uint32_t bits = m.keep[k] & 511u;
  if ((k + 1u) * 9u < all) bits |= static_cast<uint32_t>(m.keep[k + 1]) << 9;
  return bits >> (e - 9u * k);
}

// Eight values from p on, of which n are there; wide: p is aligned to 16
// bytes, and all eight are.
template <class S>
__device__ __forceinline__ void load8(const S* p, int n, bool wide, float (&v)[8]) {
  if (wide) {
    using S8 = __attribute__((ext_vector_type(8))) S;
    const S8 x = *reinterpret_cast<const S8*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? static_cast<float>(p[e]) : 0.f;
  }
}
template <class S>
__device__ __forceinline__ void store8(S* p, int n, bool wide, const float (&v)[8]) {
  if (wide) {
    using S8 = __attribute__((ext_vector_type(8))) S;
    S8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = static_cast<S>(v[e]);
    *reinterpret_cast<S8*>(p) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = static_cast<S>(v[e]);
  }
}

// elements e .. e + 7 of a weight step's update, from the new momentum
template <class S>
__device__ __forceinline__ void update8(const Mat& m, const Step& s, uint32_t e, int n, float (&u)[8]) {
  const bool wide = m.wide && n == 8 && e % 8 == 0;
  load8(m.mom_out + e, n, wide, u);
  if (!s.nesterov) return;
  const uint32_t on = kept8(m, e, static_cast<uint32_t>(m.rows) * m.cols);
  float g[8];
  load8(static_cast<const S*>(m.g) + e, n, wide, g);
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = (on >> i & 1 ? g[i] : 0.f) + s.momentum * u[i];
}

// The sum of squares of each matrix, in 64 bits, a chunk a workgroup; a
// weight step's momentum on the way.  Bound by memory: bf16 4096 x 4096 10 us,
// 3.4 TB/s; the weight step of VGG-16's pruned layers, fp32, 36 us, 4.9 TB/s.
template <class S>
__global__ __launch_bounds__(256) void norm_kernel(Table t, Step s) {
  __shared__ double sums[4];
  int chunk;
  const Mat m = get(t, find(t, kStageNorm, blockIdx.x, &chunk));
  const uint32_t all = static_cast<uint32_t>(m.rows) * m.cols, e0 = static_cast<uint32_t>(chunk) * m.chunk;
  const uint32_t e1 = e0 + m.chunk < all ? e0 + m.chunk : all;
  double sum[2] = {0., 0.};
  auto add = [&](const float (&u)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i & 1] += static_cast<double>(u[i]) * u[i];
  };
  if (m.g) {
    for (uint32_t e = e0 + 8 * threadIdx.x; e < e1; e += 2048) {
      const int n = e1 - e < 8 ? static_cast<int>(e1 - e) : 8;
      const bool wide = m.wide && n == 8;
      float g[8], mom[8];
      load8(static_cast<const S*>(m.g) + e, n, wide, g);
      load8(m.mom + e, n, wide, mom);
      const uint32_t on = kept8(m, e, all);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        g[i] = on >> i & 1 ? g[i] : 0.f;
        mom[i] = on >> i & 1 ? s.momentum * mom[i] + g[i] : 0.f;
      }
      store8(m.mom_out + e, n, wide, mom);
      if (s.nesterov) {
#pragma unroll
        for (int i = 0; i < 8; ++i) mom[i] = g[i] + s.momentum * mom[i];
      }
      add(mom);
    }
  } else if (m.u_cs == 1 && m.u_rs == m.cols) {
    for (uint32_t e = e0 + 8 * threadIdx.x; e < e1; e += 2048) {
      const int n = e1 - e < 8 ? static_cast<int>(e1 - e) : 8;
      float u[8];
      load8(static_cast<const S*>(m.u) + e, n, m.wide && n == 8, u);
      add(u);
    }
  } else {
    for (uint32_t e = e0 + threadIdx.x; e < e1; e += 256) {
      const uint32_t r = e / static_cast<uint32_t>(m.cols), c = e - r * m.cols;
      const float u = static_cast<float>(static_cast<const S*>(m.u)[r * m.u_rs + c * m.u_cs]);
      sum[0] += static_cast<double>(u) * u;
    }
  }
  double x = sum[0] + sum[1];
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = x;
  __syncthreads();
  if (threadIdx.x == 0) m.part[chunk] = sums[0] + sums[1] + sums[2] + sums[3];
}

// X = U times / (|U| + eps), for any norm of finite fp32 values: fp32 holds the
// factor itself from norms of 2^-115 on (below it is infinite) up to 2^126 (above
// it loses bits), so a power of two goes first, which is exact.  (Where that
// takes bits from an element, the element is 2^-100 of the norm.)  0 where U is.
struct Scale {
  float first, then;
  __device__ __forceinline__ float operator()(float x) const { return x * first * then; }
};
__device__ __forceinline__ Scale scale_of(double squares, float eps, float times) {
  const double norm = sqrt(squares) + static_cast<double>(eps);
  const double first = norm < 0x1p-64 ? 0x1p80 : norm > 0x1p64 ? 0x1p-64 : 1.;
  return {static_cast<float>(first), norm == 0. ? 0.f : static_cast<float>(times / (norm * first))};
}

__device__ __forceinline__ void split(float x, half_t* h, half_t* l) {
  *h = static_cast<half_t>(x);
  *l = static_cast<half_t>(x - static_cast<float>(*h));
}

// X = U / (|U| + eps), padded with zeros.  Bound by memory: bf16 4096 x 4096 21 us,
// 4.8 TB/s; VGG-16's layers 36 us (the update is formed again from the momentum:
// cheaper than a copy of it).
template <class S>
__global__ __launch_bounds__(256) void fill_kernel(Table t, Step s) {
  __shared__ float tile[64][65];
  __shared__ double sums[4];
  int id;
  const Mat m = get(t, find(t, kStageFill, blockIdx.x, &id));
  const int tid = threadIdx.x;
  double sum = 0.;
  for (int i = tid; i < m.chunks; i += 256) sum += m.part[i];
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if ((tid & 63) == 0) sums[tid >> 6] = sum;
  __syncthreads();
  const Scale scale = scale_of(sums[0] + sums[1] + sums[2] + sums[3], s.eps, kSX);

  const int tc = m.np / 64, r0 = id / tc * 64, c0 = id % tc * 64;
  // pieces of eight along the update's own rows, or down them if its columns
  // are the contiguous ones
  const bool rows = m.g || m.u_cs <= m.u_rs;
  const bool along_n = rows != static_cast<bool>(m.turned);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int u = (tid >> 3) + 32 * i, w = (tid & 7) * 8;
    const int r = r0 + (along_n ? u : w), c = c0 + (along_n ? w : u);
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (r < m.m && c < m.n) {
      const int left = along_n ? m.n - c : m.m - r, n = left < 8 ? left : 8;
      const int ur = m.turned ? c : r, uc = m.turned ? r : c;
      if (m.g) {
        update8<S>(m, s, static_cast<uint32_t>(ur) * m.cols + uc, n, x);
      } else if (rows && m.u_cs == 1) {
        load8(static_cast<const S*>(m.u) + ur * m.u_rs + uc, n, m.wide && n == 8, x);
      } else {
        const S* at = static_cast<const S*>(m.u) + ur * m.u_rs + uc * m.u_cs;
        const int64_t step = rows ? m.u_cs : m.u_rs;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < n ? static_cast<float>(at[e * step]) : 0.f;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = scale(x[e]);
      if (along_n)
        tile[u][w + e] = c + e < m.n ? v : 0.f;
      else
        tile[w + e][u] = r + e < m.m ? v : 0.f;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int u = (tid >> 3) + 32 * i, w = (tid & 7) * 8;
    if (r0 + u >= m.m) continue;
    f16x8 h, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      half_t a, b;
      split(tile[u][w + e], &a, &b);
      h[e] = a, l[e] = b;
    }
    half_t* at = m.x[0] + static_cast<int64_t>(r0 + u) * m.np + c0 + w;
    *reinterpret_cast<f16x8*>(at) = h;
    *reinterpret_cast<f16x8*>(at + static_cast<int64_t>(m.m) * m.np) = l;
  }
}

// planes [2][count][ld] as an operand whose rows (or k, by_k) are the count
__device__ __forceinline__ GemmOperand planes_of(const half_t* p, int count, int ld, bool by_k = false) {
  GemmOperand o;
  o.plane[0] = p;
  o.plane[1] = p + static_cast<int64_t>(count) * ld;
  o.plane[2] = p;
  o.ld = __builtin_amdgcn_readfirstlane(ld);
  o.rows = __builtin_amdgcn_readfirstlane(by_k ? ld : count);
  o.k = __builtin_amdgcn_readfirstlane(by_k ? count : ld);
  return o;
}

// Tile t of the lower triangle, row by row.
__device__ __forceinline__ void triangle(int t, int* ti, int* tj) {
  int r = static_cast<int>((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
  while (r * (r + 1) / 2 > t) --r;
  while ((r + 1) * (r + 2) / 2 <= t) ++r;
  *ti = r;
  *tj = t - r * (r + 1) / 2;
}

__device__ __forceinline__ void split8(const float (&v)[8], f16x8* h, f16x8* l) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    half_t a, b;
    split(v[e], &a, &b);
    (*h)[e] = a, (*l)[e] = b;
  }
}
// a pair of fp16 values as one
__device__ __forceinline__ void pair8(const half_t* h, int64_t plane, float (&v)[8]) {
  const f16x8 a = *reinterpret_cast<const f16x8*>(h), b = *reinterpret_cast<const f16x8*>(h + plane);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(a[e]) + static_cast<float>(b[e]);
}

// A = X X^T (POLY false) or B = b A + c A A^T (POLY true); P: values of X, A
// and B in the products.  Bound by the products where there are tiles for every
// CU: bf16 4096 x 4096 97 us, 0.71 PFLOP/s of one triangle, with its store twice
// (256 x 256 tiles, 136 of them: 110 us); by the length of a tile's sum where
// there are few (VGG-16, fp32, k 4608: 45 us; 313 x 256: 5 us).
template <class Tile, int P, bool POLY>
__global__ __launch_bounds__(Tile::THREADS) void gram_kernel(Table t, Step s, PlanePairs pairs, int32_t turn, Spread sp) {
  __shared__ __align__(1024) uint8_t lds[Tile::LDS_BYTES];
  int id = spread(sp, blockIdx.x);
  if (id >= sp.total) return;
  const Mat m = get(t, find(t, POLY ? kStagePoly : kStageGram, id, &id));
  int ti, tj;
  triangle(id, &ti, &tj);
  const int row0 = ti * Tile::BM, col0 = tj * Tile::BN;
  const GemmOperand x = POLY ? planes_of(m.a, m.m, m.mp) : planes_of(turn ? m.x[1] : m.x[0], m.m, m.np);
  const int ksteps = (POLY ? m.mp : m.np) / kBK;
  f32x4 acc[Tile::FM][Tile::FN];
  Tile::run(x, x, pairs, row0, col0, ksteps, 0, Tile::steps_of(ksteps, pairs), lds, acc);
  const int mm = m.m, mp = m.mp;
  const int64_t plane = static_cast<int64_t>(mm) * mp;
  const half_t* a = m.a;
  half_t* out = POLY ? m.b : m.a;
  const float fa = s.b * (kSB / kSA), fc = POLY ? s.c * (kSB / (kSA * kSA)) : kSA / (kSX * kSX);
  // Element (r, c) of the tile is also element (c, r) of the matrix: columns are
  // stored first, by their finished values, which then go out again as rows.
  // (Rows past m are zeros in both operands, so the padding comes out as zeros.)
  Tile::staged(lds, acc, [&](int rb, int cb, typename Tile::View view) {
    rb += row0, cb += col0;
#pragma unroll 4
    for (int i = 0; i < view.pieces(); ++i) {
      int r, c;
      view.col_piece(i, &r, &c);
      const int y = cb + c, x = rb + r;   // (y, x .. x + 7) of the matrix
      if (y >= mm || x >= mp) continue;
      float v[8];
      view.col(r, c, v);
      const int64_t at = static_cast<int64_t>(y) * mp + x;
      if constexpr (POLY) {
        const f16x8 h = *reinterpret_cast<const f16x8*>(a + at), l = *reinterpret_cast<const f16x8*>(a + at + plane);
        if constexpr (P == 1) {
          const float d = m.da[y];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += static_cast<float>(h[e]) * (d + m.da[x + e < mm ? x + e : mm - 1]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fc * v[e] + fa * (static_cast<float>(h[e]) + static_cast<float>(l[e]));
        if constexpr (P > 1) {   // a X comes with B X
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += x + e == y ? s.a * kSB : 0.f;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= fc;
      }
      if (ti != tj) view.put_col(r, c, v);
      f16x8 h, l;
      split8(v, &h, &l);
      *reinterpret_cast<f16x8*>(out + at) = h;
      if (!POLY || P > 1) *reinterpret_cast<f16x8*>(out + at + plane) = l;
      if (P == 1 && y >= x && y < x + 8) {
        float* d = POLY ? m.db : m.da;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (y == x + e) d[y] = static_cast<float>(l[e]);
      }
    }
    if (ti == tj) return;
    view.turn();
#pragma unroll 4
    for (int i = 0; i < view.pieces(); ++i) {
      int r, c;
      view.row_piece(i, &r, &c);
      if (rb + r >= mm || cb + c >= mp) continue;
      float v[8];
      view.row(r, c, v);
      f16x8 h, l;
      split8(v, &h, &l);
      const int64_t at = static_cast<int64_t>(rb + r) * mp + cb + c;
      *reinterpret_cast<f16x8*>(out + at) = h;
      // (else only this half's rests that may share a tile of the next product
      // with the diagonal are read)
      if (P > 1 || (!POLY && abs(rb + r - cb - c) < tile_m(1, kBig)))
        *reinterpret_cast<f16x8*>(out + at + plane) = l;
    }
  });
}

// results (r, c) .. (r, c + 7) of a matrix, of which n are there
template <class S>
__device__ __forceinline__ void put_result(const Mat& m, const Step& s, int r, int c, int n, const float (&v)[8]) {
  n = n < 8 ? n : 8;
  if (m.g) {
    const uint32_t e = static_cast<uint32_t>(r) * m.cols + c;
    const bool wide = m.wide && n == 8 && e % 8 == 0;
    const uint32_t on = kept8(m, e, static_cast<uint32_t>(m.rows) * m.cols);
    const float decay = 1.f - s.lr * s.decay;
    float w[8];
    load8(static_cast<const S*>(m.w) + e, n, wide, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = on >> i & 1 ? decay * w[i] - m.up * v[i] : 0.f;
    store8(static_cast<S*>(m.w_out) + e, n, wide, w);
  } else if (m.o_cs == 1) {
    store8(static_cast<S*>(m.o) + r * m.o_rs + c, n, m.o_wide && n == 8, v);
  } else {
    S* at = static_cast<S*>(m.o) + r * m.o_rs + c * m.o_cs;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) at[e * m.o_cs] = static_cast<S>(v[e]);
  }
}

// X <- a X + B X; the last one writes the result instead: the orthogonalised
// update, or the weights.
// (Bound by the products: bf16 4096 x 4096 131 to 144 us, 1.0 PFLOP/s; VGG-16,
// fp32, three products 54 us, 0.8 PFLOP/s.)
template <class Tile, class S, int P, bool LAST>
__global__ __launch_bounds__(Tile::THREADS) void apply_kernel(Table t, Step s, PlanePairs pairs, int32_t turn, Spread sp) {
  __shared__ __align__(1024) uint8_t lds[Tile::LDS_BYTES];
  int id = spread(sp, blockIdx.x);
  if (id >= sp.total) return;
  const Mat m = get(t, find(t, kStageApply, id, &id));
  const int mm = m.m, nn = m.n, mp = m.mp, np = m.np;
  // the tile's rows are X's columns: a lane's eight rows of a tile's column
  // follow each other in X
  int ti, tj;
  band_order(id, (np + Tile::BM - 1) / Tile::BM, (mm + Tile::BN - 1) / Tile::BN, &ti, &tj);
  const int row0 = ti * Tile::BM, col0 = tj * Tile::BN;
  const int ksteps = mp / kBK;
  f32x4 acc[Tile::FM][Tile::FN];
  const half_t* from = turn ? m.x[1] : m.x[0];
  half_t* to = turn ? m.x[0] : m.x[1];
  Tile::run(planes_of(from, mm, np, true), planes_of(m.b, mm, mp), pairs, row0, col0, ksteps, 0, Tile::steps_of(ksteps, pairs), lds, acc);
  const int64_t plane = static_cast<int64_t>(mm) * np;
  const bool turned = m.turned;
  Tile::staged(lds, acc, [&](int rb, int cb, typename Tile::View view) {
    rb += row0, cb += col0;
#pragma unroll 4
    for (int i = 0; i < view.pieces(); ++i) {
      int r, c;
      view.col_piece(i, &r, &c);
      if (cb + c >= mm || rb + r >= np) continue;
      float v[8];
      view.col(r, c, v);
      const int64_t at = static_cast<int64_t>(cb + c) * np + rb + r;
      const float fb = LAST ? 1.f / (kSB * kSX) : 1.f / kSB, fx = LAST ? s.a / kSX : s.a;
      if constexpr (P == 1) {
        float x[8];
        pair8(from + at, plane, x);
        const float d = m.db[cb + c];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fx * x[e] + fb * (v[e] + d * x[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= fb;
      }
      if constexpr (LAST) {
        if (turned)
          view.put_col(r, c, v);
        else
          put_result<S>(m, s, cb + c, rb + r, nn - (rb + r), v);
      } else {
        f16x8 h, l;
        split8(v, &h, &l);
        *reinterpret_cast<f16x8*>(to + at) = h;
        *reinterpret_cast<f16x8*>(to + at + plane) = l;
      }
    }
    if (!LAST || !turned) return;
    view.turn();
#pragma unroll 4
    for (int i = 0; i < view.pieces(); ++i) {
      int r, c;
      float v[8];
      view.row_piece(i, &r, &c);
      if (rb + r >= nn || cb + c >= mm) continue;
      view.row(r, c, v);
      put_result<S>(m, s, rb + r, cb + c, mm - (cb + c), v);
    }
  });
}

// ---------------------------------------------------------------------------
// small matrices: a workgroup does all steps of one, in LDS and in fp32
// ---------------------------------------------------------------------------

// A launch costs 3 us and more on the card, and a matrix of the staged path
// three of them a step.  Up to the sizes of tiny_fits() one CU's fp32 matrix
// instructions take less than that, and need no pairs of values.  16 x 144: 18 us
// for five steps, of which the matrix instructions are 1: bound by the latency of
// fifteen products that wait for each other.
constexpr int kTinyWaves = 8, kTinyRows = 64, kTinyFloats = 28000;
constexpr int kTinyLd = 68;     // row pitch of A and B: 4 past a multiple of the banks
__host__ __device__ constexpr int tiny_ld(int n) { return (n + 63) / 64 * 64 + 4; }

bool tiny_fits(int m, int n) {
  const int64_t m16 = (m + 15) / 16 * 16, n16 = (n + 15) / 16 * 16;
  return m16 <= kTinyRows && m16 * tiny_ld(n) <= kTinyFloats && m16 * m16 * n16 <= 600000;
}

template <class S>
__global__ __launch_bounds__(kTinyWaves * 64) void tiny_kernel(Setup su, Step s) {
  __shared__ float x[kTinyFloats];
  __shared__ float a[kTinyRows * kTinyLd], b[kTinyRows * kTinyLd];
  __shared__ f32x4 part[kTinyWaves][64];
  __shared__ double sums[kTinyWaves];
  constexpr int kThreads = kTinyWaves * 64;
  const Mat& m = su.mat[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mt = (m.m + 15) / 16, nt = (m.n + 15) / 16, ld = tiny_ld(m.n);
  const int all = m.rows * m.cols, cols = m.cols;

  // the update, and its sum of squares
  for (int e = tid; e < mt * 16 * ld; e += kThreads) x[e] = 0.f;
  __syncthreads();
  double sum = 0.;
  for (int e = tid; e < all; e += kThreads) {
    const int r = e / cols, c = e - r * cols;
    float u;
    if (m.g) {
      const bool on = kept8(m, static_cast<uint32_t>(e), static_cast<uint32_t>(all)) & 1;
      const float g = on ? static_cast<float>(static_cast<const S*>(m.g)[e]) : 0.f;
      const float mom = on ? s.momentum * m.mom[e] + g : 0.f;
      m.mom_out[e] = mom;
      u = s.nesterov ? g + s.momentum * mom : mom;
    } else {
      u = static_cast<float>(static_cast<const S*>(m.u)[r * m.u_rs + c * m.u_cs]);
    }
    sum += static_cast<double>(u) * u;
    x[m.turned ? c * ld + r : r * ld + c] = u;
  }
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  sum = 0.;
  for (int i = 0; i < kTinyWaves; ++i) sum += sums[i];
  const Scale scale = scale_of(sum, s.eps, 1.f);
  for (int e = tid; e < mt * 16 * ld; e += kThreads) x[e] = scale(x[e]);
  __syncthreads();

  // a lane's operand values: row or column lane % 16, k lane / 16
  const int l16 = lane & 15, lk = lane >> 4;
  const int tiles = mt * (mt + 1) / 2, parts = tiles < kTinyWaves ? kTinyWaves / tiles : 1;
  for (int step = 0; step < s.steps; ++step) {
    // A: tiles on and below the diagonal, k in `parts` parts
    for (int job = wave; job < tiles * parts; job += kTinyWaves) {
      const int t = job / parts, p = job - t * parts;
      int ti, tj;
      triangle(t, &ti, &tj);
      const int k0 = nt * p / parts * 16, k1 = nt * (p + 1) / parts * 16;
      f32x4 acc[4] = {};
      for (int k = k0; k < k1; k += 16)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          acc[q] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[(ti * 16 + l16) * ld + k + 4 * q + lk], x[(tj * 16 + l16) * ld + k + 4 * q + lk],
                                                        acc[q], 0, 0, 0);
      const f32x4 v = (acc[0] + acc[1]) + (acc[2] + acc[3]);
      if (parts > 1) {
        part[job][lane] = v;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a[(ti * 16 + 4 * lk + e) * kTinyLd + tj * 16 + l16] = v[e];
          a[(tj * 16 + l16) * kTinyLd + ti * 16 + 4 * lk + e] = v[e];
        }
      }
    }
    __syncthreads();
    if (parts > 1) {
      if (wave < tiles) {
        f32x4 v = part[wave * parts][lane];
        for (int p = 1; p < parts; ++p) v += part[wave * parts + p][lane];
        int ti, tj;
        triangle(wave, &ti, &tj);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a[(ti * 16 + 4 * lk + e) * kTinyLd + tj * 16 + l16] = v[e];
          a[(tj * 16 + l16) * kTinyLd + ti * 16 + 4 * lk + e] = v[e];
        }
      }
      __syncthreads();
    }
    for (int job = wave; job < mt * mt; job += kTinyWaves) {
      const int ti = job / mt, tj = job - ti * mt;
      f32x4 acc[4] = {};
      for (int k = 0; k < mt * 16; k += 16)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          acc[q] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[(ti * 16 + l16) * kTinyLd + k + 4 * q + lk],
                                                        a[(tj * 16 + l16) * kTinyLd + k + 4 * q + lk], acc[q], 0, 0, 0);
      const f32x4 v = (acc[0] + acc[1]) + (acc[2] + acc[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at = (ti * 16 + 4 * lk + e) * kTinyLd + tj * 16 + l16;
        b[at] = s.b * a[at] + s.c * v[e];
      }
    }
    __syncthreads();
    // X: a strip of 16 columns, all rows; no one else reads or writes it
    for (int job = wave; job < nt; job += kTinyWaves) {
      const int c = job * 16 + l16;
      f32x4 acc[kTinyRows / 16] = {};
      for (int k = 0; k < mt * 16; k += 4) {
        const float v = x[(k + lk) * ld + c];
#pragma unroll
        for (int i = 0; i < kTinyRows / 16; ++i)
          if (i < mt) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[(i * 16 + l16) * kTinyLd + k + lk], v, acc[i], 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < kTinyRows / 16; ++i)
        if (i < mt) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float* at = x + (i * 16 + 4 * lk + e) * ld + c;
            *at = s.a * *at + acc[i][e];
          }
        }
    }
    __syncthreads();
  }
  for (int e = tid; e < all; e += kThreads) {
    const int r = e / cols, c = e - r * cols;
    const float v = x[m.turned ? c * ld + r : r * ld + c];
    if (m.g) {
      const bool on = kept8(m, static_cast<uint32_t>(e), static_cast<uint32_t>(all)) & 1;
      const float w = on ? (1.f - s.lr * s.decay) * static_cast<float>(static_cast<const S*>(m.w)[e]) - m.up * v : 0.f;
      static_cast<S*>(m.w_out)[e] = static_cast<S>(w);
    } else {
      static_cast<S*>(m.o)[r * m.o_rs + c * m.o_cs] = static_cast<S>(v);
    }
  }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

struct Plan {
  std::vector<Mat> mats;        // those of the staged path
  std::vector<Mat> tiny;
  int gram = kSmall, poly = kSmall, apply = kSmall;   // tiles
  int64_t blocks[kStages] = {};
  std::vector<int32_t> start[kStages];
  size_t table = 0, total = 0;
};

// The tile that takes the least modelled time for a stage over all matrices;
// tiles(m, edge) and steps(m) of each.
template <class F, class G>
int pick(int np, int kinds, const std::vector<Mat>& mats, F&& tiles, G&& steps) {
  int best = kSmall;
  double least = 1e300;
  for (int k = 0; k < kinds; ++k) {
    double n = 0., work = 0., most = 0.;
    for (const Mat& m : mats) {
      const double t = static_cast<double>(tiles(m, tile_m(np, k))), s = steps(m);
      n += t, work += t * s, most = std::max(most, s);
    }
    const double t = tile_time(np, k, n, work / n, most);
    if (t < least) least = t, best = k;
  }
  return best;
}

// Fills in sizes and workspace places (as offsets from `ws`).
pp_status make_plan(Plan* p, int32_t dtype, uint8_t* ws) {
  const int planes = dtype == PP_BF16 ? 1 : 2;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t r = at;
    at += (n + 255) / 256 * 256;
    return r;
  };
  std::vector<Mat> given;
  given.swap(p->mats);
  for (Mat& m : given) {
    m.turned = m.rows > m.cols;
    m.m = std::min(m.rows, m.cols), m.n = std::max(m.rows, m.cols);
    m.mp = static_cast<int32_t>(pad64(m.m)), m.np = static_cast<int32_t>(pad64(m.n));
    const int64_t all = static_cast<int64_t>(m.rows) * m.cols;
    auto piece = [&](const void* q, int64_t pitch) { return aligned16(q) && pitch % 8 == 0; };
    m.wide = m.g ? aligned16(m.g) && aligned16(m.w) && aligned16(m.w_out) && aligned16(m.mom) && aligned16(m.mom_out)
                 : piece(m.u, m.u_rs);
    m.o_wide = piece(m.o, m.o_rs);
    // (at most 1024, whose sums each workgroup of the next kernel adds up)
    m.chunk = static_cast<int32_t>(std::max<int64_t>(4096, cdiv(cdiv(all, 1024), 2048) * 2048));
    m.chunks = static_cast<int32_t>(cdiv(all, m.chunk));
    (tiny_fits(m.m, m.n) ? p->tiny : p->mats).push_back(m);
  }
  // long sums first, so that the longest tiles do not start last
  std::stable_sort(p->mats.begin(), p->mats.end(), [](const Mat& a, const Mat& b) { return a.n > b.n; });
  auto tri = [](const Mat& m, int t) { const int64_t k = cdiv(m.mp, t); return k * (k + 1) / 2; };   // (the padding is written too)
  auto rect = [](const Mat& m, int t) { return cdiv(m.np, t) * cdiv(m.m, t); };
  p->gram = pick(planes, kTiles, p->mats, tri, [](const Mat& m) { return m.np / 64; });
  p->poly = pick(planes, kTiles, p->mats, tri, [](const Mat& m) { return m.mp / 64; });
  p->apply = pick(planes, kFit, p->mats, rect, [](const Mat& m) { return m.mp / 64; });
  for (Mat& m : p->mats) {
    const int64_t n[kStages] = {m.chunks, static_cast<int64_t>(m.mp / 64) * (m.np / 64), tri(m, tile_m(planes, p->gram)),
                                tri(m, tile_m(planes, p->poly)), rect(m, tile_m(planes, p->apply))};
    for (int k = 0; k < kStages; ++k) {
      p->start[k].push_back(static_cast<int32_t>(p->blocks[k]));
      p->blocks[k] += n[k];
      if (p->blocks[k] > (1 << 22)) return fail(PP_EUNSUPPORTED, "too many matrices, or too large, for one call");
    }
    const size_t xn = static_cast<size_t>(m.m) * m.np * 2, an = static_cast<size_t>(m.m) * m.mp * 2;
    m.x[0] = reinterpret_cast<half_t*>(ws + take(2 * xn));
    m.x[1] = reinterpret_cast<half_t*>(ws + take(2 * xn));
    m.a = reinterpret_cast<half_t*>(ws + take(2 * an));
    m.b = reinterpret_cast<half_t*>(ws + take(2 * an));
    m.da = reinterpret_cast<float*>(ws + take(m.m * 4));
    m.db = reinterpret_cast<float*>(ws + take(m.m * 4));
    m.part = reinterpret_cast<double*>(ws + take(m.chunks * 8));
  }
  p->table = take(p->mats.size() * (sizeof(Mat) + kStages * 4));
  p->total = at;   // (0: small matrices need none)
  return PP_OK;
}

Spread spread_of(int64_t tiles) {
  return {static_cast<int32_t>(tiles), static_cast<int32_t>(std::min<int64_t>(32, cdiv(tiles, 8)))};
}
dim3 grid_of(const Spread& s) { return dim3(static_cast<uint32_t>(cdiv(s.total, 8 * s.chunk) * 8 * s.chunk)); }

template <int P, bool POLY>
void gram(const Plan& p, const Table& t, const Step& s, PlanePairs pairs, int turn, hipStream_t st) {
  const Spread sp = spread_of(p.blocks[POLY ? kStagePoly : kStageGram]);
  with_tile<half_t, false, false, P, P == 1>(POLY ? p.poly : p.gram, [&](auto k) {
    using Tile = decltype(k);
    hipLaunchKernelGGL((gram_kernel<Tile, P, POLY>), grid_of(sp), dim3(Tile::THREADS), 0, st, t, s, pairs, turn, sp);
  });
}

template <class S, int P, bool LAST>
void apply(const Plan& p, const Table& t, const Step& s, PlanePairs pairs, int turn, hipStream_t st) {
  const Spread sp = spread_of(p.blocks[kStageApply]);
  with_tile<half_t, true, false, P>(p.apply, [&](auto k) {
    using Tile = decltype(k);
    hipLaunchKernelGGL((apply_kernel<Tile, S, P, LAST>), grid_of(sp), dim3(Tile::THREADS), 0, st, t, s, pairs, turn, sp);
  });
}

template <class S, int P>
pp_status enqueue(const Plan& p, const Step& s, uint8_t* ws, hipStream_t st) {
  for (size_t first = 0; first < p.tiny.size(); first += kSetup) {
    Setup su = {};
    su.count = static_cast<int32_t>(std::min<size_t>(kSetup, p.tiny.size() - first));
    std::copy_n(p.tiny.begin() + first, su.count, su.mat);
    hipLaunchKernelGGL((tiny_kernel<S>), dim3(static_cast<uint32_t>(su.count)), dim3(kTinyWaves * 64), 0, st, su, s);
  }
  if (p.mats.empty()) return launched();
  Mat* mats = reinterpret_cast<Mat*>(ws + p.table);
  int32_t* start = reinterpret_cast<int32_t*>(mats + p.mats.size());
  const int all = static_cast<int>(p.mats.size());
  for (int first = 0; first < all && all > 1; first += kSetup) {
    Setup su;
    su.first = first, su.count = std::min(kSetup, all - first), su.all = all;
    for (int i = 0; i < su.count; ++i) {
      su.mat[i] = p.mats[first + i];
      for (int k = 0; k < kStages; ++k) su.start[k][i] = p.start[k][first + i];
    }
    hipLaunchKernelGGL(setup_kernel, dim3(1), dim3(256), 0, st, su, mats, start);
  }
  const Table t = {mats, start, all, p.mats[0]};
  hipLaunchKernelGGL((norm_kernel<S>), dim3(static_cast<uint32_t>(p.blocks[kStageNorm])), dim3(256), 0, st, t, s);
  hipLaunchKernelGGL((fill_kernel<S>), dim3(static_cast<uint32_t>(p.blocks[kStageFill])), dim3(256), 0, st, t, s);
  const PlanePairs pairs = P == 1 ? kPairs1 : kPairs3;
  for (int k = 0; k < s.steps; ++k) {
    gram<P, false>(p, t, s, pairs, k & 1, st);
    gram<P, true>(p, t, s, pairs, 0, st);
    if (k + 1 < s.steps)
      apply<S, P, false>(p, t, s, pairs, k & 1, st);
    else
      apply<S, P, true>(p, t, s, pairs, k & 1, st);
  }
  return launched();
}

// The coefficients have to keep singular values of 0..1 within 0..2 and the
// intermediate matrices within their stored range.
pp_status check_step(const Step& s) {
  if (s.steps < 1 || s.steps > 64) return fail(PP_EINVAL, "steps must be 1..64");
  for (float v : {s.a, s.b, s.c, s.eps, s.lr, s.momentum, s.decay})
    if (!std::isfinite(v)) return fail(PP_EINVAL, "parameters must be finite");
  if (s.eps < 0) return fail(PP_EINVAL, "eps must be >= 0");
  // Over t = x^2 in 0..r^2, r the largest |x| the steps before can give:
  // f(x) = x (a + b t + c t^2) is largest at an end or where a + 3 b t + 5 c t^2 = 0,
  // g(t) = b t + c t^2 at an end or at -b / 2c.
  const double a = s.a, b = s.b, c = s.c;
  double r = 1.;
  for (int k = 0; k < s.steps; ++k) {
    const double end = r * r;
    double most = 0., g = 0.;
    auto f = [&](double t) { if (t >= 0. && t <= end) most = std::max(most, std::sqrt(t) * std::fabs(a + b * t + c * t * t)); };
    auto h = [&](double t) { if (t >= 0. && t <= end) g = std::max(g, std::max(std::fabs(b * t + c * t * t), std::fabs(b * t))); };
    f(end), h(end);
    if (c != 0.) {
      const double d = 9. * b * b - 20. * a * c;
      if (d >= 0.) f((-3. * b + std::sqrt(d)) / (10. * c)), f((-3. * b - std::sqrt(d)) / (10. * c));
      h(-b / (2. * c));
    } else if (b != 0.) {
      f(-a / (3. * b));
    }
    if (!(most <= 2.)) return fail(PP_EUNSUPPORTED, "the coefficients let singular values leave 0..2");
    if (!(g <= 48.)) return fail(PP_EUNSUPPORTED, "coefficients too large");
    if (most <= r) break;   // (the range does not grow any more)
    r = most;
  }
  return PP_OK;
}

pp_status run(Plan* p, int32_t dtype, const Step& s, void* workspace, size_t ws_bytes, void* hip_stream) {
  if (p->mats.empty()) return PP_OK;
  const pp_status st = make_plan(p, dtype, static_cast<uint8_t*>(workspace));
  if (st != PP_OK) return st;
  if (p->total && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256))
    return fail(PP_EINVAL, "the workspace must be 256-byte aligned");
  if (ws_bytes < p->total) return fail(PP_ESIZE, "workspace smaller than needed");
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  return dtype == PP_BF16 ? enqueue<__bf16, 1>(*p, s, static_cast<uint8_t*>(workspace), stream)
                          : enqueue<float, 2>(*p, s, static_cast<uint8_t*>(workspace), stream);
}

pp_status check_size(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0) return fail(PP_EINVAL, "negative size");
  if (rows > (1 << 21) || cols > (1 << 21) || std::min(rows, cols) > 32768)
    return fail(PP_EUNSUPPORTED, "a matrix may have up to 2^21 rows or columns, and 32768 of the fewer");
  if (rows * cols >= (int64_t(1) << 31)) return fail(PP_EUNSUPPORTED, "a matrix must have fewer than 2^31 elements");
  return PP_OK;
}

template <class F>
pp_status guarded(F&& f) {
  clear_error();
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(PP_EINVAL, std::string("out of host memory: ") + e.what());
  }
}

pp_status collect(Plan* p, const pp_ortho_mat* mats, int32_t count, int32_t dtype, bool pointers) {
  if (count < 0 || (count && !mats)) return fail(PP_EINVAL, "mats is NULL");
  if (dtype != PP_F32 && dtype != PP_BF16) return fail(PP_EINVAL, "bad dtype");
  const size_t esz = dtype == PP_BF16 ? 2 : 4;
  for (int32_t i = 0; i < count; ++i) {
    const pp_ortho_mat& q = mats[i];
    const pp_status s = check_size(q.rows, q.cols);
    if (s != PP_OK) return s;
    if (q.rows == 0 || q.cols == 0) continue;
    if (pointers) {
      if (!q.u || !q.o) return fail(PP_EINVAL, "NULL pointer");
      if (reinterpret_cast<uintptr_t>(q.u) % esz || reinterpret_cast<uintptr_t>(q.o) % esz) return fail(PP_EINVAL, "misaligned pointer");
      if (q.u_rs < 0 || q.u_cs < 0 || q.o_rs < 0 || q.o_cs < 0) return fail(PP_EINVAL, "negative stride");
    }
    Mat m;
    std::memset(&m, 0, sizeof(m));
    m.u = q.u, m.u_rs = q.u_rs, m.u_cs = q.u_cs, m.o = q.o, m.o_rs = q.o_rs, m.o_cs = q.o_cs;
    m.rows = static_cast<int32_t>(q.rows), m.cols = static_cast<int32_t>(q.cols);
    p->mats.push_back(m);
  }
  return PP_OK;
}

pp_status collect(Plan* p, const pp_muon_layer* layers, int32_t count, int32_t dtype, bool pointers, float lr) {
  if (count < 0 || (count && !layers)) return fail(PP_EINVAL, "layers is NULL");
  if (dtype != PP_F32 && dtype != PP_BF16) return fail(PP_EINVAL, "bad dtype");
  const size_t esz = dtype == PP_BF16 ? 2 : 4;
  for (int32_t i = 0; i < count; ++i) {
    const pp_muon_layer& q = layers[i];
    const pp_status s = check_size(q.rows, q.cols);
    if (s != PP_OK) return s;
    if (q.keep && q.cols % 9) return fail(PP_EINVAL, "a pruned layer has 9 columns for each input channel");
    if (q.rows == 0 || q.cols == 0) continue;
    if (pointers) {
      if (!q.w || !q.g || !q.momentum || !q.w_out || !q.momentum_out) return fail(PP_EINVAL, "NULL pointer");
      for (const void* v : {q.w, q.g, static_cast<const void*>(q.w_out)})
        if (reinterpret_cast<uintptr_t>(v) % esz) return fail(PP_EINVAL, "misaligned pointer");
      for (const void* v : {static_cast<const void*>(q.momentum), static_cast<const void*>(q.momentum_out)})
        if (reinterpret_cast<uintptr_t>(v) % 4) return fail(PP_EINVAL, "misaligned momentum");
      if (reinterpret_cast<uintptr_t>(q.keep) % 2) return fail(PP_EINVAL, "misaligned keep");
    }
    Mat m;
    std::memset(&m, 0, sizeof(m));
    m.g = q.g, m.mom = q.momentum, m.w = q.w, m.w_out = q.w_out, m.mom_out = q.momentum_out, m.keep = q.keep;
    m.rows = static_cast<int32_t>(q.rows), m.cols = static_cast<int32_t>(q.cols);
    m.up = static_cast<float>(lr * std::sqrt(std::max(1., static_cast<double>(q.rows) / q.cols)));
    p->mats.push_back(m);
  }
  return PP_OK;
}

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" pp_status pp_ortho_workspace(const pp_ortho_mat* mats, int32_t count, int32_t dtype, size_t* bytes) {
  return guarded([&]() -> pp_status {
    if (!bytes) return fail(PP_EINVAL, "bytes is NULL");
    Plan p;
    pp_status s = collect(&p, mats, count, dtype, false);
    if (s == PP_OK) s = make_plan(&p, dtype, nullptr);
    if (s == PP_OK) *bytes = p.total;
    return s;
  });
}

extern "C" pp_status pp_ortho(const pp_ortho_mat* mats, int32_t count, int32_t dtype, int32_t steps, const float* coeffs,
                              float eps, void* workspace, size_t ws_bytes, void* hip_stream) {
  return guarded([&]() -> pp_status {
    if (!coeffs) return fail(PP_EINVAL, "coeffs is NULL");
    const Step s = {0.f, 0.f, 0.f, 0, coeffs[0], coeffs[1], coeffs[2], eps, steps};
    pp_status st = check_step(s);
    if (st != PP_OK) return st;
    Plan p;
    st = collect(&p, mats, count, dtype, true);
    return st == PP_OK ? run(&p, dtype, s, workspace, ws_bytes, hip_stream) : st;
  });
}

extern "C" pp_status pp_muon_workspace(const pp_muon_layer* layers, int32_t count, int32_t dtype, size_t* bytes) {
  return guarded([&]() -> pp_status {
    if (!bytes) return fail(PP_EINVAL, "bytes is NULL");
    Plan p;
    pp_status s = collect(&p, layers, count, dtype, false, 0.f);
    if (s == PP_OK) s = make_plan(&p, dtype, nullptr);
    if (s == PP_OK) *bytes = p.total;
    return s;
  });
}

extern "C" pp_status pp_muon_step(const pp_muon_layer* layers, int32_t count, int32_t dtype, const pp_muon_desc* desc,
                                  void* workspace, size_t ws_bytes, void* hip_stream) {
  return guarded([&]() -> pp_status {
    if (!desc) return fail(PP_EINVAL, "desc is NULL");
    const Step s = {desc->lr, desc->momentum, desc->weight_decay, desc->nesterov != 0, desc->coeffs[0], desc->coeffs[1],
                    desc->coeffs[2], desc->eps, desc->steps};
    pp_status st = check_step(s);
    if (st != PP_OK) return st;
    Plan p;
    st = collect(&p, layers, count, dtype, true, desc->lr);
    return st == PP_OK ? run(&p, dtype, s, workspace, ws_bytes, hip_stream) : st;
  });
}
