// xent.hip -- pp_xent_fwd / pp_xent_bwd / pp_xent_step: softmax cross entropy
// of a linear (1x1) head over a large number of classes, with its gradient,
// without keeping the logits where they are many.
//
//   l[t][v] = x[t] . w[v] + b[v],  lse[t] = log sum_v exp l[t][v]
//   loss[t] = c[y] (lse[t] - l[t][y]),            y = target[t]
//   G[t][v] = c[y] g[t] (exp(l[t][v] - lse[t]) - [v = y])
//   dx = a G w,  dw = a G^T x,  db = a sum_t G,  a = (incoming gradient) / divisor
//
// Forward: the logits are a product on the matrix cores whose tiles never
// leave the registers: each wave reduces its tile to a maximum and a sum of
// exponentials per token (a few bytes per token and 64 to 128 classes), and a
// second kernel joins those.  Backward: the logits are computed again (a step
// in fp32 may keep them), a piece of the classes at a time, turned into G in the epilogue (the logits
// themselves are not rounded), rounded to the operands' type and stored; then
// the two products, one over classes and one over tokens.  The piece bounds
// what the workspace holds.  (Few tokens: xent_few.hpp.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <type_traits>

#include "api_internal.hpp"
#include "gemm_tile.hpp"
#include "train.hpp"

namespace pp {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

struct Tokens {   // what the kernels know of the tokens
  const int64_t* target;
  const float* class_weight;   // or null
  const float* grad;           // or null: 1
  const float* stats;          // lse of each token, then the divisor
  int64_t ignore;
  int32_t t, v;                // tokens, classes
  int32_t grad_each;           // grad has one value a token
};

// What all tokens' gradients have in common: the incoming gradient of a single
// loss over the divisor.  It is left out of G and multiplied into the fp32
// sums: most of G's weight lies in the values near -1 at the targets, which
// 16 bits hold well and which a common factor would round all alike.
//
// G's other rounding is a choice too: with bf16 features it enters the products
// with w and x as one bf16 value, like those.  It errs by 2^-8 of each value at
// most, independently, as does the output's own rounding: gradients of 8 x 4096 pixels,
// 256 channels, 313 classes are off by 2.4e-3 of their norm, with G in fp32 by
// 1.7e-3.  A second value for the rest would make either product two (1.6 of the
// 3.0 ms of 8192 tokens, 1024 channels, 50000 classes are those).
__device__ __forceinline__ float common_scale(const Tokens& k) {
  return (k.grad && !k.grad_each ? k.grad[0] : 1.f) / k.stats[k.t];
}

// Token t's own factor of G, given its class weight and its incoming gradient:
// 0 where it is ignored, NaN where its target is outside the classes.
__device__ __forceinline__ float token_scale(const Tokens& k, int64_t y, float weight, float grad) {
  return y == k.ignore ? 0.f : y < 0 || y >= k.v ? __builtin_nanf("") : weight * grad;
}

// two parts of a sum of exponentials, each with its maximum
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float top = fmaxf(a.x, b.x), ref = top == -INFINITY ? 0.f : top;
  return make_float2(top, a.y * fast_exp(a.x - ref) + b.y * fast_exp(b.x - ref));
}

// Token t's log-sum-exp (0 if it is ignored), loss and weight.
__device__ __forceinline__ float token_loss(const Tokens& k, int t, float2 s, float target_logit, float* loss, float* weight) {
  const int64_t y = k.target[t];
  *loss = *weight = 0.f;
  if (y == k.ignore) return 0.f;
  // (the loss from the maximum and the sum's logarithm, not from their sum: that
  // is rounded to 2^-24 of itself, which may be more than the loss)
  const float rest = logf(s.y);
  if (y < 0 || y >= k.v) {
    *loss = *weight = __builtin_nanf("");
  } else {
    *weight = k.class_weight ? k.class_weight[y] : 1.f;
    *loss = *weight * (s.x - target_logit + rest);
  }
  return s.x + rest;
}

// ---------------------------------------------------------------------------
// operands: [rows][cols] of any strides -> 16-bit planes, columns contiguous and
// padded with zeros to a multiple of 64
// ---------------------------------------------------------------------------

struct StageArgs {
  const void* src;
  int64_t s_hi, s_lo, s_col;   // element (r, c) at (r / inner) s_hi + (r % inner) s_lo + c s_col
  int32_t inner, rows, cols;
  const int64_t* target;       // rows whose target is `ignore` become zeros (null: none)
  int64_t ignore;
  __bf16* out;                 // [rows][cols_pad] planes
  int64_t plane;               // elements between planes
  int32_t cols_pad;
  int32_t along_cols;          // columns lie closer in memory than rows
  int32_t wide;                // pieces of eight on that axis are contiguous and 16-byte aligned
};

// An fp32 value as a sum of three bf16 values: 8 bits of it each.
template <int P>
__device__ __forceinline__ void bf16_planes(float x, __bf16 (&p)[P]) {
  p[0] = static_cast<__bf16>(x);
  if constexpr (P > 1) {
    const float h = static_cast<float>(p[0]);
    const float rest = __builtin_isfinite(h) ? x - h : 0.f;   // (an infinity has no rest)
    p[1] = static_cast<__bf16>(rest);
    if constexpr (P > 2) p[2] = static_cast<__bf16>(rest - static_cast<float>(p[1]));
  }
}

// Two arrays in one launch: the second's tiles from workgroup `first` on.
// Bound by memory.  Eight images of 256 x 4096 in bf16 10 us, 3.5 TB/s; two in
// fp32, into three planes, 8 us, 2.7 TB/s.
template <class S, int P>
__global__ __launch_bounds__(256) void stage_kernel(StageArgs one, StageArgs two, int32_t first) {
  __shared__ float tile[64][65];
  __shared__ int32_t ignored[64];
  const bool second = static_cast<int>(blockIdx.x) >= first;
  const StageArgs& a = second ? two : one;
  const int id = second ? blockIdx.x - first : blockIdx.x;
  const int tc = a.cols_pad / 64;
  const int r0 = id / tc * 64, c0 = id % tc * 64, tid = threadIdx.x;
  const S* src = static_cast<const S*>(a.src);
  if (tid < 64) ignored[tid] = a.target && r0 + tid < a.rows && a.target[r0 + tid] == a.ignore;
  // a piece of eight values along the axis that is contiguous in memory
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int u = (tid >> 3) + 32 * i, w = (tid & 7) * 8;
    const int r = r0 + (a.along_cols ? u : w), c = c0 + (a.along_cols ? w : u);
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (r < a.rows && c < a.cols) {
      const int hi = r / a.inner;
      int lo = r - hi * a.inner;
      int64_t row = hi * a.s_hi + lo * a.s_lo;
      if (a.wide && (a.along_cols ? c : lo) + 8 <= (a.along_cols ? a.cols : a.inner)) {
        using S8 = __attribute__((ext_vector_type(8))) S;
        const S8 v = *reinterpret_cast<const S8*>(src + row + c * a.s_col);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = static_cast<float>(v[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (r + (a.along_cols ? 0 : e) < a.rows && c + (a.along_cols ? e : 0) < a.cols)
            x[e] = static_cast<float>(src[row + (c + (a.along_cols ? e : 0)) * a.s_col]);
          if (!a.along_cols) {
            row += a.s_lo;
            if (++lo == a.inner) lo = 0, row += a.s_hi - a.inner * a.s_lo;
          }
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (a.along_cols)
        tile[u][w + e] = x[e];
      else
        tile[w + e][u] = x[e];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int u = (tid >> 3) + 32 * i, w = (tid & 7) * 8;
    if (r0 + u >= a.rows) continue;
    const bool off = ignored[u];
    bf16x8 o[P];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      __bf16 p[P];
      bf16_planes<P>(off ? 0.f : tile[u][w + e], p);
#pragma unroll
      for (int q = 0; q < P; ++q) o[q][e] = p[q];
    }
#pragma unroll
    for (int q = 0; q < P; ++q)
      *reinterpret_cast<bf16x8*>(a.out + q * a.plane + static_cast<int64_t>(r0 + u) * a.cols_pad + c0 + w) = o[q];
  }
}

// The loss and its divisor (sums in 64 bits, in a fixed order), by a workgroup.
struct LossArgs {
  const double2* sums;   // of n workgroups of the join
  int32_t n, mean;
  float *out, *divisor;  // (out null: each token has its loss)
};
__device__ __forceinline__ void put_loss(const LossArgs& l, double x, double w) {
  // (a mean over no token: a loss of 0)
  const double div = l.mean && !(w == 0.) ? w : 1.;
  if (l.out) *l.out = static_cast<float>(x / div);
  *l.divisor = static_cast<float>(div);
}
__device__ __forceinline__ void loss_sum(const LossArgs& l, double2* wave_sums) {
  double x = 0., w = 0.;
#pragma unroll 4
  for (int i = threadIdx.x; i < l.n; i += blockDim.x) {
    const double2 s = l.sums[i];
    x += s.x, w += s.y;
  }
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d), w += __shfl_xor(w, d);
  if ((threadIdx.x & 63) == 0) wave_sums[threadIdx.x >> 6] = make_double2(x, w);
  __syncthreads();
  if (threadIdx.x) return;
  for (unsigned i = 1; i < blockDim.x / 64; ++i) x += wave_sums[i].x, w += wave_sums[i].y;
  put_loss(l, x, w);
}

// db: 64 classes a workgroup, each wave taking every n-th part
struct ClassSums {
  const float* part;   // [parts][n]
  int32_t parts, n;
  float* out;
};
__device__ __forceinline__ void class_sum(const ClassSums& a, const Tokens& k, int block, float* wave_sums) {
  const int u = threadIdx.x & 63, w = threadIdx.x >> 6, waves = blockDim.x / 64, v = block * 64 + u;
  float s = 0.f;
  if (v < a.n) {
#pragma unroll 4
    for (int p = w; p < a.parts; p += waves) s += a.part[static_cast<int64_t>(p) * a.n + v];
  }
  wave_sums[w * 64 + u] = s;
  __syncthreads();
  if (w || v >= a.n) return;
  for (int i = 1; i < waves; ++i) s += wave_sums[i * 64 + u];
  a.out[v] = s * common_scale(k);
}

// ---------------------------------------------------------------------------
// the logits' product, rows = classes [v0, v0 + A.rows), columns = tokens
// ---------------------------------------------------------------------------

struct LogitArgs {
  GemmOperand w, x;
  PlanePairs pairs;
  int32_t ksteps, tm, tn;
  int32_t v0;
  const float* bias;
  Tokens k;
  float* logits;           // [token][l_ld], without the bias: kept, or taken from there; or null
  int64_t l_ld;
  // statistics
  float2* part;            // [class part][token]: maximum, sum of exp(l - maximum)
  float* target_logit;     // [token]
  // gradient
  __bf16* g;               // [token][v_pad] planes
  int64_t g_plane;
  int32_t v_pad;
  float* db_part;          // [token part][w.rows], or null
  LossArgs loss;           // done by a workgroup past the tiles, if there is one
  // both at once
  float *lse_out, *each;   // each: every token's loss, or null
  double2* sums;           // [64 tokens]: sums of the losses and of the weights, or null
};

// the sum over a row of 16 lanes, in all of them
__device__ __forceinline__ float sum16(float v) {
  auto turned = [](float x, auto n) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x120 + decltype(n)::value, 0xF, 0xF, true));
  };
  v += turned(v, std::integral_constant<int, 8>());   // (row_ror)
  v += turned(v, std::integral_constant<int, 4>());
  v += turned(v, std::integral_constant<int, 2>());
  v += turned(v, std::integral_constant<int, 1>());
  return v;
}

// Bound by the products.  4096 tokens, 32768 classes, 1024 channels, bf16: 220 us,
// 1.25 PFLOP/s; G of 8192 tokens, 16384 classes: 290 us, 0.95 PFLOP/s, of which
// G's store through LDS takes 45.  Sums of a few steps are short of that: fp32,
// 8192 tokens, 313 classes, 256 channels, six products: 18 to 20 us, 0.4 PFLOP/s
// (G of kept logits: 11 us, 2.8 TB/s).  With all classes in a tile, bf16, 32768
// tokens, 313 classes, 256 channels: 29 us, where statistics, join and G took 43;
// that is neither the products' time (4 us) nor the bytes' (8), but a chain of
// fetches and joins with every workgroup resident.
// A tile with all classes of 64 tokens: 8 waves of 16 FM classes each, whose rows
// of w no other wave needs: they come from memory (most of them from the L2) into
// the lanes' registers, a step ahead, and only the tokens' features, all
// channels at once, are in LDS.  So it has no barrier in its loop, and two
// workgroups fit a CU.
constexpr int kAllTokens = 64, kAllClasses = 512, kAllChannels = 512;
template <int F>
struct AllTile : GemmTile<__bf16, 128 * F, kAllTokens, 8, 1, 2, 1, false, false, false, 1, 32> {
  using Base = GemmTile<__bf16, 128 * F, kAllTokens, 8, 1, 2, 1, false, false, false, 1, 32>;
  static constexpr uint32_t FEATURES = kAllTokens * (kAllChannels + 8) * 2;
  static constexpr uint32_t LDS_BYTES = FEATURES > Base::STAGING ? FEATURES : Base::STAGING;
  static __device__ __forceinline__ void run(const GemmOperand& w, const GemmOperand& x, PlanePairs, int row0, int col0, int ksteps, int,
                                             int, uint8_t* lds, f32x4 (&acc)[Base::FM][Base::FN]) {
    const int tid = threadIdx.x, r = tid & 15, g = tid >> 4 & 3, pitch = ksteps * 64 + 8;   // (16 bytes past a multiple of the banks)
    __bf16* xs = reinterpret_cast<__bf16*>(lds);
    const __bf16* rows[Base::FM];
#pragma unroll
    for (int i = 0; i < Base::FM; ++i) {   // (what is past the last class is not used)
      const int row = min(row0 + Base::wave() * Base::TM + 16 * i + r, w.rows - 1);
      rows[i] = static_cast<const __bf16*>(w.plane[0]) + row * w.ld + 8 * g;
    }
    bf16x8 cur[Base::FM], next[Base::FM];
#pragma unroll
    for (int i = 0; i < Base::FM; ++i) cur[i] = *reinterpret_cast<const bf16x8*>(rows[i]);
    {
      const int t = tid >> 3;
      const bool on = col0 + t < x.rows;
      const __bf16* from = static_cast<const __bf16*>(x.plane[0]) + (on ? col0 + t : 0) * x.ld + (tid & 7) * 8;
      __bf16* to = xs + t * pitch + (tid & 7) * 8;
#pragma unroll 4
      for (int n = 0; n < ksteps; ++n) {
        const bf16x8 v = *reinterpret_cast<const bf16x8*>(from + 64 * n);
        *reinterpret_cast<bf16x8*>(to + 64 * n) = on ? v : bf16x8{};
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < Base::FM; ++i)
#pragma unroll
      for (int j = 0; j < Base::FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int steps = ksteps * 2;
    for (int s = 0; s < steps; ++s) {
      const int ahead = min(s + 1, steps - 1) * 32;
#pragma unroll
      for (int i = 0; i < Base::FM; ++i) next[i] = *reinterpret_cast<const bf16x8*>(rows[i] + ahead);
      bf16x8 b[Base::FN];
#pragma unroll
      for (int j = 0; j < Base::FN; ++j) b[j] = *reinterpret_cast<const bf16x8*>(xs + (16 * j + r) * pitch + 32 * s + 8 * g);
#pragma unroll
      for (int i = 0; i < Base::FM; ++i)
#pragma unroll
        for (int j = 0; j < Base::FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cur[i], b[j], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < Base::FM; ++i) cur[i] = next[i];
    }
  }
};

// kKept: G again, of logits that the statistics' kernel kept, by the same tiles
// and so with the same sums.  kWhole: a tile has all classes, so the statistics,
// the loss and G (if there is room for it: g) are one kernel's work; kWholeGrad:
// G by such tiles, given the statistics.
enum { kStats = 0, kGrad = 1, kKept = 2, kWhole = 3, kWholeGrad = 4 };
template <class Tile, int MODE, int P>
__global__ __launch_bounds__(Tile::THREADS, MODE < kWhole ? 1 : Tile::FM < 4 ? 4 : 2) void logit_kernel(LogitArgs a) {
  constexpr bool GRAD = MODE != kStats, WHOLE = MODE == kWhole;
  __shared__ __align__(1024) uint8_t lds[MODE == kKept ? Tile::STAGING : Tile::LDS_BYTES];
  if (GRAD && !WHOLE && static_cast<int>(blockIdx.x) >= a.tm * a.tn) {
    loss_sum(a.loss, reinterpret_cast<double2*>(lds));
    return;
  }
  int ti, tj;
  band_order(xcd_order(blockIdx.x, a.tm * a.tn), a.tm, a.tn, &ti, &tj);
  const int row0 = ti * Tile::BM, col0 = tj * Tile::BN;
  const int lane = Tile::lane(), wave = Tile::wave();
  const int rows = a.w.rows, nt = a.k.t;

  // this lane's columns: their targets, and for the gradient the statistics,
  // fetched ahead of the product and used after it
  int64_t target[Tile::FN];
  float lse[Tile::FN], scale[Tile::FN];
  int hit[Tile::FN];   // the target's row, from this lane's first one on (-1: not in the wave's)
#pragma unroll
  for (int j = 0; j < Tile::FN; ++j) {
    const int t = min(col0 + Tile::col_of(j), nt - 1);
    target[j] = a.k.target[t];
    if constexpr (GRAD && !WHOLE) lse[j] = a.k.stats[t];
  }

  f32x4 acc[Tile::FM][Tile::FN];
  if constexpr (MODE == kKept) {
#pragma unroll
    for (int i = 0; i < Tile::FM; ++i)
#pragma unroll
      for (int j = 0; j < Tile::FN; ++j) {
        const int t = min(col0 + Tile::col_of(j), nt - 1), r = row0 + Tile::row_of(i);
        acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (Tile::group() == 0 && r < a.v_pad) acc[i][j] = *reinterpret_cast<const f32x4*>(a.logits + t * a.l_ld + a.v0 + r);
      }
  } else {
    Tile::run(a.w, a.x, a.pairs, row0, col0, a.ksteps, 0, Tile::steps_of(a.ksteps, a.pairs), lds, acc);
    Tile::reduce(lds, acc);
  }
  if constexpr (MODE == kStats && P > 1) {
    if (a.logits && Tile::group() == 0) {
#pragma unroll
      for (int i = 0; i < Tile::FM; ++i)
#pragma unroll
        for (int j = 0; j < Tile::FN; ++j) {
          const int t = col0 + Tile::col_of(j), r = row0 + Tile::row_of(i);
          if (t < nt && r < (rows + 63) / 64 * 64) *reinterpret_cast<f32x4*>(a.logits + t * a.l_ld + a.v0 + r) = acc[i][j];
        }
    }
  }

  // (everything that has to be fetched first, without branches between)
  f32x4 bias[Tile::FM];
  if (a.bias) {
    const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(a.bias) + a.v0, 0, rows * 4, 0x00020000);   // (0 past the end)
#pragma unroll
    for (int i = 0; i < Tile::FM; ++i)
      bias[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (row0 + Tile::row_of(i)) * 4, 0, 0));
  }
  if constexpr (GRAD) {
    float weight[Tile::FN], grad[Tile::FN];
#pragma unroll
    for (int j = 0; j < Tile::FN; ++j) weight[j] = grad[j] = 1.f;
    if (a.k.class_weight) {
#pragma unroll
      for (int j = 0; j < Tile::FN; ++j) {
        const int64_t y = target[j];
        weight[j] = a.k.class_weight[y < 0 || y >= a.k.v ? 0 : y];
      }
    }
    if (a.k.grad && a.k.grad_each) {
#pragma unroll
      for (int j = 0; j < Tile::FN; ++j) grad[j] = a.k.grad[min(col0 + Tile::col_of(j), nt - 1)];
    }
#pragma unroll
    for (int j = 0; j < Tile::FN; ++j)
      scale[j] = col0 + Tile::col_of(j) < nt ? token_scale(a.k, target[j], weight[j], grad[j]) : 0.f;
  }
#pragma unroll
  for (int j = 0; j < Tile::FN; ++j) {
    const int64_t c = target[j] - a.v0, d = c - (row0 + Tile::row_of(0));
    hit[j] = d >= 0 && d < Tile::TM && c < rows && col0 + Tile::col_of(j) < nt ? static_cast<int>(d) : -1;
  }
  // the logits: bias added; classes past the end take no part
  if (a.bias) {
#pragma unroll
    for (int i = 0; i < Tile::FM; ++i)
#pragma unroll
      for (int j = 0; j < Tile::FN; ++j) acc[i][j] += bias[i];
  }
  if (row0 + Tile::BM > rows) {
#pragma unroll
    for (int i = 0; i < Tile::FM; ++i) {
      const int r = row0 + Tile::row_of(i);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < Tile::FN; ++j) acc[i][j][e] = r + e < rows ? acc[i][j][e] : -INFINITY;
    }
  }
  // the wave's part of a column: maximum, and sum of the exponentials
  [[maybe_unused]] auto column = [](int j, const f32x4 (&acc)[Tile::FM][Tile::FN]) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < Tile::FM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[i][j][e]);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    // (a column with nothing above -inf: every term is exp(-inf); NaNs reach the sum)
    const float ref = m == -INFINITY ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < Tile::FM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s += fast_exp(acc[i][j][e] - ref);
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    return make_float2(m, s);
  };
  // The target's logit.  (A lane has the rows 16 i + 4 (lane / 16) + 0..3: of the
  // others' it finds none.)
  [[maybe_unused]] auto at_hit = [&hit](int j, const f32x4 (&acc)[Tile::FM][Tile::FN]) {
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < Tile::FM; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) l = hit[j] == 16 * i + e ? acc[i][j][e] : l;
    return l;
  };
  if constexpr (WHOLE) {
    struct Shared {
      float2 part[Tile::WM][Tile::BN];
      float target[Tile::BN], lse[Tile::BN];
    };
    static_assert(sizeof(Shared) <= Tile::LDS_BYTES && Tile::BN % 64 == 0 && Tile::BN <= Tile::THREADS && Tile::WK == 1);
    Shared& sh = *reinterpret_cast<Shared*>(lds);
    gemm_sync();   // (every wave is done with the operands)
#pragma unroll
    for (int j = 0; j < Tile::FN; ++j) {
      const float2 p = column(j, acc);
      if (lane < 16) sh.part[wave / Tile::WN][Tile::col_of(j)] = p;
      if (__ballot(hit[j] >= 0)) {
        const float l = at_hit(j, acc);
        if (hit[j] >= 0 && (hit[j] & 15) < 4) sh.target[Tile::col_of(j)] = l;
      }
    }
    __syncthreads();
    const int c = threadIdx.x, t = col0 + c;
    if (c < Tile::BN) {
      float l = 0.f, loss = 0.f, weight = 0.f;
      if (t < nt) {
        float2 s = sh.part[0][c];
#pragma unroll
        for (int w = 1; w < Tile::WM; ++w) s = join(s, sh.part[w][c]);
        l = token_loss(a.k, t, s, sh.target[c], &loss, &weight);
        a.lse_out[t] = l;
        if (a.each) a.each[t] = loss;
      }
      sh.lse[c] = l;
      if (a.sums) {
        double x = loss, y = weight;
#pragma unroll
        for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d), y += __shfl_xor(y, d);
        if (lane == 0) a.sums[tj * (Tile::BN / 64) + c / 64] = make_double2(x, y);
      }
    }
    if (!a.g) return;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < Tile::FN; ++j) lse[j] = sh.lse[Tile::col_of(j)];
  }
  if constexpr (!GRAD) {
    if (Tile::group() > 0) return;
#pragma unroll
    for (int j = 0; j < Tile::FN; ++j) {
      const int t = col0 + Tile::col_of(j);
      const float2 p = column(j, acc);
      if (t < nt && lane < 16) a.part[static_cast<int64_t>(ti * Tile::WM + wave / Tile::WN) * nt + t] = p;
      if (__ballot(hit[j] >= 0)) {   // (few tiles have a target's class)
        const float l = at_hit(j, acc);
        if (hit[j] >= 0 && (hit[j] & 15) < 4) a.target_logit[t] = l;
      }
    }
  } else {
    const bool mine = Tile::group() == 0;
#pragma unroll
    for (int j = 0; j < Tile::FN; ++j) {
      const bool on = mine && scale[j] != 0.f;   // (an ignored token, whatever its logits are)
#pragma unroll
      for (int i = 0; i < Tile::FM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = fast_exp(acc[i][j][e] - lse[j]) * scale[j];
          acc[i][j][e] = on ? p : 0.f;
        }
      if (__ballot(hit[j] >= 0)) {
        const float less = on ? scale[j] : 0.f;
#pragma unroll
        for (int i = 0; i < Tile::FM; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] -= hit[j] == 16 * i + e ? less : 0.f;
      }
    }
    if (a.db_part && mine) {
#pragma unroll
      for (int i = 0; i < Tile::FM; ++i) {
        const int r = row0 + Tile::row_of(i);
        f32x4 sum = acc[i][0];
#pragma unroll
        for (int j = 1; j < Tile::FN; ++j) sum += acc[i][j];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sum[e] = sum16(sum[e]);
          if ((lane & 15) == 0 && r + e < rows)
            a.db_part[static_cast<int64_t>(tj * Tile::WN + wave % Tile::WN) * rows + r + e] = sum[e];
        }
      }
    }
    auto store = [&](__bf16* to, int64_t plane, const float (&v)[8]) {
      bf16x8 o[P];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        __bf16 p[P];
        bf16_planes<P>(v[e], p);
#pragma unroll
        for (int q = 0; q < P; ++q) o[q][e] = p[q];
      }
#pragma unroll
      for (int q = 0; q < P; ++q) *reinterpret_cast<bf16x8*>(to + q * plane) = o[q];
    };
    Tile::staged(lds, acc, [&](int rb, int cb, typename Tile::View view) {
      rb += row0, cb += col0;
#pragma unroll 4
      for (int i = 0; i < view.pieces(); ++i) {
        int r, c;
        float v[8];
        view.col_piece(i, &r, &c);
        view.col(r, c, v);
        if (cb + c < nt && rb + r < a.v_pad) store(a.g + static_cast<int64_t>(cb + c) * a.v_pad + rb + r, a.g_plane, v);
      }
    });
  }
}

// ---------------------------------------------------------------------------
// joining the parts: each token's log-sum-exp and loss
// ---------------------------------------------------------------------------

struct JoinArgs {
  Tokens k;
  const float2* part;
  const float* target_logit;
  int32_t first, parts;   // the parts [first, parts)
  float2* carry;    // [token]: the joined part goes there, and nothing else is done (or null)
  float* lse;       // [token]
  float* loss;      // [token], or null
  double2* sums;    // [workgroup]: sums of the losses and of the weights, or null
  LossArgs whole;   // one workgroup: the loss and its divisor right away (divisor null: not)
};

// 256 / W tokens a workgroup, W threads each taking every W-th part.  Bound by
// latency: 4096 tokens with 256 parts 8 us, 32768 with 4 5 us.
template <int W>
__global__ __launch_bounds__(256) void join_kernel(JoinArgs a) {
  constexpr int N = 256 / W;
  __shared__ float2 got[W][N];
  const int u = threadIdx.x % N, w = threadIdx.x / N, t = blockIdx.x * N + u;
  float2 s = make_float2(-INFINITY, 0.f);
  if (t < a.k.t)
    for (int p = a.first + w; p < a.parts; p += W) s = join(s, a.part[static_cast<int64_t>(p) * a.k.t + t]);
  got[w][u] = s;
  __syncthreads();
  if (w) return;
  float loss = 0.f, weight = 0.f;
  if (t < a.k.t) {
#pragma unroll
    for (int p = 1; p < W; ++p) s = join(s, got[p][u]);
    if (a.carry) a.carry[t] = s;
  }
  if (a.carry) return;
  if (t < a.k.t) {
    const float lse = token_loss(a.k, t, s, a.target_logit[t], &loss, &weight);
    a.lse[t] = lse;
    if (a.loss) a.loss[t] = loss;
  }
  if (!a.sums && !a.whole.divisor) return;
  // (N lanes of one wave)
  double x = loss, y = weight;
#pragma unroll
  for (int d = N / 2; d; d >>= 1) x += __shfl_xor(x, d), y += __shfl_xor(y, d);
  if (u) return;
  if (a.whole.divisor)
    put_loss(a.whole, x, y);
  else
    a.sums[blockIdx.x] = make_double2(x, y);
}

__global__ __launch_bounds__(1024) void loss_kernel(LossArgs l) {
  __shared__ double2 wave_sums[16];
  loss_sum(l, wave_sums);
}

__global__ __launch_bounds__(1024) void class_sum_kernel(ClassSums a, Tokens k) {
  __shared__ float wave_sums[16 * 64];
  class_sum(a, k, blockIdx.x, wave_sums);
}

__global__ __launch_bounds__(256) void zero_kernel(uint8_t* p, int64_t bytes) {
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < bytes; i += gridDim.x * 256ll) p[i] = 0;
}

// ---------------------------------------------------------------------------
// the gradient's products: out[c][r] = sum_k A[r][k] B[c][k]
// ---------------------------------------------------------------------------

// Where element (r, c) of a product goes: rows or columns that are tokens lie
// at (t / inner) s_hi + (t % inner) s_lo.
struct OutMap {
  void* out;
  int64_t r_hi, r_lo, c_hi, c_lo;
  int32_t r_inner, c_inner;
  int32_t wide;   // four rows follow each other in memory, aligned
};

// Partial sums to be joined: [split][n][ld] -> the output.
struct Slab {
  float* at;
  int64_t ld;
  int32_t m, n, splits;
  OutMap map;
};

struct ProductArgs {
  GemmOperand a, b;
  PlanePairs pairs;
  int32_t m, n;   // the output's size
  int32_t ksteps, tm, tn, splits;
  OutMap map;
  float* slab;    // [split][n][slab_ld] partial sums instead of the output, or null
  int64_t slab_ld;
  int32_t add;    // the slab already holds a sum
  Tokens k;       // for the common factor
  // done by workgroups past the tiles: db's sums, and another product's slab
  ClassSums db;
  int32_t db_blocks;
  Slab join;
  int32_t join_blocks;
};

template <class O>
__device__ __forceinline__ void store4(const OutMap& m, int r, int c, int rows, f32x4 v) {
  const int ch = c / m.c_inner, cl = c - ch * m.c_inner;
  const int64_t at = ch * m.c_hi + cl * m.c_lo;
  O* out = static_cast<O*>(m.out);
  if (m.wide) {
    if (r < rows) {   // (rows is a multiple of four here)
      using O4 = __attribute__((ext_vector_type(4))) O;
      const int rh = r / m.r_inner, rl = r - rh * m.r_inner;
      *reinterpret_cast<O4*>(out + at + rh * m.r_hi + rl * m.r_lo) =
          O4{static_cast<O>(v[0]), static_cast<O>(v[1]), static_cast<O>(v[2]), static_cast<O>(v[3])};
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (r + e < rows) {
      const int rh = (r + e) / m.r_inner, rl = r + e - rh * m.r_inner;
      out[at + rh * m.r_hi + rl * m.r_lo] = static_cast<O>(v[e]);
    }
}

template <class O>
__device__ __forceinline__ void join_slab(const Slab& j, const Tokens& k, int block, int blocks) {
  const float scale = common_scale(k);
  const int64_t n4 = j.ld / 4, all = n4 * j.n, step = static_cast<int64_t>(blocks) * blockDim.x;
  for (int64_t i = static_cast<int64_t>(block) * blockDim.x + threadIdx.x; i < all; i += step) {
    const int c = static_cast<int>(i / n4), r = static_cast<int>(i - c * n4) * 4;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int q = 0; q < j.splits; ++q)
      s += *reinterpret_cast<const f32x4*>(j.at + (static_cast<int64_t>(q) * j.n + c) * j.ld + r);
    store4<O>(j.map, r, c, j.m, s * scale);
  }
}

// Bound by the products, and by the transposing reads of operands that are
// stored by rows of k.  8192 tokens, 16384 classes, 1024 channels, bf16, dx or
// dw: 264 us, 1.04 PFLOP/s.  Few tiles are split over k (dx of few channels:
// its sum is over all classes), and the parts added by slab_kernel or by
// workgroups past the next product's tiles.
template <class Tile, class O>
__global__ __launch_bounds__(Tile::THREADS) void product_kernel(ProductArgs a) {
  __shared__ __align__(1024) uint8_t lds[Tile::LDS_BYTES];
  const int tiles = a.tm * a.tn;
  const int past = static_cast<int>(blockIdx.x) - tiles * a.splits;
  if (past >= 0) {
    if (past < a.db_blocks)
      class_sum(a.db, a.k, past, reinterpret_cast<float*>(lds));
    else
      join_slab<O>(a.join, a.k, past - a.db_blocks, a.join_blocks);
    return;
  }
  const int id = xcd_order(blockIdx.x, tiles * a.splits);
  const int split = id / tiles;
  int ti, tj;
  band_order(id - split * tiles, a.tm, a.tn, &ti, &tj);
  const int row0 = ti * Tile::BM, col0 = tj * Tile::BN;
  const int steps = Tile::steps_of(a.ksteps, a.pairs);
  const int s0 = static_cast<int>(static_cast<int64_t>(steps) * split / a.splits);
  const int s1 = static_cast<int>(static_cast<int64_t>(steps) * (split + 1) / a.splits);
  const float scale = a.slab ? 1.f : common_scale(a.k);
  f32x4 acc[Tile::FM][Tile::FN];
  Tile::run(a.a, a.b, a.pairs, row0, col0, a.ksteps, s0, s1, lds, acc);
  Tile::staged(lds, acc, [&](int rb, int cb, typename Tile::View view) {
    rb += row0, cb += col0;
#pragma unroll 4
    for (int i = 0; i < view.pieces(); ++i) {
      int r, c;
      float v[8];
      view.col_piece(i, &r, &c);
      view.col(r, c, v);
      r += rb, c += cb;
      if (c >= a.n) continue;
      if (a.slab) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (r + 4 * h < a.slab_ld) {   // (a multiple of four)
            f32x4* at = reinterpret_cast<f32x4*>(a.slab + (static_cast<int64_t>(split) * a.n + c) * a.slab_ld + r + 4 * h);
            const f32x4 x = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
            *at = a.add ? *at + x : x;
          }
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          store4<O>(a.map, r + 4 * h, c, a.m, f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]} * scale);
      }
    }
  });
}

// (bound by memory: dx of 8192 tokens, 1024 channels, two parts: 14 us, 6 TB/s
// with what the caches hold)
template <class O>
__global__ __launch_bounds__(256) void slab_kernel(Slab j, Tokens k) {
  join_slab<O>(j, k, blockIdx.x, gridDim.x);
}

#include "xent_few.hpp"

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

struct Plan {
  int64_t t = 0, d = 0, v = 0, dp = 0, vp = 0;   // sizes and their paddings
  int planes = 1;
  PlanePairs pairs = kPairs1;
  bool w_direct = false, x_direct = false, fwd = false, bwd = false;
  int logit = kSmall, parts = 0;      // of a forward piece
  int64_t fwd_piece = 0;              // classes of one
  int64_t piece = 0, pieces = 0;      // classes a piece
  struct Piece {
    int logit = kSmall, dx = kSmall;  // tiles
    SplitTile dw = {kSmall, 1};
  } of[2];                            // the pieces, and the last one, which may be smaller
  int dx_splits = 1;
  bool dx_slab = false;
  int all = 0;                        // tiles with all classes: their 128s (else 0)
  bool keep = false;                  // the logits are kept for the gradient
  int64_t dx_ld = 0, dw_ld = 0;       // slab pitches: the product's rows rounded up to four
  bool dx_turned = false;             // dx's product has the tokens as rows
  bool few = false, few_odd = false;  // few tokens: kernels of their own
  int few_classes = 128, few_lane = 4, few_splits = 1;   // classes a workgroup; of the gradient: channels a lane, parts of the classes
  // workspace offsets
  size_t x_k = 0, w_k = 0, logits = 0, part = 0, tl = 0, sums = 0, g = 0, db = 0, slab = 0, total = 0;
};

constexpr int64_t kPartBytes = int64_t(64) << 20;     // of the forward pass's statistics
constexpr int64_t kPieceBytes = int64_t(512) << 20;   // of G

// Modelled time of the gradient's products for nv classes.
double piece_time(const Plan& p, int64_t nv, bool turned) {
  const int64_t steps = p.dp / 64;
  const int k = pick_tile(p.planes, nv, p.t, steps);
  const double tiles = static_cast<double>(cdiv(nv, tile_m(p.planes, k)) * cdiv(p.t, tile_n(p.planes, k))), s = static_cast<double>(steps);
  // (G's epilogue: about 10 us a round of large tiles)
  double t = tile_time(p.planes, k, tiles, s, s) + (k == kBig ? 10. * static_cast<double>(cdiv(static_cast<int64_t>(tiles), kCUs)) : 0.);
  double x;
  pick_split(p.planes, turned ? p.t : p.d, turned ? p.d : p.t, cdiv(nv, 64), &x);
  t += x;
  pick_split(p.planes, p.d, nv, cdiv(p.t, 64), &x);
  return t + x;
}

// Classes a piece: all, if G fits the workspace; else the size, among a few
// that fit, whose tiles waste the least of their last rounds.
int64_t pick_piece(const Plan& p, bool turned) {
  const int64_t most = std::max<int64_t>(256, kPieceBytes / (p.t * 2 * p.planes) / 256 * 256);
  if (p.vp <= most) return p.vp;
  int64_t best = most;
  double least = 1e300;
  auto look = [&](int64_t piece) {
    if (piece < 256 || piece > most) return;
    const int64_t n = p.v / piece, rest = p.v - n * piece;
    const double t = n * piece_time(p, piece, turned) + (rest ? piece_time(p, rest, turned) : 0.);
    if (t < least) least = t, best = piece;
  };
  const int64_t few = cdiv(p.v, most);
  for (int64_t n = few; n < few + 6; ++n) look(cdiv(cdiv(p.v, n), 256) * 256);
  for (int64_t n = most / 2048 * 2048, i = 0; n > 0 && i < 12; n -= 2048, ++i) look(n);
  return best;
}

Plan make_plan(const pp_xent_desc& d, bool fwd, bool bwd, bool dw, bool x_aligned, bool w_aligned, bool w_words) {
  Plan p;
  p.fwd = fwd, p.bwd = bwd;
  p.t = d.n * d.hw, p.d = d.d, p.v = d.v;
  p.dp = pad64(p.d), p.vp = pad64(p.v);
  const bool bf16 = d.dtype == PP_BF16;
  p.planes = bf16 ? 1 : 3;
  p.pairs = bf16 ? kPairs1 : kPairs6;
  const int64_t step = d.hw == 1 ? d.x_sn : d.x_sp;
  // (dw's product reads every token's features: ignored ones are copied as zeros)
  p.x_direct = !dw && bf16 && x_aligned && d.x_sc == 1 && p.d % 64 == 0 && step % 8 == 0 && step >= p.d && step <= kMaxLd &&
               (d.n == 1 || d.hw == 1 || d.x_sn == d.hw * d.x_sp);
  p.w_direct = bf16 && w_aligned && p.d % 64 == 0 && d.w_ld % 8 == 0 && d.w_ld <= kMaxLd;
  size_t at = 0;
  auto take = [&at](size_t n) {
    const size_t r = at;
    at += (n + 255) / 256 * 256;
    return r;
  };
  // Few tokens: where reading w is the work.  1024 channels, 50000 classes, step:
  // fp32 1, 64, 128 tokens 125, 225, 420 us, by the products 438, 458, 646; bf16
  // 1, 64 tokens 72, 105, by the products 146, 154.  With few classes a token the
  // workgroups are too few, and the two ways meet at about 192 (step, us, here and
  // by the products; 96, 192, 384 classes a token):
  //   bf16 64 tokens, 256 channels      40, 46   47, 45   49, 55
  //   bf16 64 tokens, 1024 channels     59, 49   64, 61   71, 88
  //   bf16 64 tokens, 2048 channels     74, 62   84, 82   105, 126
  //   fp32 64 tokens, 256 channels      53, 49   61, 65   70, 89
  //   fp32 64 tokens, 1024 channels     91, 76   105, 105 134, 183
  //   fp32 64 tokens, 2048 channels     135, 111 163, 180 223, 377
  //   fp32 128 tokens, 256 channels     92, 71   110, 107 152, 166
  //   fp32 128 tokens, 1024 channels    185, 126 251, 240 417, 491
  // Up to 16 tokens the kernels here are ahead from 24 classes a token on (bf16 35
  // us, 42 to 46; fp32, 2048 channels, 96 a token 50, 62), so the rule gives up to
  // 12 us away there; the forward pass alone of 64 bf16 tokens with 2048 channels
  // loses by it up to 384 a token (42, 27 at 192; 42, 42).  Rows of w too far apart for the kernels' descriptors
  // (32 rows, 32-bit offsets) are left to the products, which copy them.
  p.few = p.t <= kFewTokens[bf16] && p.v >= 192 * p.t && p.d >= 8 && p.t * p.vp * 4 <= kPieceBytes && d.w_ld <= kMaxLd;
  if (p.few) {
    p.few_lane = p.t <= 64 ? 4 : 2;
    // 64 a workgroup where that leaves CUs without one (1 token, 2048 channels,
    // 8000 classes, fp32: 33 us, with 128 39; 500 channels, 20000 classes: 22, 19)
    p.few_classes = (!bf16 && p.t > 16) || p.v > 64 * kCUs ? 128 : 64;
    if (!bf16 && p.t > 16) p.x_k = take(3 * p.t * p.dp * 2);
    p.few_odd = bf16 && (!w_words || p.d % 2 || d.w_ld % 2);
    if (fwd) {
      p.parts = static_cast<int>(cdiv(p.v, p.few_classes));
      p.part = take((p.parts + 1) * p.t * 8), p.tl = take(p.t * 4), p.sums = take(cdiv(p.t, 16) * 16);
    }
    if (bwd) {
      // two workgroups a CU, 32 classes at least
      p.few_splits = static_cast<int>(std::max<int64_t>(1, std::min(cdiv(p.v, 32), 2 * kCUs / cdiv(p.d, 64 * p.few_lane))));
      p.dx_ld = cdiv(p.d, 4) * 4;
      p.g = take(p.t * p.vp * 4), p.slab = take(p.few_splits * p.t * p.dx_ld * 4);
    }
    p.total = std::max<size_t>(at, 256);
    return p;
  }
  // Few classes: a tile that has them all, whose logits are computed once and
  // joined where they are.  8 x 4096 pixels, 256 channels, 313 classes: step 71 us,
  // 81 with the logits twice.  A tile's time grows with channels and classes, and
  // few tokens leave CUs idle that the products use (step of token rows, us, here
  // and by the products; 512, 1024, 3000, 8192 tokens):
  //   130 classes, 128 channels   38, 41   38, 41   38, 41   38, 41
  //   313 classes, 256 channels   38, 41   39, 42   46, 43   44, 49
  //   313 classes, 512 channels   40, 42   43, 42   53, 49   55, 59
  //   500 classes, 256 channels   39, 42   41, 42   51, 45   51, 52
  //   500 classes, 512 channels   45, 42   49, 42   61, 51   65, 64
  // (below 512 tokens 0 to 3 us either way.)  So it loses up to a fifth in a part
  // of its range, many classes and channels of some thousand tokens.
  if (bf16 && p.t >= 512 && p.v <= kAllClasses && p.dp <= kAllChannels && (!bwd || p.t * p.vp * 2 <= kPieceBytes))
    p.all = static_cast<int>(cdiv(p.v, 128));
  const size_t e = 2 * p.planes;
  if (!p.x_direct) p.x_k = take(p.t * p.dp * e);
  if (!p.w_direct) p.w_k = take(p.v * p.dp * e);
  if (fwd && p.all) {
    p.sums = take(cdiv(p.t, 64) * 16);
  } else if (fwd) {
    p.logit = pick_tile(p.planes, p.v, p.t, p.dp / 64);
    const int64_t edge = tile_m(p.planes, p.logit), wm = tile_wm(p.planes, p.logit);
    p.fwd_piece = std::min(p.vp, std::max<int64_t>(256, kPartBytes / (p.t * 8) / wm * edge / 256 * 256));
    p.parts = static_cast<int>(cdiv(p.fwd_piece, edge) * wm);
    p.part = take((p.parts + 1) * p.t * 8);   // (and what the pieces before left)
    p.tl = take(p.t * 4), p.sums = take(cdiv(p.t, 16) * 16);
  }
  if (bwd) {
    p.piece = p.all ? p.vp : pick_piece(p, d.dx_sc != 1);
    p.pieces = cdiv(p.v, p.piece);
    p.g = take(p.t * p.piece * e);
    // A step in fp32 keeps its logits, where G fits one piece and six products
    // cost more than a store and a load: 4096 tokens, 5000 classes, 64, 128, 256
    // channels 159, 190, 256 us, computed twice 146, 190, 291; 512 tokens, 1024
    // channels, 50000 classes 1055, 1265.  (bf16: 23 us for G of the products,
    // about as many for the store and the load.)
    p.keep = fwd && !bf16 && p.dp >= 192 && p.pieces == 1 && p.t * p.vp * 4 <= kPieceBytes;
    if (p.keep) p.logits = take(p.t * p.vp * 4);
    p.dx_turned = d.dx_sc != 1;
    const int64_t dm = p.dx_turned ? p.t : p.d, dn = p.dx_turned ? p.d : p.t;
    p.dx_ld = cdiv(dm, 4) * 4;
    p.dw_ld = cdiv(p.d, 4) * 4;
    int64_t db = 0, dw_slab = 0;
    for (int i = 0; i < 2; ++i) {
      const int64_t nv = i ? p.v - (p.pieces - 1) * p.piece : std::min(p.piece, p.v);
      Plan::Piece& q = p.of[i];
      q.logit = pick_tile(p.planes, nv, p.t, p.dp / 64);
      db = std::max(db, (p.all ? cdiv(p.t, kAllTokens) : cdiv(p.t, tile_n(p.planes, q.logit)) * tile_wn(p.planes, q.logit)) * nv * 4);
      const SplitTile x = pick_split(p.planes, dm, dn, cdiv(nv, 64));
      q.dx = x.tile;
      if (i == 0) p.dx_splits = x.splits;   // (dx's partial sums are kept over the pieces)
      q.dw = pick_split(p.planes, p.d, nv, cdiv(p.t, 64));
      if (q.dw.splits > 1) dw_slab = std::max(dw_slab, q.dw.splits * p.dw_ld * nv * 4);
    }
    p.dx_slab = p.dx_splits > 1 || p.pieces > 1;
    p.db = take(db);
    p.slab = take((p.dx_slab ? p.dx_splits * p.dx_ld * dn * 4 : 0) + dw_slab);
  }
  p.total = std::max<size_t>(at, 256);
  return p;
}

template <class S, int P>
void stage(const StageArgs* a, int n, hipStream_t st) {
  int64_t blocks[2] = {0, 0};
  for (int i = 0; i < n; ++i) blocks[i] = cdiv(a[i].rows, 64) * (a[i].cols_pad / 64);
  hipLaunchKernelGGL((stage_kernel<S, P>), dim3(static_cast<uint32_t>(blocks[0] + blocks[1])), dim3(256), 0, st, a[0], a[n - 1],
                     static_cast<int32_t>(blocks[0]));
}

template <int MODE, int P>
void logits(int tile, LogitArgs& a, hipStream_t st) {
  a.tm = static_cast<int32_t>(cdiv(pad64(a.w.rows), tile_m(P, tile)));   // (G's padding is written too)
  a.tn = static_cast<int32_t>(cdiv(a.x.rows, tile_n(P, tile)));
  with_tile<__bf16, false, false, P>(tile, [&](auto t) {
    using Tile = decltype(t);
    hipLaunchKernelGGL((logit_kernel<Tile, MODE, P>), dim3(static_cast<uint32_t>(a.tm * a.tn + (a.loss.divisor ? 1 : 0))),
                       dim3(Tile::THREADS), 0, st, a);
  });
}

// f128: classes in units of 128
template <int MODE>
void whole(int f128, LogitArgs& a, hipStream_t st) {
  a.tm = 1, a.tn = static_cast<int32_t>(cdiv(a.x.rows, kAllTokens));
  auto run = [&](auto t) {
    using Tile = decltype(t);
    hipLaunchKernelGGL((logit_kernel<Tile, MODE, 1>), dim3(static_cast<uint32_t>(a.tn)), dim3(Tile::THREADS), 0, st, a);
  };
  if (f128 == 1)
    run(AllTile<1>());
  else if (f128 == 2)
    run(AllTile<2>());
  else if (f128 == 3)
    run(AllTile<3>());
  else
    run(AllTile<4>());
}

template <class O, bool AR, bool BR>
void product(int tile, ProductArgs& a, hipStream_t st) {
  constexpr int P = std::is_same_v<O, float> ? 3 : 1;
  a.tm = static_cast<int32_t>(cdiv(a.m, tile_m(P, tile)));
  a.tn = static_cast<int32_t>(cdiv(a.n, tile_n(P, tile)));
  with_tile<__bf16, AR, BR, P>(tile, [&](auto t) {
    using Tile = decltype(t);
    hipLaunchKernelGGL((product_kernel<Tile, O>), dim3(static_cast<uint32_t>(a.tm * a.tn * a.splits + a.db_blocks + a.join_blocks)),
                       dim3(Tile::THREADS), 0, st, a);
  });
}

Slab slab_of(const ProductArgs& a) { return {a.slab, a.slab_ld, a.m, a.n, a.splits, a.map}; }

template <class O>
void launch_slab(const Slab& j, const Tokens& k, hipStream_t st) {
  const uint32_t grid = static_cast<uint32_t>(std::min<int64_t>(cdiv(j.ld / 4 * j.n, 256), 4096));
  hipLaunchKernelGGL((slab_kernel<O>), dim3(grid), dim3(256), 0, st, j, k);
}

// tokens a workgroup of the join (few parts: more)
int join_tokens(const Plan& p) { return p.parts > 8 ? 16 : 64; }

struct Call {
  const pp_xent_desc* d;
  const void *x, *w;
  const float *bias, *class_weight;
  const int64_t* target;
  float *loss, *stats;
  const float* grad;
  void *dx, *dw;
  float* db;
  uint8_t* ws;
  hipStream_t st;
};

Tokens tokens_of(const Plan& p, const Call& c) {
  return {c.target, c.class_weight, c.grad, c.stats, c.d->ignore_index, static_cast<int32_t>(p.t), static_cast<int32_t>(p.v),
          c.d->reduction == PP_NONE};
}

void launch_join(const Plan& p, const JoinArgs& a, hipStream_t st) {
  const uint32_t n = static_cast<uint32_t>(join_tokens(p));
  const dim3 grid((static_cast<uint32_t>(p.t) + n - 1) / n);
  if (n == 16)
    hipLaunchKernelGGL((join_kernel<16>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((join_kernel<4>), grid, dim3(256), 0, st, a);
}

StageArgs stage_x(const Plan& p, const Call& c) {
  const pp_xent_desc& d = *c.d;
  const int64_t step = d.hw == 1 ? d.x_sn : d.x_sp;
  StageArgs a = {c.x, d.x_sn, d.x_sp, d.x_sc, static_cast<int32_t>(d.hw), static_cast<int32_t>(p.t), static_cast<int32_t>(p.d),
                 c.target, d.ignore_index, reinterpret_cast<__bf16*>(c.ws + p.x_k), p.t * p.dp, static_cast<int32_t>(p.dp)};
  a.along_cols = d.x_sc <= step;
  a.wide = aligned16(c.x) && (a.along_cols ? d.x_sc == 1 && step % 8 == 0 && (d.hw == 1 || d.x_sn % 8 == 0)
                                           : d.x_sp == 1 && d.hw % 8 == 0 && d.x_sc % 8 == 0 && d.x_sn % 8 == 0);
  return a;
}

template <class S, int NT, bool ODD>
pp_status enqueue_few(const Plan& p, const Call& c) {
  const pp_xent_desc& d = *c.d;
  constexpr int64_t N = 16 / sizeof(S);
  constexpr int C = NT > 4 ? 2 : 4;
  auto f32 = [&](size_t off) { return reinterpret_cast<float*>(c.ws + off); };
  const int64_t step = d.hw == 1 ? d.x_sn : d.x_sp;
  FewArgs a = {};
  a.w = c.w, a.w_ld = d.w_ld, a.x = c.x, a.x_sn = d.x_sn, a.x_sp = d.x_sp, a.x_sc = d.x_sc;
  a.hw = static_cast<int32_t>(d.hw), a.d = static_cast<int32_t>(d.d), a.k = tokens_of(p, c), a.bias = c.bias;
  a.x_wide = aligned16(c.x) && d.x_sc == 1 && step % N == 0 && (d.hw == 1 || d.x_sn % N == 0);
  if (p.bwd) a.logits = f32(p.g), a.l_ld = p.vp;
  if (p.fwd) a.part = reinterpret_cast<float2*>(c.ws + p.part) + p.t, a.target_logit = f32(p.tl);
  const dim3 blocks(static_cast<uint32_t>(cdiv(p.v, p.few_classes)));
  if constexpr (sizeof(S) == 4 && NT > 1) {
    const StageArgs sa = stage_x(p, c);
    stage<S, 3>(&sa, 1, c.st);
    FewArgs b = a;
    b.x = sa.out, b.x_sn = p.dp, b.x_sp = sa.plane;
    hipLaunchKernelGGL((few_logit3_kernel<NT>), blocks, dim3(256), 0, c.st, b);
  } else {
    hipLaunchKernelGGL((few_logit_kernel<S, NT, ODD>), blocks, dim3(static_cast<uint32_t>(4 * p.few_classes)), 0, c.st, a);
  }
  if (p.fwd) {
    const bool each = d.reduction == PP_NONE;
    double2* sums = each ? nullptr : reinterpret_cast<double2*>(c.ws + p.sums);
    const int32_t grid = static_cast<int32_t>(cdiv(p.t, join_tokens(p)));
    const LossArgs loss = {sums, each ? 0 : grid, d.reduction == PP_MEAN, each ? nullptr : c.loss, c.stats + p.t};
    const JoinArgs ja = {a.k, reinterpret_cast<float2*>(c.ws + p.part), a.target_logit, 1, p.parts + 1, nullptr, c.stats,
                         each ? c.loss : nullptr, sums, grid == 1 ? loss : LossArgs{}};
    launch_join(p, ja, c.st);
    if (grid > 1) hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(1024), 0, c.st, loss);
  }
  if (!p.bwd) return launched();
  a.dw = c.dw, a.db = c.db;
  a.slab = c.dx ? f32(p.slab) : nullptr, a.slab_ld = p.dx_ld;
  a.splits = p.few_splits, a.groups = static_cast<int32_t>(cdiv(p.d, 64 * C));
  hipLaunchKernelGGL((few_grad_kernel<S, NT, C, ODD>), dim3(static_cast<uint32_t>(a.splits * a.groups)), dim3(256), 0, c.st, a);
  if (c.dx) {
    const Slab s = {a.slab, p.dx_ld, a.d, static_cast<int32_t>(p.t), a.splits,
                    {c.dx, d.dx_sc, 0, d.dx_sn, d.dx_sp, 1, a.hw,
                     d.dx_sc == 1 && reinterpret_cast<uintptr_t>(c.dx) % 16 == 0 && p.d % 4 == 0 && d.dx_sn % 4 == 0 &&
                         (d.hw == 1 || d.dx_sp % 4 == 0)}};
    hipLaunchKernelGGL((few_sum_kernel<S>), dim3(static_cast<uint32_t>(cdiv(p.dx_ld / 4 * p.t, 16))), dim3(256), 0, c.st, s, a.k);
  }
  return launched();
}

template <class S>
pp_status enqueue_few(const Plan& p, const Call& c) {
  auto run = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    if constexpr (sizeof(S) == 2) {
      if (p.few_odd) return enqueue_few<S, NT, true>(p, c);
    }
    return enqueue_few<S, NT, false>(p, c);
  };
  if (p.t <= 16) return run(std::integral_constant<int, 1>());
  if (p.t <= 32) return run(std::integral_constant<int, 2>());
  if (p.t <= 48) return run(std::integral_constant<int, 3>());
  if constexpr (sizeof(S) == 4) {
    if (p.t > 96) return run(std::integral_constant<int, 8>());
    if (p.t > 64) return run(std::integral_constant<int, 6>());
  }
  return run(std::integral_constant<int, 4>());
}

template <class S, int P>
pp_status enqueue(const Plan& p, const Call& c) {
  if (p.few) return enqueue_few<S>(p, c);
  const pp_xent_desc& d = *c.d;
  hipStream_t st = c.st;
  pp_status s;
  const Tokens tok = tokens_of(p, c);
  auto bf = [&](size_t off) { return reinterpret_cast<__bf16*>(c.ws + off); };
  auto f32 = [&](size_t off) { return reinterpret_cast<float*>(c.ws + off); };

  // operands: token rows and class rows, channels contiguous
  const int64_t step = d.hw == 1 ? d.x_sn : d.x_sp;
  const GemmOperand x = p.x_direct ? operand(c.x, 0, step, p.t, p.dp, 1) : operand(bf(p.x_k), p.t * p.dp, p.dp, p.t, p.dp, P);
  const GemmOperand w = p.w_direct ? operand(c.w, 0, d.w_ld, p.v, p.dp, 1) : operand(bf(p.w_k), p.v * p.dp, p.dp, p.v, p.dp, P);
  StageArgs staged[2];
  int copies = 0;
  if (!p.x_direct) staged[copies++] = stage_x(p, c);
  if (!p.w_direct) {
    StageArgs a = {c.w, d.w_ld, 0, 1, 1, static_cast<int32_t>(p.v), static_cast<int32_t>(p.d), nullptr, 0,
                   bf(p.w_k), p.v * p.dp, static_cast<int32_t>(p.dp)};
    a.along_cols = 1;
    a.wide = aligned16(c.w) && d.w_ld % 8 == 0;
    staged[copies++] = a;
  }
  if (copies) stage<S, P>(staged, copies, st);
  if ((s = launched()) != PP_OK) return s;

  // an operand's rows from r0 on
  auto from = [](GemmOperand o, int64_t r0) {
    for (auto& q : o.plane) q = static_cast<const uint8_t*>(q) + r0 * o.ld * 2;
    return o;
  };
  LogitArgs la = {};
  if (p.keep) la.logits = f32(p.logits), la.l_ld = p.vp;
  la.x = x, la.pairs = p.pairs, la.ksteps = static_cast<int32_t>(p.dp / 64), la.k = tok;
  la.bias = c.bias;
  if (p.bwd) la.g = bf(p.g), la.g_plane = p.t * p.piece, la.v_pad = static_cast<int32_t>(p.vp), la.db_part = c.db ? f32(p.db) : nullptr;
  if (p.fwd && p.all) {
    const bool each = d.reduction == PP_NONE;
    la.w = w, la.lse_out = c.stats, la.each = each ? c.loss : nullptr;
    la.sums = each ? nullptr : reinterpret_cast<double2*>(c.ws + p.sums);
    whole<kWhole>(p.all, la, st);
    const LossArgs loss = {la.sums, each ? 0 : static_cast<int32_t>(cdiv(p.t, 64)), d.reduction == PP_MEAN, each ? nullptr : c.loss,
                           c.stats + p.t};
    hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(1024), 0, st, loss);
  } else if (p.fwd) {
    la.target_logit = f32(p.tl);
    float2* carry = reinterpret_cast<float2*>(c.ws + p.part);
    la.part = carry + p.t;
    const bool each = d.reduction == PP_NONE;
    const uint32_t grid = static_cast<uint32_t>(cdiv(p.t, join_tokens(p)));
    double2* sums = each ? nullptr : reinterpret_cast<double2*>(c.ws + p.sums);
    // The loss and its divisor: by the join, if that is one workgroup; by the
    // gradient's first product, if there is one (what the divisor scales comes
    // after it).
    const LossArgs loss = {sums, each ? 0 : static_cast<int32_t>(grid), d.reduction == PP_MEAN, each ? nullptr : c.loss, c.stats + p.t};
    const bool whole = grid == 1;
    for (int64_t v0 = 0; v0 < p.v; v0 += p.fwd_piece) {
      const int64_t nv = std::min(p.fwd_piece, p.v - v0);
      const bool last = v0 + nv == p.v;
      la.w = from(w, v0), la.w.rows = static_cast<int32_t>(nv), la.v0 = static_cast<int32_t>(v0);
      logits<kStats, P>(p.logit, la, st);
      const int32_t parts = static_cast<int32_t>(cdiv(pad64(nv), tile_m(P, p.logit)) * tile_wm(P, p.logit));
      const JoinArgs ja = {tok, carry, la.target_logit, v0 ? 0 : 1, parts + 1, last ? nullptr : carry, c.stats, each ? c.loss : nullptr,
                           sums, whole ? loss : LossArgs{}};
      launch_join(p, ja, st);
    }
    if (p.bwd && !whole)
      la.loss = loss;
    else if (!whole)
      hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(1024), 0, st, loss);
    if ((s = launched()) != PP_OK) return s;
  }
  if (!p.bwd) return PP_OK;

  const int64_t dn = p.dx_turned ? p.d : p.t;
  float* dx_slab = f32(p.slab);
  float* dw_slab = dx_slab + (p.dx_slab ? p.dx_splits * p.dx_ld * dn : 0);   // (of one piece at a time)
  // the same array as [k][rows]
  auto by_k = [](GemmOperand o, int64_t rows, int64_t k) {
    o.rows = static_cast<int32_t>(rows), o.k = static_cast<int32_t>(k);
    return o;
  };
  ProductArgs xa = {}, wa = {};
  for (int64_t k = 0; k < p.pieces; ++k) {
    const int64_t v0 = k * p.piece, nv = std::min(p.piece, p.v - v0), nvp = pad64(nv);
    const Plan::Piece& q = p.of[k + 1 == p.pieces];
    la.w = from(w, v0), la.w.rows = static_cast<int32_t>(nv), la.v0 = static_cast<int32_t>(v0);
    la.g = bf(p.g), la.v_pad = static_cast<int32_t>(nvp), la.g_plane = p.t * nvp;
    la.db_part = c.db ? f32(p.db) : nullptr;
    if (p.all) {
      if (!p.fwd) whole<kWholeGrad>(p.all, la, st);   // (else G is there)
    } else if (P > 1 && p.keep)
      logits<P == 1 ? kGrad : kKept, P>(q.logit, la, st);
    else
      logits<kGrad, P>(q.logit, la, st);
    la.loss = {};
    const ClassSums db = {la.db_part, static_cast<int32_t>(la.tn * (p.all ? 1 : tile_wn(P, q.logit))), static_cast<int32_t>(nv), c.db ? c.db + v0 : nullptr};
    const int32_t db_blocks = c.db ? static_cast<int32_t>(cdiv(nv, 64)) : 0;
    if (db_blocks && !c.dw) hipLaunchKernelGGL(class_sum_kernel, dim3(static_cast<uint32_t>(db_blocks)), dim3(1024), 0, st, db, tok);
    // a small slab of dw is joined by dx's product, which comes after it
    bool riding = false;
    const GemmOperand g = operand(la.g, la.g_plane, nvp, p.t, nvp, P);
    if (c.dw) {   // d x classes, over tokens
      wa = {};
      wa.a = by_k(x, p.dp, p.t), wa.b = by_k(g, nvp, p.t);
      wa.m = static_cast<int32_t>(p.d), wa.n = static_cast<int32_t>(nv);
      wa.k = tok, wa.pairs = p.pairs, wa.ksteps = static_cast<int32_t>(cdiv(p.t, 64)), wa.splits = q.dw.splits;
      wa.map = {static_cast<S*>(c.dw) + v0 * p.d, 1, 0, p.d, 0, 1, 1, p.d % 4 == 0 && reinterpret_cast<uintptr_t>(c.dw) % 16 == 0};
      wa.slab = wa.splits > 1 ? dw_slab : nullptr, wa.slab_ld = p.dw_ld;
      wa.db = db, wa.db_blocks = db_blocks;
      product<S, true, true>(q.dw.tile, wa, st);
      riding = wa.slab && c.dx && wa.splits * p.dw_ld * nv <= (4 << 20);
      if (wa.slab && !riding) launch_slab<S>(slab_of(wa), tok, st);
    }
    if (c.dx) {   // over classes
      xa = {};
      const GemmOperand wp = by_k(from(w, v0), p.dp, nv);
      xa.k = tok, xa.pairs = p.pairs, xa.ksteps = static_cast<int32_t>(nvp / 64);
      xa.splits = p.dx_splits;   // (a last, smaller piece may leave some without a step: they add nothing)
      xa.slab = p.dx_slab ? dx_slab : nullptr, xa.slab_ld = p.dx_ld, xa.add = k > 0;
      if (riding) xa.join = slab_of(wa), xa.join_blocks = static_cast<int32_t>(std::min<int64_t>(cdiv(p.dw_ld / 4 * nv, 512), 128));
      const bool aligned = reinterpret_cast<uintptr_t>(c.dx) % 16 == 0;
      if (p.dx_turned) {   // tokens x d
        xa.a = g, xa.b = wp, xa.m = static_cast<int32_t>(p.t), xa.n = static_cast<int32_t>(p.d);
        xa.map = {c.dx, d.dx_sn, d.dx_sp, d.dx_sc, 0, static_cast<int32_t>(d.hw), 1,
                  aligned && d.dx_sp == 1 && d.hw % 4 == 0 && d.dx_sn % 4 == 0 && d.dx_sc % 4 == 0};
        product<S, false, true>(q.dx, xa, st);
      } else {             // d x tokens
        xa.a = wp, xa.b = g, xa.m = static_cast<int32_t>(p.d), xa.n = static_cast<int32_t>(p.t);
        xa.map = {c.dx, 1, 0, d.dx_sn, d.dx_sp, 1, static_cast<int32_t>(d.hw),
                  aligned && p.d % 4 == 0 && d.dx_sn % 4 == 0 && (d.hw == 1 || d.dx_sp % 4 == 0)};
        product<S, true, false>(q.dx, xa, st);
      }
    }
    if ((s = launched()) != PP_OK) return s;
  }
  if (c.dx && p.dx_slab) launch_slab<S>(slab_of(xa), tok, st);
  return launched();
}

pp_status check_desc(const pp_xent_desc* d) {
  if (!d) return fail(PP_EINVAL, "desc is NULL");
  if (d->dtype != PP_F32 && d->dtype != PP_BF16) return fail(PP_EINVAL, "bad dtype");
  if (d->reduction != PP_MEAN && d->reduction != PP_SUM && d->reduction != PP_NONE) return fail(PP_EINVAL, "bad reduction");
  if (d->n < 0 || d->hw < 0 || d->d < 1 || d->v < 1) return fail(PP_EINVAL, "n, hw must be >= 0, d and v >= 1");
  if (d->d > kMaxLd - 64 || d->v > kMaxLd - 64 || d->n > kMaxLd || d->hw > kMaxLd || d->n * d->hw > kMaxLd - 64)
    return fail(PP_EUNSUPPORTED, "d, v and the tokens must be below 2^22 - 64 each");
  if (d->n * d->hw * pad64(d->d) > (int64_t(1) << 35) || d->v * pad64(d->d) > (int64_t(1) << 35))
    return fail(PP_EUNSUPPORTED, "x and w must have fewer than 2^35 elements each");
  if (d->w_ld < d->d) return fail(PP_EINVAL, "w_ld smaller than d");
  if (d->x_sn < 0 || d->x_sc < 0 || d->x_sp < 0 || d->dx_sn < 0 || d->dx_sc < 0 || d->dx_sp < 0)
    return fail(PP_EINVAL, "negative stride");
  return PP_OK;
}

pp_status xent_call(const Call& c, bool fwd, bool bwd, size_t ws_bytes) {
  bwd = bwd && (c.dx || c.dw || c.db);
  pp_status s = check_desc(c.d);
  if (s != PP_OK) return s;
  const pp_xent_desc& d = *c.d;
  const size_t esz = d.dtype == PP_BF16 ? 2 : 4;
  const bool empty = d.n * d.hw == 0;
  if (!c.w || !c.stats || (fwd && !c.loss && !(empty && d.reduction == PP_NONE))) return fail(PP_EINVAL, "NULL pointer");
  if (!empty && (!c.x || !c.target)) return fail(PP_EINVAL, "NULL pointer");
  for (const void* q : {c.x, c.w, static_cast<const void*>(c.dx), static_cast<const void*>(c.dw)})
    if (reinterpret_cast<uintptr_t>(q) % esz) return fail(PP_EINVAL, "misaligned pointer");
  for (const void* q : {static_cast<const void*>(c.bias), static_cast<const void*>(c.class_weight), static_cast<const void*>(c.loss),
                        static_cast<const void*>(c.stats), static_cast<const void*>(c.grad), static_cast<const void*>(c.db)})
    if (reinterpret_cast<uintptr_t>(q) % 4) return fail(PP_EINVAL, "misaligned fp32 pointer");
  if (reinterpret_cast<uintptr_t>(c.target) % 8) return fail(PP_EINVAL, "misaligned target");
  if (empty) {   // no token: a loss of 0, and gradients of 0
    auto zero = [&](void* q, int64_t bytes) {
      if (q && bytes)
        hipLaunchKernelGGL(zero_kernel, dim3(static_cast<uint32_t>(std::min<int64_t>(cdiv(bytes, 256), 4096))), dim3(256), 0, c.st,
                           static_cast<uint8_t*>(q), bytes);
    };
    if (fwd)
      hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(1024), 0, c.st, LossArgs{nullptr, 0, 0, d.reduction == PP_NONE ? nullptr : c.loss, c.stats});
    if (bwd) {
      zero(c.dw, d.v * d.d * static_cast<int64_t>(esz));
      zero(c.db, d.v * 4);
    }
    return launched();
  }
  if (!fwd && !bwd) return PP_OK;
  const Plan p = make_plan(d, fwd, bwd, bwd && c.dw, aligned16(c.x), aligned16(c.w), reinterpret_cast<uintptr_t>(c.w) % 4 == 0);
  if (!c.ws || reinterpret_cast<uintptr_t>(c.ws) % 256) return fail(PP_EINVAL, "the workspace must be 256-byte aligned");
  if (ws_bytes < p.total) return fail(PP_ESIZE, "workspace smaller than pp_xent_workspace says");
  return d.dtype == PP_BF16 ? enqueue<__bf16, 1>(p, c) : enqueue<float, 3>(p, c);
}

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" pp_status pp_xent_workspace(const pp_xent_desc* desc, int32_t parts, size_t* bytes) {
  clear_error();
  if (!bytes) return fail(PP_EINVAL, "bytes is NULL");
  pp_status s = check_desc(desc);
  if (s != PP_OK) return s;
  if (parts < 1 || parts > 3) return fail(PP_EINVAL, "parts must be PP_XENT_FWD, PP_XENT_BWD or both");
  if (desc->n * desc->hw == 0) {
    *bytes = 0;
    return PP_OK;
  }
  // (operands that are not 16-byte aligned are copied: what the call needs at most)
  *bytes = make_plan(*desc, parts & 1, parts & 2, parts & 2, false, false, false).total;
  return PP_OK;
}

extern "C" pp_status pp_xent_fwd(const pp_xent_desc* desc, const void* x, const void* w, const float* bias,
                                 const float* class_weight, const int64_t* target, float* loss, float* stats,
                                 void* workspace, size_t ws_bytes, void* hip_stream) {
  clear_error();
  return xent_call({desc, x, w, bias, class_weight, target, loss, stats, nullptr, nullptr, nullptr, nullptr,
                    static_cast<uint8_t*>(workspace), static_cast<hipStream_t>(hip_stream)}, true, false, ws_bytes);
}

extern "C" pp_status pp_xent_bwd(const pp_xent_desc* desc, const void* x, const void* w, const float* bias,
                                 const float* class_weight, const int64_t* target, const float* stats, const float* grad,
                                 void* dx, void* dw, float* db, void* workspace, size_t ws_bytes, void* hip_stream) {
  clear_error();
  return xent_call({desc, x, w, bias, class_weight, target, nullptr, const_cast<float*>(stats), grad, dx, dw, db,
                    static_cast<uint8_t*>(workspace), static_cast<hipStream_t>(hip_stream)}, false, true, ws_bytes);
}

extern "C" pp_status pp_xent_step(const pp_xent_desc* desc, const void* x, const void* w, const float* bias,
                                  const float* class_weight, const int64_t* target, const float* grad, float* loss,
                                  float* stats, void* dx, void* dw, float* db, void* workspace, size_t ws_bytes,
                                  void* hip_stream) {
  clear_error();
  return xent_call({desc, x, w, bias, class_weight, target, loss, stats, grad, dx, dw, db,
                    static_cast<uint8_t*>(workspace), static_cast<hipStream_t>(hip_stream)}, true, true, ws_bytes);
}
