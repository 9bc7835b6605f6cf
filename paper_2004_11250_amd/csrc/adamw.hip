// adamw.hip -- pp_adamw_step / pp_adamw_values / pp_grad_norm: one AdamW step of
// a list of tensors with moments of 32 or 8 bits, and the norm of a list of
// gradients.
//
//   g = s G,  m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2
//   W' = (1 - lr wd) W - lr (m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps)
//
// Everything is fp32; what does not differ between elements (1 - b, the bias
// corrections, rates) is taken in 64 bits and rounded once.  All are bound by memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <limits>
#include <string>

#include "api_internal.hpp"
#include "lists.hpp"
#include "train.hpp"

namespace pp {
namespace {

using bf16 = __bf16;

constexpr int kBlock = PP_ADAMW_BLOCK;   // elements that share their scales: 16 lanes of 8
constexpr float kTiny = 0x1p-100f;       // the least scale
constexpr int kFirstCode = 1777;         // v: code c stands for the float whose bits are (c + 1777) << 19

using half = _Float16;
using Codes = __attribute__((ext_vector_type(2))) uint32_t;   // of eight first moments

struct Tensor {
  const void* w;
  const void* g;
  void* w_out;
  bf16* copy;
  const uint16_t* keep;
  int64_t n, at;
  float decay;
};
constexpr int kTensors = 56;
using Tensors = List<Tensor, kTensors>;

struct Step {
  double lr, ln1, ln2;           // ln of the betas
  double c1;                     // 1 / (1 - beta1^t), where the step is the host's
  float c2;                      // 1 / sqrt(1 - beta2^t)
  float b1, n1, b2, n2, eps;     // betas, 1 - betas
  const float* d_lr;
  const int64_t* d_step;
  const float* d_scale;
  const void *m, *v;
  const float *ms, *vs;
  void *m_out, *v_out;
  float *ms_out, *vs_out;
  uint32_t turn;                 // turn_of(the step), where it is the host's
};
static_assert(sizeof(Tensors) + sizeof(Step) <= 4096, "kernel arguments hold 4 KB");

// The largest of a row of 16 lanes, in all of them.
__device__ __forceinline__ float row_max(float x) {
  auto turn = [](float v, auto by) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + decltype(by)::value, 0xf, 0xf, true));
  };
  x = fmaxf(x, turn(x, std::integral_constant<int, 8>()));
  x = fmaxf(x, turn(x, std::integral_constant<int, 4>()));
  x = fmaxf(x, turn(x, std::integral_constant<int, 2>()));
  return fmaxf(x, turn(x, std::integral_constant<int, 1>()));
}

// Square roots of eight v >= 0, to 1 ulp.  The hardware's takes values below fp32's
// normal range for 0; eight that hold one are scaled (one instruction and a half an
// element to find out, in place of five to scale all).
__device__ __forceinline__ void roots(const float (&v)[8], float (&r)[8]) {
  uint32_t least = ~0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    least = min(least, __builtin_bit_cast(uint32_t, v[e]) - 1u);   // (0: the largest)
    r[e] = __builtin_amdgcn_sqrtf(v[e]);
  }
  if (least < 0x007fffffu) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = v[e] < 0x1p-96f ? __builtin_amdgcn_sqrtf(v[e] * 0x1p64f) * 0x1p-32f : r[e];
  }
}

// Second moments: a root over the block's scale has 4 bits of the exponent and 4 after
// the leading one, its code c, and between codes it is held to sixths of one: c + k / 6,
// k = -3 .. 3, is the half c + (k mod 8) / 8, which holds 11 bits.  beta2 near 1 moves a
// root by far less than half a code a step (at 0.999 by 0.0005 (g^2 / v - 1) of itself; a
// code is 2^-4 to 2^-5), which codes alone would round away at every step: an element
// whose gradients grow, shrink or stop beside a steady one would be left where it was.  So
// what is held is rounded up where the part beyond a sixth is above 1 - u, u being
// spread evenly over 0..1 by step and element (multiples of the golden section and of
// another such number, modulo 1): over the steps the roundings add up to nothing.
// (u at random would do the same with errors of the root of their count.)
constexpr uint32_t kTurnStep = 0x9e3779b9u, kTurnElement = 0xc13fa9a9u;
__host__ __device__ inline uint32_t turn_of(int64_t step) { return static_cast<uint32_t>(step) * kTurnStep; }

__device__ __forceinline__ half code_of(float r, uint32_t turn) {
  const int whole = __builtin_bit_cast(int, r);
  const int bits = min(max(whole, (kFirstCode + 1) << 19), (kFirstCode + 255) << 19);           // (r = 0: 0, above it 1 at least)
  const int c = (bits + ((bits >> 19) & 1) + (0x3ffff - (kFirstCode << 19))) >> 19;
  const int k = (6 * (bits - ((c + kFirstCode) << 19)) + static_cast<int>(turn >> 13)) >> 19;   // (at most half a code: -3 .. 3)
  return static_cast<half>(static_cast<uint16_t>(whole ? c << 3 | (k & 7) : 0)) * static_cast<half>(0.125f);
}
// What is held, and what its code alone stands for.
__device__ __forceinline__ float value_of(half held) {
  const int x = __builtin_bit_cast(int, static_cast<float>(held) + 0x1p20f), c = x & 0x7f8;    // (in eighths)
  const int k = (x << 29) >> 29;
  return __builtin_bit_cast(float, c ? (kFirstCode << 19) + (c << 16) + k * 87381 : 0);        // (2^19 / 6)
}
__device__ __forceinline__ float code_value(half held) {
  const int c = static_cast<uint16_t>(held) & 255;
  return __builtin_bit_cast(float, c ? (c + kFirstCode) << 19 : 0);
}

__device__ __forceinline__ void m_values(Codes c, float s, float (&m)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int w = h ? c.y : c.x;
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    m[4 * h] = a[0] * s, m[4 * h + 1] = a[1] * s, m[4 * h + 2] = b[0] * s, m[4 * h + 3] = b[1] * s;
  }
}
template <class F>
__device__ __forceinline__ void v_values(const Eight<half>& held, float s, float (&v)[8], F&& value) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float r = value(held[e]) * s;
    v[e] = r * r;
  }
}

// Which of a pruned layer's elements x .. x + 7 from the chunk's first on are kept
// taps, bit by bit; the chunk begins at tap `tap` of kernel `cell` of `cells`.
__device__ __forceinline__ uint32_t kept8(const uint16_t* keep, int64_t cell, int tap, int64_t cells, int x) {
  const uint32_t y = static_cast<uint32_t>(tap + x), k = y / 9u;
  const uint16_t* p = keep + cell + k;
  uint32_t bits = 0;
  if (cell + k < cells) bits = p[0] & 511u;
  if (cell + k + 1 < cells) bits |= static_cast<uint32_t>(p[1]) << 9;
  return bits >> (y - 9u * k);
}

constexpr int kChunk = 2048;       // elements of a workgroup of AdamW
constexpr int kFar = kBlock / 2;   // (the second half of a lane's elements, where they are two fours)
template <bool SPLIT, bool ONCE>
__device__ __forceinline__ Codes codes(const void* p, int64_t at) {
  const uint8_t* q = static_cast<const uint8_t*>(p) + at;
  if constexpr (SPLIT)
    return {fetch<ONCE>(reinterpret_cast<const uint32_t*>(q)), fetch<ONCE>(reinterpret_cast<const uint32_t*>(q + kFar))};
  else
    return fetch<ONCE>(reinterpret_cast<const Codes*>(q));
}
template <bool SPLIT, bool ONCE>
__device__ __forceinline__ void put_codes(void* p, int64_t at, Codes c) {
  uint8_t* q = static_cast<uint8_t*>(p) + at;
  if constexpr (SPLIT)
    keep_at<ONCE>(reinterpret_cast<uint32_t*>(q), c[0]), keep_at<ONCE>(reinterpret_cast<uint32_t*>(q + kFar), c[1]);
  else
    keep_at<ONCE>(reinterpret_cast<Codes*>(q), c);
}

// Eight elements a lane, 2048 of one tensor a workgroup; a block's scales are the
// largest of 16 lanes.  Three states in turn, us a step in place / into other arrays:
// fp32 w, g and moments, VGG-16, 15 M weights 69 / 70 (6.0 TB/s), 51 M 239 / 236
// (6.1 TB/s); bf16 w and g, 8-bit moments, 102 M 209 / 199 (6.2 TB/s); fp32 w, bf16 g
// and copies, 8-bit moments, 31 M 104 / 104 (5.4 TB/s).
// Where a value has four bytes a lane's eight are two fours 64 elements apart, so that
// each access of 16 lanes is 256 bytes in a row (eight in a row are two accesses of half
// of each line: 51 M fp32 weights 263, and past the caches 362).
// Elements of a workgroup, 2048 / 4096 / 8192: fp32 w, 32 bits, 51 M 236 / 248 / 252, 8 bits
// 150 / 160 / 164; bf16 w and g, 8 bits, 102 M 207 / 214 / 228 (199 without a loop).
// With 8 bits some 60 instructions an element stand beside 12 bytes of memory, and count:
// one root serves the update and the code, what only some steps need (masks: 202 without
// the test; a tensor's end, values that are not finite, roots below the normal range) is
// looked for by eight elements together, and the update's division is a product with the
// hardware's reciprocal, 1 ulp (102 M, an exact one: 209 / 199).
template <class W, class G, int BITS, bool ONCE>
__global__ __launch_bounds__(256) void adamw_kernel(const Tensors list, const Step s) {
  constexpr bool SPLIT = kSplit<W, G> || BITS == 32;
  int chunk;
  const Tensor& t = list.item[find(list, blockIdx.x, &chunk)];
  const int64_t e0 = static_cast<int64_t>(chunk) * kChunk, n = t.n, left = n - e0;
  const int len = static_cast<int>(left < kChunk ? (left + kBlock - 1) / kBlock * kBlock : kChunk);
  const W* w_in = static_cast<const W*>(t.w) + e0;
  const G* g_in = static_cast<const G*>(t.g) + e0;
  W* w_out = static_cast<W*>(t.w_out) + e0;
  bf16* copy = t.copy ? t.copy + e0 : nullptr;
  const int64_t at = t.at + e0, block = at / kBlock;
  const uint16_t* keep = t.keep;
  const int64_t cell = keep ? e0 / 9 : 0, cells = keep ? n / 9 : 0;
  const int tap = static_cast<int>(e0 - 9 * cell);

  const float scale = s.d_scale ? *s.d_scale : 1.f;
  const bool go = fabsf(scale) < INFINITY;
  const double lr = s.d_lr ? static_cast<double>(*s.d_lr) : s.lr;
  double c1 = s.c1;
  float c2 = s.c2;
  uint32_t turn = s.turn;
  if (s.d_step) {
    const int64_t step = max(*s.d_step, int64_t(1));
    const double k = static_cast<double>(step);
    turn = turn_of(step);
    c1 = -1. / expm1(k * s.ln1);
    c2 = static_cast<float>(1. / sqrt(-expm1(k * s.ln2)));
  }
  const float rate = static_cast<float>(lr * c1), decay = static_cast<float>(1. - lr * static_cast<double>(t.decay));

  const int x = SPLIT ? 4 * (threadIdx.x & 15) + kBlock * (threadIdx.x >> 4) : 8 * threadIdx.x;
  if (x >= len) return;            // (whole blocks: rows of 16 lanes)
  const int64_t there = left - x;     // elements from here on
  float w[8], g[8], m[8], v[8];
  Codes mc;
  Eight<half> held;
  float ms, vs;
  load8<SPLIT, ONCE>(w_in + x, there, kFar, w);
  load8<SPLIT, ONCE>(g_in + x, there, kFar, g);
  if constexpr (BITS == 32) {
    load8<SPLIT, ONCE>(static_cast<const float*>(s.m) + at + x, kBlock, kFar, m);
    load8<SPLIT, ONCE>(static_cast<const float*>(s.v) + at + x, kBlock, kFar, v);
  } else {
    mc = codes<SPLIT, ONCE>(s.m, at + x);
    held = get8<SPLIT, ONCE>(static_cast<const half*>(s.v) + at + x, kBlock, kFar);
    ms = s.ms[block + x / kBlock], vs = s.vs[block + x / kBlock];
  }
  const uint32_t on = !keep ? 255u : SPLIT ? (kept8(keep, cell, tap, cells, x) & 15u) | kept8(keep, cell, tap, cells, x + kFar) << 4 : kept8(keep, cell, tap, cells, x);
  if (go) {
    if constexpr (BITS == 8) m_values(mc, ms, m), v_values(held, vs, v, [](half h) { return value_of(h); });
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float ge = scale * g[e];
      m[e] = s.b1 * m[e] + s.n1 * ge;
      v[e] = s.b2 * v[e] + s.n2 * (ge * ge);
    }
    if (keep) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (!(on >> e & 1)) m[e] = v[e] = 0.f;
    }
    if (there < (SPLIT ? kFar + 4 : 8)) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if ((SPLIT && e >= 4 ? e - 4 + kFar : e) >= there) m[e] = v[e] = 0.f;
    }
    float r[8];
    roots(v, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = decay * w[e] - rate * m[e] * __builtin_amdgcn_rcpf(r[e] * c2 + s.eps);
    if (keep) {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = on >> e & 1 ? w[e] : 0.f;
    }
    if constexpr (BITS == 8) {
      float top = 0.f, vtop = 0.f, odd = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        top = fmaxf(top, fabsf(m[e]));
        vtop = fmaxf(vtop, r[e]);
        odd += 0.f * m[e];              // NaN, if one is not finite
      }
      if (!(odd == 0.f && vtop < INFINITY)) {
        top = vtop = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool fine = fabsf(m[e]) < INFINITY;
          r[e] = fine ? fminf(r[e], 0x1.fffffep63f) : 0.f;       // (the root of fp32's largest value)
          m[e] = fine ? m[e] : __builtin_nanf("");
          top = fmaxf(top, fine ? fabsf(m[e]) : 0.f);
          vtop = fmaxf(vtop, r[e]);
        }
      }
      ms = fmaxf(row_max(top) * (1.f / 448.f), kTiny);
      vs = fmaxf(row_max(vtop), kTiny);
      const float im = 1.f / ms, iv = 1.f / vs;
      uint32_t c[2];
      const uint32_t first = static_cast<uint32_t>(at + x) * kTurnElement + turn;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int q = __builtin_amdgcn_cvt_pk_fp8_f32(m[4 * h] * im, m[4 * h + 1] * im, 0, false);
        q = __builtin_amdgcn_cvt_pk_fp8_f32(m[4 * h + 2] * im, m[4 * h + 3] * im, q, true);
        c[h] = q;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          held[4 * h + e] = code_of(r[4 * h + e] * iv, first + static_cast<uint32_t>(h * (SPLIT ? kFar : 4) + e) * kTurnElement);
      }
      mc = {c[0], c[1]};
    }
  }
  if (there > 0) {
    store8<SPLIT, ONCE>(w_out + x, there, kFar, w);
    if (copy) store8<SPLIT, ONCE>(copy + x, there, kFar, w);
  }
  if constexpr (BITS == 32) {
    store8<SPLIT, ONCE>(static_cast<float*>(s.m_out) + at + x, kBlock, kFar, m);
    store8<SPLIT, ONCE>(static_cast<float*>(s.v_out) + at + x, kBlock, kFar, v);
  } else {
    put_codes<SPLIT, ONCE>(s.m_out, at + x, mc);
    put8<SPLIT, ONCE>(static_cast<half*>(s.v_out) + at + x, kBlock, kFar, held);
    if (threadIdx.x % 16 == 0) s.ms_out[block + x / kBlock] = ms, s.vs_out[block + x / kBlock] = vs;
  }
}

// What codes stand for: 8 elements a lane.  102 M to bf16 119 us, 6 TB/s.
template <class S>
__global__ __launch_bounds__(256) void values_kernel(const uint8_t* m, const half* v, const float* ms, const float* vs,
                                                     int64_t all, S* m_out, S* v_out) {
  constexpr bool SPLIT = kSplit<S>;
  const int lane = SPLIT ? 4 * (threadIdx.x & 15) + kBlock * (threadIdx.x >> 4) : 8 * threadIdx.x;
  for (int64_t x = static_cast<int64_t>(blockIdx.x) * 2048 + lane; x < all; x += static_cast<int64_t>(gridDim.x) * 2048) {
    float a[8];
    if (m_out) {
      m_values(codes<SPLIT, false>(m, x), ms[x / kBlock], a);
      store8<SPLIT>(m_out + x, kBlock, kFar, a);
    }
    if (v_out) {
      v_values(get8<SPLIT>(v + x, kBlock, kFar), vs[x / kBlock], a, [](half h) { return code_value(h); });
      store8<SPLIT>(v_out + x, kBlock, kFar, a);
    }
  }
}

struct Grad {
  const void* g;
  int64_t n;
};
constexpr int kGrads = 192, kShort = 8;   // (a short list's launch takes 0.6 us less of the host)
static_assert(sizeof(List<Grad, kGrads>) + 16 <= 4096, "kernel arguments hold 4 KB");

template <int WAVES>
__device__ __forceinline__ double sum_of_block(double x, double* sums) {
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0.;
  for (int i = 0; i < WAVES; ++i) x += sums[i];
  return x;
}

// A chunk's sum of squares.  59 MB of fp32 11.5 us, 63 MB of bf16 13.3: 5.1 and 4.7 TB/s.
template <class G, int N>
__global__ __launch_bounds__(256) void square_kernel(const List<Grad, N> list, int32_t size, double* part) {
  __shared__ double sums[4];
  int chunk;
  const Grad& t = list.item[find(list, blockIdx.x, &chunk)];
  const int64_t e0 = static_cast<int64_t>(chunk) * size, left = t.n - e0;
  const int len = static_cast<int>(left < size ? left : size);
  const G* p = static_cast<const G*>(t.g) + e0;
  double sum[2] = {0., 0.};
  constexpr bool SPLIT = kSplit<G>;
  for (int x = SPLIT ? 4 * (threadIdx.x & 63) + 512 * (threadIdx.x >> 6) : 8 * threadIdx.x; x < len; x += 2048) {
    float g[8];
    load8<SPLIT>(p + x, len - x, 256, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e & 1] += static_cast<double>(g[e]) * g[e];
  }
  const double all = sum_of_block<4>(sum[0] + sum[1], sums);
  if (threadIdx.x == 0) part[blockIdx.x] = all;
}

// The norm of all chunks' sums (one at least of each tensor that is not empty; a chunk has
// 2048 elements, more where there are more than 2 M in all, 16384 from 15 M on), and the
// factor: 2 to 4 us, the launch.  (The first launch's last workgroup could do it, with a
// counter that something has cleared; a list so short that one workgroup reads it all
// would need no second launch, but has one here too.)
__global__ __launch_bounds__(1024) void norm_kernel(const double* part, int64_t parts, float most, float* out) {
  __shared__ double sums[16];
  double x = 0.;
  for (int64_t i = threadIdx.x; i < parts; i += 1024) x += part[i];
  x = sqrt(sum_of_block<16>(x, sums));
  if (threadIdx.x == 0) {
    out[0] = static_cast<float>(x);
    out[1] = !(x < INFINITY) ? __builtin_nanf("") : x <= most ? 1.f : static_cast<float>(most / x);
  }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

bool off(const void* p, size_t by) { return reinterpret_cast<uintptr_t>(p) % by != 0; }
size_t size_of(int32_t dtype) { return dtype == PP_BF16 ? 2 : 4; }
bool known(int32_t dtype) { return dtype == PP_F32 || dtype == PP_BF16; }
constexpr int64_t kMost = int64_t(1) << 34;   // (a launch has fewer than 2^32 threads, eight elements each at least)

// Elements that a workgroup sums: enough workgroups for the card where there is
// little to do, long ones where there is much.
int32_t chunk_of(int64_t total, int64_t most) {
  return static_cast<int32_t>(std::min<int64_t>(most, std::max<int64_t>(1, cdiv(total, 2048 * 4 * kCUs)) * 2048));
}

// The launches of a list: up to N tensors each that are not empty, a workgroup for every
// `per` elements of one.  fill(item, tensor) makes an item of the list, go(list, blocks)
// launches it.  (Lists of equal length, where one does not hold all: 72 tensors of 31 M
// elements 103.6 us a step in place of 103.0, norms of 250 tensors of 300000 58 of 54.)
template <class L, class T, class Fill, class Go>
pp_status each_launch(const T* tensors, int32_t count, int64_t per, Fill&& fill, Go&& go) {
  constexpr int N = sizeof(L::first) / 4;
  L list;
  std::memset(&list, 0, sizeof(list));
  int64_t blocks = 0;
  auto flush = [&]() -> pp_status {
    if (!list.count) return PP_OK;
    go(list, static_cast<uint32_t>(blocks));
    list.count = 0, blocks = 0;
    return launched();
  };
  for (int32_t i = 0; i < count; ++i) {
    if (tensors[i].n == 0) continue;
    const int64_t b = cdiv(tensors[i].n, per);
    if (list.count == N || blocks + b > (1 << 23)) {
      const pp_status s = flush();
      if (s != PP_OK) return s;
    }
    fill(list.item[list.count], tensors[i]);
    list.first[list.count++] = static_cast<int32_t>(blocks);
    blocks += b;
  }
  return flush();
}

pp_status check_tensor(const pp_adamw_tensor& t, const pp_adamw_desc& d) {
  if (t.n < 0 || t.at < 0 || t.at % kBlock) return fail(PP_EINVAL, "bad size, or moments that do not begin at a block");
  if (t.n >= kMost || t.at >= int64_t(1) << 40) return fail(PP_EUNSUPPORTED, "a tensor must have fewer than 2^34 elements, and the moments fewer than 2^40");
  if (!std::isfinite(t.weight_decay)) return fail(PP_EINVAL, "weight_decay must be finite");
  if (t.keep && t.n % 9) return fail(PP_EINVAL, "a pruned layer has 9 elements for each tap mask");
  if (t.n == 0) return PP_OK;
  if (!t.w || !t.g || !t.w_out) return fail(PP_EINVAL, "NULL pointer");
  if (off(t.w, size_of(d.w_dtype)) || off(t.w_out, size_of(d.w_dtype)) || off(t.g, size_of(d.g_dtype)) || off(t.copy, 2) || off(t.keep, 2))
    return fail(PP_EINVAL, "misaligned pointer");
  return PP_OK;
}

pp_status check_desc(const pp_adamw_desc& d) {
  if (!known(d.w_dtype) || !known(d.g_dtype)) return fail(PP_EINVAL, "bad dtype");
  if (d.bits != 32 && d.bits != 8) return fail(PP_EINVAL, "moments have 32 or 8 bits");
  if (!std::isfinite(d.lr) || !(d.beta1 >= 0 && d.beta1 < 1) || !(d.beta2 >= 0 && d.beta2 < 1) || !(d.eps >= 0) || !std::isfinite(d.eps))
    return fail(PP_EINVAL, "lr and eps must be finite, eps >= 0, betas in 0..1");
  if (!d.d_step && d.step < 1) return fail(PP_EINVAL, "steps count from 1");
  if (off(d.d_lr, 4) || off(d.d_step, 8) || off(d.d_grad_scale, 4)) return fail(PP_EINVAL, "misaligned scalar");
  return PP_OK;
}

pp_status check_moments(const pp_adamw_desc& d) {
  for (const void* p : {d.m, d.v, static_cast<const void*>(d.m_out), static_cast<const void*>(d.v_out)})
    if (!p || off(p, 16)) return fail(PP_EINVAL, "moments must be 16-byte aligned");
  if (d.bits == 8)
    for (const float* p : {d.m_scale, d.v_scale, static_cast<const float*>(d.m_scale_out), static_cast<const float*>(d.v_scale_out)})
      if (!p || off(p, 4)) return fail(PP_EINVAL, "moments of 8 bits need their scales");
  return PP_OK;
}

pp_status adamw(const pp_adamw_tensor* tensors, int32_t count, const pp_adamw_desc* desc, hipStream_t st) {
  if (!desc) return fail(PP_EINVAL, "desc is NULL");
  if (count < 0 || (count && !tensors)) return fail(PP_EINVAL, "tensors is NULL");
  const pp_adamw_desc& d = *desc;
  pp_status r = check_desc(d);
  int64_t total = 0;
  for (int32_t i = 0; i < count && r == PP_OK; ++i) r = check_tensor(tensors[i], d), total += tensors[i].n;
  if (r == PP_OK && total) r = check_moments(d);
  if (r != PP_OK || !total) return r;
  Step s;
  std::memset(&s, 0, sizeof(s));
  s.lr = d.lr, s.ln1 = std::log(d.beta1), s.ln2 = std::log(d.beta2);
  if (!d.d_step) {
    s.c1 = -1. / std::expm1(static_cast<double>(d.step) * s.ln1);
    s.c2 = static_cast<float>(1. / std::sqrt(-std::expm1(static_cast<double>(d.step) * s.ln2)));
    s.turn = turn_of(d.step);
  }
  s.b1 = static_cast<float>(d.beta1), s.n1 = static_cast<float>(1. - d.beta1);
  s.b2 = static_cast<float>(d.beta2), s.n2 = static_cast<float>(1. - d.beta2), s.eps = static_cast<float>(d.eps);
  s.d_lr = d.d_lr, s.d_step = d.d_step, s.d_scale = d.d_grad_scale;
  s.m = d.m, s.v = d.v, s.ms = d.m_scale, s.vs = d.v_scale;
  s.m_out = d.m_out, s.v_out = d.v_out, s.ms_out = d.m_scale_out, s.vs_out = d.v_scale_out;
  // Steps of more than the last cache holds (256 MB) go past the caches.  us, past them /
  // not, three states in turn in place: 15 M fp32 weights 69 / 79 (one again and again:
  // 74 / 60), 51 M 239 / 266, with 8-bit moments 150 / 173, 102 M bf16 weights with 8-bit
  // moments 209 / 236; 3 M fp32 weights (86 MB) 16.4 / 14.4, 8 M bf16 with 8-bit moments
  // (98 MB) 21.8 / 20.7.
  const bool past = total * static_cast<double>(2 * size_of(d.w_dtype) + size_of(d.g_dtype) + (d.bits == 8 ? 6 : 16)) > 256e6;
  auto fill = [](Tensor& x, const pp_adamw_tensor& t) {
    x = {t.w, t.g, t.w_out, static_cast<bf16*>(t.copy), t.keep, t.n, t.at, static_cast<float>(t.weight_decay)};
  };
  auto launch = [&](auto w, auto g, auto bits) {
    using W = decltype(w);
    using G = decltype(g);
    return each_launch<Tensors>(tensors, count, kChunk, fill, [&](const Tensors& list, uint32_t blocks) {
      if (past)
        hipLaunchKernelGGL((adamw_kernel<W, G, decltype(bits)::value, true>), dim3(blocks), dim3(256), 0, st, list, s);
      else
        hipLaunchKernelGGL((adamw_kernel<W, G, decltype(bits)::value, false>), dim3(blocks), dim3(256), 0, st, list, s);
    });
  };
  auto with_g = [&](auto w, auto bits) { return d.g_dtype == PP_BF16 ? launch(w, bf16(), bits) : launch(w, float(), bits); };
  auto with_w = [&](auto bits) { return d.w_dtype == PP_BF16 ? with_g(bf16(), bits) : with_g(float(), bits); };
  return d.bits == 8 ? with_w(std::integral_constant<int, 8>()) : with_w(std::integral_constant<int, 32>());
}

pp_status values(const void* m, const void* v, const float* ms, const float* vs, int64_t all, int32_t dtype, void* m_out,
                 void* v_out, hipStream_t st) {
  if (!known(dtype)) return fail(PP_EINVAL, "bad dtype");
  if (all < 0 || all % kBlock) return fail(PP_EINVAL, "elements must be whole blocks");
  if (all >= int64_t(1) << 40) return fail(PP_EUNSUPPORTED, "too many elements");
  if (!all || (!m_out && !v_out)) return PP_OK;
  if ((m_out && (!m || !ms || off(m, 16) || off(ms, 4))) || (v_out && (!v || !vs || off(v, 16) || off(vs, 4))))
    return fail(PP_EINVAL, "codes must be 16-byte aligned, with their scales");
  if (off(m_out, 16) || off(v_out, 16)) return fail(PP_EINVAL, "misaligned output");
  const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(cdiv(all, 2048), 1 << 20)));
  auto go = [&](auto o) {
    using S = decltype(o);
    hipLaunchKernelGGL((values_kernel<S>), grid, dim3(256), 0, st, static_cast<const uint8_t*>(m), static_cast<const half*>(v), ms,
                       vs, all, static_cast<S*>(m_out), static_cast<S*>(v_out));
  };
  dtype == PP_BF16 ? go(bf16()) : go(float());
  return launched();
}

// Partial sums of a list, and the elements each is of.
pp_status norm_plan(const pp_grad* grads, int32_t count, int32_t dtype, int64_t* parts, int32_t* chunk) {
  if (count < 0 || (count && !grads)) return fail(PP_EINVAL, "grads is NULL");
  if (!known(dtype)) return fail(PP_EINVAL, "bad dtype");
  int64_t total = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (grads[i].n < 0) return fail(PP_EINVAL, "negative size");
    if (grads[i].n >= kMost) return fail(PP_EUNSUPPORTED, "a tensor must have fewer than 2^34 elements");
    total += grads[i].n;
  }
  *chunk = chunk_of(total, 16384);
  *parts = 0;
  for (int32_t i = 0; i < count; ++i) *parts += cdiv(grads[i].n, *chunk);
  return PP_OK;
}

pp_status norm(const pp_grad* grads, int32_t count, int32_t dtype, float most, float* out, void* ws, size_t bytes, hipStream_t st) {
  int64_t parts;
  int32_t chunk;
  pp_status r = norm_plan(grads, count, dtype, &parts, &chunk);
  if (r != PP_OK) return r;
  if (!(most > 0)) return fail(PP_EINVAL, "max_norm must be above 0");
  if (!out || off(out, 4)) return fail(PP_EINVAL, "out must be 4-byte aligned");
  for (int32_t i = 0; i < count; ++i)
    if (grads[i].n && (!grads[i].g || off(grads[i].g, size_of(dtype)))) return fail(PP_EINVAL, "NULL or misaligned gradient");
  if (parts && (!ws || off(ws, 256))) return fail(PP_EINVAL, "the workspace must be 256-byte aligned");
  if (bytes < static_cast<size_t>(parts) * 8) return fail(PP_ESIZE, "workspace smaller than needed");
  double* part = static_cast<double*>(ws);
  auto fill = [](Grad& x, const pp_grad& t) { x = {t.g, t.n}; };
  int64_t at = 0;
  auto launch = [&](auto size) {
    constexpr int N = decltype(size)::value;
    return each_launch<List<Grad, N>>(grads, count, chunk, fill, [&](const List<Grad, N>& list, uint32_t blocks) {
      if (dtype == PP_BF16)
        hipLaunchKernelGGL((square_kernel<bf16, N>), dim3(blocks), dim3(256), 0, st, list, chunk, part + at);
      else
        hipLaunchKernelGGL((square_kernel<float, N>), dim3(blocks), dim3(256), 0, st, list, chunk, part + at);
      at += blocks;
    });
  };
  r = count <= kShort ? launch(std::integral_constant<int, kShort>()) : launch(std::integral_constant<int, kGrads>());
  if (r != PP_OK) return r;
  hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(1024), 0, st, part, parts, most, out);
  return launched();
}

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" pp_status pp_adamw_step(const pp_adamw_tensor* tensors, int32_t count, const pp_adamw_desc* desc, void* hip_stream) {
  return guarded([&] { return adamw(tensors, count, desc, static_cast<hipStream_t>(hip_stream)); });
}

extern "C" pp_status pp_adamw_values(const void* m, const void* v, const float* m_scale, const float* v_scale, int64_t elements,
                                     int32_t dtype, void* m_out, void* v_out, void* hip_stream) {
  return guarded([&] { return values(m, v, m_scale, v_scale, elements, dtype, m_out, v_out, static_cast<hipStream_t>(hip_stream)); });
}

extern "C" pp_status pp_grad_norm_workspace(const pp_grad* grads, int32_t count, int32_t dtype, size_t* bytes) {
  return guarded([&]() -> pp_status {
    if (!bytes) return fail(PP_EINVAL, "bytes is NULL");
    int64_t parts;
    int32_t chunk;
    const pp_status s = norm_plan(grads, count, dtype, &parts, &chunk);
    if (s == PP_OK) *bytes = static_cast<size_t>(parts) * 8;
    return s;
  });
}

extern "C" pp_status pp_grad_norm(const pp_grad* grads, int32_t count, int32_t dtype, float max_norm, float* out,
                                  void* workspace, size_t ws_bytes, void* hip_stream) {
  return guarded([&] { return norm(grads, count, dtype, max_norm, out, workspace, ws_bytes, static_cast<hipStream_t>(hip_stream)); });
}
