// xent_few.hpp -- the head for few tokens (at most 64, in fp32 128), where
// reading w is the work.  w is read in its own type and not copied; the logits of all classes
// are kept (they are small), so that the gradient's kernel reads w once.
//
// Both kernels use the matrix cores on what the lanes load, sixteen bytes each:
// which of the k positions of an instruction a lane's values take is free as
// long as both operands agree, so lane (r, g) = (lane % 16, lane / 16) gives
// four (or eight) neighbouring channels, one (or all) to an instruction.  fp32
// values are multiplied in fp32, whose rate is enough for that up to 16 tokens; the
// logits of more take w in three bf16 values (few_logit3_kernel).
// (Included by xent.hip, inside its namespace.)

constexpr int kFewTokens[2] = {128, 64};   // fp32, bf16

struct FewArgs {
  const void* w;        // [v][w_ld]
  int64_t w_ld;
  const void* x;        // token t, channel c at (t / hw) x_sn + (t % hw) x_sp + c x_sc
  int64_t x_sn, x_sp, x_sc;
  int32_t hw, d, x_wide;   // x_wide: pieces of a lane are contiguous and aligned
  Tokens k;
  float* logits;        // [token][l_ld], or null
  int64_t l_ld;
  // forward
  const float* bias;
  float2* part;         // [workgroup][token], or null
  float* target_logit;
  // gradient
  void* dw;             // [v][d], or null
  float* db;            // or null
  float* slab;          // [split][token][slab_ld], or null
  int64_t slab_ld;
  int32_t splits, groups;   // of the classes; of the channels (64 C each)
};

constexpr uint32_t kNowhere = 0x80000000u;   // past the end of any buffer made here
static_assert(32 * kMaxLd * 4 < int64_t(kNowhere), "32 rows of w in one descriptor");

// N values of a row of w, from byte `at` of the buffer on, which is the row's
// column `col`.  A row's last values are fetched as its last N and moved down
// when they are used (few_tail): nothing is read outside the rows, and columns
// past the end count as zeros whatever is there.  Words are fetched through the
// buffer; rows of bf16 values that do not begin at words (ODD) from memory.
template <class S, int N, bool ODD>
__device__ __forceinline__ auto few_load(__amdgpu_buffer_rsrc_t r, const S* rows, bool row, uint32_t at, int col, int cols) {
  using V = __attribute__((ext_vector_type(N))) S;
  const uint32_t off = at - static_cast<uint32_t>(max(col + N - cols, 0) * static_cast<int>(sizeof(S)));
  if constexpr (ODD) {
    using U = __attribute__((ext_vector_type(N), aligned(2))) S;
    V v = {};
    if (row && col < cols) v = *reinterpret_cast<const U*>(reinterpret_cast<const uint8_t*>(rows) + off);
    return v;
  } else if constexpr (sizeof(V) == 16) {
    return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(r, row && col < cols ? off : kNowhere, 0, 0));
  } else {
    return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(r, row && col < cols ? off : kNowhere, 0, 0));
  }
}
template <class V>
__device__ __forceinline__ V few_tail(V v, int col, int cols) {
  constexpr int N = sizeof(V) / sizeof(v[0]);
  const int by = max(col + N - cols, 0);
#pragma unroll
  for (int n = 1; n < N; n *= 2) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const auto moved = e + n < N ? v[e + n < N ? e + n : 0] : static_cast<decltype(v[0] + v[0])>(0);
      v[e] = by & n ? moved : v[e];
    }
  }
  return col < cols ? v : V{};
}

// sixteen rows of w from class c on (the same in all lanes)
template <class S>
__device__ __forceinline__ const S* few_base(const FewArgs& a, int c) {
  return static_cast<const S*>(a.w) + static_cast<int64_t>(c) * a.w_ld;
}
template <class S>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t few_rows(const FewArgs& a, int c) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<S*>(few_base<S>(a, c)), 0, static_cast<int>(16 * a.w_ld * sizeof(S)), 0x00020000);
}

// A token's features: their offset, or -1 for one that is ignored or past the end
__device__ __forceinline__ int64_t few_token(const FewArgs& a, int t) {
  if (t >= a.k.t || a.k.target[t] == a.k.ignore) return -1;
  const int hi = t / a.hw;
  return hi * a.x_sn + (t - hi * a.hw) * a.x_sp;
}
// N channels of them, 0 past the end
template <class S, int N>
__device__ __forceinline__ auto few_x(const FewArgs& a, int64_t token, int c) {
  using V = __attribute__((ext_vector_type(N))) S;
  V v = {};
  if (token < 0 || c >= a.d) return v;
  const S* at = static_cast<const S*>(a.x) + token + c * a.x_sc;
  if (a.x_wide && c + N <= a.d) return *reinterpret_cast<const V*>(at);
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (c + e < a.d) v[e] = at[e * a.x_sc];
  return v;
}

// Sixteen classes' logits: lane (r, g) has the classes c .. c + 3, c = c0 + 4 g,
// of the tokens 16 j + r.  Bias, the logits' store, and the maximum and sum of
// each token, to red[token].
template <int NT>
__device__ __forceinline__ void few_logits_out(const FewArgs& a, f32x4 (&acc)[NT], int c, float2* red) {
  const int r = threadIdx.x & 15, v = a.k.v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float bias = a.bias && c + e < v ? a.bias[c + e] : 0.f;
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j][e] = c + e < v ? acc[j][e] + bias : -INFINITY;
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int t = 16 * j + r;
    if (t < a.k.t && a.logits && c < a.l_ld) *reinterpret_cast<f32x4*>(a.logits + t * a.l_ld + c) = acc[j];
    if (!a.part) continue;
    float m = fmaxf(fmaxf(acc[j][0], acc[j][1]), fmaxf(acc[j][2], acc[j][3]));
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    const float ref = m == -INFINITY ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) s += fast_exp(acc[j][e] - ref);
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 48) == 0) red[t] = make_float2(m, s);
    const int64_t y = t < a.k.t ? a.k.target[t] : -1;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (y == c + e && c + e < v) a.target_logit[t] = acc[j][e];
  }
}

// the sixteens of a workgroup joined
template <int NT>
__device__ __forceinline__ void few_part_out(const FewArgs& a, float2 (*red)[16 * NT], int n) {
  if (!a.part) return;
  __syncthreads();
  const int t = threadIdx.x;
  if (t >= a.k.t) return;
  float2 s = red[0][t];
  for (int w = 1; w < n; ++w) s = join(s, red[w][t]);
  a.part[static_cast<int64_t>(blockIdx.x) * a.k.t + t] = s;
}

// The logits of 128 or 64 classes, 16 a wave, with their statistics: a stream of
// w against the features in LDS, a chunk of the channels at a time.  Bound by
// memory: 1024 channels, 50000 classes, fp32, 16 tokens, the whole forward pass
// 49 us (w alone at 5 TB/s: 41); bf16 34 us (20).  8000 classes of 2048 channels
// keep too few CUs busy: 33 us (13).
template <class S, int NT, bool ODD>
__global__ __launch_bounds__(512) void few_logit_kernel(FewArgs a) {
  constexpr int N = 16 / sizeof(S), KS = 4 * N, U = 4;
  constexpr int KC = 4096 / (NT * static_cast<int>(sizeof(S))) / (KS * U) * (KS * U);   // (64 KB)
  static_assert(KC % (KS * U) == 0);
  using V = __attribute__((ext_vector_type(N))) S;
  // (rows sixteen bytes apart modulo the banks)
  __shared__ __align__(16) S xs[16 * NT][KC + N];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int threads = blockDim.x, c0 = blockIdx.x * (threads / 4) + wave * 16, v = a.k.v, d = a.d;
  const auto rows = few_rows<S>(a, c0);
  const S* base = few_base<S>(a, c0);
  const bool mine = c0 + r < v;
  const uint32_t at = static_cast<uint32_t>((r * a.w_ld + N * g) * sizeof(S));
  V cur[U];
  auto load = [&](int k, V (&to)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      to[u] = few_load<S, N, ODD>(rows, base, mine, at + static_cast<uint32_t>((k + u * KS) * sizeof(S)), k + u * KS + N * g, d);
  };
  load(0, cur);
  __shared__ int64_t token[16 * NT];
  if (tid < 16 * NT) token[tid] = few_token(a, tid);
  __syncthreads();
  f32x4 acc[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bool along = a.x_sc <= (a.hw == 1 ? a.x_sn : a.x_sp);
  for (int kc = 0; kc < d; kc += KC) {
    const int kn = min(KC, (d - kc + KS * U - 1) / (KS * U) * (KS * U));
    if (kc) __syncthreads();
    // (four pieces at a time, all fetched before the first is put away)
    const int row = kn / N, all = row * 16 * NT;
    for (int i0 = tid; i0 < all; i0 += 4 * threads) {
      V got[4];
      int t[4], k[4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int i = min(i0 + n * threads, all - 1);
        t[n] = along ? i / row : i % (16 * NT), k[n] = (along ? i - t[n] * row : i / (16 * NT)) * N;
        got[n] = few_x<S, N>(a, token[t[n]], kc + k[n]);
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) *reinterpret_cast<V*>(&xs[t[n]][k[n]]) = got[n];
    }
    __syncthreads();
    for (int k = 0; k < kn; k += KS * U) {
      V next[U];
      load(kc + k + KS * U, next);   // (nothing past the last channel)
      if (kc + k + KS * U > d) {
#pragma unroll
        for (int u = 0; u < U; ++u) cur[u] = few_tail(cur[u], kc + k + u * KS + N * g, d);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        V b[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) b[j] = *reinterpret_cast<const V*>(&xs[16 * j + r][k + u * KS + N * g]);
        if constexpr (sizeof(S) == 4) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(cur[u][e], b[j][e], acc[j], 0, 0, 0);
        } else {
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cur[u], b[j], acc[j], 0, 0, 0);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) cur[u] = next[u];
    }
  }
  __syncthreads();
  float2(*red)[16 * NT] = reinterpret_cast<float2(*)[16 * NT]>(&xs[0][0]);
  few_logits_out<NT>(a, acc, c0 + 4 * g, red[wave]);
  few_part_out<NT>(a, red, threads / 64);
}

// The same for fp32 and more tokens, where the fp32 instructions' rate would be
// the bound: w's values are split into three of bf16 as they come, x's were
// before (x: its planes, x_sn apart a token, x_sp a plane), and six products of
// them are summed.  32 classes a wave, whose values serve every sixteen tokens.
// 1024 channels, 50000 classes: 64 tokens 78 us for the forward pass, in fp32
// instructions 110; 128 tokens 116.
template <int NT>
__global__ __launch_bounds__(256, 2) void few_logit3_kernel(FewArgs a) {
  constexpr int U = 2, KS = 32, KC = 512 / NT / (KS * U) * (KS * U);
  __shared__ __align__(16) __bf16 xs[3][16 * NT][KC + 8];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c0 = blockIdx.x * 128 + wave * 32, v = a.k.v, d = a.d;
  const float* base = few_base<float>(a, c0);
  const auto rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base), 0, static_cast<int>(32 * a.w_ld * 4), 0x00020000);
  f32x4 cur[U][2][2];   // [step][sixteen classes][half]
  auto load = [&](int k, f32x4 (&to)[U][2][2]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int col = k + u * KS + 8 * g + 4 * h;
          to[u][i][h] = few_load<float, 4, false>(rows, base, c0 + 16 * i + r < v, static_cast<uint32_t>(((16 * i + r) * a.w_ld + col) * 4), col, d);
        }
  };
  load(0, cur);
  f32x4 acc[2][NT];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const __bf16* x = static_cast<const __bf16*>(a.x);
  const int dp = (d + 63) / 64 * 64;
  // x's next chunk, fetched during a chunk
  constexpr int PIECES = 3 * 16 * NT * (KC / 8) / 256;
  static_assert(3 * 16 * NT * (KC / 8) % 256 == 0);
  bf16x8 ahead[PIECES];
  auto fetch = [&](int kc) {
#pragma unroll
    for (int n = 0; n < PIECES; ++n) {
      const int i = n * 256 + tid, row = i / (KC / 8), k = kc + i % (KC / 8) * 8, p = row / (16 * NT), t = row % (16 * NT);
      ahead[n] = bf16x8{};
      if (t < a.k.t && k < dp) ahead[n] = *reinterpret_cast<const bf16x8*>(x + p * a.x_sp + t * a.x_sn + k);
    }
  };
  fetch(0);
  for (int kc = 0; kc < dp; kc += KC) {
    const int kn = min(KC, dp - kc);
    if (kc) __syncthreads();
#pragma unroll
    for (int n = 0; n < PIECES; ++n) {
      const int i = n * 256 + tid, row = i / (KC / 8);
      *reinterpret_cast<bf16x8*>(&xs[row / (16 * NT)][row % (16 * NT)][i % (KC / 8) * 8]) = ahead[n];
    }
    __syncthreads();
    fetch(kc + KC);
    for (int k = 0; k < kn; k += KS * U) {
      f32x4 next[U][2][2];
      load(kc + k + KS * U, next);   // (nothing past the last channel)
      if (kc + k + KS * U > d) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) cur[u][i][h] = few_tail(cur[u][i][h], kc + k + u * KS + 8 * g + 4 * h, d);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        bf16x8 w[2][3];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            __bf16 q[3];
            bf16_planes<3>(cur[u][i][e / 4][e % 4], q);
#pragma unroll
            for (int p = 0; p < 3; ++p) w[i][p][e] = q[p];
          }
        // (two sixteens of tokens in turn: four sums, so that none waits for itself)
#pragma unroll
        for (int j0 = 0; j0 < NT; j0 += 2) {
          bf16x8 b[2][3];
#pragma unroll
          for (int j = j0; j < NT && j < j0 + 2; ++j)
#pragma unroll
            for (int p = 0; p < 3; ++p) b[j - j0][p] = *reinterpret_cast<const bf16x8*>(&xs[p][16 * j + r][k + u * KS + 8 * g]);
          // (the smallest products first)
#pragma unroll
          for (int p = 2; p >= 0; --p)
#pragma unroll
            for (int q = 0; q <= p; ++q)
#pragma unroll
              for (int j = j0; j < NT && j < j0 + 2; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                  acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[i][q], b[j - j0][p - q], acc[i][j], 0, 0, 0);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) cur[u][i][h] = next[u][i][h];
    }
  }
  __syncthreads();
  float2(*red)[16 * NT] = reinterpret_cast<float2(*)[16 * NT]>(&xs[0][0][0]);
#pragma unroll
  for (int i = 0; i < 2; ++i) few_logits_out<NT>(a, acc[i], c0 + 16 * i + 4 * g, red[2 * wave + i]);
  few_part_out<NT>(a, red, 8);
}

// G of 64 classes at a time in LDS; each wave has 16 C channels, for which it adds
// G w to dx's sums in registers and stores G^T x.  bf16 operands: G is rounded
// to bf16, as by the products (db is summed before), a lane gives four tokens or classes to one
// instruction, and the four channels that it loads of each of four classes are
// turned in its registers.  Bound by memory up to 16 tokens (1024 channels, 50000
// classes, fp32: about 75 us for w read and dw written, 5.4 TB/s), by the fp32
// instructions' rate from there on (64 tokens: 140 us, 0.1 PFLOP/s).
template <class S, int NT>
struct FewG {   // [class][token] for dw, [token][class] for dx
  __bf16 by_class[64][16 * NT + 4], by_token[16 * NT][64 + 4];
};
template <int NT>
struct FewG<float, NT> {
  float by_class[64][16 * NT + 4];
};

template <class S, int NT, int C, bool ODD>
__global__ __launch_bounds__(256, 2) void few_grad_kernel(FewArgs a) {
  using S4 = __attribute__((ext_vector_type(4))) S;
  using SC = __attribute__((ext_vector_type(C))) S;
  static_assert(C == 4 || sizeof(S) == 4);
  constexpr bool F = sizeof(S) == 4;
  __shared__ __align__(16) FewG<S, NT> gs[2];
  __shared__ float db_part[2][4][64];
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int group = blockIdx.x % a.groups, split = blockIdx.x / a.groups;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col0 = (group * 4 + wave) * 16 * C, col = col0 + C * r, v = a.k.v, d = a.d;
  const bool on = col0 < d, dx = a.slab && on, dw = a.dw && on, db = a.db && group == 0;
  const int blocks = (v + 15) / 16;
  const int b0 = static_cast<int>(static_cast<int64_t>(blocks) * split / a.splits);
  const int b1 = static_cast<int>(static_cast<int64_t>(blocks) * (split + 1) / a.splits);
  const float scale = common_scale(a.k);
  // a lane's class of load s: 4 s + g, bf16 4 g + s
  constexpr int kG = F ? 1 : 4, kS = F ? 4 : 1;
  const uint32_t at = static_cast<uint32_t>((kG * g * a.w_ld + col) * sizeof(S));
  auto load = [&](int b, SC (&to)[4]) {
    const auto rows = few_rows<S>(a, 16 * b);
#pragma unroll
    for (int s = 0; s < 4; ++s)
      to[s] = few_load<S, C, ODD>(rows, few_base<S>(a, 16 * b), b < b1 && 16 * b + kS * s + kG * g < v,
                                  at + static_cast<uint32_t>(kS * s * a.w_ld * sizeof(S)), col, d);
  };
  SC cur[4] = {};
  if (dx) load(b0, cur);
  // this thread's part of G: classes 4 q + 0..3 of a chunk, the tokens t0 + 16 i
  const int q = tid & 15, t0 = tid >> 4;
  float lse[NT], factor[NT];
  int64_t target[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int t = t0 + 16 * i;
    lse[i] = factor[i] = 0.f, target[i] = -1;
    if (t < a.k.t) {
      const int64_t y = a.k.target[t];
      const float weight = a.k.class_weight && y >= 0 && y < v ? a.k.class_weight[y] : 1.f;
      lse[i] = a.k.stats[t], target[i] = y;
      factor[i] = token_scale(a.k, y, weight, a.k.grad && a.k.grad_each ? a.k.grad[t] : 1.f);
    }
  }
  f32x4 logit[NT];
  auto fetch = [&](int b) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int t = t0 + 16 * i, c = 16 * b + 4 * q;
      logit[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (t < a.k.t && c < 16 * b1) logit[i] = *reinterpret_cast<const f32x4*>(a.logits + t * a.l_ld + c);
    }
  };
  fetch(b0);
  // x: a lane's four channels of the tokens 16 i + 4 s + g, bf16 16 i + 4 g + s
  SC x[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
#pragma unroll
    for (int s = 0; s < 4; ++s) x[i][s] = dw ? few_x<S, C>(a, few_token(a, 16 * i + kS * s + kG * g), col) : SC{};
  }
  // four values of each of four rows -> of each of four columns
  [[maybe_unused]] auto turn = [](const auto (&u)[4], S4 (&to)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) to[e] = S4{u[0][e], u[1][e], u[2][e], u[3][e]};
  };
  if constexpr (!F) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      S4 to[4];
      turn(x[i], to);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] = to[e];
    }
  }
  f32x4 sum[NT][C];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < C; ++e) sum[j][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  using I4 = __attribute__((ext_vector_type(4))) short;
  [[maybe_unused]] auto product = [](auto m, auto n, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(I4, m), __builtin_bit_cast(I4, n), c, 0, 0, 0);
  };

  int buf = 0;
  for (int b = b0; b < b1; b += 4, buf ^= 1) {
    FewG<S, NT>& now = gs[buf];
    f32x4 all = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      f32x4 p;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = 16 * b + 4 * q + e;
        p[e] = fast_exp(logit[i][e] - lse[i]) * factor[i];
        if (target[i] == c) p[e] -= factor[i];
        p[e] = factor[i] != 0.f && c < v ? p[e] : 0.f;
        now.by_class[4 * q + e][t0 + 16 * i] = static_cast<S>(p[e]);
      }
      all += p;
      if constexpr (!F)
        *reinterpret_cast<S4*>(&now.by_token[t0 + 16 * i][4 * q]) =
            S4{static_cast<S>(p[0]), static_cast<S>(p[1]), static_cast<S>(p[2]), static_cast<S>(p[3])};
    }
    if (db) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        all[e] += __shfl_xor(all[e], 16);
        all[e] += __shfl_xor(all[e], 32);
      }
      if (lane < 16) *reinterpret_cast<f32x4*>(&db_part[buf][wave][4 * q]) = all;
    }
    fetch(b + 4);
    __syncthreads();   // (the other half is written again after the next one)
    if (db && tid < 64 && tid < 16 * (b1 - b) && 16 * b + tid < v)
      a.db[16 * b + tid] = (db_part[buf][0][tid] + db_part[buf][1][tid] + db_part[buf][2][tid] + db_part[buf][3][tid]) * scale;
    if (!on) continue;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      if (b + n >= b1) break;
      SC next[4] = {};
      if (dx) load(b + n + 1, next);
      if (dw) {
        f32x4 out[C];
#pragma unroll
        for (int e = 0; e < C; ++e) out[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          if constexpr (F) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
              const float m = now.by_class[16 * n + r][16 * i + 4 * s + g];
#pragma unroll
              for (int e = 0; e < C; ++e) out[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(m, x[i][s][e], out[e], 0, 0, 0);
            }
          } else {
            const S4 m = *reinterpret_cast<const S4*>(&now.by_class[16 * n + r][16 * i + 4 * g]);
#pragma unroll
            for (int e = 0; e < C; ++e) out[e] = product(m, x[i][e], out[e]);
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = 16 * (b + n) + 4 * g + e;
          if (c >= v || col >= d) continue;
          S* to = static_cast<S*>(a.dw) + static_cast<int64_t>(c) * d + col;
          SC o;
#pragma unroll
          for (int f = 0; f < C; ++f) o[f] = static_cast<S>(out[f][e] * scale);
          if (col + C <= d) {
            using U = __attribute__((ext_vector_type(C), aligned(sizeof(S)))) S;
            *reinterpret_cast<U*>(to) = o;
          } else {
#pragma unroll
            for (int f = 0; f < C; ++f)
              if (col + f < d) to[f] = o[f];
          }
        }
      }
      if (dx) {
        if (col0 + 16 * C > d) {
#pragma unroll
          for (int s = 0; s < 4; ++s) cur[s] = few_tail(cur[s], col, d);
        }
        if constexpr (F) {
#pragma unroll
          for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              const float m = now.by_class[16 * n + 4 * s + g][16 * j + r];
#pragma unroll
              for (int e = 0; e < C; ++e) sum[j][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(m, cur[s][e], sum[j][e], 0, 0, 0);
            }
        } else {
          S4 w[4];
          turn(cur, w);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const S4 m = *reinterpret_cast<const S4*>(&now.by_token[16 * j + r][16 * n + 4 * g]);
#pragma unroll
            for (int e = 0; e < C; ++e) sum[j][e] = product(m, w[e], sum[j][e]);
          }
        }
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) cur[s] = next[s];
    }
  }
  if (!dx || col >= a.slab_ld) return;
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = 16 * j + 4 * g + e;
      if (t >= a.k.t) continue;
      __attribute__((ext_vector_type(C))) float o;
#pragma unroll
      for (int f = 0; f < C; ++f) o[f] = sum[j][f][e];
      *reinterpret_cast<decltype(o)*>(a.slab + (static_cast<int64_t>(split) * a.k.t + t) * a.slab_ld + col) = o;
    }
}

// dx of few tokens: 16 pieces of four channels a workgroup, 16 threads each
// taking every 16th partial sum
template <class O>
__global__ __launch_bounds__(256) void few_sum_kernel(Slab s, Tokens k) {
  __shared__ f32x4 got[16][16];
  const int u = threadIdx.x & 15, w = threadIdx.x >> 4;
  const int64_t n4 = s.ld / 4, i = blockIdx.x * 16ll + u, c = i / n4, r = (i - c * n4) * 4;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  if (c < s.n) {
#pragma unroll 4
    for (int q = w; q < s.splits; q += 16) x += *reinterpret_cast<const f32x4*>(s.at + (static_cast<int64_t>(q) * s.n + c) * s.ld + r);
  }
  got[w][u] = x;
  __syncthreads();
  if (w || c >= s.n) return;
#pragma unroll
  for (int q = 1; q < 16; ++q) x += got[q][u];
  store4<O>(s.map, static_cast<int>(r), static_cast<int>(c), s.m, x * common_scale(k));
}
