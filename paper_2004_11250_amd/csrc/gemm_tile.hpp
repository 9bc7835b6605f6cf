// gemm_tile.hpp -- the matrix-core product the training operators are built on:
//
//   acc[r][c] = sum over plane pairs (p, q), sum over k of A_p[r][k] B_q[c][k]
//
// Each operand is stored either with k contiguous ([row][k]) or by rows of k
// ([k][row]), so that no operand has to be kept in two orders.  16-bit operands
// multiply at the full matrix-core rate; an operand that needs more bits than
// one 16-bit value holds is stored as a sum of two or three such values
// ("planes", the first the rounded value, the next the rounded rest), and the
// product is the sum of the plane products that matter, taken one after the
// other along a longer k into the same fp32 accumulators.
//
// A workgroup owns a BM x BN tile and walks k in steps of 64.  A step's
// operands go from global memory straight into LDS (16 bytes a lane; no
// registers), steps ahead of the products.  Two layouts there:
//   k contiguous: a row of 64 values is 128 bytes; its 16-byte pieces lie at
//     position piece ^ (row & 7), so that the eight rows that an eighth of a
//     wave reads at once lie in different banks.
//   rows of k: a k holds BM (BN) values; 32-byte pieces of 16 rows lie at
//     position piece ^ swizzle(k), so that the eight k that are read at once
//     do, and the hardware's transposing LDS read gives each lane four k of
//     its row.
// The permutation is applied to the global address, since the LDS side of the
// DMA is fixed (lane after lane).  What lies past an operand's end is read
// through an offset outside the descriptor's range, which gives zeros.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace pp {

using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using f32x4 = __attribute__((ext_vector_type(4))) float;
using u32x4_t = __attribute__((ext_vector_type(4))) uint32_t;

constexpr int kBK = 64;              // k per step; operands are padded with zeros to a multiple of it
constexpr int kMaxPlanes = 3;
constexpr int64_t kMaxLd = 1 << 22;  // pitch limit: a tile stays within 31-bit byte offsets

// One operand: up to three planes of [rows][ld] with k contiguous and padded
// with zeros to whole steps, or of [k][ld] with rows contiguous, rows a
// multiple of 8.  16-byte aligned, ld a multiple of 8.
struct GemmOperand {
  const void* plane[kMaxPlanes];
  int64_t ld;
  int32_t rows;
  int32_t k;      // rows of k that are there (the second form)
};

// Which planes are multiplied, in order (the smallest products first, so that
// they are added while the sum is small): two bits of A's plane, two of B's.
struct PlanePairs {
  uint32_t code;
  int32_t n;
};
constexpr uint32_t plane_pair(int p, int q, int i) { return static_cast<uint32_t>(p | q << 2) << (4 * i); }
// one plane each: 16-bit operands
constexpr PlanePairs kPairs1 = {plane_pair(0, 0, 0), 1};
// two planes each; what is left out is the product of the two rests
constexpr PlanePairs kPairs3 = {plane_pair(1, 0, 0) | plane_pair(0, 1, 1) | plane_pair(0, 0, 2), 3};
// three bf16 planes each hold all 24 bits of an fp32 value; what is left out
// is 2^-24 of the product and less
constexpr PlanePairs kPairs6 = {plane_pair(2, 0, 0) | plane_pair(0, 2, 1) | plane_pair(1, 1, 2) | plane_pair(1, 0, 3) |
                                    plane_pair(0, 1, 4) | plane_pair(0, 0, 5), 6};

template <class T>
struct Mfma;
template <>
struct Mfma<__bf16> {
  using Frag = bf16x8;
  static __device__ __forceinline__ f32x4 mul(Frag a, Frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mfma<_Float16> {
  using Frag = f16x8;
  static __device__ __forceinline__ f32x4 mul(Frag a, Frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// 16 bytes a lane from base + voff + soff to LDS byte lds + 16 lane.  As
// assembly: the compiler would otherwise wait for every DMA in flight before
// any LDS read that follows.
__device__ __forceinline__ void gemm_dma(u32x4_t rsrc, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "s"(lds)
               : "memory", "m0");
}
#pragma clang diagnostic pop
// the wave's DMAs have landed and its LDS reads are done; then all waves meet
__device__ __forceinline__ void gemm_sync() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A value that is the same in all lanes, in scalar registers.
__device__ __forceinline__ uint64_t uniform64(uint64_t v) {
  return static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32))) << 32 |
         static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)));
}

// The plane products of operands of n planes each, in the order in which they
// are added (as kPairs1, 3 and 6).
struct PlanePair {
  int a, b;
};
template <int N>
struct PlaneProducts;
template <>
struct PlaneProducts<1> {
  static constexpr int COUNT = 1;
  static constexpr PlanePair LIST[] = {{0, 0}};
};
template <>
struct PlaneProducts<2> {
  static constexpr int COUNT = 3;
  static constexpr PlanePair LIST[] = {{1, 0}, {0, 1}, {0, 0}};
};
template <>
struct PlaneProducts<3> {
  static constexpr int COUNT = 6;
  static constexpr PlanePair LIST[] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
};

template <class T, int BM_, int BN_, int WM_, int WN_, int STAGES_, int WK_ = 1, bool PHASED_ = false, bool AR_ = false,
          bool BR_ = false, int NP_ = 1, int CR_ = 64>
struct GemmTile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int STAGES = STAGES_;                // steps held in LDS
  static constexpr bool PHASED = PHASED_;
  static constexpr bool AR = AR_, BR = BR_;             // the operand is stored by rows of k
  // Planes of each operand that a step brings; it makes all their products.
  // 1: one plane pair after the other along a longer k, as run() is told.
  static constexpr int NP = NP_;
  // WK groups of WM x WN waves: each takes every WK-th step, on operands of its
  // own, and the groups' sums are added in LDS at the end
  static constexpr int WK = WK_, NW = WM * WN, THREADS = NW * WK * 64;
  static constexpr int TM = BM / WM, TN = BN / WN;      // a wave's part
  static constexpr int FM = TM / 16, FN = TN / 16;      // in 16 x 16 blocks
  static constexpr int QA = BM / (8 * NW), QB = BN / (8 * NW);   // DMAs a wave issues for a step
  static constexpr uint32_t PLANE_A = BM * kBK * 2, PLANE_B = BN * kBK * 2, LDS_A = NP * PLANE_A, LDS_STEP = NP * (PLANE_A + PLANE_B);
  static constexpr uint32_t LDS_RING = STAGES * LDS_STEP, LDS_BYTES = WK * LDS_RING;
  static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && TM % 16 == 0 && TN % 16 == 0, "tile");
  static_assert((!AR || (FM & (FM - 1)) == 0) && (!BR || (FN & (FN - 1)) == 0) && FM <= 8 && FN <= 8, "blocks");

  // Row and column of acc[i][j][e] in the tile.  A lane holds four rows that
  // follow each other of one column.
  static __device__ __forceinline__ int row_of(int i) { return (wave() / WN) * TM + 16 * i + (lane() >> 4) * 4; }
  static __device__ __forceinline__ int col_of(int j) { return (wave() % WN) * TN + 16 * j + (lane() & 15); }
  static __device__ __forceinline__ int lane() { return threadIdx.x & 63; }
  // the wave's place in its group, and its group
  static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % NW; }
  static __device__ __forceinline__ int group() { return WK == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / NW; }

  using Frag = typename Mfma<T>::Frag;

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Wint-to-pointer-cast"   // (LDS addresses are 32 bits; the host pass does not know)
  // One operand's DMAs and LDS reads; E: rows of the tile, Q: DMAs a wave
  // issues for a step, R: stored by rows of k.
  template <int E, int Q, bool R, int TW>
  struct Side {
    static constexpr int LPR = R ? E / 8 : 8, RPI = 64 / LPR;   // lanes a stored row takes, stored rows a DMA brings
    uint64_t base[kMaxPlanes];
    int64_t step, left;       // bytes from a step to the next; bytes from the first step on (rows of k)
    int64_t now;              // bytes from the first step to the next one
    uint32_t off[Q];          // per lane
    uint32_t at;              // of this lane's LDS reads

    static __device__ __forceinline__ int swizzle(int k) {
      return E >= 128 ? (k & 3) | (k >> 3 & 1) << 2 : E == 64 ? (k >> 1 & 1) | (k >> 3 & 1) << 1 : k >> 3 & 1;
    }
    // first: first row of the tile; which(i): the group of eight rows (k
    // contiguous) that DMA i of this wave brings; wrow: first row of the
    // wave's part
    template <class F>
    __device__ __forceinline__ void init(const GemmOperand& o, int first, int wrow, F&& which) {
      const int ln = lane();
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        const int r = RPI * which(i) + ln / LPR, pos = ln % LPR;
        if constexpr (R) {
          const int piece = ((pos >> 1 ^ swizzle(r)) << 1 | (pos & 1)) * 8;
          off[i] = first + piece < o.rows ? static_cast<uint32_t>((r * static_cast<int>(o.ld) + piece) * 2) : 0x80000000u;
        } else {
          off[i] = first + r < o.rows ? static_cast<uint32_t>(r * static_cast<int>(o.ld) * 2 + (pos ^ (r & 7)) * 16) : 0x80000000u;
        }
      }
#pragma unroll
      for (int q = 0; q < kMaxPlanes; ++q)
        base[q] = uniform64(reinterpret_cast<uint64_t>(o.plane[q]) + 2 * static_cast<uint64_t>(R ? first : first * o.ld));
      step = static_cast<int64_t>(uniform64(R ? kBK * 2 * o.ld : kBK * 2));
      left = static_cast<int64_t>(uniform64(2 * (o.k * o.ld - first)));
      if constexpr (R) {
        // (k = 8 (lane / 16) + lane % 16 / 4, four rows from 4 (lane % 4) on)
        const int k = 8 * (ln >> 4) + (ln >> 2 & 3);
        at = static_cast<uint32_t>(k * (E * 2) + ((wrow / 16) ^ swizzle(k)) * 32 + (ln & 3) * 8);
      } else {
        // row lane % 16, piece lane / 16
        at = static_cast<uint32_t>((wrow + (ln & 15)) * 128 + ((ln >> 4) ^ (ln & 7)) * 16);
      }
    }
    // The descriptor's base is a sum taken in scalar registers, so a DMA has no
    // vector instruction's result to wait for.
    __device__ __forceinline__ u32x4_t rsrc(uint32_t plane) const {
      const uint64_t b = (plane == 0 ? base[0] : plane == 1 ? base[1] : base[2]) + static_cast<uint64_t>(now);
      u32x4_t r;
      r.x = static_cast<uint32_t>(b);
      r.y = static_cast<uint32_t>(b >> 32) & 0xFFFFu;
      r.z = 0x7FFFFFFFu;
      if constexpr (R) {   // (k past the end reads zeros)
        const int64_t rest = left - now;
        r.z = rest <= 0 ? 0u : rest < 0x7FFFFFFF ? static_cast<uint32_t>(rest) : 0x7FFFFFFFu;
      }
      r.w = 0x00020000u;
      return r;
    }
    // operand block i (16 rows of the wave's part), half h of the step's k,
    // from the operand's place `buf` in LDS
    // (constant parts are added to a pointer, so that they become the reads'
    // immediate offsets)
    __device__ __forceinline__ Frag read(uint32_t buf, int i, int h) const {
      using Bytes = const __attribute__((address_space(3))) uint8_t*;
      if constexpr (R) {
        using Half = __attribute__((ext_vector_type(4))) short;
        using Ptr = __attribute__((address_space(3))) Half*;
        const Bytes p = (Bytes)(buf + (at ^ (i * 32u)));
        const Half lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(p + h * (32 * E * 2)));
        const Half hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(p + h * (32 * E * 2) + 4 * E * 2));
        return __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      } else {
        const Bytes p = (Bytes)(buf + (at ^ (h * 64u)));
        return *(const __attribute__((address_space(3))) Frag*)(p + i * 2048);
      }
    }
  };

#pragma clang diagnostic pop

  struct Feed {
    Side<BM, QA, AR, TM> a;
    Side<BN, QB, BR, TN> b;
    u32x4_t ra[NP], rb[NP];
    uint32_t code;
    int ksteps, pair, kk, wv;

    __device__ __forceinline__ Feed(const GemmOperand& A, const GemmOperand& B, PlanePairs pairs, int row0, int col0,
                                    int ksteps_, int s0) {
      wv = wave();
      a.init(A, row0, (wv / WN) * TM, [&](int i) { return group_a(i, wv); });
      b.init(B, col0, (wv % WN) * TN, [&](int i) { return group_b(i, wv); });
      b.at += LDS_A;   // (a multiple of a kilobyte: the permutations are of lower bits)
      code = pairs.code;
      ksteps = __builtin_amdgcn_readfirstlane(ksteps_);
      pair = s0 / ksteps, kk = s0 - pair * ksteps;
      a.now = kk * a.step, b.now = kk * b.step;
    }
    // descriptors of the next step
    __device__ __forceinline__ void next() {
      if constexpr (NP > 1) {
#pragma unroll
        for (int q = 0; q < NP; ++q) ra[q] = a.rsrc(q), rb[q] = b.rsrc(q);
        a.now += WK * a.step, b.now += WK * b.step;
      } else {
        ra[0] = a.rsrc(code >> (4 * pair) & 3), rb[0] = b.rsrc(code >> (4 * pair + 2) & 3);
        kk += WK;
        if (kk < ksteps) {
          a.now += WK * a.step, b.now += WK * b.step;
        } else {   // the next plane pair
          while (kk >= ksteps) kk -= ksteps, ++pair;
          a.now = kk * a.step, b.now = kk * b.step;
        }
      }
    }
    template <int I>
    __device__ __forceinline__ void dma_a(uint32_t buf) const {
#pragma unroll
      for (int q = 0; q < NP; ++q) gemm_dma(ra[q], a.off[I], buf + q * PLANE_A + 1024u * group_a(I, wv));
    }
    template <int I>
    __device__ __forceinline__ void dma_b(uint32_t buf) const {
#pragma unroll
      for (int q = 0; q < NP; ++q) gemm_dma(rb[q], b.off[I], buf + LDS_A + q * PLANE_B + 1024u * group_b(I, wv));
    }
    template <int I = 0>
    __device__ __forceinline__ void all(uint32_t buf) const {
      if constexpr (I < QA) dma_a<I>(buf);
      if constexpr (I < QB) dma_b<I>(buf);
      if constexpr (I + 1 < QA || I + 1 < QB) all<I + 1>(buf);
    }
  };
  // Which kilobyte of the operand's place DMA i of wave w brings.  In the
  // phased loop, k contiguous: DMAs 0 and 1 bring the halves of every wave's
  // rows (columns) that its first products read, 2 and 3 the others.
  static __device__ __forceinline__ int group_a(int i, int w) {
    if constexpr (PHASED && !AR) return (i & 1) * (TM / 8) + (i >> 1) * (TM / 16) + w;
    return NW * i + w;
  }
  static __device__ __forceinline__ int group_b(int i, int w) {
    if constexpr (PHASED && !BR) return (2 * (i & 1) + (w >> 2)) * (TN / 8) + (i >> 1) * (TN / 16) + (w & 3);
    return NW * i + w;
  }

  // how many steps a product of ksteps k steps takes
  static __device__ __forceinline__ int steps_of(int ksteps, PlanePairs pairs) { return NP > 1 ? ksteps : ksteps * pairs.n; }

  // steps [s0, s1) of the flattened (plane pair, k step) range; ksteps k steps
  // a pair.  lds: LDS_BYTES of shared memory.
  static __device__ __forceinline__ void run(const GemmOperand& A, const GemmOperand& B, PlanePairs pairs, int row0,
                                             int col0, int ksteps, int s0, int s1, uint8_t* lds, f32x4 (&acc)[FM][FN]) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    s0 = __builtin_amdgcn_readfirstlane(s0), s1 = __builtin_amdgcn_readfirstlane(s1);
    if (s0 >= s1) return;
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)lds));
    const int g = group();
    Feed feed(A, B, pairs, row0, col0, ksteps, s0 + g);
    if constexpr (PHASED)
      phased(feed, s1 - s0, lds0, acc);
    else
      ring(feed, s1 - s0, g, lds0 + g * LDS_RING, acc);
  }

  // A ring of STAGES steps a group, STAGES - 1 of them in flight; one barrier
  // for a step of every group.
  static __device__ __forceinline__ void ring(Feed& feed, int steps, int g, uint32_t lds0, f32x4 (&acc)[FM][FN]) {
    const int rounds = (steps + WK - 1) / WK, n = WK == 1 ? steps : (steps - g + WK - 1) / WK;   // this group's steps
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
      if (i < n) {
        feed.next();
        feed.all(lds0 + i * LDS_STEP);
      }
    uint32_t cur = 0;                              // the step's place in the ring
    uint32_t put = (STAGES - 1) * LDS_STEP;        // where the step STAGES - 1 on goes: the last one's place
    for (int s = 0; s < rounds; ++s) {
      // this step has landed once at most the later ones' DMAs are in flight
      if (s + STAGES - 1 <= n)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * NP * (QA + QB)) : "memory");
      else
        gemm_sync();
      if (s + STAGES - 1 < n) {
        feed.next();
        feed.all(lds0 + put);
      }
      if (WK > 1 && s >= n) break;   // (the last round, for groups without a step in it)
      const uint32_t la = lds0 + cur;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Frag a[NP][FM], b[NP][FN];
#pragma unroll
        for (int q = NP - 1; q >= 0; --q) {
#pragma unroll
          for (int j = 0; j < FN; ++j) b[q][j] = feed.b.read(la + q * PLANE_B, j, h);
#pragma unroll
          for (int i = 0; i < FM; ++i) a[q][i] = feed.a.read(la + q * PLANE_A, i, h);
        }
#pragma unroll
        for (int k = 0; k < PlaneProducts<NP>::COUNT; ++k)
#pragma unroll
          for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
              acc[i][j] = Mfma<T>::mul(a[PlaneProducts<NP>::LIST[k].a][i], b[PlaneProducts<NP>::LIST[k].b][j], acc[i][j]);
      }
      put = cur;
      cur = cur + LDS_STEP == LDS_RING ? 0 : cur + LDS_STEP;
    }
  }

  // Two groups of four waves, one wave of each on every SIMD, half a phase
  // apart: while one group's waves feed the matrix cores, the other's read
  // their next operands from LDS and start DMAs.  A step is four phases, each
  // a quarter of the wave's tile (2 x 2 blocks of FM/2 x FN/2) over the whole
  // step's k.  What has been read is overwritten from the next phase on by the
  // step after next, so that a DMA has a step and more to land.
  static __device__ __forceinline__ void phased(Feed& feed, int n, uint32_t lds0, f32x4 (&acc)[FM][FN]) {
    static_assert(!PHASED || (NP == 1 && NW == 8 && WK == 1 && STAGES == 2 && QA == 4 && QB == 4 && FM == 8 && FN == 4), "phases");
    const int wv = wave();
    constexpr int HM = FM / 2, HN = FN / 2;
    auto fetch = [&](uint32_t buf) {   // (columns first: the counts below)
      feed.next();
      feed.template dma_b<0>(buf), feed.template dma_b<1>(buf), feed.template dma_b<2>(buf), feed.template dma_b<3>(buf);
      feed.template dma_a<0>(buf), feed.template dma_a<1>(buf), feed.template dma_a<2>(buf), feed.template dma_a<3>(buf);
    };
    fetch(lds0);
    if (n > 1) {
      fetch(lds0 + LDS_STEP);
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(QA + QB) : "memory");
    } else {
      gemm_sync();
    }
    if (wv >= 4) asm volatile("s_barrier" ::: "memory");
    uint32_t cur = lds0;
    Frag a[2][HM], b0[2][HN], b1[2][HN];
    auto read_a = [&](int half) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < HM; ++i) a[h][i] = feed.a.read(cur, half * HM + i, h);
    };
    auto read_b = [&](uint32_t buf, int half, Frag (&b)[2][HN]) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < HN; ++j) b[h][j] = feed.b.read(buf, half * HN + j, h);
    };
    auto products = [&](int mh, int nh, const Frag (&b)[2][HN]) {
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < HM; ++i)
#pragma unroll
          for (int j = 0; j < HN; ++j)
            acc[mh * HM + i][nh * HN + j] = Mfma<T>::mul(a[h][i], b[h][j], acc[mh * HM + i][nh * HN + j]);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_barrier" ::: "memory");
    };
    for (int s = 0; s < n; ++s) {
      const bool more = s + 2 < n;
      read_b(cur, 0, b0);
      read_a(0);
      products(0, 0, b0);
      read_b(cur, 1, b1);
      if (more) {
        feed.next();
        if constexpr (!AR) feed.template dma_a<0>(cur), feed.template dma_a<1>(cur);
        if constexpr (!BR) feed.template dma_b<0>(cur), feed.template dma_b<1>(cur);
      }
      products(0, 1, b1);
      read_a(1);
      if (more) {
        if constexpr (BR) feed.template dma_b<0>(cur), feed.template dma_b<1>(cur);
        feed.template dma_b<2>(cur), feed.template dma_b<3>(cur);
      }
      products(1, 1, b1);
      if (more) {
        if constexpr (AR) feed.template dma_a<0>(cur), feed.template dma_a<1>(cur);
        feed.template dma_a<2>(cur), feed.template dma_a<3>(cur);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(QA + QB) : "memory");   // the next step has landed
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      products(1, 0, b0);
      cur = lds0 + (LDS_STEP - (cur - lds0));
    }
    if (wv < 4) asm volatile("s_barrier" ::: "memory");
  }

  // After run(), for what is done with the accumulators in registers: the
  // groups' sums in the first group's, zeros in the others'.
  static __device__ __forceinline__ void reduce(uint8_t* lds, f32x4 (&acc)[FM][FN]) {
    if constexpr (WK > 1) {
      gemm_sync();   // (every wave is done with the operands)
      const int g = group();
      f32x4* at = reinterpret_cast<f32x4*>(lds) + (wave() * FM * FN) * 64 + lane();
      constexpr int STRIDE = NW * FM * FN * 64;
      if (g > 0) {
#pragma unroll
        for (int k = 0; k < FM * FN; ++k) {
          at[(g - 1) * STRIDE + k * 64] = acc[k / FN][k % FN];
          acc[k / FN][k % FN] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
      }
      gemm_sync();
      if (g == 0) {
#pragma unroll
        for (int k = 0; k < FM * FN; ++k)
#pragma unroll
          for (int q = 0; q < WK - 1; ++q) acc[k / FN][k % FN] += at[q * STRIDE + k * 64];
      }
    }
  }

  // After run(): the accumulators by way of LDS, for stores along columns or
  // rows (a lane holds four rows of a column, too short a piece for either).  Each wave has a region of its own, of CR x CC values; f(row,
  // col, View) is called for each CR x CC part of the wave's tile, whose first
  // element is (row, col) of the workgroup's tile.
  static constexpr int CR = TM % 64 == 0 && CR_ >= 64 ? 64 : TM % 32 == 0 ? 32 : 16, CC = TN;
  // pieces of eight values a lane takes (a small part has work for SHARERS
  // groups only)
  static constexpr int SHARERS = CR * CC / 512 < WK ? CR * CC / 512 : WK, PIECES = CR * CC / 512 / SHARERS;
  static constexpr uint32_t STAGING = CR * CC * 4 * NW * WK;   // bytes of LDS
  static_assert(CC <= 64 && STAGING <= LDS_BYTES && (WK == 1 || TM <= 64), "staging area");
  struct View {
    float* at;
    // Element (r, c): columns one after the other, rows in groups of four
    // (what a lane's accumulator holds) that are turned round with the column,
    // so that 16 lanes with one row group of 16 columns reach all banks.
    static __device__ __forceinline__ int place(int r, int c) { return c * CR + ((r >> 2 ^ (c & (CR / 4 - 1))) << 2) + (r & 3); }
    // how many pieces this lane takes
    static __device__ __forceinline__ int pieces() { return SHARERS == WK || group() < SHARERS ? PIECES : 0; }
    // the i-th of them: eight rows of a column ...
    static __device__ __forceinline__ void col_piece(int i, int* r, int* c) {
      const int k = (i * SHARERS + group()) * 64 + lane();
      *c = k / (CR / 8), *r = k % (CR / 8) * 8;
    }
    // ... or eight columns of a row
    static __device__ __forceinline__ void row_piece(int i, int* r, int* c) {
      const int k = (i * SHARERS + group()) * 64 + lane();
      *r = k / (CC / 8), *c = k % (CC / 8) * 8;
    }
    __device__ __forceinline__ void col(int r, int c, float (&v)[8]) const {
      const f32x4 a = *reinterpret_cast<const f32x4*>(at + place(r, c)), b = *reinterpret_cast<const f32x4*>(at + place(r + 4, c));
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
    }
    __device__ __forceinline__ void put_col(int r, int c, const float (&v)[8]) const {
      *reinterpret_cast<f32x4*>(at + place(r, c)) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4*>(at + place(r + 4, c)) = f32x4{v[4], v[5], v[6], v[7]};
    }
    __device__ __forceinline__ void row(int r, int c, float (&v)[8]) const {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = at[place(r, c + e)];
    }
    // what lanes wrote is read by others from here on (one wave's LDS
    // accesses are done in order: only the compiler has to keep it)
    static __device__ __forceinline__ void turn() {
      if constexpr (WK > 1) {
        gemm_sync();   // (the groups share a region)
      } else {
        __builtin_amdgcn_wave_barrier();
        asm volatile("" ::: "memory");
      }
    }
  };
  template <class F>
  static __device__ __forceinline__ void staged(uint8_t* lds, const f32x4 (&acc)[FM][FN], F&& f) {
    gemm_sync();   // (every wave is done with the operands)
    const int ln = lane(), wv = wave();
    float* region = reinterpret_cast<float*>(lds) + wv * (CR * CC);
    const View view = {region}, mine = {region + group() * (NW * CR * CC)};
#pragma unroll
    for (int part = 0; part < TM / CR; ++part) {
#pragma unroll
      for (int i = 0; i < CR / 16; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          *reinterpret_cast<f32x4*>(mine.at + View::place(16 * i + 4 * (ln >> 4), 16 * j + (ln & 15))) = acc[part * (CR / 16) + i][j];
      View::turn();
      if constexpr (WK > 1) {   // the groups' sums
        for (int i = 0; i < View::pieces(); ++i) {
          int r, c;
          float v[8];
          View::col_piece(i, &r, &c);
          view.col(r, c, v);
#pragma unroll
          for (int q = 1; q < WK; ++q) {
            float x[8];
            View{region + q * (NW * CR * CC)}.col(r, c, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += x[e];
          }
          view.put_col(r, c, v);
        }
        View::turn();
      }
      f((wv / WN) * TM + part * CR, (wv % WN) * TN, view);
      View::turn();
    }
  }
};

// Workgroups are dealt to the eight XCDs in turn, each with an L2 of its own:
// consecutive logical tiles are put on one XCD.
__device__ __forceinline__ int xcd_order(int id, int n) {
  const int q = n >> 3, r = n & 7, x = id & 7;
  return x * q + (x < r ? x : r) + (id >> 3);
}

// Tile t of a tm x tn grid, in bands of eight rows walked column by column, so
// that tiles that run together share operand rows of both sides.
__device__ __forceinline__ void band_order(int t, int tm, int tn, int* ti, int* tj) {
  constexpr int kBand = 8;
  const int per = kBand * tn, band = t / per, first = band * kBand;
  const int h = tm - first < kBand ? tm - first : kBand, in = t - band * per;
  *ti = first + in % h;
  *tj = in / h;
}

}  // namespace pp
