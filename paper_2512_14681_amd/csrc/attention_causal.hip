// Causal grouped-query attention of packed sequences (jf_attention_causal) and
// its gradient (jf_attention_causal_grad): row i of a sequence sees the rows
// j <= i of its own sequence.
//
//   s_ij = q_i k_j / sqrt(hd), p = softmax_j, o_i = sum_j p_ij v_j
//   D_i = o_i do_i, ds_ij = p_ij (do_i v_j - D_i)
//   dv_j = sum_i p_ij do_i, dq_i = sum_j ds_ij k_j / sqrt(hd), dk_j = sum_i ds_ij q_i / sqrt(hd)
//
// The outputs and dq are computed by workgroups of 128, 64 or 32 queries of
// one head that go over the keys; dk and dv by workgroups of as many keys that
// go over the queries, so that no sum depends on the order in which
// workgroups run.  Scores come out of the matrix cores transposed (keys x
// queries for the former, queries x keys for the latter), such that a lane
// holds one query's (one key's) weights in the order in which the second
// product takes them.  The row-major tiles in LDS serve as both operands: as
// they are, and read transposed.
//
// bf16: weights p and ds enter the second products rounded to bf16, as the
// inputs there are (2^-8 at most of each of many terms of a sum; the result
// is rounded to as much itself).  Sums, maxima and statistics are fp32.  Each
// of these two roundings adds 0.0015 to 0.0017 to the gradients' relative
// error, D from the rounded outputs 0.001 to that of dq, and the gradients' own
// rounding 0.0017 (errors that add up as squares); two terms for each would
// double the second products.
//
// Figures below are of traced launches, 7b heads being 28 query and 4 KV heads
// of 128 dims in bf16; a matrix product of 8192^3 reaches 1236 TFLOP/s.
#include <algorithm>
#include <type_traits>

#include "jf_internal.h"
#include "jf_tile32.h"

namespace jf {

// A block of a sequence's rows: rows r0 .. r0 + n - 1 of the row tensors are
// the sequence's, block t (of `blocks`) is meant.
struct RowBlock {
  int r0, n, t, blocks;
};

// The block that workgroup number `rank` works on (none: no blocks).  Among up to
// 64 sequences the ones with the most work come first: work grows with a
// block's number (kFirst: with its distance from the sequence's end).  Among
// more, sequence s's blocks have the numbers from (its start) / kBlock + s on,
// which no two sequences share, and s is searched for, 64 places at a time.
// The first workgroup raises JF_FLAG_CAPACITY for row starts beyond the rows
// or decreasing ones; no address is formed from those.  Only where there are
// such can sequences overlap: among up to 64, one that starts before an
// earlier one's end has no blocks then.
template <int kBlock, bool kFirst> __device__ __forceinline__ RowBlock search_block(const CausalArgs& a, int rank) {
  constexpr int kMostSearched = 256;  // blocks of a sequence, for which the order is looked for
  const int lane = threadIdx.x & 63;
  const uint64_t before = (1ull << lane) - 1;
  auto valid = [&](int r0, int r1) { return r0 >= 0 && r1 >= r0 && r1 <= a.n_rows; };
  if (blockIdx.x == 0 && a.flags) {
    bool bad = false;
    for (int s = threadIdx.x; s < a.n_seqs; s += 256) bad |= !valid(a.row_start[s], a.row_start[s + 1]);
    if (bad) atomicOr(a.flags, kFlagCapacity);
  }
  if (a.n_seqs <= 64) {
    int r0 = 0, r1 = 0;
    if (lane < a.n_seqs) {
      r0 = a.row_start[lane];
      r1 = a.row_start[lane + 1];
    }
    bool good = valid(r0, r1);
    if (__any(!good)) {
      int end = good ? r1 : 0;  // the latest one up to here
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int before = __shfl_up(end, d);
        if (lane >= d) end = max(end, before);
      }
      end = __shfl_up(end, 1);
      good = good && (lane == 0 || r0 >= end);
    }
    const int blocks = good ? (r1 - r0 + kBlock - 1) / kBlock : 0;
    int total = blocks, most = blocks;
    if (a.n_seqs > 1) {
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        total += __shfl_xor(total, d);
        most = max(most, __shfl_xor(most, d));
      }
    }
    total = __builtin_amdgcn_readfirstlane(total);
    most = __builtin_amdgcn_readfirstlane(most);
    if (rank >= total) return RowBlock{0, 0, 0, 0};
    int l = 0, u = most - 1 - rank;  // of one sequence
    if (a.n_seqs > 1) {
      int left = rank;
      if (most <= kMostSearched) {   // of every sequence its longest, then of every one its next, ...
        for (u = most - 1;; --u) {
          const int n = __builtin_popcountll(__ballot(blocks > u));
          if (left < n) break;
          left -= n;
        }
        const uint64_t has = __ballot(blocks > u);
        l = __builtin_ctzll(__ballot(blocks > u && __builtin_popcountll(has & before) == left));
      } else {                       // one sequence after the other
        for (;; ++l) {
          const int n = __builtin_amdgcn_readlane(blocks, l);
          if (left < n) break;
          left -= n;
        }
        u = __builtin_amdgcn_readlane(blocks, l) - 1 - left;
      }
    }
    const int n = __builtin_amdgcn_readlane(blocks, l), at = __builtin_amdgcn_readlane(r0, l);
    return RowBlock{at, __builtin_amdgcn_readlane(r1, l) - at, kFirst ? n - 1 - u : u, n};
  }
  // the last sequence whose blocks start at `rank` or before: in [lo, lo + span)
  const int r = a.row_start[0];
  int lo = 0, span = a.n_seqs;
  auto number = [&](int s) { return (int)(((int64_t)a.row_start[s] - r) / kBlock) + s; };
  while (span > 1) {
    const int step = (span + 63) / 64, at = lane * step;
    const uint64_t has = __ballot(at < span && number(lo + at) <= rank);
    if (!has) return RowBlock{0, 0, 0, 0};
    const int l = 63 - __builtin_clzll(has);
    span = min(step, span - l * step);
    lo += l * step;
  }
  const int r0 = a.row_start[lo], r1 = a.row_start[lo + 1], t = rank - number(lo);
  const int blocks = valid(r0, r1) ? (r1 - r0 + kBlock - 1) / kBlock : 0;
  return t >= 0 && t < blocks ? RowBlock{r0, r1 - r0, kFirst ? t : blocks - 1 - t, blocks} : RowBlock{0, 0, 0, 0};
}
template <int kBlock, bool kFirst> __device__ __forceinline__ bool find_block(const CausalArgs& a, int rank, RowBlock& b) {
  const RowBlock x = search_block<kBlock, kFirst>(a, rank);
  b = RowBlock{__builtin_amdgcn_readfirstlane(x.r0), __builtin_amdgcn_readfirstlane(x.n),   // in scalar registers,
               __builtin_amdgcn_readfirstlane(x.t), __builtin_amdgcn_readfirstlane(x.blocks)};  // as loads to LDS take them
  return b.blocks > 0;
}

// Workgroups go around the 8 XCDs in order: the heads of a group, which read
// the same keys, follow each other on one of them.
struct Work {
  int rank, g, h;
};
__device__ __forceinline__ Work work_of(int G, int heads) {
  const int i = blockIdx.x >> 3, pair = i / heads * 8 + (blockIdx.x & 7);
  return Work{pair / G, pair % G, i % heads};
}
static unsigned work_grid(int blocks, int G, int heads) {
  return (unsigned)(((int64_t)blocks * G + 7) / 8 * 8 * heads);
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Weights are 2^(s - m - kDown).  m follows a row's maximum only when a lane's
// weights of a step sum to more than kMost: most steps look for no maximum
// and leave sums and outputs as they are.  kDown keeps sums of weights below
// 1, so that no sum of values overflows that has a finite mean.
// A maximum beyond kFar is too coarse to hold kDown beside it: the weights are
// held below 2^(4 - kDown) one by one.
constexpr float kDown = 32.f, kMost = 0x1p-22f, kFar = 1 << 20;

// Four waves work on blocks of 32 NQ queries (keys, for dk and dv): NQ = 4
// gives each wave 32 of its own; with fewer, kShare waves have the same ones
// and take other rows of each step, and join at the end.  A step brings kRows
// rows, 32 kTiles for a wave.
template <typename T, int NQ> struct Shape {
  static constexpr int kBlock = 32 * NQ, kShare = 4 / NQ;
  static constexpr int kTiles = NQ == 4 && sizeof(T) == 2 ? 2 : 1;
  static constexpr int kRows = 32 * kTiles * kShare;
};
// Workgroups of a compute unit: registers and LDS of fp32 tiles hold one.
template <typename T> constexpr int kResident = sizeof(T) == 2 ? 2 : 1;
using First = std::integral_constant<int, 0>;
using Second = std::integral_constant<int, 1>;

// Steps over the keys up to `last` for queries from `first` on, those before
// it without masks.  The buffers by turns, in pairs of steps: their addresses
// are constants.
template <int kRows, typename F> __device__ __forceinline__ void all_steps(int first, int last, F step) {
  int j0 = 0;
#pragma unroll 1
  for (; j0 + 2 * kRows - 1 <= first; j0 += 2 * kRows) {
    step(std::false_type{}, First{}, j0);
    step(std::false_type{}, Second{}, j0 + kRows);
  }
#pragma unroll 1
  for (; j0 <= last; j0 += 2 * kRows) {
    step(std::true_type{}, First{}, j0);
    if (j0 + kRows <= last) step(std::true_type{}, Second{}, j0 + kRows);
  }
}

// Values of the waves that share a block's rows, as columns of 32 lanes: slot
// 0 .. kShare - 2 of them in LDS.
template <int ND> __device__ __forceinline__ void put_shared(float* at, const f32x16_t (&x)[ND]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) at[(32 * d + acc_row(i) + 4 * (lane >> 5)) * 32 + (lane & 31)] = x[d][i];
}
template <int ND> __device__ __forceinline__ void add_shared(const float* at, float f, f32x16_t (&x)[ND]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) x[d][i] += f * at[(32 * d + acc_row(i) + 4 * (lane >> 5)) * 32 + (lane & 31)];
}

// Outputs, in one pass over the keys.  Bound by the matrix and vector
// instructions, which two waves a SIMD overlap in part: 8192 rows of 7b heads
// (481 GFLOP) take 462 us, 1040 TFLOP/s; the matrix cores are busy in about 60%
// of the cycles, at 1.8 GHz (the chip's power sets the clock), and no LDS access
// waits for a bank.  2048 rows take 50 us: 448 workgroups on 512 places, of
// which the longest has 32 steps.  A wave holds its 32 queries (32 registers),
// 64 x 32 scores and weights (64) and 32 outputs of 128 dims (64); the keys'
// and values' next step comes to LDS meanwhile.  Not kept: scores of the next
// step beside the weights of this one inside one wave (2048 rows 7% slower),
// wave priorities (no change), operands further ahead (no change).
template <typename T, int HD, int NQ, bool kVec>
__global__ void __launch_bounds__(256, kResident<T>) k_causal(CausalArgs a) {
  using Tile = RowTile<T, HD>;
  using S = Shape<T, NQ>;
  constexpr int KT = S::kTiles, kRows = S::kRows, NS = HD / 16, ND = HD / 32, kTileBytes = Tile::kRowBytes * kRows;
  using Loader = RowLoader<T, HD, kRows, 4, kVec>;
  __shared__ __align__(1024) char s_kv[2][2][kTileBytes];
  const int grp = a.H / a.G;
  const Work job = work_of(a.G, grp);
  RowBlock b;
  if (!find_block<S::kBlock, false>(a, job.rank, b)) return;
  const int head = job.g * grp + job.h;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const int share = wave / NQ, from = share * 32 * KT; // the wave's rows of a step
  const int q0 = b.t * S::kBlock + wave % NQ * 32;     // the wave's queries
  const int qi = min(q0 + (lane & 31), b.n - 1);       // the lane's: past the end the last one again
  const int last = min(b.t * S::kBlock + S::kBlock, b.n) - 1;
  const T* kp = reinterpret_cast<const T*>(a.k) + (size_t)b.r0 * a.ld_k + job.g * HD;
  const T* vp = reinterpret_cast<const T*>(a.v) + (size_t)b.r0 * a.ld_v + job.g * HD;
  auto load = [&](int j0, int buf) {
    Loader::load(kp + (size_t)j0 * a.ld_k, a.ld_k * sizeof(T), last - j0, s_kv[buf][0]);
    Loader::load(vp + (size_t)j0 * a.ld_v, a.ld_v * sizeof(T), last - j0, s_kv[buf][1]);
  };
  load(0, 0);
  Frag<T> q[NS];
  {
    const T* p = reinterpret_cast<const T*>(a.q) + (size_t)(b.r0 + qi) * a.ld_q + head * HD + 8 * h;
#pragma unroll
    for (int s = 0; s < NS; ++s) q[s] = row_frag<T>(p + 16 * s, kVec);
    settle(q);
  }
  const float c = kLog2e / sqrtf((float)HD);
  float m = -INFINITY, l = 0.f;
  bool far = false;
  f32x16_t o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zero16();

  auto step = [&](auto edge, auto which, int j0) {
    constexpr bool kEdge = decltype(edge)::value;
    constexpr int kBuf = decltype(which)::value;
    // every wave's pieces have arrived, and its work on the step before is done
    if constexpr (kVec) wait_vm<0>();
    __syncthreads();
    if (j0 + kRows <= last) load(j0 + kRows, kBuf ^ 1);
    const uint32_t keys = Tile::row_base(lds_address(s_kv) + from * Tile::kRowBytes) + kBuf * 2 * kTileBytes;
    const uint32_t values = Tile::column_base(lds_address(s_kv) + from * Tile::kRowBytes) + (kBuf * 2 + 1) * kTileBytes;
    if (kEdge && j0 + from > q0 + 31) return;
    f32x16_t st[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) st[kt] = zero16();
    stream<T, KT * NS, kAhead<T>>([&](int n) { return Tile::rows(keys, n % KT * 32, n / KT); },
                                  [&](int n, const Frag<T>& k) { mfma32(st[n % KT], k, q[n / KT]); });
    const int lim = qi - j0 - from - 4 * h;
    if constexpr (kEdge) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) st[kt][i] = 32 * kt + acc_row(i) <= lim ? st[kt][i] : -INFINITY;
    }
    f32x16_t w[KT];
    float sum;
    auto weights = [&](float off) {
      sum = 0.f;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          w[kt][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kt][i], c, off));
          sum += w[kt][i];
        }
    };
    weights(-kDown - m);  // nothing seen yet: infinite or NaN
    if (__builtin_expect(__any(!(sum <= kMost)) || far, 0)) {
      float mx = st[0][0];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[kt][i]);
      mx = pair_max(mx);
      float top = mx * c;
      // beyond 2^24 the rounded product may lie far above the score itself, which would lose all weight
      if (__builtin_fmaf(mx, c, -top) < -1.f) top -= fabsf(top) * 0x1p-23f;
      const float m_new = fmaxf(m, top), m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m - m_use);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= alpha;
      far = __any(fabsf(m_use) > kFar);
      if (far) {
        sum = 0.f;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float d = __builtin_fmaf(st[kt][i], c, -m_use);
            w[kt][i] = __builtin_amdgcn_exp2f((d > 4.f ? 4.f : d) - kDown);  // NaN stays
            sum += w[kt][i];
          }
      } else {
        weights(-kDown - m_use);
      }
    }
    l += sum;
    bool finite = true;
    if constexpr (kEdge) {  // 0 times a value that is not finite would reach rows that do not see it
      uint32_t top = 0;
#pragma unroll
      for (int n = 0; n < 2 * KT * ND; ++n) magnitude(Tile::columns(values, n / ND * 16, n % ND), top);
      finite = !__any(!all_finite<T>(top));
    }
    Frag<T> pf[2 * KT];
#pragma unroll
    for (int j = 0; j < 2 * KT; ++j) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = w[j / 2][8 * (j % 2) + e];
      frag_of(p, pf[j]);
    }
    if (!kEdge || finite) {
      stream<T, 2 * KT * ND, kAhead<T>>([&](int n) { return Tile::columns(values, n / ND * 16, n % ND); },
                                        [&](int n, const Frag<T>& v) { mfma32(o[n % ND], v, pf[n / ND]); });
    } else {
#pragma unroll
      for (int n = 0; n < 2 * KT * ND; ++n) {
        __builtin_amdgcn_sched_barrier(0);
        Frag<T> v = Tile::columns(values, n / ND * 16, n % ND);
        keep_finite(v);
        mfma32(o[n % ND], v, pf[n / ND]);
      }
#pragma unroll 1
      for (int j = 0; j < 2 * KT; ++j) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = 16 * j + acc_row(e) <= lim ? 1.f : 0.f;
        Frag<T> seen;
        frag_of(p, seen);
#pragma unroll
        for (int d = 0; d < ND; ++d) add_infinite<T>(o[d], Tile::columns(values, 16 * j, d), seen);
      }
    }
  };
  all_steps<kRows>(b.t * S::kBlock, last, step);

  l = pair_sum(l);
  if constexpr (S::kShare > 1) {
    __shared__ float s_ml[S::kShare - 1][NQ][2][32];
    float* s_o = reinterpret_cast<float*>(s_kv);
    static_assert((S::kShare - 1) * NQ * 32 * HD * 4 <= (int)sizeof(s_kv), "the parts fit");
    __syncthreads();
    if (share > 0) {
      put_shared<ND>(s_o + ((share - 1) * NQ + wave % NQ) * 32 * HD, o);
      if (h == 0) {
        s_ml[share - 1][wave % NQ][0][lane] = m;
        s_ml[share - 1][wave % NQ][1][lane] = l;
      }
    }
    __syncthreads();
    if (share > 0) return;
    float m_all = m;
#pragma unroll
    for (int i = 0; i < S::kShare - 1; ++i) m_all = fmaxf(m_all, s_ml[i][wave][0][lane & 31]);
    const float m_use = m_all == -INFINITY ? 0.f : m_all, f = __builtin_amdgcn_exp2f(m - m_use);
    l *= f;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] *= f;
#pragma unroll
    for (int i = 0; i < S::kShare - 1; ++i) {
      const float fi = __builtin_amdgcn_exp2f(s_ml[i][wave][0][lane & 31] - m_use);
      l += fi * s_ml[i][wave][1][lane & 31];
      add_shared<ND>(s_o + (i * NQ + wave) * 32 * HD, fi, o);
    }
    m = m_all;
  }
  if (q0 + (lane & 31) >= b.n) return;
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  T* out = reinterpret_cast<T*>(a.out) + (size_t)(b.r0 + qi) * a.ld_out + head * HD + 4 * h;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = inv == 0.f ? 0.f : o[d][i + e] * inv;
      row_store4<T>(out + 32 * d + acc_row(i), a.vec_out, v[0], v[1], v[2], v[3]);
    }
  if (a.lse && h == 0)
    a.lse[(size_t)head * a.n_rows + b.r0 + qi] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l * 0x1p32f)) * kLn2;
}

// ---- gradient ------------------------------------------------------------------------

// 2^x, at most 1: scores beyond 2^20 are too coarse beside the rounded lse.
// The bound is part of the instruction, and gives 0 for NaN: a row with a NaN
// score has NaN for its lse and D, which bring it to dq and dk; dv looks for it.
// (A minimum that keeps NaN costs 1.4% of 4096 rows' forward and gradient, that look 0.3%.)
__device__ __forceinline__ float weight(float x) { return __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(x), 0.f, 1.f); }

// dq; and of each row and head, for dk and dv, what the accumulators of its
// scores and of do v start from: -lse sqrt(hd) (-inf for a row without
// weights, whose weights then are 0), and -D.  sum_j ds_ij is 0 but for what the
// rounded outputs lack in D, and is added to it for dk.
// Three products a pair where the forward pass has two: 4096 rows of 7b heads
// (180 GFLOP) take 192 us, 940 TFLOP/s, bound as the forward pass is (which
// takes 136 us there).  Of these the sum of ds takes 1% of a forward and
// backward pass (in four sums; in one 1.5%, and 4% for heads of 64), and
// the gradients' error falls from 0.0025 to 0.0024.
template <typename T, int HD, int NQ, bool kVec>
__global__ void __launch_bounds__(256, kResident<T>) k_causal_dq(CausalGradArgs a) {
  using Tile = RowTile<T, HD>;
  using S = Shape<T, NQ>;
  constexpr int KT = S::kTiles, kRows = S::kRows, NS = HD / 16, ND = HD / 32, kTileBytes = Tile::kRowBytes * kRows;
  using Loader = RowLoader<T, HD, kRows, 4, kVec>;
  __shared__ __align__(1024) char s_kv[2][2][kTileBytes];
  const int grp = a.f.H / a.f.G;
  const Work job = work_of(a.f.G, grp);
  RowBlock b;
  if (!find_block<S::kBlock, false>(a.f, job.rank, b)) return;
  const int head = job.g * grp + job.h;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const int share = wave / NQ, from = share * 32 * KT;
  const int q0 = b.t * S::kBlock + wave % NQ * 32;
  const int qi = min(q0 + (lane & 31), b.n - 1);
  const int last = min(b.t * S::kBlock + S::kBlock, b.n) - 1;
  const T* kp = reinterpret_cast<const T*>(a.f.k) + (size_t)b.r0 * a.f.ld_k + job.g * HD;
  const T* vp = reinterpret_cast<const T*>(a.f.v) + (size_t)b.r0 * a.f.ld_v + job.g * HD;
  auto load = [&](int j0, int buf) {
    Loader::load(kp + (size_t)j0 * a.f.ld_k, a.f.ld_k * sizeof(T), last - j0, s_kv[buf][0]);
    Loader::load(vp + (size_t)j0 * a.f.ld_v, a.f.ld_v * sizeof(T), last - j0, s_kv[buf][1]);
  };
  load(0, 0);
  Frag<T> q[NS], g[NS];
  {
    const T* p = reinterpret_cast<const T*>(a.f.q) + (size_t)(b.r0 + qi) * a.f.ld_q + head * HD + 8 * h;
    const T* r = reinterpret_cast<const T*>(a.g_out) + (size_t)(b.r0 + qi) * a.ld_g_out + head * HD + 8 * h;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      q[s] = row_frag<T>(p + 16 * s, kVec);
      g[s] = row_frag<T>(r + 16 * s, kVec);
    }
    settle(q);
    settle(g);
  }
  const float c = kLog2e / sqrtf((float)HD);
  float lse, dot = 0.f, rest[4] = {0.f, 0.f, 0.f, 0.f};  // rest: sum of ds
  {
    const T* p = reinterpret_cast<const T*>(a.f.out) + (size_t)(b.r0 + qi) * a.f.ld_out + head * HD + 8 * h;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const Frag<T> x = row_frag<T>(p + 16 * s, a.vec_dot);
      float xs[8], gs[8];
      frag_values(x, xs);
      frag_values(g[s], gs);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot = __builtin_fmaf(xs[e], gs[e], dot);
    }
    dot = pair_sum(dot);
    lse = a.f.lse[(size_t)head * a.f.n_rows + b.r0 + qi];
    lse = lse == -INFINITY ? INFINITY : lse * kLog2e;
  }
  f32x16_t dq[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) dq[d] = zero16();

  auto step = [&](auto edge, auto which, int j0) {
    constexpr bool kEdge = decltype(edge)::value;
    constexpr int kBuf = decltype(which)::value;
    if constexpr (kVec) wait_vm<0>();
    __syncthreads();
    if (j0 + kRows <= last) load(j0 + kRows, kBuf ^ 1);
    const uint32_t tile = lds_address(s_kv) + from * Tile::kRowBytes;
    const uint32_t keys = Tile::row_base(tile) + kBuf * 2 * kTileBytes, values = keys + kTileBytes;
    const uint32_t key_columns = Tile::column_base(tile) + kBuf * 2 * kTileBytes;
    if (kEdge && j0 + from > q0 + 31) return;
    const int lim = qi - j0 - from - 4 * h;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      f32x16_t st = zero16(), dp = zero16();
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        mfma32(st, Tile::rows(keys, 32 * kt, s), q[s]);
        mfma32(dp, Tile::rows(values, 32 * kt, s), g[s]);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float ds = weight(__builtin_fmaf(st[i], c, -lse)) * (dp[i] - dot);
        st[i] = kEdge && 32 * kt + acc_row(i) > lim ? 0.f : ds;
        rest[i % 4] += st[i];
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = st[8 * j + e];
        Frag<T> pf;
        frag_of(p, pf);
#pragma unroll
        for (int d = 0; d < ND; ++d) mfma32(dq[d], Tile::columns(key_columns, 32 * kt + 16 * j, d), pf);
      }
    }
  };
  all_steps<kRows>(b.t * S::kBlock, last, step);

  float left = pair_sum((rest[0] + rest[1]) + (rest[2] + rest[3]));
  if constexpr (S::kShare > 1) {
    __shared__ float s_rest[S::kShare - 1][NQ][32];
    float* s_o = reinterpret_cast<float*>(s_kv);
    static_assert((S::kShare - 1) * NQ * 32 * HD * 4 <= (int)sizeof(s_kv), "the parts fit");
    __syncthreads();
    if (share > 0) {
      put_shared<ND>(s_o + ((share - 1) * NQ + wave % NQ) * 32 * HD, dq);
      if (h == 0) s_rest[share - 1][wave % NQ][lane] = left;
    }
    __syncthreads();
    if (share > 0) return;
#pragma unroll
    for (int i = 0; i < S::kShare - 1; ++i) {
      add_shared<ND>(s_o + (i * NQ + wave) * 32 * HD, 1.f, dq);
      left += s_rest[i][wave][lane & 31];
    }
  }
  if (q0 + (lane & 31) >= b.n) return;
  if (h == 0)
    a.dots[(size_t)head * a.f.n_rows + b.r0 + qi] =
        make_float2(lse == INFINITY ? -INFINITY : lse * (kLn2 * -sqrtf((float)HD)), -(dot + left));
  const float f = 1.f / sqrtf((float)HD);
  T* out = reinterpret_cast<T*>(a.g_q) + (size_t)(b.r0 + qi) * a.ld_g_q + head * HD + 4 * h;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      row_store4<T>(out + 32 * d + acc_row(i), a.vec_q, dq[d][i] * f, dq[d][i + 1] * f, dq[d][i + 2] * f, dq[d][i + 3] * f);
}

// dk and dv of a block of keys of a KV head, over the queries of the heads of
// `part` (part, part + parts, ... of the group's).
// Four products a pair: 4096 rows of 7b heads (241 GFLOP) take 260 to 287 us,
// 840 to 930 TFLOP/s.  The 128 registers of dk and dv beside 64 of keys and values leave
// room for one tile of scores at a time, so that the matrix cores wait for the
// weights more often than in the forward pass.
template <typename T, int HD, int NQ, bool kVec>
__global__ void __launch_bounds__(256, kResident<T>) k_causal_dkv(CausalGradArgs a) {
  using Tile = RowTile<T, HD>;
  using S = Shape<T, NQ>;
  constexpr int KT = S::kTiles, kRows = S::kRows, NS = HD / 16, ND = HD / 32;
  using Loader = RowLoader<T, HD, kRows, 4, kVec>;
  __shared__ __align__(1024) char s_qg[2][2][Tile::kRowBytes * kRows];
  __shared__ __align__(16) float s_dots[2][2][kRows];
  const int grp = a.f.H / a.f.G;
  const Work job = work_of(a.f.G, a.parts);
  RowBlock b;
  if (!find_block<S::kBlock, true>(a.f, job.rank, b)) return;  // the first keys have the most queries
  const int part = job.h;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const int share = wave / NQ, from = share * 32 * KT;  // the wave's rows of a step
  const int k0 = b.t * S::kBlock + wave % NQ * 32;
  const int ki = min(k0 + (lane & 31), b.n - 1);
  Frag<T> k[NS], v[NS];
  {
    const T* p = reinterpret_cast<const T*>(a.f.k) + (size_t)(b.r0 + ki) * a.f.ld_k + job.g * HD + 8 * h;
    const T* r = reinterpret_cast<const T*>(a.f.v) + (size_t)(b.r0 + ki) * a.f.ld_v + job.g * HD + 8 * h;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      k[s] = row_frag<T>(p + 16 * s, kVec);
      v[s] = row_frag<T>(r + 16 * s, kVec);
    }
  }
  const float c = kLog2e / sqrtf((float)HD);
  f32x16_t dk[ND], dv[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    dk[d] = zero16();
    dv[d] = zero16();
  }
  // The steps: every head's rows from the sequence's end to the block's first
  // key, one head after the other.  From the end, as workgroups that run at
  // once then read the same rows at about the same time (4096 rows, 28 query
  // and 4 KV heads: 27% of the accesses miss the L2, in the other order 56%,
  // and a forward and backward pass takes 1.3% longer).
  const int first = b.t * S::kBlock, steps = (b.n - first + kRows - 1) / kRows, top = first + (steps - 1) * kRows;
  int head = job.g * grp + part, i0 = top;
  float2 dots = make_float2(-INFINITY, 0.f);
  auto load = [&](int buf) {
    const int row = i0 + (int)threadIdx.x;
    if ((int)threadIdx.x < kRows) {
      dots = make_float2(-INFINITY, 0.f);
      if (row < b.n) dots = a.dots[(size_t)head * a.f.n_rows + b.r0 + row];
    }
    Loader::load(reinterpret_cast<const T*>(a.f.q) + (size_t)(b.r0 + i0) * a.f.ld_q + head * HD, a.f.ld_q * sizeof(T),
                 b.n - 1 - i0, s_qg[buf][0]);
    Loader::load(reinterpret_cast<const T*>(a.g_out) + (size_t)(b.r0 + i0) * a.ld_g_out + head * HD,
                 a.ld_g_out * sizeof(T), b.n - 1 - i0, s_qg[buf][1]);
    i0 -= kRows;
    if (i0 < first) {
      i0 = top;
      head += a.parts;
    }
  };
  auto put_dots = [&](int buf) {
    if ((int)threadIdx.x < kRows) {
      s_dots[buf][0][threadIdx.x] = dots.x;
      s_dots[buf][1][threadIdx.x] = dots.y;
    }
  };
  load(0);
  put_dots(0);
  settle(k);
  settle(v);
  const int heads = (grp - part + a.parts - 1) / a.parts, total = heads * steps;
  int at = top, buf = 0;
#pragma unroll 1
  for (int it = 0; it < total; ++it) {
    if constexpr (kVec) wait_vm<0>();
    __syncthreads();
    if (it + 1 < total) load(buf ^ 1);
    const int mine = at + from;          // the wave's first row
    const bool edge = mine < k0 + 31;    // rows before some of the wave's keys
    if (mine + 32 * KT > k0 && mine < b.n) {
#pragma unroll 1
      for (int kt = 0; kt < KT; ++kt) {  // not unrolled: registers
        const int skip = from + 32 * kt;
        const uint32_t q_tile = lds_address(s_qg[buf][0]) + skip * Tile::kRowBytes;
        const uint32_t g_tile = lds_address(s_qg[buf][1]) + skip * Tile::kRowBytes;
        const float start = s_dots[buf][0][skip + (lane & 31)];
        if (const uint32_t nans = (uint32_t)__ballot(start != start); __builtin_expect(nans != 0, 0)) {
          // rows without numbers: the gradients of the values that they see have none
          const float f = 31 - __builtin_clz(nans) >= ki - at - skip ? NAN : 0.f;
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) dv[d][i] += f;
        }
        const uint32_t qs = Tile::row_base(q_tile), gs = Tile::row_base(g_tile);
        const uint32_t q_columns = Tile::column_base(q_tile), g_columns = Tile::column_base(g_tile);
        f32x16_t st, dp, off;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 x = *reinterpret_cast<const float4*>(&s_dots[buf][0][skip + acc_row(i) + 4 * h]);
          const float4 y = *reinterpret_cast<const float4*>(&s_dots[buf][1][skip + acc_row(i) + 4 * h]);
          st[i] = x.x; st[i + 1] = x.y; st[i + 2] = x.z; st[i + 3] = x.w;
          dp[i] = y.x; dp[i + 1] = y.y; dp[i + 2] = y.z; dp[i + 3] = y.w;
        }
        if constexpr (sizeof(T) == 4) {  // sums next to lse sqrt(hd) would lose last digits of fp32 scores
          off = st;
          st = zero16();
        }
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          mfma32(st, Tile::rows(qs, 0, s), k[s]);
          mfma32(dp, Tile::rows(gs, 0, s), v[s]);
        }
        __builtin_amdgcn_sched_barrier(0);
        const int lim = ki - at - skip - 4 * h;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool hidden = edge && acc_row(i) < lim;
          st[i] = weight(sizeof(T) == 4 ? (st[i] + off[i]) * c : st[i] * c);
          dp[i] = hidden ? 0.f : st[i] * dp[i];
          st[i] = hidden ? 0.f : st[i];
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float x[8], y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = st[8 * j + e];
            y[e] = dp[8 * j + e];
          }
          Frag<T> pf, df;
          frag_of(x, pf);
          frag_of(y, df);
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            mfma32(dv[d], Tile::columns(g_columns, 16 * j, d), pf);
            mfma32(dk[d], Tile::columns(q_columns, 16 * j, d), df);
          }
        }
      }
    }
    if (it + 1 < total) put_dots(buf ^ 1);
    buf ^= 1;
    at -= kRows;
    if (at < first) at = top;
  }

  if constexpr (S::kShare > 1) {
    float* s_o = reinterpret_cast<float*>(s_qg);
    static_assert((S::kShare - 1) * NQ * 64 * HD * 4 <= (int)sizeof(s_qg), "the parts fit");
    __syncthreads();
    if (share > 0) {
      put_shared<ND>(s_o + ((share - 1) * NQ + wave % NQ) * 64 * HD, dk);
      put_shared<ND>(s_o + ((share - 1) * NQ + wave % NQ) * 64 * HD + 32 * HD, dv);
    }
    __syncthreads();
    if (share > 0) return;
#pragma unroll
    for (int i = 0; i < S::kShare - 1; ++i) {
      add_shared<ND>(s_o + (i * NQ + wave) * 64 * HD, 1.f, dk);
      add_shared<ND>(s_o + (i * NQ + wave) * 64 * HD + 32 * HD, 1.f, dv);
    }
  }
  if (k0 + (lane & 31) >= b.n) return;
  const float f = 1.f / sqrtf((float)HD);
  const int col = job.g * HD + 4 * h;
  if (a.parts == 1) {
    T* pk = reinterpret_cast<T*>(a.g_k) + (size_t)(b.r0 + ki) * a.ld_g_k + col;
    T* pv = reinterpret_cast<T*>(a.g_v) + (size_t)(b.r0 + ki) * a.ld_g_v + col;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        row_store4<T>(pk + 32 * d + acc_row(i), a.vec_kv, dk[d][i] * f, dk[d][i + 1] * f, dk[d][i + 2] * f, dk[d][i + 3] * f);
        row_store4<T>(pv + 32 * d + acc_row(i), a.vec_kv, dv[d][i], dv[d][i + 1], dv[d][i + 2], dv[d][i + 3]);
      }
  } else {
    const size_t width = (size_t)a.f.G * HD, at_row = ((size_t)part * a.f.n_rows + b.r0 + ki) * width + col;
    float *pk = a.kv_part + at_row, *pv = pk + (size_t)a.parts * a.f.n_rows * width;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        *reinterpret_cast<float4*>(pk + 32 * d + acc_row(i)) =
            make_float4(dk[d][i] * f, dk[d][i + 1] * f, dk[d][i + 2] * f, dk[d][i + 3] * f);
        *reinterpret_cast<float4*>(pv + 32 * d + acc_row(i)) = make_float4(dv[d][i], dv[d][i + 1], dv[d][i + 2], dv[d][i + 3]);
      }
  }
}

// Sums the parts of a block's rows in order, four columns a thread; kSlices
// workgroups share a block.  Reads what k_causal_dkv wrote: 117 MB of 4096
// rows of 7b heads in 19 us, 6.1 TB/s, the last of it from the caches.
constexpr int kSlices = 8;
template <typename T, int NQ> __global__ void __launch_bounds__(256) k_causal_join(CausalGradArgs a) {
  const Work job = work_of(a.f.G, kSlices);
  RowBlock b;
  if (!find_block<32 * NQ, true>(a.f, job.rank, b)) return;
  constexpr int kRows = 32 * NQ / kSlices;
  const int chunks = a.f.hd / 4, col = job.g * a.f.hd + threadIdx.x % chunks * 4;
  const size_t width = (size_t)a.f.G * a.f.hd, plane = a.f.n_rows * width;
  for (int i = threadIdx.x / chunks; i < 2 * kRows; i += 256 / chunks) {  // the keys', then the values'
    const int r = b.t * 32 * NQ + job.h * kRows + i % kRows;
    if (r >= b.n) continue;
    const size_t row = b.r0 + r;
    const float* p = a.kv_part + row * width + col + (i < kRows ? 0 : a.parts * plane);
    float4 s = *reinterpret_cast<const float4*>(p);
    for (int k = 1; k < a.parts; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(p + k * plane);
      s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
    T* out = i < kRows ? reinterpret_cast<T*>(a.g_k) + row * a.ld_g_k : reinterpret_cast<T*>(a.g_v) + row * a.ld_g_v;
    row_store4<T>(out + col, a.vec_kv, s.x, s.y, s.z, s.w);
  }
}

// ---- launch --------------------------------------------------------------------------
// Bound on the blocks' numbers (search_block): among more than 64 sequences
// empty ones count too.
static int blocks_of(int n_rows, int n_seqs, int rows) {
  if (n_seqs > 64) return (int)std::min<int64_t>((int64_t)n_rows / rows + n_seqs, 1 << 30);
  return (int)std::min<int64_t>((int64_t)n_rows / rows + std::min(n_seqs, n_rows), n_rows);
}

// Wide blocks read the keys least often; narrow ones make the longest
// workgroup short, which counts where there are too few to fill the chip.
// Blocks of 128 rows from `wide` of them (times heads) on.  Where the two are
// even depends on the lengths as well: one long sequence gains from narrow
// blocks longer, many short ones not as long, and the bounds lie between.
// Whole passes, us in blocks of 128 and of 64 rows, 28 query and 4 KV heads:
//                          `wide`  one sequence                     nine of different lengths
//   bf16, 128 dims            320  364: 38 and 36, 448: 44 and 46   364: 12 and 11, 448: 14 and 17
//   its gradient              450  476: 200 and 167, 700: 316, 319  448: 50 and 50, 560: 59 and 66
//   bf16, 64 dims             600  476: 31 and 28, 700: 52 and 55   672: 14.3 and 16.0
//   its gradient              900  896: 271 and 265, 1176: 431, 445 868: 60 and 62, 1148: 83 and 82
//   bf16, 32 dims             600  476: 24 and 20, 1176: 90 and 91  672: 11 and 10, 1148: 19.1 and 19.5
//   its gradient              900  896: 187 and 171, 1792: 595, 968 868: 43.0 and 42.4, 1764: 97 and 110
//   fp32, 32 dims            1000  980: 352 and 311, 1288: 559, 523 952: 51 and 46, 1260: 76 and 71
//   its gradient             1000  980: 1187, 1082, 1288: 2021, 2054  952: 164 and 146, 1260: 248, 252
// (fp32, 128 dims: nine sequences, 952: 178 and 187, its gradient 566 and 591;
// one sequence, 784: 835 and 811, 3003 and 2845).
// Blocks of 32 rows where these all run at once, up to 512 of them: 4 heads of
// 32 dims, fp32, 2048 rows 89, 48 and 28 us in blocks of 128, 64 and 32; beyond,
// 28 heads of 64, bf16, 768 rows (700 blocks) 12.3 us in blocks of 64 and 15.2
// of 32, but 16 heads of 32, 1024 rows (528) 12.0 and 9.7.  At head_dim 128
// blocks of 32 rows fill the LDS, or gain nothing (20.1 us for 512 rows, blocks
// of 64 12.7).
static int causal_groups(int n_rows, int n_seqs, int H, int hd, bool f32, bool grad) {
  const int wide = f32 ? 1000 : hd == 128 ? (grad ? 450 : 320) : grad ? 900 : 600;
  if ((int64_t)blocks_of(n_rows, n_seqs, 128) * H >= wide) return 4;
  return (int64_t)blocks_of(n_rows, n_seqs, 32) * H > 512 || hd == 128 ? 2 : 1;
}
static void causal_shape(CausalArgs& a, bool grad) {
  a.groups = causal_groups(a.n_rows, a.n_seqs, a.H, a.hd, a.f32, grad);
  a.blocks = blocks_of(a.n_rows, a.n_seqs, 32 * a.groups);
}
void causal_plan(CausalArgs& a) { causal_shape(a, false); }
// dk and dv: one part where its workgroups (500 and more) fill the chip, else a
// group's heads in parts of as many as leave enough of them, and a pass that
// adds the parts.  The gradient's passes in us, 28 query and 4 KV heads of 128
// dims: 4096 rows (132 workgroups a part) 1511 in one part, 480 in seven; 12
// sequences of 1000 rows (420) 548 in one, 480 in four as here, 561 in seven; 32
// of 500 rows (628) 376 in one, 398 in two, 566 in seven.  One sequence of 16200
// rows (508), whose last keys have little to do, would take 6.7 ms in seven
// parts instead of 9.2.
static int grad_parts(int64_t one, int64_t grp) {  // one: workgroups of one part; fewer parts the more there are
  const int64_t heads = one >= 500 ? grp : std::max<int64_t>(grp * one / 1024, 1);
  return (int)((grp + heads - 1) / heads);
}
void causal_grad_plan(CausalGradArgs& a) {
  causal_shape(a.f, true);
  a.parts = grad_parts((int64_t)a.f.blocks * a.f.G, a.f.H / a.f.G);
}
// Bound on parts times rows of the calls with n_rows rows or fewer (those with
// one part have no parts to hold).  Rows between 128 (b - 1) and 128 b - 1, of
// however many sequences, make b blocks or more.
size_t causal_most_part_rows(int n_rows, int H, int G) {
  size_t most = 0;
  for (int64_t b = 1;; ++b) {
    const int64_t rows = std::min<int64_t>(128 * b - 1, n_rows);
    const int parts = grad_parts(b * G, H / G);
    if (parts == 1) return most;
    most = std::max(most, (size_t)(parts * rows));
    if (rows == n_rows) return most;
  }
}

template <typename F> static hipError_t with_shape(int hd, int groups, bool vec, F f) {
  auto by_vec = [&](auto d, auto n) {
    if (vec) f(d, n, std::true_type{});
    else f(d, n, std::false_type{});
  };
  auto by_groups = [&](auto d) {
    if (groups == 4) by_vec(d, std::integral_constant<int, 4>{});
    else if (groups == 2) by_vec(d, std::integral_constant<int, 2>{});
    else by_vec(d, std::integral_constant<int, 1>{});
  };
  if (hd == 32) by_groups(std::integral_constant<int, 32>{});
  else if (hd == 64) by_groups(std::integral_constant<int, 64>{});
  else by_groups(std::integral_constant<int, 128>{});
  return hipGetLastError();
}
// No kernel for what causal_groups does not choose.
template <int HD, int NQ> constexpr int kGroups = HD == 128 && NQ == 1 ? 2 : NQ;

template <typename T> static hipError_t causal_type(const CausalArgs& a, hipStream_t st) {
  const unsigned grid = work_grid(a.blocks, a.G, a.H / a.G);
  return with_shape(a.hd, a.groups, a.vec, [&](auto hd, auto nq, auto vec) {
    constexpr int HD = decltype(hd)::value;
    k_causal<T, HD, kGroups<HD, decltype(nq)::value>, decltype(vec)::value><<<grid, 256, 0, st>>>(a);
  });
}
hipError_t launch_causal(int dtype, const CausalArgs& a, hipStream_t st) {
  return dtype == 0 ? causal_type<float>(a, st) : causal_type<bf16_t>(a, st);
}

template <typename T> static hipError_t causal_grad_type(const CausalGradArgs& a, hipStream_t st) {
  const unsigned dq = work_grid(a.f.blocks, a.f.G, a.f.H / a.f.G), dkv = work_grid(a.f.blocks, a.f.G, a.parts);
  const hipError_t e = with_shape(a.f.hd, a.f.groups, a.f.vec, [&](auto hd, auto nq, auto vec) {
    constexpr int HD = decltype(hd)::value, NQ = kGroups<HD, decltype(nq)::value>;
    k_causal_dq<T, HD, NQ, decltype(vec)::value><<<dq, 256, 0, st>>>(a);
    k_causal_dkv<T, HD, NQ, decltype(vec)::value><<<dkv, 256, 0, st>>>(a);
  });
  if (e != hipSuccess || a.parts == 1) return e;
  const unsigned join = work_grid(a.f.blocks, a.f.G, kSlices);
  if (a.f.groups == 4) k_causal_join<T, 4><<<join, 256, 0, st>>>(a);
  else if (a.f.groups == 2) k_causal_join<T, 2><<<join, 256, 0, st>>>(a);
  else k_causal_join<T, 1><<<join, 256, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_causal_grad(int dtype, const CausalGradArgs& a, hipStream_t st) {
  return dtype == 0 ? causal_grad_type<float>(a, st) : causal_grad_type<bf16_t>(a, st);
}

}  // namespace jf
