// Causal grouped-query attention of packed sequences (jf_attention_causal) and
// its gradient (jf_attention_causal_grad): row i of a sequence sees the rows
// j <= i of its own sequence.
//
//   s_ij = q_i k_j / sqrt(hd), p = softmax_j, o_i = sum_j p_ij v_j
//   D_i = o_i do_i, ds_ij = p_ij (do_i v_j - D_i)
//   dv_j = sum_i p_ij do_i, dq_i = sum_j ds_ij k_j / sqrt(hd), dk_j = sum_i ds_ij q_i / sqrt(hd)
//
// The outputs and dq are computed by workgroups of 128 queries of one head,
// 32 a wave, that go over the keys; dk and dv by workgroups of 128 keys that
// go over the queries, so that no sum depends on the order in which
// workgroups run.  Scores come out of the matrix cores transposed (keys x
// queries for the former, queries x keys for the latter), such that a lane
// holds one query's (one key's) weights in the order in which the second
// product takes them.  The row-major tiles in LDS serve as both operands: as
// they are, and read transposed.
//
// bf16: weights p and ds enter the second products rounded to bf16, as the
// inputs there are (2^-9 of each of many terms of a sum; the result is
// rounded to as much itself).  Sums, maxima and statistics are fp32.
#include <algorithm>
#include <type_traits>

#include "jf_internal.h"
#include "jf_tile32.h"

namespace jf {

constexpr int kBlock = 128;  // queries of a workgroup (keys, for dk and dv): 32 a wave

// A block of a sequence's rows: rows r0 .. r0 + n - 1 of the row tensors are
// the sequence's, block t (of `blocks`) is meant.
struct RowBlock {
  int r0, n, t, blocks;
};

// Block number `rank` of all sequences' blocks, one after the other.  The
// first workgroup raises JF_FLAG_CAPACITY for row starts beyond the rows or
// decreasing ones; no address is formed from those.
__device__ __forceinline__ bool find_block(const CausalArgs& a, int rank, RowBlock& b) {
  const int lane = threadIdx.x & 63;
  const bool first = blockIdx.x == 0;
  int base = 0;
  bool found = false, bad = false;
  for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
    const int s = s0 + lane;
    int r0 = 0, r1 = 0;
    if (s < a.n_seqs) {
      r0 = a.row_start[s];
      r1 = a.row_start[s + 1];
    }
    const bool ok = r0 >= 0 && r1 >= r0 && r1 <= a.n_rows;
    bad |= !ok;
    const int blocks = ok ? (r1 - r0 + kBlock - 1) / kBlock : 0;
    int upto = blocks;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int v = __shfl_up(upto, d);
      if (lane >= d) upto += v;
    }
    const uint64_t hit = __ballot(base + upto > rank);
    if (!found && hit) {
      const int l = __builtin_ctzll(hit);
      b.blocks = __builtin_amdgcn_readlane(blocks, l);
      b.t = rank - base - (__builtin_amdgcn_readlane(upto, l) - b.blocks);
      b.r0 = __builtin_amdgcn_readlane(r0, l);
      b.n = __builtin_amdgcn_readlane(r1, l) - b.r0;
      found = true;
      if (!first) break;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
  }
  if (first && a.flags && (__any(bad) || base > a.blocks) && threadIdx.x == 0) atomicOr(a.flags, kFlagCapacity);
  return found;
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
constexpr float kDown = 32.f, kMost = 0x1p-22f;

template <typename T> struct Steps {
  static constexpr int KT = sizeof(T) == 2 ? 2 : 1;  // 32-row tiles of a step
  static constexpr int kRows = 32 * KT;
};

template <typename T, int HD, bool kVec>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) k_causal(CausalArgs a) {
  using Tile = RowTile<T, HD>;
  constexpr int KT = Steps<T>::KT, kRows = Steps<T>::kRows, NS = HD / 16, ND = HD / 32;
  using Loader = RowLoader<T, HD, kRows, 4, kVec>;
  __shared__ __align__(1024) char s_kv[2][2][kRows * HD * sizeof(T)];
  const int grp = a.H / a.G;
  const Work job = work_of(a.G, grp);
  RowBlock b;
  if (!find_block(a, job.rank, b)) return;
  b.t = b.blocks - 1 - b.t;  // the longest first
  const int head = job.g * grp + job.h;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const int q0 = b.t * kBlock + wave * 32;             // the wave's queries
  const int qi = min(q0 + (lane & 31), b.n - 1);       // the lane's: past the end the last one again
  const int last = min(b.t * kBlock + kBlock, b.n) - 1;
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
    const uint32_t keys = Tile::row_base(lds_address(s_kv)) + kBuf * 2 * Tile::kRowBytes * kRows;
    const uint32_t values = Tile::column_base(lds_address(s_kv)) + (kBuf * 2 + 1) * Tile::kRowBytes * kRows;
    if (kEdge && j0 > q0 + 31) return;
    f32x16_t st[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      st[kt] = zero16();
#pragma unroll
      for (int s = 0; s < NS; ++s) mfma32(st[kt], Tile::rows(keys, 32 * kt, s), q[s]);
    }
    const int lim = qi - j0 - 4 * h;
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
    if (__builtin_expect(__any(!(sum <= kMost)), 0)) {
      float mx = st[0][0];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[kt][i]);
      const float m_new = fmaxf(m, pair_max(mx) * c), m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m - m_use);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= alpha;
      weights(-kDown - m_use);
    }
    l += sum;
    bool finite = true;
    if constexpr (kEdge) {  // 0 times a value that is not finite would reach rows that do not see it
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 2 * KT; ++j)
#pragma unroll
        for (int d = 0; d < ND; ++d) magnitude(Tile::columns(values, 16 * j, d), top);
      finite = !__any(!all_finite<T>(top));
    }
#pragma unroll
    for (int j = 0; j < 2 * KT; ++j) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = w[j / 2][8 * (j % 2) + e];
      Frag<T> pf;
      frag_of(p, pf);
      if (!kEdge || finite) {
#pragma unroll
        for (int d = 0; d < ND; ++d) mfma32(o[d], Tile::columns(values, 16 * j, d), pf);
      } else {
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          __builtin_amdgcn_sched_barrier(0);
          Frag<T> v = Tile::columns(values, 16 * j, d);
          keep_finite(v);
          mfma32(o[d], v, pf);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if (kEdge && !finite) {
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
  // The buffers by turns, in pairs of steps: their addresses are constants.
  using First = std::integral_constant<int, 0>;
  using Second = std::integral_constant<int, 1>;
  static_assert(kBlock % (2 * kRows) == 0, "whole pairs before the edge");
  int j0 = 0;
#pragma unroll 1
  for (; j0 < b.t * kBlock; j0 += 2 * kRows) {
    step(std::false_type{}, First{}, j0);
    step(std::false_type{}, Second{}, j0 + kRows);
  }
#pragma unroll 1
  for (; j0 <= last; j0 += 2 * kRows) {
    step(std::true_type{}, First{}, j0);
    if (j0 + kRows <= last) step(std::true_type{}, Second{}, j0 + kRows);
  }

  if (q0 + (lane & 31) >= b.n) return;
  l = pair_sum(l);
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
    a.lse[(size_t)head * a.n_rows + b.r0 + qi] = l == 0.f ? -INFINITY : (m + kDown + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---- gradient ------------------------------------------------------------------------

// dq; and of each row and head, for dk and dv, what the accumulators of its
// scores and of do v start from: -lse sqrt(hd) (-inf for a row without
// weights, whose weights then are 0), and -D.
template <typename T, int HD, bool kVec>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) k_causal_dq(CausalGradArgs a) {
  using Tile = RowTile<T, HD>;
  constexpr int KT = Steps<T>::KT, kRows = Steps<T>::kRows, NS = HD / 16, ND = HD / 32;
  using Loader = RowLoader<T, HD, kRows, 4, kVec>;
  __shared__ __align__(1024) char s_kv[2][2][kRows * HD * sizeof(T)];
  const int grp = a.f.H / a.f.G;
  const Work w = work_of(a.f.G, grp);
  RowBlock b;
  if (!find_block(a.f, w.rank, b)) return;
  b.t = b.blocks - 1 - b.t;  // the longest first
  const int head = w.g * grp + w.h;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const int q0 = b.t * kBlock + wave * 32;
  const int qi = min(q0 + (lane & 31), b.n - 1);
  const int last = min(b.t * kBlock + kBlock, b.n) - 1;
  const T* kp = reinterpret_cast<const T*>(a.f.k) + (size_t)b.r0 * a.f.ld_k + w.g * HD;
  const T* vp = reinterpret_cast<const T*>(a.f.v) + (size_t)b.r0 * a.f.ld_v + w.g * HD;
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
  float lse, dot = 0.f;
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
    const size_t at = (size_t)head * a.f.n_rows + b.r0 + qi;
    lse = a.f.lse[at];
    if (h == 0 && q0 + lane < b.n) a.dots[at] = make_float2(lse == -INFINITY ? -INFINITY : -lse * sqrtf((float)HD), -dot);
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
    const uint32_t keys = Tile::row_base(lds_address(s_kv)) + kBuf * 2 * Tile::kRowBytes * kRows;
    const uint32_t values = keys + Tile::kRowBytes * kRows;
    const uint32_t key_columns = Tile::column_base(lds_address(s_kv)) + kBuf * 2 * Tile::kRowBytes * kRows;
    if (kEdge && j0 > q0 + 31) return;
    const int lim = qi - j0 - 4 * h;
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
        const float ds = __builtin_amdgcn_exp2f(__builtin_fmaf(st[i], c, -lse)) * (dp[i] - dot);
        st[i] = kEdge && 32 * kt + acc_row(i) > lim ? 0.f : ds;
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
  // The buffers by turns, in pairs of steps: their addresses are constants.
  using First = std::integral_constant<int, 0>;
  using Second = std::integral_constant<int, 1>;
  static_assert(kBlock % (2 * kRows) == 0, "whole pairs before the edge");
  int j0 = 0;
#pragma unroll 1
  for (; j0 < b.t * kBlock; j0 += 2 * kRows) {
    step(std::false_type{}, First{}, j0);
    step(std::false_type{}, Second{}, j0 + kRows);
  }
#pragma unroll 1
  for (; j0 <= last; j0 += 2 * kRows) {
    step(std::true_type{}, First{}, j0);
    if (j0 + kRows <= last) step(std::true_type{}, Second{}, j0 + kRows);
  }

  if (q0 + (lane & 31) >= b.n) return;
  const float f = 1.f / sqrtf((float)HD);
  T* out = reinterpret_cast<T*>(a.g_q) + (size_t)(b.r0 + qi) * a.ld_g_q + head * HD + 4 * h;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      row_store4<T>(out + 32 * d + acc_row(i), a.vec_q, dq[d][i] * f, dq[d][i + 1] * f, dq[d][i + 2] * f, dq[d][i + 3] * f);
}

// dk and dv of 128 keys of a KV head, over the queries of the heads of `part`
// (part, part + parts, ... of the group's).
template <typename T, int HD, bool kVec>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) k_causal_dkv(CausalGradArgs a) {
  using Tile = RowTile<T, HD>;
  constexpr int KT = Steps<T>::KT, kRows = Steps<T>::kRows, NS = HD / 16, ND = HD / 32;
  using Loader = RowLoader<T, HD, kRows, 4, kVec>;
  __shared__ __align__(1024) char s_qg[2][2][kRows * HD * sizeof(T)];
  __shared__ __align__(16) float s_dots[2][2][kRows];
  const int grp = a.f.H / a.f.G;
  const Work w = work_of(a.f.G, a.parts);
  RowBlock b;
  if (!find_block(a.f, w.rank, b)) return;  // in order: the first keys have the most queries
  const int part = w.h;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const int k0 = b.t * kBlock + wave * 32;
  const int ki = min(k0 + (lane & 31), b.n - 1);
  Frag<T> k[NS], v[NS];
  {
    const T* p = reinterpret_cast<const T*>(a.f.k) + (size_t)(b.r0 + ki) * a.f.ld_k + w.g * HD + 8 * h;
    const T* r = reinterpret_cast<const T*>(a.f.v) + (size_t)(b.r0 + ki) * a.f.ld_v + w.g * HD + 8 * h;
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
  // The steps: every head's rows from the block's first key on, one head after the other.
  const int first = b.t * kBlock, steps = (b.n - first + kRows - 1) / kRows;
  int head = w.g * grp + part, i0 = first;
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
    i0 += kRows;
    if (i0 >= b.n) {
      i0 = first;
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
  int at = first, buf = 0;
#pragma unroll 1
  for (int it = 0; it < total; ++it) {
    if constexpr (kVec) wait_vm<0>();
    __syncthreads();
    if (it + 1 < total) load(buf ^ 1);
    const uint32_t qs = Tile::row_base(lds_address(s_qg[buf][0])), gs = Tile::row_base(lds_address(s_qg[buf][1]));
    const uint32_t q_columns = Tile::column_base(lds_address(s_qg[buf][0]));
    const uint32_t g_columns = Tile::column_base(lds_address(s_qg[buf][1]));
    const bool edge = at < k0 + 31;  // rows before some of the wave's keys
    if (at + kRows > k0) {
#pragma unroll 1
      for (int kt = 0; kt < KT; ++kt) {
        constexpr int kSkip = 32 * Tile::kRowBytes;
        f32x16_t st, dp;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 x = *reinterpret_cast<const float4*>(&s_dots[buf][0][32 * kt + acc_row(i) + 4 * h]);
          const float4 y = *reinterpret_cast<const float4*>(&s_dots[buf][1][32 * kt + acc_row(i) + 4 * h]);
          st[i] = x.x; st[i + 1] = x.y; st[i + 2] = x.z; st[i + 3] = x.w;
          dp[i] = y.x; dp[i + 1] = y.y; dp[i + 2] = y.z; dp[i + 3] = y.w;
        }
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          mfma32(st, Tile::rows(qs + kt * kSkip, 0, s), k[s]);
          mfma32(dp, Tile::rows(gs + kt * kSkip, 0, s), v[s]);
        }
        __builtin_amdgcn_sched_barrier(0);
        const int lim = ki - at - 32 * kt - 4 * h;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool hidden = edge && acc_row(i) < lim;
          st[i] = __builtin_amdgcn_exp2f(st[i] * c);
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
            mfma32(dv[d], Tile::columns(g_columns + kt * kSkip, 16 * j, d), pf);
            mfma32(dk[d], Tile::columns(q_columns + kt * kSkip, 16 * j, d), df);
          }
          
        }
      }
    }
    if (it + 1 < total) put_dots(buf ^ 1);
    buf ^= 1;
    at += kRows;
    if (at >= b.n) at = first;
  }

  if (k0 + (lane & 31) >= b.n) return;
  const float f = 1.f / sqrtf((float)HD);
  const int col = w.g * HD + 4 * h;
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

// Sums the parts in order, four columns a thread.
template <typename T>
__global__ void __launch_bounds__(256) k_causal_join(CausalGradArgs a) {
  const int width = a.f.G * a.f.hd, chunks = width / 4;
  const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int row = (int)(item / chunks), col = (int)(item % chunks) * 4;
  if (row >= a.f.n_rows || row < a.f.row_start[0] || row >= a.f.row_start[a.f.n_seqs]) return;
  const size_t plane = (size_t)a.f.n_rows * width;
  const float* p = a.kv_part + (size_t)row * width + col;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float4 s = *reinterpret_cast<const float4*>(p);
    for (int i = 1; i < a.parts; ++i) {
      const float4 x = *reinterpret_cast<const float4*>(p + i * plane);
      s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
    T* out = which ? reinterpret_cast<T*>(a.g_v) + (size_t)row * a.ld_g_v : reinterpret_cast<T*>(a.g_k) + (size_t)row * a.ld_g_k;
    row_store4<T>(out + col, a.vec_kv, s.x, s.y, s.z, s.w);
    p += a.parts * plane;
  }
}

// ---- launch --------------------------------------------------------------------------
int causal_blocks(int n_rows, int n_seqs) {
  return (int)std::min<int64_t>((int64_t)n_rows / kBlock + std::min(n_seqs, n_rows), n_rows);
}

// One part where the workgroups fill the chip; else one head a workgroup, and
// a pass that adds the heads' shares.
int causal_parts(int n_rows, int n_seqs, int H, int G) {
  return (int64_t)causal_blocks(n_rows, n_seqs) * G >= 1024 ? 1 : H / G;
}

template <typename T, int HD> static void causal_vec(const CausalArgs& a, hipStream_t st) {
  const unsigned grid = work_grid(a.blocks, a.G, a.H / a.G);
  if (a.vec) k_causal<T, HD, true><<<grid, 256, 0, st>>>(a);
  else k_causal<T, HD, false><<<grid, 256, 0, st>>>(a);
}
template <typename T> static hipError_t causal_hd(const CausalArgs& a, hipStream_t st) {
  if (a.hd == 32) causal_vec<T, 32>(a, st);
  else if (a.hd == 64) causal_vec<T, 64>(a, st);
  else causal_vec<T, 128>(a, st);
  return hipGetLastError();
}
hipError_t launch_causal(int dtype, const CausalArgs& a, hipStream_t st) {
  return dtype == 0 ? causal_hd<float>(a, st) : causal_hd<bf16_t>(a, st);
}

template <typename T, int HD> static void causal_grad_vec(const CausalGradArgs& a, hipStream_t st) {
  const unsigned dq = work_grid(a.f.blocks, a.f.G, a.f.H / a.f.G), dkv = work_grid(a.f.blocks, a.f.G, a.parts);
  if (a.f.vec) {
    k_causal_dq<T, HD, true><<<dq, 256, 0, st>>>(a);
    k_causal_dkv<T, HD, true><<<dkv, 256, 0, st>>>(a);
  } else {
    k_causal_dq<T, HD, false><<<dq, 256, 0, st>>>(a);
    k_causal_dkv<T, HD, false><<<dkv, 256, 0, st>>>(a);
  }
}
template <typename T> static hipError_t causal_grad_hd(const CausalGradArgs& a, hipStream_t st) {
  if (a.f.hd == 32) causal_grad_vec<T, 32>(a, st);
  else if (a.f.hd == 64) causal_grad_vec<T, 64>(a, st);
  else causal_grad_vec<T, 128>(a, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  const int64_t quads = (int64_t)a.f.n_rows * a.f.G * a.f.hd / 4;
  k_causal_join<T><<<(unsigned)((quads + 255) / 256), 256, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_causal_grad(int dtype, const CausalGradArgs& a, hipStream_t st) {
  return dtype == 0 ? causal_grad_hd<float>(a, st) : causal_grad_hd<bf16_t>(a, st);
}

}  // namespace jf
