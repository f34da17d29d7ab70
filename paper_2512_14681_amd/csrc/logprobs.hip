// Log probabilities of given tokens with entropy and best alternatives
// (jf_token_logprobs), and their gradient (jf_token_logprobs_grad).
//
// One pass over a row's logits x with m = max x, s = sum e^(x - m) and
// u = sum e^(x - m) (x - m), all in fp32 and relative to the running maximum:
//   log p_t = (x_t - m) - log s,   entropy = log s - u / s.
// The alternatives are the k largest 64-bit keys (value, then lowest index).
// Bound by memory without alternatives (512 rows of 152064 fp32 logits 55 us,
// 5.6 TB/s, kept in the caches for the gradient; 50 us if loaded as read once,
// which calls with alternatives do), by the vector unit with them where the
// rows are few (64 rows in bf16: k = 0 8 us, k = 8 12.4 us; 400 rows in fp32 and
// k = 8 46 us, 5.2 TB/s).  A row is split until there are about four
// workgroups a compute unit; a second launch joins (4 us).
#include <algorithm>

#include "jf_device.h"
#include "jf_internal.h"

namespace jf {

constexpr int kTileElems = 16;  // elements of a lane in one step
constexpr int kTile = 256 * kTileElems;

// Sixteen bytes at any address of the elements' alignment.
typedef float f32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(2)));

// The column of element j of a lane's tile: runs of 16 bytes.
template <typename T> __device__ __forceinline__ int tile_col(int base, int tid, int j) {
  constexpr int N = 16 / (int)sizeof(T);
  return base + 256 * N * (j / N) + N * tid + j % N;
}
template <typename T, bool ONCE> __device__ __forceinline__ void load_run(const T* p, float* x) {
  if constexpr (sizeof(T) == 4) {
    const auto* q = reinterpret_cast<const f32x4_any_t*>(p);
    const f32x4_any_t w = ONCE ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = w[e];
  } else {
    const auto* q = reinterpret_cast<const u32x4_any_t*>(p);
    const u32x4_any_t w = ONCE ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
  }
}
template <typename T> __device__ __forceinline__ void store_run(T* p, const float* y) {
  if constexpr (sizeof(T) == 4) {
    __builtin_nontemporal_store(f32x4_any_t{y[0], y[1], y[2], y[3]}, reinterpret_cast<f32x4_any_t*>(p));
  } else {
    const u32x4_any_t w = {pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]),
                           pack_bf16x2(y[6], y[7])};
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_any_t*>(p));
  }
}
// A lane's sixteen elements of a row from column base on; -inf at and past v1.
template <typename T, bool ONCE> __device__ __forceinline__ void load_tile(const T* row, int base, int tid, int v1, float (&x)[kTileElems]) {
  constexpr int N = 16 / (int)sizeof(T);
  if (base + kTile <= v1) {
#pragma unroll
    for (int j = 0; j < kTileElems; j += N) load_run<T, ONCE>(row + tile_col<T>(base, tid, j), x + j);
  } else {
#pragma unroll
    for (int j = 0; j < kTileElems; j += N) {
      const int c = tile_col<T>(base, tid, j);
      if (c + N <= v1) {
        load_run<T, ONCE>(row + c, x + j);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[j + e] = c + e < v1 ? to_f32<T>(row[c + e]) : -INFINITY;
      }
    }
  }
}

// A lane's value in every lane, and the value of the lane below, on the
// vector unit (through LDS the latency of six exchanges is in every insert).
__device__ __forceinline__ uint64_t from_lane(uint64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t from_lane_below(uint64_t v) {
  constexpr int kWaveShiftRight1 = 0x138;
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, kWaveShiftRight1, 0xF, 0xF, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), kWaveShiftRight1, 0xF, 0xF, true);
  return (uint64_t)hi << 32 | lo;
}

// A logit's key: rising with the value, then with a falling column.  -0 and +0
// are one value: the sum makes both +0.
__device__ __forceinline__ uint64_t logit_key(float v, uint32_t col) { return argmax_key(v + 0.f, col); }
// The value of a key.
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}

// Keys larger than `key` among n in LDS (zeros up to the next multiple of 8):
// its place in their order.
__device__ __forceinline__ int key_rank(const uint64_t* keys, int n, uint64_t key) {
  int rank = 0;
  for (int i = 0; i < n; i += 8)
#pragma unroll
    for (int j = 0; j < 8; ++j) rank += keys[i + j] > key;
  return rank;
}

// A wave's best keys.  It collects candidates side by side in LDS, elements
// above a value that k earlier ones reach, and ranks them by counting when
// they are too many and at the end, so that most tiles cost a comparison an
// element (kept sorted over the lanes instead, key by key, 64 rows of 152064
// bf16 logits took 15.2 us for k = 8 and 20.7 for k = 20, now 12.6 and 16.3).
constexpr int kCand = 128;
template <typename T> struct TopList {
  uint64_t* cand;  // kCand of this wave: `sorted` keys, then pairs of value and column
  uint64_t* best;  // kMaxTop of this wave: scratch
  int k, n, sorted;
  float least;     // k candidates reach it (-inf: not known of k)
  __device__ __forceinline__ void init(int k_, uint64_t* cand_, uint64_t* best_) {
    k = k_; cand = cand_; best = best_;
    n = sorted = 0;
    least = -INFINITY;
  }
  static __device__ __forceinline__ void fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

  // This lane's of the k best candidates in order (0: none), which alone stay.
  __device__ __forceinline__ uint64_t rank() {
    const int lane = threadIdx.x & 63;
    if (lane < kMaxTop) best[lane] = 0;
    uint64_t mine[kCand / 64];
#pragma unroll
    for (int h = 0; h < kCand / 64; ++h) {
      const int i = 64 * h + lane;
      const uint64_t c = cand[i];
      mine[h] = i >= n ? 0 : (i < sorted ? c : logit_key(__uint_as_float((uint32_t)(c >> 32)), (uint32_t)c));
      cand[i] = mine[h];
    }
    fence();
#pragma unroll
    for (int h = 0; h < kCand / 64; ++h)
      if (mine[h]) {
        const int at = key_rank(cand, n, mine[h]);
        if (at < k) best[at] = mine[h];
      }
    fence();
    const uint64_t key = lane < k ? best[lane] : 0;
    keep(key);
    return key;
  }
  // The candidates become these: the k best in order, one a lane.
  __device__ __forceinline__ void keep(uint64_t key) {
    const int lane = threadIdx.x & 63;
    n = sorted = __popcll(__ballot(lane < k && key));
    if (lane < k) cand[lane] = key;
    const uint64_t kth = from_lane(key, k - 1);
    if (kth) least = key_value(kth);
    fence();
  }
  // Adds the elements for which in(value), as they are; false (and nothing added) if they do not fit.
  template <typename F>
  __device__ __forceinline__ bool add(const float (&x)[kTileElems], int base, int tid, F in) {
    int to = n;
#pragma unroll
    for (int j = 0; j < kTileElems; ++j) {
      const bool it = in(x[j]);
      const uint64_t mask = __ballot(it);
      if (mask) {
        const int at = to + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
        if (it && at < kCand)
          cand[at] = (uint64_t)__float_as_uint(x[j]) << 32 | (uint32_t)tile_col<T>(base, tid, j);
        to += __popcll(mask);
      }
    }
    if (to > kCand) return false;
    n = to;
    return true;
  }
  // A value that k of the tile's elements reach (-inf: not known of k): the
  // k-th largest of the lanes' maxima, searched bit by bit in the upper half
  // of the ordered values only; a little lower, which admits a few more.
  __device__ __forceinline__ float reached(float mx) const {
    const uint32_t u = __float_as_uint(mx), om = mx > -INFINITY ? ((u & 0x80000000u) ? ~u : (u | 0x80000000u)) : 0;
    uint32_t t = 0;
#pragma unroll
    for (int b = 31; b >= 16; --b) {
      const uint32_t with = t | 1u << b;
      t = __popcll(__ballot(om >= with)) >= k ? with : t;
    }
    return t ? key_value((uint64_t)t << 32) : -INFINITY;
  }
  // A tile's elements, mx their maximum in this lane.  Tiles come by rising
  // column, so an element that only equals `least` comes after k others.
  __device__ __forceinline__ void offer(const float (&x)[kTileElems], float mx, int base, int tid) {
    if (!__any(mx > least)) return;
    if (n >= 2 * k) {  // a better `least` (400 rows of fp32, 13 tiles a split: 46 us, 54 without)
      rank();
      if (!__any(mx > least)) return;
    }
    const float above = least;  // -inf admits the finite ones
    if (n && add(x, base, tid, [&](float v) { return v > above; })) return;
    if (n) rank();
    const float reach = fmaxf(reached(mx), least), low = fmaxf(reach, -3.402823466e38f);  // only finite ones
    if (add(x, base, tid, [&](float v) { return v >= low; })) {
      least = reach;
      return;
    }
    // the best sit in few lanes, or many are equal: one by one into the sorted list
    const int lane = tid & 63;
    uint64_t key = lane < n ? cand[lane] : 0, kth = from_lane(key, k - 1);
#pragma unroll
    for (int j = 0; j < kTileElems; ++j) {
      const uint64_t c = x[j] >= low ? logit_key(x[j], (uint32_t)tile_col<T>(base, tid, j)) : 0;
      uint64_t left = __ballot(c > kth);
      while (left) {
        const uint64_t y = from_lane(c, __builtin_ctzll(left));
        left &= left - 1;
        if (y <= kth) continue;
        const int at = __popcll(__ballot(key > y));
        const uint64_t up = from_lane_below(key);
        key = lane < at ? key : (lane == at ? y : up);
        kth = from_lane(key, k - 1);
      }
    }
    keep(key);
  }
};

struct Stat { float m, s, u; };
// The statistics of two sets together.
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b) {
  const float m = fmaxf(a.m, b.m), mu = m == -INFINITY ? 0.f : m;
  // max keeps 0 * inf away: a set without a finite element has s = u = 0
  const float da = fmaxf(a.m - mu, -1e4f), db = fmaxf(b.m - mu, -1e4f);
  const float fa = __expf(da), fb = __expf(db);
  return {m, a.s * fa + b.s * fb, (a.u + a.s * da) * fa + (b.u + b.s * db) * fb};
}

// A row's outputs from its statistics and best keys (in LDS).  A row that is
// no distribution (its maximum not finite, or a NaN among its logits) has NaN
// everywhere and no alternatives.
__device__ __forceinline__ void finish_row(const LogprobArgs& a, int r, const Stat& st, float xt, const uint64_t* best) {
  const bool good = st.m > -INFINITY && st.m < INFINITY && st.s == st.s;
  const float ls = good ? logf(st.s) : NAN;
  if (threadIdx.x == 0) {
    if (a.logprob) {
      const int t = a.tokens[r];
      a.logprob[r] = t == -1 ? 0.f : (t >= 0 && t < a.V && good ? (xt - st.m) - ls : NAN);
    }
    if (a.entropy) a.entropy[r] = good ? ls - st.u / st.s : NAN;
    if (a.norm) {
      a.norm[2 * (size_t)r] = good ? st.m : NAN;
      a.norm[2 * (size_t)r + 1] = ls;
    }
  }
  const int i = threadIdx.x;
  if (i < a.k) {
    const uint64_t key = good ? best[i] : 0;
    if (a.top_ids) a.top_ids[(size_t)r * a.k + i] = key ? (int32_t)argmax_key_index(key) : -1;
    if (a.top_logprob)
      a.top_logprob[(size_t)r * a.k + i] = key ? (key_value(key) - st.m) - ls : (good ? -INFINITY : NAN);
  }
}

// Workgroup: one row's columns [split * per, (split + 1) * per).
template <typename T, bool TOP>
__global__ void __launch_bounds__(256) k_logprobs(LogprobArgs a, int per) {
  __shared__ Stat s_st[4];
  __shared__ uint64_t s_top[4][kMaxTop], s_cand[TOP ? 4 : 1][kCand];
  const int r = blockIdx.x, split = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const T* row = reinterpret_cast<const T*>(a.x) + (size_t)r * a.ld;
  const int v0 = split * per, v1 = min(a.V, v0 + per);
  Stat st = {-INFINITY, 0.f, 0.f};
  TopList<T> top;
  if constexpr (TOP) top.init(a.k, s_cand[wave], s_top[wave]);
  float next[kTileElems];
  load_tile<T, TOP>(row, v0, tid, v1, next);
  for (int base = v0; base < v1; base += kTile) {
    float x[kTileElems];
#pragma unroll
    for (int j = 0; j < kTileElems; ++j) x[j] = next[j];
    if (base + kTile < v1) load_tile<T, TOP>(row, base + kTile, tid, v1, next);  // in flight during this tile's work
    float mt = x[0];
#pragma unroll
    for (int j = 1; j < kTileElems; ++j) mt = fmaxf(mt, x[j]);
    const float m = fmaxf(st.m, mt), mu = m == -INFINITY ? 0.f : m;
    const float d0 = fmaxf(st.m - mu, -1e4f), f = __expf(d0);
    st.u = (st.u + st.s * d0) * f;
    st.s *= f;
    st.m = m;
#pragma unroll
    for (int j = 0; j < kTileElems; ++j) {
      const float d = x[j] - mu, e = __expf(d);
      st.s += e;
      st.u = __builtin_fmaf(e, fmaxf(d, -1e4f), st.u);  // max: 0 * inf
    }
    if constexpr (TOP) {
      top.offer(x, mt, base, tid);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
    st = join(st, Stat{__shfl_xor(st.m, d), __shfl_xor(st.s, d), __shfl_xor(st.u, d)});
  if (lane == 0) s_st[wave] = st;
  if constexpr (TOP) top.rank();  // into s_top[wave]
  __syncthreads();
  st = join(join(s_st[0], s_st[1]), join(s_st[2], s_st[3]));
  uint64_t* best = s_cand[0];
  if constexpr (TOP) {
    // the waves' lists, ranked by counting
    if (tid < a.k) best[tid] = 0;
    uint64_t key = 0;
    int rank = 0;
    if (tid < 4 * a.k) {
      key = s_top[tid / a.k][tid % a.k];
      if (key)
        for (int w = 0; w < 4; ++w) rank += key_rank(s_top[w], a.k, key);
    }
    __syncthreads();
    if (key && rank < a.k) best[rank] = key;
    __syncthreads();
  }
  if (a.splits == 1) {
    const int t = a.logprob ? a.tokens[r] : -1;
    finish_row(a, r, st, t >= 0 && t < a.V ? to_f32<T>(row[t]) : 0.f, best);
    return;
  }
  const size_t at = (size_t)r * a.splits + split;
  if (tid == 0) *reinterpret_cast<float4*>(a.part + at * 4) = make_float4(st.m, st.s, st.u, 0.f);
  if (TOP && tid < a.k) a.top_part[at * a.k + tid] = best[tid];
}

// Joins a row's splits.  Of S lists, with q = ceil(k / S), the ceil(k / q)-th
// largest of their q-th keys has k keys at or above it; those that reach it
// are ranked by counting.
constexpr int kWantBlocks = 1024, kMaxRowSplits = 64;
template <typename T>
__global__ void __launch_bounds__(256) k_logprobs_join(LogprobArgs a) {
  __shared__ uint64_t s_key[kMaxRowSplits * kMaxTop], s_best[kMaxTop], s_least;
  __shared__ int s_n;
  __shared__ Stat s_st;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const T* row = reinterpret_cast<const T*>(a.x) + (size_t)r * a.ld;
  const int t = a.logprob ? a.tokens[r] : -1;
  const float xt = t >= 0 && t < a.V ? to_f32<T>(row[t]) : 0.f;
  if (tid < 64) {  // kMaxRowSplits: one a lane
    Stat st = {-INFINITY, 0.f, 0.f};
    if (lane < a.splits) {
      const float4 p = *reinterpret_cast<const float4*>(a.part + ((size_t)r * a.splits + lane) * 4);
      st = Stat{p.x, p.y, p.z};
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
      st = join(st, Stat{__shfl_xor(st.m, d), __shfl_xor(st.s, d), __shfl_xor(st.u, d)});
    if (tid == 0) {
      s_st = st;
      s_n = 0;
    }
  }
  if (a.k) {
    const uint64_t* p = a.top_part + (size_t)r * a.splits * a.k;
    const int q = (a.k + a.splits - 1) / a.splits, nth = (a.k + q - 1) / q;
    const uint64_t mine = tid < a.splits ? p[tid * a.k + q - 1] : 0;
    if (tid < kMaxRowSplits) s_key[tid] = mine;
    if (tid < a.k) s_best[tid] = 0;
    if (tid == 0) s_least = 0;
    __syncthreads();
    if (mine && key_rank(s_key, a.splits, mine) == nth - 1) s_least = mine;  // fewer keys: 0, all of them
    __syncthreads();
    const uint64_t least = s_least;
    for (int i = tid; i < a.splits * a.k; i += 256) {
      const uint64_t key = p[i];
      if (key && key >= least) s_key[atomicAdd(&s_n, 1)] = key;  // in any order: ranks do not depend on it
    }
    __syncthreads();
    if (tid < 8 && (s_n & 7) && tid >= (s_n & 7)) s_key[s_n / 8 * 8 + tid] = 0;
    __syncthreads();
    for (int i = tid; i < s_n; i += 256) {
      const uint64_t key = s_key[i];
      const int rank = key_rank(s_key, s_n, key);
      if (rank < a.k) s_best[rank] = key;
    }
  }
  __syncthreads();
  finish_row(a, r, s_st, xt, s_best);
}

// ---- gradient ------------------------------------------------------------------------
// dx_j = g (1[j = t] - p_j) - h p_j (log p_j + H); nothing read and zeros
// written for a row whose g and h are both 0.  Bound by memory: 512 rows of
// 152064 fp32 logits 89 us, 7.0 TB/s.  The gradient is stored without being
// kept in the caches (97 us when it is), and the last rows come first: they
// are what the forward pass left there.
template <typename T>
__global__ void __launch_bounds__(256) k_logprobs_grad(LogprobGradArgs a, int tiles) {
  constexpr int N = 16 / (int)sizeof(T);
  const unsigned block = gridDim.x - 1 - blockIdx.x;
  const int r = block / tiles, tid = threadIdx.x, base = block % tiles * kTile;
  const T* row = reinterpret_cast<const T*>(a.x) + (size_t)r * a.ld;
  T* out = reinterpret_cast<T*>(a.grad) + (size_t)r * a.ld_g;
  const int t = a.tokens ? a.tokens[r] : -1;
  float g = a.g_logprob ? a.g_logprob[r] : 0.f;
  const float h = a.g_entropy ? a.g_entropy[r] : 0.f;
  if (t == -1) g = 0.f;                       // no token: its log probability is a constant
  else if (t < -1 || t >= a.V) g = g == 0.f ? 0.f : NAN;
  const float m = a.norm[2 * (size_t)r], ls = a.norm[2 * (size_t)r + 1], H = a.entropy ? a.entropy[r] : 0.f;
  float y[kTileElems];
  if (g == 0.f && h == 0.f) {
#pragma unroll
    for (int j = 0; j < kTileElems; ++j) y[j] = 0.f;
  } else {
    float x[kTileElems];
    load_tile<T, true>(row, base, tid, a.V, x);
#pragma unroll
    for (int j = 0; j < kTileElems; ++j) {
      const float lp = (x[j] - m) - ls, p = __expf(lp);
      float d = -g * p;
      if (h != 0.f) d -= h * p * (fmaxf(lp, -1e4f) + H);  // max: 0 * inf
      y[j] = tile_col<T>(base, tid, j) == t ? d + g : d;
    }
  }
#pragma unroll
  for (int j = 0; j < kTileElems; j += N) {
    const int c = tile_col<T>(base, tid, j);
    if (c + N <= a.V) {
      store_run<T>(out + c, y + j);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (c + e < a.V) out[c + e] = from_f32<T>(y[j + e]);
    }
  }
}

// ---- launches ------------------------------------------------------------------------
// Splits of a row: about four workgroups a compute unit, each with a tile or more.
static int row_splits(int V) { return (int)std::min<int64_t>(((int64_t)V + kTile - 1) / kTile, kMaxRowSplits); }
int logprob_splits(int R, int V) { return std::min(row_splits(V), (kWantBlocks + R - 1) / R); }
size_t logprob_parts(int R, int V) {
  return std::min((size_t)R * row_splits(V), (size_t)R + kWantBlocks);
}

template <typename T> static hipError_t logprobs(const LogprobArgs& a, hipStream_t st) {
  const int tiles = (int)(((int64_t)a.V + kTile - 1) / kTile);
  const int per = (tiles + a.splits - 1) / a.splits * kTile;
  const dim3 grid((unsigned)a.R, (unsigned)a.splits);
  if (a.k) k_logprobs<T, true><<<grid, 256, 0, st>>>(a, per);
  else k_logprobs<T, false><<<grid, 256, 0, st>>>(a, per);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  k_logprobs_join<T><<<(unsigned)a.R, 256, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_logprobs(int dtype, const LogprobArgs& a, hipStream_t st) {
  return dtype == 0 ? logprobs<float>(a, st) : logprobs<bf16_t>(a, st);
}

template <typename T> static hipError_t logprobs_grad(const LogprobGradArgs& a, hipStream_t st) {
  const int tiles = (int)(((int64_t)a.V + kTile - 1) / kTile);
  const unsigned grid = (unsigned)((int64_t)tiles * a.R);
  k_logprobs_grad<T><<<grid, 256, 0, st>>>(a, tiles);
  return hipGetLastError();
}
hipError_t launch_logprobs_grad(int dtype, const LogprobGradArgs& a, hipStream_t st) {
  return dtype == 0 ? logprobs_grad<float>(a, st) : logprobs_grad<bf16_t>(a, st);
}

}  // namespace jf
