// Log probabilities of given tokens with entropy and best alternatives
// (jf_token_logprobs), and their gradient (jf_token_logprobs_grad).
//
// One pass over a row's logits x with m = max x, s = sum e^(x - m) and
// u = sum e^(x - m) (x - m), all in fp32 and relative to the running maximum:
//   log p_t = (x_t - m) - log s,   entropy = log s - u / s.
// The alternatives are the k largest 64-bit keys (value, then lowest index);
// a wave keeps its k best sorted over its lanes and looks at an element only
// if it beats the k-th.
#include <algorithm>

#include "jf_device.h"
#include "jf_internal.h"

namespace jf {

constexpr int kTileElems = 16;  // elements of a lane in one step

// Sixteen elements of a lane: columns base + 4 * 256 * j + 4 * tid + e of the
// row for VEC, base + 256 * j + tid otherwise; -inf at and past v1.
template <typename T, bool VEC>
__device__ __forceinline__ void load_tile(const T* row, int base, int tid, int v1, float (&x)[kTileElems]) {
  if constexpr (VEC && sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = base + 1024 * j + 4 * tid;
      if (c + 4 <= v1) {
        const float4 w = *reinterpret_cast<const float4*>(row + c);
        x[4 * j] = w.x; x[4 * j + 1] = w.y; x[4 * j + 2] = w.z; x[4 * j + 3] = w.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * j + e] = c + e < v1 ? row[c + e] : -INFINITY;
      }
    }
  } else if constexpr (VEC) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = base + 2048 * j + 8 * tid;
      if (c + 8 <= v1) {
        const uint4 w = *reinterpret_cast<const uint4*>(row + c);
        const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[8 * j + 2 * e] = __uint_as_float(a[e] << 16);
          x[8 * j + 2 * e + 1] = __uint_as_float(a[e] & 0xFFFF0000u);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[8 * j + e] = c + e < v1 ? to_f32<T>(row[c + e]) : -INFINITY;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < kTileElems; ++j) {
      const int c = base + 256 * j + tid;
      x[j] = c < v1 ? to_f32<T>(row[c]) : -INFINITY;
    }
  }
}
// The column of element j of load_tile.
template <typename T, bool VEC> __device__ __forceinline__ int tile_col(int base, int tid, int j) {
  if constexpr (VEC && sizeof(T) == 4) return base + 1024 * (j >> 2) + 4 * tid + (j & 3);
  else if constexpr (VEC) return base + 2048 * (j >> 3) + 8 * tid + (j & 7);
  else return base + 256 * j + tid;
}

__device__ __forceinline__ uint64_t shfl64(uint64_t v, int lane) {
  const uint32_t lo = __shfl((int)(uint32_t)v, lane), hi = __shfl((int)(uint32_t)(v >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}

// A wave's best keys, largest first, one a lane (0: none).
struct TopList {
  uint64_t key, kth;  // this lane's; the k-th best (every lane)
  int k;
  __device__ __forceinline__ void init(int k_) { key = kth = 0; k = k_; }
  // Puts one key (the same in every lane) in its place.
  __device__ __forceinline__ void insert(uint64_t c) {
    const int lane = threadIdx.x & 63;
    const int at = __popcll(__ballot(key > c));
    const uint64_t up = shfl64(key, max(lane - 1, 0));
    key = lane < at ? key : (lane == at ? c : up);
    kth = shfl64(key, k - 1);
  }
  // Offers one key a lane (0: none).
  __device__ __forceinline__ void offer(uint64_t c) {
    uint64_t left = __ballot(c > kth);
    while (left) {
      const uint64_t x = shfl64(c, __builtin_ctzll(left));
      left &= left - 1;
      if (x > kth) insert(x);
    }
  }
};

// -inf is no alternative: key 0.
__device__ __forceinline__ uint64_t top_key(float v, int col) {
  return v > -INFINITY ? argmax_key(v, (uint32_t)col) : 0;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}

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
template <typename T, bool VEC, bool TOP>
__global__ void __launch_bounds__(256) k_logprobs(LogprobArgs a, int per) {
  __shared__ Stat s_st[4];
  __shared__ uint64_t s_top[4][kMaxTop];
  const int r = blockIdx.x, split = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const T* row = reinterpret_cast<const T*>(a.x) + (size_t)r * a.ld;
  const int v0 = split * per, v1 = min(a.V, v0 + per);
  Stat st = {-INFINITY, 0.f, 0.f};
  TopList top;
  top.init(a.k);
  for (int base = v0; base < v1; base += 256 * kTileElems) {
    float x[kTileElems];
    load_tile<T, VEC>(row, base, tid, v1, x);
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
      if (__any(top_key(mt, 0) > top.kth)) {
#pragma unroll
        for (int j = 0; j < kTileElems; ++j) top.offer(top_key(x[j], tile_col<T, VEC>(base, tid, j)));
      }
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
    st = join(st, Stat{__shfl_xor(st.m, d), __shfl_xor(st.s, d), __shfl_xor(st.u, d)});
  if (lane == 0) s_st[wave] = st;
  if (TOP && lane < a.k) s_top[wave][lane] = top.key;
  __syncthreads();
  st = join(join(s_st[0], s_st[1]), join(s_st[2], s_st[3]));
  if constexpr (TOP) {
    if (wave == 0)
#pragma unroll
      for (int w = 1; w < 4; ++w) top.offer(lane < a.k ? s_top[w][lane] : 0);
    if (wave == 0 && lane < a.k) s_top[0][lane] = top.key;
    __syncthreads();
  }
  if (a.splits == 1) {
    const int t = a.logprob ? a.tokens[r] : -1;
    finish_row(a, r, st, t >= 0 && t < a.V ? to_f32<T>(row[t]) : 0.f, s_top[0]);
    return;
  }
  const size_t at = (size_t)r * a.splits + split;
  if (tid == 0) *reinterpret_cast<float4*>(a.part + at * 4) = make_float4(st.m, st.s, st.u, 0.f);
  if (TOP && tid < a.k) a.top_part[at * a.k + tid] = s_top[0][tid];
}

// Joins a row's splits: one wave a row.
template <typename T>
__global__ void __launch_bounds__(64) k_logprobs_join(LogprobArgs a) {
  __shared__ uint64_t s_top[kMaxTop];
  const int r = blockIdx.x, lane = threadIdx.x;
  Stat st = {-INFINITY, 0.f, 0.f};
  for (int i = lane; i < a.splits; i += 64) {
    const float4 p = *reinterpret_cast<const float4*>(a.part + ((size_t)r * a.splits + i) * 4);
    st = join(st, Stat{p.x, p.y, p.z});
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
    st = join(st, Stat{__shfl_xor(st.m, d), __shfl_xor(st.s, d), __shfl_xor(st.u, d)});
  if (a.k) {
    TopList top;
    top.init(a.k);
    const uint64_t* p = a.top_part + (size_t)r * a.splits * a.k;
    for (int i = 0; i < a.splits * a.k; i += 64) top.offer(i + lane < a.splits * a.k ? p[i + lane] : 0);
    if (lane < a.k) s_top[lane] = top.key;
    __syncthreads();
  }
  const int t = a.logprob ? a.tokens[r] : -1;
  const T* row = reinterpret_cast<const T*>(a.x) + (size_t)r * a.ld;
  finish_row(a, r, st, t >= 0 && t < a.V ? to_f32<T>(row[t]) : 0.f, s_top);
}

// ---- gradient ------------------------------------------------------------------------
// dx_j = g (1[j = t] - p_j) - h p_j (log p_j + H); nothing read and zeros
// written for a row whose g and h are both 0.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) k_logprobs_grad(LogprobGradArgs a, int tiles) {
  const int r = blockIdx.x / tiles, tid = threadIdx.x, base = blockIdx.x % tiles * 256 * kTileElems;
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
    load_tile<T, VEC>(row, base, tid, a.V, x);
#pragma unroll
    for (int j = 0; j < kTileElems; ++j) {
      const float lp = (x[j] - m) - ls, p = __expf(lp);
      float d = -g * p;
      if (h != 0.f) d -= h * p * (fmaxf(lp, -1e4f) + H);  // max: 0 * inf
      y[j] = tile_col<T, VEC>(base, tid, j) == t ? d + g : d;
    }
  }
  if constexpr (VEC && sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = base + 1024 * j + 4 * tid;
      if (c + 4 <= a.V) {
        *reinterpret_cast<float4*>(out + c) = make_float4(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < a.V) out[c + e] = y[4 * j + e];
      }
    }
  } else if constexpr (VEC) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = base + 2048 * j + 8 * tid;
      if (c + 8 <= a.V) {
        *reinterpret_cast<uint4*>(out + c) =
            make_uint4(pack_bf16x2(y[8 * j], y[8 * j + 1]), pack_bf16x2(y[8 * j + 2], y[8 * j + 3]),
                       pack_bf16x2(y[8 * j + 4], y[8 * j + 5]), pack_bf16x2(y[8 * j + 6], y[8 * j + 7]));
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < a.V) out[c + e] = from_f32<T>(y[8 * j + e]);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < kTileElems; ++j) {
      const int c = base + 256 * j + tid;
      if (c < a.V) out[c] = from_f32<T>(y[j]);
    }
  }
}

// ---- launches ------------------------------------------------------------------------
constexpr int kTile = 256 * kTileElems;

// Splits of a row: about four workgroups a compute unit, each with a tile or more.
constexpr int kWantBlocks = 1024, kMaxRowSplits = 64;
static int row_splits(int V) { return (int)std::min<int64_t>(((int64_t)V + kTile - 1) / kTile, kMaxRowSplits); }
int logprob_splits(int R, int V) { return std::min(row_splits(V), (kWantBlocks + R - 1) / R); }
size_t logprob_parts(int R, int V) {
  return std::min((size_t)R * row_splits(V), (size_t)R + kWantBlocks);
}

static bool vector_rows(const void* p, size_t ld, size_t esz) { return (((uintptr_t)p | (ld * esz)) & 15) == 0; }

template <typename T> static hipError_t logprobs(const LogprobArgs& a, hipStream_t st) {
  const int tiles = (int)(((int64_t)a.V + kTile - 1) / kTile);
  const int per = (tiles + a.splits - 1) / a.splits * kTile;
  const dim3 grid((unsigned)a.R, (unsigned)a.splits);
  const bool vec = vector_rows(a.x, a.ld, sizeof(T));
  if (vec && a.k) k_logprobs<T, true, true><<<grid, 256, 0, st>>>(a, per);
  else if (vec) k_logprobs<T, true, false><<<grid, 256, 0, st>>>(a, per);
  else if (a.k) k_logprobs<T, false, true><<<grid, 256, 0, st>>>(a, per);
  else k_logprobs<T, false, false><<<grid, 256, 0, st>>>(a, per);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  k_logprobs_join<T><<<(unsigned)a.R, 64, 0, st>>>(a);
  return hipGetLastError();
}
hipError_t launch_logprobs(int dtype, const LogprobArgs& a, hipStream_t st) {
  return dtype == 0 ? logprobs<float>(a, st) : logprobs<bf16_t>(a, st);
}

template <typename T> static hipError_t logprobs_grad(const LogprobGradArgs& a, hipStream_t st) {
  const int tiles = (int)(((int64_t)a.V + kTile - 1) / kTile);
  const unsigned grid = (unsigned)((int64_t)tiles * a.R);
  if (vector_rows(a.x, a.ld, sizeof(T)) && vector_rows(a.grad, a.ld_g, sizeof(T)))
    k_logprobs_grad<T, true><<<grid, 256, 0, st>>>(a, tiles);
  else
    k_logprobs_grad<T, false><<<grid, 256, 0, st>>>(a, tiles);
  return hipGetLastError();
}
hipError_t launch_logprobs_grad(int dtype, const LogprobGradArgs& a, hipStream_t st) {
  return dtype == 0 ? logprobs_grad<float>(a, st) : logprobs_grad<bf16_t>(a, st);
}

}  // namespace jf
