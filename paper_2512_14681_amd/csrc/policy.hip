// Clipped policy loss with a KL term, and its gradient (jf_policy_loss).
//
//   r = e^(lp - old), policy = -min(r A, clip(r, 1 - low, 1 + high) A)
//   k = ref - lp, kl = e^k - k - 1 (an estimate of the KL divergence that is never negative)
//   loss = scale sum w (policy + kl_weight kl - entropy_weight H)
//   dloss/dlp = scale w (-A r unless clipped + kl_weight (1 - e^k)), dloss/dH = -scale entropy_weight w
//
// Clipped: A > 0 and r > 1 + high, or A < 0 and r < 1 - low.  All of it in 64
// bits: log probabilities lie close together, so that ratios are next to 1
// and KL terms next to 0, and a rounded ratio would take the wrong side of a
// border.  A row takes up to 32 bytes and two exponentials of 64 bits, which
// bound a large batch: 960 thousand rows, 31 MB, take 3.0 us to count, 12 us
// here and 3.9 us to add up, where a copy of them takes 6.
//
// Sums add up in an order that does not depend on timing: a thread's rows, a
// workgroup's threads, then the workgroups.  What is counted with atomics is
// whole numbers.
#include <algorithm>

#include "jf_device.h"
#include "jf_internal.h"

namespace jf {

constexpr int kTerms = 5;       // policy, KL, entropy, clipped (weighted), tokens
constexpr int kRowsBlock = 1024;  // rows of a workgroup, four a thread
constexpr int kSmallRows = 4096;  // rows and sequences that one workgroup takes in one launch

// Workspace: the number of sequences with tokens, a count for every block of rows, a count for
// every sequence, then the workgroups' sums.
struct PolicyWs {
  int32_t *seqs, *block, *count;
  double* part;
};
static int policy_blocks(int n_rows) { return (n_rows + kRowsBlock - 1) / kRowsBlock; }
static __host__ __device__ size_t policy_part_at(int n_seqs, int blocks) { return ((size_t)(4 + blocks + n_seqs) * 4 + 15) / 16 * 16; }
static __device__ PolicyWs policy_ws(const PolicyArgs& a) {
  int32_t* p = reinterpret_cast<int32_t*>(a.ws);
  return PolicyWs{p, p + 4, p + 4 + a.blocks, reinterpret_cast<double*>(reinterpret_cast<char*>(a.ws) + policy_part_at(a.n_seqs, a.blocks))};
}
size_t policy_ws_bytes(int n_seqs, int n_rows) {
  const int blocks = policy_blocks(n_rows);
  return policy_part_at(n_seqs, blocks) + (size_t)blocks * kTerms * 8;
}

// The sequence of a row between the first start and the last one.
__device__ __forceinline__ int seq_of(const int32_t* start, int lo, int hi, int row) {  // start[lo] <= row < start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= row) lo = mid;
    else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ bool start_bad(const PolicyArgs& a, int s) {
  const int r0 = a.row_start[s], r1 = a.row_start[s + 1];
  return r0 < 0 || r1 < r0 || r1 > a.n_rows;
}

// What a row brings, in registers before anything is computed.
struct PolicyRow {
  float lp, old, ref, entropy, adv;
};

// A row's terms with weight w, added to sum; its gradient.
__device__ __forceinline__ void policy_row(const PolicyArgs& a, const PolicyRow& x, double w, double (&sum)[kTerms],
                                           float& g_lp, float& g_entropy) {
  const double lp = x.lp, adv = x.adv;
  const double ratio = exp(lp - (double)x.old);
  const bool clipped = (adv > 0.0 && ratio > 1.0 + a.high) || (adv < 0.0 && ratio < 1.0 - a.low);
  const double used = clipped ? (adv > 0.0 ? 1.0 + a.high : 1.0 - a.low) : ratio;
  double g = clipped || adv == 0.0 ? 0.0 : -adv * ratio;  // an advantage of 0 takes no ratio, infinite ones among them
  sum[0] += adv == 0.0 ? 0.0 : -w * (used * adv);
  if (a.ref) {
    const double k = (double)x.ref - lp;
    // e^k - 1 - k: the difference cancels for small k, the series does not
    const double series = k * k * (0.5 + k * (1.0 / 6 + k * (1.0 / 24 + k * (1.0 / 120 + k * (1.0 / 720)))));
    const double e = exp(k) - 1.0;
    const bool small = fabs(k) < 0.02;
    sum[1] += w * (small ? series : e - k);
    if (a.kl_weight != 0.0) g -= a.kl_weight * (small ? k + series : e);  // an infinite e among others
  }
  if (a.entropy) sum[2] += w * (double)x.entropy;
  sum[3] += clipped ? w : 0.0;
  sum[4] += 1.0;
  g_lp = (float)(a.scale * w * g);
  g_entropy = (float)(-a.scale * a.entropy_weight * w);
}
__device__ __forceinline__ void policy_stats(const PolicyArgs& a, const double (&t)[kTerms]) {
  const double loss = t[0] + (a.kl_weight != 0.0 ? a.kl_weight * t[1] : 0.0) - (a.entropy_weight != 0.0 ? a.entropy_weight * t[2] : 0.0);
  a.stats[0] = (float)(a.scale * loss);
#pragma unroll
  for (int i = 0; i < kTerms; ++i) a.stats[1 + i] = (float)t[i];
}
__device__ __forceinline__ void policy_bad(const PolicyArgs& a) {
  for (int i = 0; i < 1 + kTerms; ++i) a.stats[i] = NAN;
  if (a.flags) atomicOr(a.flags, kFlagCapacity);
}

// Sum of every thread's terms, in the first thread.
template <int N> __device__ __forceinline__ void block_sum(double (&t)[kTerms], double (*s_part)[kTerms]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < kTerms; ++i)
#pragma unroll
    for (int d = 32; d; d /= 2) t[i] += __shfl_down(t[i], d);
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < kTerms; ++i) s_part[wave][i] = t[i];
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < N / 64; ++w)
#pragma unroll
      for (int i = 0; i < kTerms; ++i) t[i] += s_part[w][i];
}

// All of it in one workgroup: one launch for a small batch (512 rows: 6.1 us,
// of which the barriers and loads one after the other take most).
__global__ void __launch_bounds__(1024) k_policy_small(PolicyArgs a) {
  __shared__ int s_count[kSmallRows], s_tokens, s_seqs, s_bad;
  __shared__ double s_part[16][kTerms];
  const int tid = threadIdx.x;
  if (tid == 0) s_tokens = s_seqs = s_bad = 0;
  for (int s = tid; s < a.n_seqs; s += 1024) s_count[s] = 0;
  __syncthreads();
  bool bad = false;
  for (int s = tid; s < a.n_seqs; s += 1024) bad |= start_bad(a, s);
  if (bad) s_bad = 1;
  __syncthreads();
  if (s_bad) {
    if (tid == 0) policy_bad(a);
    return;
  }
  const int first = a.n_seqs ? a.row_start[0] : 0, end = a.n_seqs ? a.row_start[a.n_seqs] : 0;
  constexpr int kEach = kSmallRows / 1024;
  int seq[kEach];  // -1: no sequence, -2 - s: sequence s without a token
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int row = tid + i * 1024;
    seq[i] = -1;
    if (row < first || row >= end) continue;
    const int s = seq_of(a.row_start, 0, a.n_seqs, row);
    seq[i] = s;
    if (a.tokens && a.tokens[row] == -1) seq[i] = -2 - s;
    else if (a.mean == 0) atomicAdd(&s_tokens, 1);
    else if (a.mean == 1 && atomicAdd(&s_count[s], 1) == 0) atomicAdd(&s_seqs, 1);
  }
  __syncthreads();
  double t[kTerms] = {0, 0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int row = tid + i * 1024;
    if (seq[i] == -1) continue;
    float g = 0.f, ge = 0.f;
    if (seq[i] >= 0) {
      const double w = a.mean == 0 ? 1.0 / s_tokens : a.mean == 1 ? 1.0 / ((double)s_count[seq[i]] * s_seqs) : 1.0;
      const PolicyRow x = {a.lp[row], a.old[row], a.ref ? a.ref[row] : 0.f, a.entropy ? a.entropy[row] : 0.f,
                           a.adv[a.adv_rows ? row : seq[i]]};
      policy_row(a, x, w, t, g, ge);
    }
    if (a.g_lp) a.g_lp[row] = g;
    if (a.g_entropy) a.g_entropy[row] = ge;
  }
  block_sum<1024>(t, s_part);
  if (tid == 0) policy_stats(a, t);
}

// Four elements of a row array from `row` (a multiple of 4) on; vec: all arrays start on 16-byte boundaries.
template <typename V> __device__ __forceinline__ void load_rows(const V* p, int row, int n_rows, bool vec, V (&v)[4]) {
  if (vec && row + 4 <= n_rows) {
    const uint4 x = *reinterpret_cast<const uint4*>(p + row);
    v[0] = __builtin_bit_cast(V, x.x); v[1] = __builtin_bit_cast(V, x.y);
    v[2] = __builtin_bit_cast(V, x.z); v[3] = __builtin_bit_cast(V, x.w);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = row + i < n_rows ? p[row + i] : V(0);
  }
}
__device__ __forceinline__ void store_rows(float* p, int row, int from, int to, bool vec, const float (&v)[4]) {
  if (vec && row >= from && row + 3 <= to) {
    *reinterpret_cast<float4*>(p + row) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (row + i >= from && row + i <= to) p[row + i] = v[i];
  }
}

__global__ void __launch_bounds__(256) k_policy_clear(PolicyArgs a) {
  const PolicyWs ws = policy_ws(a);
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < a.n_seqs) ws.count[i] = 0;
  if (i == 0) *ws.seqs = 0;
}

// Counts the tokens of every block of rows (the sign bit: row starts that
// cannot be) and, for the mean over sequences, of every sequence.
__global__ void __launch_bounds__(256) k_policy_count(PolicyArgs a) {
  __shared__ int s_n[4];
  const PolicyWs ws = policy_ws(a);
  const int tid = threadIdx.x, lane = tid & 63, row0 = blockIdx.x * kRowsBlock + tid * 4;
  bool bad = false;
  for (int s = blockIdx.x * 256 + tid; s < a.n_seqs; s += gridDim.x * 256) bad |= start_bad(a, s);
  const int first = a.row_start[0], end = a.row_start[a.n_seqs];
  int n = 0, seq = -1, token[4] = {0, 0, 0, 0};
  if (a.tokens) load_rows(a.tokens, row0, a.n_rows, a.vec, token);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = row0 + i;
    if (row >= a.n_rows || row < first || row >= end || token[i] == -1) continue;
    ++n;
    if (a.mean == 1) {
      if (seq < 0) seq = seq_of(a.row_start, 0, a.n_seqs, row);
      while (seq + 1 < a.n_seqs && row >= a.row_start[seq + 1]) ++seq;
      if (__hip_atomic_fetch_add(ws.count + seq, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0)
        __hip_atomic_fetch_add(ws.seqs, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  if (bad) n = INT32_MIN;
#pragma unroll
  for (int d = 32; d; d /= 2) {
    const int o = __shfl_xor(n, d);
    n = ((n | o) & INT32_MIN) | ((n & INT32_MAX) + (o & INT32_MAX));
  }
  if (lane == 0) s_n[tid >> 6] = n;
  __syncthreads();
  if (tid == 0) {
    int sum = 0, sign = 0;
    for (int w = 0; w < 4; ++w) {
      sum += s_n[w] & INT32_MAX;
      sign |= s_n[w] & INT32_MIN;
    }
    ws.block[blockIdx.x] = sum | sign;
  }
}

__global__ void __launch_bounds__(256) k_policy(PolicyArgs a) {
  __shared__ double s_part[4][kTerms];
  __shared__ int s_n[4], s_bad, s_span[2];
  const PolicyWs ws = policy_ws(a);
  const int tid = threadIdx.x, lane = tid & 63, block0 = blockIdx.x * kRowsBlock, row0 = block0 + tid * 4;
  // everything that the rows need is on its way before the first wait
  float lp[4], old[4], ref[4] = {0, 0, 0, 0}, entropy[4] = {0, 0, 0, 0}, adv[4] = {0, 0, 0, 0};
  int token[4] = {0, 0, 0, 0};
  load_rows(a.lp, row0, a.n_rows, a.vec, lp);
  load_rows(a.old, row0, a.n_rows, a.vec, old);
  if (a.tokens) load_rows(a.tokens, row0, a.n_rows, a.vec, token);
  if (a.ref) load_rows(a.ref, row0, a.n_rows, a.vec, ref);
  if (a.entropy) load_rows(a.entropy, row0, a.n_rows, a.vec, entropy);
  if (a.adv_rows) load_rows(a.adv, row0, a.n_rows, a.vec, adv);
  const int first = a.row_start[0], end = a.row_start[a.n_seqs];
  int n = 0, sign = 0;
  for (int i = tid; i < a.blocks; i += 256) {
    n += ws.block[i] & INT32_MAX;
    sign |= ws.block[i];
  }
  if (tid == 0) s_bad = 0;
  __syncthreads();
  if (sign < 0) s_bad = 1;
#pragma unroll
  for (int d = 32; d; d /= 2) n += __shfl_xor(n, d);
  if (lane == 0) s_n[tid >> 6] = n;
  __syncthreads();
  if (s_bad) return;
  const int from = max(block0, first), to = min(block0 + kRowsBlock, end) - 1;
  const bool some = from <= to, need_seq = !a.adv_rows || a.mean == 1;
  if (need_seq) {  // the sequences of the workgroup's first and last row, by two waves at once
    if (some && lane == 0 && tid < 128) s_span[tid >> 6] = seq_of(a.row_start, 0, a.n_seqs, tid ? to : from);
    __syncthreads();
  }
  double t[kTerms] = {0, 0, 0, 0, 0};
  if (some && row0 <= to && row0 + 3 >= from) {
    const double tokens = (double)(s_n[0] + s_n[1] + s_n[2] + s_n[3]), seqs = a.mean == 1 ? (double)*ws.seqs : 0.0;
    double w = a.mean == 0 ? 1.0 / tokens : 1.0;
    int seq = -1;
    float g[4], ge[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = row0 + i;
      g[i] = ge[i] = 0.f;
      if (row < from || row > to || token[i] == -1) continue;
      if (need_seq) {
        const int was = seq;
        if (seq < 0) seq = seq_of(a.row_start, s_span[0], s_span[1] + 1, row);
        while (seq < s_span[1] && row >= a.row_start[seq + 1]) ++seq;
        if (a.mean == 1 && seq != was) w = 1.0 / (ws.count[seq] * seqs);
        if (!a.adv_rows) adv[i] = a.adv[seq];
      }
      policy_row(a, PolicyRow{lp[i], old[i], ref[i], entropy[i], adv[i]}, w, t, g[i], ge[i]);
    }
    if (a.g_lp) store_rows(a.g_lp, row0, from, to, a.vec, g);
    if (a.g_entropy) store_rows(a.g_entropy, row0, from, to, a.vec, ge);
  }
  block_sum<256>(t, s_part);
  if (tid == 0)
#pragma unroll
    for (int i = 0; i < kTerms; ++i) ws.part[(size_t)blockIdx.x * kTerms + i] = t[i];
}

// The workgroups' sums, in order.  A launch of its own: that the workgroup
// which ends last does it needs a release by each of them, which writes its
// L2's changed lines back (960 thousand rows: 49 us for k_policy, 11 without).
__global__ void __launch_bounds__(256) k_policy_stats(PolicyArgs a) {
  __shared__ double s_part[4][kTerms];
  __shared__ int s_bad;
  const PolicyWs ws = policy_ws(a);
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  double t[kTerms] = {0, 0, 0, 0, 0};
  for (int b = threadIdx.x; b < a.blocks; b += 256) {
    if (ws.block[b] < 0) s_bad = 1;
#pragma unroll
    for (int i = 0; i < kTerms; ++i) t[i] += ws.part[(size_t)b * kTerms + i];
  }
  block_sum<256>(t, s_part);
  if (threadIdx.x == 0) {
    if (s_bad) policy_bad(a);
    else policy_stats(a, t);
  }
}

hipError_t launch_policy(PolicyArgs& a, hipStream_t st) {
  a.blocks = policy_blocks(a.n_rows);
  if (a.n_rows <= kSmallRows && a.n_seqs <= kSmallRows) {
    k_policy_small<<<1, 1024, 0, st>>>(a);
    return hipGetLastError();
  }
  if (a.mean == 1) k_policy_clear<<<(unsigned)((a.n_seqs + 255) / 256), 256, 0, st>>>(a);
  k_policy_count<<<(unsigned)a.blocks, 256, 0, st>>>(a);
  k_policy<<<(unsigned)a.blocks, 256, 0, st>>>(a);
  k_policy_stats<<<1, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace jf
