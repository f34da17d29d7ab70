// Grouped-query attention of a batch of sequences over an e4m3 paged cache
// (jf_attention_kv8): row i of a sequence sees its committed slots and the
// in-step slots that its mask marks.
//
// A page's 64 keys are four 16-row operands of S^T = K Q^T.  A lane then holds
// the scores of one query for keys 16 t + 4 kg + i (t, i < 4; kg = lane / 16),
// the page keeps a lane's value bytes in that same order, and so the softmax
// weights go on to O^T += V^T P^T without leaving their lanes.  One pass over
// the pages with a running maximum and sum, both in fp32.
//
// Precision: e4m3 codes are exact in fp16.  A row of Q, scaled by a power of
// two to a largest element in [1, 2), and the weights, which are at most 2^14,
// enter the matrix cores as two fp16 terms each, which hold 22 bits.  The
// values' scales are applied relative to the largest one met so far; a page's
// codes lose bits by that only 2^11 and more below it.
#include <algorithm>

#include "jf_batch.h"

namespace jf {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void mfma16(f32x4_t& acc, const f16x8_t& a, const f16x8_t& b) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, acc, 0, 0, 0);
}

union F16x8 {
  f16x8_t v;
  f16x2_t p[4];
  uint32_t w[4];
};

// Eight codes times a power of two.
__device__ __forceinline__ f16x8_t f8_to_f16(uint32_t lo, uint32_t hi, float scale) {
  F16x8 r;
  r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false);
  r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
  r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false);
  r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
  return r.v;
}

// Eight values as two fp16 terms.  Both are rounded towards zero (one
// instruction for two): the second holds what the first leaves, so 21 bits
// or more are kept.
__device__ __forceinline__ void split16(const float* x, f16x8_t& hi, f16x8_t& lo) {
  F16x8 h, l;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h.p[i] = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_cvt_pkrtz(x[2 * i], x[2 * i + 1]));
    l.p[i] = __builtin_bit_cast(
        f16x2_t, __builtin_amdgcn_cvt_pkrtz(__builtin_fmaf((float)h.p[i][0], -1.f, x[2 * i]),
                                            __builtin_fmaf((float)h.p[i][1], -1.f, x[2 * i + 1])));
  }
  hi = h.v;
  lo = l.v;
}

// Low n bits, n clamped to [0, 64].
__device__ __forceinline__ uint64_t low_bits(int n) { return n >= 64 ? ~0ull : (n <= 0 ? 0ull : (1ull << n) - 1); }

// Bits j0 .. j0 + 63 of what a row sees (j0 > -64): slots before the in-step
// ones, then those of its mask (causal for vis null), none past the
// sequence's n rows.
__device__ __forceinline__ uint64_t seen_bits(const uint64_t* vis, int i, int n, int j0) {
  uint64_t w;
  if (vis) {
    const int k = j0 >> 6, sh = j0 & 63;  // floor: k = -1 for a window that starts before the in-step slots
    const uint64_t a = k >= 0 && k < kVisWords ? vis[k] : 0, b = k + 1 < kVisWords ? vis[k + 1] : 0;
    w = sh ? (a >> sh) | (b << (64 - sh)) : a;
    w &= low_bits(n - j0);
  } else {
    w = low_bits(min(i + 1, n) - j0);
  }
  return w | low_bits(-j0);
}

// NaN codes of four bytes, as 0x80 in each.
__device__ __forceinline__ uint32_t f8_nans(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

template <typename A> __device__ __forceinline__ void load_q8(const A* p, size_t plane, float (&v)[8]);
template <> __device__ __forceinline__ void load_q8<bf16_t>(const bf16_t* p, size_t plane, float (&v)[8]) {
  const uint4 h = *reinterpret_cast<const uint4*>(p), l = *reinterpret_cast<const uint4*>(p + plane);
  const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(hw[i] << 16) + __uint_as_float(lw[i] << 16);
    v[2 * i + 1] = __uint_as_float(hw[i] & 0xFFFF0000u) + __uint_as_float(lw[i] & 0xFFFF0000u);
  }
}
template <> __device__ __forceinline__ void load_q8<float>(const float* p, size_t, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

constexpr float kWeightBits = 14.f;  // weights are 2^14 e^(s - m)
constexpr int kWaves = 4;

// Workgroup: KV head, up to QT (kShare: 4 QT) query tiles, one key split.
// kShare: every wave has QT tiles of its own and all the split's pages; else
// the waves share QT tiles and take every fourth page, and merge in LDS.
// Query j of a head group is row j / grp, head j % grp of the group, so a
// tile's queries have neighbouring rows.
template <typename A, int HD, int QT, bool kShare>
__global__ void __launch_bounds__(256, 2) k_attention_kv8(Kv8Args a) {
  constexpr int NS = HD / 32;  // matrix steps along the head
  constexpr int NP = HD / 16;  // 1 KB pieces of a page's keys (and values)
  const int grp = a.H / a.G;
  const int s = blockIdx.x / (a.G * a.groups), g = blockIdx.x / a.groups % a.G, group = blockIdx.x % a.groups;
  const int split = blockIdx.y;
  Seq q;
  if (!batch_seq(a.b, s, q)) return;
  const int nq = grp * q.n;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int ql = lane & 15, kg = lane >> 4;
  const int tile0 = kShare ? (group * kWaves + wave) * QT : group * QT;
  if (tile0 * 16 >= nq) return;  // kShare: this wave only, which shares nothing with the others
  const int pages = (q.C + q.n + kPage - 1) / kPage;
  const int p0 = split * a.chunk;
  int p1 = min(p0 + a.chunk, pages);
  if (p0 >= pages) return;

  f16x8_t qh[QT][NS], qlo[QT][NS];
  float cq[QT];       // score units: 2^(row's exponent) log2(e) / sqrt(hd)
  int qi[QT], qhd[QT];
  bool valid[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int j = (tile0 + t) * 16 + ql;
    valid[t] = j < nq;
    qi[t] = valid[t] ? j / grp : 0;
    qhd[t] = g * grp + (valid[t] ? j - qi[t] * grp : 0);
    float v[NS][8], amax = 0.f;
    const A* p = reinterpret_cast<const A*>(a.q) + ((size_t)(q.r0 + qi[t]) * a.H + qhd[t]) * HD + kg * (HD / 4);
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      load_q8<A>(p + 8 * c, a.q_plane, v[c]);
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(v[c][e]));
    }
    amax = fmaxf(amax, __shfl_xor(amax, 16));
    amax = fmaxf(amax, __shfl_xor(amax, 32));
    // an infinite row stays as it is (and its output becomes NaN)
    int ex = 0;
    if (amax > 0.f && amax < INFINITY) {
      (void)frexpf(amax, &ex);
      ex = max(ex - 1, -100);
    }
    const float down = ldexpf(1.f, -ex);
    cq[t] = ldexpf(1.4426950408889634f / sqrtf((float)HD), ex);
#pragma unroll
    for (int c = 0; c < NS; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] *= down;
      split16(v[c], qh[t][c], qlo[t][c]);
    }
  }
  if (kShare && !a.vis) {  // causal: no slot past the wave's last row
    const int last = min((tile0 + QT) * 16, nq) - 1;
    p1 = min(p1, (q.C + last / grp) / kPage + 1);
  }

  float m_run[QT], l_run[QT];
  f32x4_t o[QT][NP];
  float unit = 0.f;  // the largest value scale so far: o holds sums in it
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m_run[t] = -INFINITY;
    l_run[t] = 0.f;
#pragma unroll
    for (int d = 0; d < NP; ++d) o[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  for (int p = p0 + (kShare ? 0 : wave); p < p1; p += kShare ? 1 : kWaves) {
    const int id = __builtin_amdgcn_readfirstlane(batch_page(a.b, q, p));
    if (id < 0) continue;
    const uint8_t* page = a.kv + (size_t)id * a.page_bytes;
    u32x4_t kr[NP], vr[NP];
#pragma unroll
    for (int n = 0; n < NP; ++n)
      kr[n] = *reinterpret_cast<const u32x4_t*>(page + (size_t)g * kPage * HD + n * 1024 + lane * 16);
#pragma unroll
    for (int n = 0; n < NP; ++n)
      vr[n] = *reinterpret_cast<const u32x4_t*>(page + (size_t)(a.G + g) * kPage * HD + n * 1024 + lane * 16);
    const float2 sc = reinterpret_cast<const float2*>(page + (size_t)2 * a.G * kPage * HD)[g];
    const bool edge = (p + 1) * kPage > q.C;  // holds slots that not every row sees

    f32x4_t st[QT][4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
      for (int t = 0; t < QT; ++t) st[t][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NS; ++c) {
        const int w = kt * (HD / 16) + 2 * c;
        const f16x8_t kf = f8_to_f16(kr[w >> 2][w & 3], kr[w >> 2][(w & 3) + 1], 1.f);
#pragma unroll
        for (int t = 0; t < QT; ++t) mfma16(st[t][kt], kf, qh[t][c]);
#pragma unroll
        for (int t = 0; t < QT; ++t) mfma16(st[t][kt], kf, qlo[t][c]);
      }
    }
    // values relative to the largest scale so far
    if (sc.y > unit) {
      const float f = unit / sc.y;
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int d = 0; d < NP; ++d) o[t][d] *= f;
      unit = sc.y;
    }
    const float vscale = sc.y / unit;

    f16x8_t ph[QT][2], pl[QT][2];
    uint64_t seen[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float x[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = st[t][e >> 2][e & 3];
      if (edge) {
        seen[t] = seen_bits(a.vis ? a.vis + (size_t)(q.r0 + qi[t]) * kVisWords : nullptr, qi[t], q.n,
                            p * kPage - q.C) >> (4 * kg);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = (seen[t] >> (16 * (e >> 2) + (e & 3))) & 1 ? x[e] : -INFINITY;
      }
      const float f = cq[t] * sc.x;
      float mx = x[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m_run[t], mx * f);
      // nothing visible yet: weights 0 and m = -inf
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run[t] - m_use);
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], f, kWeightBits - m_use));
        sum += x[e];
      }
      l_run[t] = l_run[t] * alpha + sum;
      m_run[t] = m_new;
#pragma unroll
      for (int d = 0; d < NP; ++d) o[t][d] *= alpha;
      split16(x, ph[t][0], pl[t][0]);
      split16(x + 8, ph[t][1], pl[t][1]);
    }

    if (edge) {
      // A slot that a row does not see must not reach it, and 0 times NaN is
      // NaN: NaN codes are taken out, and the rows that do see one get it back.
      uint32_t any = 0;
#pragma unroll
      for (int n = 0; n < NP; ++n) any |= f8_nans(vr[n][0]) | f8_nans(vr[n][1]) | f8_nans(vr[n][2]) | f8_nans(vr[n][3]);
      if (__any(any != 0)) {
#pragma unroll
        for (int n = 0; n < NP; ++n) {
          uint32_t one[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t nan = f8_nans(vr[n][i]) >> 7;   // 1 in each such byte
            vr[n][i] &= ~(nan * 0xFFu);
            one[i] = nan * 0x38u;                      // code of 1.0
          }
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            f32x4_t hit = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              f16x8_t b;
#pragma unroll
              for (int e = 0; e < 8; ++e) b[e] = (seen[t] >> (16 * (2 * j + (e >> 2)) + (e & 3))) & 1 ? 1.f : 0.f;
              mfma16(hit, f8_to_f16(one[2 * j], one[2 * j + 1], 1.f), b);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (hit[i] > 0.f) o[t][n][i] = NAN;
          }
        }
      }
    }

#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f16x8_t vf = f8_to_f16(vr[n][2 * j], vr[n][2 * j + 1], vscale);
#pragma unroll
        for (int t = 0; t < QT; ++t) mfma16(o[t][n], vf, ph[t][j]);
#pragma unroll
        for (int t = 0; t < QT; ++t) mfma16(o[t][n], vf, pl[t][j]);
      }
  }

#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l_run[t] += __shfl_xor(l_run[t], 16);
    l_run[t] += __shfl_xor(l_run[t], 32);
  }

  // a query's maximum, sum and 4 of its outputs: the result, or the split's partial one
  auto put = [&](int t, int dim, float m, float l, float (&v)[4]) {
    const int row = q.r0 + qi[t];
    if (a.splits == 1) {
      const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = inv == 0.f ? 0.f : v[i] * inv;
      act_store4(reinterpret_cast<A*>(a.out) + act_offset(row, qhd[t] * HD + dim, a.H * HD), a.out_plane, v);
    } else {
      const size_t at = ((size_t)split * a.b.n_rows + row) * a.H + qhd[t];
      *reinterpret_cast<float4*>(a.o_part + at * HD + dim) = make_float4(v[0], v[1], v[2], v[3]);
      if (dim == 0) *reinterpret_cast<float2*>(a.ml_part + at * 2) = make_float2(m, l);
    }
  };
  if constexpr (kShare) {
#pragma unroll
    for (int t = 0; t < QT; ++t)
      if (valid[t])
#pragma unroll
        for (int n = 0; n < NP; ++n) {
          float v[4] = {o[t][n][0] * unit, o[t][n][1] * unit, o[t][n][2] * unit, o[t][n][3] * unit};
          put(t, 16 * n + 4 * kg, m_run[t], l_run[t], v);
        }
  } else {
    __shared__ float s_o[kWaves][16][HD + 4], s_m[kWaves][16], s_l[kWaves][16];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (t) __syncthreads();
#pragma unroll
      for (int n = 0; n < NP; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s_o[wave][ql][16 * n + 4 * kg + i] = o[t][n][i] * unit;
      if (kg == 0) {
        s_m[wave][ql] = m_run[t];
        s_l[wave][ql] = l_run[t];
      }
      __syncthreads();
      // wave w merges dims of pieces w, w + 4, ...; its lanes keep their query
      float m = -INFINITY, l = 0.f, f[kWaves];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_m[w][ql]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        f[w] = s_m[w][ql] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][ql] - m);
        l += s_l[w][ql] * f[w];
      }
      if (valid[t])
        for (int n = wave; n < NP; n += kWaves) {
          float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < kWaves; ++w)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += f[w] * s_o[w][ql][16 * n + 4 * kg + i];
          put(t, 16 * n + 4 * kg, m, l, v);
        }
    }
  }
}

// Merges the key splits of a sequence, four dims of one row and head a
// thread, in split order.
template <typename A>
__global__ void __launch_bounds__(256) k_attention_kv8_merge(Kv8Args a, int blocks) {
  const int s = blockIdx.x / blocks;
  Seq q;
  if (!batch_seq(a.b, s, q)) return;
  const int chunks = a.hd / 4;
  const int item = blockIdx.x % blocks * 256 + threadIdx.x;
  const int dim = item % chunks * 4, h = item / chunks % a.H, i = item / chunks / a.H;
  if (i >= q.n) return;
  const int row = q.r0 + i;
  const int n = ((q.C + q.n + kPage - 1) / kPage + a.chunk - 1) / a.chunk;
  const size_t stride = (size_t)a.b.n_rows * a.H, at = (size_t)row * a.H + h;
  float m = -INFINITY;
  for (int k = 0; k < n; ++k) m = fmaxf(m, a.ml_part[(k * stride + at) * 2]);
  float l = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < n; ++k) {
    const float2 ml = *reinterpret_cast<const float2*>(a.ml_part + (k * stride + at) * 2);
    const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
    const float4 o = *reinterpret_cast<const float4*>(a.o_part + (k * stride + at) * a.hd + dim);
    l += ml.y * f;
    v[0] += o.x * f; v[1] += o.y * f; v[2] += o.z * f; v[3] += o.w * f;
  }
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = inv == 0.f ? 0.f : v[e] * inv;
  act_store4(reinterpret_cast<A*>(a.out) + act_offset(row, h * a.hd + dim, a.H * a.hd), a.out_plane, v);
}

// ---- launch --------------------------------------------------------------------------
constexpr int kMaxSplits = 64;

void kv8_plan(Kv8Args& a) {
  const int tiles = (int)(((int64_t)a.H / a.G * a.b.max_rows + 15) / 16);
  a.share = tiles > 4;
  a.qt = tiles > 1 && a.hd < 128 ? 2 : 1;  // two tiles of head_dim 128 do not fit the registers
  const int per = a.qt * (a.share ? kWaves : 1);
  a.groups = (tiles + per - 1) / per;
  const int pages = (a.b.max_ctx + kPage - 1) / kPage;
  const int64_t base = (int64_t)a.b.n_seqs * a.G * a.groups;
  // about four workgroups a compute unit, each with four pages or more
  const int64_t want = std::min<int64_t>(std::max<int64_t>((1024 + base - 1) / base, 1), kMaxSplits);
  a.chunk = std::max<int>((int)((pages + want - 1) / want), 4);
  a.chunk = (a.chunk + 3) / 4 * 4;
  a.splits = (pages + a.chunk - 1) / a.chunk;
}

template <typename A, int HD>
static void attention_qt(const Kv8Args& a, dim3 grid, hipStream_t st) {
  constexpr int kMore = HD == 128 ? 1 : 2;
  if (a.share) k_attention_kv8<A, HD, kMore, true><<<grid, 256, 0, st>>>(a);
  else if (a.qt == kMore) k_attention_kv8<A, HD, kMore, false><<<grid, 256, 0, st>>>(a);
  else k_attention_kv8<A, HD, 1, false><<<grid, 256, 0, st>>>(a);
}
template <typename A> static hipError_t attention_act(const Kv8Args& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.b.n_seqs * a.G * a.groups), (unsigned)a.splits);
  if (a.hd == 32) attention_qt<A, 32>(a, grid, st);
  else if (a.hd == 64) attention_qt<A, 64>(a, grid, st);
  else attention_qt<A, 128>(a, grid, st);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int blocks = (a.b.max_rows * a.H * (a.hd / 4) + 255) / 256;
  k_attention_kv8_merge<A><<<(unsigned)(a.b.n_seqs * blocks), 256, 0, st>>>(a, blocks);
  return hipGetLastError();
}
hipError_t launch_attention_kv8(int act, const Kv8Args& a, hipStream_t st) {
  return act == 0 ? attention_act<float>(a, st) : attention_act<bf16_t>(a, st);
}

}  // namespace jf
