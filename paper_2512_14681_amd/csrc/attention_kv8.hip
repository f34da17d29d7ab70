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
// two to a largest element in [1, 2), and the weights, which are at most 2^15,
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

// Eight values as two fp16 terms, the second one what the first one's
// rounding left.  minus_one (-1, unknown to the compiler) makes that
// difference one instruction with an fp16 operand.
__device__ __forceinline__ void split16(const float* x, float minus_one, f16x8_t& hi, f16x8_t& lo) {
  F16x8 h, l;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h.p[i] = __builtin_convertvector((f32x2_t{x[2 * i], x[2 * i + 1]}), f16x2_t);
    const f32x2_t left = {__builtin_fmaf((float)h.p[i][0], minus_one, x[2 * i]),
                          __builtin_fmaf((float)h.p[i][1], minus_one, x[2 * i + 1])};
    l.p[i] = __builtin_convertvector(left, f16x2_t);
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

// Maximum over the four lanes that share a query (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float query_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t x = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Weights are 2^kWeightBits e^(s - m), and m follows a row's maximum only
// when that has grown by more than 2^kSlack: most pages leave the sums and
// outputs as they are.
constexpr float kWeightBits = 12.f, kSlack = 3.f;
constexpr int kWaves = 4;

// QT tiles of 16 queries of one KV head in a wave.  Query j of the head group
// is row j / grp, head j % grp of the group, so that a tile's queries have
// neighbouring rows.  Lane l holds query l % 16; of a page's scores it has
// keys 16 t + 4 kg + i (kg = l / 16), of the outputs dims 16 n + 4 kg + i.
template <typename A, int HD, int QT> struct Tiles {
  static constexpr int NS = HD / 32;  // matrix steps along the head
  static constexpr int NP = HD / 16;  // 1 KB pieces of a page's keys (and values)
  f16x8_t qh[QT][NS], qlo[QT][NS];
  float cq[QT];                       // score units: 2^(row's exponent) log2(e) / sqrt(hd)
  int qi[QT], qhd[QT];
  bool valid[QT];
  float m[QT], l[QT];
  f32x4_t o[QT][NP];                  // in the units of the value scale `unit`
  float unit, minus_one;

  __device__ __forceinline__ void init(const Kv8Args& a, const Seq& q, int g, int tile0) {
    const int grp = a.H / a.G, nq = grp * q.n, lane = threadIdx.x & 63, ql = lane & 15, kg = lane >> 4;
    unit = 0.f;
    minus_one = -1.f;
    asm("" : "+s"(minus_one));
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
      amax = query_max(amax);
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
        split16(v[c], minus_one, qh[t][c], qlo[t][c]);
      }
      m[t] = -INFINITY;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < NP; ++d) o[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Scores of a page; kf(kt, c): its keys 16 kt .., dims of matrix step c.
  template <typename F> __device__ __forceinline__ void scores(F kf, f32x4_t (&st)[QT][4]) const {
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
      for (int t = 0; t < QT; ++t) st[t][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NS; ++c) {
        const f16x8_t k = kf(kt, c);
#pragma unroll
        for (int t = 0; t < QT; ++t) mfma16(st[t][kt], k, qh[t][c]);
#pragma unroll
        for (int t = 0; t < QT; ++t) mfma16(st[t][kt], k, qlo[t][c]);
      }
    }
  }

  // The slots of page p that tile t's queries see, this lane's keys at bits 16 t' + i.
  __device__ __forceinline__ uint64_t seen(const Kv8Args& a, const Seq& q, int t, int p) const {
    return seen_bits(a.vis ? a.vis + (size_t)(q.r0 + qi[t]) * kVisWords : nullptr, qi[t], q.n, p * kPage - q.C) >>
           (4 * ((threadIdx.x & 63) >> 4));
  }

  // -inf for the slots of page p that a query does not see.
  __device__ __forceinline__ void mask(const Kv8Args& a, const Seq& q, int p, f32x4_t (&st)[QT][4]) const {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const uint64_t sees = seen(a, q, t, p);
      const uint32_t half[2] = {(uint32_t)sees, (uint32_t)(sees >> 32)};
#pragma unroll
      for (int e = 0; e < 16; ++e)
        st[t][e >> 2][e & 3] = (half[e >> 3] >> (16 * ((e >> 2) & 1) + (e & 3))) & 1 ? st[t][e >> 2][e & 3] : -INFINITY;
    }
  }

  // Scores to weights; key_scale: the page's.
  __device__ __forceinline__ void softmax(const f32x4_t (&st)[QT][4], float key_scale, f16x8_t (&ph)[QT][2],
                                          f16x8_t (&pl)[QT][2]) {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float x[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = st[t][e >> 2][e & 3];
      const float f = cq[t] * key_scale;
      float mx = x[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
      mx = query_max(mx) * f;
      if (__any(mx > m[t] + kSlack)) {
        const float m_new = fmaxf(m[t], mx);
        const float alpha = __builtin_amdgcn_exp2f(m[t] - (m_new == -INFINITY ? 0.f : m_new));
        l[t] *= alpha;
        m[t] = m_new;
#pragma unroll
        for (int d = 0; d < NP; ++d) o[t][d] *= alpha;
      }
      // nothing visible yet: weights 0
      const float off = kWeightBits - (m[t] == -INFINITY ? 0.f : m[t]);
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], f, off));
        sum += x[e];
      }
      l[t] += sum;
      split16(x, minus_one, ph[t][0], pl[t][0]);
      split16(x + 8, minus_one, ph[t][1], pl[t][1]);
    }
  }

  // A page's value scale: the outputs' unit becomes the larger of the two.
  __device__ __forceinline__ float value_scale(float s) {
    if (s > unit) {
      const float f = unit / s;
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int d = 0; d < NP; ++d) o[t][d] *= f;
      unit = s;
    }
    return s / unit;
  }

  // Weighted values; vf(n, j): the page's dims 16 n .., keys of tiles 2 j and 2 j + 1.
  template <typename F>
  __device__ __forceinline__ void outputs(F vf, const f16x8_t (&ph)[QT][2], const f16x8_t (&pl)[QT][2]) {
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f16x8_t v = vf(n, j);
#pragma unroll
        for (int t = 0; t < QT; ++t) mfma16(o[t][n], v, ph[t][j]);
#pragma unroll
        for (int t = 0; t < QT; ++t) mfma16(o[t][n], v, pl[t][j]);
      }
  }

  // NaN for the queries that see a NaN among the values that ones(n) marks
  // with the code of 1.
  template <typename F>
  __device__ __forceinline__ void poison(const Kv8Args& a, const Seq& q, int p, F ones) {
    uint64_t sees[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) sees[t] = seen(a, q, t, p);
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const u32x4_t w = ones(n);
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        f32x4_t hit = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          f16x8_t b;
#pragma unroll
          for (int e = 0; e < 8; ++e) b[e] = (sees[t] >> (16 * (2 * j + (e >> 2)) + (e & 3))) & 1 ? 1.f : 0.f;
          mfma16(hit, f8_to_f16(w[2 * j], w[2 * j + 1], 1.f), b);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (hit[i] > 0.f) o[t][n][i] = NAN;
      }
    }
  }

  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      l[t] += __shfl_xor(l[t], 16);
      l[t] += __shfl_xor(l[t], 32);
    }
  }
};

// A value page's NaN codes as codes of 1, and the codes without them.
__device__ __forceinline__ u32x4_t nan_ones(const u32x4_t& w) {
  u32x4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (f8_nans(w[i]) >> 7) * 0x38u;
  return r;
}
__device__ __forceinline__ u32x4_t without_nans(const u32x4_t& w) {
  u32x4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = w[i] & ~((f8_nans(w[i]) >> 7) * 0xFFu);
  return r;
}
__device__ __forceinline__ bool has_nans(const u32x4_t& w) {
  return (f8_nans(w[0]) | f8_nans(w[1]) | f8_nans(w[2]) | f8_nans(w[3])) != 0;
}

// A query's maximum, sum and 4 of its outputs: the result, or the split's partial one.
template <typename A>
__device__ __forceinline__ void put_outputs(const Kv8Args& a, int row, int head, int split, int dim, float m, float l,
                                            float (&v)[4]) {
  if (a.splits == 1) {
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = inv == 0.f ? 0.f : v[i] * inv;
    act_store4(reinterpret_cast<A*>(a.out) + act_offset(row, head * a.hd + dim, a.H * a.hd), a.out_plane, v);
  } else {
    const size_t at = ((size_t)split * a.b.n_rows + row) * a.H + head;
    *reinterpret_cast<float4*>(a.o_part + at * a.hd + dim) = make_float4(v[0], v[1], v[2], v[3]);
    if (dim == 0) *reinterpret_cast<float2*>(a.ml_part + at * 2) = make_float2(m, l);
  }
}

template <bool ONCE> __device__ __forceinline__ u32x4_t load16(const uint8_t* p) {
  const auto* q = reinterpret_cast<const u32x4_t*>(p);
  return ONCE ? __builtin_nontemporal_load(q) : *q;
}

// One query tile (few rows: bound by the cache's bytes).  Workgroup: KV head,
// tile, key split; the waves take every fourth page straight into registers,
// the next page's keys in flight from when this one's scores are done, and
// merge in LDS.
template <typename A, int HD>
__global__ void __launch_bounds__(256, 2) k_attention_kv8_few(Kv8Args a) {
  using T = Tiles<A, HD, 1>;
  constexpr int NP = T::NP;
  __shared__ float s_o[kWaves][16][HD + 4], s_m[kWaves][16], s_l[kWaves][16];
  const int s = blockIdx.x / a.G, g = blockIdx.x % a.G, split = blockIdx.y;
  Seq q;
  if (!batch_seq(a.b, s, q)) return;
  const int pages = (q.C + q.n + kPage - 1) / kPage;
  const int p0 = split * a.chunk, p1 = min(p0 + a.chunk, pages);
  if (p0 >= pages) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, ql = lane & 15, kg = lane >> 4;
  T w;

  int id = -1;
  u32x4_t kr[NP], vr[NP];
  float2 sc;
  const uint8_t* page = nullptr;
  auto find = [&](int p) {  // the wave's first valid page from p on
    id = -1;
    for (; p < p1; p += kWaves)
      if ((id = __builtin_amdgcn_readfirstlane(batch_page(a.b, q, p))) >= 0) break;
    return p;
  };
  auto load_keys = [&] {
    page = a.kv + (size_t)id * a.page_bytes;
#pragma unroll
    for (int n = 0; n < NP; ++n) kr[n] = load16<true>(page + (size_t)g * kPage * HD + n * 1024 + lane * 16);
    sc = reinterpret_cast<const float2*>(page + (size_t)2 * a.G * kPage * HD)[g];
  };
  int p = find(p0 + wave);
  if (p < p1) load_keys();
  w.init(a, q, g, 0);
  while (p < p1) {
#pragma unroll
    for (int n = 0; n < NP; ++n) vr[n] = load16<true>(page + (size_t)(a.G + g) * kPage * HD + n * 1024 + lane * 16);
    f32x4_t st[1][4];
    w.scores([&](int kt, int c) {
      const int i = kt * (HD / 16) + 2 * c;
      return f8_to_f16(kr[i >> 2][i & 3], kr[i >> 2][(i & 3) + 1], 1.f);
    }, st);
    const int now = p;
    const float2 scale = sc;
    p = find(p + kWaves);
    if (p < p1) load_keys();
    const float vscale = w.value_scale(scale.y);
    f16x8_t ph[1][2], pl[1][2];
    const bool edge = (now + 1) * kPage > q.C;  // holds slots that not every row sees
    if (edge) w.mask(a, q, now, st);
    w.softmax(st, scale.x, ph, pl);
    if (edge) {
      // 0 times NaN is NaN: NaN codes are taken out, and the rows that see one get it back
      bool any = false;
#pragma unroll
      for (int n = 0; n < NP; ++n) any |= has_nans(vr[n]);
      if (__any(any)) {
        w.poison(a, q, now, [&](int n) { return nan_ones(vr[n]); });
#pragma unroll
        for (int n = 0; n < NP; ++n) vr[n] = without_nans(vr[n]);
      }
    }
    w.outputs([&](int n, int j) { return f8_to_f16(vr[n][2 * j], vr[n][2 * j + 1], vscale); }, ph, pl);
  }
  w.finish();

#pragma unroll
  for (int n = 0; n < NP; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s_o[wave][ql][16 * n + 4 * kg + i] = w.o[0][n][i] * w.unit;
  if (kg == 0) {
    s_m[wave][ql] = w.m[0];
    s_l[wave][ql] = w.l[0];
  }
  __syncthreads();
  // wave w merges pieces w, w + 4, ...; its lanes keep their query
  float m = -INFINITY, l = 0.f, f[kWaves];
#pragma unroll
  for (int i = 0; i < kWaves; ++i) m = fmaxf(m, s_m[i][ql]);
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    f[i] = s_m[i][ql] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[i][ql] - m);
    l += s_l[i][ql] * f[i];
  }
  if (w.valid[0])
    for (int n = wave; n < NP; n += kWaves) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kWaves; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += f[i] * s_o[i][ql][16 * n + 4 * kg + e];
      put_outputs<A>(a, q.r0 + w.qi[0], w.qhd[0], split, 16 * n + 4 * kg, m, l, v);
    }
}

// More tiles: QT of its own for each wave.  Workgroup: KV head, 4 QT tiles,
// key split.  A page is turned to fp16 once for all of them, on its way into
// one of two LDS buffers: the next page's loads are in flight during a page's
// work, and one barrier separates two pages.
template <typename A, int HD, int QT>
__global__ void __launch_bounds__(256, 2) k_attention_kv8_many(Kv8Args a) {
  using T = Tiles<A, HD, QT>;
  constexpr int NS = T::NS, NP = T::NP;
  constexpr int kItems = 2 * NP / kWaves;      // 16-byte pieces of a page for each thread
  __shared__ f16x8_t s_kv[2][4 * NP][64];      // operands: keys kt NS + c, then values 2 NP + 2 n + j
  __shared__ int s_nan[2];                     // page + 1 whose values hold a NaN that not every row sees
  const int grp = a.H / a.G;
  const int s = blockIdx.x / (a.G * a.groups), g = blockIdx.x / a.groups % a.G, group = blockIdx.x % a.groups;
  const int split = blockIdx.y;
  Seq q;
  if (!batch_seq(a.b, s, q)) return;
  const int nq = grp * q.n;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, kg = lane >> 4;
  if (group * kWaves * QT * 16 >= nq) return;
  const int pages = (q.C + q.n + kPage - 1) / kPage;
  const int p0 = split * a.chunk;
  int p1 = min(p0 + a.chunk, pages);
  if (p0 >= pages) return;
  const int tile0 = (group * kWaves + wave) * QT;
  int mine = tile0 * 16 < nq ? p1 : p0;        // the wave's tiles need pages [p0, mine)
  if (!a.vis) {                                // causal: no slot past the last row
    const int last_wave = min((tile0 + QT) * 16, nq) - 1, last = min((group + 1) * kWaves * QT * 16, nq) - 1;
    mine = min(mine, (q.C + last_wave / grp) / kPage + 1);
    p1 = min(p1, (q.C + last / grp) / kPage + 1);
  }
  if (threadIdx.x < 2) s_nan[threadIdx.x] = 0;
  T w;
  w.init(a, q, g, tile0);

  u32x4_t raw[kItems];
  float2 sc = {0.f, 0.f};
  const uint8_t* page = nullptr;
  auto load = [&](int p) {  // the first valid page from p on
    int id = -1;
    for (; p < p1; ++p)
      if ((id = __builtin_amdgcn_readfirstlane(batch_page(a.b, q, p))) >= 0) break;
    if (id >= 0) {
      page = a.kv + (size_t)id * a.page_bytes;
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        const int piece = i * kWaves + wave;   // keys 0 .. NP - 1, then values
        raw[i] = load16<false>(page + (size_t)(piece < NP ? g : a.G + g) * kPage * HD + (piece % NP) * 1024 + lane * 16);
      }
      sc = reinterpret_cast<const float2*>(page + (size_t)2 * a.G * kPage * HD)[g];
    }
    return p;
  };
  auto store = [&](int buf, int p, float vscale) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int piece = i * kWaves + wave;
      if (piece >= NP && (p + 1) * kPage > q.C && __any(has_nans(raw[i]))) {
        raw[i] = without_nans(raw[i]);
        s_nan[buf] = p + 1;
      }
      const float f = piece < NP ? 1.f : vscale;
      s_kv[buf][2 * piece][lane] = f8_to_f16(raw[i][0], raw[i][1], f);
      s_kv[buf][2 * piece + 1][lane] = f8_to_f16(raw[i][2], raw[i][3], f);
    }
  };
  __syncthreads();  // s_nan
  int p = load(p0), buf = 0;
  float vscale = 0.f, key_scale = 0.f;
  const uint8_t* base = nullptr;
  if (p < p1) {
    vscale = w.value_scale(sc.y);
    key_scale = sc.x;
    base = page;
    store(0, p, vscale);
  }
  __syncthreads();
  while (p < p1) {
    const int next = load(p + 1);
    if (p < mine) {
      f32x4_t st[QT][4];
      w.scores([&](int kt, int c) { return s_kv[buf][kt * NS + c][lane]; }, st);
      f16x8_t ph[QT][2], pl[QT][2];
      if ((p + 1) * kPage > q.C) w.mask(a, q, p, st);
      w.softmax(st, key_scale, ph, pl);
      if (s_nan[buf] == p + 1)
        w.poison(a, q, p, [&](int n) {
          return nan_ones(load16<false>(base + (size_t)(a.G + g) * kPage * HD + n * 1024 + lane * 16));
        });
      w.outputs([&](int n, int j) { return s_kv[buf][2 * NP + 2 * n + j][lane]; }, ph, pl);
    }
    if (next < p1) {
      vscale = w.value_scale(sc.y);
      key_scale = sc.x;
      base = page;
      store(buf ^ 1, next, vscale);
    }
    __syncthreads();
    p = next;
    buf ^= 1;
  }
  w.finish();
#pragma unroll
  for (int t = 0; t < QT; ++t)
    if (w.valid[t])
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        float v[4] = {w.o[t][n][0] * w.unit, w.o[t][n][1] * w.unit, w.o[t][n][2] * w.unit, w.o[t][n][3] * w.unit};
        put_outputs<A>(a, q.r0 + w.qi[t], w.qhd[t], split, 16 * n + 4 * kg, w.m[t], w.l[t], v);
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

#ifndef WB_FEW
#define WB_FEW 1024
#define WB_MANY 512
#define CH_FEW 4
#define CH_MANY 4
#endif
void kv8_plan(Kv8Args& a) {
  const int tiles = (int)(((int64_t)a.H / a.G * a.b.max_rows + 15) / 16);
  a.qt = tiles == 1 ? 0 : tiles <= kWaves ? 1 : 2;
  a.groups = a.qt == 0 ? 1 : (tiles + kWaves * a.qt - 1) / (kWaves * a.qt);
  const int pages = (a.b.max_ctx + kPage - 1) / kPage;
  const int64_t base = (int64_t)a.b.n_seqs * a.G * a.groups;
  const int wb = a.qt == 0 ? WB_FEW : WB_MANY, ch = a.qt == 0 ? CH_FEW : CH_MANY;
  const int64_t want = std::min<int64_t>(std::max<int64_t>((wb + base - 1) / base, 1), kMaxSplits);
  a.chunk = std::max<int>((int)((pages + want - 1) / want), ch);
  if (a.qt == 0) a.chunk = (a.chunk + kWaves - 1) / kWaves * kWaves;
  a.splits = (pages + a.chunk - 1) / a.chunk;
}

template <typename A, int HD>
static void attention_qt(const Kv8Args& a, dim3 grid, hipStream_t st) {
  if (a.qt == 0) k_attention_kv8_few<A, HD><<<grid, 256, 0, st>>>(a);
  else if (a.qt == 1) k_attention_kv8_many<A, HD, 1><<<grid, 256, 0, st>>>(a);
  else k_attention_kv8_many<A, HD, 2><<<grid, 256, 0, st>>>(a);
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
