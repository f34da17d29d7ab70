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
// values' scales are applied to the codes, relative to a unit that follows the
// scales where fp16 would not hold the codes exactly: no page's scale costs
// another page's codes bits, whoever sees what set it.
#include <algorithm>
#include <type_traits>

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

// Values that all lanes share, kept in scalar registers.
__device__ __forceinline__ int same(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float same(float v) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}
// The bits of a power of two over those of another, as their ratio (0 below
// the normal range).
__device__ __forceinline__ float power_ratio(int a, int b) {
  const int d = a - b + 0x3F800000;
  return __uint_as_float(d > 0 ? d : 0);
}

// Maximum over the four lanes that share a query (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float query_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t x = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Weights are 2^kWeightBits e^(s - m).  m follows a row's maximum only when a
// lane's 16 weights of a page sum to more than kMostWeight, which fp16 still
// holds: most pages look for no maximum and leave sums and outputs as they
// are.
// A maximum beyond kFarScore is too coarse to hold kWeightBits beside it: the
// weights are held to what fp16 holds one by one.
constexpr float kWeightBits = 10.f, kMostWeight = 32768.f, kFarScore = 1 << 20;
constexpr int kWaves = 4, kXcds = 8;
// In the bits of a float: codes times 2^-11 .. 2^7 are exact in fp16 (448 2^7
// is below its largest value, 2^-9 2^-11 above its smallest), outputs may
// reach 2^124, and 2^-126 is the least normal number.
constexpr int kScaleAbove = 7 << 23, kScaleBelow = 11 << 23, kMostOutput = (127 + 124) << 23, kLeastScale = 1 << 23;

// A wave's tile: 16 queries of one KV head.  Query j of the head group is row
// j / grp, head j % grp of the group, so that a tile's queries have
// neighbouring rows.  Lane l holds query l % 16; of a page's scores it has
// keys 16 t + 4 kg + i (kg = l / 16), of the outputs dims 16 n + 4 kg + i.
template <typename A, int HD> struct Tile {
  static constexpr int NS = HD / 32;  // matrix steps along the head
  static constexpr int NP = HD / 16;  // 1 KB pieces of a page's keys (and values)
  f16x8_t qh[NS], qlo[NS];
  float cq;         // score units: 2^(row's exponent) log2(e) / sqrt(hd)
  int qi, qhd;      // the lane's query: row in the sequence, head
  bool valid;
  float m, l;
  f32x4_t o[NP];    // in units of the value scale `unit`
  int unit;         // the bits of a power of two (the least one before the first page)
  int last;         // the page before's value scale, and that scale in units
  float ratio;
  float minus_one;

  __device__ __forceinline__ void init(const Kv8Args& a, const Seq& q, int g, int tile0) {
    const int grp = a.H / a.G, nq = grp * q.n, lane = threadIdx.x & 63, ql = lane & 15, kg = lane >> 4;
    unit = last = kLeastScale;
    ratio = 1.f;
    minus_one = -1.f;
    asm("" : "+s"(minus_one));
    const int j = tile0 * 16 + ql;
    valid = j < nq;
    qi = valid ? j / grp : 0;
    qhd = g * grp + (valid ? j - qi * grp : 0);
    float v[NS][8], amax = 0.f;
    const A* p = reinterpret_cast<const A*>(a.q) + ((size_t)(q.r0 + qi) * a.H + qhd) * HD + kg * (HD / 4);
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
    cq = ldexpf(1.4426950408889634f / sqrtf((float)HD), ex);
#pragma unroll
    for (int c = 0; c < NS; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] *= down;
      split16(v[c], minus_one, qh[c], qlo[c]);
    }
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < NP; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // Scores of a page; piece(n): the lane's 16 key bytes of piece n.
  template <typename F> __device__ __forceinline__ void scores(F piece, f32x4_t (&st)[4]) const {
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) st[kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const u32x4_t w = piece(n);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int kt = (2 * n + h) / NS, c = (2 * n + h) % NS;
        const f16x8_t k = f8_to_f16(w[2 * h], w[2 * h + 1], 1.f);
        mfma16(st[kt], k, qh[c]);
        mfma16(st[kt], k, qlo[c]);
      }
    }
  }

  // The slots of page p that the lane's query sees, this lane's keys at bits 16 t + i.
  __device__ __forceinline__ uint64_t seen(const Kv8Args& a, const Seq& q, int p) const {
    return seen_bits(a.vis ? a.vis + (size_t)(q.r0 + qi) * kVisWords : nullptr, qi, q.n, p * kPage - q.C) >>
           (4 * ((threadIdx.x & 63) >> 4));
  }

  // -inf for the slots of page p that a query does not see.
  __device__ __forceinline__ void mask(const Kv8Args& a, const Seq& q, int p, f32x4_t (&st)[4]) const {
    const uint64_t sees = seen(a, q, p);
    const uint32_t half[2] = {(uint32_t)sees, (uint32_t)(sees >> 32)};
#pragma unroll
    for (int e = 0; e < 16; ++e)
      st[e >> 2][e & 3] = (half[e >> 3] >> (16 * ((e >> 2) & 1) + (e & 3))) & 1 ? st[e >> 2][e & 3] : -INFINITY;
  }

  // Weights of a page with that key scale.
  __device__ __forceinline__ void weights(const f32x4_t (&st)[4], float key_scale, f16x8_t (&ph)[2],
                                          f16x8_t (&pl)[2]) {
    const float f = fmaxf(cq * key_scale, 1.17549435e-38f);  // 0 times the -inf of an unseen slot would be NaN
    float x[16], sum;
    auto compute = [&](float off) {
      sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e >> 2][e & 3], f, off));
        sum += x[e];
      }
    };
    compute(kWeightBits - m);  // nothing seen yet: infinity or NaN
    if (__any(!(sum <= kMostWeight))) {
      float mx = st[0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, st[e >> 2][e & 3]);
      mx = query_max(mx);
      float top = mx * f;
      // beyond 2^24 the rounded product may lie far above the score itself, which would lose all weight
      if (__builtin_fmaf(mx, f, -top) < -1.f) top -= fabsf(top) * 0x1p-23f;
      const float m_new = fmaxf(m, top), m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m - m_use);
      l *= alpha;
      m = m_new;
#pragma unroll
      for (int d = 0; d < NP; ++d) o[d] *= alpha;
      if (__any(fabsf(m_use) > kFarScore)) {
        sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float d = __builtin_fmaf(st[e >> 2][e & 3], f, -m_use);
          x[e] = __builtin_amdgcn_exp2f((d > 4.f ? 4.f : d) + kWeightBits);  // NaN stays
          sum += x[e];
        }
      } else {
        compute(kWeightBits - m_use);
      }
    }
    l += sum;
    split16(x, minus_one, ph[0], pl[0]);
    split16(x + 8, minus_one, ph[1], pl[1]);
  }

  // A page's value scale relative to the outputs' unit (both in scalar
  // registers; powers of two divide by their exponents).
  __device__ __forceinline__ float value_scale(float scale) {
    const int s = max(same((int)__float_as_uint(scale)), kLeastScale);
    if (__builtin_expect(s != last, 0)) {
      last = s;
      if (s > unit + kScaleAbove || s < unit - kScaleBelow) follow(s);
      ratio = power_ratio(s, unit);
    }
    return ratio;
  }
  // The unit becomes s, or goes down as far as the outputs' range allows.
  __device__ __forceinline__ void follow(int s) {
    int to = s;
    if (s < unit) {
      float mine = 0.f;
#pragma unroll
      for (int d = 0; d < NP; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine = fmaxf(mine, fabsf(o[d][i]));
      int top = 0;  // over the lanes, one by one: exchanges would hold registers throughout the loop
#pragma unroll 1
      for (int i = 0; i < 64; ++i) top = max(top, __builtin_amdgcn_readlane((int)__float_as_uint(mine), i));
      to = max(s, unit - min((kMostOutput - top) >> 23 << 23, 127 << 23));
    }
    const float f = power_ratio(unit, to);
#pragma unroll
    for (int d = 0; d < NP; ++d) o[d] *= f;
    unit = to;
  }

  // Weighted values; piece(n): the lane's 16 value bytes of piece n.
  template <typename F>
  __device__ __forceinline__ void outputs(F piece, float vscale, const f16x8_t (&ph)[2], const f16x8_t (&pl)[2]) {
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const u32x4_t w = piece(n);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f16x8_t v = f8_to_f16(w[2 * j], w[2 * j + 1], vscale);
        mfma16(o[n], v, ph[j]);
        mfma16(o[n], v, pl[j]);
      }
    }
  }

  // The same two for pieces that come from LDS, in a fixed order: a piece's
  // reads run two pieces ahead, its conversions beside the matrix
  // instructions of the piece before.  mul(n, i, k) is matrix instruction i of
  // piece n on its operands k.  (The compiler's own order waits for each read.
  // That an instruction adds to the result of the one before costs nothing:
  // two results in turn took the same time.)
  template <typename F, typename M> __device__ __forceinline__ static void feed(F piece, float scale, M mul) {
    u32x4_t w[3];
    F16x8 k[2][2];
    auto convert = [&](int n, int u) {  // conversion u of piece n
      const int h = u >> 2, i = u & 3;
      const uint32_t d = w[n % 3][2 * h + (i >> 1)];
      k[n & 1][h].p[i] = i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(d, scale, true)
                               : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(d, scale, false);
    };
    w[0] = piece(0);
    if (NP > 1) w[1] = piece(1);
#pragma unroll
    for (int u = 0; u < 8; ++u) convert(0, u);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      if (n + 2 < NP) w[(n + 2) % 3] = piece(n + 2);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mul(n, i, k[n & 1]);
        if (n + 1 < NP)
#pragma unroll
          for (int u = 0; u < 2; ++u) convert(n + 1, 2 * i + u);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  template <typename F> __device__ __forceinline__ void scores_fed(F piece, f32x4_t (&st)[4]) const {
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) st[kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    feed(piece, 1.f, [&](int n, int i, const F16x8 (&k)[2]) {
      const int h = i / 2, lo = i % 2, kt = (2 * n + h) / NS, c = (2 * n + h) % NS;
      mfma16(st[kt], k[h].v, lo ? qlo[c] : qh[c]);
    });
  }
  template <typename F>
  __device__ __forceinline__ void outputs_fed(F piece, float vscale, const f16x8_t (&ph)[2],
                                              const f16x8_t (&pl)[2]) {
    feed(piece, vscale, [&](int n, int i, const F16x8 (&k)[2]) {
      const int j = i / 2, lo = i % 2;
      mfma16(o[n], k[j].v, lo ? pl[j] : ph[j]);
    });
  }

  // NaN for the queries that see a NaN among the values that ones(n) marks
  // with the code of 1.
  template <typename F>
  __device__ __forceinline__ void poison(const Kv8Args& a, const Seq& q, int p, F ones) {
    f16x8_t b[2];  // 1 for the keys that a query sees
    const uint64_t sees = seen(a, q, p);
    const uint32_t half[2] = {(uint32_t)sees, (uint32_t)(sees >> 32)};
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) b[j][e] = (half[j] >> (16 * (e >> 2) + (e & 3))) & 1 ? 1.f : 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const u32x4_t w = ones(n);
      f32x4_t hit = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 2; ++j) mfma16(hit, f8_to_f16(w[2 * j], w[2 * j + 1], 1.f), b[j]);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][i] = hit[i] > 0.f ? NAN : o[n][i];
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Sums and outputs (times factor()) as they are merged and divided: 2^-24 of
  // what was summed, as values next to the largest number times weights of
  // 2^kWeightBits would not fit.
  __device__ __forceinline__ void finish() {
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    l *= 0x1p-24f;
  }
  __device__ __forceinline__ float factor() const { return __uint_as_float(unit) * 0x1p-24f; }
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
// key split; the waves take every fourth page straight into registers, as
// nobody shares it, the next page's keys in flight from when this one's scores
// are done, and merge in LDS.  64 sequences of up to 8192 tokens, 28 query and
// 4 KV heads of 128 dims: 58.0 us, 5.7 TB/s.
template <typename A, int HD>
__global__ void __launch_bounds__(256, 2) k_attention_kv8_few(Kv8Args a) {
  using T = Tile<A, HD>;
  constexpr int NP = T::NP;
  __shared__ float s_o[kWaves][16][HD + 4], s_m[kWaves][16], s_l[kWaves][16];
  const int s = blockIdx.x / a.G, g = blockIdx.x % a.G, split = blockIdx.y;
  Seq q;
  if (!batch_seq(a.b, s, q)) return;
  const int pages = (q.C + q.n + kPage - 1) / kPage;
  const int p0 = split * a.chunk, p1 = min(p0 + a.chunk, pages);
  if (p0 >= pages) return;
  const int lane = threadIdx.x & 63, wave = same((int)threadIdx.x >> 6), ql = lane & 15, kg = lane >> 4;
  T w;

  // Page ids: this page's, the next one's and (on its way) the one after; a
  // bad one becomes page 0, of which nothing is used.
  auto entry = [&](int p) { return q.table[min(p, p1 - 1)]; };  // no branch: it would wait for every load
  u32x4_t kr[NP], vr[NP];
  float2 sc = {1.f, 1.f};
  const uint8_t* page = a.kv;
  auto load_keys = [&](int id) {
    page = a.kv + (size_t)max(id, 0) * a.page_bytes;
#pragma unroll
    for (int n = 0; n < NP; ++n) kr[n] = load16<true>(page + (size_t)g * kPage * HD + n * 1024 + lane * 16);
    sc = reinterpret_cast<const float2*>(page + (size_t)2 * a.G * kPage * HD)[g];
  };
  int p = p0 + wave, id = 0, after = 0;
  if (p < p1) {
    const int first = entry(p);
    after = entry(p + kWaves);
    id = batch_page_id(a.b, same(first));
    load_keys(id);
  }
  w.init(a, q, g, 0);
  // Page p; kEdge: it holds slots that not every row sees.
  auto step = [&](auto edge) {
    constexpr bool kEdge = decltype(edge)::value;
    const int next = batch_page_id(a.b, same(after));
    after = entry(p + 2 * kWaves);
#pragma unroll
    for (int n = 0; n < NP; ++n) vr[n] = load16<true>(page + (size_t)(a.G + g) * kPage * HD + n * 1024 + lane * 16);
    f32x4_t st[4];
    w.scores([&](int n) { return kr[n]; }, st);
    const float2 scale = {same(sc.x), same(sc.y)};
    if (p + kWaves < p1) load_keys(next);
    if (id >= 0) {  // a bad page's slots are seen by nobody
      const float vscale = w.value_scale(scale.y);
      f16x8_t ph[2], pl[2];
      if constexpr (kEdge) {
        w.mask(a, q, p, st);
        // 0 times NaN is NaN: NaN codes are taken out, and the rows that see one get it back
        bool any = false;
#pragma unroll
        for (int n = 0; n < NP; ++n) any |= has_nans(vr[n]);
        if (__any(any)) {
          w.poison(a, q, p, [&](int n) { return nan_ones(vr[n]); });
#pragma unroll
          for (int n = 0; n < NP; ++n) vr[n] = without_nans(vr[n]);
        }
      }
      w.weights(st, scale.x, ph, pl);
      w.outputs([&](int n) { return vr[n]; }, vscale, ph, pl);
    }
    id = next;
    p += kWaves;
  };
  const int whole = min(q.C / kPage, p1);
#pragma unroll 1
  while (p < whole) step(std::false_type{});
#pragma unroll 1
  while (p < p1) step(std::true_type{});
  w.finish();

#pragma unroll
  for (int n = 0; n < NP; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s_o[wave][ql][16 * n + 4 * kg + i] = w.o[n][i] * w.factor();
  if (kg == 0) {
    s_m[wave][ql] = w.m;
    s_l[wave][ql] = w.l;
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
  if (w.valid)
    for (int n = wave; n < NP; n += kWaves) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kWaves; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += f[i] * s_o[i][ql][16 * n + 4 * kg + e];
      put_outputs<A>(a, q.r0 + w.qi, w.qhd, split, 16 * n + 4 * kg, m, l, v);
    }
}

// More tiles: one of its own for each of W waves.  Workgroup: KV head, W
// tiles, key split.  A page's codes go from memory to one of two LDS buffers
// without passing registers, while the page before is worked on; the waves
// read them as operands and turn them to fp16 (as fp16 in LDS the writes
// alone, 32 KB a page at the 31 bytes a cycle that they reach, took a quarter
// of the time).  512 rows after up to 8000 keys, heads as above: 128 us, 122
// GFLOP issued at 0.95 PFLOP/s.  Bound by issue: a page's 64 matrix
// instructions of a wave take 1020 cycles, its 230 vector instructions 1150,
// and the three waves of a SIMD overlap these in part.  Two tiles a wave share
// the conversions, but leave registers for two waves a SIMD: 2% more, and 49.1
// against 35.0 for 512 rows after 1000 keys, 17.0 against 11.0 for 16 rows.
template <typename A, int HD, int W>
__global__ void __launch_bounds__(64 * W, 2) k_attention_kv8_many(Kv8Args a) {
  using T = Tile<A, HD>;
  constexpr int NP = T::NP;
  constexpr int kItems = 2 * NP / W;      // 1 KB pieces of a page that each wave brings
  __shared__ u32x4_t s_kv[2][2 * NP][64];      // pieces: keys, then values
  const int grp = a.H / a.G;
  // Workgroups go around the 8 XCDs in order: each gets a run of consecutive
  // work, so that the groups that read the same pages share an L2.
  const int work = blockIdx.x % kXcds * (gridDim.x / kXcds) + blockIdx.x / kXcds;
  const int group = work % a.groups, split = work / a.groups % a.splits, g = work / (a.groups * a.splits) % a.G;
  const int s = work / (a.groups * a.splits * a.G);
  if (s >= a.b.n_seqs) return;
  Seq q;
  if (!batch_seq(a.b, s, q)) return;
  const int nq = grp * q.n;
  const int lane = threadIdx.x & 63, wave = same((int)threadIdx.x >> 6), kg = lane >> 4;
  if (group * W * 16 >= nq) return;
  const int pages = (q.C + q.n + kPage - 1) / kPage;
  const int p0 = split * a.chunk;
  int p1 = min(p0 + a.chunk, pages);
  if (p0 >= pages) return;
  const int tile0 = group * W + wave;
  int mine = tile0 * 16 < nq ? p1 : p0;        // the wave's tiles need pages [p0, mine)
  if (!a.vis) {                                // causal: no slot past the last row
    const int last_wave = min((tile0 + 1) * 16, nq) - 1, last = min((group + 1) * W * 16, nq) - 1;
    mine = min(mine, (q.C + last_wave / grp) / kPage + 1);
    p1 = min(p1, (q.C + last / grp) / kPage + 1);
  }
  T w;
  w.init(a, q, g, tile0);

  // Page ids: the next page's and (on its way) the one after; a bad one
  // becomes page 0, of which nothing is used.
  auto entry = [&](int p) { return q.table[min(p, p1 - 1)]; };  // no branch: it would wait for every load
  float2 sc = {1.f, 1.f};
  const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)reinterpret_cast<char*>(s_kv) +
                        wave * 1024;
  auto load = [&](int buf, int id) {  // a page on its way into a buffer, and its scales
    const uint8_t* page = a.kv + (size_t)max(id, 0) * a.page_bytes;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int piece = i * W + wave;
      dma_1k<false>(reinterpret_cast<const char*>(page) + ((piece < NP ? g : a.G + g) * kPage * HD + piece % NP * 1024),
                    lane * 16, ring + (buf * 2 * NP + i * W) * 1024);
    }
    sc = reinterpret_cast<const float2*>(page + (size_t)2 * a.G * kPage * HD)[g];
  };
  int buf = 0, id = 0, after = 0;
  if (p0 < p1) {
    const int first = entry(p0);
    after = entry(p0 + 1);
    id = batch_page_id(a.b, same(first));
    load(0, id);
  }
  // Page p; kEdge: it holds slots that not every row sees.
  auto step = [&](auto edge, int p) {
    constexpr bool kEdge = decltype(edge)::value;
    // every wave's pieces of page p have arrived, and its work on the page before is done
    wait_vm<0>();
    __syncthreads();
    const float2 scale = {same(sc.x), same(sc.y)};
    const bool work = id >= 0 && p < mine;  // a bad page's slots are seen by nobody
    const int next = batch_page_id(a.b, same(after));
    if (p + 1 < p1) load(buf ^ 1, next);
    after = entry(p + 2);
    if (work) {
      auto key = [&](int n) { return s_kv[buf][n][lane]; };
      auto value = [&](int n) { return s_kv[buf][NP + n][lane]; };
      const float vscale = w.value_scale(scale.y);
      f32x4_t st[4];
      w.scores_fed(key, st);
      if constexpr (kEdge) w.mask(a, q, p, st);
      f16x8_t ph[2], pl[2];
      w.weights(st, scale.x, ph, pl);
      if constexpr (kEdge) {
        // 0 times NaN is NaN: NaN codes are taken out, and the rows that see one get it back
        bool any = false;
#pragma unroll
        for (int n = 0; n < NP; ++n) any |= has_nans(value(n));
        if (__any(any)) {
          w.poison(a, q, p, [&](int n) { return nan_ones(value(n)); });
          w.outputs_fed([&](int n) { return without_nans(value(n)); }, vscale, ph, pl);
        } else {
          w.outputs_fed(value, vscale, ph, pl);
        }
      } else {
        w.outputs_fed(value, vscale, ph, pl);
      }
    }
    id = next;
    buf ^= 1;
  };
  int p = p0;
#pragma unroll 1
  for (const int whole = min(q.C / kPage, p1); p < whole; ++p) step(std::false_type{}, p);
#pragma unroll 1
  for (; p < p1; ++p) step(std::true_type{}, p);
  w.finish();
  if (w.valid)
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const float unit = w.factor();
      float v[4] = {w.o[n][0] * unit, w.o[n][1] * unit, w.o[n][2] * unit, w.o[n][3] * unit};
      put_outputs<A>(a, q.r0 + w.qi, w.qhd, split, 16 * n + 4 * kg, w.m, w.l, v);
    }
}

// Merges a row's key splits, four dims of one row and head a thread.  SG
// threads share an item, each taking every SG-th split, at most kMaxSplits /
// SG of them with all loads in flight at once, and join in LDS.  Splits are
// added in the same order whatever the timing.
constexpr int kMaxSplits = 64;
template <typename A, int SG>
__global__ void __launch_bounds__(256) k_attention_kv8_merge(Kv8Args a, int blocks) {
  constexpr int kEach = SG == 1 ? 8 : kMaxSplits / SG;
  __shared__ float s_part[SG > 1 ? 256 : 1][6];
  const int s = blockIdx.x / blocks;
  Seq q;
  if (!batch_seq(a.b, s, q)) return;
  const int chunks = a.hd / 4, per = 256 / (chunks * SG);  // items of a workgroup
  const int tid = threadIdx.x, dim = tid % chunks * 4, group = tid / chunks % SG;
  const int item = blockIdx.x % blocks * per + tid / (chunks * SG);
  const bool valid = item < q.n * a.H;
  const int h = valid ? item % a.H : 0, row = q.r0 + (valid ? item / a.H : 0);
  const int n = ((q.C + q.n + kPage - 1) / kPage + a.chunk - 1) / a.chunk;
  const size_t stride = (size_t)a.b.n_rows * a.H, at = (size_t)row * a.H + h;
  float2 ml[kEach];
  float4 o[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int k = group + j * SG;
    ml[j] = make_float2(-INFINITY, 0.f);
    o[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (k < n) {
      ml[j] = *reinterpret_cast<const float2*>(a.ml_part + (k * stride + at) * 2);
      o[j] = *reinterpret_cast<const float4*>(a.o_part + (k * stride + at) * a.hd + dim);
    }
  }
  float m = -INFINITY, l = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kEach; ++j) m = fmaxf(m, ml[j].x);
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const float f = ml[j].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[j].x - m);
    l += ml[j].y * f;
    v[0] += o[j].x * f; v[1] += o[j].y * f; v[2] += o[j].z * f; v[3] += o[j].w * f;
  }
  if constexpr (SG > 1) {
    float* p = s_part[tid];
    p[0] = m; p[1] = l; p[2] = v[0]; p[3] = v[1]; p[4] = v[2]; p[5] = v[3];
    __syncthreads();
    if (group) return;
    const float* g = s_part[tid];  // the groups' parts are chunks threads apart
    float mm = -INFINITY;
#pragma unroll
    for (int j = 0; j < SG; ++j) mm = fmaxf(mm, g[j * chunks * 6]);
    l = v[0] = v[1] = v[2] = v[3] = 0.f;
#pragma unroll
    for (int j = 0; j < SG; ++j) {
      const float* x = g + j * chunks * 6;
      const float f = x[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[0] - mm);
      l += x[1] * f;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += x[2 + e] * f;
    }
  }
  if (!valid) return;
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = inv == 0.f ? 0.f : v[e] * inv;
  act_store4(reinterpret_cast<A*>(a.out) + act_offset(row, h * a.hd + dim, a.H * a.hd), a.out_plane, v);
}

// ---- launch --------------------------------------------------------------------------

// One tile: up to 20 pages in one workgroup a head, which saves the merge (1
// row after 1024 keys 9.7 us, split five ways 6.0 and 3.2 for the merge);
// beyond, 512 workgroups of 4 to 24 pages (64 ragged sequences of up to 8192:
// 24 pages 57.6 us, 64 pages 61.7).
// More tiles: as many splits as fill the chip's places, three workgroups of
// four waves a compute unit (64 sequences of 6 rows after up to 4000 keys 54.1
// us, 62.0 with two), of 8 pages or more (192 rows after 2048 keys: 8 pages
// 25.8 us and 6.4 for the merge, 4 pages 24.1 and 12.9), or of 4 where these
// leave most of the chip free (16 rows after 1024 keys: 10.5 against 14.7 us).
// Two tiles have workgroups of two waves, four a compute unit, as two more
// waves would only load (64 sequences of 4 rows 41.9 us, 57.6 with four waves).
void kv8_plan(Kv8Args& a) {
  const int tiles = (int)(((int64_t)a.H / a.G * a.b.max_rows + 15) / 16);
  a.waves = tiles <= 2 ? tiles : kWaves;
  a.groups = (tiles + a.waves - 1) / a.waves;
  const int pages = (a.b.max_ctx + kPage - 1) / kPage;
  const int64_t base = (int64_t)a.b.n_seqs * a.G * a.groups;
  if (tiles == 1) {
    const int64_t c = (base * pages / 512 + 2) / 4 * 4;
    a.chunk = pages <= 20 ? pages : (int)std::min<int64_t>(std::max<int64_t>(c, 4), 24);
  } else {
    const int64_t want = std::max<int64_t>((a.waves == 2 ? 1024 : 768) / base, 1);
    a.chunk = std::max<int>((int)((pages + want - 1) / want), base * pages <= 1024 ? 4 : 8);
  }
  a.chunk = std::max(a.chunk, (pages + kMaxSplits - 1) / kMaxSplits);
  a.splits = (pages + a.chunk - 1) / a.chunk;
}

template <typename A, int HD>
static void attention_qt(const Kv8Args& a, hipStream_t st) {
  const dim3 few((unsigned)(a.b.n_seqs * a.G), (unsigned)a.splits);
  const unsigned many = (unsigned)((a.b.n_seqs * a.G * a.groups * a.splits + kXcds - 1) / kXcds * kXcds);
  if (a.waves == 1) k_attention_kv8_few<A, HD><<<few, 256, 0, st>>>(a);
  else if (a.waves == 2) k_attention_kv8_many<A, HD, 2><<<many, 128, 0, st>>>(a);
  else k_attention_kv8_many<A, HD, 4><<<many, 256, 0, st>>>(a);
}
template <typename A> static hipError_t attention_act(const Kv8Args& a, hipStream_t st) {
  if (a.hd == 32) attention_qt<A, 32>(a, st);
  else if (a.hd == 64) attention_qt<A, 64>(a, st);
  else attention_qt<A, 128>(a, st);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int per = 256 / (a.hd / 4 * (a.splits > 8 ? 8 : 1));
  const int blocks = (a.b.max_rows * a.H + per - 1) / per;
  if (a.splits > 8) k_attention_kv8_merge<A, 8><<<(unsigned)(a.b.n_seqs * blocks), 256, 0, st>>>(a, blocks);
  else k_attention_kv8_merge<A, 1><<<(unsigned)(a.b.n_seqs * blocks), 256, 0, st>>>(a, blocks);
  return hipGetLastError();
}
hipError_t launch_attention_kv8(int act, const Kv8Args& a, hipStream_t st) {
  return act == 0 ? attention_act<float>(a, st) : attention_act<bf16_t>(a, st);
}

}  // namespace jf
