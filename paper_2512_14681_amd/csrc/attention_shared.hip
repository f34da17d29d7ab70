// Grouped-query attention of a batch of sequences over a paged fp32 or bf16
// cache in which groups of sequences share their first pages
// (jf_attention_shared).
//
// The rows of all sequences of a group go over the shared pages together, as
// one product, and the rows of each sequence over the pages of its own; what
// the parts give (maximum, sum, weighted values) is merged.  Both kinds of
// work are in one launch.
//
// A wave works on 32 queries (row, head) of one KV head.  Scores come out of
// the matrix cores transposed (keys x queries), with a page's keys in an
// order that gives a lane 8 consecutive keys of its query: these weights and
// 8 consecutive keys of V^T, as the page holds it, are operands of O^T += V^T P^T.
//
// Precision: bf16 queries come as two terms (hi and lo) and the weights enter
// the second product as two, which keeps 16 bits of either; keys and values
// are exact.  Sums and maxima are fp32.
#include <algorithm>
#include <type_traits>

#include "jf_batch.h"
#include "jf_tile32.h"

namespace jf {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
// Weights are 2^(s - m - kDown).  m follows a row's maximum only when a lane's
// weights of a step sum to more than kMost.  kDown keeps sums of weights below
// 1, so that no sum of values overflows that has a finite mean.  A maximum
// beyond kFar is too coarse to hold kDown beside it: the weights are held
// below 2^(4 - kDown) one by one.
constexpr float kDown = 32.f, kMost = 0x1p-22f, kFar = 1 << 20;
constexpr int kChunk = 4;      // pages of a part at least
constexpr int kWorkgroups = 512;  // as many as run at once
constexpr int kFewTiles = 32;     // tiles of a group's or sequence's queries that have workgroups of their own

// Queries as operands: bf16 in two terms.
template <typename T> struct Query;
template <> struct Query<bf16_t> { Frag<bf16_t> hi, lo; };
template <> struct Query<float> { Frag<float> v; };
__device__ __forceinline__ void load_query(const bf16_t* p, size_t plane, Query<bf16_t>& q) {
  q.hi = frag_load<bf16_t>(p);
  q.lo = frag_load<bf16_t>(p + plane);
}
__device__ __forceinline__ void load_query(const float* p, size_t, Query<float>& q) { q.v = frag_load<float>(p); }
__device__ __forceinline__ void settle_query(Query<bf16_t>& q) {
  settle(reinterpret_cast<Frag<bf16_t>(&)[1]>(q.hi));
  settle(reinterpret_cast<Frag<bf16_t>(&)[1]>(q.lo));
}
__device__ __forceinline__ void settle_query(Query<float>& q) { settle(reinterpret_cast<Frag<float>(&)[1]>(q.v)); }
__device__ __forceinline__ void split_query(const float* x, Query<bf16_t>& q) {
  split2(x[0], x[1], q.hi.v.x, q.lo.v.x);
  split2(x[2], x[3], q.hi.v.y, q.lo.v.y);
  split2(x[4], x[5], q.hi.v.z, q.lo.v.z);
  split2(x[6], x[7], q.hi.v.w, q.lo.v.w);
}
__device__ __forceinline__ void split_query(const float* x, Query<float>& q) { frag_of(x, q.v); }
__device__ __forceinline__ void mul(f32x16_t& acc, const Frag<bf16_t>& a, const Query<bf16_t>& b) {
  mfma32(acc, a, b.hi);
  mfma32(acc, a, b.lo);
}
__device__ __forceinline__ void mul(f32x16_t& acc, const Frag<float>& a, const Query<float>& b) { mfma32(acc, a, b.v); }

// What a sequence shares: the first `pages` pages, if its group is what the
// host announced, no group before starts behind it (it then overlaps none,
// whose work it would do once more) and the sequence's rows are among the
// group's, r0 .. r1 - 1 (else false, with JF_FLAG_CAPACITY raised).
__device__ __forceinline__ bool group_ok(const SharedArgs& a, int s0, int s1, int pages, int& r0, int& r1) {
  if (s0 < 0 || s1 < s0 || s1 > a.b.n_seqs || pages < 0 || pages > a.max_pages) return false;
  r0 = a.b.row_start[s0];
  r1 = a.b.row_start[s1];
  return r0 >= 0 && r1 >= r0 && r1 <= a.b.n_rows && r1 - r0 <= a.max_group_rows;
}
__device__ __forceinline__ bool shared_pages(const SharedArgs& a, int s, const Seq& q, int& pages) {
  const int lane = threadIdx.x & 63;
  int top = 0;  // of the starts looked through before
  pages = 0;
  bool ok = true;
  for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
    const int g = g0 + lane;
    const int s0 = g < a.n_groups ? a.seq_start[g] : 0, s1 = g < a.n_groups ? a.seq_start[g + 1] : 0;
    const uint64_t hit = __ballot(s0 <= s && s < s1);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      const int at = __builtin_amdgcn_readlane(s0, l);
      int r0, r1;
      pages = a.pages[g0 + l];
      ok = group_ok(a, at, __builtin_amdgcn_readlane(s1, l), pages, r0, r1) && pages <= q.C / kPage && q.r0 >= r0 &&
           q.r0 + q.n <= r1 &&  // row starts within a group may go beyond its ends
           !(__ballot(s0 > at) & ((1ull << l) - 1)) && !__any(top > at);
      break;
    }
    top = max(top, s0);
  }
  if (!ok && a.b.flags && threadIdx.x == 0) atomicOr(a.b.flags, kFlagCapacity);
  return ok;
}
// Values that all lanes share, in scalar registers.
__device__ __forceinline__ int same(int v) { return __builtin_amdgcn_readfirstlane(v); }
// Pages of a part, when `splits` parts at most share n pages.
__device__ __forceinline__ int part_pages(int n, int splits) {
  return max((n + splits - 1) / max(splits, 1), kChunk);
}

}  // namespace

// A wave's 32 queries of KV head g: query j is row j / grp, head j % grp of
// the group's.  Lane l holds query l % 32.
template <typename T, int HD> struct SharedTile {
  static constexpr int NS = HD / 16, ND = HD / 32;
  Query<T> q[NS];
  int qi, qhd;    // the lane's query: row among the job's, head
  bool valid, far;  // far (of all lanes): maxima beyond kFar
  float m, l;
  f32x16_t o[ND];

  __device__ __forceinline__ void init(const SharedArgs& a, int r0, int n, int g, int tile) {
    const int grp = a.H / a.G, nq = grp * n, lane = threadIdx.x & 63;
    const int j0 = tile * 32 + (lane & 31), j = min(j0, nq - 1);
    valid = j0 < nq;
    qi = j / grp;
    qhd = g * grp + j - qi * grp;
    const T* p = reinterpret_cast<const T*>(a.q) + ((size_t)(r0 + qi) * a.H + qhd) * HD + 8 * (lane >> 5);
#pragma unroll
    for (int s = 0; s < NS; ++s) load_query(p + 16 * s, a.q_plane, q[s]);
#pragma unroll
    for (int s = 0; s < NS; ++s) settle_query(q[s]);
    m = -INFINITY;
    l = 0.f;
    far = false;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] = zero16();
  }

  // Scores of 32 KT keys in LDS (in PageLoader's order).
  template <int KT> __device__ __forceinline__ void scores(const char* tile, f32x16_t (&st)[KT]) const {
    const uint32_t keys = RowTile<T, HD>::row_base(lds_address(tile));
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) st[kt] = zero16();
    stream<T, KT * NS, kAhead<T>>([&](int n) { return RowTile<T, HD>::rows(keys, n % KT * 32, n / KT); },
                                  [&](int n, const Frag<T>& k) { mul(st[n % KT], k, q[n / KT]); });
  }
  // Their weights, and the weighted values (V^T in LDS, there once arrive() is
  // back).  kEdge: seen holds a bit for each key that the lane's query sees.
  // False if there were values that are not finite, which count as 0 here.
  template <int KT, bool kEdge, typename F>
  __device__ __forceinline__ bool outputs(f32x16_t (&st)[KT], const char* tile, uint64_t seen, F arrive) {
    using Values = RowTile<T, 32 * KT>;
    const float c = kLog2e / sqrtf((float)HD);
    seen >>= 8 * ((threadIdx.x & 63) >> 5);
    const uint32_t bits[2] = {(uint32_t)seen, (uint32_t)(seen >> 32)};
    if constexpr (kEdge) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) st[kt][i] = (bits[kt] >> (16 * (i / 8) + i % 8)) & 1 ? st[kt][i] : -INFINITY;
    }
    float sum;
    f32x16_t w[KT];
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
    arrive();
    const uint32_t values = Values::row_base(lds_address(tile));
    bool finite = true;
    if constexpr (kEdge) {  // 0 times a value that is not finite would reach rows that do not see it
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 2 * KT; ++j)
#pragma unroll
        for (int d = 0; d < ND; ++d) magnitude(Values::rows(values, 32 * d, j), top);
      finite = !__any(!all_finite<T>(top));
      asm volatile("" ::: "memory");  // read again rather than kept: registers
    }
    Query<T> pf[2 * KT];
#pragma unroll
    for (int j = 0; j < 2 * KT; ++j) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = w[j / 2][8 * (j % 2) + e];
      split_query(p, pf[j]);
    }
    if (!kEdge || finite) {
      stream<T, 2 * KT * ND, kAhead<T>>([&](int n) { return Values::rows(values, n % ND * 32, n / ND); },
                                        [&](int n, const Frag<T>& v) { mul(o[n % ND], v, pf[n / ND]); });
    } else {
#pragma unroll
      for (int n = 0; n < 2 * KT * ND; ++n) {
        __builtin_amdgcn_sched_barrier(0);
        Frag<T> v = Values::rows(values, n % ND * 32, n / ND);
        keep_finite(v);
        mul(o[n % ND], v, pf[n / ND]);
      }
    }
    return finite;
  }
  // What the queries see of infinities and NaN among the values that outputs left out.
  template <int KT> __device__ __forceinline__ void infinite(const char* tile, uint64_t seen) {
    const uint32_t values = RowTile<T, 32 * KT>::row_base(lds_address(tile));
    seen >>= 8 * ((threadIdx.x & 63) >> 5);
#pragma unroll 1
    for (int j = 0; j < 2 * KT; ++j) {
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = (seen >> (16 * j + e)) & 1 ? 1.f : 0.f;
      Frag<T> sees;
      frag_of(p, sees);
#pragma unroll
      for (int d = 0; d < ND; ++d) add_infinite<T>(o[d], RowTile<T, 32 * KT>::rows(values, 32 * d, j), sees);
    }
  }
};

// Brings 32 KT keys of a page from token t0 on, and their V^T, into LDS, by W
// waves of which this is number `wave`.  LDS row r of the keys holds the key
// with bits 2 and 3 of r exchanged: a result's elements 8 j .. + 7 of lane l
// then are keys 16 j + 8 (l / 32) .. + 7.
template <typename T, int HD, int KT, int W> struct PageLoader {
  static constexpr int kKeyRow = HD * (int)sizeof(T), kValueRow = 32 * KT * (int)sizeof(T);
  static constexpr int kBytes = 32 * KT * kKeyRow;                     // of the keys, and of the values
  static constexpr int kPieces = kBytes / 1024 / W;                    // 1 KB pieces a wave, of either
  static constexpr int kKeyRows = 1024 / kKeyRow, kValueRows = 1024 / kValueRow;  // rows of a piece
  static_assert(kPieces * W * 1024 == kBytes, "whole pieces");
  static_assert(kKeyRows <= 16 && kValueRows <= 16, "places repeat after 16 rows");
  // Few offsets in registers: they repeat every 16 rows, the rest is the same for all lanes.
  static __device__ __forceinline__ void keys(const T* page, int t0, int wave, char* tile) {
    constexpr int kPeriod = std::max(16 / (kKeyRows * W), 1);
    const int lane = threadIdx.x & 63;
    const uint32_t at = lds_address(tile) + wave * 1024;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int row = ((i % kPeriod * W + wave) * kKeyRows) % 16 + lane * 16 / kKeyRow;
      const int c = (lane * 16 % kKeyRow / 16) ^ turn<kKeyRow>(row), key = (row & ~12) | ((row & 4) << 1) | ((row & 8) >> 1);
      const int skip = (i * W + wave) * kKeyRows / 16 * 16;
      dma_1k<false>(reinterpret_cast<const char*>(page + (size_t)t0 * HD) + skip * kKeyRow, key * kKeyRow + c * 16, at + i * W * 1024);
    }
  }
  static __device__ __forceinline__ void values(const T* page, int t0, int wave, char* tile) {
    constexpr int kPeriod = std::max(16 / (kValueRows * W), 1), kStride = kPage * (int)sizeof(T);
    const int lane = threadIdx.x & 63;
    const uint32_t at = lds_address(tile) + wave * 1024;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int row = ((i % kPeriod * W + wave) * kValueRows) % 16 + lane * 16 / kValueRow;
      const int c = (lane * 16 % kValueRow / 16) ^ turn<kValueRow>(row), skip = (i * W + wave) * kValueRows / 16 * 16;
      dma_1k<false>(reinterpret_cast<const char*>(page + t0) + skip * kStride, row * kStride + c * 16, at + i * W * 1024);
    }
  }
};

// Four outputs of a query: the result, or a part of it.
template <typename T>
__device__ __forceinline__ void put_outputs(const SharedArgs& a, int row, int head, int part, int dim, float m, float l,
                                            float (&v)[4]) {
  if (part < 0) {
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = inv == 0.f ? 0.f : v[i] * inv;
    act_store4(reinterpret_cast<T*>(a.out) + act_offset(row, head * a.hd + dim, a.H * a.hd), a.out_plane, v);
  } else {
    const size_t at = ((size_t)part * a.b.n_rows + row) * a.H + head;
    *reinterpret_cast<float4*>(a.o_part + at * a.hd + dim) = make_float4(v[0], v[1], v[2], v[3]);
    if (dim == 0) *reinterpret_cast<float2*>(a.ml_part + at * 2) = make_float2(m, l);
  }
}

// 64 samples of one row over 128 shared pages and 1 to 500 slots of their own
// (28 query and 4 KV heads of 128 dims, bf16): 32 us.  The shared pages are a
// product of 448 queries a KV head with two terms of each operand (16 GFLOP),
// the rest reads 44 MB: neither fills the chip.  What bounds it is the length
// of a wave's chain (table entry, page, scores, weights, outputs) over every
// fourth page of a part, 8 of 32 here: shorter parts are more than run at once
// or more than the merge can join as fast.  Three samples of two rows in fp32:
// 11 us, one such chain.
template <typename T, int HD>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) k_attention_shared(SharedArgs a) {
  using Tile = SharedTile<T, HD>;
  constexpr int KT = HD * sizeof(T) == 64 ? 2 : 1, ND = HD / 32;  // a 1 KB piece of a step's keys for every wave
  constexpr int kOne = 2 * 32 * HD * (int)sizeof(T);   // 32 keys and their values
  constexpr int kBytes = std::max(4 * KT * kOne, 4 * 32 * HD * 4);  // 4 waves' steps, or 4 stages; the waves' outputs
  __shared__ __align__(1024) char s_kv[kBytes];
  __shared__ float s_ml[4][2][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  // The jobs: shared pages first.
  const bool shared = (int)blockIdx.x < a.shared_jobs;
  int job = shared ? blockIdx.x : blockIdx.x - a.shared_jobs;
  const int splits = shared ? a.shared_splits : a.own_splits, groups = shared ? a.shared_groups : a.own_groups;
  const int g = job % a.G, split = job / a.G % splits, group = job / (a.G * splits) % groups;
  const int unit = job / (a.G * splits * groups);
  int r0, n, p0, p1, part;
  const int32_t* table;
  Seq q{};
  if (shared) {
    const int s0 = a.seq_start[unit], s1 = a.seq_start[unit + 1], pages = a.pages[unit];
    int r1;
    bool behind = false;  // a group before starts behind this one
#pragma unroll 4
    for (int i = lane; i < unit; i += 64) behind |= a.seq_start[i] > s0;
    if (!group_ok(a, s0, s1, pages, r0, r1) || __any(behind)) {
      if (a.b.flags && threadIdx.x == 0) atomicOr(a.b.flags, kFlagCapacity);
      return;
    }
    if (s0 == s1) return;
    n = r1 - r0;
    table = a.b.table + (size_t)s0 * a.b.stride;
    const int chunk = part_pages(pages, splits);
    p0 = split * chunk;
    p1 = min(p0 + chunk, pages);
    part = split;
  } else {
    int pages;
    if (!batch_seq(a.b, unit, q) || !shared_pages(a, unit, q, pages)) return;
    r0 = q.r0;
    n = q.n;
    table = q.table;
    const int end = (q.C + q.n + kPage - 1) / kPage, chunk = part_pages(end - pages, splits);
    p0 = pages + split * chunk;
    p1 = min(p0 + chunk, end);
    part = a.parts == 1 ? -1 : a.shared_splits + split;
  }
  const int nq = a.H / a.G * n;
  const bool few = shared ? a.shared_few : a.own_few;
  if (p0 >= p1 || group * (few ? 32 : 128) >= nq) return;
  const int whole = shared ? p1 : max(min(q.C / kPage, p1), p0);   // pages below are seen by all
  const T* pool = reinterpret_cast<const T*>(a.kv);
  const size_t page_elems = (size_t)2 * a.G * kPage * HD, values_at = (size_t)a.G * kPage * HD;
  // slots of page p that the lane's query sees
  auto seen = [&](const Tile& w, int p) {
    return seen_bits(a.vis ? a.vis + (size_t)(r0 + w.qi) * kVisWords : nullptr, w.qi, n, p * kPage - q.C);
  };
  Tile w;
  if (few) {
    // One tile (few of them read a page): the waves take every fourth page, each in LDS of its own, half
    // a page a step.  The next step's keys come as soon as this one's scores
    // are done, its values once this one's are used.
    using Loader = PageLoader<T, HD, 1, 1>;
    w.init(a, r0, n, g, group);
    constexpr int kFly = Loader::kPieces;
    char *keys = s_kv + wave * kOne, *values = keys + kOne / 2;
    auto entry = [&](int p) { return table[min(p, p1 - 1)]; };
    auto read_done = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };  // before a load takes the place
    bool finite = true;
    // Pages p, p + 4, ... below `to`.
    auto pages = [&](auto edge, int p, int to) {
      if (p >= to) return;
      constexpr bool kEdge = decltype(edge)::value;
      int id = batch_page_id(a.b, same(entry(p))), after = entry(p + 4);
      const T* page = pool + (size_t)max(id, 0) * page_elems + (size_t)g * kPage * HD;
      Loader::keys(page, 0, 0, keys);
      Loader::values(page + values_at, 0, 0, values);
#pragma unroll 1
      for (; p < to; p += 4) {
        uint64_t bits = 0;
        if constexpr (kEdge) bits = id >= 0 ? seen(w, p) : 0;
        const int next = p + 4 < to ? batch_page_id(a.b, same(after)) : id;
        after = entry(p + 8);
        const T* next_page = pool + (size_t)max(next, 0) * page_elems + (size_t)g * kPage * HD;
#pragma unroll 1
        for (int t0 = 0; t0 < kPage; t0 += 32) {
          const T* from = t0 ? next_page : page;  // where the next step's are (once more the last one's at the end)
          const int at = t0 ? 0 : 32;
          f32x16_t st[1];
          wait_vm<kFly>();
          w.template scores<1>(keys, st);
          read_done();
          Loader::keys(from, at, 0, keys);
          if (kEdge || id >= 0) finite &= w.template outputs<1, kEdge>(st, values, bits >> t0, [] { wait_vm<kFly>(); });
          else wait_vm<kFly>();  // a bad page's slots are seen by nobody
          read_done();
          Loader::values(from + values_at, at, 0, values);
        }
        id = next;
        page = next_page;
      }
      wait_vm<0>();
    };
    pages(std::false_type{}, p0 + wave, whole);
    const int edges = p0 + wave + (max(whole - p0 - wave, 0) + 3) / 4 * 4;
    pages(std::true_type{}, edges, p1);
    if (!finite)
#pragma unroll 1
      for (int p = edges; p < p1; p += 4) {
        const int id = batch_page_id(a.b, same(entry(p)));
        if (id < 0) continue;
        const uint64_t bits = seen(w, p);
#pragma unroll 1
        for (int t0 = 0; t0 < kPage; t0 += 32) {
          Loader::values(pool + (size_t)id * page_elems + (size_t)g * kPage * HD + values_at, t0, 0, values);
          wait_vm<0>();
          w.template infinite<1>(values, bits >> t0);
          read_done();
        }
      }
    // The waves' parts, dims by queries; each wave merges a quarter of the dims.
    w.l = pair_sum(w.l);
    __syncthreads();
    float* s_o = reinterpret_cast<float*>(s_kv);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) s_o[(wave * HD + 32 * d + acc_row(i) + 4 * h) * 32 + (lane & 31)] = w.o[d][i];
    if (h == 0) {
      s_ml[wave][0][lane] = w.m;
      s_ml[wave][1][lane] = w.l;
    }
    __syncthreads();
    if (!w.valid) return;
    float m = -INFINITY, l = 0.f, f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, s_ml[i][0][lane & 31]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = s_ml[i][0][lane & 31] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_ml[i][0][lane & 31] - m);
      l += s_ml[i][1][lane & 31] * f[i];
    }
#pragma unroll
    for (int k = 0; k < HD / 32; ++k) {
      const int dim = wave * (HD / 4) + 8 * k + 4 * h;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += f[i] * s_o[(i * HD + dim + e) * 32 + (lane & 31)];
      put_outputs<T>(a, r0 + w.qi, w.qhd, part, dim, m, l, v);
    }
    return;
  }
  // Four tiles, one a wave, over pages that all share: steps of 32 KT keys,
  // kStages - 1 of them on their way.
  using Loader = PageLoader<T, HD, KT, 4>;
  constexpr int kStep = 32 * KT, kTile = KT * kOne, kStages = 4, kFly = 2 * Loader::kPieces, kPerPage = kPage / kStep;
  w.init(a, r0, n, g, group * 4 + wave);
  const bool work = (group * 4 + wave) * 32 < nq;
  // Pages [from, to).
  auto pages = [&](auto edge, int from, int to, auto use) {
    constexpr bool kEdge = decltype(edge)::value;
    if (from >= to) return;
    const int steps = (to - from) * kPerPage;
    auto entry = [&](int p) { return table[min(p, to - 1)]; };
    // what is to be loaded next: its page, and the entry after that
    int ahead = 0, id = batch_page_id(a.b, same(entry(from))), after = entry(from + 1);
    uint32_t good = 0;   // whether the steps' pages can be used, the latest at bit 0
    auto load = [&] {
      const T* page = pool + (size_t)max(id, 0) * page_elems + (size_t)g * kPage * HD;
      char* tile = s_kv + ahead % kStages * kTile;
      const int t0 = ahead % kPerPage * kStep;
      Loader::keys(page, t0, wave, tile);
      Loader::values(page + values_at, t0, wave, tile + kTile / 2);
      good = good << 1 | (id >= 0 ? 1 : 0);
      if (++ahead % kPerPage == 0 && ahead < steps) {
        id = batch_page_id(a.b, same(after));
        after = entry(from + ahead / kPerPage + 1);
      }
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) load();   // past the end: the last page once more
    uint64_t bits = 0;
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
      if constexpr (kEdge)
        if (i % kPerPage == 0) bits = seen(w, from + i / kPerPage);
      wait_vm<(kStages - 2) * kFly>();
      __syncthreads();
      const bool usable = work && (good >> (kStages - 2) & 1);
      load();
      if (usable) use(s_kv + i % kStages * kTile, bits >> (i % kPerPage * kStep));
    }
    wait_vm<0>();
    __syncthreads();
  };
  bool finite = true;
  pages(std::false_type{}, p0, whole, [&](const char* t, uint64_t bits) {
    f32x16_t st[KT];
    w.template scores<KT>(t, st);
    w.template outputs<KT, false>(st, t + kTile / 2, bits, [] {});
  });
  if (whole < p1) {
    pages(std::true_type{}, whole, p1, [&](const char* t, uint64_t bits) {
      f32x16_t st[KT];
      w.template scores<KT>(t, st);
      finite &= w.template outputs<KT, true>(st, t + kTile / 2, bits, [] {});
    });
    if (__syncthreads_or(!finite))
      pages(std::true_type{}, whole, p1, [&](const char* t, uint64_t bits) { w.template infinite<KT>(t + kTile / 2, bits); });
  }
  if (!w.valid) return;
  w.l = pair_sum(w.l);
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      float v[4] = {w.o[d][i], w.o[d][i + 1], w.o[d][i + 2], w.o[d][i + 3]};
      put_outputs<T>(a, r0 + w.qi, w.qhd, part, 32 * d + acc_row(i) + 4 * h, w.m, w.l, v);
    }
}

// Merges a row's parts, four dims of one row and head a thread.  SG threads
// share an item, each taking every SG-th part, and join in LDS: the order does
// not depend on timing.  Bound by two loads that depend on each other (the
// batch's tables, then the parts) and its launch: 4 to 7 us.
template <typename T, int SG>
__global__ void __launch_bounds__(256) k_attention_shared_merge(SharedArgs a, int blocks) {
  __shared__ float s_part[SG > 1 ? 256 : 1][6];
  const int s = blockIdx.x / blocks;
  Seq q;
  int pages;
  if (!batch_seq(a.b, s, q) || !shared_pages(a, s, q, pages)) return;
  const int chunks = a.hd / 4, per = 256 / (chunks * SG), tid = threadIdx.x;
  const int item = blockIdx.x % blocks * per + tid / (chunks * SG), group = tid / chunks % SG, dim = tid % chunks * 4;
  const bool valid = item < q.n * a.H;
  const int head = valid ? item % a.H : 0, row = q.r0 + (valid ? item / a.H : 0);
  const int own = (q.C + q.n + kPage - 1) / kPage - pages;
  const int c0 = part_pages(pages, a.shared_splits), c1 = part_pages(own, a.own_splits);
  const int n0 = (pages + c0 - 1) / c0, n = n0 + (own + c1 - 1) / c1;
  const size_t stride = (size_t)a.b.n_rows * a.H, at = (size_t)row * a.H + head;
  constexpr int kFlight = 8;  // parts on their way at once
  float m = -INFINITY, l = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int i0 = group; i0 < n; i0 += kFlight * SG) {
    float2 ml[kFlight];
    float4 o[kFlight];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const int i = min(i0 + j * SG, n - 1);
      const size_t k = (i < n0 ? i : a.shared_splits + i - n0) * stride + at;
      ml[j] = *reinterpret_cast<const float2*>(a.ml_part + k * 2);
      o[j] = *reinterpret_cast<const float4*>(a.o_part + k * a.hd + dim);
    }
    float m_new = m;
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      if (i0 + j * SG >= n) ml[j] = make_float2(-INFINITY, 0.f);
      m_new = fmaxf(m_new, ml[j].x);
    }
    const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= alpha;
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      if (ml[j].x == -INFINITY && ml[j].y == 0.f) continue;  // nothing seen there (or no part)
      const float f = __builtin_amdgcn_exp2f(ml[j].x - m);
      l += ml[j].y * f;
      v[0] += o[j].x * f; v[1] += o[j].y * f; v[2] += o[j].z * f; v[3] += o[j].w * f;
    }
  }
  if constexpr (SG > 1) {
    float* p = s_part[tid];
    p[0] = m; p[1] = l; p[2] = v[0]; p[3] = v[1]; p[4] = v[2]; p[5] = v[3];
    __syncthreads();
    if (group) return;
    const float* x = s_part[tid];  // the groups' shares are `chunks` threads apart
#pragma unroll
    for (int j = 1; j < SG; ++j) m = fmaxf(m, x[j * chunks * 6]);
    l = v[0] = v[1] = v[2] = v[3] = 0.f;
#pragma unroll
    for (int j = 0; j < SG; ++j) {
      const float* y = x + j * chunks * 6;
      if (y[0] == -INFINITY && y[1] == 0.f) continue;
      const float f = __builtin_amdgcn_exp2f(y[0] - m);
      l += y[1] * f;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += y[2 + e] * f;
    }
  }
  if (!valid) return;
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = inv == 0.f ? 0.f : v[e] * inv;
  act_store4(reinterpret_cast<T*>(a.out) + act_offset(row, head * a.hd + dim, a.H * a.hd), a.out_plane, v);
}

// ---- launch --------------------------------------------------------------------------
// Up to kFewTiles tiles of queries have a workgroup each, whose waves split
// its pages and join in LDS; more of them go four to a workgroup, one a wave,
// which read a page once for all (7b heads, 128 shared pages: 64 sequences of
// 2 rows, 28 tiles, 52 us and 57; of 4 rows, 56 tiles, 84 and 66).
// Parts of kChunk pages or more, as many as give two workgroups a compute
// unit (64 sequences of one row: 37 us, with twice as many parts 46); how many
// pages there are to split is known on the device, and the host's bounds stand
// for it here.  Where the sequences' own pages alone take those places, shared
// pages are split all the same, into as many as give one workgroup a compute
// unit, or two by parts of 32 pages and more (16 with four tiles a workgroup):
// the sequences' own parts, which come last, then start later, which costs
// less than long parts do (128 shared pages: 64 sequences of 8 rows 275 us with
// one part, 98; 8 of 64 rows 273 and 96).
void shared_plan(SharedArgs& a) {
  const int grp = a.H / a.G;
  auto tiles = [&](int64_t rows) { return (int)((rows * grp + 31) / 32); };
  const bool prefix = a.n_groups > 0 && a.max_pages > 0 && a.max_group_rows > 0;
  const int ts = prefix ? tiles(a.max_group_rows) : 0, to = tiles(a.b.max_rows);
  a.shared_few = ts <= kFewTiles;
  a.own_few = to <= kFewTiles;
  a.shared_groups = a.shared_few ? std::max(ts, 1) : (ts + 3) / 4;
  a.own_groups = a.own_few ? to : (to + 3) / 4;
  const int shared = prefix ? a.max_pages : 0, all = (a.b.max_ctx + kPage - 1) / kPage;
  const int64_t base_s = prefix ? (int64_t)a.n_groups * a.G * a.shared_groups : 0;
  const int64_t base_o = (int64_t)a.b.n_seqs * a.G * a.own_groups;
  const int own = std::max(all - shared, 1);
  auto parts = [](int pages, int chunk) { return (pages + chunk - 1) / chunk; };
  auto longer = [](int chunk) { return chunk + std::max(chunk / 8, 4) / 4 * 4; };
  const int least = std::max(kChunk, (std::max(shared, all) + 63) / 64);
  int chunk = least;
  while (chunk < std::max(shared, own) && base_s * parts(shared, chunk) + base_o * parts(own, chunk) > kWorkgroups)
    chunk = longer(chunk);
  int chunk_s = least;
  const int enough = a.shared_few ? 32 : 16;
  while (chunk_s < chunk && base_s * parts(shared, chunk_s) > (chunk_s < enough ? kWorkgroups / 2 : kWorkgroups))
    chunk_s = longer(chunk_s);
  a.shared_splits = prefix ? parts(shared, chunk_s) : 0;
  a.own_splits = parts(own, chunk);
  a.parts = a.shared_splits + a.own_splits;
  a.shared_jobs64 = base_s * a.shared_splits;
  a.own_jobs64 = base_o * a.own_splits;
}

template <typename T> static hipError_t shared_type(const SharedArgs& a, hipStream_t st) {
  const unsigned jobs = (unsigned)(a.shared_jobs64 + a.own_jobs64);
  if (a.hd == 32) k_attention_shared<T, 32><<<jobs, 256, 0, st>>>(a);
  else if (a.hd == 64) k_attention_shared<T, 64><<<jobs, 256, 0, st>>>(a);
  else k_attention_shared<T, 128><<<jobs, 256, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  const bool many = a.parts > 16;
  const int per = 256 / (a.hd / 4 * (many ? 4 : 1)), blocks = (a.b.max_rows * a.H + per - 1) / per;
  if (many) k_attention_shared_merge<T, 4><<<(unsigned)(a.b.n_seqs * blocks), 256, 0, st>>>(a, blocks);
  else k_attention_shared_merge<T, 1><<<(unsigned)(a.b.n_seqs * blocks), 256, 0, st>>>(a, blocks);
  return hipGetLastError();
}
hipError_t launch_attention_shared(int dtype, SharedArgs& a, hipStream_t st) {
  a.shared_jobs = (int)a.shared_jobs64;
  return dtype == 0 ? shared_type<float>(a, st) : shared_type<bf16_t>(a, st);
}

}  // namespace jf
