// Keys and values of a batch of sequences: appended to a paged cache with the
// position rotation applied on the way (jf_kv_append), and read back
// (jf_kv_read).
//
// Rotation: dims i and i + hd / 2 of a head turn by pos * base^(-2 i / hd).
// The angle is a number of turns in 64 bits, of which only the fraction is
// kept, so that far positions lose nothing.
//
// A workgroup takes one head of one page: it alone writes that head's codes
// and scale there, so the scale needs no other workgroup.  The queries'
// rotation runs in further workgroups of the same launch.
//
// Both are bound by memory for many rows and by three dependent loads (the
// sequence, its page table entry, the page) for few.  Append: 14458 rows of 16
// + 2 x 4 heads of 128 dims in fp32 to an e4m3 cache 67 us, 310 MB at 4.7
// TB/s; one row 4.7 us, 64 sequences of one row 10.1 us.  Read: the 14458 rows
// to bf16 14.6 us, 44 MB at 3.0 TB/s; the last pages of 64 sequences 6.5 us.
#include <algorithm>

#include "jf_batch.h"

namespace jf {

// Sine and cosine of x turns: Taylor polynomials on an eighth of a turn to
// either side of the nearest quarter, 1.2e-10 off at most, about 25
// instructions at the rate of 32 bits.  The queries take them rounded to fp32.
// The keys are turned in 64 bits, as every error before the rounding to e4m3
// sends some of them to its other side, for half a microsecond of 64.
template <typename R> __device__ __forceinline__ void sincos_turns(double x, R& sn, R& cs) {
  const double y = 4.0 * (x - rint(x)), n = rint(y), r = (y - n) * 1.5707963267948966, z = r * r;
  const double ps = 1.0 / 362880 - z * (1.0 / 39916800), pc = 1.0 / 40320 - z * (1.0 / 3628800);
  const R s = (R)(r + r * z * (-1.0 / 6 + z * (1.0 / 120 + z * (-1.0 / 5040 + z * ps))));
  const R c = (R)(1.0 + z * (-0.5 + z * (1.0 / 24 + z * (-1.0 / 720 + z * pc))));
  const int k = (int)n;  // -2 .. 2
  const R u = k & 1 ? c : s, v = k & 1 ? s : c;
  sn = k & 2 ? -u : u;
  cs = (k + 1) & 2 ? -v : v;
}

// Sine and cosine of four consecutive pairs at a position.
template <typename R>
__device__ __forceinline__ void angles4(const double* freq, int i, int pos, R (&cs)[4], R (&sn)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) sincos_turns<R>((double)pos * freq[i + e], sn[e], cs[e]);
}

template <typename T> __device__ __forceinline__ void store4(T* p, const float (&v)[4]);
template <> __device__ __forceinline__ void store4<float>(float* p, const float (&v)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
template <> __device__ __forceinline__ void store4<bf16_t>(bf16_t* p, const float (&v)[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

constexpr int kQHeads = 4;  // heads that share a thread's sines and cosines

// The queries: a thread rotates four pairs of up to kQHeads heads of a row.
template <typename X, typename A, int HD>
__device__ __forceinline__ void append_queries(const AppendArgs& a, const Seq& q, int block) {
  constexpr int kChunks = HD / 8;
  const int hb = (a.H + kQHeads - 1) / kQHeads;
  const int item = block * 256 + threadIdx.x;
  const int c = item % kChunks, h0 = item / kChunks % hb * kQHeads, i = item / kChunks / hb;
  if (i >= q.n) return;
  const int row = q.r0 + i;
  const int pos = a.pos ? a.pos[row] : q.C + i;
  const X* x = reinterpret_cast<const X*>(a.q) + (size_t)row * a.ld_q;
  A* out = reinterpret_cast<A*>(a.q_out) + (size_t)row * a.H * HD;
  // all loads before the first store, which they could not pass
  float u[kQHeads][4], w[kQHeads][4];
#pragma unroll
  for (int hh = 0; hh < kQHeads; ++hh) {
    const int h = min(h0 + hh, a.H - 1);
    load4(x + (size_t)h * HD + 4 * c, a.vec_q, u[hh]);
    load4(x + (size_t)h * HD + HD / 2 + 4 * c, a.vec_q, w[hh]);
  }
  float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
  if (a.rotate) angles4(a.freq, 4 * c, pos, cs, sn);
#pragma unroll
  for (int hh = 0; hh < kQHeads; ++hh) {
    const int h = h0 + hh;
    if (h >= a.H) break;
    float y[4], z[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] = a.rotate ? u[hh][e] * cs[e] - w[hh][e] * sn[e] : u[hh][e];
      z[e] = a.rotate ? w[hh][e] * cs[e] + u[hh][e] * sn[e] : w[hh][e];
    }
    act_store4(out + (size_t)h * HD + 4 * c, a.q_plane, y);
    act_store4(out + (size_t)h * HD + HD / 2 + 4 * c, a.q_plane, z);
  }
}

template <int HD, typename T> struct AppendShared { alignas(16) T v[HD][kPage + 16 / sizeof(T)]; };   // values transposed
template <int HD> struct AppendShared<HD, uint8_t> {
  alignas(16) uint32_t code[2][16 * HD];  // a head's key and value codes in the page's order
  float amax[2][4];
};

// A turned key in 32 bits: the nearest value, but for codes the neighbour with
// an odd last bit where bits were lost, so that the second rounding, to e4m3,
// is that of the 64-bit value (a tie in 32 bits is one in 64).
template <typename KV> __device__ __forceinline__ float round_key(double y) {
  const float t = (float)y;
  if constexpr (sizeof(KV) == 1) {
    const double left = y - (double)t;
    const uint32_t b = __float_as_uint(t);
    if (left != 0.0 && !(b & 1) && t != 0.f && fabsf(t) < INFINITY)
      return __uint_as_float((left > 0.0) == (t > 0.f) ? b + 1 : b - 1);
  }
  return t;
}

// The tokens of a head's code word i of an e4m3 page: a key word is four dims
// of one token, a value word four tokens (this one and the next three) of a dim.
template <int HD> __device__ __forceinline__ int key_token(int i) {
  return ((i >> 8) * 16 + (i & 3) * 4) / (HD / 4) * 16 + ((i >> 2) & 15);
}
__device__ __forceinline__ int value_token(int i) { return (i & 3) * 16 + (i >> 6 & 3) * 4; }

// Whether a head's keys (w = 0) or values are 0 in every token below t0: such
// tokens got scale 1 for want of a value, and must not hold later ones to it.
template <int HD> __device__ __forceinline__ bool kept_zeros(const uint32_t* codes, int w, int t0) {
  uint32_t any = 0;
  for (int i = threadIdx.x; i < 16 * HD; i += 256) {
    const int n = w ? min(t0 - value_token(i), 4) : (key_token<HD>(i) < t0 ? 4 : 0);  // bytes of tokens below t0
    if (n > 0) any |= codes[i] & (0x7F7F7F7Fu >> (32 - 8 * n));
  }
  return !__syncthreads_or((int)any);
}

// KV: float, bf16_t (pages of jf_model_load) or uint8_t (e4m3 pages).
template <typename X, typename A, typename KV, int HD>
__global__ void __launch_bounds__(256) k_kv_append(AppendArgs a) {
  constexpr int kItems = HD / 32;  // a thread's items: four pairs of one token
  __shared__ AppendShared<HD, KV> sh;
  const int per = a.n_cache + a.n_q;
  const int s = blockIdx.x / per, it = blockIdx.x % per;
  Seq q;
  if (!batch_seq(a.b, s, q)) return;
  if (it >= a.n_cache) {
    append_queries<X, A, HD>(a, q, it - a.n_cache);
    return;
  }
  const int g = it % a.G, page = q.C / kPage + it / a.G;
  const int t0 = max(q.C - page * kPage, 0);                 // first new token of the page
  const int t1 = min(q.C + q.n - page * kPage, kPage);       // past the last one
  if (t1 <= t0) return;
  const int entry = q.table[page];                           // looked at when the rows are on their way
  const int tid = threadIdx.x;
  const int row0 = q.r0 + page * kPage - q.C;                // the row of the page's token 0

  // the new keys and values, in registers
  float x[kItems][2][8];
  float kmax = 0.f, vmax = 0.f;
#pragma unroll
  for (int n = 0; n < kItems; ++n) {
    const int item = n * 256 + tid, c = item % (HD / 8), t = item / (HD / 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[n][0][e] = x[n][1][e] = 0.f;
    if (t >= t0 && t < t1) {
      const int row = row0 + t;
      const X* kp = reinterpret_cast<const X*>(a.k) + (size_t)row * a.ld_k + (size_t)g * HD + 4 * c;
      const X* vp = reinterpret_cast<const X*>(a.v) + (size_t)row * a.ld_v + (size_t)g * HD + 4 * c;
      load4(kp, a.vec_k, reinterpret_cast<float(&)[4]>(x[n][0][0]));
      load4(kp + HD / 2, a.vec_k, reinterpret_cast<float(&)[4]>(x[n][0][4]));
      load4(vp, a.vec_v, reinterpret_cast<float(&)[4]>(x[n][1][0]));
      load4(vp + HD / 2, a.vec_v, reinterpret_cast<float(&)[4]>(x[n][1][4]));
    }
  }
  const int id = batch_page_id(a.b, entry);
  if (id < 0) return;
  if (a.rotate) {
#pragma unroll
    for (int n = 0; n < kItems; ++n) {
      const int item = n * 256 + tid, c = item % (HD / 8), t = item / (HD / 8);
      if (t < t0 || t >= t1) continue;
      const int row = row0 + t;
      double cs[4], sn[4];
      angles4(a.freq, 4 * c, a.pos ? a.pos[row] : q.C + row - q.r0, cs, sn);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float u = x[n][0][e], w = x[n][0][4 + e];
        x[n][0][e] = round_key<KV>((double)u * cs[e] - (double)w * sn[e]);
        x[n][0][4 + e] = round_key<KV>((double)w * cs[e] + (double)u * sn[e]);
      }
    }
  }
  char* base = reinterpret_cast<char*>(a.kv) + (size_t)id * a.page_bytes;

  if constexpr (sizeof(KV) > 1) {
    KV* kd = reinterpret_cast<KV*>(base) + (size_t)g * kPage * HD;
    KV* vd = reinterpret_cast<KV*>(base) + (size_t)(a.G + g) * kPage * HD;
#pragma unroll
    for (int n = 0; n < kItems; ++n) {
      const int item = n * 256 + tid, c = item % (HD / 8), t = item / (HD / 8);
      if (t < t0 || t >= t1) continue;
      store4<KV>(kd + (size_t)t * HD + 4 * c, {x[n][0][0], x[n][0][1], x[n][0][2], x[n][0][3]});
      store4<KV>(kd + (size_t)t * HD + HD / 2 + 4 * c, {x[n][0][4], x[n][0][5], x[n][0][6], x[n][0][7]});
#pragma unroll
      for (int e = 0; e < 8; ++e) sh.v[(e / 4) * (HD / 2) + 4 * c + e % 4][t] = from_f32<KV>(x[n][1][e]);
    }
    __syncthreads();
    // 16 bytes along the tokens of a dim where all of them are new
    constexpr int N = 16 / (int)sizeof(KV);
    for (int i = tid; i < HD * (kPage / N); i += 256) {
      const int d = i / (kPage / N), t = i % (kPage / N) * N;
      KV* p = vd + (size_t)d * kPage + t;
      if (t >= t0 && t + N <= t1) {
        *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&sh.v[d][t]);
      } else {
        for (int e = max(t0 - t, 0); e < min(t1 - t, N); ++e) p[e] = sh.v[d][t + e];
      }
    }
  } else {
    float* scales = reinterpret_cast<float*>(base + (size_t)2 * a.G * kPage * HD) + 2 * g;
    const float held[2] = {scales[0], scales[1]};
#pragma unroll
    for (int n = 0; n < kItems; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        // infinities saturate and NaN stays NaN: neither sets the scale
        const float ka = fabsf(x[n][0][e]), va = fabsf(x[n][1][e]);
        kmax = ka < INFINITY ? fmaxf(kmax, ka) : kmax;
        vmax = va < INFINITY ? fmaxf(vmax, va) : vmax;
      }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      kmax = fmaxf(kmax, __shfl_xor(kmax, d));
      vmax = fmaxf(vmax, __shfl_xor(vmax, d));
    }
    if ((tid & 63) == 0) {
      sh.amax[0][tid >> 6] = kmax;
      sh.amax[1][tid >> 6] = vmax;
    }
    __syncthreads();
    uint32_t* codes[2] = {reinterpret_cast<uint32_t*>(base + (size_t)g * kPage * HD),
                          reinterpret_cast<uint32_t*>(base + (size_t)(a.G + g) * kPage * HD)};
    int from[2];          // first token whose codes are written
    float inv[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float amax = fmaxf(fmaxf(sh.amax[w][0], sh.amax[w][1]), fmaxf(sh.amax[w][2], sh.amax[w][3]));
      const float need = f8_block_scale(amax);
      const bool keeps = t0 > 0 && !(held[w] == 1.f && need < 1.f && kept_zeros<HD>(codes[w], w, t0));
      const float old = keeps ? held[w] : need;
      const float sc = fmaxf(old, need);
      inv[w] = 1.f / sc;  // a power of two: exact
      from[w] = t0;
      if (sc > old) {     // the kept tokens' codes on the larger scale
        const float ratio = old * inv[w];
        for (int i = tid; i < 16 * HD; i += 256) {
          float v[4];
          f8_unpack4(codes[w][i], v);
          sh.code[w][i] = f8_pack4(v[0] * ratio, v[1] * ratio, v[2] * ratio, v[3] * ratio);
        }
        from[w] = 0;
      }
    }
    __syncthreads();      // scales read, kept codes staged
    if (tid == 0) {
      scales[0] = 1.f / inv[0];
      scales[1] = 1.f / inv[1];
    }
    uint8_t* kc = reinterpret_cast<uint8_t*>(sh.code[0]);
    uint8_t* vc = reinterpret_cast<uint8_t*>(sh.code[1]);
#pragma unroll
    for (int n = 0; n < kItems; ++n) {
      const int item = n * 256 + tid, c = item % (HD / 8), t = item / (HD / 8);
      if (t < t0 || t >= t1) continue;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const float* k4 = &x[n][0][4 * hf];
        const float* v4 = &x[n][1][4 * hf];
        const int i = hf * (HD / 2) + 4 * c;
        *reinterpret_cast<uint32_t*>(kc + kv8_key_offset(t, i, HD)) =
            f8_pack4(k4[0] * inv[0], k4[1] * inv[0], k4[2] * inv[0], k4[3] * inv[0]);
        const uint32_t w = f8_pack4(v4[0] * inv[1], v4[1] * inv[1], v4[2] * inv[1], v4[3] * inv[1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) vc[kv8_value_offset(t, i + e)] = (uint8_t)(w >> (8 * e));
      }
    }
    __syncthreads();
    if (from[0] == 0 && from[1] == 0 && t1 == kPage) {  // a whole page
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < HD / 64; ++i)
          reinterpret_cast<uint4*>(codes[w])[i * 256 + tid] = reinterpret_cast<const uint4*>(sh.code[w])[i * 256 + tid];
      if constexpr (HD < 64)
        if (tid < 128)
#pragma unroll
          for (int w = 0; w < 2; ++w)
            reinterpret_cast<uint4*>(codes[w])[tid] = reinterpret_cast<const uint4*>(sh.code[w])[tid];
      return;
    }
    // Words of four dims of one token (keys), of four tokens of one dim
    // (values); only the tokens written change.
    for (int i = tid; i < 16 * HD; i += 256) {
      const int tk = key_token<HD>(i), tv = value_token(i);
      if (tk >= from[0] && tk < t1) codes[0][i] = sh.code[0][i];
      if (tv >= from[1] && tv + 4 <= t1) {
        codes[1][i] = sh.code[1][i];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (tv + e >= from[1] && tv + e < t1)
            reinterpret_cast<uint8_t*>(codes[1] + i)[e] = (uint8_t)(sh.code[1][i] >> (8 * e));
      }
    }
  }
}

// ---- reading back --------------------------------------------------------------------
template <typename X> __device__ __forceinline__ void put4(X* p, bool vec, const float (&v)[4]) {
  if (vec) {
    store4<X>(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = from_f32<X>(v[e]);
  }
}

// Eight values of a row in one store (two for fp32).
typedef uint32_t u32x4_part_t __attribute__((ext_vector_type(4), aligned(8)));
__device__ __forceinline__ void put8(float* p, bool vec, const float (&v)[8]) {
  put4(p, vec, {v[0], v[1], v[2], v[3]});
  put4(p + 4, vec, {v[4], v[5], v[6], v[7]});
}
__device__ __forceinline__ void put8(bf16_t* p, bool vec, const float (&v)[8]) {
  if (vec) {
    *reinterpret_cast<u32x4_part_t*>(p) = u32x4_part_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                       pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = from_f32<bf16_t>(v[e]);
  }
}

// The head's codes of an e4m3 page.  A lane's 16 bytes of the keys are 16 dims
// of one token (head_dim 32: 8 dims of two) and go straight to its row; those
// of the values are 16 tokens of one dim and pass through LDS, where the low
// bits of a slot are turned by the piece so that the dims of a token lie in
// different banks (14458 rows to bf16 14.6 us; byte by byte, in the page's own order, 20.8).
template <typename X, int HD>
__device__ __forceinline__ void read_codes(const ReadArgs& a, const char* base, int g, int row0, int t0, int t1,
                                           uint4* sh) {
  constexpr int kEach = (4 * HD + 255) / 256, W = HD / 4, kRun = W < 16 ? W : 16;
  const int tid = threadIdx.x;
  const uint4* kp = reinterpret_cast<const uint4*>(base + (size_t)g * kPage * HD);
  const uint4* vp = reinterpret_cast<const uint4*>(base + (size_t)(a.G + g) * kPage * HD);
  uint4 r[2][kEach];
#pragma unroll
  for (int n = 0; n < kEach; ++n)
    if (n * 256 + tid < 4 * HD) {
      r[0][n] = kp[n * 256 + tid];
      r[1][n] = vp[n * 256 + tid];
    }
  const float2 scale = reinterpret_cast<const float2*>(base + (size_t)2 * a.G * kPage * HD)[g];
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int i = n * 256 + tid, piece = i >> 6, l = i & 63;
    if (i >= 4 * HD) break;
    sh[(piece << 6) + (l ^ (piece & 3))] = r[1][n];
    const uint32_t w[4] = {r[0][n].x, r[0][n].y, r[0][n].z, r[0][n].w};
#pragma unroll
    for (int b = 0; b < 16; b += 8) {
      const int at = piece * 16 + b / kRun * kRun, t = at / W * 16 + (l & 15), d = (l >> 4) * W + at % W + b % kRun;
      if (t < t0 || t >= t1) continue;
      float lo[4], hi[4];
      f8_unpack4(w[b / 4], lo);
      f8_unpack4(w[b / 4 + 1], hi);
      put8(reinterpret_cast<X*>(a.k) + (size_t)(row0 + t) * a.ld_k + (size_t)g * HD + d, a.vec_k,
           {lo[0] * scale.x, lo[1] * scale.x, lo[2] * scale.x, lo[3] * scale.x,
            hi[0] * scale.x, hi[1] * scale.x, hi[2] * scale.x, hi[3] * scale.x});
    }
  }
  __syncthreads();
  // four dims (c) of four tokens: 16 j + 4 kg + m
#pragma unroll
  for (int n = 0; n < kEach; ++n) {
    const int i = n * 256 + tid, c = i % W, j = i / W % 4, kg = i / W / 4;
    if (i >= 4 * HD) break;
    const int t = 16 * j + 4 * kg;
    if (t + 3 < t0 || t >= t1) continue;
    float v[4][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int piece = c >> 2, l = 4 * (c & 3) + e + 16 * kg;
      f8_unpack4(reinterpret_cast<const uint32_t*>(sh + (piece << 6) + (l ^ (piece & 3)))[j], v[e]);
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
      if (t + m >= t0 && t + m < t1)
        put4(reinterpret_cast<X*>(a.v) + (size_t)(row0 + t + m) * a.ld_v + (size_t)g * HD + 4 * c, a.vec_v,
             {v[0][m] * scale.y, v[1][m] * scale.y, v[2][m] * scale.y, v[3][m] * scale.y});
  }
}

// A workgroup: one head of one page.  KV as above; X: float or bf16_t rows.
// The values, transposed in the page, pass through LDS.
template <typename X, typename KV, int HD>
__global__ void __launch_bounds__(256) k_kv_read(ReadArgs a) {
  constexpr int N = 16 / (int)sizeof(KV);                 // elements of 16 bytes
  constexpr int kRow = kPage + N;                         // a dim's tokens in LDS
  __shared__ alignas(16) KV sh[sizeof(KV) > 1 ? HD * kRow : HD * kPage];
  const int per = a.pages * a.G;
  const int s = blockIdx.x / per, it = blockIdx.x % per;
  Seq q;
  if (!batch_seq(a.b, s, q)) return;
  const int g = it % a.G, page = q.C / kPage + it / a.G;
  const int t0 = max(q.C - page * kPage, 0), t1 = min(q.C + q.n - page * kPage, kPage);
  if (t1 <= t0) return;
  const int id = batch_page(a.b, q, page);
  if (id < 0) return;
  const int tid = threadIdx.x;
  const int row0 = q.r0 + page * kPage - q.C;
  const char* base = reinterpret_cast<const char*>(a.kv) + (size_t)id * a.page_bytes;
  if constexpr (sizeof(KV) == 1) {
    read_codes<X, HD>(a, base, g, row0, t0, t1, reinterpret_cast<uint4*>(sh));
  } else {
    const KV* kp = reinterpret_cast<const KV*>(base) + (size_t)g * kPage * HD;
    const KV* vp = reinterpret_cast<const KV*>(base) + (size_t)(a.G + g) * kPage * HD;
#pragma unroll 4
    for (int i = tid; i < HD * (kPage / N); i += 256) {
      const int d = i / (kPage / N), t = i % (kPage / N) * N;
      if (t < t1 && t + N > t0)
        *reinterpret_cast<uint4*>(sh + d * kRow + t) = *reinterpret_cast<const uint4*>(vp + (size_t)d * kPage + t);
    }
    __syncthreads();
    for (int i = tid; i < (t1 - t0) * (HD / 4); i += 256) {
      const int t = t0 + i / (HD / 4), d = i % (HD / 4) * 4;
      float k[4], v[4];
      load4(kp + (size_t)t * HD + d, true, k);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = to_f32<KV>(sh[(d + e) * kRow + t]);
      put4(reinterpret_cast<X*>(a.k) + (size_t)(row0 + t) * a.ld_k + (size_t)g * HD + d, a.vec_k, k);
      put4(reinterpret_cast<X*>(a.v) + (size_t)(row0 + t) * a.ld_v + (size_t)g * HD + d, a.vec_v, v);
    }
  }
}

// ---- launches ------------------------------------------------------------------------
// Pages that n consecutive slots can touch.
static int pages_of(int n) { return (int)(((int64_t)n + kPage - 2) / kPage) + 1; }

template <typename X, typename A, typename KV>
static hipError_t append_hd(const AppendArgs& a, unsigned grid, hipStream_t st) {
  if (a.hd == 32) k_kv_append<X, A, KV, 32><<<grid, 256, 0, st>>>(a);
  else if (a.hd == 64) k_kv_append<X, A, KV, 64><<<grid, 256, 0, st>>>(a);
  else k_kv_append<X, A, KV, 128><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}
template <typename X, typename A>
static hipError_t append_kv(int kv, const AppendArgs& a, unsigned grid, hipStream_t st) {
  if (kv == 0) return append_hd<X, A, float>(a, grid, st);
  if (kv == 1) return append_hd<X, A, bf16_t>(a, grid, st);
  return append_hd<X, A, uint8_t>(a, grid, st);
}
hipError_t launch_kv_append(int kv, int x, int act, AppendArgs& a, hipStream_t st) {
  a.n_cache = pages_of(a.b.max_rows) * a.G;
  a.n_q = a.q ? (int)(((int64_t)a.b.max_rows * ((a.H + kQHeads - 1) / kQHeads) * (a.hd / 8) + 255) / 256) : 0;
  const unsigned n = (unsigned)(a.b.n_seqs * (a.n_cache + a.n_q));
  if (x == 0) return act == 0 ? append_kv<float, float>(kv, a, n, st) : append_kv<float, bf16_t>(kv, a, n, st);
  return act == 0 ? append_kv<bf16_t, float>(kv, a, n, st) : append_kv<bf16_t, bf16_t>(kv, a, n, st);
}

template <typename X, typename KV> static hipError_t read_hd(const ReadArgs& a, unsigned grid, hipStream_t st) {
  if (a.hd == 32) k_kv_read<X, KV, 32><<<grid, 256, 0, st>>>(a);
  else if (a.hd == 64) k_kv_read<X, KV, 64><<<grid, 256, 0, st>>>(a);
  else k_kv_read<X, KV, 128><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}
template <typename X> static hipError_t read_kv(int kv, const ReadArgs& a, unsigned grid, hipStream_t st) {
  if (kv == 0) return read_hd<X, float>(a, grid, st);
  if (kv == 1) return read_hd<X, bf16_t>(a, grid, st);
  return read_hd<X, uint8_t>(a, grid, st);
}
hipError_t launch_kv_read(int kv, int x, ReadArgs& a, hipStream_t st) {
  a.pages = pages_of(a.b.max_rows);
  const unsigned n = (unsigned)(a.b.n_seqs * a.pages * a.G);
  return x == 0 ? read_kv<float>(kv, a, n, st) : read_kv<bf16_t>(kv, a, n, st);
}

}  // namespace jf
