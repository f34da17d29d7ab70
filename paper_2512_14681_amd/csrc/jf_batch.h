// A batch of sequences over one paged cache, on the device: whose rows are
// whose, and where their pages are.
#pragma once

#include "jf_device.h"
#include "jf_internal.h"

namespace jf {

// One sequence of the batch: its rows are r0 .. r0 + n - 1 of the row
// tensors, row r0 + i at slot C + i.
struct Seq {
  int r0, n, C;
  const int32_t* table;   // its pages
};

// False if sequence s has no rows, or (with JF_FLAG_CAPACITY raised) if what
// the device holds about it does not fit what the host announced: no address
// is formed from it then.
__device__ __forceinline__ bool batch_seq(const BatchArgs& b, int s, Seq& q) {
  const int r0 = b.row_start[s], r1 = b.row_start[s + 1], C = b.ctx[s];
  const bool ok = r0 >= 0 && r1 >= r0 && r1 <= b.n_rows && r1 - r0 <= b.max_rows && C >= 0 &&
                  C <= b.max_ctx - (r1 - r0);
  if (!ok && b.flags && threadIdx.x == 0) atomicOr(b.flags, kFlagCapacity);
  q = Seq{r0, r1 - r0, C, b.table + (size_t)s * b.stride};
  return ok && r1 > r0;
}

// A page table entry's page; -1 (with JF_FLAG_BAD_PAGE raised) if it names
// none of the pool's.
__device__ __forceinline__ int batch_page_id(const BatchArgs& b, int id) {
  if ((unsigned)id < (unsigned)b.n_pages) return id;
  if (b.flags) atomicOr(b.flags, kFlagBadPage);
  return -1;
}
__device__ __forceinline__ int batch_page(const BatchArgs& b, const Seq& q, int p) { return batch_page_id(b, q.table[p]); }

// ---- what a row sees ---------------------------------------------------------------
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

// ---- 8-bit pages ------------------------------------------------------------------
// Codes of the keys [G][64 hd], of the values [G][64 hd], then the scales
// [G][2] (key, value; powers of two), padded to 128 bytes.  A head's 64 hd
// codes are hd / 16 pieces of 64 lanes x 16 bytes, so that one load of a wave
// is one contiguous 1 KB and arrives as matrix-core operands:
//   key t, dim i:    lane t % 16 + 16 (i / (hd / 4)), byte (t / 16) (hd / 4) + i % (hd / 4)
//   value t, dim i:  lane i % 16 + 16 ((t / 4) % 4),  byte 16 (i / 16) + 4 (t / 16) + t % 4
// with byte b of a lane at piece b / 16.  A lane's 16 value bytes are the
// keys that the same lane's scores belong to (jf_attention_kv8).
__host__ __device__ inline size_t kv8_page_bytes(int G, int hd) {
  return ((size_t)2 * G * kPage * hd + (size_t)8 * G + 127) / 128 * 128;
}
__device__ __forceinline__ int kv8_key_offset(int t, int i, int hd) {
  const int w = hd / 4, b = (t >> 4) * w + i % w;
  return (b >> 4) * 1024 + ((t & 15) + 16 * (i / w)) * 16 + (b & 15);
}
__device__ __forceinline__ int kv8_value_offset(int t, int i) {
  return (i >> 4) * 1024 + ((i & 15) + 16 * ((t >> 2) & 3)) * 16 + 4 * (t >> 4) + (t & 3);
}

constexpr float kF8Max = 448.f;

// Four values (already divided by the scale) as e4m3 codes: round to nearest,
// ties to even, saturating; NaN stays NaN.  (The conversion itself turns what
// is above the largest value into NaN.)
__device__ __forceinline__ float f8_clamp(float x) {
  const float c = fminf(fmaxf(x, -kF8Max), kF8Max);
  return x != x ? x : c;
}
__device__ __forceinline__ uint32_t f8_pack4(float a, float b, float c, float d) {
  uint32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(f8_clamp(a), f8_clamp(b), 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(f8_clamp(c), f8_clamp(d), w, true);
}
__device__ __forceinline__ void f8_unpack4(uint32_t w, float (&v)[4]) {
  const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
}

// The smallest power of two 2^k with amax <= 448 2^k (1 for amax = 0), from
// the significands: a division's rounding could move amax across the border.
__device__ __forceinline__ float f8_block_scale(float amax) {
  if (!(amax > 0.f)) return 1.f;
  int e;
  const float m = frexpf(amax, &e);             // amax = m 2^e, m in [0.5, 1)
  const int k = m > 0.875f ? e - 8 : e - 9;     // 448 = 0.875 2^9
  return ldexpf(1.f, max(k, -100));             // scales stay far from the denormals
}

// Four consecutive elements; vec: the address is aligned to all four.
template <typename T> __device__ __forceinline__ void load4(const T* p, bool vec, float (&v)[4]);
template <> __device__ __forceinline__ void load4<float>(const float* p, bool vec, float (&v)[4]) {
  if (vec) {
    const float4 x = *reinterpret_cast<const float4*>(p);
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = p[i];
  }
}
template <> __device__ __forceinline__ void load4<bf16_t>(const bf16_t* p, bool vec, float (&v)[4]) {
  if (vec) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(x.x << 16); v[1] = __uint_as_float(x.x & 0xFFFF0000u);
    v[2] = __uint_as_float(x.y << 16); v[3] = __uint_as_float(x.y & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = bf16_to_f32(p[i]);
  }
}

}  // namespace jf
