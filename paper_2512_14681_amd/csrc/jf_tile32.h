// 32 x 32 matrix-core tiles whose operands come from row-major tiles in LDS:
// the attention over packed rows and over shared prefixes.
//
// A tile's contraction runs in steps of 16: lane l gives row (or column)
// l % 32 and elements 8 (l / 32) .. + 7 of the step.  In the result lane l
// holds column l % 32 of rows 8 (i / 4) + 4 (l / 32) + i % 4, i < 16.
#pragma once

#include "jf_device.h"

namespace jf {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

// fp32: eight instructions of two elements each (element e of both halves).
__device__ __forceinline__ void mfma32(f32x16_t& acc, const Frag<bf16_t>& a, const Frag<bf16_t>& b) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a.v), __builtin_bit_cast(bf16x8_t, b.v),
                                                acc, 0, 0, 0);
}
__device__ __forceinline__ void mfma32(f32x16_t& acc, const Frag<float>& a, const Frag<float>& b) {
  const float x[8] = {a.lo.x, a.lo.y, a.lo.z, a.lo.w, a.hi.x, a.hi.y, a.hi.z, a.hi.w};
  const float y[8] = {b.lo.x, b.lo.y, b.lo.z, b.lo.w, b.hi.x, b.hi.y, b.hi.z, b.hi.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
// Row of element i in a result, without the 4 (l / 32) of the lane.
__device__ __forceinline__ constexpr int acc_row(int i) { return 8 * (i / 4) + i % 4; }

// Eight values as an operand.
__device__ __forceinline__ void frag_of(const float* x, Frag<bf16_t>& f) {
  f.v = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ void frag_of(const float* x, Frag<float>& f) {
  f.lo = make_float4(x[0], x[1], x[2], x[3]);
  f.hi = make_float4(x[4], x[5], x[6], x[7]);
}

// The values of an operand.
__device__ __forceinline__ void frag_values(const Frag<bf16_t>& f, float (&x)[8]) {
  const uint32_t w[4] = {f.v.x, f.v.y, f.v.z, f.v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void frag_values(const Frag<float>& f, float (&x)[8]) {
  x[0] = f.lo.x; x[1] = f.lo.y; x[2] = f.lo.z; x[3] = f.lo.w;
  x[4] = f.hi.x; x[5] = f.hi.y; x[6] = f.hi.z; x[7] = f.hi.w;
}

// Maximum over, and sum over, the two lanes that hold one column.
__device__ __forceinline__ float pair_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float pair_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// A tile of rows in LDS, kRowBytes each, in 16-byte chunks: chunk c of row r
// lies at place c ^ turn(r) of its row.  16 rows' chunks of one column, and
// four rows' runs of four chunks, then fill the 64 banks (with turns that
// tell apart 8 rows only, half of the cycles of LDS reads were conflicts).
template <int kRowBytes> __device__ __forceinline__ constexpr int turn(int r) {
  return kRowBytes >= 256   ? ((r & 3) << 2) | ((r >> 2) & 3)
         : kRowBytes == 128 ? ((r & 2) << 1) | ((r >> 2) & 3)
                            : (r >> 2) & 3;
}

typedef __attribute__((address_space(3))) char lds_char_t;
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(lds_char_t*)reinterpret_cast<char*>(const_cast<void*>(p));
}

// Operand reads from a row-major tile [rows][HD] of T.  `base` is the tile's
// LDS address (a multiple of 1024) plus the lane's part of the place, for all
// reads of a tile the same: what else there is to it are constants, exclusive
// or'ed where chunks are turned, and few registers hold addresses.
template <typename T, int HD> struct RowTile {
  static constexpr int kRowBytes = HD * (int)sizeof(T);
  static_assert(kRowBytes >= 64, "a row holds four chunks or more");
  template <typename V> static __device__ __forceinline__ V at(uint32_t address) {
    return *reinterpret_cast<__attribute__((address_space(3))) V*>((uintptr_t)address);
  }

  // Rows r0 + l % 32 (r0 a multiple of 16), dims 16 s + 8 (l / 32) .. + 7.
  static __device__ __forceinline__ uint32_t row_base(uint32_t tile) {
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    return tile + r * kRowBytes + (((sizeof(T) == 2 ? h : 2 * h) ^ turn<kRowBytes>(r)) << 4);
  }
  static __device__ __forceinline__ Frag<T> rows(uint32_t base, int r0, int s) {
    if constexpr (sizeof(T) == 2) {
      return Frag<T>{__builtin_bit_cast(uint4, at<u32x4_t>((base ^ (s << 5)) + r0 * kRowBytes))};
    } else {
      return Frag<T>{__builtin_bit_cast(float4, at<f32x4v_t>((base ^ (s << 6)) + r0 * kRowBytes)),
                     __builtin_bit_cast(float4, at<f32x4v_t>((base ^ (s << 6 | 16)) + r0 * kRowBytes))};
    }
  }
  // The transposed tile: dims 32 t + l % 32, of the 16 tile rows from r0 (a
  // multiple of 16) those that a result's elements 0 .. 7 stand for:
  // r0 + 8 (e / 4) + 4 (l / 32) + e % 4.  bf16: a group of 16 lanes reads 4
  // rows of 16 dims, and each lane gets its dim of the 4 rows.
  static __device__ __forceinline__ uint32_t column_base(uint32_t tile) {
    const int lane = threadIdx.x & 63, h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      const int i = lane & 15, r = 4 * h + (i >> 2), c = ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
      return tile + r * kRowBytes + ((c ^ turn<kRowBytes>(r)) << 4) + (i & 1) * 8;
    } else {
      const int d = lane & 31;
      return tile + 4 * h * kRowBytes + (((d >> 2) ^ turn<kRowBytes>(4 * h)) << 4) + (d & 3) * 4;
    }
  }
  static __device__ __forceinline__ Frag<T> columns(uint32_t base, int r0, int t) {
    if constexpr (sizeof(T) == 2) {
      typedef short s16x4_t __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
      auto read = [&](int row) {  // 8 more rows turn the chunks by 2 more
        const uint32_t a = (base ^ (t << 6) ^ (turn<kRowBytes>(row) << 4)) + (r0 + row) * kRowBytes;
        return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(uintptr_t)a));
      };
      const uint2 a = read(0), b = read(8);
      return Frag<T>{make_uint4(a.x, a.y, b.x, b.y)};
    } else {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int r = 8 * (e / 4) + e % 4;
        x[e] = at<float>((base ^ (t << 7) ^ (turn<kRowBytes>(r) << 4)) + (r0 + r) * kRowBytes);
      }
      return Frag<T>{make_float4(x[0], x[1], x[2], x[3]), make_float4(x[4], x[5], x[6], x[7])};
    }
  }
};

// Largest magnitude bits of an operand's elements, kept over several
// operands (pairs of bf16, or one fp32), and whether they were all finite.
__device__ __forceinline__ void magnitude(const Frag<bf16_t>& f, uint32_t& top) {
  const uint32_t w[4] = {f.v.x, f.v.y, f.v.z, f.v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
    top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, top),
                                                                 __builtin_bit_cast(u16x2_t, w[i] & 0x7FFF7FFFu)));
  }
}
__device__ __forceinline__ void magnitude(const Frag<float>& f, uint32_t& top) {
  const float x[8] = {f.lo.x, f.lo.y, f.lo.z, f.lo.w, f.hi.x, f.hi.y, f.hi.z, f.hi.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
}
template <typename T> __device__ __forceinline__ bool all_finite(uint32_t top);
template <> __device__ __forceinline__ bool all_finite<bf16_t>(uint32_t top) {
  return (top & 0xFFFFu) < 0x7F80u && (top >> 16) < 0x7F80u;
}
template <> __device__ __forceinline__ bool all_finite<float>(uint32_t top) { return top < 0x7F800000u; }

// An operand with its infinities and NaN as 0.
__device__ __forceinline__ void keep_finite(Frag<bf16_t>& f) {
  uint32_t w[4] = {f.v.x, f.v.y, f.v.z, f.v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = (w[i] & 0x7F80u) == 0x7F80u ? w[i] & 0xFFFF0000u : w[i];
    w[i] = (w[i] & 0x7F800000u) == 0x7F800000u ? w[i] & 0xFFFFu : w[i];
  }
  f.v = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void keep_finite(Frag<float>& f) {
  float x[8] = {f.lo.x, f.lo.y, f.lo.z, f.lo.w, f.hi.x, f.hi.y, f.hi.z, f.hi.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (__float_as_uint(x[i]) & 0x7F800000u) == 0x7F800000u ? 0.f : x[i];
  frag_of(x, f);
}
// 1 where an operand is NaN or the infinity with that sign bit, else 0.
__device__ __forceinline__ void mark_infinite(const Frag<bf16_t>& f, uint32_t sign, Frag<bf16_t>& mark) {
  const uint32_t w[4] = {f.v.x, f.v.y, f.v.z, f.v.w}, other = 0x7F80u | (sign ? 0u : 0x8000u);
  uint32_t m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0xFFFFu, hi = w[i] >> 16;
    m[i] = (lo & 0x7F80u) == 0x7F80u && lo != other ? 0x3F80u : 0u;
    m[i] |= (hi & 0x7F80u) == 0x7F80u && hi != other ? 0x3F800000u : 0u;
  }
  mark.v = make_uint4(m[0], m[1], m[2], m[3]);
}
__device__ __forceinline__ void mark_infinite(const Frag<float>& f, uint32_t sign, Frag<float>& mark) {
  float x[8] = {f.lo.x, f.lo.y, f.lo.z, f.lo.w, f.hi.x, f.hi.y, f.hi.z, f.hi.w};
  const float other = sign ? INFINITY : -INFINITY;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (__float_as_uint(x[i]) & 0x7F800000u) == 0x7F800000u && x[i] != other ? 1.f : 0.f;
  frag_of(x, mark);
}
// Adds to a column's outputs what it sees (1 in `seen`) of an operand's
// infinities and NaN.  A rare path: its parts run one after the other, so that
// it costs the common one no registers.
template <typename T> __device__ __forceinline__ void add_infinite(f32x16_t& o, const Frag<T>& f, const Frag<T>& seen) {
#pragma unroll
  for (int sign = 0; sign < 2; ++sign) {
    __builtin_amdgcn_sched_barrier(0);
    Frag<T> mark;
    mark_infinite(f, sign, mark);
    f32x16_t hit = zero16();
    mfma32(hit, mark, seen);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] += hit[i] > 0.f ? (sign ? -INFINITY : INFINITY) : 0.f;
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Eight consecutive elements of a row in memory; vec: on a boundary of all eight.
template <typename T> __device__ __forceinline__ Frag<T> row_frag(const T* p, bool vec);
template <> __device__ __forceinline__ Frag<bf16_t> row_frag<bf16_t>(const bf16_t* p, bool vec) {
  if (vec) return frag_load<bf16_t>(p);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
  Frag<bf16_t> f;
  f.v = make_uint4(w[0], w[1], w[2], w[3]);
  return f;
}
template <> __device__ __forceinline__ Frag<float> row_frag<float>(const float* p, bool vec) {
  if (vec) return frag_load<float>(p);
  Frag<float> f;
  f.lo = make_float4(p[0], p[1], p[2], p[3]);
  f.hi = make_float4(p[4], p[5], p[6], p[7]);
  return f;
}

// Operands that a loop only reads, arrived before it: the compiler's waits for
// their loads would otherwise stay in the loop, where they wait for every
// load in flight there too.
template <int N> __device__ __forceinline__ void settle(Frag<bf16_t> (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i].v.x), "+v"(f[i].v.y), "+v"(f[i].v.z), "+v"(f[i].v.w));
}
template <int N> __device__ __forceinline__ void settle(Frag<float> (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    asm volatile("" : "+v"(f[i].lo.x), "+v"(f[i].lo.y), "+v"(f[i].lo.z), "+v"(f[i].lo.w));
    asm volatile("" : "+v"(f[i].hi.x), "+v"(f[i].hi.y), "+v"(f[i].hi.z), "+v"(f[i].hi.w));
  }
}

// mul(n, read(n)) for n < N, in a fixed order: reads run D - 1 ahead of the
// matrix instructions that take them.  (The compiler's own order waits for
// most reads right before their use.)
template <typename T, int N, int D, typename R, typename M> __device__ __forceinline__ void stream(R read, M mul) {
  Frag<T> f[D];
#pragma unroll
  for (int n = 0; n < D - 1 && n < N; ++n) f[n] = read(n);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n + D - 1 < N) f[(n + D - 1) % D] = read(n + D - 1);
    mul(n, f[n % D]);
    __builtin_amdgcn_sched_barrier(0);
  }
}
template <typename T> constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;

// Brings rows of a matrix (HD of its columns, ld elements a row) into an LDS
// tile of ROWS rows, by W waves; rows past `last` repeat row `last`.  kVec:
// rows on 16-byte boundaries go to LDS without passing registers, and the
// reader waits for them (wait_vm).
template <typename T, int HD, int ROWS, int W, bool kVec> struct RowLoader {
  static constexpr int kRowBytes = HD * (int)sizeof(T);
  static constexpr int kPieces = ROWS * kRowBytes / 1024 / W;  // 1 KB pieces a wave
  static constexpr int kPieceRows = 1024 / kRowBytes;
  static constexpr int kPeriod = kPieceRows * W >= 16 ? 1 : 16 / (kPieceRows * W);  // chunks are turned alike every 16 rows
  static_assert(ROWS * kRowBytes % (1024 * W) == 0 && kPieceRows <= 16, "whole pieces");

  // `stride` is ld in bytes.
  static __device__ __forceinline__ void load(const T* base, size_t stride, int last, char* tile) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const char* p = reinterpret_cast<const char*>(base);
    const uint32_t at = lds_address(tile) + wave * 1024;
    auto chunk = [&](int i) {  // of the lane's row in piece i: its row within 16 of them decides
      return (lane * 16 % kRowBytes / 16) ^ turn<kRowBytes>((i * W + wave) * kPieceRows % 16 + lane * 16 / kRowBytes);
    };
    if (kVec && last >= ROWS - 1) {  // few offsets in registers, the rest is the same for all lanes
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int row = (i % kPeriod * W + wave) * kPieceRows + lane * 16 / kRowBytes;
        dma_1k<false>(p + (size_t)(i / kPeriod * kPeriod * W * kPieceRows) * stride, row * (int)stride + chunk(i % kPeriod) * 16,
                      at + i * W * 1024);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int row = min((i * W + wave) * kPieceRows + lane * 16 / kRowBytes, last);
      if constexpr (kVec) {
        dma_1k<false>(p, row * (int)stride + chunk(i) * 16, at + i * W * 1024);
      } else {
        const T* from = reinterpret_cast<const T*>(p + row * stride + chunk(i) * 16);
        T x[16 / sizeof(T)];
#pragma unroll
        for (int e = 0; e < 16 / (int)sizeof(T); ++e) x[e] = from[e];
        *reinterpret_cast<uint4*>(tile + (i * W + wave) * 1024 + lane * 16) = *reinterpret_cast<const uint4*>(x);
      }
    }
  }
};

// Four consecutive columns of a row; vec: on a boundary of all four.
template <typename T> __device__ __forceinline__ void row_store4(T* p, bool vec, float a, float b, float c, float d);
template <> __device__ __forceinline__ void row_store4<bf16_t>(bf16_t* p, bool vec, float a, float b, float c, float d) {
  const uint32_t x = pack_bf16x2(a, b), y = pack_bf16x2(c, d);
  if (vec) {
    *reinterpret_cast<uint2*>(p) = make_uint2(x, y);
  } else {
    p[0] = (bf16_t)x; p[1] = (bf16_t)(x >> 16); p[2] = (bf16_t)y; p[3] = (bf16_t)(y >> 16);
  }
}
template <> __device__ __forceinline__ void row_store4<float>(float* p, bool vec, float a, float b, float c, float d) {
  if (vec) {
    *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
  } else {
    p[0] = a; p[1] = b; p[2] = c; p[3] = d;
  }
}

}  // namespace jf
