// Shared pieces of the window attention kernels (k_window.hip,
// k_window_backward.hip): 32 x 32 matrix-core products over bf16 or fp32
// operands, tiles of rows in LDS that are read along rows and across them, and
// the rows and keys a workgroup covers.
//
// Sample i has N_i queries and M_i keys (its key length may be given on the
// device); query t sits at position p = M_i - N_i + t.  The G query heads that
// share a key/value head are taken as rows r = t G + g of one problem, so a
// tile of keys is read once for all of them and their key gradients are summed
// in one accumulator.
#pragma once

#include "nt_device.h"
#include "nt_internal.h"

namespace nt {
namespace win {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// D(32 x 32, fp32) += A(32 x 16) B(16 x 32).  Lane l supplies row (A) or column
// (B) l % 32 with the eight k values of group l / 32; it receives column l % 32,
// rows 8 (i / 4) + 4 (l / 32) + i % 4, i = 0 .. 15.  fp32 operands go through
// eight products over two k each, which pair the same k of A and B.
template <typename T> struct Frag;
template <> struct Frag<bf16> { typedef bf16x8 type; };
template <> struct Frag<float> { typedef f32x8 type; };

__device__ __forceinline__ f32x16 mma32(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(const f32x8& a, const f32x8& b, f32x16 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// Elements i = 8 n .. 8 n + 7 of an accumulator as the B operand of a product
// over its rows 16 n .. 16 n + 15: the operand's k order is the accumulator's
// row order {16 n + 4 h + 0..3, 16 n + 8 + 4 h + 0..3}, h = l / 32, and the A
// operand is read in that order too (Tile::across).  bf16 rounds here: a weight
// or score gradient is off by at most 2^-8 of itself, half a step, as the inputs
// and outputs of a bf16 call are; sums stay in fp32.  One rounding more than the
// stored outputs': the normwise error against 64 bits is 2.3e-3 for o, 2.5e-3 for
// dq and dk and 2.3e-3 for dv, where the rounding of the outputs alone gives 1.7e-3,
// 1.8e-3 and 1.7e-3.  Both parts of each weight as two operands reach that, at half
// as many products again: 64 samples of about 230 tokens 40 -> 46 us, causal window
// to 8192 236 -> 296, chunk over 30000 106 -> 133, training N 200 .. 1024 87 -> 97, to
// 8192 1264 -> 1600.
__device__ __forceinline__ void to_operand(const f32x16& s, int n, bf16x8& out) {
#pragma unroll
  for (int e = 0; e < 8; ++e) out[e] = (bf16)s[8 * n + e];
}
__device__ __forceinline__ void to_operand(const f32x16& s, int n, f32x8& out) {
#pragma unroll
  for (int e = 0; e < 8; ++e) out[e] = s[8 * n + e];
}

__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}

// Rows of DP elements in LDS, read in 16-byte pieces along a row (row l % 32 of
// a 32-row block, k values of a product over the row's elements) and across
// rows (element l % 32 of a 32-element block, k values of a product over rows).
template <typename T, int DP> struct Tile;

// bf16: rows without padding, the piece at column c of row r stored at column
// c ^ f(r).  f makes both reads free of bank conflicts: the 16 rows of a quarter
// of a row read go to 16 different 16-byte slots, and the four rows x 64 bytes
// of half of a transposed read to four different 64-byte blocks.
template <int DP> struct Tile<bf16, DP> {
  static constexpr int kLd = DP;                       // elements per row
  static constexpr int kPieces = DP / 8;               // 16-byte pieces per row
  static __device__ __forceinline__ int f(int r) {
    if (DP == 32) return (r >> 2) & 3;
    if (DP == 64) return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
    return (r & 3) << 2 | ((r >> 2) & 3);
  }
  static __device__ __forceinline__ void put(bf16* s, int r, int c, const u32x4& v) {
    *reinterpret_cast<u32x4*>(s + r * DP + ((c ^ f(r)) << 3)) = v;
  }
  // row base + l % 32, elements 16 ks + 8 (l / 32) ..
  static __device__ __forceinline__ bf16x8 along(const bf16* s, int base, int ks, int lane) {
    const int r = lane & 31;
    return *reinterpret_cast<const bf16x8*>(s + (base + r) * DP + (((2 * ks + (lane >> 5)) ^ f(r)) << 3));
  }
  // element 32 dt + l % 32 of rows base + 4 h + 0..3 and base + 8 + 4 h + 0..3,
  // h = l / 32 (base a multiple of 16).  ds_read_b64_tr_b16: lane i of a
  // 16-lane group points at row i / 4, elements 4 (i % 4) and receives four
  // rows of element i.
  static __device__ __forceinline__ void across_addr(int lane, uint32_t (&a)[2]) {
    const int i = lane & 15, h = lane >> 5, half = (lane >> 4) & 1;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int r = 8 * x + 4 * h + (i >> 2), c = 2 * half + ((i & 3) >> 1);
      a[x] = (uint32_t)((r * DP + ((c ^ f(r)) << 3) + (i & 1) * 4) * 2);
    }
  }
};

// fp32: rows padded by four elements (row reads of 16 rows fall on different
// banks); the transposed read is eight 4-byte reads, 32 lanes along a row.
template <int DP> struct Tile<float, DP> {
  static constexpr int kLd = DP + 4;
  static constexpr int kPieces = DP / 4;
  static __device__ __forceinline__ void put(float* s, int r, int c, const u32x4& v) {
    *reinterpret_cast<u32x4*>(s + r * kLd + 4 * c) = v;
  }
  static __device__ __forceinline__ f32x8 along(const float* s, int base, int ks, int lane) {
    const float* p = s + (base + (lane & 31)) * kLd + 16 * ks + 8 * (lane >> 5);
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
    return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
  static __device__ __forceinline__ void across_addr(int, uint32_t (&)[2]) {}
};

template <int DP>
__device__ __forceinline__ bf16x8 across(const bf16* s, int base, int dt, int lane, const uint32_t (&a)[2]) {
  typedef __attribute__((address_space(3))) bf16x4 lds4;
  const uint32_t b = lds_offset(s + base * DP);
  const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(uintptr_t)(b + (a[0] ^ (uint32_t)(dt << 6))));
  const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(uintptr_t)(b + (a[1] ^ (uint32_t)(dt << 6))));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <int DP>
__device__ __forceinline__ f32x8 across(const float* s, int base, int dt, int lane, const uint32_t (&)[2]) {
  const float* p = s + (base + 4 * (lane >> 5)) * Tile<float, DP>::kLd + (lane & 31) + 32 * dt;
  f32x8 out;
#pragma unroll
  for (int e = 0; e < 8; ++e) out[e] = p[((e >> 2) * 8 + (e & 3)) * Tile<float, DP>::kLd];
  return out;
}

// x / group for 0 <= x < 2^20: the quotient of x + 1/2 stays at least 1 / (2 group)
// away from a whole number, far more than the product's rounding.
__device__ __forceinline__ int div_group(int x, float inv_group) { return (int)(((float)x + 0.5f) * inv_group); }

// Buffer resource over `bytes` bytes from a uniform address: loads outside give
// zero (raw buffer, 32-bit data).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* base, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00027000);
}
constexpr uint32_t kOutside = 0x80000000u;         // an offset past every such buffer

// Row strides up to which a tile of at most 129 rows lies within 2^31 bytes.
inline bool narrow_stride(int64_t ld, int size) { return ld * size <= (int64_t)1 << 23; }

// A tile of ROWS rows x DP elements on its way from memory to LDS through the
// registers of THREADS threads.  Rows past the end and elements past d are zero,
// whatever memory holds there: buffer loads return zero outside their range,
// which costs no instruction, where row strides allow 32-bit offsets (narrow),
// and the others select.
template <typename T, int DP, int ROWS, int THREADS> struct Stage {
  static constexpr int kP = Tile<T, DP>::kPieces, kPer = ROWS * kP / THREADS, kE = 16 / sizeof(T), kStep = THREADS / kP;
  static_assert(kPer * THREADS == ROWS * kP && kStep * kP == THREADS, "whole pieces per thread");
  u32x4 v[kPer];
  // rows >= 1 rows from `base` (uniform), ld apart
  __device__ __forceinline__ void load(int tid, const T* base, int64_t ld, int rows, int d, bool narrow) {
    const int r0 = tid / kP, c = tid % kP;
    if (narrow) {
      const auto rs = buffer(base, ((int64_t)(rows - 1) * ld + d) * (int)sizeof(T));
      const uint32_t ldb = (uint32_t)ld * sizeof(T), at = r0 * ldb + c * 16 + (c * kE < d ? 0 : kOutside);
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        v[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, at + i * (kStep * ldb), 0, 0));
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i * kStep;
        v[i] = u32x4{0, 0, 0, 0};
        if (r < rows && c * kE < d) v[i] = *reinterpret_cast<const u32x4*>(base + r * ld + c * kE);
      }
    }
  }
  // rows x = g0 .. of `queries` tokens from `base` (uniform; first token, first head
  // of the group): row x is token x / group, head x % group
  __device__ __forceinline__ void load_group(int tid, const T* base, int64_t ld, int queries, int g0, int group,
                                             float inv_group, int d, bool narrow) {
    const int r0 = tid / kP, c = tid % kP;
    if (narrow) {
      const auto rs = buffer(base, ((int64_t)(queries - 1) * ld + (int64_t)group * d) * (int)sizeof(T));
      const uint32_t ldb = (uint32_t)ld * sizeof(T), db = (uint32_t)d * sizeof(T), c16 = c * 16 + (c * kE < d ? 0 : kOutside);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int x = g0 + r0 + i * kStep, tg = div_group(x, inv_group);
        const uint32_t at = tg * ldb + (x - tg * group) * db + c16;
        v[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, 0));
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int x = g0 + r0 + i * kStep, tg = div_group(x, inv_group);
        v[i] = u32x4{0, 0, 0, 0};
        if (tg < queries && c * kE < d)
          v[i] = *reinterpret_cast<const u32x4*>(base + tg * ld + (int64_t)(x - tg * group) * d + c * kE);
      }
    }
  }
  __device__ __forceinline__ void store(int tid, T* s) const {
    const int r0 = tid / kP, c = tid % kP;
#pragma unroll
    for (int i = 0; i < kPer; ++i) Tile<T, DP>::put(s, r0 + i * kStep, c, v[i]);
  }
};

// Nothing is moved across by the compiler.  The product loops read the fragments
// of a step before the products of the step before it; left alone the compiler
// sinks each read to its product, which then waits for LDS.
__device__ __forceinline__ void pin() { __builtin_amdgcn_sched_barrier(0); }

// by: 1, -1 or 0 (exact)
template <typename T, typename F, int N>
__device__ __forceinline__ void multiply(F (&x)[N], float by) {
  if (by != 1.f)
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int u = 0; u < 8; ++u) x[k][u] = (T)((float)x[k][u] * by);
}

template <int DP, typename T, typename F>
__device__ __forceinline__ void read_along(const T* s, int base, int lane, F (&out)[DP / 16]) {
#pragma unroll
  for (int ks = 0; ks < DP / 16; ++ks) out[ks] = Tile<T, DP>::along(s, base, ks, lane);
}
template <int DP, typename T, typename F, int M>
__device__ __forceinline__ void read_across(const T* s, int base, int lane, const uint32_t (&tr)[2], F (&out)[M]) {
#pragma unroll
  for (int dt = 0; dt < DP / 32; ++dt) out[dt] = across<DP>(s, base, dt, lane, tr);
}
// fragments ks0 .. ks0 + N - 1 of a row block
template <int DP, int N, typename T, typename F, int M>
__device__ __forceinline__ void read_part(const T* s, int base, int ks0, int lane, F (&out)[M]) {
#pragma unroll
  for (int k = 0; k < N; ++k) out[k] = Tile<T, DP>::along(s, base, ks0 + k, lane);
}
template <int N, typename F>
__device__ __forceinline__ f32x16 product_part(const F* a, const F* b, f32x16 s) {
#pragma unroll
  for (int k = 0; k < N; ++k) s = mma32(a[k], b[k], s);
  return s;
}
template <int N, typename F>
__device__ __forceinline__ f32x16 product(const F (&a)[N], const F (&b)[N], f32x16 s = f32x16{}) {
#pragma unroll
  for (int k = 0; k < N; ++k) s = mma32(a[k], b[k], s);
  return s;
}
template <int N, typename F, int M>
__device__ __forceinline__ void add_products(const F (&a)[M], const F& b, f32x16 (&acc)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) acc[k] = mma32(a[k], b, acc[k]);
}

// Sum over the two lanes l, l ^ 32 that hold one column of an accumulator.
__device__ __forceinline__ float pair_sum(float v) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float pair_max(float v) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The sample that block b of `size` rows belongs to, where sample i's blocks
// start at floor(cu_i mul / size) + i: room for every sample's last, partial
// block without a table of block counts (at most one block per sample is idle).
// All lanes of the wave look at 64 samples in a step.
__device__ __forceinline__ int64_t block_start(const int32_t* cu, int i, int mul, int shift) {
  return (((int64_t)cu[i] * mul) >> shift) + i;
}
__device__ __forceinline__ int find_sample(const int32_t* cu, int batch, int mul, int shift, int64_t b, int lane) {
  int lo = 0, n = batch;
  while (n > 1) {
    const int step = (n + 63) >> 6, x = lane * step;
    const bool ok = x < n && block_start(cu, lo + x, mul, shift) <= b;
    const int c = __popcll(__ballot(ok)) - 1;
    lo += c * step;
    n = min(step, n - c * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}
inline int64_t block_count(int64_t total, int batch, int mul, int shift) { return ((total * mul) >> shift) + batch; }

// The keys that a block of rows at positions p0 .. p1 of m keys sees: tiles of
// the sinks before the window (none where the two touch), then of the window.
struct KeyTiles {
  int sink_end, lo, hi, n_sink, n;             // sinks [0, sink_end), window [lo, hi)
  __device__ __forceinline__ KeyTiles(int p0, int p1, int m, int left, int right, int sinks, int kt) {
    hi = right >= 0 ? min(m, p1 + right + 1) : m;
    hi = max(hi, 0);
    lo = left >= 0 ? max(0, p0 - left) : 0;
    sink_end = min(sinks, hi);
    if (lo <= sink_end) lo = sink_end = 0;
    n_sink = (sink_end + kt - 1) / kt;
    n = n_sink + (hi > lo ? (hi - lo + kt - 1) / kt : 0);
  }
  __device__ __forceinline__ int first(int t, int kt) const { return t < n_sink ? t * kt : lo + (t - n_sink) * kt; }
  __device__ __forceinline__ int end(int t) const { return t < n_sink ? sink_end : hi; }
};

// Which keys of a tile (first key j0, keys below jend) a lane's row does not see.
// Key offsets of an accumulator's elements are constants, so each bound that cuts
// the tile costs a comparison and a selection per score; which ones do is the same
// for the whole wave (hi_a, lo_b: the first row's last key, the last row's first).
// Only a tile that holds both sinks and keys before the window needs a third.
struct TileMask {
  bool cut_hi, cut_lo, mixed;
  int hi, lo, sink;              // relative to the lane's first key offset
  __device__ __forceinline__ TileMask(int j0, int kt, int jend, int row_lo, int row_hi, int hi_a, int lo_b, int sinks, int h32) {
    cut_hi = j0 + kt - 1 > min(hi_a, jend - 1);
    cut_lo = j0 < lo_b && jend > sinks && j0 + kt > sinks;
    mixed = j0 < sinks;
    const int base = j0 + 4 * h32;
    hi = min(row_hi, jend - 1) - base;
    lo = row_lo - base;
    sink = sinks - base;
  }
  __device__ __forceinline__ void hide(f32x16& s, int kb) const {
    if (cut_hi)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 32 * kb + 8 * (e >> 2) + (e & 3) <= hi ? s[e] : -INFINITY;
    if (cut_lo) {
      if (mixed) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int k = 32 * kb + 8 * (e >> 2) + (e & 3);
          s[e] = k >= lo || k < sink ? s[e] : -INFINITY;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 32 * kb + 8 * (e >> 2) + (e & 3) >= lo ? s[e] : -INFINITY;
      }
    }
  }
};

}  // namespace win
}  // namespace nt
