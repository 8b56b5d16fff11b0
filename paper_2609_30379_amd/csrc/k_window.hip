// Sliding-window attention over the packed tokens of each sample, with a few
// first keys that stay visible and shared key/value heads (window_device.h).
//
//   s_j = scale q . k_j,  o = sum_j exp(s_j - m) v_j / l,  lse = m + log l
// over the visible keys j of a query, m the running maximum and l the running
// sum of one pass over the keys.  A wave holds 32 query rows as columns of the
// products S^T = K Q^T and O^T = V^T P^T, so that a row's scores, maximum and
// sum stay in two lanes and the weights P^T go from the accumulators of the
// first product into the operand of the second without leaving the registers.
#include <algorithm>
#include <type_traits>

#include "window_device.h"

namespace nt {
namespace {
using namespace win;

struct WindowParams {
  const int32_t *cu_q, *cu_k, *kv_lengths;
  int batch, heads, kv_heads, group, d, left, right, sinks;
  float c, qmul;                 // |scale| log2(e) (1 for scale 0), and what Q is multiplied by: 1, -1 or 0
  const void *q, *k, *v;
  void* o;
  int64_t ld_q, ld_k, ld_v, ld_o, ld_lse;
  float* lse;
  int64_t items;
  bool narrow;
  // a block's key tiles cut over workgroups: split s takes tiles [s chunk, (s + 1) chunk)
  int splits, chunk;
  float2* part_ml;               // [splits][rows of q x heads]: maximum, sum
  float* part_o;                 // [splits][rows of q x heads][d]: unnormalised output
  int64_t part_rows;
};

constexpr int kBlockShift = 7;                 // query rows per workgroup: 4 waves x 32

constexpr int kFewShift = 5;                   // query rows per workgroup of the few-rows kernel
// At most so many blocks of 128 rows: blocks of 32 instead.  About 90 blocks (fp32,
// 8 samples of 66 .. 317 tokens, 4 heads of 32): 8.4 us in blocks of 32, 21 in blocks
// of 128; about 600 (bf16, 16 of 200 .. 1024, 8 heads of 64): 33 and 19.
constexpr int kFewBlocks = 128;
// Key tiles of a split, at least: eight per wave of few rows, two of fp32 past 64
// channels, whose products take 5 us a tile (3 tokens over 366 .. 733 keys, 16 heads on
// 2 of 128: 34 us in splits of 32 tiles, 29 of 16, 20 of 8; 28 samples of 46 over to
// 503 keys, 3 heads of 64: 17 of 32, 20 of 8).  And workgroups that a
// call with few blocks is cut into: four per compute unit of few rows (64 tokens over
// 500 .. 32000 keys, 8 key/value heads of 128: 816 us in 512, 769 in 1024, 796 in
// 2048), else as many as are resident, three up to 64 channels (chunks of 300 .. 700
// tokens over 8000 .. 30000, 16 heads of 64: 135 us in 512, 114 in 768, 122 in 1024)
// and two past that.
constexpr int kFewChunk = 32, kFewChunkWide = 8, kRowsChunk = 8, kFewItems = 1024, kRowsItems = 256;

// One tile of KB x 32 keys against the wave's 32 rows: scores S become weights, O
// and l are brought to the maximum in use.
template <int KB, int ND>
__device__ __forceinline__ void online_softmax(f32x16 (&S)[KB], f32x16 (&O)[ND], float& mx, float& l, float c,
                                               const TileMask& mask) {
  if (mask.cut_hi || mask.cut_lo)
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) mask.hide(S[kb], kb);
  float top = S[0][0];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, S[kb][e]);
  top *= c;
  // The maximum in use only has to keep the weights within range: it moves on
  // when a row's score passes it by 8 (weights up to 2^8), which after the
  // first tiles is rare, and the accumulators are rescaled only then.
  if (__any(top > mx + 8.f)) {
    const float m_new = fmaxf(mx, pair_max(top));
    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mx - m_new);
    mx = m_new;
    l *= alpha;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) O[dt][e] *= alpha;
  }
  const float sub = mx == -INFINITY ? 0.f : mx;
  float sum = 0.f;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      S[kb][e] = __builtin_amdgcn_exp2f(fmaf(S[kb][e], c, -sub));
      sum += S[kb][e];
    }
  l += sum;
}

// o and lse of four channels of a row from its unnormalised output.  A row that
// saw nothing has sum 0.
template <typename T>
__device__ __forceinline__ void write_out(const WindowParams& p, int64_t token, int head, int c, const f32x4& o, float mx,
                                          float l) {
  typedef T vec4 __attribute__((ext_vector_type(4)));
  const float inv = l == 0.f ? 0.f : 1.f / l;
  vec4 w;
#pragma unroll
  for (int u = 0; u < 4; ++u) w[u] = (T)(o[u] * inv);
  *reinterpret_cast<vec4*>((T*)p.o + token * p.ld_o + (int64_t)head * p.d + c) = w;
  if (p.lse && c == 0)
    p.lse[(int64_t)head * p.ld_lse + token] = l == 0.f ? -INFINITY : (mx + __builtin_amdgcn_logf(l)) * kLn2;
}

// 128 rows per workgroup, 32 per wave, all four on the same tile of 64 keys (fp32:
// 32), which lies in LDS twice: the next tile is stored while this one is read, one
// barrier per tile.  Shared tiles quarter the reads of the keys, and S^T = K Q^T
// needs only K from LDS, since Q stays in registers.  Bound by the products and the
// exponentials together: of a wave's time the matrix cores take 38 .. 40 % and the
// vector instructions as much (no LDS bank conflicts), which two or three waves per
// SIMD overlap in part; a wave in its products goes first (s_setprio), so that the
// others' exponentials fill the time around them (without and with, in turn: causal
// window to 8192, 128 channels, 233 and 229 us; chunk over 30000 107 and 104; the
// encoder's window the same).  Tiles of 32 keys at 128 channels cost 14 %, four waves
// per SIMD at 64 channels a third (spills).  Each fragment read from LDS feeds one
// product, 1.75 LDS instructions a product; more rows per wave is not tried.  155
// registers at 64 channels and 253 at 128, no spills.  A call among many, on two cards:
//   64 samples of about 230 tokens, 12 heads of 64, left = right = 64: 41 us, 2.4 TB/s
//   4 samples to 8192, 16 heads on 4 of 128, causal window of 1024: 233 .. 247 us, 694 ..
//   734 TFLOP/s
//   two chunks of 300 .. 700 tokens over 8000 .. 30000, 16 heads on 4 of 64, the join of
//   their splits included: 103 .. 108 us, 555 .. 580 TFLOP/s
template <typename T, int DP>
__global__ void __launch_bounds__(256, DP == 128 ? (sizeof(T) == 4 ? 1 : 2) : DP == 64 && sizeof(T) == 4 ? 2 : 3)
window_rows_kernel(WindowParams p) {
  typedef typename Frag<T>::type frag;
  constexpr int KT = sizeof(T) == 2 ? 64 : 32, KB = KT / 32, NS = DP / 16, ND = DP / 32, kG = NS < 4 ? NS : 4;
  __shared__ __attribute__((aligned(16))) T Kb[2][KT * Tile<T, DP>::kLd];
  __shared__ __attribute__((aligned(16))) T Vb[2][KT * Tile<T, DP>::kLd];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h32 = lane >> 5;
  const int64_t item = block_id();
  if (item >= p.items) return;
  const int hk = (int)(item % p.kv_heads), split = p.splits > 1 ? (int)(item / p.kv_heads % p.splits) : 0;
  const int64_t b = p.splits > 1 ? item / p.kv_heads / p.splits : item / p.kv_heads;
  const int i = find_sample(p.cu_q, p.batch, p.group, kBlockShift, b, lane);
  const int q0 = p.cu_q[i], n = p.cu_q[i + 1] - q0, k0 = p.cu_k[i];
  int m = p.cu_k[i + 1] - k0;
  if (p.kv_lengths) m = min(max(p.kv_lengths[i], 0), m);
  const int64_t rows = (int64_t)n * p.group, r0 = (b - block_start(p.cu_q, i, p.group, kBlockShift)) << kBlockShift;
  if (r0 >= rows) return;
  const int t0 = (int)(r0 / p.group), g0 = (int)(r0 - (int64_t)t0 * p.group);
  const int last = (int)min((int64_t)127, rows - 1 - r0);       // last row of the block
  const int off = m - n;

  // this lane's row: the one of a lane past the last row is the last row, not stored
  const int x = min(wave * 32 + (lane & 31), last), tg = (g0 + x) / p.group;
  const int t = t0 + tg, g = g0 + x - tg * p.group, pos = off + t;
  const int lo = p.left >= 0 ? pos - p.left : 0, hi = p.right >= 0 ? min(pos + p.right, m - 1) : m - 1;
  const bool live = wave * 32 <= last;
  // the same of the wave's first and last row: positions only grow along the rows
  const int pos_a = off + t0 + (g0 + min(wave * 32, last)) / p.group, pos_b = off + t0 + (g0 + min(wave * 32 + 31, last)) / p.group;
  const int lo_a = p.left >= 0 ? pos_a - p.left : 0, hi_a = p.right >= 0 ? min(pos_a + p.right, m - 1) : m - 1;
  const int lo_b = p.left >= 0 ? pos_b - p.left : 0, hi_b = p.right >= 0 ? min(pos_b + p.right, m - 1) : m - 1;

  frag Q[NS];
  {
    const T* src = (const T*)p.q + (int64_t)(q0 + t) * p.ld_q + (int64_t)(hk * p.group + g) * p.d;
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
      const int e = 16 * ks + 8 * h32;
      frag z = {};
      Q[ks] = e < p.d ? *reinterpret_cast<const frag*>(src + e) : z;
    }
    multiply<T>(Q, p.qmul);
  }
  uint32_t tr[2];
  Tile<T, DP>::across_addr(lane, tr);

  f32x16 O[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) O[dt] = f32x16{};
  float mx = -INFINITY, l = 0.f;

  const KeyTiles kt(off + t0, off + t0 + (g0 + last) / p.group, m, p.left, p.right, p.sinks, KT);
  const T* kbase = (const T*)p.k + (int64_t)hk * p.d;
  const T* vbase = (const T*)p.v + (int64_t)hk * p.d;
  // The next tile's keys travel while the scores of this one are computed, its
  // values while the weights are applied: one set of registers for both.
  Stage<T, DP, KT, 256> stage, values;
  auto load = [&](auto& to, const T* base, int64_t ld, int tile) {
    const int j0 = kt.first(tile, KT), cnt = min(kt.end(tile) - j0, KT);
    to.load(tid, base + (int64_t)(k0 + j0) * ld, ld, cnt, p.d, p.narrow);
  };
  const int first = split * p.chunk, end = min(kt.n, first + p.chunk);
  if (first < end) {
    load(stage, kbase, p.ld_k, first);
    load(values, vbase, p.ld_v, first);
    stage.store(tid, Kb[0]);
    values.store(tid, Vb[0]);
  }
  // one tile from buffer B while the next one is on its way into the other: a
  // constant, so that all LDS addresses of the loop are offsets of a few registers
  auto body = [&](auto B, int tile) {
    __syncthreads();
    const T *Ks = Kb[B.value], *Vs = Vb[B.value];
    if (tile + 1 < end) {
      load(stage, kbase, p.ld_k, tile + 1);
      if (KB == 1) load(values, vbase, p.ld_v, tile + 1);
    }
    const int j0 = kt.first(tile, KT), jend = kt.end(tile);
    // unless nothing of the tile is visible to any row of the wave
    const bool seen = live && j0 <= hi_b && (min(j0 + KT, jend) > lo_a || j0 < p.sinks);
    const TileMask mask(j0, KT, jend, lo, hi, hi_a, lo_b, p.sinks, h32);
    // steps of at most four fragments, the reads of a step before the products of
    // the one before
    f32x16 S[KB];
    frag X[kG], Y[kG];
    if (seen) {
      __builtin_amdgcn_s_setprio(1);
      read_part<DP, kG>(Ks, 0, 0, lane, X);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        S[kb] = f32x16{};
        if constexpr (NS > kG) {
          read_part<DP, kG>(Ks, 32 * kb, kG, lane, Y);
          pin();
          S[kb] = product_part<kG>(X, Q, S[kb]);
          pin();
          if (kb + 1 < KB) read_part<DP, kG>(Ks, 32 * kb + 32, 0, lane, X);
          pin();
          S[kb] = product_part<kG>(Y, Q + kG, S[kb]);
          pin();
        } else {
          if (kb + 1 < KB) read_part<DP, kG>(Ks, 32 * kb + 32, 0, lane, Y);
          pin();
          S[kb] = product_part<kG>(X, Q, S[kb]);
          pin();
          if (kb + 1 < KB)
#pragma unroll
            for (int k = 0; k < kG; ++k) X[k] = Y[k];
        }
      }
      __builtin_amdgcn_s_setprio(0);
      online_softmax<KB, ND>(S, O, mx, l, p.c, mask);
    }
    if (tile + 1 < end) {
      stage.store(tid, Kb[1 - B.value]);
      if (KB > 1) load(stage, vbase, p.ld_v, tile + 1);
    }
    if (seen) {
      __builtin_amdgcn_s_setprio(1);
      read_across<DP>(Vs, 0, lane, tr, X);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        frag P;
        read_across<DP>(Vs, 32 * kb + 16, lane, tr, Y);
        to_operand(S[kb], 0, P);
        pin();
        add_products(X, P, O);
        to_operand(S[kb], 1, P);
        pin();
        if (kb + 1 < KB) read_across<DP>(Vs, 32 * kb + 32, lane, tr, X);
        pin();
        add_products(Y, P, O);
      }
      __builtin_amdgcn_s_setprio(0);
    }
    if (tile + 1 < end) (KB > 1 ? stage : values).store(tid, Vb[1 - B.value]);
  };
  for (int tile = first; tile < end; tile += 2) {
    body(std::integral_constant<int, 0>{}, tile);
    if (tile + 1 < end) body(std::integral_constant<int, 1>{}, tile + 1);
  }

  if (wave * 32 + (lane & 31) > last) return;
  l = pair_sum(l);
  if (p.splits > 1) {
    const int64_t row = (int64_t)(q0 + t) * p.heads + hk * p.group + g, at = split * p.part_rows + row;
    if (h32 == 0) p.part_ml[at] = make_float2(mx, l);
    if (l != 0.f) {
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const int c = 32 * dt + 2 * e + 4 * h32;
          if (c < p.d)
            *reinterpret_cast<f32x4*>(p.part_o + at * p.d + c) = f32x4{O[dt][e], O[dt][e + 1], O[dt][e + 2], O[dt][e + 3]};
        }
    }
    return;
  }
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int c = 32 * dt + 2 * e + 4 * h32;
      if (c < p.d)
        write_out<T>(p, q0 + t, hk * p.group + g, c, f32x4{O[dt][e], O[dt][e + 1], O[dt][e + 2], O[dt][e + 3]}, mx, l);
    }
}

// Few rows: one block of 32 rows per workgroup (the query heads of one or a few
// tokens), its four waves on different key tiles, each with its own tile in LDS,
// so no wave waits for another before the end, where the four running sums are
// joined through LDS.  Bound by the cache's bytes: a wave keeps a whole tile in
// flight while it works on the one before, eight waves per compute unit together
// 256 KB; that takes all 256 registers, of bf16 at 64 channels 6 and at 128 channels 30
// are spilled and read back in the tile loop.  64 tokens over 500 .. 32000 keys, 32 heads on 8 of 128: 759 us, 5.0 TB/s
// (a large copy reaches 4.7 here, a large read alone 4.0); one token over a window
// of 1023 keys, 12 heads of 64: 10 us, the latency of four dependent tiles and the
// launch.  Eight waves per workgroup: 9 us for that token, 794 .. 815 for the 64.
template <typename T, int DP> struct FewShape {
  static constexpr int KT = sizeof(T) == 2 && DP < 128 ? 64 : 32;
  static constexpr int kTileBytes = KT * Tile<T, DP>::kLd * (int)sizeof(T);
  static constexpr int kOutLd = DP + 4;                          // padded: rows start on different banks
};
template <typename T, int DP>
__global__ void __launch_bounds__(256, sizeof(T) == 4 && DP == 128 ? 1 : 2)
window_few_kernel(WindowParams p) {
  typedef typename Frag<T>::type frag;
  typedef FewShape<T, DP> F;
  constexpr int KT = F::KT, KB = KT / 32, NS = DP / 16, ND = DP / 32, kG = NS < 4 ? NS : 4;
  union Shared {
    char tile[4][2][F::kTileBytes];
    struct {
      float o[4][32 * F::kOutLd], m[4][32], l[4][32];
    } out;
  };
  __shared__ __attribute__((aligned(16))) Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h32 = lane >> 5;
  const int64_t item = block_id();
  if (item >= p.items) return;
  const int hk = (int)(item % p.kv_heads), split = p.splits > 1 ? (int)(item / p.kv_heads % p.splits) : 0;
  const int64_t b = p.splits > 1 ? item / p.kv_heads / p.splits : item / p.kv_heads;
  const int i = find_sample(p.cu_q, p.batch, p.group, kFewShift, b, lane);
  const int q0 = p.cu_q[i], n = p.cu_q[i + 1] - q0, k0 = p.cu_k[i];
  int m = p.cu_k[i + 1] - k0;
  if (p.kv_lengths) m = min(max(p.kv_lengths[i], 0), m);
  const int64_t rows = (int64_t)n * p.group, r0 = (b - block_start(p.cu_q, i, p.group, kFewShift)) << kFewShift;
  if (r0 >= rows) return;
  const int t0 = (int)(r0 / p.group), g0 = (int)(r0 - (int64_t)t0 * p.group);
  const int last = (int)min((int64_t)31, rows - 1 - r0), off = m - n;
  const int x = min(lane & 31, last), tg = (g0 + x) / p.group;
  const int t = t0 + tg, g = g0 + x - tg * p.group, pos = off + t;
  const int lo = p.left >= 0 ? pos - p.left : 0, hi = p.right >= 0 ? min(pos + p.right, m - 1) : m - 1;
  const int pos_a = off + t0, pos_b = off + t0 + (g0 + last) / p.group;
  const int hi_a = p.right >= 0 ? min(pos_a + p.right, m - 1) : m - 1, lo_b = p.left >= 0 ? pos_b - p.left : 0;

  const KeyTiles kt(pos_a, pos_b, m, p.left, p.right, p.sinks, KT);
  const int first = split * p.chunk, end = min(kt.n, first + p.chunk);
  const T* kbase = (const T*)p.k + (int64_t)hk * p.d;
  const T* vbase = (const T*)p.v + (int64_t)hk * p.d;
  Stage<T, DP, KT, 64> sk, sv;
  auto load = [&](int tile) {
    const int j0 = kt.first(tile, KT), cnt = min(kt.end(tile) - j0, KT);
    sk.load(lane, kbase + (int64_t)(k0 + j0) * p.ld_k, p.ld_k, cnt, p.d, p.narrow);
    sv.load(lane, vbase + (int64_t)(k0 + j0) * p.ld_v, p.ld_v, cnt, p.d, p.narrow);
  };
  if (first + wave < end) load(first + wave);
  frag Q[NS];
  {
    const T* src = (const T*)p.q + (int64_t)(q0 + t) * p.ld_q + (int64_t)(hk * p.group + g) * p.d;
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
      const int e = 16 * ks + 8 * h32;
      frag z = {};
      Q[ks] = e < p.d ? *reinterpret_cast<const frag*>(src + e) : z;
    }
    multiply<T>(Q, p.qmul);
  }
  uint32_t tr[2];
  Tile<T, DP>::across_addr(lane, tr);
  f32x16 O[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) O[dt] = f32x16{};
  float mx = -INFINITY, l = 0.f;
  T* Ks = reinterpret_cast<T*>(sh.tile[wave][0]);
  T* Vs = reinterpret_cast<T*>(sh.tile[wave][1]);
  // the tile is the wave's own: its LDS accesses stay in order, only the compiler
  // has to keep them so
  auto own = [] {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  for (int tile = first + wave; tile < end; tile += 4) {
    own();
    sk.store(lane, Ks);
    sv.store(lane, Vs);
    own();
    if (tile + 4 < end) load(tile + 4);
    const int j0 = kt.first(tile, KT), jend = kt.end(tile);
    const TileMask mask(j0, KT, jend, lo, hi, hi_a, lo_b, p.sinks, h32);
    f32x16 S[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      S[kb] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < NS; ks += kG) {
        frag A[kG];
        read_part<DP, kG>(Ks, 32 * kb, ks, lane, A);
        S[kb] = product_part<kG>(A, Q + ks, S[kb]);
      }
    }
    online_softmax<KB, ND>(S, O, mx, l, p.c, mask);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int nn = 0; nn < 2; ++nn) {
        frag P, X[ND];
        read_across<DP>(Vs, 32 * kb + 16 * nn, lane, tr, X);
        to_operand(S[kb], nn, P);
        add_products(X, P, O);
      }
  }
  l = pair_sum(l);
  __syncthreads();
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<f32x4*>(&sh.out.o[wave][(lane & 31) * F::kOutLd + 32 * dt + 2 * e + 4 * h32]) =
          f32x4{O[dt][e], O[dt][e + 1], O[dt][e + 2], O[dt][e + 3]};
  if (h32 == 0) {
    sh.out.m[wave][lane] = mx;
    sh.out.l[wave][lane] = l;
  }
  __syncthreads();
  for (int u = tid; u < (last + 1) * (DP / 4); u += 256) {
    const int r = u / (DP / 4), c = u % (DP / 4) * 4;
    float top = sh.out.m[0][r], sum = 0.f;
#pragma unroll
    for (int w = 1; w < 4; ++w) top = fmaxf(top, sh.out.m[w][r]);
    const float sub = top == -INFINITY ? 0.f : top;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(sh.out.m[w][r] - sub);
      sum += f * sh.out.l[w][r];
      o += f * *reinterpret_cast<const f32x4*>(&sh.out.o[w][r * F::kOutLd + c]);
    }
    if (c >= p.d) continue;
    const int rt = (g0 + r) / p.group, head = hk * p.group + g0 + r - rt * p.group;
    const int64_t token = q0 + t0 + rt;
    if (p.splits > 1) {
      const int64_t at = split * p.part_rows + token * p.heads + head;
      if (c == 0) p.part_ml[at] = make_float2(top, sum);
      *reinterpret_cast<f32x4*>(p.part_o + at * p.d + c) = o;
    } else {
      write_out<T>(p, token, head, c, o, top, sum);
    }
  }
}

// The splits' sums joined: o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s, four
// channels of a row per thread, the splits in order.  Bound by the partial outputs'
// bytes: 8 us for the chunks above (26 MB written, read from the caches).
template <typename T>
__global__ void __launch_bounds__(256)
window_join_kernel(WindowParams p) {
  const int64_t blk = block_id();
  if (blk >= p.items) return;
  const int dv = p.d / 4;
  const int64_t u = blk * 256 + threadIdx.x, row = u / dv;
  const int c = (int)(u - row * dv) * 4;
  if (row >= p.part_rows) return;
  float top = -INFINITY, sum = 0.f;
  for (int s = 0; s < p.splits; ++s) top = fmaxf(top, p.part_ml[s * p.part_rows + row].x);
  const float sub = top == -INFINITY ? 0.f : top;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < p.splits; ++s) {
    const int64_t at = s * p.part_rows + row;
    const float2 ml = p.part_ml[at];
    if (ml.y == 0.f) continue;                             // no visible key in this split: its output was not written
    const float f = __builtin_amdgcn_exp2f(ml.x - sub);
    sum += f * ml.y;
    o += f * *reinterpret_cast<const f32x4*>(p.part_o + at * p.d + c);
  }
  write_out<T>(p, row / p.heads, (int)(row % p.heads), c, o, top, sum);
}

// How a call is laid out: the kernel, and over how many workgroups a block's keys
// are cut.
struct WindowPlan {
  bool few;
  int splits, chunk;
  int64_t blocks;                // per key/value head
  size_t ml_bytes, o_bytes;
};

// Key tiles of the blocks of `size` rows: all of them, and the most of one block.
// With a window a block's keys begin `left` before its first query and end `right`
// past its last; without a bound on the right (none given, or one that no query
// needs) they end with the sample, which is at most N past the first query.
void count_tiles(const nt_window_args& a, int shift, int kt, int64_t* total, int64_t* most) {
  const nt_layout &Lq = *a.q_layout, &Lk = *a.kv_layout;
  const int64_t G = a.heads / a.kv_heads, size = (int64_t)1 << shift;
  *total = *most = 0;
  for (int i = 0; i < Lq.batch; ++i) {
    const int64_t rows = Lq.lengths[i] * G, m = Lk.lengths[i];
    if (rows == 0 || m == 0) continue;
    int64_t keys = m;
    if (a.left >= 0) {
      const int64_t past = a.right >= 0 ? a.right + (size - 1) / G + 2 : Lq.lengths[i];
      keys = std::min(m, a.left + past + a.sinks);
    }
    const int64_t tiles = (keys + kt - 1) / kt + (a.left >= 0 && a.sinks > 0 ? 1 : 0);
    *total += (rows + size - 1) / size * tiles;
    *most = std::max(*most, tiles);
  }
  *total *= a.kv_heads;
}

WindowPlan window_plan(const nt_window_args& a) {
  WindowPlan w{};
  const nt_layout& Lq = *a.q_layout;
  const int G = a.heads / a.kv_heads;
  int64_t most_rows = 0, blocks = 0;
  for (int i = 0; i < Lq.batch; ++i) {
    const int64_t r = (int64_t)Lq.lengths[i] * G;
    most_rows = std::max(most_rows, r);
    blocks += (r + 127) >> 7;
  }
  // Blocks of 32 rows where no sample has more, and where blocks of 128 would
  // leave most of the card idle.
  w.few = most_rows <= 32 || blocks * a.kv_heads <= kFewBlocks;
  const int shift = w.few ? kFewShift : kBlockShift;
  const bool bf = a.dtype == NT_BF16;
  const int kt = bf && !(w.few && a.head_dim > 64) ? 64 : 32;
  w.blocks = win::block_count(Lq.sum_n, Lq.batch, G, shift);
  int64_t total, most;
  count_tiles(a, shift, kt, &total, &most);
  const int items = w.few ? kFewItems : kRowsItems * (a.head_dim <= 64 ? 3 : 2);
  w.chunk = (int)std::max<int64_t>(w.few ? (!bf && a.head_dim > 64 ? kFewChunkWide : kFewChunk) : kRowsChunk, (total + items - 1) / items);
  // every block gets the splits of the longest one, most of them empty where lengths
  // differ much: bounded, so that empty workgroups never outweigh the work
  const int64_t room = std::max<int64_t>(1, 16 * (int64_t)items / std::max<int64_t>(1, w.blocks * a.kv_heads));
  w.splits = (int)std::max<int64_t>(1, std::min(room, (most + w.chunk - 1) / w.chunk));
  w.chunk = (int)std::max<int64_t>(w.chunk, (most + w.splits - 1) / w.splits);
  if (w.splits == 1) {
    w.chunk = INT32_MAX;
    return w;
  }
  const size_t rows = (size_t)Lq.sum_n * a.heads;
  w.ml_bytes = (rows * w.splits * sizeof(float2) + 15) / 16 * 16;
  w.o_bytes = rows * w.splits * a.head_dim * sizeof(float);
  return w;
}

template <typename T, int DP>
hipError_t launch(const WindowParams& p, bool few, hipStream_t s) {
  if (few) window_few_kernel<T, DP><<<folded_grid(p.items), 256, 0, s>>>(p);
  else window_rows_kernel<T, DP><<<folded_grid(p.items), 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

size_t window_workspace_bytes(const nt_window_args& a) {
  const WindowPlan w = window_plan(a);
  return w.ml_bytes + w.o_bytes;
}

hipError_t launch_window(const nt_window_args& a, hipStream_t s) {
  const nt_layout &Lq = *a.q_layout, &Lk = *a.kv_layout;
  const WindowPlan w = window_plan(a);
  WindowParams p{};
  p.cu_q = Lq.d_cu_seqlens;
  p.cu_k = Lk.d_cu_seqlens;
  p.kv_lengths = a.kv_lengths;
  p.batch = Lq.batch;
  p.heads = a.heads;
  p.kv_heads = a.kv_heads;
  p.group = a.heads / a.kv_heads;
  p.d = a.head_dim;
  p.left = a.left;
  p.right = a.right;
  p.sinks = a.sinks;
  p.c = a.scale == 0.f ? 1.f : fabsf(a.scale) * win::kLog2e;
  p.qmul = a.scale == 0.f ? 0.f : a.scale < 0.f ? -1.f : 1.f;
  p.q = a.q; p.k = a.k; p.v = a.v; p.o = a.o;
  p.ld_q = a.ld_q; p.ld_k = a.ld_k; p.ld_v = a.ld_v; p.ld_o = a.ld_o; p.ld_lse = a.ld_lse;
  p.lse = a.lse;
  p.items = w.blocks * p.kv_heads * w.splits;
  p.splits = w.splits;
  p.chunk = w.chunk;
  p.part_ml = (float2*)a.workspace;
  p.part_o = (float*)((char*)a.workspace + w.ml_bytes);
  p.part_rows = Lq.sum_n * p.heads;
  const bool bf = a.dtype == NT_BF16;
  const int size = bf ? 2 : 4;
  p.narrow = win::narrow_stride(a.ld_k, size) && win::narrow_stride(a.ld_v, size);
  hipError_t e;
  if (p.d <= 32) e = bf ? launch<bf16, 32>(p, w.few, s) : launch<float, 32>(p, w.few, s);
  else if (p.d <= 64) e = bf ? launch<bf16, 64>(p, w.few, s) : launch<float, 64>(p, w.few, s);
  else e = bf ? launch<bf16, 128>(p, w.few, s) : launch<float, 128>(p, w.few, s);
  if (e != hipSuccess || w.splits == 1) return e;
  p.items = (p.part_rows * (p.d / 4) + 255) / 256;
  if (bf) window_join_kernel<bf16><<<folded_grid(p.items), 256, 0, s>>>(p);
  else window_join_kernel<float><<<folded_grid(p.items), 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace nt
