// Backward of the sliding-window attention (k_window.hip): the weights are
// recomputed from the forward's lse,
//   P = exp(s - lse),  D = sum_c dO O,  dS = P (dO V^T - D)
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO.
// Two passes without atomics: one over the keys of 128 query rows (dQ, and D for
// the second pass), one over the query rows of 128 keys (dK, dV; the rows of all
// query heads that share the keys are one sequence, so a shared head's gradient
// is one accumulator).  Both hold their 32 rows or keys per wave as columns of
// the products, so P and dS go from accumulators into the next operand in
// registers.
#include <algorithm>

#include "window_device.h"

namespace nt {
namespace {
using namespace win;

struct WindowBwdParams {
  const int32_t *cu_q, *cu_k;
  int batch, heads, kv_heads, group, d, left, right, sinks;
  float scale, c, qmul;          // c = |scale| log2(e) (1 for scale 0); qmul: 1, -1 or 0, what one operand of q . k is multiplied by
  float inv_group;
  const void *q, *k, *v, *o, *dout;
  void *dq, *dk, *dv;
  int64_t ld_q, ld_k, ld_v, ld_o, ld_dout, ld_dq, ld_dk, ld_dv, ld_lse;
  const float* lse;
  float* delta;                  // [heads][sum N] workspace
  int64_t sum_q;
  int64_t items;
  bool narrow;
  // gradients of the sinks from the queries past their window (window_dkv_few_kernel<SINKS>, sink_sum_kernel)
  int split;                     // done apart, in pieces of `piece` rows
  int subs, pieces;              // blocks of 32 sinks, most pieces of a sample
  int64_t piece;                 // rows per piece
  // the rows of a block of keys cut over workgroups
  int parts;
  float* key_part;               // [parts][2][sum M][kv_heads][d]
  int64_t sum_k;
  float *sink_part, *sink_sum;   // [batch][kv_heads][subs][pieces][2][32][DP], [batch][kv_heads][subs][2][32][DP]
};

// At most so many blocks of 128 rows, or of 128 keys, of all heads: blocks of 32
// instead.  dQ: about 90 blocks (fp32, N 66 .. 317, 4 heads of 32) 12 us in blocks of
// 32, 25 in blocks of 128; 600 (bf16, N 200 .. 1024, 8 heads on 2 of 64) 36 and 27.
// dK, dV: 90 blocks 13 and 31; 170 (the bf16 ones) 28 and 54; 384 (N to 8192, 16 heads
// on 4 of 128) 873 and 793.
constexpr int kFewRowBlocks = 128, kFewKeyBlocks = 256;

// First query past the window of the keys jb .. jl; the queries before it are
// gone through by the keys' own workgroup.
__device__ __forceinline__ int window_end(int jl, int left, int off, int n) { return min(n, max(0, jl + left - off + 1)); }

constexpr int kBlockShift = 7, kFewShift = 5;   // rows or keys per workgroup: four waves x 32, or 32 in all

// A row's q and dout as operands, and D.
template <typename T, int DP>
__device__ __forceinline__ void load_row(const WindowBwdParams& p, int64_t token, int head, int h32,
                                         typename Frag<T>::type (&Q)[DP / 16], typename Frag<T>::type (&G)[DP / 16],
                                         float& delta) {
  typedef typename Frag<T>::type frag;
  const T* src = (const T*)p.q + token * p.ld_q + (int64_t)head * p.d;
  const T* dsrc = (const T*)p.dout + token * p.ld_dout + (int64_t)head * p.d;
  const T* osrc = (const T*)p.o + token * p.ld_o + (int64_t)head * p.d;
#pragma unroll
  for (int ks = 0; ks < DP / 16; ++ks) {
    const int e = 16 * ks + 8 * h32;
    frag z = {}, o = {};
    Q[ks] = e < p.d ? *reinterpret_cast<const frag*>(src + e) : z;
    G[ks] = e < p.d ? *reinterpret_cast<const frag*>(dsrc + e) : z;
    if (e < p.d) o = *reinterpret_cast<const frag*>(osrc + e);
#pragma unroll
    for (int u = 0; u < 8; ++u) delta = fmaf((float)o[u], (float)G[ks][u], delta);
  }
  delta = pair_sum(delta);
  multiply<T>(Q, p.qmul);
}
// Four channels of dq, rounded once.
template <typename T>
__device__ __forceinline__ void write_row(const WindowBwdParams& p, int64_t token, int head, int at, const f32x4& dq) {
  typedef T vec4 __attribute__((ext_vector_type(4)));
  vec4 w;
#pragma unroll
  for (int u = 0; u < 4; ++u) w[u] = (T)(dq[u] * p.scale);
  *reinterpret_cast<vec4*>((T*)p.dq + token * p.ld_dq + (int64_t)head * p.d + at) = w;
}

// dQ of 128 rows, 32 per wave: S^T = K Q^T, dP^T = V dO^T and dQ^T += K^T dS^T of one
// tile of keys after another, the tiles twice in LDS as in the forward; dP starts from
// -D, which saves the subtraction.  Q and dO stay in registers, so past 64 channels
// bf16 tiles of 64 keys spill 31 registers; tiles of 32 spill 10, some of them read back
// in the loop, and both K and V of the next tile can be on their way at once (N to 8192,
// 16 heads on 4 of 128, the whole training step: 1301 us in tiles of 64, 1260 in tiles
// of 32; dQ 351 .. 424, median 372, 790 TFLOP/s).  Bound as the forward is: matrix cores
// 38 %, vector instructions 27 % of the time.  64 channels, N 200 .. 1024: 27 us.
template <typename T, int DP>
__global__ void __launch_bounds__(256, DP == 32 ? 3 : DP == 128 && sizeof(T) == 4 ? 1 : 2)
window_dq_kernel(WindowBwdParams p) {
  typedef typename Frag<T>::type frag;
  constexpr int KT = sizeof(T) == 2 && DP < 128 ? 64 : 32, KB = KT / 32, NS = DP / 16, ND = DP / 32, kG = NS < 4 ? NS : 4;
  __shared__ __attribute__((aligned(16))) T Kb[2][KT * Tile<T, DP>::kLd];
  __shared__ __attribute__((aligned(16))) T Vb[2][KT * Tile<T, DP>::kLd];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h32 = lane >> 5;
  const int64_t item = block_id();
  if (item >= p.items) return;
  const int hk = (int)(item % p.kv_heads);
  const int64_t b = item / p.kv_heads;
  const int i = find_sample(p.cu_q, p.batch, p.group, kBlockShift, b, lane);
  const int q0 = p.cu_q[i], n = p.cu_q[i + 1] - q0, k0 = p.cu_k[i], m = p.cu_k[i + 1] - k0;
  const int64_t rows = (int64_t)n * p.group, r0 = (b - block_start(p.cu_q, i, p.group, kBlockShift)) << kBlockShift;
  if (r0 >= rows) return;
  const int t0 = (int)(r0 / p.group), g0 = (int)(r0 - (int64_t)t0 * p.group);
  const int last = (int)min((int64_t)127, rows - 1 - r0), off = m - n;
  const int x = min(wave * 32 + (lane & 31), last), tg = div_group(g0 + x, p.inv_group);
  const int t = t0 + tg, g = g0 + x - tg * p.group, pos = off + t, head = hk * p.group + g;
  const int lo = p.left >= 0 ? pos - p.left : 0, hi = p.right >= 0 ? min(pos + p.right, m - 1) : m - 1;
  const int pos_a = off + t0 + (g0 + min(wave * 32, last)) / p.group, pos_b = off + t0 + (g0 + min(wave * 32 + 31, last)) / p.group;
  const int lo_a = p.left >= 0 ? pos_a - p.left : 0, hi_a = p.right >= 0 ? min(pos_a + p.right, m - 1) : m - 1;
  const int lo_b = p.left >= 0 ? pos_b - p.left : 0, hi_b = p.right >= 0 ? min(pos_b + p.right, m - 1) : m - 1;
  const bool live = wave * 32 <= last, mine = wave * 32 + (lane & 31) <= last;

  frag Q[NS], G[NS];
  float delta = 0.f;
  load_row<T, DP>(p, q0 + t, head, h32, Q, G, delta);
  const float lse = p.lse[(int64_t)head * p.ld_lse + q0 + t], nlse2 = lse == -INFINITY ? 0.f : -lse * kLog2e;
  if (mine && h32 == 0) p.delta[(int64_t)head * p.sum_q + q0 + t] = delta;
  uint32_t tr[2];
  Tile<T, DP>::across_addr(lane, tr);

  f32x16 dQ[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) dQ[dt] = f32x16{};

  const KeyTiles kt(off + t0, off + t0 + (g0 + last) / p.group, m, p.left, p.right, p.sinks, KT);
  const T* kbase = (const T*)p.k + (int64_t)hk * p.d;
  const T* vbase = (const T*)p.v + (int64_t)hk * p.d;
  // the next tile's keys travel during the first half of this one, its values
  // during the second, through the same registers (tiles of 32 keys: both at once)
  Stage<T, DP, KT, 256> stage, values;
  auto load = [&](auto& to, const T* base, int64_t ld, int tile) {
    const int j0 = kt.first(tile, KT), cnt = min(kt.end(tile) - j0, KT);
    to.load(tid, base + (int64_t)(k0 + j0) * ld, ld, cnt, p.d, p.narrow);
  };
  if (kt.n > 0) {
    load(stage, kbase, p.ld_k, 0);
    load(values, vbase, p.ld_v, 0);
    stage.store(tid, Kb[0]);
    values.store(tid, Vb[0]);
  }
  for (int tile = 0; tile < kt.n; ++tile) {
    __syncthreads();
    const int buf = tile & 1;
    const T *Ks = Kb[buf], *Vs = Vb[buf];
    if (tile + 1 < kt.n) {
      load(stage, kbase, p.ld_k, tile + 1);
      if (KB == 1) load(values, vbase, p.ld_v, tile + 1);
    }
    const int j0 = kt.first(tile, KT), jend = kt.end(tile);
    const bool seen = live && j0 <= hi_b && (min(j0 + KT, jend) > lo_a || j0 < p.sinks);
    const TileMask mask(j0, KT, jend, lo, hi, hi_a, lo_b, p.sinks, h32);
    // Block by block of 32 keys in steps of at most four fragments, the reads of a
    // step before the products of the one before; a hidden pair's score starts
    // from -inf, dP from -D.
    frag X[kG], Y[kG];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if (seen) {
        read_part<DP, kG>(Ks, 32 * kb, 0, lane, X);
        f32x16 S = f32x16{}, dP;
        mask.hide(S, kb);
#pragma unroll
        for (int e = 0; e < 16; ++e) dP[e] = -delta;
        if constexpr (NS > kG) {
          read_part<DP, kG>(Ks, 32 * kb, kG, lane, Y);
          S = product_part<kG>(X, Q, S);
          read_part<DP, kG>(Vs, 32 * kb, 0, lane, X);
          S = product_part<kG>(Y, Q + kG, S);
          read_part<DP, kG>(Vs, 32 * kb, kG, lane, Y);
          dP = product_part<kG>(X, G, dP);
          read_across<DP>(Ks, 32 * kb, lane, tr, X);
          dP = product_part<kG>(Y, G + kG, dP);
        } else {
          read_part<DP, kG>(Vs, 32 * kb, 0, lane, Y);
          S = product_part<kG>(X, Q, S);
          read_across<DP>(Ks, 32 * kb, lane, tr, X);
          dP = product_part<kG>(Y, G, dP);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) S[e] = __builtin_amdgcn_exp2f(fmaf(S[e], p.c, nlse2));
        read_across<DP>(Ks, 32 * kb + 16, lane, tr, Y);
#pragma unroll
        for (int e = 0; e < 16; ++e) S[e] *= dP[e];
        frag D;
        to_operand(S, 0, D);
        add_products(X, D, dQ);
        to_operand(S, 1, D);
        add_products(Y, D, dQ);
      }
      if (kb == (KB - 1) / 2 && tile + 1 < kt.n) {
        stage.store(tid, Kb[1 - buf]);
        if (KB > 1) load(stage, vbase, p.ld_v, tile + 1);
      }
    }
    if (tile + 1 < kt.n) (KB > 1 ? stage : values).store(tid, Vb[1 - buf]);
  }
  if (!mine) return;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int at = 32 * dt + 2 * e + 4 * h32;
      if (at < p.d) write_row<T>(p, q0 + t, head, at, f32x4{dQ[dt][e], dQ[dt][e + 1], dQ[dt][e + 2], dQ[dt][e + 3]});
    }
}

// dQ of 32 rows per workgroup, its four waves on different key tiles, each with its
// own tile in LDS, their sums joined in order at the end: for calls whose blocks of
// 128 rows would leave most of the card idle.  Bound by latency: 12 us for fp32, N
// 66 .. 317, 4 heads of 32 (25 in blocks of 128).
template <typename T, int DP>
__global__ void __launch_bounds__(256, DP == 128 || (DP == 64 && sizeof(T) == 4) ? 1 : 2)
window_dq_few_kernel(WindowBwdParams p) {
  typedef typename Frag<T>::type frag;
  constexpr int KT = 32, NS = DP / 16, ND = DP / 32, kOutLd = DP + 4;
  union Shared {
    T tile[4][2][KT * Tile<T, DP>::kLd];
    float sum[4][32 * kOutLd];
  };
  __shared__ __attribute__((aligned(16))) Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h32 = lane >> 5;
  const int64_t item = block_id();
  if (item >= p.items) return;
  const int hk = (int)(item % p.kv_heads);
  const int64_t b = item / p.kv_heads;
  const int i = find_sample(p.cu_q, p.batch, p.group, kFewShift, b, lane);
  const int q0 = p.cu_q[i], n = p.cu_q[i + 1] - q0, k0 = p.cu_k[i], m = p.cu_k[i + 1] - k0;
  const int64_t rows = (int64_t)n * p.group, r0 = (b - block_start(p.cu_q, i, p.group, kFewShift)) << kFewShift;
  if (r0 >= rows) return;
  const int t0 = (int)(r0 / p.group), g0 = (int)(r0 - (int64_t)t0 * p.group);
  const int last = (int)min((int64_t)31, rows - 1 - r0), off = m - n;
  const int x = min(lane & 31, last), tg = div_group(g0 + x, p.inv_group);
  const int t = t0 + tg, g = g0 + x - tg * p.group, pos = off + t, head = hk * p.group + g;
  const int lo = p.left >= 0 ? pos - p.left : 0, hi = p.right >= 0 ? min(pos + p.right, m - 1) : m - 1;
  const int pos_a = off + t0, pos_b = off + t0 + (g0 + last) / p.group;
  const int hi_a = p.right >= 0 ? min(pos_a + p.right, m - 1) : m - 1, lo_b = p.left >= 0 ? pos_b - p.left : 0;

  const KeyTiles kt(pos_a, pos_b, m, p.left, p.right, p.sinks, KT);
  const T* kbase = (const T*)p.k + (int64_t)hk * p.d;
  const T* vbase = (const T*)p.v + (int64_t)hk * p.d;
  Stage<T, DP, KT, 64> sk, sv;
  auto load = [&](int tile) {
    const int j0 = kt.first(tile, KT), cnt = min(kt.end(tile) - j0, KT);
    sk.load(lane, kbase + (int64_t)(k0 + j0) * p.ld_k, p.ld_k, cnt, p.d, p.narrow);
    sv.load(lane, vbase + (int64_t)(k0 + j0) * p.ld_v, p.ld_v, cnt, p.d, p.narrow);
  };
  if (wave < kt.n) load(wave);
  frag Q[NS], G[NS];
  float delta = 0.f;
  load_row<T, DP>(p, q0 + t, head, h32, Q, G, delta);
  const float lse = p.lse[(int64_t)head * p.ld_lse + q0 + t], nlse2 = lse == -INFINITY ? 0.f : -lse * kLog2e;
  if (wave == 0 && h32 == 0 && (lane & 31) <= last) p.delta[(int64_t)head * p.sum_q + q0 + t] = delta;
  uint32_t tr[2];
  Tile<T, DP>::across_addr(lane, tr);
  f32x16 dQ[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) dQ[dt] = f32x16{};
  T *Ks = sh.tile[wave][0], *Vs = sh.tile[wave][1];
  auto own = [] {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  for (int tile = wave; tile < kt.n; tile += 4) {
    own();
    sk.store(lane, Ks);
    sv.store(lane, Vs);
    own();
    if (tile + 4 < kt.n) load(tile + 4);
    const int j0 = kt.first(tile, KT), jend = kt.end(tile);
    const TileMask mask(j0, KT, jend, lo, hi, hi_a, lo_b, p.sinks, h32);
    f32x16 S = f32x16{}, dP;
#pragma unroll
    for (int e = 0; e < 16; ++e) dP[e] = -delta;
    mask.hide(S, 0);
    frag A[NS], X[ND], D;
    read_along<DP>(Ks, 0, lane, A);
    S = product(A, Q, S);
    read_along<DP>(Vs, 0, lane, A);
    dP = product(A, G, dP);
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = __builtin_amdgcn_exp2f(fmaf(S[e], p.c, nlse2)) * dP[e];
#pragma unroll
    for (int nn = 0; nn < 2; ++nn) {
      read_across<DP>(Ks, 16 * nn, lane, tr, X);
      to_operand(S, nn, D);
      add_products(X, D, dQ);
    }
  }
  __syncthreads();
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<f32x4*>(&sh.sum[wave][(lane & 31) * kOutLd + 32 * dt + 2 * e + 4 * h32]) =
          f32x4{dQ[dt][e], dQ[dt][e + 1], dQ[dt][e + 2], dQ[dt][e + 3]};
  __syncthreads();
  for (int u = tid; u < (last + 1) * (DP / 4); u += 256) {
    const int r = u / (DP / 4), at = u % (DP / 4) * 4;
    f32x4 a = *reinterpret_cast<f32x4*>(&sh.sum[0][r * kOutLd + at]);
#pragma unroll
    for (int w = 1; w < 4; ++w) a += *reinterpret_cast<f32x4*>(&sh.sum[w][r * kOutLd + at]);
    if (at >= p.d) continue;
    const int rt = div_group(g0 + r, p.inv_group);
    write_row<T>(p, q0 + t0 + rt, hk * p.group + g0 + r - rt * p.group, at, a);
  }
}

// One block of 32 rows (in LDS from row r0) against the wave's 32 keys, in steps of
// at most four fragments: each step issues the reads of the next one before its
// products, and the exponentials and score gradients run under products (the
// compiler keeps to that order by itself here).  lse_s holds -lse log2(e) (-inf for a
// row past the end: weight 0), delta_s -D, pos_s the rows' positions; a hidden pair's
// score starts from -inf.
template <typename T, int DP>
__device__ __forceinline__ void key_block(const T* Qs, const T* Gs, const float* lse_s, const float* delta_s,
                                          const int* pos_s, int r0, bool cut_lo, bool cut_hi, int plo, int phi, float c,
                                          const typename Frag<T>::type (&K)[DP / 16],
                                          const typename Frag<T>::type (&V)[DP / 16], f32x16 (&dK)[DP / 32],
                                          f32x16 (&dV)[DP / 32], int lane, const uint32_t (&tr)[2]) {
  typedef typename Frag<T>::type frag;
  constexpr int NS = DP / 16, ND = DP / 32, kG = NS < 4 ? NS : 4;
  const int h32 = lane >> 5;
  frag X[kG], Y[kG], W;
  read_part<DP, kG>(Qs, r0, 0, lane, X);
  f32x16 S = f32x16{}, dP;
  if (cut_lo || cut_hi) {
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const int4 ps = *reinterpret_cast<const int4*>(pos_s + r0 + 8 * e4 + 4 * h32);
      const int pr[4] = {ps.x, ps.y, ps.z, ps.w};
      if (cut_lo)
#pragma unroll
        for (int u = 0; u < 4; ++u) S[4 * e4 + u] = pr[u] >= plo ? 0.f : -INFINITY;
      if (cut_hi)
#pragma unroll
        for (int u = 0; u < 4; ++u) S[4 * e4 + u] = pr[u] <= phi ? S[4 * e4 + u] : -INFINITY;
    }
  }
  if constexpr (NS > kG) {
    read_part<DP, kG>(Qs, r0, kG, lane, Y);
    S = product_part<kG>(X, K, S);
    read_part<DP, kG>(Gs, r0, 0, lane, X);
    S = product_part<kG>(Y, K + kG, S);
  } else {
    read_part<DP, kG>(Gs, r0, 0, lane, Y);
    S = product_part<kG>(X, K, S);
#pragma unroll
    for (int k = 0; k < kG; ++k) X[k] = Y[k];
  }
#pragma unroll
  for (int e4 = 0; e4 < 4; ++e4) {
    const f32x4 de = *reinterpret_cast<const f32x4*>(delta_s + r0 + 8 * e4 + 4 * h32);
#pragma unroll
    for (int u = 0; u < 4; ++u) dP[4 * e4 + u] = de[u];
  }
  if constexpr (NS > kG) {
    read_part<DP, kG>(Gs, r0, kG, lane, Y);
    dP = product_part<kG>(X, V, dP);
    read_across<DP>(Gs, r0, lane, tr, X);
    dP = product_part<kG>(Y, V + kG, dP);
  } else {
    read_across<DP>(Gs, r0, lane, tr, Y);
    dP = product_part<kG>(X, V, dP);
#pragma unroll
    for (int k = 0; k < ND; ++k) X[k] = Y[k];
  }
#pragma unroll
  for (int e4 = 0; e4 < 4; ++e4) {
    const f32x4 ls = *reinterpret_cast<const f32x4*>(lse_s + r0 + 8 * e4 + 4 * h32);
#pragma unroll
    for (int u = 0; u < 4; ++u) S[4 * e4 + u] = __builtin_amdgcn_exp2f(fmaf(S[4 * e4 + u], c, ls[u]));
  }
  to_operand(S, 0, W);
  read_across<DP>(Gs, r0 + 16, lane, tr, Y);
  add_products(X, W, dV);
#pragma unroll
  for (int e = 0; e < 16; ++e) dP[e] *= S[e];
  to_operand(S, 1, W);
  read_across<DP>(Qs, r0, lane, tr, X);
  add_products(Y, W, dV);
  to_operand(dP, 0, W);
  read_across<DP>(Qs, r0 + 16, lane, tr, Y);
  add_products(X, W, dK);
  to_operand(dP, 1, W);
  add_products(Y, W, dK);
}

// Positions of the rows that see a key: plo .. phi.
__device__ __forceinline__ int first_seeing(const WindowBwdParams& p, int j) {
  return p.right >= 0 ? j - p.right : INT32_MIN + 1;
}
__device__ __forceinline__ int last_seeing(const WindowBwdParams& p, int j) {
  return p.left >= 0 && j >= p.sinks ? j + p.left : INT32_MAX;
}
// The same for all keys ja .. je: first of the last key, last of the first key that is no sink.
__device__ __forceinline__ int last_seeing_all(const WindowBwdParams& p, int ja, int je) {
  return p.left >= 0 && je >= p.sinks ? max(ja, p.sinks) + p.left : INT32_MAX;
}

template <typename T, int DP>
__device__ __forceinline__ void load_keys(const WindowBwdParams& p, int64_t row, int hk, int h32,
                                          typename Frag<T>::type (&K)[DP / 16], typename Frag<T>::type (&V)[DP / 16]) {
  typedef typename Frag<T>::type frag;
  const T* ksrc = (const T*)p.k + row * p.ld_k + (int64_t)hk * p.d;
  const T* vsrc = (const T*)p.v + row * p.ld_v + (int64_t)hk * p.d;
#pragma unroll
  for (int ks = 0; ks < DP / 16; ++ks) {
    const int e = 16 * ks + 8 * h32;
    frag z = {};
    K[ks] = e < p.d ? *reinterpret_cast<const frag*>(ksrc + e) : z;
    V[ks] = e < p.d ? *reinterpret_cast<const frag*>(vsrc + e) : z;
  }
  multiply<T>(K, p.qmul);
}

// Four channels of dk and dv of a key (the row of the packed keys), rounded once.
template <typename T>
__device__ __forceinline__ void write_keys(const WindowBwdParams& p, int64_t row, int hk, int at, const f32x4& dk,
                                           const f32x4& dv) {
  typedef T vec4 __attribute__((ext_vector_type(4)));
  vec4 a, w;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    a[u] = (T)(dk[u] * p.scale);
    w[u] = (T)dv[u];
  }
  *reinterpret_cast<vec4*>((T*)p.dk + row * p.ld_dk + (int64_t)hk * p.d + at) = a;
  *reinterpret_cast<vec4*>((T*)p.dv + row * p.ld_dv + (int64_t)hk * p.d + at) = w;
}

// The same of one part of the rows, for key_join_kernel.
__device__ __forceinline__ void write_part(const WindowBwdParams& p, int part, int64_t row, int hk, int at,
                                           const f32x4& dk, const f32x4& dv) {
  const int64_t width = (int64_t)p.kv_heads * p.d;
  float* out = p.key_part + ((int64_t)part * 2 * p.sum_k + row) * width + (int64_t)hk * p.d + at;
  *reinterpret_cast<f32x4*>(out) = dk;
  *reinterpret_cast<f32x4*>(out + p.sum_k * width) = dv;
}

// The rows of a tile on their way into LDS: q and dout of all query heads that
// share the keys, and the rows' statistics.  THREADS threads of index tid.
template <typename T, int DP, int RT, int THREADS> struct RowTile {
  Stage<T, DP, RT, THREADS> q, g;
  float lse, delta;              // as loaded: touching them here would wait for all loads of the tile
  int pos;
  bool inside;
  // cnt rows from row g0 of query t0 of the sample that begins at q0
  __device__ __forceinline__ void load(const WindowBwdParams& p, int tid, int hk, int q0, int t0, int g0, int queries,
                                       int cnt, int off) {
    const int first = q0 + t0, h0 = hk * p.group;
    q.load_group(tid, (const T*)p.q + (int64_t)first * p.ld_q + (int64_t)h0 * p.d, p.ld_q, queries, g0, p.group,
                 p.inv_group, p.d, p.narrow);
    g.load_group(tid, (const T*)p.dout + (int64_t)first * p.ld_dout + (int64_t)h0 * p.d, p.ld_dout, queries, g0, p.group,
                 p.inv_group, p.d, p.narrow);
    if (tid < RT) {
      const int r = min(tid, cnt - 1), tg = div_group(g0 + r, p.inv_group), head = h0 + g0 + r - tg * p.group;
      lse = p.lse[(int64_t)head * p.ld_lse + first + tg];
      delta = p.delta[(int64_t)head * p.sum_q + first + tg];
      pos = off + t0 + tg;
      inside = tid < cnt;
    }
  }
  __device__ __forceinline__ void store(int tid, T* qs, T* gs, float* lse_s, float* delta_s, int* pos_s) const {
    q.store(tid, qs);
    g.store(tid, gs);
    if (tid < RT) {
      // a row past the end has weight 0; one that sees nothing (-inf) is hidden everywhere
      lse_s[tid] = !inside ? -INFINITY : lse == -INFINITY ? 0.f : lse * -kLog2e;
      delta_s[tid] = -delta;
      pos_s[tid] = pos;
    }
  }
};

// dK and dV of 128 keys, 32 per wave; the workgroup walks the rows that see them, 64
// (fp32: 32) at a time through one tile of q and dout in LDS while the next is on its
// way in registers.  K, V and both gradients of a wave's keys are 192 registers at 128
// bf16 channels, and 371 of 512 are used, so one wave per SIMD; two waves, forced, spill
// (1130 us for N to 8192, 16 heads on 4 of 128, against 800 then), and dK and dV in
// workgroups of their own compute S twice (907).  fp32 past 64 channels uses all 512 and
// spills 24.  Bound by the products' latency with nothing else to issue: matrix cores
// 33 % of the time it runs.  The 428 workgroups on 256 compute units would take two
// turns, so their rows are cut in four parts: 761 .. 800 us uncut, now 621 .. 756, median
// 660, 595 TFLOP/s, and 46 in the join.  Without any new rows to read it takes 9 % less;
// workgroups that walk shared rows at the same time gain nothing.
template <typename T, int DP>
__global__ void __launch_bounds__(256, DP == 128 || (DP == 64 && sizeof(T) == 4) ? 1 : 2)
window_dkv_kernel(WindowBwdParams p) {
  typedef typename Frag<T>::type frag;
  constexpr int RT = sizeof(T) == 2 ? 64 : 32, ND = DP / 32;
  __shared__ __attribute__((aligned(16))) T Qs[RT * Tile<T, DP>::kLd];
  __shared__ __attribute__((aligned(16))) T Gs[RT * Tile<T, DP>::kLd];
  __shared__ __attribute__((aligned(16))) float lse_s[RT];
  __shared__ __attribute__((aligned(16))) float delta_s[RT];
  __shared__ __attribute__((aligned(16))) int pos_s[RT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h32 = lane >> 5;
  const int64_t item = block_id();
  if (item >= p.items) return;
  const int hk = (int)(item % p.kv_heads), part = p.parts > 1 ? (int)(item / p.kv_heads % p.parts) : 0;
  const int64_t b = p.parts > 1 ? item / p.kv_heads / p.parts : item / p.kv_heads;
  const int i = find_sample(p.cu_k, p.batch, 1, kBlockShift, b, lane);
  const int q0 = p.cu_q[i], n = p.cu_q[i + 1] - q0, k0 = p.cu_k[i], m = p.cu_k[i + 1] - k0, off = m - n;
  const int64_t jb64 = (b - block_start(p.cu_k, i, 1, kBlockShift)) << kBlockShift;
  if (jb64 >= m) return;
  const int jb = (int)jb64, jl = min(jb + 127, m - 1);          // keys jb .. jl
  const int j = min(jb + wave * 32 + (lane & 31), m - 1);       // a lane past the last key takes the last one, not stored
  const bool live = jb + wave * 32 < m, mine = jb + wave * 32 + (lane & 31) < m;
  const int plo = first_seeing(p, j), phi = last_seeing(p, j);
  const int ja = min(jb + wave * 32, m - 1), je = min(jb + wave * 32 + 31, m - 1);      // the wave's keys
  const int plo_a = first_seeing(p, ja), plo_b = first_seeing(p, je), phi_a = last_seeing_all(p, ja, je);
  const int phi_b = p.left >= 0 && ja >= p.sinks ? je + p.left : INT32_MAX;
  frag K[DP / 16], V[DP / 16];
  load_keys<T, DP>(p, k0 + j, hk, h32, K, V);
  uint32_t tr[2];
  Tile<T, DP>::across_addr(lane, tr);
  f32x16 dK[ND], dV[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) dK[dt] = dV[dt] = f32x16{};

  // queries that see a key of the block, as rows [ra, rb)
  const int ta = p.right >= 0 ? min(max(0, jb - p.right - off), n) : 0;
  const int tb = max(ta, p.left >= 0 && (jb >= p.sinks || p.split) ? window_end(jl, p.left, off, n) : n);
  const int64_t rows = (int64_t)(tb - ta) * p.group;
  int first = 0, tiles = (int)((rows + RT - 1) / RT);
  if (p.parts > 1) {
    first = (int)((int64_t)tiles * part / p.parts);
    tiles = (int)((int64_t)tiles * (part + 1) / p.parts);
  }
  RowTile<T, DP, RT, 256> in;
  // a tile's first row as (t0, g0), moved on by RT rows per tile
  const int step_t = RT / p.group, step_g = RT - step_t * p.group;
  int t0 = ta + (int)((int64_t)first * RT / p.group), g0 = (int)((int64_t)first * RT % p.group);
  auto load = [&](int tile) {
    in.load(p, tid, hk, q0, t0, g0, min(tb - t0, RT + 1), (int)min((int64_t)RT, rows - (int64_t)tile * RT), off);
  };
  if (first < tiles) load(first);
  for (int tile = first; tile < tiles; ++tile) {
    __syncthreads();
    in.store(tid, Qs, Gs, lse_s, delta_s, pos_s);
    __syncthreads();
    const int cnt = (int)min((int64_t)RT, rows - (int64_t)tile * RT);
    const int pa = off + t0, pe = off + t0 + (g0 + cnt - 1) / p.group;
    t0 += step_t;
    g0 += step_g;
    if (g0 >= p.group) {
      g0 -= p.group;
      ++t0;
    }
    if (tile + 1 < tiles) load(tile + 1);
    if (!live || pe < plo_a || pa > phi_b) continue;       // no row of the tile sees a key of the wave
    const bool cut_lo = pa < plo_b, cut_hi = pe > phi_a;
#pragma unroll 1
    for (int r0 = 0; r0 < RT; r0 += 32)
      key_block<T, DP>(Qs, Gs, lse_s, delta_s, pos_s, r0, cut_lo, cut_hi, plo, phi, p.c, K, V, dK, dV, lane, tr);
  }
  if (!mine) return;
  const bool more = part == 0 && p.split && j < p.sinks && tb < n;      // what the queries past the window add to a sink
  const float* sum = p.sink_sum + (((int64_t)(i * p.kv_heads + hk) * p.subs + (j >> 5)) * 64 + (j & 31)) * DP;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int at = 32 * dt + 2 * e + 4 * h32;
      if (at >= p.d) continue;
      f32x4 a = {dK[dt][e], dK[dt][e + 1], dK[dt][e + 2], dK[dt][e + 3]};
      f32x4 w = {dV[dt][e], dV[dt][e + 1], dV[dt][e + 2], dV[dt][e + 3]};
      if (more) {
        a += *reinterpret_cast<const f32x4*>(sum + at);
        w += *reinterpret_cast<const f32x4*>(sum + 32 * DP + at);
      }
      if (p.parts > 1) {
        write_part(p, part, k0 + j, hk, at, a, w);
      } else {
        write_keys<T>(p, k0 + j, hk, at, a, w);
      }
    }
}

// The parts' sums of dK and dV, added in order, four channels of a key per thread.
// Bound by the partial sums' bytes: 219 MB for the four parts above, 47 us, 5.3 TB/s
// with what is written.
template <typename T>
__global__ void __launch_bounds__(256)
key_join_kernel(WindowBwdParams p) {
  const int64_t blk = block_id();
  if (blk >= p.items) return;
  const int dv = p.kv_heads * (p.d / 4);
  const int64_t u = blk * 256 + threadIdx.x, row = u / dv, plane = p.sum_k * dv * 4;
  if (row >= p.sum_k) return;
  const int c = (int)(u - row * dv) * 4, hk = c / p.d;
  f32x4 a = {0.f, 0.f, 0.f, 0.f}, w = a;
  for (int x = 0; x < p.parts; ++x) {
    a += *reinterpret_cast<const f32x4*>(p.key_part + 2 * x * plane + u * 4);
    w += *reinterpret_cast<const f32x4*>(p.key_part + (2 * x + 1) * plane + u * 4);
  }
  write_keys<T>(p, row, hk, c - hk * p.d, a, w);
}

// dK and dV of 32 keys per workgroup, its four waves on different tiles of rows,
// each with its own tile in LDS, their sums joined in order at the end.  Two uses:
// - calls whose blocks of 128 keys would leave most of the card idle;
// - SINKS: the sinks' gradients from the queries past their window, few keys and
//   all the later rows of the sample, which the workgroup of a block of keys would
//   walk alone while the others have left.  A workgroup takes a piece of the rows
//   (every row sees every sink there) and leaves its sums for sink_sum_kernel.
// Bound by latency, four walks instead of one: 13 us for fp32, N 66 .. 317, 4 heads of
// 32 (31 in blocks of 128 keys); 28 for N 200 .. 1024, 8 heads on 2 of 64 (54); the
// sinks of N to 8192, 16 heads on 4 of 128: 23.  fp32 past 64 channels spills: 121
// registers here, stored and read back in the loop, and 38 in the dQ of few rows.
template <typename T, int DP, bool SINKS>
__global__ void __launch_bounds__(256, sizeof(T) == 4 || DP == 128 ? 1 : 2)
window_dkv_few_kernel(WindowBwdParams p) {
  typedef typename Frag<T>::type frag;
  constexpr int RT = 32, ND = DP / 32, kOutLd = DP + 4;
  struct Rows {
    T q[RT * Tile<T, DP>::kLd], g[RT * Tile<T, DP>::kLd];
    float lse[RT], delta[RT];
    int pos[RT];
  };
  union Shared {
    Rows tile[4];
    float sum[4][32 * kOutLd];
  };
  __shared__ __attribute__((aligned(16))) Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h32 = lane >> 5;
  const int64_t item = block_id();
  if (item >= p.items) return;
  const int hk = (int)(item % p.kv_heads);
  int i, sub = 0, piece = 0, part = 0, jb;
  if (SINKS) {
    piece = (int)(item / p.kv_heads % p.pieces);
    sub = (int)(item / p.kv_heads / p.pieces % p.subs);
    i = (int)(item / p.kv_heads / p.pieces / p.subs);
    jb = 32 * sub;
  } else {
    part = p.parts > 1 ? (int)(item / p.kv_heads % p.parts) : 0;
    const int64_t b = p.parts > 1 ? item / p.kv_heads / p.parts : item / p.kv_heads;
    i = find_sample(p.cu_k, p.batch, 1, kFewShift, b, lane);
    jb = (int)((b - block_start(p.cu_k, i, 1, kFewShift)) << kFewShift);
  }
  const int q0 = p.cu_q[i], n = p.cu_q[i + 1] - q0, k0 = p.cu_k[i], m = p.cu_k[i + 1] - k0, off = m - n;
  const int keys = SINKS ? min(p.sinks, m) : m;            // the keys that matter here
  if (jb >= keys) return;
  const int je = min(jb + 31, keys - 1), j = min(jb + (lane & 31), keys - 1);
  const int plo = first_seeing(p, j), phi = last_seeing(p, j);
  const int plo_b = first_seeing(p, je), phi_a = last_seeing_all(p, jb, je);
  // the rows: with a window up to its end, where the sinks' own call begins
  const int blk_end = min((jb & ~127) + 127, m - 1);       // last key of the block of 128, which sets that end
  const int ta = p.right >= 0 ? min(max(0, (SINKS ? jb & ~127 : jb) - p.right - off), n) : 0;
  const int far = p.left >= 0 ? max(ta, window_end(blk_end, p.left, off, n)) : n;
  int64_t ra, rb;
  if (SINKS) {
    ra = (int64_t)far * p.group + piece * p.piece;
    rb = min((int64_t)n * p.group, ra + p.piece);
  } else {
    ra = (int64_t)ta * p.group;
    rb = (int64_t)(jb < p.sinks ? (p.split ? far : n) : p.left >= 0 ? max(ta, window_end(je, p.left, off, n)) : n) * p.group;
    if (p.parts > 1) {
      const int64_t tiles = max((int64_t)0, rb - ra + RT - 1) / RT, end = ra + tiles * (part + 1) / p.parts * RT;
      ra += tiles * part / p.parts * RT;
      rb = min(rb, end);
    }
  }
  if (SINKS && ra >= rb) return;
  frag K[DP / 16], V[DP / 16];
  load_keys<T, DP>(p, k0 + j, hk, h32, K, V);
  uint32_t tr[2];
  Tile<T, DP>::across_addr(lane, tr);
  f32x16 dK[ND], dV[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) dK[dt] = dV[dt] = f32x16{};
  RowTile<T, DP, RT, 64> in;
  Rows& my = sh.tile[wave];
  const int64_t first = ra + RT * wave;
  int t0 = (int)(first / p.group), g0 = (int)(first - (int64_t)t0 * p.group);
  const int step_t = 4 * RT / p.group, step_g = 4 * RT - step_t * p.group;
  const int t_end = (int)((rb + p.group - 1) / p.group);
  auto load = [&](int64_t r) {
    in.load(p, lane, hk, q0, t0, g0, min(t_end - t0, RT + 1), (int)min((int64_t)RT, rb - r), off);
  };
  auto own = [] {                                          // the tile is the wave's own
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  if (first < rb) load(first);
  for (int64_t r = first; r < rb; r += 4 * RT) {
    own();
    in.store(lane, my.q, my.g, my.lse, my.delta, my.pos);
    own();
    const int pa = off + t0, pe = off + t0 + (g0 + (int)min((int64_t)RT, rb - r) - 1) / p.group;
    t0 += step_t;
    g0 += step_g;
    if (g0 >= p.group) {
      g0 -= p.group;
      ++t0;
    }
    if (r + 4 * RT < rb) load(r + 4 * RT);
    key_block<T, DP>(my.q, my.g, my.lse, my.delta, my.pos, 0, !SINKS && pa < plo_b, !SINKS && pe > phi_a, plo, phi,
                     p.c, K, V, dK, dV, lane, tr);
  }
  // the four waves' sums: dK, then dV, four channels per thread and turn
  constexpr int kTurns = 32 * DP / 4 / 256 > 0 ? 32 * DP / 4 / 256 : 1;
  f32x4 total[2][kTurns];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    __syncthreads();
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const f32x16& a = x ? dV[dt] : dK[dt];
        *reinterpret_cast<f32x4*>(&sh.sum[wave][(lane & 31) * kOutLd + 32 * dt + 2 * e + 4 * h32]) =
            f32x4{a[e], a[e + 1], a[e + 2], a[e + 3]};
      }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
      const int y = tid + 256 * u, at = y / (DP / 4) * kOutLd + y % (DP / 4) * 4;
      total[x][u] = *reinterpret_cast<f32x4*>(&sh.sum[0][at]);
#pragma unroll
      for (int w = 1; w < 4; ++w) total[x][u] += *reinterpret_cast<f32x4*>(&sh.sum[w][at]);
    }
  }
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    const int y = tid + 256 * u, key = y / (DP / 4), at = y % (DP / 4) * 4;
    if (SINKS) {
      float* out = p.sink_part + ((((int64_t)i * p.kv_heads + hk) * p.subs + sub) * p.pieces + piece) * 64 * DP;
      *reinterpret_cast<f32x4*>(out + key * DP + at) = total[0][u];
      *reinterpret_cast<f32x4*>(out + (32 + key) * DP + at) = total[1][u];
    } else if (jb + key < m && at < p.d) {
      if (part == 0 && p.split && jb + key < p.sinks && far < n) {
        const float* sum = p.sink_sum + (((int64_t)(i * p.kv_heads + hk) * p.subs + (jb >> 5)) * 64 + key) * DP + at;
        total[0][u] += *reinterpret_cast<const f32x4*>(sum);
        total[1][u] += *reinterpret_cast<const f32x4*>(sum + 32 * DP);
      }
      if (p.parts > 1) write_part(p, part, k0 + jb + key, hk, at, total[0][u], total[1][u]);
      else write_keys<T>(p, k0 + jb + key, hk, at, total[0][u], total[1][u]);
    }
  }
}

// The pieces' sums, added in order, four channels per thread: 5 .. 7 us, the latency of
// its loads.
template <int DP>
__global__ void __launch_bounds__(256)
sink_sum_kernel(WindowBwdParams p) {
  const int64_t item = block_id();
  if (item >= p.items) return;
  constexpr int kParts = 64 * DP / 1024;                   // workgroups per block of sinks
  const int part = (int)(item % kParts);
  const int64_t blk = item / kParts;
  const int sub = (int)(blk % p.subs), i = (int)(blk / p.subs / p.kv_heads);
  const int n = p.cu_q[i + 1] - p.cu_q[i], m = p.cu_k[i + 1] - p.cu_k[i], off = m - n;
  if (sub * 32 >= min(p.sinks, m)) return;
  const int jb = sub * 32 & ~127, jl = min(jb + 127, m - 1);
  const int ta = p.right >= 0 ? min(max(0, jb - p.right - off), n) : 0;
  const int64_t rows = (int64_t)(n - max(ta, window_end(jl, p.left, off, n))) * p.group;
  const int pieces = (int)((rows + p.piece - 1) / p.piece);
  const float* src = p.sink_part + blk * p.pieces * 64 * DP + part * 1024 + threadIdx.x * 4;
  f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int x = 0; x < pieces; ++x) a += *reinterpret_cast<const f32x4*>(src + (int64_t)x * 64 * DP);
  if (pieces > 0) *reinterpret_cast<f32x4*>(p.sink_sum + blk * 64 * DP + part * 1024 + threadIdx.x * 4) = a;
}

// How the sinks' part past the window is cut: pieces of at least kSinkPiece rows, or
// kSinkCut where those would leave compute units idle, fewer and longer ones where
// there are many blocks of sinks.  (N to 8192, 16 heads on 4 of 128, pieces of 512 and
// 256: 22 and 29 us; N 200 .. 1024, 8 on 2 of 64: 10 and 8; the backward of fp32, 2
// samples of 463, 3 heads on 1 of 128, window of 110 to both sides: 190 us in pieces of
// 512 and uncut parts, 137 with both.)
// The partial sums, two of 32 keys each for dK and dV per block at least, may take 64
// MB or as much as q, k and v in fp32; where blocks of short samples or of many sinks
// would take more, the keys' own workgroups walk all the rows.  (1100 samples of 40
// tokens and one of 20000, 4 sinks, 8 heads of 64: 553 us cut, 973 not; 1100 and one of
// 2000, 341 and 335.)
constexpr int kSinkPiece = 512, kSinkCut = 256, kSinkItems = 1024;
constexpr int64_t kSinkFloats = 1 << 24;

struct BackwardPlan {
  bool few_q, few_k;
  int parts;
  int split, subs, pieces, dp;
  int64_t piece;
  size_t delta_bytes, part_bytes, sum_bytes, key_bytes;
};

// Parts that the rows of a block of keys are cut into, where the blocks take few turns
// on the compute units and the last turn leaves many idle: a part keeps at least
// kPartRows rows, and each step up has to save a tenth of the turns.  Whole backward,
// uncut and cut: N 8192 and 4500, window 2048, 16 heads on 4 of 128 (400 blocks on 256
// places, 3 parts) 1070 and 961 us; N 9000 causal, 32 heads on 4 of 128 (284, 3 parts)
// 4037 and 2950; three of 4000, fp32, 16 heads on 4 of 64 (384, 2 parts) 7249 and 6048.
// Where the turns are even, four parts all the same: 8192 causal, 16 heads on 8 of 128
// (512 blocks) 1230 and 1347; four of 2048, every key (512) 587 and 700.
// Blocks of 32 keys are cut where they leave room, in parts of kFewPartRows: the join's
// launch has to pay (fp32, N 66 .. 317, 4 heads of 32, parts of 256: 34 and 40 us).
constexpr int kPartRows = 1024, kMostParts = 4, kFewPartRows = 512, kMostFewParts = 8;
int key_parts(const nt_window_args& a, int64_t blocks, bool few, int dp) {
  // workgroups that are resident, by registers
  const int64_t slots = 256 * (dp == 128 || (dp == 64 && a.dtype == NT_F32) ? 1 : dp == 64 ? 2 : 3);
  int64_t rows = 0;                                        // that a block of keys is seen by
  for (int32_t n : a.q_layout->lengths) rows = std::max<int64_t>(rows, n);
  if (a.left >= 0 && a.right >= 0) rows = std::min<int64_t>(rows, (int64_t)a.left + a.right + 128);
  rows *= a.heads / a.kv_heads;
  if (few) return (int)std::max<int64_t>(1, std::min({slots / std::max<int64_t>(1, blocks), rows / kFewPartRows, (int64_t)kMostFewParts}));
  int best = 1;
  double turns = (double)((blocks + slots - 1) / slots);
  for (int x = 2; x <= kMostParts && rows / x >= kPartRows; ++x) {
    const double t = (double)((blocks * x + slots - 1) / slots) / x;
    if (t < 0.9 * turns) best = x, turns = t;
  }
  return best;
}

BackwardPlan backward_plan(const nt_window_args& a) {
  BackwardPlan s{};
  const nt_layout &Lq = *a.q_layout, &Lk = *a.kv_layout;
  s.delta_bytes = ((size_t)a.heads * Lq.sum_n * sizeof(float) + 15) / 16 * 16;
  s.dp = a.head_dim <= 32 ? 32 : a.head_dim <= 64 ? 64 : 128;
  // blocks of 128 rows or keys, or of 32 where those would leave most of the card idle
  auto blocks_of = [&](const nt_layout& L, int mul, int shift) {
    int64_t n = 0;
    for (int32_t x : L.lengths) n += ((int64_t)x * mul + (1 << shift) - 1) >> shift;
    return n * a.kv_heads;
  };
  s.few_q = blocks_of(Lq, a.heads / a.kv_heads, kBlockShift) <= kFewRowBlocks;
  s.few_k = blocks_of(Lk, 1, kBlockShift) <= kFewKeyBlocks;
  s.parts = key_parts(a, blocks_of(Lk, 1, s.few_k ? kFewShift : kBlockShift), s.few_k, s.dp);
  if (s.parts > 1) s.key_bytes = (size_t)s.parts * 2 * Lk.sum_n * a.kv_heads * a.head_dim * sizeof(float);
  if (a.left < 0 || a.sinks == 0) return s;
  int64_t rows = 0;                                        // most rows past the window of the first keys
  for (int i = 0; i < Lq.batch; ++i) {
    const int64_t n = Lq.lengths[i], m = Lk.lengths[i];
    if (m == 0) continue;
    const int64_t end = (m < 128 ? m : 128) - 1 + a.left - (m - n) + 1;
    rows = std::max(rows, (n - std::max<int64_t>(0, std::min(n, end))) * (a.heads / a.kv_heads));
  }
  const int subs = (a.sinks + 31) / 32;
  const int64_t blocks = (int64_t)Lq.batch * a.kv_heads * subs;
  const int64_t operands = (Lq.sum_n * a.heads + 2 * Lk.sum_n * a.kv_heads) * a.head_dim;
  if (rows <= kSinkPiece || blocks * 128 * s.dp > std::max(kSinkFloats, operands)) return s;
  s.split = 1;
  s.subs = subs;
  const int64_t cut = blocks * (rows / kSinkPiece) < 256 ? kSinkCut : kSinkPiece;
  const int64_t want = std::max<int64_t>(1, std::min(rows / cut, kSinkItems / blocks));
  s.piece = ((rows + want - 1) / want + 127) / 128 * 128;
  s.pieces = (int)((rows + s.piece - 1) / s.piece);
  s.part_bytes = (size_t)blocks * s.pieces * 64 * s.dp * sizeof(float);
  s.sum_bytes = (size_t)blocks * 64 * s.dp * sizeof(float);
  return s;
}

template <typename T, int DP>
hipError_t launch_backward(WindowBwdParams p, const BackwardPlan& w, const nt_layout& Lq, const nt_layout& Lk,
                           hipStream_t s) {
  auto items = [&](const nt_layout& L, int mul, int shift) {
    return L.sum_n ? block_count(L.sum_n, L.batch, mul, shift) * p.kv_heads : 0;
  };
  p.items = items(Lq, p.group, w.few_q ? kFewShift : kBlockShift);
  if (p.items > 0) {
    if (w.few_q) window_dq_few_kernel<T, DP><<<folded_grid(p.items), 256, 0, s>>>(p);
    else window_dq_kernel<T, DP><<<folded_grid(p.items), 256, 0, s>>>(p);
  }
  if (hipError_t e = hipGetLastError()) return e;
  if (p.split) {
    p.items = (int64_t)p.batch * p.kv_heads * p.subs * p.pieces;
    window_dkv_few_kernel<T, DP, true><<<folded_grid(p.items), 256, 0, s>>>(p);
    if (hipError_t e = hipGetLastError()) return e;
    p.items = (int64_t)p.batch * p.kv_heads * p.subs * (64 * DP / 1024);
    sink_sum_kernel<DP><<<folded_grid(p.items), 256, 0, s>>>(p);
    if (hipError_t e = hipGetLastError()) return e;
  }
  p.items = items(Lk, 1, w.few_k ? kFewShift : kBlockShift) * p.parts;
  if (p.items > 0) {
    if (w.few_k) window_dkv_few_kernel<T, DP, false><<<folded_grid(p.items), 256, 0, s>>>(p);
    else window_dkv_kernel<T, DP><<<folded_grid(p.items), 256, 0, s>>>(p);
  }
  if (hipError_t e = hipGetLastError()) return e;
  if (p.parts > 1) {
    p.items = (p.sum_k * p.kv_heads * (p.d / 4) + 255) / 256;
    key_join_kernel<T><<<folded_grid(p.items), 256, 0, s>>>(p);
  }
  return hipGetLastError();
}

}  // namespace

size_t window_backward_workspace_bytes(const nt_window_args& a) {
  const BackwardPlan s = backward_plan(a);
  return s.delta_bytes + s.part_bytes + s.sum_bytes + s.key_bytes;
}

hipError_t launch_window_backward(const nt_window_args& a, hipStream_t s) {
  const nt_layout &Lq = *a.q_layout, &Lk = *a.kv_layout;
  WindowBwdParams p{};
  p.cu_q = Lq.d_cu_seqlens;
  p.cu_k = Lk.d_cu_seqlens;
  p.batch = Lq.batch;
  p.heads = a.heads;
  p.kv_heads = a.kv_heads;
  p.group = a.heads / a.kv_heads;
  p.d = a.head_dim;
  p.left = a.left;
  p.right = a.right;
  p.sinks = a.sinks;
  p.scale = a.scale;
  p.inv_group = 1.f / (float)p.group;
  p.c = a.scale == 0.f ? 1.f : fabsf(a.scale) * win::kLog2e;
  p.qmul = a.scale == 0.f ? 0.f : a.scale < 0.f ? -1.f : 1.f;
  p.q = a.q; p.k = a.k; p.v = a.v; p.o = a.o; p.dout = a.dout;
  p.dq = a.dq; p.dk = a.dk; p.dv = a.dv;
  p.ld_q = a.ld_q; p.ld_k = a.ld_k; p.ld_v = a.ld_v; p.ld_o = a.ld_o; p.ld_dout = a.ld_dout;
  p.ld_dq = a.ld_dq; p.ld_dk = a.ld_dk; p.ld_dv = a.ld_dv; p.ld_lse = a.ld_lse;
  p.lse = a.lse;
  p.delta = (float*)a.workspace;
  p.sum_q = Lq.sum_n;
  const BackwardPlan sp = backward_plan(a);
  p.parts = sp.parts;
  p.sum_k = Lk.sum_n;
  p.split = sp.split;
  p.subs = sp.subs;
  p.pieces = sp.pieces;
  p.piece = sp.piece;
  p.sink_part = (float*)((char*)a.workspace + sp.delta_bytes);
  p.sink_sum = (float*)((char*)a.workspace + sp.delta_bytes + sp.part_bytes);
  p.key_part = (float*)((char*)a.workspace + sp.delta_bytes + sp.part_bytes + sp.sum_bytes);
  const bool bf = a.dtype == NT_BF16;
  const int size = bf ? 2 : 4;
  p.narrow = win::narrow_stride(a.ld_q, size) && win::narrow_stride(a.ld_dout, size) &&
             win::narrow_stride(a.ld_k, size) && win::narrow_stride(a.ld_v, size);
  if (p.d <= 32) return bf ? launch_backward<bf16, 32>(p, sp, Lq, Lk, s) : launch_backward<float, 32>(p, sp, Lq, Lk, s);
  if (p.d <= 64) return bf ? launch_backward<bf16, 64>(p, sp, Lq, Lk, s) : launch_backward<float, 64>(p, sp, Lq, Lk, s);
  return bf ? launch_backward<bf16, 128>(p, sp, Lq, Lk, s) : launch_backward<float, 128>(p, sp, Lq, Lk, s);
}

}  // namespace nt
