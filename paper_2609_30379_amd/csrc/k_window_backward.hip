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
#include <type_traits>

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
  // gradients of the sinks from the queries past their window (window_sink_kernel)
  int split;                     // done apart, in pieces of `piece` rows
  int subs, pieces, piece;       // blocks of 32 sinks, most pieces of a sample, rows per piece
  float *sink_part, *sink_sum;   // [batch][kv_heads][subs][pieces][2][32][DP], [batch][kv_heads][subs][2][32][DP]
};

// First query past the window of the keys jb .. jl; the queries before it are
// gone through by the keys' own workgroup.
__device__ __forceinline__ int window_end(int jl, int left, int off, int n) { return min(n, max(0, jl + left - off + 1)); }

constexpr int kBlockShift = 7;

template <typename T, int DP>
__global__ void __launch_bounds__(256, DP == 32 ? 3 : DP == 128 ? 1 : 2)
window_dq_kernel(WindowBwdParams p) {
  typedef typename Frag<T>::type frag;
  constexpr int KT = sizeof(T) == 2 ? 64 : 32, KB = KT / 32, NS = DP / 16, ND = DP / 32;
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
  {
    const T* src = (const T*)p.q + (int64_t)(q0 + t) * p.ld_q + (int64_t)head * p.d;
    const T* dsrc = (const T*)p.dout + (int64_t)(q0 + t) * p.ld_dout + (int64_t)head * p.d;
    const T* osrc = (const T*)p.o + (int64_t)(q0 + t) * p.ld_o + (int64_t)head * p.d;
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
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
  Stage<T, DP, KT, 256> sk, sv;
  auto load = [&](int tile) {
    const int j0 = kt.first(tile, KT), cnt = min(kt.end(tile) - j0, KT);
    sk.load(tid, kbase + (int64_t)(k0 + j0) * p.ld_k, p.ld_k, cnt, p.d, p.narrow);
    sv.load(tid, vbase + (int64_t)(k0 + j0) * p.ld_v, p.ld_v, cnt, p.d, p.narrow);
  };
  if (kt.n > 0) {
    load(0);
    sk.store(tid, Kb[0]);
    sv.store(tid, Vb[0]);
  }
  for (int tile = 0; tile < kt.n; ++tile) {
    __syncthreads();
    const T *Ks = Kb[tile & 1], *Vs = Vb[tile & 1];
    if (tile + 1 < kt.n) load(tile + 1);
    const int j0 = kt.first(tile, KT), jend = kt.end(tile);
    if (live && j0 <= hi_b && (min(j0 + KT, jend) > lo_a || j0 < p.sinks)) {
    const bool whole = j0 + KT <= jend && j0 + KT - 1 <= hi_a && (j0 >= lo_b || j0 + KT <= p.sinks);
    // Block by block of 32 keys, the reads of a step before the products of the
    // one before; a hidden pair's score starts from -inf, dP from -D.
    frag A[NS], B[NS], X[ND], Y[ND];
    read_along<DP>(Ks, 0, lane, A);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      f32x16 S = f32x16{}, dP;
      if (!whole) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = j0 + 32 * kb + 8 * (e >> 2) + 4 * h32 + (e & 3);
          S[e] = j < jend && j <= hi && (j >= lo || j < p.sinks) ? 0.f : -INFINITY;
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) dP[e] = -delta;
      pin();
      read_along<DP>(Vs, 32 * kb, lane, B);
      pin();
      S = product(A, Q, S);
      pin();
      read_across<DP>(Ks, 32 * kb, lane, tr, X);
      pin();
      dP = product(B, G, dP);
#pragma unroll
      for (int e = 0; e < 16; ++e) S[e] = __builtin_amdgcn_exp2f(fmaf(S[e], p.c, nlse2));
      pin();
      read_across<DP>(Ks, 32 * kb + 16, lane, tr, Y);
      pin();
#pragma unroll
      for (int e = 0; e < 16; ++e) S[e] *= dP[e];
      frag D;
      to_operand(S, 0, D);
      add_products(X, D, dQ);
      to_operand(S, 1, D);
      pin();
      if (kb + 1 < KB) read_along<DP>(Ks, 32 * kb + 32, lane, A);
      pin();
      add_products(Y, D, dQ);
    }
    }
    if (tile + 1 < kt.n) {
      sk.store(tid, Kb[~tile & 1]);
      sv.store(tid, Vb[~tile & 1]);
    }
  }
  if (!mine) return;
  T* dst = (T*)p.dq + (int64_t)(q0 + t) * p.ld_dq + (int64_t)head * p.d;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int at = 32 * dt + 2 * e + 4 * h32;
      if (at < p.d) {
        typedef T vec4 __attribute__((ext_vector_type(4)));
        vec4 w;
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = (T)(dQ[dt][e + u] * p.scale);
        *reinterpret_cast<vec4*>(dst + at) = w;
      }
    }
}

template <typename T, int DP>
__global__ void __launch_bounds__(256, DP == 128 || (DP == 64 && sizeof(T) == 4) ? 1 : 2)
window_dkv_kernel(WindowBwdParams p) {
  typedef typename Frag<T>::type frag;
  constexpr int RT = sizeof(T) == 2 ? 64 : 32, RB = RT / 32, NS = DP / 16, ND = DP / 32;
  __shared__ __attribute__((aligned(16))) T Qb[2][RT * Tile<T, DP>::kLd];
  __shared__ __attribute__((aligned(16))) T Gb[2][RT * Tile<T, DP>::kLd];
  __shared__ __attribute__((aligned(16))) float lse_b[2][RT];
  __shared__ __attribute__((aligned(16))) float delta_b[2][RT];
  __shared__ __attribute__((aligned(16))) int pos_b[2][RT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h32 = lane >> 5;
  const int64_t item = block_id();
  if (item >= p.items) return;
  const int hk = (int)(item % p.kv_heads);
  const int64_t b = item / p.kv_heads;
  const int i = find_sample(p.cu_k, p.batch, 1, kBlockShift, b, lane);
  const int q0 = p.cu_q[i], n = p.cu_q[i + 1] - q0, k0 = p.cu_k[i], m = p.cu_k[i + 1] - k0;
  const int64_t jb64 = (b - block_start(p.cu_k, i, 1, kBlockShift)) << kBlockShift;
  if (jb64 >= m) return;
  const int jb = (int)jb64, jl = min(jb + 127, m - 1);          // keys jb .. jl
  const int off = m - n;
  const int j = min(jb + wave * 32 + (lane & 31), m - 1);       // a lane past the last key takes the last one, not stored
  const bool live = jb + wave * 32 < m, mine = jb + wave * 32 + (lane & 31) < m;
  // positions of the rows that see key j
  const int plo = p.right >= 0 ? j - p.right : INT32_MIN + 1;
  const int phi = p.left >= 0 && j >= p.sinks ? j + p.left : INT32_MAX;

  // the same bounds over the wave's keys
  const int ja = min(jb + wave * 32, m - 1), je = min(jb + wave * 32 + 31, m - 1);
  const int plo_a = p.right >= 0 ? ja - p.right : INT32_MIN + 1, plo_b = p.right >= 0 ? je - p.right : INT32_MIN + 1;
  const int phi_a = p.left >= 0 && je >= p.sinks ? max(ja, p.sinks) + p.left : INT32_MAX;
  const int phi_b = p.left >= 0 && ja >= p.sinks ? je + p.left : INT32_MAX;

  frag K[NS], V[NS];
  {
    const T* ksrc = (const T*)p.k + (int64_t)(k0 + j) * p.ld_k + (int64_t)hk * p.d;
    const T* vsrc = (const T*)p.v + (int64_t)(k0 + j) * p.ld_v + (int64_t)hk * p.d;
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
      const int e = 16 * ks + 8 * h32;
      frag z = {};
      K[ks] = e < p.d ? *reinterpret_cast<const frag*>(ksrc + e) : z;
      V[ks] = e < p.d ? *reinterpret_cast<const frag*>(vsrc + e) : z;
    }
    multiply<T>(K, p.qmul);
  }
  uint32_t tr[2];
  Tile<T, DP>::across_addr(lane, tr);
  f32x16 dK[ND], dV[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) dK[dt] = dV[dt] = f32x16{};

  // queries that see a key of the block, as rows [ra, rb)
  const int ta = p.right >= 0 ? min(max(0, jb - p.right - off), n) : 0;
  const int tb = p.left >= 0 && (jb >= p.sinks || p.split) ? window_end(jl, p.left, off, n) : n;
  const int64_t ra = (int64_t)ta * p.group, rb = (int64_t)max(ta, tb) * p.group;
  const int tiles = (int)((rb - ra + RT - 1) / RT);
  Stage<T, DP, RT, 256> sq, sg;
  float r_lse = 0.f, r_delta = 0.f;
  int r_pos = 0;
  // the tile's first row as (t0, g0), moved on by RT rows per tile
  const int step_t = RT / p.group, step_g = RT - step_t * p.group;
  int lt0 = ta, lg0 = 0;
  int64_t left_rows = rb - ra;
  auto load = [&]() {
    const int cnt = (int)min((int64_t)RT, left_rows), queries = min(tb - lt0, RT + 1);
    const int first = q0 + lt0, h0 = hk * p.group;
    sq.load_group(tid, (const T*)p.q + (int64_t)first * p.ld_q + (int64_t)h0 * p.d, p.ld_q, queries, lg0, p.group,
                  p.inv_group, p.d, p.narrow);
    sg.load_group(tid, (const T*)p.dout + (int64_t)first * p.ld_dout + (int64_t)h0 * p.d, p.ld_dout, queries, lg0,
                  p.group, p.inv_group, p.d, p.narrow);
    if (tid < RT) {
      const int r = min(tid, cnt - 1), tg = div_group(lg0 + r, p.inv_group), head = h0 + lg0 + r - tg * p.group;
      r_lse = p.lse[(int64_t)head * p.ld_lse + first + tg];
      r_delta = p.delta[(int64_t)head * p.sum_q + first + tg];
      r_pos = tid < cnt ? off + lt0 + tg : INT32_MIN;           // no key sees a row past the end
    }
    left_rows -= RT;
    lt0 += step_t;
    lg0 += step_g;
    if (lg0 >= p.group) {
      lg0 -= p.group;
      ++lt0;
    }
  };
  auto store = [&](int buf) {
    sq.store(tid, Qb[buf]);
    sg.store(tid, Gb[buf]);
    if (tid < RT) {
      lse_b[buf][tid] = r_lse == -INFINITY ? 0.f : r_lse * -kLog2e;   // -inf: a row that sees nothing
      delta_b[buf][tid] = -r_delta;
      pos_b[buf][tid] = r_pos;
    }
  };
  int nt0 = ta, ng0 = 0;                                        // the tile that is worked on next
  if (tiles > 0) {
    load();
    store(0);
  }
  for (int tile = 0; tile < tiles; ++tile) {
    __syncthreads();
    const T *Qs = Qb[tile & 1], *Gs = Gb[tile & 1];
    const float *lse_s = lse_b[tile & 1], *delta_s = delta_b[tile & 1];
    const int* pos_s = pos_b[tile & 1];
    const int cur_rows = (int)min((int64_t)RT, rb - ra - (int64_t)tile * RT);
    const int pa = off + nt0, pe = off + nt0 + (ng0 + cur_rows - 1) / p.group;
    nt0 = lt0;
    ng0 = lg0;
    if (tile + 1 < tiles) load();
    if (live && pe >= plo_a && pa <= phi_b) {
    const bool whole = cur_rows == RT && pa >= plo_b && pe <= phi_a;
    // One 32-row block after the other; each step issues the reads of the next
    // one before its products, and the exponentials and score gradients run
    // under products.  A hidden pair's score starts from -inf, so its weight is 0;
    // dP starts from -D.
    frag A[NS], B[NS], X[ND], Y[ND];
    read_along<DP>(Qs, 0, lane, A);
#pragma unroll
    for (int rbk = 0; rbk < RB; ++rbk) {
      const int r0 = 32 * rbk;
      f32x16 S = f32x16{}, dP;
      if (!whole) {
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const int4 ps = *reinterpret_cast<const int4*>(pos_s + r0 + 8 * e4 + 4 * h32);
          const int pr[4] = {ps.x, ps.y, ps.z, ps.w};
#pragma unroll
          for (int u = 0; u < 4; ++u) S[4 * e4 + u] = pr[u] >= plo && pr[u] <= phi ? 0.f : -INFINITY;
        }
      }
      pin();
      read_along<DP>(Gs, r0, lane, B);
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4) {
        const f32x4 de = *reinterpret_cast<const f32x4*>(delta_s + r0 + 8 * e4 + 4 * h32);
#pragma unroll
        for (int u = 0; u < 4; ++u) dP[4 * e4 + u] = de[u];
      }
      pin();
      S = product(A, K, S);
      pin();
      read_across<DP>(Gs, r0, lane, tr, X);
      pin();
      dP = product(B, V, dP);
      frag W, D;
#pragma unroll
      for (int e4 = 0; e4 < 4; ++e4) {
        const f32x4 ls = *reinterpret_cast<const f32x4*>(lse_s + r0 + 8 * e4 + 4 * h32);
#pragma unroll
        for (int u = 0; u < 4; ++u) S[4 * e4 + u] = __builtin_amdgcn_exp2f(fmaf(S[4 * e4 + u], p.c, ls[u]));
      }
      to_operand(S, 0, W);
      pin();
      read_across<DP>(Gs, r0 + 16, lane, tr, Y);
      pin();
      add_products(X, W, dV);
#pragma unroll
      for (int e = 0; e < 16; ++e) dP[e] *= S[e];
      to_operand(S, 1, W);
      pin();
      read_across<DP>(Qs, r0, lane, tr, X);
      pin();
      add_products(Y, W, dV);
      to_operand(dP, 0, D);
      pin();
      read_across<DP>(Qs, r0 + 16, lane, tr, Y);
      pin();
      add_products(X, D, dK);
      to_operand(dP, 1, D);
      pin();
      if (rbk + 1 < RB) read_along<DP>(Qs, r0 + 32, lane, A);
      pin();
      add_products(Y, D, dK);
    }
    }
    if (tile + 1 < tiles) store(~tile & 1);
  }
  if (!mine) return;
  if (p.split && j < p.sinks && max(ta, tb) < n) {         // what the queries past the window add to a sink
    const float* sum = p.sink_sum + (((int64_t)(i * p.kv_heads + hk) * p.subs + (j >> 5)) * 64 + (j & 31)) * DP;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int at = 32 * dt + 2 * e + 4 * h32;
        const f32x4 a = *reinterpret_cast<const f32x4*>(sum + at), w = *reinterpret_cast<const f32x4*>(sum + 32 * DP + at);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          dK[dt][e + u] += a[u];
          dV[dt][e + u] += w[u];
        }
      }
  }
  T* kd = (T*)p.dk + (int64_t)(k0 + j) * p.ld_dk + (int64_t)hk * p.d;
  T* vd = (T*)p.dv + (int64_t)(k0 + j) * p.ld_dv + (int64_t)hk * p.d;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int at = 32 * dt + 2 * e + 4 * h32;
      if (at < p.d) {
        typedef T vec4 __attribute__((ext_vector_type(4)));
        vec4 a, w;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          a[u] = (T)(dK[dt][e + u] * p.scale);
          w[u] = (T)dV[dt][e + u];
        }
        *reinterpret_cast<vec4*>(kd + at) = a;
        *reinterpret_cast<vec4*>(vd + at) = w;
      }
    }
}

// The sinks' gradients from the queries past their window: few keys and all the
// later rows of the sample, which one workgroup per block of keys would walk
// alone while the others have left.  A workgroup takes 32 sinks and a piece of
// the rows, 32 rows of each tile of 128 per wave; every row sees every sink here,
// so there is no mask.  The waves' sums are added in order through LDS, the
// pieces' by sink_sum_kernel.
template <typename T, int DP>
__global__ void __launch_bounds__(256)
window_sink_kernel(WindowBwdParams p) {
  typedef typename Frag<T>::type frag;
  constexpr int RT = 128, NS = DP / 16, ND = DP / 32;
  union Shared {
    struct {
      T q[RT * Tile<T, DP>::kLd], g[RT * Tile<T, DP>::kLd];
      float lse[RT], delta[RT];
    } t;
    float sum[4][32 * DP];
  };
  __shared__ __attribute__((aligned(16))) Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h32 = lane >> 5;
  const int64_t item = block_id();
  if (item >= p.items) return;
  const int hk = (int)(item % p.kv_heads), piece = (int)(item / p.kv_heads % p.pieces);
  const int sub = (int)(item / p.kv_heads / p.pieces % p.subs), i = (int)(item / p.kv_heads / p.pieces / p.subs);
  const int q0 = p.cu_q[i], n = p.cu_q[i + 1] - q0, k0 = p.cu_k[i], m = p.cu_k[i + 1] - k0, off = m - n;
  const int sinks = min(p.sinks, m);
  if (sub * 32 >= sinks) return;
  const int jb = sub * 32 & ~127, jl = min(jb + 127, m - 1);
  const int ta = p.right >= 0 ? min(max(0, jb - p.right - off), n) : 0;
  const int64_t ra = (int64_t)max(ta, window_end(jl, p.left, off, n)) * p.group + (int64_t)piece * p.piece;
  const int64_t rb = min((int64_t)n * p.group, ra + p.piece);
  if (ra >= rb) return;
  const int j = min(sub * 32 + (lane & 31), sinks - 1);
  frag K[NS], V[NS];
  {
    const T* ksrc = (const T*)p.k + (int64_t)(k0 + j) * p.ld_k + (int64_t)hk * p.d;
    const T* vsrc = (const T*)p.v + (int64_t)(k0 + j) * p.ld_v + (int64_t)hk * p.d;
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
      const int e = 16 * ks + 8 * h32;
      frag z = {};
      K[ks] = e < p.d ? *reinterpret_cast<const frag*>(ksrc + e) : z;
      V[ks] = e < p.d ? *reinterpret_cast<const frag*>(vsrc + e) : z;
    }
    multiply<T>(K, p.qmul);
  }
  uint32_t tr[2];
  Tile<T, DP>::across_addr(lane, tr);
  f32x16 dK[ND], dV[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) dK[dt] = dV[dt] = f32x16{};
  Stage<T, DP, RT, 256> sq, sg;
  for (int64_t r0 = ra; r0 < rb; r0 += RT) {
    const int t0 = (int)(r0 / p.group), g0 = (int)(r0 - (int64_t)t0 * p.group);
    const int cnt = (int)min((int64_t)RT, rb - r0), first = q0 + t0, h0 = hk * p.group;
    const int queries = min(n - t0, RT + 1);
    sq.load_group(tid, (const T*)p.q + (int64_t)first * p.ld_q + (int64_t)h0 * p.d, p.ld_q, queries, g0, p.group,
                  p.inv_group, p.d, p.narrow);
    sg.load_group(tid, (const T*)p.dout + (int64_t)first * p.ld_dout + (int64_t)h0 * p.d, p.ld_dout, queries, g0, p.group,
                  p.inv_group, p.d, p.narrow);
    float lse2 = INFINITY, delta = 0.f;                    // a row past the piece has weight 0
    if (tid < cnt) {
      const int tg = div_group(g0 + tid, p.inv_group), head = h0 + g0 + tid - tg * p.group;
      lse2 = p.lse[(int64_t)head * p.ld_lse + first + tg] * kLog2e;
      delta = p.delta[(int64_t)head * p.sum_q + first + tg];
    }
    __syncthreads();
    sq.store(tid, sh.t.q);
    sg.store(tid, sh.t.g);
    if (tid < RT) {
      sh.t.lse[tid] = lse2;
      sh.t.delta[tid] = delta;
    }
    __syncthreads();
    const int rw = 32 * wave;
    if (rw >= cnt) continue;
    f32x16 S = f32x16{}, dP = f32x16{};
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
      S = mma32(Tile<T, DP>::along(sh.t.q, rw, ks, lane), K[ks], S);
      dP = mma32(Tile<T, DP>::along(sh.t.g, rw, ks, lane), V[ks], dP);
    }
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const int r = rw + 8 * e4 + 4 * h32;
      const f32x4 ls = *reinterpret_cast<const f32x4*>(sh.t.lse + r), de = *reinterpret_cast<const f32x4*>(sh.t.delta + r);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float w = __builtin_amdgcn_exp2f(fmaf(S[4 * e4 + u], p.c, -ls[u]));
        S[4 * e4 + u] = w;
        dP[4 * e4 + u] = w * (dP[4 * e4 + u] - de[u]);
      }
    }
#pragma unroll
    for (int nn = 0; nn < 2; ++nn) {
      frag W, D;
      to_operand(S, nn, W);
      to_operand(dP, nn, D);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        dV[dt] = mma32(across<DP>(sh.t.g, rw + 16 * nn, dt, lane, tr), W, dV[dt]);
        dK[dt] = mma32(across<DP>(sh.t.q, rw + 16 * nn, dt, lane, tr), D, dK[dt]);
      }
    }
  }
  float* out = p.sink_part + ((((int64_t)i * p.kv_heads + hk) * p.subs + sub) * p.pieces + piece) * 64 * DP;
#pragma unroll
  for (int x = 0; x < 2; ++x) {                            // dK, then dV
    __syncthreads();
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const f32x16& a = x ? dV[dt] : dK[dt];
        *reinterpret_cast<f32x4*>(&sh.sum[wave][(lane & 31) * DP + 32 * dt + 2 * e + 4 * h32]) =
            f32x4{a[e], a[e + 1], a[e + 2], a[e + 3]};
      }
    __syncthreads();
    for (int u = tid * 4; u < 32 * DP; u += 1024) {
      f32x4 a = *reinterpret_cast<f32x4*>(&sh.sum[0][u]);
#pragma unroll
      for (int w = 1; w < 4; ++w) a += *reinterpret_cast<f32x4*>(&sh.sum[w][u]);
      *reinterpret_cast<f32x4*>(out + x * 32 * DP + u) = a;
    }
  }
}

// The pieces' sums, added in order.
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

// How the sinks' part past the window is cut: pieces of at least kSinkPiece rows,
// fewer and longer ones where there are many blocks of sinks, so that the partial
// sums stay bounded.
constexpr int kSinkPiece = 512, kSinkItems = 1024;
struct SinkPlan {
  int split, subs, pieces, piece, dp;
  size_t delta_bytes, part_bytes, sum_bytes;
};
SinkPlan sink_plan(const nt_window_args& a) {
  SinkPlan s{};
  const nt_layout &Lq = *a.q_layout, &Lk = *a.kv_layout;
  s.delta_bytes = ((size_t)a.heads * Lq.sum_n * sizeof(float) + 15) / 16 * 16;
  s.dp = a.head_dim <= 32 ? 32 : a.head_dim <= 64 ? 64 : 128;
  if (a.left < 0 || a.sinks == 0) return s;
  int64_t rows = 0;                                        // most rows past the window of the first keys
  for (int i = 0; i < Lq.batch; ++i) {
    const int64_t n = Lq.lengths[i], m = Lk.lengths[i];
    if (m == 0) continue;
    const int64_t end = (m < 128 ? m : 128) - 1 + a.left - (m - n) + 1;
    rows = std::max(rows, (n - std::max<int64_t>(0, std::min(n, end))) * (a.heads / a.kv_heads));
  }
  if (rows <= kSinkPiece) return s;
  s.split = 1;
  s.subs = (a.sinks + 31) / 32;
  const int64_t blocks = (int64_t)Lq.batch * a.kv_heads * s.subs;
  const int64_t want = std::max<int64_t>(1, std::min(rows / kSinkPiece, kSinkItems / blocks));
  s.piece = (int)((rows + want - 1) / want + 127) / 128 * 128;
  s.pieces = (int)((rows + s.piece - 1) / s.piece);
  s.part_bytes = (size_t)blocks * s.pieces * 64 * s.dp * sizeof(float);
  s.sum_bytes = (size_t)blocks * 64 * s.dp * sizeof(float);
  return s;
}

template <typename T, int DP>
hipError_t launch_backward(WindowBwdParams p, int64_t q_items, int64_t k_items, hipStream_t s) {
  p.items = q_items;
  if (q_items > 0) window_dq_kernel<T, DP><<<folded_grid(q_items), 256, 0, s>>>(p);
  if (hipError_t e = hipGetLastError()) return e;
  if (p.split) {
    p.items = (int64_t)p.batch * p.kv_heads * p.subs * p.pieces;
    window_sink_kernel<T, DP><<<folded_grid(p.items), 256, 0, s>>>(p);
    if (hipError_t e = hipGetLastError()) return e;
    p.items = (int64_t)p.batch * p.kv_heads * p.subs * (64 * DP / 1024);
    sink_sum_kernel<DP><<<folded_grid(p.items), 256, 0, s>>>(p);
    if (hipError_t e = hipGetLastError()) return e;
  }
  p.items = k_items;
  if (k_items > 0) window_dkv_kernel<T, DP><<<folded_grid(k_items), 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

size_t window_backward_workspace_bytes(const nt_window_args& a) {
  const SinkPlan s = sink_plan(a);
  return s.delta_bytes + s.part_bytes + s.sum_bytes;
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
  const SinkPlan sp = sink_plan(a);
  p.split = sp.split;
  p.subs = sp.subs;
  p.pieces = sp.pieces;
  p.piece = sp.piece;
  p.sink_part = (float*)((char*)a.workspace + sp.delta_bytes);
  p.sink_sum = (float*)((char*)a.workspace + sp.delta_bytes + sp.part_bytes);
  const int64_t qi = Lq.sum_n ? win::block_count(Lq.sum_n, Lq.batch, p.group, kBlockShift) * p.kv_heads : 0;
  const int64_t ki = Lk.sum_n ? win::block_count(Lk.sum_n, Lk.batch, 1, kBlockShift) * p.kv_heads : 0;
  const bool bf = a.dtype == NT_BF16;
  const int size = bf ? 2 : 4;
  p.narrow = win::narrow_stride(a.ld_q, size) && win::narrow_stride(a.ld_dout, size) &&
             win::narrow_stride(a.ld_k, size) && win::narrow_stride(a.ld_v, size);
  if (p.d <= 32) return bf ? launch_backward<bf16, 32>(p, qi, ki, s) : launch_backward<float, 32>(p, qi, ki, s);
  if (p.d <= 64) return bf ? launch_backward<bf16, 64>(p, qi, ki, s) : launch_backward<float, 64>(p, qi, ki, s);
  return bf ? launch_backward<bf16, 128>(p, qi, ki, s) : launch_backward<float, 128>(p, qi, ki, s);
}

}  // namespace nt
