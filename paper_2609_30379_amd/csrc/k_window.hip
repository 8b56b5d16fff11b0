// Sliding-window attention over the packed tokens of each sample, with a few
// first keys that stay visible and shared key/value heads (window_device.h).
//
//   s_j = scale q . k_j,  o = sum_j exp(s_j - m) v_j / l,  lse = m + log l
// over the visible keys j of a query, m the running maximum and l the running
// sum of one pass over the keys.  A wave holds 32 query rows as columns of the
// products S^T = K Q^T and O^T = V^T P^T, so that a row's scores, maximum and
// sum stay in two lanes and the weights P^T go from the accumulators of the
// first product into the operand of the second without leaving the registers.
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
};

constexpr int kBlockShift = 7;                 // query rows per workgroup: 4 waves x 32

template <typename T, int DP>
__global__ void __launch_bounds__(256, DP == 128 ? 2 : 3)
window_rows_kernel(WindowParams p) {
  typedef typename Frag<T>::type frag;
  constexpr int KT = sizeof(T) == 2 ? 64 : 32, KB = KT / 32, NS = DP / 16, ND = DP / 32;
  __shared__ __attribute__((aligned(16))) T Ks[KT * Tile<T, DP>::kLd];
  __shared__ __attribute__((aligned(16))) T Vs[KT * Tile<T, DP>::kLd];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h32 = lane >> 5;
  const int64_t item = block_id();
  if (item >= p.items) return;
  const int hk = (int)(item % p.kv_heads);
  const int64_t b = item / p.kv_heads;
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

  frag Q[NS];
  {
    const T* src = (const T*)p.q + (int64_t)(q0 + t) * p.ld_q + (int64_t)(hk * p.group + g) * p.d;
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
      const int e = 16 * ks + 8 * h32;
      frag z = {};
      Q[ks] = e < p.d ? *reinterpret_cast<const frag*>(src + e) : z;
    }
    if (p.qmul != 1.f)
#pragma unroll
      for (int ks = 0; ks < NS; ++ks)
#pragma unroll
        for (int u = 0; u < 8; ++u) Q[ks][u] = (T)((float)Q[ks][u] * p.qmul);
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
  Stage<T, DP, KT, 256> sk, sv;
  auto load = [&](int tile) {
    const int j0 = kt.first(tile, KT), cnt = kt.end(tile) - j0;
    sk.load(tid, cnt, p.d, [&](int r) { return kbase + (int64_t)(k0 + j0 + r) * p.ld_k; });
    sv.load(tid, cnt, p.d, [&](int r) { return vbase + (int64_t)(k0 + j0 + r) * p.ld_v; });
  };
  if (kt.n > 0) load(0);
  for (int tile = 0; tile < kt.n; ++tile) {
    __syncthreads();
    sk.store(tid, Ks);
    sv.store(tid, Vs);
    __syncthreads();
    const int j0 = kt.first(tile, KT), jend = kt.end(tile);
    if (tile + 1 < kt.n) load(tile + 1);
    if (!live) continue;
    // nothing of the tile visible to any row of the wave, or all of it to all
    const int je = min(j0 + KT, jend);
    if (!__any(j0 <= hi && (je > lo || j0 < p.sinks))) continue;
    const bool whole = __all(j0 + KT <= jend && j0 + KT - 1 <= hi && (j0 >= lo || j0 + KT <= p.sinks));
    f32x16 S[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      S[kb] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < NS; ++ks) S[kb] = mma32(Tile<T, DP>::along(Ks, 32 * kb, ks, lane), Q[ks], S[kb]);
    }
    if (!whole)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = j0 + 32 * kb + 8 * (e >> 2) + 4 * h32 + (e & 3);
          S[kb][e] = j < jend && j <= hi && (j >= lo || j < p.sinks) ? S[kb][e] : -INFINITY;
        }
    float top = S[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, S[kb][e]);
    top *= p.c;
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
        S[kb][e] = __builtin_amdgcn_exp2f(fmaf(S[kb][e], p.c, -sub));
        sum += S[kb][e];
      }
    l += sum;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int nn = 0; nn < 2; ++nn) {
        frag P;
        to_operand(S[kb], nn, P);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
          O[dt] = mma32(across<DP>(Vs, 32 * kb + 16 * nn, dt, lane, tr), P, O[dt]);
      }
  }

  if (wave * 32 + (lane & 31) > last) return;
  l = pair_sum(l);
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const int head = hk * p.group + g;
  T* dst = (T*)p.o + (int64_t)(q0 + t) * p.ld_o + (int64_t)head * p.d;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const int at = 32 * dt + 2 * e + 4 * h32;
      if (at < p.d) {
        typedef T vec4 __attribute__((ext_vector_type(4)));
        vec4 w;
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = (T)(O[dt][e + u] * inv);
        *reinterpret_cast<vec4*>(dst + at) = w;
      }
    }
  if (p.lse && h32 == 0)
    p.lse[(int64_t)head * p.ld_lse + q0 + t] = l > 0.f ? (mx + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

template <typename T, int DP>
hipError_t launch_rows(const WindowParams& p, hipStream_t s) {
  window_rows_kernel<T, DP><<<folded_grid(p.items), 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

size_t window_workspace_bytes(const nt_window_args& a) { return 0; }

hipError_t launch_window(const nt_window_args& a, hipStream_t s) {
  const nt_layout &Lq = *a.q_layout, &Lk = *a.kv_layout;
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
  p.items = win::block_count(Lq.sum_n, Lq.batch, p.group, kBlockShift) * p.kv_heads;
  const bool bf = a.dtype == NT_BF16;
  if (p.d <= 32) return bf ? launch_rows<bf16, 32>(p, s) : launch_rows<float, 32>(p, s);
  if (p.d <= 64) return bf ? launch_rows<bf16, 64>(p, s) : launch_rows<float, 64>(p, s);
  return bf ? launch_rows<bf16, 128>(p, s) : launch_rows<float, 128>(p, s);
}

}  // namespace nt
