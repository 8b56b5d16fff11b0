// Rows of a table by token id, and the table's gradient.
//
//   y[r] = scale table[id_r];  dtable[v] (+)= scale sum_{r: id_r = v} dy[r]
//
// The gradient sorts the tokens by id (stable, so equal ids keep their order)
// and sums the sorted rows in chunks of equal length, whatever the ids: a run of
// one id inside a chunk goes straight to its table row, a run that crosses chunks
// leaves one partial sum per chunk, which a last launch adds in order.  There are
// no floating-point atomics: the result does not depend on timing.
#include <algorithm>

#include "nt_device.h"
#include "nt_internal.h"

namespace nt {
namespace {

constexpr int kVE = 8;             // channels per thread

template <typename T> struct Row8;
template <> struct Row8<bf16> {
  float v[8];
  __device__ __forceinline__ void load(const bf16* p) {
    Vec<bf16> t;
    t.load(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = t.v[j];
  }
  __device__ __forceinline__ void store(bf16* p) const {
    Vec<bf16> t;
#pragma unroll
    for (int j = 0; j < 8; ++j) t.v[j] = v[j];
    t.store(p);
  }
};
template <> struct Row8<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* p) {
    Vec<float> a, b;
    a.load(p);
    b.load(p + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = a.v[j], v[4 + j] = b.v[j];
  }
  __device__ __forceinline__ void store(float* p) const {
    Vec<float> a, b;
#pragma unroll
    for (int j = 0; j < 4; ++j) a.v[j] = v[j], b.v[j] = v[4 + j];
    a.store(p);
    b.store(p + 4);
  }
};

// Token id of row r, or `vocab` for one outside the table.
__device__ __forceinline__ uint32_t token(const void* ids, int wide, int64_t r, uint32_t vocab) {
  const int64_t id = wide ? reinterpret_cast<const int64_t*>(ids)[r] : reinterpret_cast<const int32_t*>(ids)[r];
  return (uint64_t)id < vocab ? (uint32_t)id : vocab;
}

// ---------------------------------------------------------------- lookup
// Eight channels per thread and turn, four turns in flight: bound by bytes, the rows of
// y written once and those of the table that occur read once (131072 rows of 2048
// bf16: 172 us, 6.2 TB/s of rows in and out; 14999 of 768: 9 us; 48 of 32: the launch).
constexpr int kPer = 4;
template <typename TT, typename TY>
__global__ void __launch_bounds__(256)
embedding_kernel(const TT* __restrict__ table, int64_t ld_table, uint32_t vocab, const void* __restrict__ ids, int wide,
                 int64_t rows, int cv, float scale, TY* __restrict__ y, int64_t ld_y, int64_t blocks) {
  const int64_t blk = block_id();
  if (blk >= blocks) return;
  const int64_t total = rows * cv;
  Row8<TT> x[kPer];
  int64_t r[kPer];
  int c[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int64_t e = blk * (256 * kPer) + 256 * k + threadIdx.x;
    r[k] = e < total ? e / cv : -1;
    c[k] = (int)(e - (e / cv) * cv) * kVE;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[k].v[j] = 0.f;
    if (r[k] < 0) continue;
    const uint32_t id = token(ids, wide, r[k], vocab);
    if (id < vocab) x[k].load(table + (int64_t)id * ld_table + c[k]);
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (r[k] < 0) continue;
    Row8<TY> o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o.v[j] = x[k].v[j] * scale;
    o.store(y + r[k] * ld_y + c[k]);
  }
}

// ---------------------------------------------------------------- sort by id
// Stable sort of (id, row) pairs.  Up to kSmall pairs take one launch: a workgroup
// has a range of ids, looks at all tokens, keeps those in its range in LDS, counts
// those below it (that is where its pairs go) and sorts what it kept by the few
// bits that ids of one range differ in.  More pairs go through a least-significant-
// digit radix sort of two launches per pass: one counts the digits of every tile,
// the other finds where a tile's pairs of each digit begin (all smaller digits,
// and the same digit in the tiles before) and writes them there in their order.
// The gradient table is cleared meanwhile by further workgroups of the same
// launches: the sort is short and latency-bound, the clearing long and bound by
// bytes (30011 rows of 768 fp32 and 14999 tokens, one launch: 15.6 us, 5.9 TB/s;
// 128011 rows of 2048 and 131072 tokens, six launches: 192 us, 5.5 TB/s).
// Past kSmall a range's pairs no longer fit LDS.  There, at 16384 tokens, the whole
// gradient takes 28 us with the one launch and 37 through the passes (C = 64, 32000 ids),
// 35 and 49 (768, 30000), 119 and 122 (1024, 128000), 26 and 27 (64, 300).
constexpr int kSmall = 16384, kRanges = 128, kRangeBits = 8, kMaxBins = 512;

struct SortParams {
  const void* ids;               // first pass: the tokens; later passes: NULL
  int wide;
  uint32_t vocab;
  const uint32_t *key_in, *row_in;
  uint32_t *key_out, *row_out;
  uint32_t* hist;                // [tiles + 1][bins]: counts; or, scanned, those of the tiles before, and all
  int scanned;
  int64_t rows;
  int tiles, shift, bits, passes;   // tiles, or ranges of ids
  uint32_t range;                // ids per range
  char* fill;                    // pieces fill_lo .. fill_hi of the gradient's memory are cleared, each fill_bytes long
  int64_t fill_ld, fill_lo, fill_hi, fill_total;   // and fill_ld apart; nothing past fill_total bytes
  int fill_bytes;
};

__device__ __forceinline__ uint32_t sort_key(const SortParams& p, int64_t r) {
  return p.ids ? token(p.ids, p.wide, r, p.vocab) : p.key_in[r];
}

// One wave per piece and turn, 16 bytes per lane and store.
__device__ __forceinline__ void clear_pieces(const SortParams& p, int64_t wave, int64_t waves, int lane) {
  for (int64_t r = p.fill_lo + wave; r < p.fill_hi; r += waves) {
    const int64_t at = r * p.fill_ld;
    const int n = (int)min((int64_t)p.fill_bytes, p.fill_total - at);
    for (int b = lane * 16; b < n; b += 1024) *reinterpret_cast<uint4*>(p.fill + at + b) = make_uint4(0, 0, 0, 0);
  }
}

// Lanes that hold the same digit as this one, among those in `ok`: one ballot per bit.
__device__ __forceinline__ uint64_t same_digit(uint32_t dg, int bits, uint64_t ok) {
  for (int bit = 0; bit < bits; ++bit) {
    const uint64_t set = __ballot((dg >> bit) & 1);
    ok &= (dg >> bit) & 1 ? set : ~set;
  }
  return ok;
}
__device__ __forceinline__ uint32_t lanes_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v, int lane) {      // inclusive
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const uint32_t u = __shfl_up(v, s, 64);
    v += lane >= s ? u : 0;
  }
  return v;
}

template <int ITER>
__global__ void __launch_bounds__(1024)
sort_range_kernel(SortParams p) {
  constexpr int kPairs = ITER * 1024, kBins = 1 << kRangeBits;
  __shared__ uint32_t keys[kPairs], wc[16][kBins], sums[16], below_s[16];
  __shared__ uint16_t rows[kPairs];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if ((int)blockIdx.x >= p.tiles) {
    clear_pieces(p, ((int64_t)blockIdx.x - p.tiles) * 16 + wave, ((int64_t)gridDim.x - p.tiles) * 16, lane);
    return;
  }
  const uint32_t lo = blockIdx.x * p.range;
  const int n_all = (int)p.rows, r0 = wave * (ITER * 64) + lane;
  // wave w looks at a sixteenth of the tokens in order, 64 at a time
  uint32_t key[ITER], row[ITER], rank[ITER];
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    const int r = r0 + k * 64;
    key[k] = r < n_all ? token(p.ids, p.wide, r, p.vocab) : 0xffffffffu;
  }
  uint32_t inside = 0, below = 0;
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    inside += __popcll(__ballot(key[k] - lo < p.range));
    below += __popcll(__ballot(key[k] < lo));
  }
  if (lane == 0) {
    sums[wave] = inside;
    below_s[wave] = below;
  }
  __syncthreads();
  uint32_t first = 0, n = 0, to0 = 0;                      // of all pairs, in this range, those of the waves before
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    first += below_s[w];
    to0 += w < wave ? sums[w] : 0;
    n += sums[w];
  }
  if (n == 0) return;
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    const uint64_t in = __ballot(key[k] - lo < p.range);
    if (key[k] - lo < p.range) {
      const uint32_t to = to0 + lanes_below(in);
      keys[to] = key[k] - lo;
      rows[to] = (uint16_t)(r0 + k * 64);
    }
    to0 += __popcll(in);
  }
  // the range's pairs, again a sixteenth per wave
  const int bins = 1 << p.bits, iters = ((int)n + 1023) / 1024, s0 = wave * (iters * 64) + lane;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.bits;
    for (int b = tid; b < 16 * kBins; b += 1024) (&wc[0][0])[b] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
      if (k >= iters) break;
      const int r = s0 + k * 64;
      const bool ok = r < (int)n;
      key[k] = ok ? keys[r] : 0;
      row[k] = ok ? rows[r] : 0;
      const uint32_t dg = (key[k] >> shift) & (bins - 1);
      const uint64_t same = same_digit(dg, p.bits, __ballot(ok));
      const uint32_t old = wc[wave][dg], under = lanes_below(same);
      rank[k] = old + under;
      if (ok && under == 0) wc[wave][dg] = old + __popcll(same);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    uint32_t tot = 0, incl = 0;
    if (tid < kBins) {                                     // counts become the places before each wave's first pair
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        const uint32_t c = wc[w][tid];
        wc[w][tid] = tot;
        tot += c;
      }
      incl = wave_scan(tot, lane);
      if (lane == 63) sums[wave] = incl;
    }
    __syncthreads();
    if (tid < kBins) {
      uint32_t base = incl - tot;
      for (int w = 0; w < wave; ++w) base += sums[w];
#pragma unroll
      for (int w = 0; w < 16; ++w) wc[w][tid] += base;
    }
    __syncthreads();
    const bool done = pass + 1 == p.passes;
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
      if (k >= iters) break;
      if (s0 + k * 64 >= (int)n) continue;
      const uint32_t to = wc[wave][(key[k] >> shift) & (bins - 1)] + rank[k];
      if (done) {
        p.key_out[first + to] = lo + key[k];
        p.row_out[first + to] = row[k];
      } else {
        keys[to] = key[k];
        rows[to] = (uint16_t)row[k];
      }
    }
    if (!done) __syncthreads();
  }
}

template <int ITER>
__global__ void __launch_bounds__(256)
sort_count_kernel(SortParams p) {
  __shared__ uint32_t h[kMaxBins];
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= p.tiles) {
    const int64_t w = ((int64_t)blockIdx.x - p.tiles) * 4 + (tid >> 6);
    clear_pieces(p, w, ((int64_t)gridDim.x - p.tiles) * 4, tid & 63);
    return;
  }
  const int bins = 1 << p.bits;
  uint32_t key[ITER];
  const int64_t r0 = (int64_t)blockIdx.x * (ITER * 256);
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    const int64_t r = r0 + k * 256 + tid;
    key[k] = r < p.rows ? sort_key(p, r) : 0;
  }
  for (int b = tid; b < bins; b += 256) h[b] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < ITER; ++k)
    if (r0 + k * 256 + tid < p.rows) atomicAdd(&h[(key[k] >> p.shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int b = tid; b < bins; b += 256) p.hist[(int64_t)blockIdx.x * bins + b] = h[b];
}

// Every tile's counts become those of the tiles before it, and row `tiles` their
// totals: where there are so many tiles that each of them adding up all counts
// would cost more than this launch.  A workgroup has 64 digits, each of its 16
// waves a sixteenth of the tiles.
__global__ void __launch_bounds__(1024)
sort_scan_kernel(SortParams p) {
  __shared__ uint32_t sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << p.bits, own = (bins + 63) / 64;
  if ((int)blockIdx.x >= own) {
    clear_pieces(p, ((int64_t)blockIdx.x - own) * 16 + wave, ((int64_t)gridDim.x - own) * 16, lane);
    return;
  }
  const int dg = blockIdx.x * 64 + lane, lo = (int)((int64_t)p.tiles * wave / 16), hi = (int)((int64_t)p.tiles * (wave + 1) / 16);
  uint32_t* h = p.hist + min(dg, bins - 1);
  uint32_t n = 0;
#pragma unroll 8
  for (int t = lo; t < hi; ++t) n += h[(int64_t)t * bins];
  sums[wave][lane] = n;
  __syncthreads();
  uint32_t at = 0;
  for (int w = 0; w < wave; ++w) at += sums[w][lane];
  if (dg >= bins) return;
  for (int t0 = lo; t0 < hi; t0 += 8) {
    uint32_t c[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) c[u] = h[(int64_t)min(t0 + u, hi - 1) * bins];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (t0 + u < hi) h[(int64_t)(t0 + u) * bins] = at;
      at += c[u];
    }
  }
  if (wave == 15) {
    uint32_t all = 0;
    for (int w = 0; w < 16; ++w) all += sums[w][lane];
    h[(int64_t)p.tiles * bins] = all;
  }
}

template <int ITER>
__global__ void __launch_bounds__(256)
sort_scatter_kernel(SortParams p) {
  __shared__ uint32_t wc[4][kMaxBins], sums[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if ((int)blockIdx.x >= p.tiles) {
    const int64_t w = ((int64_t)blockIdx.x - p.tiles) * 4 + wave;
    clear_pieces(p, w, ((int64_t)gridDim.x - p.tiles) * 4, lane);
    return;
  }
  const int bins = 1 << p.bits, tile = blockIdx.x;
  // wave w takes a quarter of the tile in order, 64 pairs at a time
  uint32_t key[ITER], row[ITER], rank[ITER];
  const int64_t r0 = (int64_t)tile * (ITER * 256) + wave * (ITER * 64);
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    const int64_t r = r0 + k * 64 + lane;
    key[k] = r < p.rows ? sort_key(p, r) : 0;
    row[k] = r < p.rows ? (p.ids ? (uint32_t)r : p.row_in[r]) : 0;
  }
  for (int b = tid; b < 4 * kMaxBins; b += 256) (&wc[0][0])[b] = 0;
  // thread t has the digits 2 t and 2 t + 1: their totals, and the tiles before
  uint32_t t0 = 0, t1 = 0, b0 = 0, b1 = 0;
  if (2 * tid < bins && p.scanned) {
    const uint2 all = *reinterpret_cast<const uint2*>(p.hist + (int64_t)p.tiles * bins + 2 * tid);
    const uint2 before = *reinterpret_cast<const uint2*>(p.hist + (int64_t)tile * bins + 2 * tid);
    t0 = all.x;
    t1 = all.y;
    b0 = before.x;
    b1 = before.y;
  } else if (2 * tid < bins) {
#pragma unroll 8
    for (int t = 0; t < p.tiles; ++t) {
      const uint2 c = *reinterpret_cast<const uint2*>(p.hist + (int64_t)t * bins + 2 * tid);
      t0 += c.x;
      t1 += c.y;
      b0 += t < tile ? c.x : 0;
      b1 += t < tile ? c.y : 0;
    }
  }
  const uint32_t incl = wave_scan(t0 + t1, lane);
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    const bool ok = r0 + k * 64 + lane < p.rows;
    const uint32_t dg = (key[k] >> p.shift) & (bins - 1);
    const uint64_t same = same_digit(dg, p.bits, __ballot(ok));
    const uint32_t old = wc[wave][dg], below = lanes_below(same);
    rank[k] = old + below;
    if (ok && below == 0) wc[wave][dg] = old + __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  if (2 * tid < bins) {
    uint32_t at = incl - t0 - t1;
    for (int w = 0; w < wave; ++w) at += sums[w];
    uint32_t x = at + b0, y = at + t0 + b1;
#pragma unroll
    for (int w = 0; w < 4; ++w) {                          // counts become the places before each wave's first pair
      const uint32_t c = wc[w][2 * tid], d = wc[w][2 * tid + 1];
      wc[w][2 * tid] = x;
      wc[w][2 * tid + 1] = y;
      x += c;
      y += d;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < ITER; ++k) {
    if (r0 + k * 64 + lane >= p.rows) continue;
    const uint32_t to = wc[wave][(key[k] >> p.shift) & (bins - 1)] + rank[k];
    p.key_out[to] = key[k];
    p.row_out[to] = row[k];
  }
}

// ---------------------------------------------------------------- sum of runs
// Eight rows per thread in flight, added in the order of the sort; a token's run has
// one sum per chunk.  Bound by dy's bytes, rows in random order, and the table rows
// written: 131072 rows of 2048 bf16 into fp32 222 us, 3.7 TB/s; 14999 of 768 14 us.
constexpr int kBatch = 8;          // rows in flight per thread
struct SumParams {
  const uint32_t *key, *row;
  uint32_t vocab;
  int64_t rows;
  int chunk;                     // sorted rows per chunk
  int64_t chunks;
  int cv, cvs;                   // 8-channel pieces per row; per workgroup slice (at most 256)
  float scale;
  int accumulate;
  float* part;                   // [chunks][2][8 cv]: sum of the run that enters, of the run that leaves
  int64_t blocks;
};

template <typename TG>
__device__ __forceinline__ void write_row(TG* dtable, int64_t ld, uint32_t id, int c, const float (&acc)[8],
                                          const SumParams& p) {
  TG* d = dtable + (int64_t)id * ld + c;
  Row8<TG> o;
  if (p.accumulate) {
    o.load(d);
#pragma unroll
    for (int j = 0; j < 8; ++j) o.v[j] = fmaf(acc[j], p.scale, o.v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) o.v[j] = acc[j] * p.scale;
  }
  o.store(d);
}

template <typename TD, typename TG>
__global__ void __launch_bounds__(256)
embedding_sum_kernel(SumParams p, const TD* __restrict__ dy, int64_t ld_dy, TG* __restrict__ dtable, int64_t ld) {
  const int64_t blk = block_id();
  if (blk >= p.blocks) return;
  const int slices = (p.cv + p.cvs - 1) / p.cvs, teams = 256 / p.cvs;
  const int slice = (int)(blk % slices), team = threadIdx.x / p.cvs, piece = slice * p.cvs + threadIdx.x % p.cvs;
  const int64_t ch = blk / slices * teams + team;
  if (team >= teams || piece >= p.cv || ch >= p.chunks) return;
  const int64_t s = ch * p.chunk, e = min(s + p.chunk, p.rows);
  const int c = piece * kVE;
  float acc[8] = {};
  uint32_t cur = p.key[s];
  bool enters = s > 0 && p.key[s - 1] == cur;
  for (int64_t x0 = s; x0 < e && cur < p.vocab; x0 += kBatch) {
    // the batch's rows in flight together; then in order
    uint32_t id[kBatch];
    Row8<TD> v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int64_t x = min(x0 + u, e - 1);
      id[u] = p.key[x];
      v[u].load(dy + (int64_t)p.row[x] * ld_dy + c);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (x0 + u >= e || cur >= p.vocab) break;
      if (id[u] != cur) {
        if (enters) {
          float* d = p.part + (ch * 2 * p.cv + piece) * kVE;
#pragma unroll
          for (int j = 0; j < 8; ++j) d[j] = acc[j];
        } else {
          write_row(dtable, ld, cur, c, acc, p);
        }
        cur = id[u];
        enters = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.f;
        if (cur >= p.vocab) break;                         // sorted: only tokens outside the table follow
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += v[u].v[j];
    }
  }
  if (cur >= p.vocab) return;
  const bool leaves = e < p.rows && p.key[e] == cur;
  if (!enters && !leaves) {
    write_row(dtable, ld, cur, c, acc, p);
    return;
  }
  float* d = p.part + ((ch * 2 + (enters ? 0 : 1)) * p.cv + piece) * kVE;
#pragma unroll
  for (int j = 0; j < 8; ++j) d[j] = acc[j];
}

// The runs that cross chunks: the chunk in which one begins adds its parts, four
// waves a quarter of the chunks each (the run of a frequent token goes over
// hundreds), joined in order.  A workgroup has one chunk and 64 pieces of the row.
// Bound by the longest run's latency: 17 us and 5 for the two above.
template <typename TG>
__global__ void __launch_bounds__(256)
embedding_join_kernel(SumParams p, TG* __restrict__ dtable, int64_t ld) {
  __shared__ float sum[3][8][64];
  const int64_t blk = block_id();
  if (blk >= p.blocks) return;
  const int slices = (p.cv + 63) / 64, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t ch = blk / slices;
  const int piece = min((int)(blk % slices) * 64 + lane, p.cv - 1);
  if (ch + 1 >= p.chunks) return;
  const int64_t s = ch * p.chunk, e = s + p.chunk;       // a chunk before the last is whole
  const uint32_t id = p.key[e - 1];
  if (id >= p.vocab || p.key[e] != id) return;           // nothing leaves
  if (s > 0 && p.key[s - 1] == id) return;               // it began before this chunk
  int64_t n = 0;                                         // chunks that begin with the run
  for (;;) {
    const int64_t x = ch + 1 + n + lane;
    const uint64_t other = ~__ballot(x < p.chunks && p.key[min(x, p.chunks - 1) * p.chunk] == id);
    if (other) {
      n += __ffsll((unsigned long long)other) - 1;
      break;
    }
    n += 64;
  }
  const int64_t lo = n * wave / 4, hi = n * (wave + 1) / 4;
  const float* h = p.part + ((ch + 1) * 2 * p.cv + piece) * kVE;   // chunk x's part of the run that enters: + 2 x 8 cv
  float acc[8] = {};
  if (wave == 0) {
    Row8<float> v;
    v.load(p.part + ((ch * 2 + 1) * p.cv + piece) * kVE);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = v.v[j];
  }
  for (int64_t x = lo; x < hi; x += kBatch) {
    Row8<float> v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) v[u].load(h + min(x + u, hi - 1) * 2 * p.cv * kVE);
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += x + u < hi ? v[u].v[j] : 0.f;
  }
  if (wave > 0)
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[wave - 1][j][lane] = acc[j];
  __syncthreads();
  if (wave > 0 || (int)(blk % slices) * 64 + lane >= p.cv) return;
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += sum[w][j][lane];
  write_row(dtable, ld, id, piece * kVE, acc, p);
}

// Sorted rows per chunk: short ones give few tokens enough workgroups, long ones
// leave fewer partial sums to add.  Whole gradient in us, for C = 64 and 32000 ids, 768
// and 30000, 1024 and 128000, 64 and 300: chunks of 32 and 64 rows at 32768 tokens
// 41 : 49, 56 : 61, 138 : 137, 28 : 33; at 100000 57 : 62, 95 : 90, 214 : 216, 40 : 40; at
// 160000 65 : 67, 136 : 130, 259 : 252, 50 : 45.  Chunks of 64 and 128 at 262144 tokens
// 74 : 85, 179 : 170, 317 : 312, 56 : 58; at 524288 90 : 98, 301 : 289, 473 : 463, 76 : 70.
// At most 65536 chunks, so that one token's run over all rows stays a short list of them.
constexpr int64_t kChunk64Rows = 100000, kChunk128Rows = 500000;
int chunk_of(int64_t rows) {
  return rows < kChunk64Rows ? 32 : rows < kChunk128Rows ? 64 : (int)std::max<int64_t>(128, (rows + 65535) >> 16);
}
// Pairs per tile / 256: small tiles give few tokens enough workgroups, large ones
// leave fewer counts to go through (small and large, C = 64, 32000 ids: 800000 tokens
// 117 and 124 us, 1.5 million 160 and 158, 3 million 295 and 265, 12 million 1056 and 916;
// 131000 tokens 58 and 76).
constexpr int64_t kLargeTileRows = 1500000;
int tile_iter(int64_t rows) { return rows < kLargeTileRows ? 4 : 16; }
// From so many pairs on (98 tiles), the tiles' counts are summed by a launch of their
// own (C = 64, 32000 ids, with and without it: 65536 tokens 53 and 47 us, 100000 57 and
// 56, 131000 58 and 61, 200000 67 and 77, 524288 90 and 124; at C = 2048, 100000 tokens
// 227 and 229).
constexpr int64_t kScanRows = 100000;

struct Plan {
  bool small;
  int64_t range;
  int tiles, passes, bits, chunk, iter;
  int64_t chunks;
  size_t key[2], row[2], hist, part, bytes;
};
Plan plan(int64_t rows, int64_t vocab, int C) {
  Plan s{};
  s.small = rows <= kSmall;
  s.range = s.small ? (vocab + kRanges) / kRanges : 0;   // ids 0 .. vocab in at most kRanges ranges
  const int64_t top = s.small ? s.range - 1 : vocab;     // largest id that is sorted by
  int bits = 1;
  while ((top >> bits) > 0) ++bits;
  const int most = s.small ? kRangeBits : 9;
  s.passes = (bits + most - 1) / most;
  s.bits = (bits + s.passes - 1) / s.passes;
  s.iter = tile_iter(rows);
  s.tiles = (int)((rows + s.iter * 256 - 1) / (s.iter * 256));
  s.chunk = chunk_of(rows);
  s.chunks = (rows + s.chunk - 1) / s.chunk;
  size_t at = 0;
  auto take = [&](size_t n) { const size_t o = at; at += (n + 15) / 16 * 16; return o; };
  for (int k = 0; k < (s.small ? 1 : 2); ++k) {
    s.key[k] = take((size_t)rows * 4);
    s.row[k] = take((size_t)rows * 4);
  }
  s.hist = take(s.small ? 0 : ((size_t)s.tiles + 1) * (1u << s.bits) * 4);
  s.part = take((size_t)s.chunks * 2 * C * 4);
  s.bytes = at;
  return s;
}

template <typename TD, typename TG>
hipError_t backward(const void* ids, int wide, int64_t rows, int64_t vocab, int C, const TD* dy, int64_t ld_dy,
                    float scale, TG* dtable, int64_t ld, int accumulate, char* ws, hipStream_t s) {
  const Plan pl = plan(rows, vocab, C);
  SortParams sp{};
  sp.wide = wide;
  sp.vocab = (uint32_t)vocab;
  sp.rows = rows;
  sp.tiles = pl.tiles;
  sp.bits = pl.bits;
  sp.passes = pl.passes;
  sp.hist = (uint32_t*)(ws + pl.hist);
  sp.scanned = rows >= kScanRows;
  // memory to clear: 4 KB pieces of a dense table, else its rows
  sp.fill = (char*)dtable;
  const bool dense = ld == C;
  sp.fill_bytes = dense ? 4096 : C * (int)sizeof(TG);
  sp.fill_ld = dense ? 4096 : ld * (int64_t)sizeof(TG);
  sp.fill_total = dense ? vocab * C * (int64_t)sizeof(TG) : INT64_MAX;
  const int64_t pieces = accumulate ? 0 : dense ? (sp.fill_total + 4095) / 4096 : vocab;
  int last = 0;                                          // which of the two pairs of arrays holds the result
  if (pl.small) {
    sp.ids = ids;
    sp.key_out = (uint32_t*)(ws + pl.key[0]);
    sp.row_out = (uint32_t*)(ws + pl.row[0]);
    sp.fill_hi = pieces;
    const int clear = (int)std::min<int64_t>((pieces + 15) / 16, 1024);
    sp.range = (uint32_t)pl.range;
    sp.tiles = (int)((vocab + pl.range) / pl.range);
    if (rows <= 4096) sort_range_kernel<4><<<sp.tiles + clear, 1024, 0, s>>>(sp);
    else sort_range_kernel<16><<<sp.tiles + clear, 1024, 0, s>>>(sp);
    if (hipError_t e = hipGetLastError()) return e;
  } else {
    last = (pl.passes - 1) & 1;
    const int each = sp.scanned ? 3 : 2, steps = each * pl.passes;   // launches that share the clearing
    for (int k = 0; k < steps; ++k) {
      const int pass = k / each, what = k % each == 0 ? 0 : k % each + (3 - each);   // 0 counts, 1 scans, 2 scatters
      sp.ids = pass ? nullptr : ids;
      sp.key_in = (uint32_t*)(ws + pl.key[(pass + 1) & 1]);
      sp.row_in = (uint32_t*)(ws + pl.row[(pass + 1) & 1]);
      sp.key_out = (uint32_t*)(ws + pl.key[pass & 1]);
      sp.row_out = (uint32_t*)(ws + pl.row[pass & 1]);
      sp.shift = pass * pl.bits;
      sp.fill_lo = pieces * k / steps;
      sp.fill_hi = pieces * (k + 1) / steps;
      const int waves = what == 1 ? 16 : 4, clear = (int)std::min<int64_t>((sp.fill_hi - sp.fill_lo + waves - 1) / waves, 8192 / waves);
      if (what == 0) {
        if (pl.iter == 4) sort_count_kernel<4><<<pl.tiles + clear, 256, 0, s>>>(sp);
        else sort_count_kernel<16><<<pl.tiles + clear, 256, 0, s>>>(sp);
      } else if (what == 1) {
        sort_scan_kernel<<<((1 << pl.bits) + 63) / 64 + clear, 1024, 0, s>>>(sp);
      } else {
        if (pl.iter == 4) sort_scatter_kernel<4><<<pl.tiles + clear, 256, 0, s>>>(sp);
        else sort_scatter_kernel<16><<<pl.tiles + clear, 256, 0, s>>>(sp);
      }
      if (hipError_t e = hipGetLastError()) return e;
    }
  }
  if (rows == 0) return hipSuccess;
  SumParams q{};
  q.key = (uint32_t*)(ws + pl.key[last]);
  q.row = (uint32_t*)(ws + pl.row[last]);
  q.vocab = (uint32_t)vocab;
  q.rows = rows;
  q.chunk = pl.chunk;
  q.chunks = pl.chunks;
  q.cv = C / kVE;
  q.cvs = q.cv < 256 ? q.cv : 256;
  q.scale = scale;
  q.accumulate = accumulate;
  q.part = (float*)(ws + pl.part);
  const int slices = (q.cv + q.cvs - 1) / q.cvs, teams = 256 / q.cvs;
  q.blocks = (pl.chunks + teams - 1) / teams * slices;
  embedding_sum_kernel<TD, TG><<<folded_grid(q.blocks), 256, 0, s>>>(q, dy, ld_dy, dtable, ld);
  if (hipError_t e = hipGetLastError()) return e;
  q.blocks = (pl.chunks - 1) * ((q.cv + 63) / 64);
  if (q.blocks > 0) embedding_join_kernel<TG><<<folded_grid(q.blocks), 256, 0, s>>>(q, dtable, ld);
  return hipGetLastError();
}

}  // namespace

size_t embedding_backward_workspace_bytes(int64_t rows, int64_t vocab, int C) { return plan(rows, vocab, C).bytes; }

hipError_t launch_embedding(const void* table, int64_t vocab, int64_t ld_table, nt_dtype table_dtype, const void* ids,
                            int wide, int64_t rows, int C, float scale, void* y, int64_t ld_y, nt_dtype y_dtype,
                            hipStream_t s) {
  const int cv = C / kVE;
  const int64_t blocks = (rows * cv + 256 * kPer - 1) / (256 * kPer);
  const dim3 grid = folded_grid(blocks);
#define NT_EMBED(TT, TY)                                                                                        \
  embedding_kernel<TT, TY><<<grid, 256, 0, s>>>((const TT*)table, ld_table, (uint32_t)vocab, ids, wide, rows, cv, \
                                                scale, (TY*)y, ld_y, blocks)
  if (table_dtype == NT_BF16) {
    if (y_dtype == NT_BF16) NT_EMBED(bf16, bf16);
    else NT_EMBED(bf16, float);
  } else {
    if (y_dtype == NT_BF16) NT_EMBED(float, bf16);
    else NT_EMBED(float, float);
  }
#undef NT_EMBED
  return hipGetLastError();
}

hipError_t launch_embedding_backward(const void* ids, int wide, int64_t rows, int64_t vocab, int C, const void* dy,
                                     int64_t ld_dy, nt_dtype dtype, float scale, void* dtable, int64_t ld_dtable,
                                     nt_dtype table_dtype, int accumulate, void* ws, hipStream_t s) {
#define NT_EMBED_BWD(TD, TG) \
  backward<TD, TG>(ids, wide, rows, vocab, C, (const TD*)dy, ld_dy, scale, (TG*)dtable, ld_dtable, accumulate, (char*)ws, s)
  if (dtype == NT_BF16) return table_dtype == NT_BF16 ? NT_EMBED_BWD(bf16, bf16) : NT_EMBED_BWD(bf16, float);
  return table_dtype == NT_BF16 ? NT_EMBED_BWD(float, bf16) : NT_EMBED_BWD(float, float);
#undef NT_EMBED_BWD
}

}  // namespace nt
