// Rows of a table by token id, and the table's gradient.
//
//   y[r] = scale table[id_r];  dtable[v] (+)= scale sum_{r: id_r = v} dy[r]
//
// The gradient sorts the tokens by id (stable, so equal ids keep their order)
// and sums the sorted rows in chunks of equal length, whatever the ids: a run of
// one id inside a chunk goes straight to its table row, a run that crosses chunks
// leaves one partial sum per chunk, which a last launch adds in order.  There are
// no floating-point atomics: the result does not depend on timing.
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
constexpr int kPer = 4;            // 16-byte chunks in flight per thread
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
// Least-significant-digit radix sort of (id, row) pairs, kTile pairs per
// workgroup.  A pass counts the digits of every tile, then every tile finds
// where its pairs of each digit begin (all smaller digits, and the same digit in
// the tiles before) and writes them there in their order.
constexpr int kTile = 4096, kMaxBins = 512;

struct SortParams {
  const void* ids;               // first pass: the tokens; later passes: NULL
  int wide;
  uint32_t vocab;
  const uint32_t *key_in, *row_in;
  uint32_t *key_out, *row_out;
  uint32_t* hist;                // [tiles][bins]
  int64_t rows;
  int tiles, shift, bits;
  char* fill;                    // a share of the gradient's memory to clear: rows fill_lo .. fill_hi
  int64_t fill_ld, fill_lo, fill_hi;   // bytes per row, first row, end
  int fill_bytes;                // bytes of a row that are cleared
};

__device__ __forceinline__ uint32_t sort_key(const SortParams& p, int64_t r) {
  return p.ids ? token(p.ids, p.wide, r, p.vocab) : p.key_in[r];
}

// Workgroups past the tiles clear the gradient table's rows: one wave per row
// and turn, 16 bytes per lane.
__device__ __forceinline__ void clear_rows(const SortParams& p, int64_t wave, int64_t waves, int lane) {
  for (int64_t r = p.fill_lo + wave; r < p.fill_hi; r += waves) {
    char* d = p.fill + r * p.fill_ld;
    for (int b = lane * 16; b < p.fill_bytes; b += 1024) *reinterpret_cast<uint4*>(d + b) = make_uint4(0, 0, 0, 0);
  }
}

__global__ void __launch_bounds__(256)
sort_count_kernel(SortParams p) {
  __shared__ uint32_t h[kMaxBins];
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= p.tiles) {
    const int64_t w = ((int64_t)blockIdx.x - p.tiles) * 4 + (tid >> 6);
    clear_rows(p, w, ((int64_t)gridDim.x - p.tiles) * 4, tid & 63);
    return;
  }
  const int bins = 1 << p.bits;
  for (int b = tid; b < bins; b += 256) h[b] = 0;
  __syncthreads();
  const int64_t r0 = (int64_t)blockIdx.x * kTile;
#pragma unroll
  for (int k = 0; k < kTile / 256; ++k) {
    const int64_t r = r0 + k * 256 + tid;
    if (r < p.rows) atomicAdd(&h[(sort_key(p, r) >> p.shift) & (bins - 1)], 1u);
  }
  __syncthreads();
  for (int b = tid; b < bins; b += 256) p.hist[(int64_t)blockIdx.x * bins + b] = h[b];
}

__global__ void __launch_bounds__(256)
sort_scatter_kernel(SortParams p) {
  __shared__ uint32_t base[kMaxBins], wc[4][kMaxBins], part[256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if ((int)blockIdx.x >= p.tiles) {
    const int64_t w = ((int64_t)blockIdx.x - p.tiles) * 4 + wave;
    clear_rows(p, w, ((int64_t)gridDim.x - p.tiles) * 4, lane);
    return;
  }
  const int bins = 1 << p.bits, per = (bins + 255) / 256, tile = blockIdx.x;
  // thread b takes bins b per .. b per + per - 1: totals, and the tiles before
  uint32_t tot[2] = {0, 0}, before[2] = {0, 0};
  for (int u = 0; u < per; ++u) {
    const int b = tid * per + u;
    if (b < bins)
      for (int t = 0; t < p.tiles; ++t) {
        const uint32_t c = p.hist[(int64_t)t * bins + b];
        tot[u] += c;
        before[u] += t < tile ? c : 0;
      }
  }
  part[tid] = tot[0] + tot[1];
  for (int b = tid; b < 4 * kMaxBins; b += 256) (&wc[0][0])[b] = 0;
  __syncthreads();
  for (int s = 1; s < 256; s <<= 1) {                    // inclusive scan of the threads' totals
    const uint32_t v = tid >= s ? part[tid - s] : 0;
    __syncthreads();
    part[tid] += v;
    __syncthreads();
  }
  uint32_t at = part[tid] - tot[0] - tot[1];
  for (int u = 0; u < per; ++u) {
    const int b = tid * per + u;
    if (b < bins) base[b] = at + before[u];
    at += tot[u];
  }
  // ranks: wave w takes a quarter of the tile in order, 64 pairs at a time; the
  // lanes that hold equal digits are found by one ballot per digit bit
  constexpr int kIter = kTile / 256;
  uint32_t key[kIter], rank[kIter];
  const int64_t r0 = (int64_t)tile * kTile + wave * (kTile / 4);
#pragma unroll
  for (int k = 0; k < kIter; ++k) {
    const int64_t r = r0 + k * 64 + lane;
    const bool ok = r < p.rows;
    key[k] = ok ? sort_key(p, r) : 0;
    const uint32_t dg = (key[k] >> p.shift) & (bins - 1);
    uint64_t same = __ballot(ok);
    for (int bit = 0; bit < p.bits; ++bit) {
      const uint64_t set = __ballot((dg >> bit) & 1);
      same &= (dg >> bit) & 1 ? set : ~set;
    }
    const uint32_t old = wc[wave][dg], below = __popcll(same & ((1ull << lane) - 1));
    rank[k] = old + below;
    if (ok && below == 0) wc[wave][dg] = old + __popcll(same);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kIter; ++k) {
    const int64_t r = r0 + k * 64 + lane;
    if (r >= p.rows) continue;
    const uint32_t dg = (key[k] >> p.shift) & (bins - 1);
    uint32_t to = base[dg] + rank[k];
    for (int w = 0; w < wave; ++w) to += wc[w][dg];
    p.key_out[to] = key[k];
    p.row_out[to] = p.ids ? (uint32_t)r : p.row_in[r];
  }
}

// ---------------------------------------------------------------- sum of runs
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
  for (int64_t x = s; x < e; ++x) {
    const uint32_t k = p.key[x];
    if (k != cur) {
      if (cur < p.vocab) {
        if (enters) {
#pragma unroll
          for (int j = 0; j < 8; ++j) p.part[((ch * 2) * p.cv + piece) * kVE + j] = acc[j];
        } else {
          write_row(dtable, ld, cur, c, acc, p);
        }
      }
      cur = k;
      enters = false;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    }
    if (k >= p.vocab) break;                             // sorted: only tokens outside the table follow
    Row8<TD> v;
    v.load(dy + (int64_t)p.row[x] * ld_dy + c);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += v.v[j];
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

// The runs that cross chunks: the chunk in which one begins adds its parts.
template <typename TG>
__global__ void __launch_bounds__(256)
embedding_join_kernel(SumParams p, TG* __restrict__ dtable, int64_t ld) {
  const int64_t blk = block_id();
  if (blk >= p.blocks) return;
  const int slices = (p.cv + p.cvs - 1) / p.cvs, teams = 256 / p.cvs;
  const int slice = (int)(blk % slices), team = threadIdx.x / p.cvs, piece = slice * p.cvs + threadIdx.x % p.cvs;
  const int64_t ch = blk / slices * teams + team;
  if (team >= teams || piece >= p.cv || ch + 1 >= p.chunks) return;
  const int64_t s = ch * p.chunk, e = s + p.chunk;       // a chunk before the last is whole
  const uint32_t id = p.key[e - 1];
  if (id >= p.vocab || p.key[e] != id) return;           // nothing leaves
  if (s > 0 && p.key[s - 1] == id) return;               // it began before this chunk
  float acc[8];
  const float* d = p.part + ((ch * 2 + 1) * p.cv + piece) * kVE;
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = d[j];
  for (int64_t x = ch + 1; x < p.chunks && p.key[x * p.chunk] == id; ++x) {
    const float* h = p.part + ((x * 2) * p.cv + piece) * kVE;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += h[j];
  }
  write_row(dtable, ld, id, piece * kVE, acc, p);
}

constexpr int kChunk = 32;

struct Plan {
  int tiles, passes, bits;
  int64_t chunks;
  size_t key[2], row[2], hist, part, bytes;
};
Plan plan(int64_t rows, int64_t vocab, int C) {
  Plan s{};
  int bits = 1;
  while ((vocab >> bits) > 0) ++bits;                    // ids 0 .. vocab
  s.passes = (bits + 8) / 9;
  s.bits = (bits + s.passes - 1) / s.passes;
  s.tiles = (int)((rows + kTile - 1) / kTile);
  s.chunks = (rows + kChunk - 1) / kChunk;
  size_t at = 0;
  auto take = [&](size_t n) { const size_t o = at; at += (n + 15) / 16 * 16; return o; };
  for (int k = 0; k < 2; ++k) {
    s.key[k] = take((size_t)rows * 4);
    s.row[k] = take((size_t)rows * 4);
  }
  s.hist = take((size_t)s.tiles * (1u << s.bits) * 4);
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
  sp.hist = (uint32_t*)(ws + pl.hist);
  sp.fill = (char*)dtable;
  sp.fill_ld = ld * (int64_t)sizeof(TG);
  sp.fill_bytes = C * (int)sizeof(TG);
  const int steps = 2 * pl.passes;                       // launches that share the clearing
  for (int k = 0; k < steps; ++k) {
    const int pass = k / 2;
    sp.ids = pass ? nullptr : ids;
    sp.key_in = (uint32_t*)(ws + pl.key[(pass + 1) & 1]);
    sp.row_in = (uint32_t*)(ws + pl.row[(pass + 1) & 1]);
    sp.key_out = (uint32_t*)(ws + pl.key[pass & 1]);
    sp.row_out = (uint32_t*)(ws + pl.row[pass & 1]);
    sp.shift = pass * pl.bits;
    sp.fill_lo = accumulate ? 0 : vocab * k / steps;
    sp.fill_hi = accumulate ? 0 : vocab * (k + 1) / steps;
    const int64_t share = sp.fill_hi - sp.fill_lo;
    const int clear = (int)(share <= 0 ? 0 : share < 8192 ? (share + 3) / 4 : 2048);
    if (pl.tiles + clear == 0) continue;
    if (k & 1) sort_scatter_kernel<<<pl.tiles + clear, 256, 0, s>>>(sp);
    else sort_count_kernel<<<pl.tiles + clear, 256, 0, s>>>(sp);
    if (hipError_t e = hipGetLastError()) return e;
  }
  if (rows == 0) return hipSuccess;
  SumParams q{};
  q.key = (uint32_t*)(ws + pl.key[(pl.passes - 1) & 1]);
  q.row = (uint32_t*)(ws + pl.row[(pl.passes - 1) & 1]);
  q.vocab = (uint32_t)vocab;
  q.rows = rows;
  q.chunk = kChunk;
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
  if (pl.chunks > 1) embedding_join_kernel<TG><<<folded_grid(q.blocks), 256, 0, s>>>(q, dtable, ld);
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
