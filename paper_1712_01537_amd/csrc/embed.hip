// Table rows by id (oc_embed_fwd), y[r] = scale table[id[r]], and the table's gradient
// (oc_embed_bwd), dtable[v] = scale times the sum of dy[r] over the rows r with id v.
//
// The gradient without atomics, so that its bits do not depend on the order of the
// workgroups: the rows are sorted by id (stable, so that those of one id stay in order),
// the sorted list is cut into chunks of equal length, and each chunk's runs of one id
// are summed in order.  A run inside one chunk is written to the table's row; one that
// goes on over a border leaves a partial sum a chunk, added by k_embed_join.  However
// many rows share an id, no thread's chain of additions is longer than a chunk.
//
// The sort takes the ids' bits in digits, lowest first, with one counter a digit value
// and tile of rows: count, scan over the tiles, and scatter.  A tile is one wave's: it
// takes 64 rows at a time, in order, so that the place of a row among those of its digit
// is a count of the lanes before it with the same digit.
#include <algorithm>

#include "rows.h"

namespace {

using oc::cdiv;

constexpr int TB = 256;
constexpr int64_t MOST_BLOCKS = (int64_t)1 << 22;
constexpr uint32_t KEY_BITS = 0xffffffu;  // a shuffle key without its shape

__device__ __forceinline__ uint32_t id_of(const int32_t* ids, int64_t r, uint32_t mask) {
  return (uint32_t)ids[r] & mask;
}

__global__ __launch_bounds__(TB) void k_embed(const int32_t* ids, uint32_t mask, int64_t rows,
                                              int64_t num, int c, const void* table, bool bf16,
                                              float scale, void* y) {
  const int nv = (c + 7) / 8;
  const int64_t groups = rows * nv;
  for (int64_t i = (int64_t)blockIdx.x * TB + threadIdx.x; i < groups;
       i += (int64_t)gridDim.x * TB) {
    const int64_t row = i / nv;
    const int col = (int)(i - row * nv) * 8;
    const uint32_t id = id_of(ids, row, mask);
    float v[8] = {};
    if (id < num) oc::load8n(table, bf16, (int64_t)id * c + col, c - col, num * c, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = id < num ? v[k] * scale : 0.f;
    oc::store8n(y, bf16, row * c + col, c - col, v);
  }
}

// --- the sort -----------------------------------------------------------------------

struct Pair {
  uint32_t id, row;
};
// One digit of the sort: `bits` bits from `shift` on.  in NULL: the first, from the ids,
// of which those outside the table are left out; else *count pairs.
struct Digit {
  const int32_t* ids;
  uint32_t mask;
  const Pair* in;
  Pair* out;
  uint32_t *hist, *total, *count;  // [tiles][1 << bits], [1 << bits]
  int64_t rows, num;
  int tiles, shift, bits;
};
constexpr int MOST_BITS = 12;

__device__ __forceinline__ bool pair_at(const Digit& a, int64_t i, int64_t n, Pair& p) {
  if (i >= n) return false;
  if (a.in) {
    p = a.in[i];
    return true;
  }
  p = Pair{id_of(a.ids, i, a.mask), (uint32_t)i};
  return p.id < a.num;
}
// The rows of tile t: multiples of 64 but for the last.
__device__ __forceinline__ void tile_range(int64_t n, int tiles, int t, int64_t& i0, int64_t& i1) {
  const int64_t steps = (n + 63) / 64;
  i0 = steps * t / tiles * 64;
  i1 = steps * (t + 1) / tiles * 64;
  if (i1 > n) i1 = n;
}

__global__ __launch_bounds__(64) void k_embed_count(Digit a) {
  __shared__ uint32_t cnt[1 << MOST_BITS];
  const int D = 1 << a.bits, t = blockIdx.x;
  for (int d = threadIdx.x; d < D; d += 64) cnt[d] = 0;
  __syncthreads();
  const int64_t n = a.in ? (int64_t)*a.count : a.rows;
  int64_t i0, i1;
  tile_range(n, a.tiles, t, i0, i1);
#pragma unroll 4
  for (int64_t i = i0 + threadIdx.x; i < i1; i += 64) {
    Pair p;
    if (pair_at(a, i, n, p)) atomicAdd(&cnt[p.id >> a.shift & (D - 1)], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < D; d += 64) a.hist[(int64_t)t * D + d] = cnt[d];
}

// hist[t][d] becomes the number of pairs of digit d in the tiles before t; total[d] theirs
// in all.
__global__ __launch_bounds__(TB) void k_embed_scan(Digit a) {
  const int D = 1 << a.bits, d = blockIdx.x * TB + threadIdx.x;
  if (d >= D) return;
  uint32_t sum = 0;
  for (int t0 = 0; t0 < a.tiles; t0 += 16) {
    uint32_t v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = t0 + j < a.tiles ? a.hist[(int64_t)(t0 + j) * D + d] : 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if (t0 + j < a.tiles) a.hist[(int64_t)(t0 + j) * D + d] = sum;
      sum += v[j];
    }
  }
  a.total[d] = sum;
}

__global__ __launch_bounds__(64) void k_embed_scatter(Digit a) {
  __shared__ uint32_t at[1 << MOST_BITS];
  const int D = 1 << a.bits, t = blockIdx.x, lane = threadIdx.x;
  const int64_t n = a.in ? (int64_t)*a.count : a.rows;
  uint32_t before = 0;
  for (int d0 = 0; d0 < D; d0 += 64) {
    const int d = d0 + lane;
    const uint32_t v = d < D ? a.total[d] : 0;
    uint32_t s = v;
    for (int k = 1; k < 64; k <<= 1) {
      const uint32_t u = __shfl_up(s, k);
      if (lane >= k) s += u;
    }
    if (d < D) at[d] = before + s - v + a.hist[(int64_t)t * D + d];
    before += __shfl(s, 63);
  }
  if (!a.in && t == 0 && lane == 0) *a.count = before;
  __syncthreads();
  int64_t i0, i1;
  tile_range(n, a.tiles, t, i0, i1);
  for (int64_t i = i0; i < i1; i += 64) {
    Pair p{0, 0};
    const bool in = pair_at(a, i + lane, i1, p);
    const uint32_t d = p.id >> a.shift & (D - 1);
    uint64_t same = __ballot(in);
    for (int b = 0; b < a.bits; ++b) {
      const bool one = d >> b & 1;
      const uint64_t ones = __ballot(one);
      same &= one ? ones : ~ones;
    }
    const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
    uint32_t pos = 0;
    if (in) pos = at[d] + rank;
    __syncthreads();
    if (in && rank == 0) at[d] = pos + __popcll(same);
    __syncthreads();
    if (in) a.out[pos] = p;
  }
}

// --- the sums -------------------------------------------------------------------------

struct Sums {
  const Pair* sorted;
  const uint32_t* count;
  const void* dy;
  void* out;
  float* part;  // [chunks][2][c]: of the run open at the chunk's start, and at its end
  int64_t num, rows;
  int c, len;  // len: pairs of a chunk
  bool bf16, out_bf16;
  float scale;
  int64_t chunk_blocks;
};

// A thread's sums of eight columns: at most MOST_ADDED values in fp32, the rest in double.
constexpr int MOST_ADDED = 64;
struct Acc {
  float f[8];
  double d[8];
  int n;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = 0.f, d[k] = 0.0;
    n = 0;
  }
  __device__ __forceinline__ void add(const float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] += v[k];
    if (++n == MOST_ADDED) {
#pragma unroll
      for (int k = 0; k < 8; ++k) d[k] += (double)f[k], f[k] = 0.f;
      n = 0;
    }
  }
};

// Zeros in the table's rows that no id names.  A wave has 64 rows, each lane looks for one
// of them among the sorted ids.
__device__ __forceinline__ void zero_rows(const Sums& a, int64_t n, int64_t wave) {
  const int lane = threadIdx.x & 63;
  const int64_t v = wave * 64 + lane;
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if ((int64_t)a.sorted[mid].id < v) lo = mid + 1;
    else hi = mid;
  }
  const bool none = v < a.num && !(lo < n && (int64_t)a.sorted[lo].id == v);
  const float zero[8] = {};
  for (uint64_t m = __ballot(none); m; m &= m - 1) {
    const int64_t row = wave * 64 + __builtin_ctzll(m);
    for (int col = lane * 8; col < a.c; col += 512)
      oc::store8n(a.out, a.out_bf16, row * a.c + col, a.c - col, zero);
  }
}

// Groups of tpr lanes, each with 8 tpr columns of a chunk (slabs of them where rows are
// longer).  The blocks behind the chunks' zero the table's other rows.
__global__ __launch_bounds__(TB) void k_embed_sums(Sums a, int tpr, int slabs) {
  const int64_t n = *a.count;
  if (blockIdx.x >= a.chunk_blocks) {
    zero_rows(a, n, (int64_t)(blockIdx.x - a.chunk_blocks) * (TB / 64) + threadIdx.x / 64);
    return;
  }
  const int64_t unit = (int64_t)blockIdx.x * (TB / tpr) + threadIdx.x / tpr;
  const int64_t chunk = unit / slabs;
  const int col = ((int)(unit - chunk * slabs) * tpr + threadIdx.x % tpr) * 8;
  const int64_t i0 = chunk * a.len, i1 = i0 + a.len < n ? i0 + a.len : n;
  if (i0 >= i1 || col >= a.c) return;
  const int cnt = a.c - col;
  const int64_t all = a.rows * a.c;
  uint32_t id = a.sorted[i0].id;
  bool first = i0 > 0 && a.sorted[i0 - 1].id == id;  // the run began in a chunk before
  const bool goes_on = i1 < n && a.sorted[i1].id == a.sorted[i1 - 1].id;
  Acc acc;
  acc.clear();
  const auto flush = [&](bool open) {
    float v[8];
    if (first || open) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = (float)((double)acc.f[k] + acc.d[k]);
      oc::store8n(a.part, false, (chunk * 2 + (first ? 0 : 1)) * a.c + col, cnt, v);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = (float)(((double)acc.f[k] + acc.d[k]) * a.scale);
      oc::store8n(a.out, a.out_bf16, (int64_t)id * a.c + col, cnt, v);
    }
  };
  constexpr int U = 8;  // rows in flight
  for (int64_t i = i0; i < i1; i += U) {
    Pair p[U];
    float v[U][8];
#pragma unroll
    for (int j = 0; j < U; ++j) p[j] = a.sorted[i + j < i1 ? i + j : i1 - 1];
#pragma unroll
    for (int j = 0; j < U; ++j)
      oc::load8n(a.dy, a.bf16, (int64_t)p[j].row * a.c + col, cnt, all, v[j]);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (i + j >= i1) break;
      if (p[j].id != id) {
        flush(false);
        acc.clear();
        id = p[j].id;
        first = false;
      }
      acc.add(v[j]);
    }
  }
  flush(goes_on);
}

// The runs that go on over a chunk's end: the workgroup of the chunk where one begins adds
// its partial sums, rl lanes a column, in double and in a fixed order.
__global__ __launch_bounds__(TB) void k_embed_join(Sums a, int tpr) {
  __shared__ double red[TB][9];
  const int64_t n = *a.count, chunk = blockIdx.x;
  const int64_t i0 = chunk * a.len, i1 = i0 + a.len;
  if (i1 >= n) return;
  const uint32_t id = a.sorted[i1 - 1].id;
  if (a.sorted[i1].id != id) return;
  if (a.sorted[i0].id == id && i0 > 0 && a.sorted[i0 - 1].id == id) return;
  int64_t more = 0;  // chunks that the run goes on in
  for (;;) {
    const int64_t at = (chunk + 1 + more + threadIdx.x) * a.len;
    const int k = __syncthreads_count(at < n && a.sorted[at].id == id);
    more += k;
    if (k < TB) break;
  }
  const int tc = threadIdx.x % tpr, tr = threadIdx.x / tpr, rl = TB / tpr;
  for (int col = (blockIdx.y * tpr + tc) * 8; col - tc * 8 < a.c; col += gridDim.y * tpr * 8) {
    double s[8] = {};
    if (col < a.c)
      for (int64_t j = tr; j <= more; j += rl) {
        float v[8];
        oc::load8n(a.part, false, ((chunk + j) * 2 + (j ? 0 : 1)) * a.c + col, a.c - col,
                   INT64_MAX, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += (double)v[k];
      }
#pragma unroll
    for (int k = 0; k < 8; ++k) red[threadIdx.x][k] = s[k];
    __syncthreads();
    if (tr == 0 && col < a.c) {
      float v[8];
      for (int r = 1; r < rl; ++r)
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += red[r * tpr + tc][k];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = (float)(s[k] * a.scale);
      oc::store8n(a.out, a.out_bf16, (int64_t)id * a.c + col, a.c - col, v);
    }
    __syncthreads();
  }
}

// Up to 64 rows: a wave finds a table row's among them at once.
__global__ __launch_bounds__(TB) void k_embed_few(const int32_t* ids, uint32_t mask, int rows,
                                                  Sums a) {
  const int lane = threadIdx.x & 63;
  const uint32_t id = lane < rows ? id_of(ids, lane, mask) : 0;
  for (int64_t v = (int64_t)blockIdx.x * (TB / 64) + threadIdx.x / 64; v < a.num;
       v += (int64_t)gridDim.x * (TB / 64)) {
    const uint64_t mine = __ballot(lane < rows && id == (uint64_t)v);
    for (int col = lane * 8; col < a.c; col += 512) {
      float s[8] = {};
      for (uint64_t m = mine; m; m &= m - 1) {
        float g[8];
        oc::load8n(a.dy, a.bf16, (int64_t)__builtin_ctzll(m) * a.c + col, a.c - col, a.rows * a.c,
                   g);
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += g[k];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] *= a.scale;
      oc::store8n(a.out, a.out_bf16, v * a.c + col, a.c - col, s);
    }
  }
}

// --- the plan ---------------------------------------------------------------------------

struct Plan {
  int passes, bits, tiles, len, tpr, slabs;
  int64_t chunks;
  size_t hist, total, count, a, b, part, bytes;
};
constexpr int FEW = 64;
Plan plan_of(int64_t rows, int64_t num, int c) {
  Plan p{};
  int bits = 1;
  while (((int64_t)1 << bits) < num) ++bits;
  p.passes = (int)cdiv(bits, MOST_BITS);
  p.bits = (int)cdiv(bits, p.passes);
  // (a tile's steps follow one another, the scan over the tiles too)
  p.tiles = (int)std::max<int64_t>(
      1, rows <= (1 << 20) ? std::min<int64_t>(cdiv(rows, 512), 128)
                           : std::min<int64_t>(cdiv(rows, 8192), 1024));
  p.len = (int)std::max<int64_t>(32, cdiv(rows, 2048));
  p.chunks = cdiv(rows, p.len);
  const int nv = (int)cdiv(c, 8);
  p.tpr = 1;
  while (p.tpr < nv && p.tpr < 64) p.tpr *= 2;
  p.slabs = (int)cdiv(nv, p.tpr);
  size_t at = 0;
  const auto take = [&](size_t n) {
    const size_t was = at;
    at += oc::align256(n);
    return was;
  };
  p.count = take(4);
  p.total = take((size_t)4 << p.bits);
  p.hist = take(((size_t)4 << p.bits) * p.tiles);
  p.a = take((size_t)rows * sizeof(Pair));
  p.b = p.passes > 1 ? take((size_t)rows * sizeof(Pair)) : p.a;
  p.part = take((size_t)p.chunks * 2 * c * sizeof(float) + 32);
  p.bytes = at;
  return p;
}

oc_status check(const char* who, int32_t flags, oc_dtype dt, int64_t rows, int64_t num,
                int32_t c) {
  OC_TRY(oc::check_rows(who, dt, rows, c));
  if (flags & ~OC_IDS_KEYS) return oc::fail(OC_ERR_ARG, "%s: flags %d", who, flags);
  if (num < 1 || num >= oc::ROWS_MOST)
    return oc::fail(OC_ERR_ARG, "%s: a table of %lld rows", who, (long long)num);
  if (num * c >= (int64_t)1 << 40)
    return oc::fail(OC_ERR_UNSUPPORTED, "%s: %lld table rows of %d channels are too many", who,
                    (long long)num, c);
  return OC_OK;
}
uint32_t id_mask(int32_t flags) { return flags & OC_IDS_KEYS ? KEY_BITS : ~0u; }

}  // namespace

extern "C" {

oc_status oc_embed_fwd(oc_dtype dt, int32_t flags, int64_t rows, int64_t num, int32_t c,
                       const int32_t* ids, const void* table, float scale, void* y,
                       hipStream_t s) {
  const char* who = "oc_embed_fwd";
  OC_TRY(check(who, flags, dt, rows, num, c));
  if (rows == 0) return OC_OK;
  if (!ids || !table || !y) return oc::fail(OC_ERR_ARG, "%s: NULL buffer", who);
  const size_t e = oc::value_bytes(dt);
  const oc::Span sp[] = {{"y", y, (size_t)rows * c * e, true, nullptr},
                         {"ids", ids, (size_t)rows * 4, false, nullptr},
                         {"table", table, (size_t)num * c * e, false, nullptr}};
  OC_TRY(oc::check_spans(who, sp));
  const int64_t groups = rows * cdiv(c, 8);
  oc::launch_main(k_embed, dim3((unsigned)std::min(cdiv(groups, TB), MOST_BLOCKS)), dim3(TB), s,
                  ids, id_mask(flags), rows, num, (int)c, table, dt == OC_BF16, scale, y);
  OC_LAUNCH_CHECK();
  return OC_OK;
}

size_t oc_embed_bwd_workspace(int64_t rows, int64_t num, int32_t c) {
  if (rows <= FEW || rows >= oc::ROWS_MOST || num < 1 || num >= oc::ROWS_MOST || c < 1 ||
      c > oc::COLS_MOST)
    return 0;
  return plan_of(rows, num, c).bytes;
}

oc_status oc_embed_bwd(oc_dtype dt, int32_t flags, int64_t rows, int64_t num, int32_t c,
                       const int32_t* ids, const void* dy, float scale, oc_dtype dtable_dt,
                       void* dtable, void* ws, size_t ws_bytes, hipStream_t s) {
  const char* who = "oc_embed_bwd";
  OC_TRY(check(who, flags, dt, rows, num, c));
  if (dtable_dt != OC_F32 && dtable_dt != dt)
    return oc::fail(OC_ERR_ARG, "%s: the gradient has dtype %d", who, (int)dtable_dt);
  if (!dtable || (rows > 0 && (!ids || !dy))) return oc::fail(OC_ERR_ARG, "%s: NULL buffer", who);
  const size_t need = oc_embed_bwd_workspace(rows, num, c);
  OC_TRY(oc::check_row_ws(who, ws, ws_bytes, need));
  const oc::Span sp[] = {
      {"dtable", dtable, (size_t)num * c * oc::value_bytes(dtable_dt), true, nullptr},
      {"the workspace", need ? ws : nullptr, need, true, nullptr},
      {"ids", ids, (size_t)rows * 4, false, nullptr},
      {"dy", dy, (size_t)rows * c * oc::value_bytes(dt), false, nullptr}};
  OC_TRY(oc::check_spans(who, sp));
  Sums a{};
  a.dy = dy;
  a.out = dtable;
  a.num = num;
  a.rows = rows;
  a.c = c;
  a.bf16 = dt == OC_BF16;
  a.out_bf16 = dtable_dt == OC_BF16;
  a.scale = scale;
  if (rows <= FEW) {
    oc::launch_main(k_embed_few, dim3((unsigned)std::min(cdiv(num, TB / 64), MOST_BLOCKS)),
                    dim3(TB), s, ids, id_mask(flags), (int)rows, a);
    OC_LAUNCH_CHECK();
    return OC_OK;
  }
  const Plan p = plan_of(rows, num, c);
  char* w = (char*)ws;
  Digit d{ids, id_mask(flags), nullptr, nullptr, (uint32_t*)(w + p.hist),
          (uint32_t*)(w + p.total), (uint32_t*)(w + p.count), rows, num, p.tiles, 0, p.bits};
  for (int i = 0; i < p.passes; ++i) {
    d.out = (Pair*)(w + (i & 1 ? p.b : p.a));
    d.shift = i * p.bits;
    oc::launch(k_embed_count, dim3((unsigned)p.tiles), dim3(64), 0, s, d);
    oc::launch(k_embed_scan, dim3((unsigned)cdiv(1 << p.bits, TB)), dim3(TB), 0, s, d);
    oc::launch(k_embed_scatter, dim3((unsigned)p.tiles), dim3(64), 0, s, d);
    d.in = d.out;
  }
  a.sorted = d.in;
  a.count = d.count;
  a.part = (float*)(w + p.part);
  a.len = p.len;
  a.chunk_blocks = cdiv(p.chunks * p.slabs, TB / p.tpr);
  const int64_t zero_blocks = cdiv(num, TB);
  oc::launch_main(k_embed_sums, dim3((unsigned)(a.chunk_blocks + zero_blocks)), dim3(TB), s, a,
                  p.tpr, p.slabs);
  if (p.chunks > 1)
    oc::launch(k_embed_join, dim3((unsigned)p.chunks, (unsigned)std::min(p.slabs, 16)), dim3(TB),
               0, s, a, p.tpr);
  OC_LAUNCH_CHECK();
  return OC_OK;
}

}  // extern "C"
