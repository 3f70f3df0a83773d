// Table rows by id (oc_embed_fwd), y[r] = scale table[id[r]], and the table's gradient
// (oc_embed_bwd), dtable[v] = scale times the sum of dy[r] over the rows r with id v.
//
// The gradient without floating-point atomics, so that its bits do not depend on the order
// of the workgroups: the rows are sorted by id (stable, so that those of one id stay in
// order) and the sorted list is cut into pieces of equal length, one for a group of
// lanes, whose runs of one id are summed in order.  A run inside one piece is written to
// the table's row; one that goes on over a border leaves a partial sum a piece, added
// through LDS where the run stays in the workgroup's chunk, else by k_embed_join.
// A run's chain of additions: a piece's rows, at most 64 of them in fp32 and the rest in
// double; the pieces of a chunk one after another (up to 256 of 8 columns, 4 of 512 and
// more) in double; and in double up to nine chunks one after another, or of up to 2048
// chunks every 16th to 512th and then those 16 to 512 sums.  Each piece's and each chunk's
// sum is rounded to fp32 on its way.
//
// The sort takes the ids' bits in digits of up to nine, lowest first.  A tile of rows is
// one workgroup's: count writes each tile's number of rows of every digit value, and
// scatter adds those numbers up itself (all values below its own, and its own in the tiles
// before), so that a digit takes two launches.  (Counting the next digit by atomics where
// the scatter puts the rows saves a launch of 3 to 5 us and costs 6 us for 65536 rows and
// 14 for 260000.)  A wave takes its rows 64 at a time, in order: the place of a row among
// those of its digit is a count of the lanes before it with the same digit.  Up to SMALL
// rows are sorted by one workgroup in LDS (4000 rows, two digits: 9.3 us; the four
// launches take 17).
//
// The lookup and the sums are bound by memory, the sort by its chain of launches.  65536
// rows of 1024 bf16 channels, a table of 32768 rows, skewed ids: lookup 39 us (4.5 TB/s of
// what is read and written), sort 22, sums with the zeros 55 (3.7 TB/s), joins 7.
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

// A group of tpr lanes has ROWS rows, whose ids and then whose vectors are in flight
// together; lanes step over the columns.
template <bool BF, int ROWS>
__global__ __launch_bounds__(TB) void k_embed(const int32_t* ids, uint32_t mask, int64_t rows,
                                              int64_t num, int c, const void* table, int tpr,
                                              float scale, void* y) {
  const int per = TB / tpr, tc = threadIdx.x % tpr;
  const int64_t all = num * c, step = (int64_t)gridDim.x * per * ROWS;
  for (int64_t r0 = (int64_t)blockIdx.x * per * ROWS + threadIdx.x / tpr; r0 < rows; r0 += step) {
    uint32_t id[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
      const int64_t r = r0 + j * per;
      id[j] = r < rows ? id_of(ids, r, mask) : ~0u;
    }
    for (int col = tc * 8; col < c; col += tpr * 8) {
      const int cnt = c - col;
      oc::Raw<BF> raw[ROWS];
#pragma unroll
      for (int j = 0; j < ROWS; ++j) {
        const int64_t at = (int64_t)id[j] * c;
        if (id[j] < num) oc::raw_load(raw[j], table, oc::Place{at, col, cnt, all - at});
      }
#pragma unroll
      for (int j = 0; j < ROWS; ++j) {
        const int64_t r = r0 + j * per;
        if (r >= rows) break;
        float v[8];
        oc::unpack(raw[j], v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = id[j] < num ? v[k] * scale : 0.f;
        oc::row_store<BF>(y, oc::Place{r * c, col, cnt, 0}, v);
      }
    }
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
  uint32_t *hist, *count;  // hist[tiles][1 << bits]
  int64_t rows, num;
  int tiles, shift, bits, passes;
};
constexpr int MOST_BITS = 9, MOST_D = 1 << MOST_BITS;
constexpr int SB = 1024, SW = SB / 64;  // threads and waves of a sorting workgroup
constexpr int SMALL = 4096;

__device__ __forceinline__ bool pair_at(const Digit& a, int64_t i, int64_t n, Pair& p) {
  if (i >= n) return false;
  if (a.in) {
    p = a.in[i];
    return true;
  }
  p = Pair{id_of(a.ids, i, a.mask), (uint32_t)i};
  return p.id < a.num;
}
// Part t of the rows in `parts`: multiples of 64 but for the last.
__device__ __forceinline__ void part_of(int64_t from, int64_t to, int parts, int t, int64_t& i0,
                                        int64_t& i1) {
  const int64_t steps = (to - from + 63) / 64;
  i0 = from + steps * t / parts * 64;
  i1 = from + steps * (t + 1) / parts * 64;
  if (i1 > to) i1 = to;
}
// The lanes with this lane's digit, of those that have one.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, int bits, bool in) {
  uint64_t same = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const bool one = d >> b & 1;
    const uint64_t ones = __ballot(one);
    same &= one ? ones : ~ones;
  }
  return same;
}
__device__ __forceinline__ int lanes_before(uint64_t m) {
  return __popcll(m & (((uint64_t)1 << (threadIdx.x & 63)) - 1));
}
// What this wave wrote to LDS is there for its next reads.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// v[d] of D values becomes the sum of those before it, by one wave (PER a lane).
// Returns the sum of all, in each lane.
__device__ __forceinline__ uint32_t scan_digits(uint32_t* v, int D) {
  constexpr int PER = MOST_D / 64;
  const int lane = threadIdx.x & 63;
  uint32_t x[PER], sum = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const uint32_t y = lane * PER + k < D ? v[lane * PER + k] : 0;
    x[k] = sum;
    sum += y;
  }
  uint32_t upto = sum;
  for (int k = 1; k < 64; k <<= 1) {
    const uint32_t u = __shfl_up(upto, k);
    if (lane >= k) upto += u;
  }
#pragma unroll
  for (int k = 0; k < PER; ++k)
    if (lane * PER + k < D) v[lane * PER + k] = upto - sum + x[k];
  return __shfl(upto, 63);
}

// at[w] of this thread's digit value becomes `sum` and the counts of the waves before w;
// returns the sum with all.
__device__ __forceinline__ uint32_t before_waves(uint32_t (*at)[MOST_D], uint32_t sum) {
  uint32_t v[SW];
#pragma unroll
  for (int u = 0; u < SW; ++u) v[u] = at[u][threadIdx.x];
#pragma unroll
  for (int u = 0; u < SW; ++u) {
    at[u][threadIdx.x] = sum;
    sum += v[u];
  }
  return sum;
}

__global__ __launch_bounds__(SB) void k_embed_count(Digit a) {
  __shared__ uint32_t cnt[MOST_D];
  const int D = 1 << a.bits, t = blockIdx.x;
  if ((int)threadIdx.x < D) cnt[threadIdx.x] = 0;
  __syncthreads();
  const int64_t n = a.in ? (int64_t)*a.count : a.rows;
  int64_t i0, i1;
  part_of(0, n, a.tiles, t, i0, i1);
#pragma unroll 4
  for (int64_t i = i0 + threadIdx.x; i < i1; i += SB) {
    Pair p;
    if (pair_at(a, i, n, p)) atomicAdd(&cnt[p.id >> a.shift & (D - 1)], 1u);
  }
  __syncthreads();
  if ((int)threadIdx.x < D) a.hist[(int64_t)t * D + threadIdx.x] = cnt[threadIdx.x];
}

__global__ __launch_bounds__(SB) void k_embed_scatter(Digit a) {
  __shared__ uint32_t total[MOST_D], before[MOST_D], at[SW][MOST_D];
  const int D = 1 << a.bits, t = blockIdx.x, w = threadIdx.x / 64;
  const int64_t n = a.in ? (int64_t)*a.count : a.rows;
  for (int i = threadIdx.x; i < SW << a.bits; i += SB) at[i >> a.bits][i & (D - 1)] = 0;
  if ((int)threadIdx.x < D) total[threadIdx.x] = before[threadIdx.x] = 0;
  __syncthreads();
  int64_t i0, i1, j0, j1;
  part_of(0, n, a.tiles, t, i0, i1);
  part_of(i0, i1, SW, w, j0, j1);
  // the wave's rows of each digit value
  for (int64_t i = j0 + (threadIdx.x & 63); i < j1; i += 64) {
    Pair p;
    if (pair_at(a, i, n, p)) atomicAdd(&at[w][p.id >> a.shift & (D - 1)], 1u);
  }
  {  // every tile's, by threads of digit value d and every SB / D-th tile
    const int d = threadIdx.x & (D - 1);
    uint32_t all = 0, early = 0;
#pragma unroll 8
    for (int u = threadIdx.x >> a.bits; u < a.tiles; u += SB >> a.bits) {
      const uint32_t v = a.hist[(int64_t)u * D + d];
      all += v;
      early += u < t ? v : 0;
    }
    atomicAdd(&total[d], all);
    atomicAdd(&before[d], early);
  }
  __syncthreads();
  if (w == 0) {
    const uint32_t sum = scan_digits(total, D);
    if (!a.in && t == 0 && threadIdx.x == 0) *a.count = sum;
  }
  __syncthreads();
  if ((int)threadIdx.x < D) {
    before_waves(at, total[threadIdx.x] + before[threadIdx.x]);
  }
  __syncthreads();
  for (int64_t i = j0; i < j1; i += 64) {
    Pair p{0, 0};
    const bool in = pair_at(a, i + (threadIdx.x & 63), j1, p);
    const uint32_t d = p.id >> a.shift & (D - 1);
    const uint64_t same = same_digit(d, a.bits, in);
    const int rank = lanes_before(same);
    uint32_t pos = 0;
    if (in) pos = at[w][d] + rank;
    wave_sync();
    if (in && rank == 0) at[w][d] = pos + __popcll(same);
    wave_sync();
    if (in) a.out[pos] = p;
  }
}

// Up to SMALL rows, every digit: a thread's pairs are rows 256 w + 64 j + lane of the list.
__global__ __launch_bounds__(SB) void k_embed_sort_small(Digit a) {
  __shared__ Pair list[SMALL];
  __shared__ uint32_t at[SW][MOST_D], total[MOST_D], valid;
  constexpr int J = SMALL / SB;
  const int D = 1 << a.bits, w = threadIdx.x / 64, lane = threadIdx.x & 63;
  const int rows = (int)a.rows, i0 = w * 64 * J + lane;
  if (threadIdx.x == 0) valid = 0;
  __syncthreads();
  Pair p[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int i = i0 + j * 64;
    // ids outside the table go behind the others, where *count leaves them out
    p[j] = Pair{i < rows ? id_of(a.ids, i, a.mask) : ~0u, (uint32_t)i};
    const bool in = i < rows && p[j].id < a.num;
    if (!in) p[j].id = (uint32_t)a.num;
    const uint64_t m = __ballot(in);
    if (lane == 0 && m) atomicAdd(&valid, (uint32_t)__popcll(m));
  }
  for (int s = 0; s < a.passes; ++s) {
    for (int i = threadIdx.x; i < SW << a.bits; i += SB) at[i >> a.bits][i & (D - 1)] = 0;
    __syncthreads();
    uint32_t rank[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const uint32_t d = p[j].id >> s * a.bits & (D - 1);
      const uint64_t same = same_digit(d, a.bits, true);
      const int r = lanes_before(same);
      rank[j] = at[w][d] + r;
      wave_sync();
      if (r == 0) at[w][d] = rank[j] + __popcll(same);
      wave_sync();
    }
    __syncthreads();
    if ((int)threadIdx.x < D) {
      total[threadIdx.x] = before_waves(at, 0);
    }
    __syncthreads();
    if (w == 0) scan_digits(total, D);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const uint32_t d = p[j].id >> s * a.bits & (D - 1);
      list[total[d] + at[w][d] + rank[j]] = p[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j) p[j] = list[i0 + j * 64];
  }
#pragma unroll
  for (int j = 0; j < J; ++j)
    if (i0 + j * 64 < rows) a.out[i0 + j * 64] = p[j];
  if (threadIdx.x == 0) *a.count = valid;
}

// --- the sums -------------------------------------------------------------------------

struct Sums {
  const Pair* sorted;
  const uint32_t* count;
  const void* dy;
  void* out;
  float* part;  // [chunks][2][c]: sums of the run open at the chunk's start, and its end
  int64_t num, rows;
  int c, len, chunk;  // len, chunk: pairs of a piece and of a chunk
  bool bf16, out_bf16;
  float scale;
  int64_t zero_blocks;
};

// A thread's sums of eight columns: at most MOST_ADDED values in fp32, the rest in double
// (LONG: there may be more).
constexpr int MOST_ADDED = 64;
template <bool LONG>
struct Acc {
  float f[8];
  double d[LONG ? 8 : 1];
  int n;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      f[k] = 0.f;
      if (LONG) d[LONG ? k : 0] = 0.0;
    }
    n = 0;
  }
  __device__ __forceinline__ void add(const float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] += v[k];
    if (LONG && ++n == MOST_ADDED) {
#pragma unroll
      for (int k = 0; k < 8; ++k) d[LONG ? k : 0] += (double)f[k], f[k] = 0.f;
      n = 0;
    }
  }
  __device__ __forceinline__ void times(float scale, float (&v)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      v[k] = LONG ? (float)(((double)f[k] + d[LONG ? k : 0]) * scale) : f[k] * scale;
  }
};

// The first place in the sorted list whose id is at least v, by a wave: 64 probes a step.
__device__ __forceinline__ int64_t place_of(const Sums& a, int64_t n, int64_t v) {
  const int lane = threadIdx.x & 63;
  int64_t lo = 0, len = n;  // it is lo .. lo + len
  while (len > 0) {
    const int64_t step = (len + 63) / 64, at = lo + step * (lane + 1) - 1;
    const bool below = at < lo + len && (int64_t)a.sorted[at].id < v;
    const int k = __popcll(__ballot(below));
    const int64_t skip = k * step;
    lo += skip;
    len = len - skip < step - 1 ? len - skip : step - 1;
    if (len < 0) len = 0;
  }
  return lo;
}

// Zeros in the table's rows that no id names, 64 rows a wave: the part of the sorted list
// with their ids is read where it is short, else each lane looks for its own row's there.
__device__ __forceinline__ void zero_rows(const Sums& a, int64_t n, int64_t wave) {
  __shared__ unsigned long long named[TB / 64];
  const int lane = threadIdx.x & 63, w = threadIdx.x / 64;
  const int64_t v0 = wave * 64, v = v0 + lane;
  if (v0 >= a.num) return;
  const int64_t from = place_of(a, n, v0), to = place_of(a, n, v0 + 64);
  uint64_t none;
  if (to - from <= 256) {
    if (lane == 0) named[w] = 0;
    wave_sync();
    for (int64_t i = from + lane; i < to; i += 64)
      atomicOr(&named[w], 1ull << (a.sorted[i].id - (uint32_t)v0));
    wave_sync();
    none = ~named[w] & __ballot(v < a.num);
  } else {
    int64_t lo = from, hi = to;
    while (lo < hi) {
      const int64_t mid = (lo + hi) >> 1;
      if ((int64_t)a.sorted[mid].id < v) lo = mid + 1;
      else hi = mid;
    }
    none = __ballot(v < a.num && !(lo < to && (int64_t)a.sorted[lo].id == v));
  }
  const float zero[8] = {};
  for (uint64_t m = none; m; m &= m - 1) {
    const int64_t row = v0 + __builtin_ctzll(m);
    for (int col = lane * 8; col < a.c; col += 512)
      oc::store8n(a.out, a.out_bf16, row * a.c + col, a.c - col, zero);
  }
}

// A workgroup has a chunk of the sorted list and 8 tpr columns (a slab of them where rows
// are longer), each of its groups of tpr lanes a piece of the chunk.  The first
// workgroups zero the table's other rows.
template <bool BF, bool LONG>
__global__ __launch_bounds__(TB) void k_embed_sums(Sums a, int tpr, int slabs) {
  __shared__ float open[2][8][TB];  // sums of the run open at the piece's start, and its end
  __shared__ bool through[TB];      // the first is the second: all of the piece
  const int64_t n = *a.count;
  if (blockIdx.x < a.zero_blocks) {
    zero_rows(a, n, (int64_t)blockIdx.x * (TB / 64) + threadIdx.x / 64);
    return;
  }
  const int64_t unit = blockIdx.x - a.zero_blocks, chunk = unit / slabs;
  const int g = threadIdx.x / tpr, tc = threadIdx.x % tpr, G = TB / tpr;
  const int col = ((int)(unit - chunk * slabs) * tpr + tc) * 8, cnt = a.c - col;
  const int64_t b0 = chunk * G * a.len, i0 = b0 + (int64_t)g * a.len;
  const int64_t i1 = i0 + a.len < n ? i0 + a.len : n;
  if (b0 >= n) return;
  uint32_t id = 0;
  bool first = false, goes_on = false, begun = false;  // begun: the last run began here
  const auto store = [&](uint32_t row, const float(&v)[8]) {
    oc::store8n(a.out, a.out_bf16, (int64_t)row * a.c + col, cnt, v);
  };
  if (i0 < i1) {
    constexpr int U = BF ? 8 : 4;  // rows in flight
    Pair p[U];
    const auto pairs = [&](int64_t i) {
#pragma unroll
      for (int j = 0; j < U; ++j) p[j] = a.sorted[i + j < i1 ? i + j : i1 - 1];
    };
    pairs(i0);
    id = p[0].id;
    first = i0 > 0 && a.sorted[i0 - 1].id == id;  // the run began in a piece before
    goes_on = i1 < n && a.sorted[i1].id == a.sorted[i1 - 1].id;
    begun = !first;
    Acc<LONG> acc;
    acc.clear();
    const auto flush = [&](bool left_open) {
      float v[8];
      if (cnt <= 0) return;
      if (begun && !left_open) {
        acc.times(a.scale, v);
        store(id, v);
      } else {
        acc.times(1.f, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) open[begun ? 1 : 0][k][threadIdx.x] = v[k];
      }
    };
    for (int64_t i = i0; i < i1; i += U) {
      oc::Raw<BF> raw[U];
      uint32_t ids[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int64_t at = (int64_t)p[j].row * a.c;
        if (cnt > 0) oc::raw_load(raw[j], a.dy, oc::Place{at, col, cnt, a.rows * a.c - at});
        ids[j] = p[j].id;
      }
      if (i + U < i1) pairs(i + U);
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (i + j >= i1) break;
        if (ids[j] != id) {
          flush(false);
          acc.clear();
          id = ids[j];
          begun = true;
        }
        float v[8];
        oc::unpack(raw[j], v);
        acc.add(v);
      }
    }
    flush(goes_on);
  }
  if (tc == 0) through[g] = first && !begun && goes_on;
  __syncthreads();
  if (cnt <= 0) return;
  double sum[8];
  // pieces from g + 1 on, to the run's end: whether that is in this chunk
  const auto add_on = [&]() {
    for (int h = g + 1; h < G; ++h) {
#pragma unroll
      for (int k = 0; k < 8; ++k) sum[k] += (double)open[0][k][h * tpr + tc];
      if (!through[h]) return true;
    }
    return false;
  };
  const auto store_part = [&](int which) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)sum[k];
    oc::store8n(a.part, false, (chunk * 2 + which) * a.c + col, cnt, v);
  };
  if (goes_on && begun) {
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = (double)open[1][k][threadIdx.x];
    if (add_on()) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = (float)(sum[k] * a.scale);
      store(id, v);
    } else {
      store_part(1);
    }
  }
  if (g == 0 && first) {
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = (double)open[0][k][threadIdx.x];
    if (through[0]) add_on();
    store_part(0);
  }
}

// The runs that go on over a chunk's end, whose partial sums are added in double and in a
// fixed order.  Each wave looks at the end of one chunk.  Where a run begins in it and goes
// on in at most WAVE_MORE chunks, as nearly all do, the wave adds it; the others it leaves
// to the workgroup, which has rl lanes a column.
constexpr int JB = 512, JW = JB / 64, WAVE_MORE = 8;
__global__ __launch_bounds__(JB, 4) void k_embed_join(Sums a, int tpr) {
  __shared__ double red[8][JB];
  __shared__ bool longer[JW];
  const int64_t n = *a.count;
  const int w = threadIdx.x / 64, lane = threadIdx.x & 63;
  const auto load = [&](int64_t chunk, int which, int col, float(&v)[8]) {
    oc::load8n(a.part, false, (chunk * 2 + which) * a.c + col, a.c - col, INT64_MAX, v);
  };
  const auto finish = [&](uint32_t id, int col, const double(&s)[8]) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)(s[k] * a.scale);
    oc::store8n(a.out, a.out_bf16, (int64_t)id * a.c + col, a.c - col, v);
  };
  {
    const int64_t chunk = (int64_t)blockIdx.x * JW + w, i0 = chunk * a.chunk, i1 = i0 + a.chunk;
    bool left = false;
    if (i1 < n) {
      const uint32_t id = a.sorted[i1].id, was = a.sorted[i1 - 1].id, from = a.sorted[i0].id;
      const uint32_t before = i0 > 0 ? a.sorted[i0 - 1].id : ~0u;  // (no id)
      const int64_t at = i1 + (int64_t)lane * a.chunk;
      const uint64_t on = __ballot(at < n && a.sorted[at].id == id);
      if (was == id && !(from == id && before == id)) {
        const int more = on == ~0ull ? 64 : __builtin_ctzll(~on);  // chunks it goes on in
        left = more > WAVE_MORE;
        for (int col = (blockIdx.y * tpr + lane) * 8; !left && lane < tpr && col < a.c;
             col += gridDim.y * tpr * 8) {
          float v[8];
          double s[8];
          load(chunk, 1, col, v);
#pragma unroll
          for (int k = 0; k < 8; ++k) s[k] = (double)v[k];
#pragma unroll 4
          for (int j = 1; j <= more; ++j) {
            load(chunk + j, 0, col, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k] += (double)v[k];
          }
          finish(id, col, s);
        }
      }
    }
    if (lane == 0) longer[w] = left;
  }
  __syncthreads();
  const int tc = threadIdx.x % tpr, tr = threadIdx.x / tpr, rl = JB / tpr;
  for (int q = 0; q < JW; ++q) {
    if (!longer[q]) continue;
    const int64_t chunk = (int64_t)blockIdx.x * JW + q;
    const uint32_t id = a.sorted[(chunk + 1) * a.chunk].id;
    int64_t more = 0;  // chunks that the run goes on in
    for (;;) {
      const int64_t at = (chunk + 1 + more + threadIdx.x) * a.chunk;
      const int k = __syncthreads_count(at < n && a.sorted[at].id == id);
      more += k;
      if (k < JB) break;
    }
    for (int c0 = blockIdx.y * tpr * 8; c0 < a.c; c0 += gridDim.y * tpr * 8) {
      const int col = c0 + tc * 8;
      double s[8] = {};
      if (col < a.c) {
#pragma unroll 4
        for (int64_t j = tr; j <= more; j += rl) {
          float v[8];
          load(chunk + j, j ? 0 : 1, col, v);
#pragma unroll
          for (int k = 0; k < 8; ++k) s[k] += (double)v[k];
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) red[k][threadIdx.x] = s[k];
      __syncthreads();
      if (tr == 0 && col < a.c) {
        const int most = more < rl - 1 ? (int)more : rl - 1;
        for (int r = 1; r <= most; ++r)
#pragma unroll
          for (int k = 0; k < 8; ++k) s[k] += red[k][r * tpr + tc];
        finish(id, col, s);
      }
      __syncthreads();
    }
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
  size_t hist, count, a, b, part, bytes;
};
constexpr int FEW = 64;
Plan plan_of(int64_t rows, int64_t num, int c) {
  Plan p{};
  const bool small = rows <= SMALL;
  int bits = 1;
  while (((int64_t)1 << bits) < num + (small ? 1 : 0)) ++bits;  // (small: num is a key too)
  p.passes = (int)cdiv(bits, MOST_BITS);
  p.bits = (int)cdiv(bits, p.passes);
  // a tile is one step of a workgroup's waves where there are few rows; every scatter
  // reads all tiles' counts, so there are at most 128 of them up to 2^20 rows
  p.tiles = (int)(rows <= (1 << 20) ? std::min<int64_t>(cdiv(rows, SB), 128)
                                    : std::min<int64_t>(cdiv(rows, 8192), 512));
  const int nv = (int)cdiv(c, 8);
  p.tpr = 1;
  while (p.tpr < nv && p.tpr < 64) p.tpr *= 2;
  p.slabs = (int)cdiv(nv, p.tpr);
  // pieces of 16 rows, or of 8 where those would leave CUs without a workgroup or two
  // (35472 x 256 fp32: sums 10.2 us instead of 12.8; 65536 x 1024 bf16, with twice the
  // chunks: joins 13.2 instead of 7.3)
  const int G = TB / p.tpr;
  const int64_t least = cdiv(rows, 16 * G) * p.slabs < 512 ? 8 : 16;
  p.len = (int)std::max<int64_t>(least, cdiv(rows, 2048 * G));
  p.chunks = cdiv(rows, (int64_t)p.len * G);
  size_t at = 0;
  const auto take = [&](size_t n) {
    const size_t was = at;
    at += oc::align256(n);
    return was;
  };
  p.count = take(4);
  p.hist = take(small ? 0 : ((size_t)4 << p.bits) * p.tiles);
  p.a = take((size_t)rows * sizeof(Pair));
  p.b = !small && p.passes > 1 ? take((size_t)rows * sizeof(Pair)) : p.a;
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
  int tpr = 1;
  while (tpr < TB && tpr * 8 < c) tpr *= 2;
  const auto go = [&](auto kernel, int each) {
    oc::launch_main(kernel, dim3((unsigned)std::min(cdiv(rows, each * (TB / tpr)), MOST_BLOCKS)),
                    dim3(TB), s, ids, id_mask(flags), rows, num, (int)c, table, tpr, scale, y);
  };
  // Several rows a group where workgroups are enough, counted with four rows a group for
  // both types.  35472 x 256, just below: bf16 7.1 us with one, 6.7 with four, fp32 11.9
  // with one or two; 17700 x 256: 4.6 and 4.7, 7.7 both; above it, 140000 x 256: bf16 18.4
  // with one, 16.7 with four, fp32 35.6 both.
  const bool many = cdiv(rows, 4 * (TB / tpr)) >= 2048;
  if (dt == OC_BF16)
    many ? go(k_embed<true, 4>, 4) : go(k_embed<true, 1>, 1);
  else
    many ? go(k_embed<false, 2>, 2) : go(k_embed<false, 1>, 1);
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
  Digit d{ids, id_mask(flags), nullptr, (Pair*)(w + p.a), (uint32_t*)(w + p.hist),
          (uint32_t*)(w + p.count), rows, num, p.tiles, 0, p.bits, p.passes};
  if (rows <= SMALL) {
    oc::launch(k_embed_sort_small, dim3(1), dim3(SB), 0, s, d);
    d.in = d.out;
  } else {
    for (int i = 0; i < p.passes; ++i) {
      d.out = (Pair*)(w + (i & 1 ? p.b : p.a));
      d.shift = i * p.bits;
      oc::launch(k_embed_count, dim3((unsigned)p.tiles), dim3(SB), 0, s, d);
      oc::launch(k_embed_scatter, dim3((unsigned)p.tiles), dim3(SB), 0, s, d);
      d.in = d.out;
    }
  }
  a.sorted = d.in;
  a.count = d.count;
  a.part = (float*)(w + p.part);
  a.len = p.len;
  a.chunk = p.len * (TB / p.tpr);
  a.zero_blocks = cdiv(num, TB);
  const int64_t blocks = a.zero_blocks + p.chunks * p.slabs;
  const auto sums = [&](auto kernel) {
    oc::launch_main(kernel, dim3((unsigned)blocks), dim3(TB), s, a, p.tpr, p.slabs);
  };
  if (p.len > MOST_ADDED)
    a.bf16 ? sums(k_embed_sums<true, true>) : sums(k_embed_sums<false, true>);
  else
    a.bf16 ? sums(k_embed_sums<true, false>) : sums(k_embed_sums<false, false>);
  if (p.chunks > 1) {
    // few columns a workgroup, so that a long run's partial sums have many lanes, and no
    // more workgroups than the card holds at once
    const int jt = std::min(p.tpr, 32);
    const int64_t blocks = cdiv(p.chunks, JW), most = std::max<int64_t>(1, 512 / blocks);
    oc::launch(k_embed_join,
               dim3((unsigned)blocks, (unsigned)std::min(cdiv(cdiv(c, 8), jt), most)), dim3(JB), 0,
               s, a, jt);
  }
  OC_LAUNCH_CHECK();
  return OC_OK;
}

}  // extern "C"
