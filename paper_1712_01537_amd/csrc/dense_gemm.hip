// Which tiles a dense layer's product runs on, and the sum of a split reduction.
#include <algorithm>
#include <cmath>

#include "dense_tile.h"

namespace {

using oc::Epi;
using oc::cdiv;

constexpr int TB = 256;

// out = the epilogue of the sums of the shared tiles' partial sums, the workgroups'
// in order.  A thread has eight columns of a row (gated: and the eight of the other
// half) and every `lanes`-th partial sum; the lanes' sums are added in order through
// LDS: the same order whatever runs beside it.  lanes grows with their number so that
// a few outputs of many are not one long chain of loads (32 x 128 outputs of 230: 80
// us with one).
template <bool GLU>
__global__ __launch_bounds__(TB) void k_part_sum(oc::TileArgs t, int bm, int bn, int lanes) {
  __shared__ float red[GLU ? 2 : 1][8][TB];
  const Epi& e = t.epi;
  const int per = TB / lanes, tid = threadIdx.x, l = tid / per;
  const int cols = GLU ? bn / 2 : bn, nc = cols / 8;  // a tile's output columns
  const int i = blockIdx.x * per + tid % per;
  const int row = i / nc, oc = i % nc * 8;
  const int64_t nth = blockIdx.y / t.members, member = blockIdx.y - nth * t.members;
  const int64_t first = nth * t.steps / t.share, last = ((nth + 1) * t.steps - 1) / t.share;
  if (first == last) return;  // one workgroup's, done
  const oc::TilePos pos = oc::tile_pos(t.ntm, t.ntn, t.whole + blockIdx.y);
  const int64_t p = (int64_t)pos.m * bm + row;
  const int c = pos.n * cols + oc;
  const bool live = row < bm && p < t.P && c < e.n;
  const float* src = t.part + (((first + l + nth) * t.members + member) * bm + row) * bn +
                     (GLU ? oc / 32 * 64 + oc % 32 : oc);
  float v[1][8] = {}, u[1][8] = {};
  if (live) {
#pragma unroll 4
    for (int64_t w = first + l; w <= last; w += lanes, src += (int64_t)lanes * t.members * bm * bn) {
      float x[8];
      oc::load8(src, false, 0, x);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[0][k] += x[k];
      if (GLU) {
        oc::load8(src, false, 32, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) u[0][k] += x[k];
      }
    }
  }
  if (lanes > 1) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      red[0][k][tid] = v[0][k];
      if (GLU) red[GLU][k][tid] = u[0][k];
    }
    __syncthreads();
    if (l > 0) return;
    for (int j = 1; j < lanes; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[0][k] += red[0][k][tid + j * per];
        if (GLU) u[0][k] += red[GLU][k][tid + j * per];
      }
  }
  if (!live) return;
  float b0[8] = {}, b1[8] = {};
  if (e.bias) {
    oc::load8n(e.bias, false, c, e.n - c, GLU ? 2 * e.n : e.n, b0);
    if (GLU) oc::load8n(e.bias, false, e.n + c, e.n - c, 2 * e.n, b1);
  }
  const int64_t m[1] = {p};
  oc::epilogue<1, GLU>(e, m, t.P, c, b0, b1, v, u);
}

struct Plan {
  int shape;
  int ntm, ntn, whole, members, run, classes;
  int64_t steps, share;
  double us;  // expected
  bool sums() const { return share < steps; }
  size_t ws(oc_dtype dt) const {  // bytes of partial sums
    if (!sums()) return 0;
    const oc::TileInfo i = dt == OC_BF16 ? oc::tile_info<uint16_t>(shape)
                                         : oc::tile_info<float>(shape);
    return oc::align256((size_t)(classes + run - 1) * members * i.bm * i.bn * 4);
  }
};

// What make() returns for these sizes on this device: the plans of a call's products are
// asked for by its workspace and by its launches, and took the host 6 us a backward in
// all (bf16 2048 x 256 -> 256: 22 us a call, its kernels 15).  Every thread remembers the
// last ones.
struct Asked {
  int64_t kind, P, Q, R;
  bool operator==(const Asked& o) const {
    return kind == o.kind && P == o.P && Q == o.Q && R == o.R;
  }
};
template <typename V, typename F>
V remembered(oc_dtype dt, int flags, int64_t P, int64_t Q, int64_t R, F&& make) {
  constexpr int N = 64;
  static thread_local Asked asked[N];
  static thread_local V value[N];
  const Asked a{((int64_t)oc::cu_count() << 8 | flags << 2 | (int)dt) + 1, P, Q, R};
  const uint64_t h = (uint64_t)(a.kind + P * 31 + Q * 1009 + R * 30011) * 0x9e3779b97f4a7c15ull;
  const int at = (int)(h >> 58);
  if (!(asked[at] == a)) {
    value[at] = make();
    asked[at] = a;
  }
  return value[at];
}

// Expected time of each shape, and of each way to deal out the tiles that do not fill
// the card; the least is taken.  Measured, in microseconds: a step of BK terms of a
// workgroup alone on its CU (step) and with all that fit there (full), and what a
// workgroup takes to start and finish (ends).  (As many workgroups as fit, all three
// layouts within 5%: bf16 256x256 1430 TFLOP/s, 256x128 1190, 128x128 1180, 64x64 715;
// fp32 256x128 250, 128x64 168, 128x128 202, 64x64 140.)  Partial sums are written and
// read at 4 TB/s and take another launch of 4 us.
// There is no term for what the epilogue writes and reads, so the expectation holds where
// the reduction is long (35472 x 512 -> 1024 fp32, dx and dw: 199 and 181 us, measured 202
// and 187; 65536 x 1024 -> 4096 bf16: 416 and 430, measured 436 and 440) and is too short
// where the epilogue moves much (the forwards of these 216 and 512, measured 281 and 557;
// 35472 x 256 -> 1024 bf16 GELU with its fp32 values kept 41, measured 74; the gated
// 32768 x 1024 -> 2 x 2816 352, measured 458).  There shapes that differ by less than that
// are in an order of no meaning.
struct Cost {
  double step, full;
  int fit;
  double ends;
};
const Cost kCost[2][oc::TILE_SHAPES] = {
    {{1.75, 2.16, 1, 9.}, {1.02, 1.6, 2, 5.5}, {1.18, 1.33, 1, 6.}, {0.74, 1.45, 3, 4.}},
    {{1.22, 1.5, 1, 8.}, {0.6, 0.9, 2, 7.}, {0.64, 0.91, 2, 4.5}, {0.47, 0.74, 4, 2.5}}};
// A step where wgs workgroups run at a time.
double step_of(const Cost& c, int64_t cus, int64_t wgs) {
  const int64_t calm = c.fit > 1 ? cus : cus / 4;  // workgroups that run as if alone
  const double crowd =
      wgs > calm ? std::min(1.0, (double)(wgs - calm) / (double)(cus * c.fit - calm)) : 0.0;
  return c.step + (c.full - c.step) * crowd;
}
double sums_us(int64_t slots, const oc::TileInfo& i) {
  return 4.0 + (double)slots * i.bm * i.bn * 8 / 4e6;
}

// direct: bf16 operands that go straight to LDS; the larger tiles take only those.
// apart: every tile has a workgroup (for dz, whose epilogue is the tile kernel's alone).
Plan make_plan(oc_dtype dt, bool direct, int64_t P, int64_t Q, int64_t R, bool glu, bool apart) {
  const int64_t cus = oc::cu_count(), n = glu ? Q / 2 : Q;
  Plan best{};
  double least = 1e300;
  for (int k = dt == OC_BF16 && !direct ? oc::TILE_SMALL : oc::TILE_LARGE; k < oc::TILE_SHAPES;
       ++k) {
    const oc::TileInfo i = dt == OC_BF16 ? oc::tile_info<uint16_t>(k) : oc::tile_info<float>(k);
    const Cost& c = kCost[dt == OC_BF16][k];
    const int64_t ntm = cdiv(P, i.bm), ntn = cdiv(n, glu ? i.bn / 2 : i.bn), tiles = ntm * ntn;
    const int64_t steps = cdiv(R, i.bk), slots = cus * c.fit;
    const int64_t whole = tiles / slots * slots, rest = tiles - whole;
    const double rounds = (double)(whole / slots) * (steps * c.full + c.ends);
    auto offer = [&](int64_t run, int64_t share) {
      const int64_t members = cdiv(rest, run), classes = cdiv(run * steps, share);
      const int64_t wgs = members * classes;
      double us = rounds;
      if (rest > 0) {
        us += share * (whole > 0 ? c.full : step_of(c, cus, wgs)) + c.ends;
      }
      if (share < steps)
        us += (run > 1 ? c.ends : 0.0) + sums_us((classes + run - 1) * members, i);
      if (us < least) {
        least = us;
        best = Plan{k, (int)ntm, (int)ntn, (int)whole, (int)members, (int)run, (int)classes,
                    steps, share, us};
      }
    };
    offer(1, steps);
    for (int64_t run = 1; run <= 8 && run <= rest && !apart; ++run) {
      const int64_t members = cdiv(rest, run);
      for (int64_t classes = slots / members; classes > run; classes = classes * 3 / 4) {
        const int64_t share = cdiv(run * steps, classes);
        if (share < steps) offer(run, share);
      }
    }
  }
  return best;
}

Plan plan(oc_dtype dt, bool direct, int64_t P, int64_t Q, int64_t R, bool glu,
          bool apart = false) {
  return remembered<Plan>(dt, direct | glu << 1 | apart << 2, P, Q, R,
                          [&] { return make_plan(dt, direct, P, Q, R, glu, apart); });
}

// Both products of a backward in one launch, on tiles of one shape, with the
// reductions of either dealt out to workgroups of about the time that the whole takes
// on a full card: or two launches, unless that is expected to take less by 5% (what the
// expectations are worth: at 3%, fp32 8383 x 513 -> 1027, one launch took 177 us, two
// 158).  One and two, both products: fp32 8384 x 128 -> 682 41 us, 59; 256 x 512 -> 512
// 17, 22; 139800 x 32 -> 128 59, 66; bf16 5000 x 2048 -> 2048 94, 115; 8384 x 128 -> 688
// 19, 24; 1000 x 512 -> 512 10, 15.  From a few rounds of tiles on there is no difference
// (bf16 65536 x 1024 -> 4096).
struct Plan2 {
  Plan dx, dw;
  bool one, swapped;  // swapped: the input gradient's workgroups first
  size_t ws(oc_dtype dt) const {
    return one ? dx.ws(dt) + dw.ws(dt) : std::max(dx.ws(dt), dw.ws(dt));
  }
};
// Time of n1 workgroups of t1 each and then n2 of t2, `slots` at a time.
double queue_us(int64_t slots, int64_t n1, double t1, int64_t n2, double t2) {
  const int64_t rounds = n1 / slots, late = n1 % slots;
  int64_t m = n2 / slots;
  const auto done = [&](int64_t k) {
    return (slots - late) * k +
           (k * t2 > t1 ? late * (int64_t)((k * t2 - t1) / t2) : 0);
  };
  while (done(m) < n2) ++m;
  return std::max(rounds * t1 + m * t2, (rounds + (late > 0)) * t1);
}
Plan2 make_plan2(oc_dtype dt, bool direct, int64_t rows, int64_t cin, int64_t nz) {
  Plan2 best{plan(dt, direct, rows, cin, nz, false), plan(dt, direct, cin, nz, rows, false), false,
             false};
  double least = 0.95 * (best.dx.us + best.dw.us + 2.0);  // (another launch)
  const int64_t cus = oc::cu_count();
  for (int k = dt == OC_BF16 && !direct ? oc::TILE_SMALL : oc::TILE_LARGE; k < oc::TILE_SHAPES;
       ++k) {
    // (bf16 256 x 128 tiles were not the least for any of 3000 sizes of 33 to 140000 rows)
    if (dt == OC_BF16 && k == oc::TILE_TWO) continue;
    const oc::TileInfo i = dt == OC_BF16 ? oc::tile_info<uint16_t>(k) : oc::tile_info<float>(k);
    const Cost& c = kCost[dt == OC_BF16][k];
    const int64_t slots = cus * c.fit;
    const auto whole = [&](int64_t P, int64_t Q, int64_t R) {
      const int64_t ntm = cdiv(P, i.bm), ntn = cdiv(Q, i.bn), steps = cdiv(R, i.bk);
      return Plan{k, (int)ntm, (int)ntn, (int)(ntm * ntn), 1, 1, 0, steps, steps, 0.};
    };
    const Plan x = whole(rows, cin, nz), w = whole(cin, nz, rows);
    if ((int64_t)x.whole + w.whole > 1 << 20) continue;
    const double even = (double)(x.whole * x.steps + w.whole * w.steps) / (double)slots;
    // each tile's steps dealt out to about n workgroups
    const auto dealt = [&](Plan p, int64_t n) {
      n = std::min(n, p.steps);
      if (n <= 1 || p.whole * n > 2 * slots) return p;
      p.share = cdiv(p.steps, n);
      p.classes = (int)cdiv(p.steps, p.share);
      if (p.classes == 1) return p.classes = 0, p;
      p.members = p.whole;
      p.whole = 0;
      return p;
    };
    const auto count = [](const Plan& p) { return p.whole + (int64_t)p.classes * p.members; };
    const int64_t nx = (int64_t)std::ceil(x.steps / even), nw = (int64_t)std::ceil(w.steps / even);
    for (int64_t fx : {(int64_t)1, nx, 2 * nx})
      for (int64_t fw : {(int64_t)1, nw, nw + cdiv(nw, 2), 2 * nw}) {
        Plan2 p{dealt(x, fx), dealt(w, fw), true, false};
        const int64_t n = count(p.dx), m = count(p.dw);
        const double step = step_of(c, cus, n + m);
        const double tx = p.dx.share * step + c.ends, tw = p.dw.share * step + c.ends;
        if (std::max(tx, tw) >= least) continue;
        p.swapped = tx > tw;
        double us = p.swapped ? queue_us(slots, n, tx, m, tw) : queue_us(slots, m, tw, n, tx);
        for (const Plan* q : {&p.dx, &p.dw})
          if (q->sums()) us += sums_us(count(*q), i);
        if (us < least) least = us, best = p;
      }
  }
  return best;
}

Plan2 plan2(oc_dtype dt, bool direct, int64_t rows, int64_t cin, int64_t nz) {
  return remembered<Plan2>(dt, direct, rows, cin, nz,
                           [&] { return make_plan2(dt, direct, rows, cin, nz); });
}

// bf16 rows that are whole 16-byte vectors at 16-byte addresses.
bool vectors(const void* p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0; }

}  // namespace

namespace oc {

size_t gemm_ws(oc_dtype dt, int64_t P, int64_t Q, int64_t R, bool glu) {
  // for whichever plan the operands' alignment asks for
  const size_t a = plan(dt, false, P, Q, R, glu).ws(dt);
  const size_t b = dt == OC_BF16 ? plan(dt, true, P, Q, R, glu).ws(dt) : 0;
  return std::max(a, b);
}

bool gemm_direct(oc_dtype dt, const void* a, int64_t lda, const void* b, int64_t ldb, bool glu,
                 int64_t half) {
  return dt == OC_BF16 && vectors(a, lda) && vectors(b, ldb) && (!glu || half % 8 == 0);
}

int64_t gemm_dz_tiles(oc_dtype dt, bool direct, int64_t P, int64_t Q, int64_t R, bool glu) {
  return plan(dt, direct, P, Q, R, glu, true).ntm;
}

namespace {

TileArgs tile_args(const Gemm& g, const Plan& p, void* ws) {
  return TileArgs{g.a,    g.b,       g.P,   g.R,       g.Q,     g.lda,   g.ldb,      g.half, p.ntm,
                  p.ntn,  p.whole,   p.members, p.run, p.classes, p.steps, p.share, (float*)ws,
                  g.epi};
}
void run(const Gemm& g, const Plan& p, bool direct, void* ws, bool main, hipStream_t s) {
  const TileArgs t = tile_args(g, p, ws);
  if (g.dt == OC_F32) tile_f32(p.shape, g.a_rs, g.b_rs, main, t, s);
  else tile_bf16(p.shape, g.a_rs, g.b_rs, direct, main, t, s);
}
void add_sums(const Gemm& g, const Plan& p, void* ws, hipStream_t s) {
  if (!p.sums()) return;
  const TileArgs t = tile_args(g, p, ws);
  const TileInfo i = g.dt == OC_BF16 ? tile_info<uint16_t>(p.shape) : tile_info<float>(p.shape);
  const int64_t each = cdiv(p.steps, p.share);  // partial sums of a tile, about
  int lanes = 1;
  while (lanes < 64 && lanes * 4 < each) lanes *= 2;
  const int per = TB / lanes, vecs = i.bm * (g.epi.glu ? i.bn / 2 : i.bn) / 8;
  const dim3 grid((unsigned)cdiv(vecs, per), (unsigned)(p.ntm * p.ntn - p.whole));
  if (g.epi.glu) launch(k_part_sum<true>, grid, dim3(TB), 0, s, t, i.bm, i.bn, lanes);
  else launch(k_part_sum<false>, grid, dim3(TB), 0, s, t, i.bm, i.bn, lanes);
}

}  // namespace

void gemm(const Gemm& g, void* ws, bool main, hipStream_t s) {
  const bool direct = gemm_direct(g.dt, g.a, g.lda, g.b, g.ldb, g.epi.glu, g.half);
  const Plan p = plan(g.dt, direct, g.P, g.Q, g.R, g.epi.glu, g.epi.dy != nullptr);
  run(g, p, direct, ws, main, s);
  add_sums(g, p, ws, s);
}

size_t gemm2_ws(oc_dtype dt, int64_t rows, int64_t cin, int64_t nz) {
  const size_t a = plan2(dt, false, rows, cin, nz).ws(dt);
  const size_t b = dt == OC_BF16 ? plan2(dt, true, rows, cin, nz).ws(dt) : 0;
  return std::max(a, b);
}

void gemm2(const Gemm& dx, const Gemm& dw, void* ws, hipStream_t s) {
  const bool direct = gemm_direct(dx.dt, dx.a, dx.lda, dx.b, dx.ldb, false, 0);
  const bool same = direct == gemm_direct(dw.dt, dw.a, dw.lda, dw.b, dw.ldb, false, 0);
  if (!same) {
    gemm(dx, ws, true, s);
    gemm(dw, ws, false, s);
    return;
  }
  const Plan2 p = plan2(dx.dt, direct, dx.P, dx.Q, dx.R);
  if (!p.one) {
    run(dx, p.dx, direct, ws, true, s);
    add_sums(dx, p.dx, ws, s);
    run(dw, p.dw, direct, ws, false, s);
    add_sums(dw, p.dw, ws, s);
    return;
  }
  char* const behind = (char*)ws + p.dx.ws(dx.dt);
  const TileArgs x = tile_args(dx, p.dx, ws), w = tile_args(dw, p.dw, behind);
  if (dx.dt == OC_F32) tiles2_f32(p.dx.shape, x, w, p.swapped, s);
  else tiles2_bf16(p.dx.shape, direct, x, w, p.swapped, s);
  add_sums(dx, p.dx, ws, s);
  add_sums(dw, p.dw, behind, s);
}

}  // namespace oc
