// Which tiles a dense layer's product runs on, and the sum of a split reduction.
#include <algorithm>

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
  bool sums() const { return share < steps; }
  size_t ws(oc_dtype dt) const {  // bytes of partial sums
    if (!sums()) return 0;
    const oc::TileInfo i = dt == OC_BF16 ? oc::tile_info<uint16_t>(shape)
                                         : oc::tile_info<float>(shape);
    return oc::align256((size_t)(classes + run - 1) * members * i.bm * i.bn * 4);
  }
};

// Expected time of each shape, and of each way to deal out the tiles that do not fill
// the card; the least is taken.  Measured, in microseconds: a step of BK terms of a
// workgroup alone on its CU and with all that fit there, and what a workgroup takes
// to start and finish.  (As many workgroups as fit, all three layouts within 5%: bf16
// 256x256 1430 TFLOP/s, 256x128 1190, 128x128 1180, 64x64 715; fp32 256x128 250,
// 128x64 168, 128x128 202, 64x64 140.)  Partial sums are written and read at 4 TB/s
// and take another launch of 4 us.
// direct: bf16 operands that go straight to LDS; the larger tiles take only those.
// apart: every tile has a workgroup (for dz, whose epilogue is the tile kernel's alone).
Plan plan(oc_dtype dt, bool direct, int64_t P, int64_t Q, int64_t R, bool glu,
          bool apart = false) {
  struct Cost {
    double step, full;
    int fit;
    double ends;
  };
  static const Cost cost[2][oc::TILE_SHAPES] = {
      {{1.75, 2.16, 1, 9.}, {1.02, 1.6, 2, 5.5}, {1.18, 1.33, 1, 6.}, {0.74, 1.45, 3, 4.}},
      {{1.22, 1.5, 1, 8.}, {0.6, 0.9, 2, 7.}, {0.64, 0.91, 2, 4.5}, {0.47, 0.74, 4, 2.5}}};
  const int64_t cus = oc::cu_count(), n = glu ? Q / 2 : Q;
  Plan best{};
  double least = 1e300;
  for (int k = dt == OC_BF16 && !direct ? oc::TILE_SMALL : oc::TILE_LARGE; k < oc::TILE_SHAPES;
       ++k) {
    const oc::TileInfo i = dt == OC_BF16 ? oc::tile_info<uint16_t>(k) : oc::tile_info<float>(k);
    const Cost& c = cost[dt == OC_BF16][k];
    const int64_t ntm = cdiv(P, i.bm), ntn = cdiv(n, glu ? i.bn / 2 : i.bn), tiles = ntm * ntn;
    const int64_t steps = cdiv(R, i.bk), slots = cus * c.fit;
    const int64_t whole = tiles / slots * slots, rest = tiles - whole;
    const double rounds = (double)(whole / slots) * (steps * c.full + c.ends);
    auto offer = [&](int64_t run, int64_t share) {
      const int64_t members = cdiv(rest, run), classes = cdiv(run * steps, share);
      const int64_t wgs = members * classes;
      double us = rounds;
      if (rest > 0) {
        const int64_t calm = c.fit > 1 ? cus : cus / 4;  // workgroups that run as if alone
        const double crowd =
            wgs > calm ? std::min(1.0, (double)(wgs - calm) / (double)(slots - calm)) : 0.0;
        us += share * (whole > 0 ? c.full : c.step + (c.full - c.step) * crowd) + c.ends;
      }
      if (share < steps)
        us += (run > 1 ? c.ends : 0.0) + 4.0 +
              (double)(classes + run - 1) * members * i.bm * i.bn * 8 / 4e6;
      if (us < least) {
        least = us;
        best = Plan{k, (int)ntm, (int)ntn, (int)whole, (int)members, (int)run, (int)classes,
                    steps, share};
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

void gemm(const Gemm& g, void* ws, bool main, hipStream_t s) {
  const bool direct = gemm_direct(g.dt, g.a, g.lda, g.b, g.ldb, g.epi.glu, g.half);
  const Plan p = plan(g.dt, direct, g.P, g.Q, g.R, g.epi.glu, g.epi.dy != nullptr);
  const TileArgs t{g.a,     g.b,       g.P,   g.R,       g.Q,     g.lda,   g.ldb,      g.half, p.ntm,
                   p.ntn,   p.whole,   p.members, p.run, p.classes, p.steps, p.share, (float*)ws,
                   g.epi};
  if (g.dt == OC_F32) tile_f32(p.shape, g.a_rs, g.b_rs, main, t, s);
  else tile_bf16(p.shape, g.a_rs, g.b_rs, direct, main, t, s);
  if (!p.sums()) return;
  const TileInfo i = g.dt == OC_BF16 ? tile_info<uint16_t>(p.shape) : tile_info<float>(p.shape);
  const int64_t each = cdiv(p.steps, p.share);  // partial sums of a tile, about
  int lanes = 1;
  while (lanes < 64 && lanes * 4 < each) lanes *= 2;
  const int per = TB / lanes, vecs = i.bm * (g.epi.glu ? i.bn / 2 : i.bn) / 8;
  const dim3 grid((unsigned)cdiv(vecs, per), (unsigned)(p.ntm * p.ntn - p.whole));
  if (g.epi.glu) launch(k_part_sum<true>, grid, dim3(TB), 0, s, t, i.bm, i.bn, lanes);
  else launch(k_part_sum<false>, grid, dim3(TB), 0, s, t, i.bm, i.bn, lanes);
}

}  // namespace oc
