// Which tiles a dense layer's product runs on, and the sum of a split reduction.
#include <algorithm>

#include "dense_tile.h"

namespace {

using oc::Epi;
using oc::cdiv;

constexpr int TB = 256;

// out = the epilogue of the sum of the splits' partial sums, in index order: a
// thread per row and eight columns.
template <bool GLU>
__global__ __launch_bounds__(TB) void k_split_sum(const float* part, int splits, int64_t P, int Q,
                                                  Epi e) {
  const int nc = (e.n + 7) / 8;
  const int64_t i = (int64_t)blockIdx.x * TB + threadIdx.x;
  if (i >= P * nc) return;
  const int64_t p = i / nc;
  const int c = (int)(i - p * nc) * 8;
  const int64_t step = P * Q;
  const float* src = part + p * Q + c;
  float v[8] = {}, u[8] = {};
  for (int s = 0; s < splits; ++s, src += step) {
    float w[8];
    oc::load8n(src, false, 0, e.n - c, w);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += w[k];
    if (GLU) {
      oc::load8n(src, false, e.n, e.n - c, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) u[k] += w[k];
    }
  }
  if (GLU) oc::epi8_glu(e, p, c, v, u);
  else oc::epi8(e, p, c, v);
}

struct Plan {
  int shape;
  int ntm, ntn, splits;
  int64_t per;
};

// Expected time of each shape and number of splits; the least is taken.  A step
// of BK terms takes a workgroup `step` microseconds with `fit` of them on a CU,
// a workgroup 3 more to start and finish; splits write and read their partial
// sums at 4 TB/s and take another launch of 3.
Plan plan(oc_dtype dt, int64_t P, int64_t Q, int64_t R, bool glu) {
  struct Cost {
    double step;
    int fit;
  };
  static const Cost cost[2][oc::TILE_SHAPES] = {{{2.4, 1}, {1.5, 1}, {1.4, 3}},
                                                {{1.6, 1}, {0.9, 2}, {0.7, 4}}};
  const int cus = oc::cu_count();
  const int64_t n = glu ? Q / 2 : Q;
  Plan best{};
  double least = 1e300;
  for (int k = 0; k < oc::TILE_SHAPES; ++k) {
    const oc::TileInfo i = dt == OC_BF16 ? oc::tile_info<uint16_t>(k) : oc::tile_info<float>(k);
    const Cost& c = cost[dt == OC_BF16][k];
    const int64_t ntm = cdiv(P, i.bm), ntn = cdiv(n, glu ? i.bn / 2 : i.bn);
    const int64_t steps = cdiv(R, i.bk), slots = (int64_t)cus * c.fit;
    int64_t last = 0;
    for (int64_t want = 1; want <= 256 && want <= steps; want = want < 8 ? want + 1 : want * 5 / 4) {
      const int64_t each = cdiv(steps, want), splits = cdiv(steps, each);
      if (splits == last || (splits > 1 && ntm * ntn * splits > 4 * slots)) continue;
      last = splits;
      const double rounds = (double)cdiv(ntm * ntn * splits, slots);
      double us = rounds * (each * c.step + 3.0);
      if (splits > 1) us += 3.0 + (double)splits * P * Q * 8 / 4e6;
      if (us < least) {
        least = us;
        best = Plan{k, (int)ntm, (int)ntn, (int)splits, each * i.bk};
      }
    }
  }
  return best;
}

// Rows that are whole 16-byte vectors at 16-byte addresses.
bool vectors(const void* p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0; }

}  // namespace

namespace oc {

size_t gemm_ws(oc_dtype dt, int64_t P, int64_t Q, int64_t R, bool, bool, bool glu) {
  const Plan p = plan(dt, P, Q, R, glu);
  return p.splits > 1 ? align256((size_t)p.splits * P * Q * 4) : 0;
}

void gemm(const Gemm& g, void* ws, bool main, hipStream_t s) {
  const Plan p = plan(g.dt, g.P, g.Q, g.R, g.epi.glu);
  const TileArgs t{g.a, g.b, g.P, g.R, g.Q, p.ntm, p.ntn, p.splits, p.per,
                   p.splits > 1 ? (float*)ws : nullptr, g.epi};
  if (g.dt == OC_F32) {
    tile_f32(p.shape, g.a_rs, g.b_rs, main, t, s);
  } else {
    const bool direct = vectors(g.a, g.a_rs ? g.P : g.R) && vectors(g.b, g.b_rs ? g.Q : g.R) &&
                        (!g.epi.glu || g.epi.n % 8 == 0);
    tile_bf16(p.shape, g.a_rs, g.b_rs, direct, main, t, s);
  }
  if (p.splits == 1) return;
  const dim3 grid((unsigned)cdiv(g.P * cdiv(g.epi.n, 8), TB));
  if (g.epi.glu)
    launch(k_split_sum<true>, grid, dim3(TB), 0, s, (const float*)ws, p.splits, g.P, g.Q, g.epi);
  else
    launch(k_split_sum<false>, grid, dim3(TB), 0, s, (const float*)ws, p.splits, g.P, g.Q, g.epi);
}

}  // namespace oc
