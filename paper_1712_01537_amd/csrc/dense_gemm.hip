// Which tiles a dense layer's product runs on, and the sum of a split reduction.
#include <algorithm>

#include "dense_tile.h"

namespace {

using oc::Epi;
using oc::cdiv;

constexpr int TB = 256;

// out = the epilogue of the sum of the splits' partial sums.  A thread has eight
// columns of a row (gated: and the eight of the other half) and every `lanes`-th
// split; the lanes' sums are added in order through LDS: the same order whatever
// runs beside it.  lanes grows with the splits so that a few outputs of many splits
// are not one long chain of loads (32 x 128 outputs of 230 splits: 80 us with one).
template <bool GLU>
__global__ __launch_bounds__(TB) void k_split_sum(const float* part, int splits, int lanes,
                                                  int64_t P, int Q, Epi e) {
  __shared__ float red[GLU ? 2 : 1][8][TB];
  const int per = TB / lanes, tid = threadIdx.x, l = tid / per;
  const int nc = (e.n + 7) / 8;
  const int64_t i = (int64_t)blockIdx.x * per + tid % per;
  const bool live = i < P * nc;
  const int64_t p = live ? i / nc : 0;
  const int c = live ? (int)(i - p * nc) * 8 : 0, cnt = e.n - c;
  const int64_t step = P * Q;
  const float* src = part + (int64_t)l * step + p * Q + c;
  float v[1][8] = {}, u[1][8] = {};
  if (live) {
#pragma unroll 4
    for (int s = l; s < splits; s += lanes, src += lanes * step) {
      float w[8];
      oc::load8n(src, false, 0, cnt, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[0][k] += w[k];
      if (GLU) {
        oc::load8n(src, false, e.n, cnt, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) u[0][k] += w[k];
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
    oc::load8n(e.bias, false, c, cnt, b0);
    if (GLU) oc::load8n(e.bias, false, e.n + c, cnt, b1);
  }
  const int64_t m[1] = {p};
  oc::epilogue<1, GLU>(e, m, P, c, b0, b1, v, u);
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
// direct: bf16 operands that go straight to LDS; the largest tiles take only those.
Plan plan(oc_dtype dt, bool direct, int64_t P, int64_t Q, int64_t R, bool glu) {
  struct Cost {
    double step;
    int fit;
  };
  static const Cost cost[2][oc::TILE_SHAPES] = {{{2.4, 1}, {1.4, 2}, {1.5, 1}, {1.4, 3}},
                                                {{1.6, 1}, {0.9, 2}, {0.9, 2}, {0.7, 4}}};
  const int cus = oc::cu_count();
  const int64_t n = glu ? Q / 2 : Q;
  Plan best{};
  double least = 1e300;
  for (int k = dt == OC_BF16 && !direct ? oc::TILE_MEDIUM : oc::TILE_LARGE; k < oc::TILE_SHAPES;
       ++k) {
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
  int splits = 1;  // of whichever plan the operands' alignment asks for
  for (int direct = 0; direct < 2; ++direct) {
    const Plan p = plan(dt, direct, P, Q, R, glu);
    if (p.splits > splits) splits = p.splits;
  }
  return splits > 1 ? align256((size_t)splits * P * Q * 4) : 0;
}

void gemm(const Gemm& g, void* ws, bool main, hipStream_t s) {
  const bool direct = g.dt == OC_BF16 && vectors(g.a, g.a_rs ? g.P : g.R) &&
                      vectors(g.b, g.b_rs ? g.Q : g.R) && (!g.epi.glu || g.epi.n % 8 == 0);
  const Plan p = plan(g.dt, direct, g.P, g.Q, g.R, g.epi.glu);
  const TileArgs t{g.a, g.b, g.P, g.R, g.Q, p.ntm, p.ntn, p.splits, p.per,
                   p.splits > 1 ? (float*)ws : nullptr, g.epi};
  if (g.dt == OC_F32) tile_f32(p.shape, g.a_rs, g.b_rs, main, t, s);
  else tile_bf16(p.shape, g.a_rs, g.b_rs, direct, main, t, s);
  if (p.splits == 1) return;
  int lanes = 1;
  while (lanes < 64 && lanes * 4 < p.splits) lanes *= 2;
  const dim3 grid((unsigned)cdiv(g.P * cdiv(g.epi.n, 8), TB / lanes));
  if (g.epi.glu)
    launch(k_split_sum<true>, grid, dim3(TB), 0, s, (const float*)ws, p.splits, lanes, g.P, g.Q,
           g.epi);
  else
    launch(k_split_sum<false>, grid, dim3(TB), 0, s, (const float*)ws, p.splits, lanes, g.P, g.Q,
           g.epi);
}

}  // namespace oc
