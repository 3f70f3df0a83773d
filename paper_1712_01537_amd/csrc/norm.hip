// Layer norm over the channels of each row (oc_ln_*) and the residual step around it,
// h = res + dropout(x), y = layer norm of h (oc_drop_ln_*).
//
//   mean = sum h / c,  var = sum (h - mean)^2 / c,  invstd = 1 / sqrt(var + eps)
//   z = (h - mean) invstd,  y = z gamma + beta
//   g = dy gamma,  dn = invstd (g - mean(g) - z mean(g z)),  dgamma = sum dy z, dbeta =
//   sum dy over the rows;  dres = dn + dh,  dx = dropout's mask on dres
//
// The mean is formed twice: m from the values (each divided by c before it is added, so
// that the sum does not overflow), then delta = mean of h - m; h - m - delta has no
// rounding of the mean in it, whatever the size of the mean beside the deviations.
// The stored mean is m + delta rounded; the backward forms its delta again (times invstd,
// as its deviations are), as one more sum of the pass it makes anyway.  Squared deviations
// are divided by c before they are added too, in fp32: the variance is in range for
// deviations up to 2^63, whatever c.
#include <algorithm>

#include "norm.h"

namespace {

using oc::cdiv;
using oc::Drop;
using oc::MOST_ADDED;
using oc::Norm;
using oc::NormBwd;

constexpr int TB = 256;
constexpr int64_t MOST_BLOCKS = (int64_t)1 << 22;  // (a launch has fewer than 2^32 threads)

// The sums of K values over the block's threads, in every thread: lanes first, then the
// waves in order.  Two calls in a row need different halves of `red`.
template <int K>
__device__ __forceinline__ void block_sums(float (&v)[K], float (*red)[K]) {
#pragma unroll
  for (int k = 0; k < K; ++k)
    for (int m = 32; m > 0; m >>= 1) v[k] += __shfl_xor(v[k], m);
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) red[threadIdx.x >> 6][k] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] = red[0][k];
    for (int w = 1; w < (int)(blockDim.x >> 6); ++w) v[k] += red[w][k];
  }
}

// --- rows of any length ----------------------------------------------------------
// One workgroup a row, which it reads once a pass (from the caches but for the first): for
// rows that fit no workgroup's registers.

// The values 8 i .. 8 i + 7 of a row's h; keep: which of them dropout has kept.
template <typename Args>
__device__ __forceinline__ void load_h(const Args& a, const oc::DropKey& key, int64_t row, int i,
                                       float (&v)[8], bool (&keep)[8]) {
  const int c = i * 8, cnt = a.c - c;
  const int64_t at = row * a.c + c, n = a.rows * a.c;
  oc::load8n(a.x, a.bf16, at, cnt, n, v);
  if (a.drop.on) {
    oc::keep8(a.drop, key, (uint64_t)row * ((a.c + 7) / 8) + i, keep);
    oc::drop8(a.drop, keep, v);
  }
  if (a.res) {
    float r[8];
    oc::load8n(a.res, a.bf16, at, cnt, n, r);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += r[k];
  }
}

__global__ __launch_bounds__(TB) void k_ln_fwd_any(Norm a) {
  __shared__ float red0[TB / 64][1], red1[TB / 64][2];
  const int nv = (a.c + 7) / 8;
  const oc::DropKey key = a.drop.on ? oc::drop_key(a.drop) : oc::DropKey{};
  const float rc = 1.f / (float)a.c;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float v[8];
    bool keep[8];
    float m[1] = {0.f};
    for (int i = threadIdx.x; i < nv; i += TB) {
      load_h(a, key, row, i, v, keep);
#pragma unroll
      for (int k = 0; k < 8; ++k) m[0] = fmaf(v[k], rc, m[0]);
    }
    block_sums(m, red0);
    float s[2] = {0.f, 0.f};
    for (int i = threadIdx.x; i < nv; i += TB) {
      load_h(a, key, row, i, v, keep);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float d = i * 8 + k < a.c ? v[k] - m[0] : 0.f;
        s[0] += d;
        s[1] = fmaf(d * rc, d, s[1]);
      }
    }
    block_sums(s, red1);
    const float delta = s[0] * rc;
    float var = fmaf(-delta, delta, s[1]);
    if (var < 0.f) var = 0.f;  // (NaN stays NaN)
    const float invstd = 1.f / sqrtf(var + a.eps);
    for (int i = threadIdx.x; i < nv; i += TB) {
      load_h(a, key, row, i, v, keep);
      const int c = i * 8, cnt = a.c - c;
      const int64_t at = row * a.c + c;
      if (a.h) oc::store8n(a.h, a.bf16, at, cnt, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float z = ((v[k] - m[0]) - delta) * invstd;
        const bool in = c + k < a.c;
        v[k] = fmaf(z, a.gamma && in ? a.gamma[c + k] : 1.f, a.beta && in ? a.beta[c + k] : 0.f);
      }
      oc::store8n(a.y, a.bf16, at, cnt, v);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = m[0] + delta;
      if (a.invstd) a.invstd[row] = invstd;
    }
  }
}

__global__ __launch_bounds__(TB) void k_ln_bwd_any(NormBwd a) {
  __shared__ float red[TB / 64][3];
  const int64_t n = a.rows * a.c;
  const int nv = (a.c + 7) / 8;
  const oc::DropKey key = a.drop.on ? oc::drop_key(a.drop) : oc::DropKey{};
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    __syncthreads();  // the sums of the row before have been read
    const float m = a.mean[row], r = a.invstd[row], rc = 1.f / (float)a.c;
    float d[8], g[8];
    bool keep[8];
    const auto load = [&](int i) {
      const int c = i * 8, cnt = a.c - c;
      load_h(a, key, row, i, d, keep);
      oc::load8n(a.dy, a.bf16, row * a.c + c, cnt, n, g);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        d[k] = k < cnt ? (d[k] - m) * r : 0.f;
        if (a.gamma && k < cnt) g[k] *= a.gamma[c + k];
      }
    };
    float s[3] = {0.f, 0.f, 0.f};
    for (int i = threadIdx.x; i < nv; i += TB) {
      load(i);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        s[0] += g[k];
        s[1] = fmaf(g[k], d[k], s[1]);
        s[2] += d[k];
      }
    }
    block_sums(s, red);
    const float delta = s[2] * rc, gm = s[0] * rc, zm = fmaf(-delta, s[0], s[1]) * rc;
    if (threadIdx.x == 0 && a.delta) a.delta[row] = delta;
    if (!a.dx && !a.dres) continue;
    for (int i = threadIdx.x; i < nv; i += TB) {
      load(i);
      const int c = i * 8, cnt = a.c - c;
      const int64_t at = row * a.c + c;
#pragma unroll
      for (int k = 0; k < 8; ++k) g[k] = r * (g[k] - gm - (d[k] - delta) * zm);
      if (a.dh) {
        oc::load8n(a.dh, a.bf16, at, cnt, n, d);
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] += d[k];
      }
      if (a.dres) oc::store8n(a.dres, a.bf16, at, cnt, g);
      if (a.dx) {
        if (a.drop.on) oc::drop8(a.drop, keep, g);
        oc::store8n(a.dx, a.bf16, at, cnt, g);
      }
    }
  }
}

// Sums over the rows: a thread has eight columns and every rl-th row of the block's
// range, at most MOST_ADDED of them, in fp32; the row lanes are added in double, and
// k_ln_colsum adds the blocks' part[b][2][c] (dgamma, dbeta), in a fixed order.
struct ColShape {
  int ct, rl, kb;  // column threads, row lanes, column blocks
  int64_t nb;      // row blocks
};
ColShape col_shape(int64_t rows, int c) {
  ColShape d;
  const int chunks = (int)cdiv(c, 8);
  d.ct = 1;
  while (d.ct < chunks && d.ct < 32) d.ct *= 2;
  d.rl = TB / d.ct;
  d.kb = (int)cdiv(chunks, d.ct);
  const int64_t most = std::max<int64_t>(64, 2048 / d.kb);
  d.nb = std::max(std::min<int64_t>(most, cdiv(rows, 4 * d.rl)), cdiv(rows, MOST_ADDED * d.rl));
  return d;
}
__global__ __launch_bounds__(TB) void k_ln_cols_any(NormBwd a, int ct, float* part) {
  __shared__ float red[2][8][TB];
  const int tid = threadIdx.x, tc = tid % ct, tr = tid / ct, rl = TB / ct;
  const int64_t nb = gridDim.x, b = blockIdx.x;
  const int64_t r0 = a.rows * b / nb, r1 = a.rows * (b + 1) / nb, n = a.rows * a.c;
  const int c = (blockIdx.y * ct + tc) * 8, cnt = a.c - c;
  const oc::DropKey key = a.drop.on ? oc::drop_key(a.drop) : oc::DropKey{};
  float sg[8] = {}, sb[8] = {};
  if (cnt > 0)
    for (int64_t r = r0 + tr; r < r1; r += rl) {
      float x[8], g[8];
      bool keep[8];
      load_h(a, key, r, c / 8, x, keep);
      oc::load8n(a.dy, a.bf16, r * a.c + c, cnt, n, g);
      const float m = a.mean[r], is = a.invstd[r], de = a.delta[r];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        sg[k] = fmaf(g[k], (x[k] - m) * is - de, sg[k]);
        sb[k] += g[k];
      }
    }
#pragma unroll
  for (int k = 0; k < 8; ++k) red[0][k][tid] = sg[k], red[1][k][tid] = sb[k];
  __syncthreads();
  for (int i = tid; i < ct * 16; i += TB) {
    const int h = i >= ct * 8, j = h ? i - ct * 8 : i, cc = blockIdx.y * ct * 8 + j;
    if (cc >= a.c) continue;
    double s = 0.0;
    for (int r = 0; r < rl; ++r) s += (double)red[h][j & 7][r * ct + (j >> 3)];
    part[(b * 2 + h) * a.c + cc] = (float)s;
  }
}

// dgamma[c], dbeta[c] = the sums of part[b][0 / 1][c] over the nb blocks, in double: 32
// lanes a column take every 32nd block, then a fixed tree through LDS.  A workgroup has 32
// columns, 128 bytes of a row of part (with 16, 512 blocks of 4096 channels took 14 us
// instead of 9).
constexpr int CB = 1024, CC = 32;
__global__ __launch_bounds__(CB) void k_ln_colsum(const float* part, int64_t nb, int c,
                                                  float* dgamma, float* dbeta) {
  __shared__ double red[CB];
  const int cl = threadIdx.x % CC, l = threadIdx.x / CC;
  const int64_t j = (int64_t)blockIdx.x * CC + cl, n = 2 * (int64_t)c;
  double a = 0.0;
  if (j < n) {
#pragma unroll 16
    for (int64_t b = l; b < nb; b += CB / CC) a += (double)part[b * n + j];
  }
  red[threadIdx.x] = a;
  __syncthreads();
  for (int h = CB / 2; h >= CC; h >>= 1) {
    if ((int)threadIdx.x < h) red[threadIdx.x] += red[threadIdx.x + h];
    __syncthreads();
  }
  if (l != 0 || j >= n) return;
  if (j < c) {
    if (dgamma) dgamma[j] = (float)red[cl];
  } else if (dbeta) {
    dbeta[j - c] = (float)red[cl];
  }
}

// --- the calls ---------------------------------------------------------------------

struct BwdWs {
  int64_t blocks;
  size_t delta, total;
};
BwdWs bwd_ws(int64_t rows, int c) {
  BwdWs w{};
  const bool rows_fit = c <= oc::NORM_ROWS_MOST;
  w.blocks = rows_fit ? oc::norm_rows_blocks(rows, c) : col_shape(rows, c).nb;
  w.delta = oc::align256((size_t)w.blocks * 2 * c * sizeof(float));
  w.total = w.delta + (rows_fit ? 0 : oc::align256((size_t)rows * sizeof(float)));
  return w;
}

void fwd(const Norm& a, hipStream_t s) {
  if (a.c <= oc::NORM_ROWS_MOST)
    oc::norm_rows_fwd(a, s);
  else
    oc::launch_main(k_ln_fwd_any, dim3((unsigned)std::min(a.rows, MOST_BLOCKS)), dim3(TB), s, a);
}

void bwd(NormBwd a, float* dgamma, float* dbeta, void* ws, hipStream_t s) {
  const BwdWs w = bwd_ws(a.rows, a.c);
  const bool cols = dgamma || dbeta;
  float* part = cols ? (float*)ws : nullptr;
  if (a.rows > 0 && a.c <= oc::NORM_ROWS_MOST) {
    oc::norm_rows_bwd(a, part, s);
  } else if (a.rows > 0) {
    const ColShape d = col_shape(a.rows, a.c);
    a.delta = cols ? (float*)((char*)ws + w.delta) : nullptr;
    oc::launch_main(k_ln_bwd_any, dim3((unsigned)std::min(a.rows, MOST_BLOCKS)), dim3(TB), s, a);
    if (cols)
      oc::launch(k_ln_cols_any, dim3((unsigned)d.nb, (unsigned)d.kb), dim3(TB), 0, s, a, d.ct,
                 part);
  }
  if (cols)
    oc::launch(k_ln_colsum, dim3((unsigned)cdiv(2 * (int64_t)a.c, CC)), dim3(CB), 0, s,
               (const float*)part, a.rows > 0 ? w.blocks : 0, a.c, dgamma, dbeta);
}

}  // namespace

extern "C" {

oc_status oc_ln_fwd(oc_dtype dt, int64_t rows, int32_t c, const void* x, const float* gamma,
                    const float* beta, float eps, void* y, float* mean, float* invstd,
                    hipStream_t s) {
  const char* who = "oc_ln_fwd";
  OC_TRY(oc::check_rows(who, dt, rows, c));
  if (!(eps > 0.f)) return oc::fail(OC_ERR_ARG, "%s: eps must be positive", who);
  if (rows == 0) return OC_OK;
  if (!x || !y) return oc::fail(OC_ERR_ARG, "%s: NULL buffer", who);
  const size_t n = (size_t)rows * c * oc::value_bytes(dt), nc = (size_t)c * 4, nr = rows * 4;
  const oc::Span sp[] = {{"y", y, n, true, "x"},           {"mean", mean, nr, true, nullptr},
                         {"invstd", invstd, nr, true, nullptr}, {"x", x, n, false, nullptr},
                         {"gamma", gamma, nc, false, nullptr},  {"beta", beta, nc, false, nullptr}};
  OC_TRY(oc::check_spans(who, sp));
  fwd(Norm{x, nullptr, nullptr, y, gamma, beta, mean, invstd, rows, c, dt == OC_BF16, eps, Drop{}},
      s);
  OC_LAUNCH_CHECK();
  return OC_OK;
}

oc_status oc_drop_ln_fwd(oc_dtype dt, int64_t rows, int32_t c, const void* x, const void* res,
                         double p, const uint64_t* rng, int32_t site, const float* gamma,
                         const float* beta, float eps, void* h, void* y, float* mean,
                         float* invstd, hipStream_t s) {
  const char* who = "oc_drop_ln_fwd";
  OC_TRY(oc::check_rows(who, dt, rows, c));
  Drop drop;
  OC_TRY(oc::make_drop(who, p, rng, site, &drop));
  if (!(eps > 0.f)) return oc::fail(OC_ERR_ARG, "%s: eps must be positive", who);
  if (rows == 0) return OC_OK;
  if (!x || !h || !y) return oc::fail(OC_ERR_ARG, "%s: NULL buffer", who);
  const size_t n = (size_t)rows * c * oc::value_bytes(dt), nc = (size_t)c * 4, nr = rows * 4;
  const oc::Span sp[] = {{"h", h, n, true, "res"},
                         {"y", y, n, true, "x"},
                         {"mean", mean, nr, true, nullptr},
                         {"invstd", invstd, nr, true, nullptr},
                         {"x", x, n, false, nullptr},
                         {"res", res, n, false, nullptr},
                         {"gamma", gamma, nc, false, nullptr},
                         {"beta", beta, nc, false, nullptr},
                         {"rng", rng, drop.on ? (size_t)16 : 0, false, nullptr}};
  OC_TRY(oc::check_spans(who, sp));
  fwd(Norm{x, res, h, y, gamma, beta, mean, invstd, rows, c, dt == OC_BF16, eps, drop}, s);
  OC_LAUNCH_CHECK();
  return OC_OK;
}

size_t oc_ln_bwd_workspace(int64_t rows, int32_t c) {
  if (rows < 1 || rows >= oc::ROWS_MOST || c < 1 || c > oc::COLS_MOST) return 0;
  return bwd_ws(rows, c).total;
}

oc_status oc_ln_bwd(oc_dtype dt, int64_t rows, int32_t c, const void* x, const void* dy,
                    const float* gamma, const float* mean, const float* invstd, void* dx,
                    float* dgamma, float* dbeta, void* ws, size_t ws_bytes, hipStream_t s) {
  const char* who = "oc_ln_bwd";
  OC_TRY(oc::check_rows(who, dt, rows, c));
  if (rows > 0 && (!x || !dy || !mean || !invstd))
    return oc::fail(OC_ERR_ARG, "%s: NULL buffer", who);
  const size_t need = dgamma || dbeta ? oc_ln_bwd_workspace(rows, c) : 0;
  OC_TRY(oc::check_row_ws(who, ws, ws_bytes, need));
  const size_t n = (size_t)rows * c * oc::value_bytes(dt), nc = (size_t)c * 4, nr = rows * 4;
  const oc::Span sp[] = {{"dx", dx, n, true, nullptr},
                         {"dgamma", dgamma, nc, true, nullptr},
                         {"dbeta", dbeta, nc, true, nullptr},
                         {"the workspace", need ? ws : nullptr, need, true, nullptr},
                         {"x", x, n, false, nullptr},
                         {"dy", dy, n, false, nullptr},
                         {"gamma", gamma, nc, false, nullptr},
                         {"mean", mean, nr, false, nullptr},
                         {"invstd", invstd, nr, false, nullptr}};
  OC_TRY(oc::check_spans(who, sp));
  if ((rows == 0 || !dx) && !dgamma && !dbeta) return OC_OK;
  bwd(NormBwd{x, nullptr, dy, nullptr, nullptr, dx, gamma, mean, invstd, nullptr, rows, c,
              dt == OC_BF16, Drop{}},
      dgamma, dbeta, ws, s);
  OC_LAUNCH_CHECK();
  return OC_OK;
}

oc_status oc_drop_ln_bwd(oc_dtype dt, int64_t rows, int32_t c, const void* x, const void* res,
                         const void* dy, const void* dh, double p, const uint64_t* rng,
                         int32_t site, const float* gamma, const float* mean,
                         const float* invstd, void* dx, void* dres, float* dgamma, float* dbeta,
                         void* ws, size_t ws_bytes, hipStream_t s) {
  const char* who = "oc_drop_ln_bwd";
  OC_TRY(oc::check_rows(who, dt, rows, c));
  Drop drop;
  OC_TRY(oc::make_drop(who, p, rng, site, &drop));
  if (rows > 0 && (!x || !dy || !mean || !invstd))
    return oc::fail(OC_ERR_ARG, "%s: NULL buffer", who);
  const size_t need = dgamma || dbeta ? oc_ln_bwd_workspace(rows, c) : 0;
  OC_TRY(oc::check_row_ws(who, ws, ws_bytes, need));
  const size_t n = (size_t)rows * c * oc::value_bytes(dt), nc = (size_t)c * 4, nr = rows * 4;
  const oc::Span sp[] = {{"dx", dx, n, true, nullptr},
                         {"dres", dres, n, true, nullptr},
                         {"dgamma", dgamma, nc, true, nullptr},
                         {"dbeta", dbeta, nc, true, nullptr},
                         {"the workspace", need ? ws : nullptr, need, true, nullptr},
                         {"x", x, n, false, nullptr},
                         {"res", res, n, false, nullptr},
                         {"dy", dy, n, false, nullptr},
                         {"dh", dh, n, false, nullptr},
                         {"gamma", gamma, nc, false, nullptr},
                         {"mean", mean, nr, false, nullptr},
                         {"invstd", invstd, nr, false, nullptr},
                         {"rng", rng, drop.on ? (size_t)16 : 0, false, nullptr}};
  OC_TRY(oc::check_spans(who, sp));
  if ((rows == 0 || (!dx && !dres)) && !dgamma && !dbeta) return OC_OK;
  bwd(NormBwd{x, res, dy, dh, dx, dres, gamma, mean, invstd, nullptr, rows, c, dt == OC_BF16, drop},
      dgamma, dbeta, ws, s);
  OC_LAUNCH_CHECK();
  return OC_OK;
}

}  // extern "C"
