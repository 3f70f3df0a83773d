// Dense layers over rows (oc_dense_*, oc_glu_*): argument checks, the
// elementwise part of the backward and the order of the launches.  The
// products are in dense_gemm.hip.
//
// Backward: dz = dy act'(z) (gated: dg = dy u act'(g), du = dy act(g), dz = [dg
// | du]) is written once, in the type of the products' operands, and read by
// both of them: dx = dz w^T and dw = x^T dz.  Forming dz inside the products
// instead would read z (fp32) and dy once per tile column of each.  In bf16
// that rounds dz once (half a step, 2^-8), as the matrix cores' operand has to
// be; z itself is kept in fp32, since a rounded z would move the slope and so
// round the gradients a second time.  dbias is summed from the unrounded dz in
// the same pass.
#include <algorithm>

#include "dense.h"

namespace {

using oc::cdiv;

constexpr int TB = 256;

// --- dz and its column sums -------------------------------------------------
//
// A thread has eight columns and every rl-th row of the block's range; block
// (b, k) has rows M b / nb .. and columns 8 ct k ..  Column sums: per thread
// fp32 over its rows (at most MOST_ADDED, whatever M is: as many blocks as that takes),
// then in double the row lanes in order through LDS into part[b][column] and, by
// k_colsum, the blocks: a fixed order.
// Bound by memory: dy and z read, dz written (65536 x 4096 bf16 ReLU from y 346 us, 4.7
// TB/s; 32768 x 2816 bf16 gated 288 us, 4.5 TB/s).
constexpr int64_t MOST_ADDED = 64;
struct DzShape {
  int ct, rl, kb, nb;  // column threads, row lanes, column blocks, row blocks
};
DzShape dz_shape(int64_t M, int n) {
  DzShape d;
  const int chunks = (int)cdiv(n, 8);
  d.ct = 1;
  while (d.ct < chunks && d.ct < 32) d.ct *= 2;
  d.rl = TB / d.ct;
  d.kb = (int)cdiv(chunks, d.ct);
  const int64_t most = std::max<int64_t>(64, 2048 / d.kb);
  d.nb = (int)std::max(std::min<int64_t>(most, cdiv(M, 4 * d.rl)), cdiv(M, MOST_ADDED * d.rl));
  return d;
}

// glu 0: z, dz [M][n]; 1: z, dz [M][2 n].  dz has rows of ld elements, those past the
// columns zero (bf16 rows padded to whole vectors); NULL: column sums only (dz = dy).
// A ReLU's slope comes from the forward's bits (Z_BITS) or from its output, of dy's type
// (Z_OUT); the others' from z.
enum { Z_F32, Z_OUT, Z_BITS };
template <bool GLU, int ACT, int Z>
__global__ __launch_bounds__(TB) void k_dz(const void* dy, const void* z, bool bf16, int64_t M,
                                           int n, int ct, void* dz, int64_t ld, float* part) {
  __shared__ float red[GLU ? 2 : 1][8][TB];
  constexpr int U = GLU ? 2 : 4;  // rows whose loads are in flight together
  const int tid = threadIdx.x, tc = tid % ct, tr = tid / ct, rl = TB / ct;
  const int nb = gridDim.x, b = blockIdx.x;
  const int64_t r0 = M * b / nb, r1 = M * (b + 1) / nb;
  const int c = (blockIdx.y * ct + tc) * 8, cnt = n - c;
  float s0[8] = {}, s1[8] = {};
  if (cnt > 0)
    for (int64_t m0 = r0 + tr; m0 < r1; m0 += U * rl) {
      float g[U][8], v[U][8], u[U][8];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int64_t m = m0 + i * rl;
        if (m >= r1) continue;
        oc::load8n(dy, bf16, m * n + c, cnt, M * n, g[i]);
        if (GLU) {
          oc::load8n(z, false, m * 2 * n + c, cnt, M * 2 * n, v[i]);
          oc::load8n(z, false, m * 2 * n + n + c, cnt, M * 2 * n, u[i]);
        } else if (Z == Z_BITS) {
          const uint32_t bits = ((const uint8_t*)z)[m * ((n + 7) / 8) + c / 8];
#pragma unroll
          for (int k = 0; k < 8; ++k) v[i][k] = bits >> k & 1 ? 1.f : 0.f;
        } else if (ACT != OC_ACT_NONE) {
          oc::load8n(z, Z == Z_OUT && bf16, m * n + c, cnt, M * n, v[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int64_t m = m0 + i * rl;
        if (m >= r1) continue;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float d = g[i][k];
          if (GLU) {
            g[i][k] = oc::act_grad(ACT, d * u[i][k], v[i][k]);
            u[i][k] = d * oc::act_value(ACT, v[i][k]);
            s1[k] += u[i][k];
          } else if (ACT != OC_ACT_NONE) {
            g[i][k] = oc::act_grad(ACT, d, v[i][k]);
          }
          s0[k] += g[i][k];
        }
        if (GLU) {
          oc::store8n(dz, bf16, m * ld + c, cnt, g[i]);
          oc::store8n(dz, bf16, m * ld + n + c, cnt, u[i]);
          if (cnt <= 8)
            for (int64_t k = 2 * n; k < ld; ++k) oc::store1(dz, bf16, m * ld + k, 0.f);
        } else if (dz) {
          oc::store8n(dz, bf16, m * ld + c, (int)(ld - c), g[i]);
        }
      }
    }
  if (!part) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    red[0][k][tid] = s0[k];
    if (GLU) red[GLU][k][tid] = s1[k];
  }
  __syncthreads();
  const int nz = GLU ? 2 * n : n;
  for (int i = tid; i < ct * 8; i += TB) {  // column i of the block
    const int cc = blockIdx.y * ct * 8 + i;
    if (cc >= n) continue;
    for (int h = 0; h < (GLU ? 2 : 1); ++h) {
      double a = 0.0;
      for (int r = 0; r < rl; ++r) a += (double)red[h][i & 7][r * ct + (i >> 3)];
      part[(int64_t)b * nz + h * n + cc] = (float)a;
    }
  }
}

// out[c] = sum of part[b][c] over the nb blocks, in double: 64 lanes per column
// take every 64th block, then a fixed tree through LDS.
__global__ __launch_bounds__(TB) void k_colsum(const float* part, int nb, int nz, float* out) {
  __shared__ double red[TB];
  const int cl = threadIdx.x & 3, l = threadIdx.x >> 2, c = blockIdx.x * 4 + cl;
  double a = 0.0;
  if (c < nz) {
#pragma unroll 8
    for (int b = l; b < nb; b += 64) a += (double)part[(int64_t)b * nz + c];
  }
  red[threadIdx.x] = a;
  __syncthreads();
  for (int h = TB / 2; h >= 4; h >>= 1) {
    if ((int)threadIdx.x < h) red[threadIdx.x] += red[threadIdx.x + h];
    __syncthreads();
  }
  if (l == 0 && c < nz) out[c] = (float)red[cl];
}

// --- arguments ---------------------------------------------------------------

constexpr int64_t MOST_ROWS = (int64_t)1 << 28;
constexpr int32_t MOST_COLS = 1 << 16;
// A launch has fewer than 2^32 threads: 64x64 tiles of the largest product.
bool too_many_tiles(int64_t rows, int64_t cin, int64_t nz) {
  return cdiv(rows, 64) * cdiv(std::max(cin, nz), 64) >= (int64_t)1 << 24;
}

oc_status check(const char* who, oc_dtype dt, int32_t act, bool glu, int64_t rows, int32_t cin,
                int32_t cout) {
  if (dt != OC_F32 && dt != OC_BF16) return oc::fail(OC_ERR_ARG, "%s: dtype %d", who, (int)dt);
  if (act < OC_ACT_NONE || act > OC_ACT_GELU)
    return oc::fail(OC_ERR_ARG, "%s: activation %d", who, act);
  const int32_t most = glu ? MOST_COLS / 2 : MOST_COLS;
  if (rows < 0 || rows >= MOST_ROWS || cin < 1 || cin > MOST_COLS || cout < 1 || cout > most)
    return oc::fail(OC_ERR_ARG, "%s: %lld rows, %d -> %d channels", who, (long long)rows, cin,
                    cout);
  if (too_many_tiles(rows, cin, glu ? 2 * cout : cout))
    return oc::fail(OC_ERR_UNSUPPORTED, "%s: %lld rows of %d -> %d channels are too many", who,
                    (long long)rows, cin, cout);
  return OC_OK;
}

bool sizes_ok(oc_dtype dt, int64_t rows, int32_t cin, int32_t cout, bool glu) {
  return (dt == OC_F32 || dt == OC_BF16) && rows > 0 && rows < MOST_ROWS && cin >= 1 &&
         cin <= MOST_COLS && cout >= 1 && cout <= (glu ? MOST_COLS / 2 : MOST_COLS) &&
         !too_many_tiles(rows, cin, glu ? 2 * cout : cout);
}

oc_status check_ws(const char* who, const void* ws, size_t have, size_t need) {
  if (need && (!ws || have < need))
    return oc::fail(OC_ERR_ARG, "%s: workspace %zu bytes < %zu", who, ws ? have : 0, need);
  if (need && (uintptr_t)ws % 16)
    return oc::fail(OC_ERR_ARG, "%s: the workspace is not 16-byte aligned", who);
  return OC_OK;
}

// n values of the type set to zero (two bytes a thread: bf16 buffers are not
// aligned to four).
__global__ __launch_bounds__(TB) void k_zero16(uint16_t* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * TB + threadIdx.x; i < n; i += (int64_t)gridDim.x * TB)
    p[i] = 0;
}
void zero(void* p, oc_dtype dt, int64_t n, hipStream_t s) {
  const int64_t halves = dt == OC_F32 ? 2 * n : n;
  oc::launch(k_zero16, dim3((unsigned)std::min<int64_t>(cdiv(halves, TB), 4096)), dim3(TB), 0, s,
             (uint16_t*)p, halves);
}

// --- copies to rows of whole vectors ------------------------------------------

// Two bf16 matrices [rows][cols] copied to rows of ld elements (a multiple of
// eight), zero past the columns; with halves, the columns' second half starts at ld / 2
// (zero between).  A thread writes one vector; grid y picks the matrix.
struct Pad {
  const void* src;
  uint16_t* dst;
  int64_t rows, ld;
  int32_t cols, halves;
};
struct Pads {
  Pad p[2];
};
__global__ __launch_bounds__(TB) void k_pad(Pads a) {
  const Pad p = blockIdx.y ? a.p[1] : a.p[0];
  const int64_t nv = p.ld / 8, total = p.src ? p.rows * nv : 0;
  for (int64_t i = (int64_t)blockIdx.x * TB + threadIdx.x; i < total; i += (int64_t)gridDim.x * TB) {
    const int64_t r = i / nv;
    int c = (int)(i - r * nv) * 8, lim = p.cols, add = 0;
    if (p.halves) {
      lim = p.cols / 2;
      if (c >= p.ld / 2) c -= (int)(p.ld / 2), add = lim;
    }
    float v[8];
    const int cnt = lim - c < 0 ? 0 : lim - c;
    oc::load8n(p.src, true, cnt ? r * p.cols + add + c : 0, cnt, p.rows * p.cols, v);
    oc::store8(p.dst, true, i * 8, v);
  }
}
void pad(const Pads& a, hipStream_t s) {
  int64_t most = 1;
  for (const Pad& p : a.p) most = std::max(most, p.src ? p.rows * p.ld / 8 : 0);
  oc::launch(k_pad, dim3((unsigned)std::min<int64_t>(cdiv(most, TB), 8192), 2), dim3(TB), 0, s, a);
}
size_t pad_bytes(int64_t rows, int64_t ld) { return oc::align256((size_t)rows * ld * 2); }

// --- the two layers -----------------------------------------------------------

// x and w as the forward's product takes them, copied to xp and wp where they are padded.
struct Operands {
  const void *x, *w;
  int64_t lda, ldb;
  int32_t half;
};
Operands operands(oc_dtype dt, int64_t rows, int32_t cin, int32_t cout, bool glu, const void* x,
                  const void* w, void* xp, void* wp, hipStream_t s) {
  const int32_t nz = glu ? 2 * cout : cout;
  Operands f{x, w, cin, nz, cout};
  if (!oc::pads(dt, rows, cin, cout, glu)) return f;
  Pads p{};
  if (cin % 8) {
    f.lda = oc::pad8(cin);
    f.x = xp;
    p.p[0] = Pad{x, (uint16_t*)xp, rows, f.lda, cin, 0};
  }
  if (cout % 8) {
    f.half = (int32_t)oc::pad8(cout);
    f.ldb = glu ? 2 * f.half : f.half;
    f.w = wp;
    p.p[1] = Pad{w, (uint16_t*)wp, cin, f.ldb, nz, glu};
  }
  pad(p, s);
  return f;
}

struct FwdWs {
  size_t x, w, gemm, total;  // offsets, bytes in all
};
FwdWs fwd_ws(oc_dtype dt, int64_t rows, int32_t cin, int32_t cout, bool glu) {
  const int64_t nz = glu ? 2 * cout : cout;
  if (oc::few_rows(dt, rows, cin, cout)) return FwdWs{0, 0, 0, 0};
  const bool pd = oc::pads(dt, rows, cin, cout, glu);
  FwdWs f;
  f.x = 0;
  f.w = pd && cin % 8 ? pad_bytes(rows, oc::pad8(cin)) : 0;
  f.gemm = f.w + (pd && cout % 8 ? pad_bytes(cin, (glu ? 2 : 1) * oc::pad8(cout)) : 0);
  f.total = f.gemm + oc::gemm_ws(dt, rows, nz, cin, glu);
  return f;
}

oc_status fwd(const char* who, bool glu, oc_dtype dt, int32_t act, int64_t rows, int32_t cin,
              int32_t cout, const void* x, const void* w, const float* bias, const void* res,
              void* y, void* pre, void* ws, size_t ws_bytes, hipStream_t s) {
  oc_status st = check(who, dt, act, glu, rows, cin, cout);
  if (st != OC_OK) return st;
  if (rows == 0) return OC_OK;
  if (!x || !w || !y) return oc::fail(OC_ERR_ARG, "%s: NULL buffer", who);
  const FwdWs o = fwd_ws(dt, rows, cin, cout, glu);
  st = check_ws(who, ws, ws_bytes, o.total);
  if (st != OC_OK) return st;
  const int32_t bf16 = dt == OC_BF16, nz = glu ? 2 * cout : cout;
  const oc::Epi epi{act, glu, cout, bf16, act == OC_ACT_RELU && !glu, bias, res, y, pre, nullptr, 0,
                    nullptr};
  if (oc::few_rows(dt, rows, cin, cout)) {
    oc::gemm_rows(dt, (int32_t)rows, cin, nz, x, w, epi, s);
    OC_LAUNCH_CHECK();
    return OC_OK;
  }
  char* base = (char*)ws;
  const Operands f = operands(dt, rows, cin, cout, glu, x, w, base + o.x, base + o.w, s);
  oc::gemm(oc::Gemm{dt, rows, cin, nz, f.x, f.w, f.lda, f.ldb, f.half, false, true, epi},
           base + o.gemm, true, s);
  OC_LAUNCH_CHECK();
  return OC_OK;
}

struct BwdWs {
  size_t dz, part, x, w, gemm, total;  // offsets, bytes in all
};
BwdWs bwd_ws(oc_dtype dt, int32_t act, int64_t rows, int32_t cin, int32_t cout, bool glu) {
  const int64_t nz = glu ? 2 * cout : cout;
  const DzShape d = dz_shape(rows, cout);
  const bool pd = oc::pads(dt, rows, cin, cout, glu);
  BwdWs b;
  b.dz = 0;
  b.part = glu || act != OC_ACT_NONE || (pd && nz % 8)
               ? oc::align256((size_t)rows * (pd ? oc::pad8(nz) : nz) * (dt == OC_BF16 ? 2 : 4)) : 0;
  // (a product formed again leaves a sum for each tile of 64 rows or more)
  b.x = b.part + oc::align256((size_t)std::max<int64_t>(d.nb, cdiv(rows, 64)) * nz * 4);
  b.w = b.x + (pd && cin % 8 ? pad_bytes(rows, oc::pad8(cin)) : 0);
  b.gemm = b.w + (pd && nz % 8 ? pad_bytes(cin, oc::pad8(nz)) : 0);
  const size_t again = pd && cout % 8 ? pad_bytes(cin, (glu ? 2 : 1) * oc::pad8(cout)) : 0;
  b.total = b.gemm + oc::align256(std::max({oc::gemm_ws(dt, rows, cin, nz, false),
                                            oc::gemm_ws(dt, cin, nz, rows, false),
                                            oc::gemm2_ws(dt, rows, cin, nz), again}));
  return b;
}

oc_status bwd(const char* who, bool glu, oc_dtype dt, int32_t act, int64_t rows, int32_t cin,
              int32_t cout, const void* x, const void* w, const float* bias, const void* pre,
              const void* y, const void* dy, void* dx, oc_dtype dw_dt, void* dw, float* dbias,
              void* ws, size_t ws_bytes, hipStream_t s) {
  oc_status st = check(who, dt, act, glu, rows, cin, cout);
  if (st != OC_OK) return st;
  if (dw && dw_dt != OC_F32 && dw_dt != dt)
    return oc::fail(OC_ERR_ARG, "%s: dw of dtype %d", who, (int)dw_dt);
  const int32_t nz = glu ? 2 * cout : cout;
  if (rows == 0) {  // sums over no rows
    if (dw) zero(dw, dw_dt, (int64_t)cin * nz, s);
    if (dbias) zero(dbias, OC_F32, nz, s);
    OC_LAUNCH_CHECK();
    return OC_OK;
  }
  const bool slope = glu || act != OC_ACT_NONE;
  const bool from_y = !glu && act == OC_ACT_RELU && y;
  if (pre && from_y) return oc::fail(OC_ERR_ARG, "%s: both pre and y", who);
  const bool again = slope && !pre && !from_y;  // x w + bias is formed once more
  if (!dy || ((dx || again) && !w) || ((dw || again) && !x))
    return oc::fail(OC_ERR_ARG, "%s: NULL buffer", who);
  if (!dx && !dw && !dbias) return OC_OK;
  const BwdWs o = bwd_ws(dt, act, rows, cin, cout, glu);
  st = check_ws(who, ws, ws_bytes, o.total);
  if (st != OC_OK) return st;
  char* base = (char*)ws;
  const bool bf16 = dt == OC_BF16, pd = oc::pads(dt, rows, cin, cout, glu);
  const bool apart = slope || (pd && nz % 8);  // dz is not dy itself
  const int64_t ldz = pd ? oc::pad8(nz) : nz;
  const void* dz = apart ? base + o.dz : dy;
  float* part = dbias ? (float*)(base + o.part) : nullptr;
  if (again) {
    const Operands f =
        operands(dt, rows, cin, cout, glu, x, w, base + o.x, base + o.gemm, s);
    const int64_t tiles = oc::gemm_dz_tiles(
        dt, oc::gemm_direct(dt, f.x, f.lda, f.w, f.ldb, glu, f.half), rows, nz, cin, glu);
    oc::gemm(oc::Gemm{dt, rows, cin, nz, f.x, f.w, f.lda, f.ldb, f.half, false, true,
                      {act, glu, cout, bf16, 0, bias, nullptr, base + o.dz, nullptr, dy, ldz,
                       part}},
             nullptr, false, s);
    if (dbias)
      oc::launch(k_colsum, dim3((unsigned)cdiv(nz, 4)), dim3(TB), 0, s, (const float*)part,
                 (int)tiles, nz, dbias);
  } else if (apart || dbias) {
    const DzShape d = dz_shape(rows, cout);
    void* out = glu || (apart && (dx || dw)) ? base + o.dz : nullptr;
    // the sums of a single block of rows are the result
    if (dbias && d.nb == 1) part = dbias;
    const auto run = [&](auto k) {
      oc::launch(k, dim3(d.nb, d.kb), dim3(TB), 0, s, dy, from_y ? y : pre, bf16, rows, cout, d.ct,
                 out, ldz, part);
    };
    if (glu) {
      if (act == OC_ACT_NONE) run(k_dz<true, OC_ACT_NONE, Z_F32>);
      else if (act == OC_ACT_RELU) run(k_dz<true, OC_ACT_RELU, Z_F32>);
      else if (act == OC_ACT_SILU) run(k_dz<true, OC_ACT_SILU, Z_F32>);
      else run(k_dz<true, OC_ACT_GELU, Z_F32>);
    } else {
      if (act == OC_ACT_NONE) run(k_dz<false, OC_ACT_NONE, Z_F32>);
      else if (from_y) run(k_dz<false, OC_ACT_RELU, Z_OUT>);
      else if (act == OC_ACT_RELU) run(k_dz<false, OC_ACT_RELU, Z_BITS>);
      else if (act == OC_ACT_SILU) run(k_dz<false, OC_ACT_SILU, Z_F32>);
      else run(k_dz<false, OC_ACT_GELU, Z_F32>);
    }
    if (dbias && d.nb > 1)
      oc::launch(k_colsum, dim3((unsigned)cdiv(nz, 4)), dim3(TB), 0, s, (const float*)part, d.nb,
                 nz, dbias);
  }
  int64_t ldx = cin, ldw = nz;
  if (pd && ((dw && cin % 8) || (dx && nz % 8))) {
    Pads p{};
    if (dw && cin % 8) {
      ldx = oc::pad8(cin);
      if (!again) p.p[0] = Pad{x, (uint16_t*)(base + o.x), rows, ldx, cin, 0};
      x = base + o.x;
    }
    if (dx && nz % 8) {
      ldw = oc::pad8(nz);
      p.p[1] = Pad{w, (uint16_t*)(base + o.w), cin, ldw, nz, 0};
      w = base + o.w;
    }
    pad(p, s);
  }
  const oc::Gemm gx{dt, rows, nz, cin, dz, w, ldz, ldw, 0, false, false,
                    {OC_ACT_NONE, 0, cin, bf16, 0, nullptr, nullptr, dx, nullptr, nullptr, 0,
                     nullptr}};
  const oc::Gemm gw{dt, cin, rows, nz, x, dz, ldx, ldz, 0, true, true,
                    {OC_ACT_NONE, 0, nz, dw_dt == OC_BF16, 0, nullptr, nullptr, dw, nullptr,
                     nullptr, 0, nullptr}};
  if (dx && dw) oc::gemm2(gx, gw, base + o.gemm, s);
  else if (dx) oc::gemm(gx, base + o.gemm, true, s);
  else if (dw) oc::gemm(gw, base + o.gemm, true, s);
  OC_LAUNCH_CHECK();
  return OC_OK;
}

}  // namespace

extern "C" {

size_t oc_dense_fwd_workspace(oc_dtype dt, int64_t rows, int32_t cin, int32_t cout) {
  return sizes_ok(dt, rows, cin, cout, false) ? fwd_ws(dt, rows, cin, cout, false).total : 0;
}

oc_status oc_dense_fwd(oc_dtype dt, int32_t act, int64_t rows, int32_t cin, int32_t cout,
                       const void* x, const void* w, const float* bias, const void* res, void* y,
                       void* pre, void* ws, size_t ws_bytes, hipStream_t s) {
  return fwd("oc_dense_fwd", false, dt, act, rows, cin, cout, x, w, bias, res, y, pre, ws,
             ws_bytes, s);
}

size_t oc_dense_bwd_workspace(oc_dtype dt, int32_t act, int64_t rows, int32_t cin, int32_t cout) {
  return sizes_ok(dt, rows, cin, cout, false) ? bwd_ws(dt, act, rows, cin, cout, false).total : 0;
}

oc_status oc_dense_bwd(oc_dtype dt, int32_t act, int64_t rows, int32_t cin, int32_t cout,
                       const void* x, const void* w, const float* bias, const void* pre,
                       const void* y, const void* dy, void* dx, oc_dtype dw_dt, void* dw,
                       float* dbias, void* ws, size_t ws_bytes, hipStream_t s) {
  return bwd("oc_dense_bwd", false, dt, act, rows, cin, cout, x, w, bias, pre, y, dy, dx, dw_dt,
             dw, dbias, ws, ws_bytes, s);
}

size_t oc_glu_fwd_workspace(oc_dtype dt, int64_t rows, int32_t cin, int32_t cout) {
  return sizes_ok(dt, rows, cin, cout, true) ? fwd_ws(dt, rows, cin, cout, true).total : 0;
}

oc_status oc_glu_fwd(oc_dtype dt, int32_t act, int64_t rows, int32_t cin, int32_t cout,
                     const void* x, const void* w, const float* bias, void* y, float* pre,
                     void* ws, size_t ws_bytes, hipStream_t s) {
  return fwd("oc_glu_fwd", true, dt, act, rows, cin, cout, x, w, bias, nullptr, y, pre, ws,
             ws_bytes, s);
}

size_t oc_glu_bwd_workspace(oc_dtype dt, int64_t rows, int32_t cin, int32_t cout) {
  return sizes_ok(dt, rows, cin, cout, true)
             ? bwd_ws(dt, OC_ACT_NONE, rows, cin, cout, true).total : 0;
}

oc_status oc_glu_bwd(oc_dtype dt, int32_t act, int64_t rows, int32_t cin, int32_t cout,
                     const void* x, const void* w, const float* bias, const float* pre,
                     const void* dy, void* dx, oc_dtype dw_dt, void* dw, float* dbias, void* ws,
                     size_t ws_bytes, hipStream_t s) {
  return bwd("oc_glu_bwd", true, dt, act, rows, cin, cout, x, w, bias, pre, nullptr, dy, dx,
             dw_dt, dw, dbias, ws, ws_bytes, s);
}

}  // extern "C"
