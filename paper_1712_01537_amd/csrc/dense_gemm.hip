// The matrix products of the dense layers, in plain fp32 FMAs: a 64 x 64 tile
// per workgroup, 16 terms of the reduction at a time through LDS.  Each thread
// forms 2 rows of eight columns (with glu: eight gate columns and the eight of
// the other half).  Every 1024 terms the running sum is added to the total and
// starts again, so that a sum of 10^6 terms rounds like one of 10^3.
#include "dense.h"

namespace {

using oc::Epi;

constexpr int TB = 256, BM = 64, BN = 64, BK = 16;

__device__ __forceinline__ float at(const void* p, bool bf16, int64_t i) {
  return oc::load1(p, bf16, i);
}

__global__ __launch_bounds__(TB) void k_gemm(const void* a, const void* b, bool bf16, bool a_rs,
                                             bool b_rs, int64_t P, int Q, int64_t R, Epi e) {
  __shared__ float A[BK][BM + 1], B[BK][BN + 1];
  const int tid = threadIdx.x;
  const int64_t p0 = (int64_t)blockIdx.x * BM;
  const int half = BN / 2;
  // column of tile position j: glu tiles hold 32 gate columns, then the other half's 32
  const int q0 = blockIdx.y * (e.glu ? half : BN);
  auto col = [&](int j) {
    if (!e.glu) return q0 + j < Q ? q0 + j : -1;
    const int c = q0 + (j & (half - 1));
    return c < e.n ? c + (j >= half ? e.n : 0) : -1;
  };
  const int tm = tid >> 3, tn = tid & 7;
  float acc[2][8] = {}, sum[2][8] = {};
  for (int64_t r0 = 0; r0 < R; r0 += BK) {
    for (int i = tid; i < BK * BM; i += TB) {
      const int r = a_rs ? i / BM : i % BK, p = a_rs ? i % BM : i / BK;
      const bool ok = p0 + p < P && r0 + r < R;
      A[r][p] = ok ? at(a, bf16, a_rs ? (r0 + r) * P + p0 + p : (p0 + p) * R + r0 + r) : 0.f;
    }
    for (int i = tid; i < BK * BN; i += TB) {
      const int r = b_rs ? i / BN : i % BK, j = b_rs ? i % BN : i / BK;
      const int q = col(j);
      const bool ok = q >= 0 && r0 + r < R;
      B[r][j] = ok ? at(b, bf16, b_rs ? (r0 + r) * Q + q : q * R + r0 + r) : 0.f;
    }
    __syncthreads();
    for (int r = 0; r < BK; ++r)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          acc[i][j] = fmaf(A[r][tm + 32 * i], B[r][tn * 8 + j], acc[i][j]);
    __syncthreads();
    if (r0 + BK >= R || (r0 / BK + 1) % 64 == 0)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          sum[i][j] += acc[i][j];
          acc[i][j] = 0.f;
        }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = sum[i][j];
  if (!e.glu) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t m = p0 + tm + 32 * i;
      if (m < P) oc::epi8(e, m, q0 + tn * 8, acc[i]);
    }
    return;
  }
  __shared__ float U[BM][half + 1];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (tn >= 4) U[tm + 32 * i][(tn - 4) * 8 + j] = acc[i][j];
  __syncthreads();
  if (tn < 4)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t m = p0 + tm + 32 * i;
      float u[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = U[tm + 32 * i][tn * 8 + j];
      if (m < P) oc::epi8_glu(e, m, q0 + tn * 8, acc[i], u);
    }
}

}  // namespace

namespace oc {

size_t gemm_ws(oc_dtype, int64_t, int64_t, int64_t, bool, bool, bool) { return 0; }

void gemm(const Gemm& g, void*, bool main, hipStream_t s) {
  const dim3 grid((unsigned)cdiv(g.P, BM), (unsigned)cdiv(g.epi.n, g.epi.glu ? BN / 2 : BN));
  if (main)
    launch_main(k_gemm, grid, dim3(TB), s, g.a, g.b, g.dt == OC_BF16, g.a_rs, g.b_rs, g.P, g.Q,
                g.R, g.epi);
  else
    launch(k_gemm, grid, dim3(TB), 0, s, g.a, g.b, g.dt == OC_BF16, g.a_rs, g.b_rs, g.P, g.Q, g.R,
           g.epi);
}

}  // namespace oc
