// The dense layers' forward for a few rows (a service's answer, a loop's single
// step): every weight is used once or a few times, so the time is that of
// reading them, and a matrix core would be fed with padding.
//
// A workgroup has up to four rows and 16 columns (gated: and the 16 of the other
// half); a thread has eight of the columns and every 128th group of four terms of
// the reduction, in fp32 FMAs.  The threads of a column meet through shuffles and
// then LDS, in a fixed order, and one of them runs the epilogue: one launch, no
// workspace.  Neighbouring workgroups, which share the weights' cache lines, run on
// one XCD.  Bound by memory once the weights are many, by latency below: one row on
// bf16 1024 x 1024 takes 4.1 us, 4096 x 4096 8.7 us (3.9 TB/s), fp32 14.8 us (4.5
// TB/s); with 64 columns a workgroup, whole cache lines, 5.1, 17.3 and 17.1 us (too
// few workgroups).  The 64 x 64 tile takes 7.7, 13.3 and 28.8 us.
#include <type_traits>

#include "dense.h"

namespace {

constexpr int TB = 256, WAVES = TB / 64;
constexpr int CL = 2, LK = TB / CL;  // threads along the columns, along the reduction

// Four consecutive elements i .. i + 3.
template <bool BF16>
__device__ __forceinline__ void load4(const void* p, int64_t i, float (&v)[4]) {
  if (BF16) {
    typedef oc::d_v2u v2u_any __attribute__((aligned(2)));
    const oc::d_v2u u = *(const v2u_any*)((const uint16_t*)p + i);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      v[2 * k] = oc::bf_up(u[k] & 0xffffu);
      v[2 * k + 1] = __builtin_bit_cast(float, u[k] & 0xffff0000u);
    }
  } else {
    const oc::d_v4f u = *(const oc::d_v4f_any*)((const float*)p + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = u[k];
  }
}

template <bool BF16, int ROWS, bool GLU>
__global__ __launch_bounds__(TB) void k_dense_rows(const void* x, const void* w, int rows, int R,
                                                   int Q, oc::Epi e) {
  constexpr int H = GLU ? 2 : 1;
  __shared__ float red[WAVES][H][ROWS][CL][8];
  const int tid = threadIdx.x, tc = tid % CL, kl = tid / CL;
  const int row0 = blockIdx.y * ROWS, left = rows - row0 < ROWS ? rows - row0 : ROWS;
  const int c = (oc::xcd_order(blockIdx.x, gridDim.x) * CL + tc) * 8;
  const int64_t all = (int64_t)R * Q;
  // rows of w whose vectors are all inside it, however short the rows
  const int safe = Q % 8 == 0 && e.n % 8 == 0 ? R : R - (8 + Q - 1) / Q, Rv = safe < 4 ? 0 : safe / 4 * 4;
  float acc[H][ROWS][8] = {};
  if (c < e.n) {
    auto add = [&](int h, const float (&xv)[ROWS], const float (&wv)[8]) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[h][r][j] = fmaf(xv[r], wv[j], acc[h][r][j]);
    };
    // G groups of four terms, all their loads started before the first is used
    auto group = [&](auto g, int k) __attribute__((always_inline)) {
      constexpr int G = decltype(g)::value, V = BF16 ? 1 : 2;
      oc::d_v4u raw[G][4][H][V];
      float xv[G][ROWS][4];
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int v = 0; v < V; ++v) {
              const int64_t at = (int64_t)(k + i * 4 * LK + j) * Q + h * e.n + c + 4 * v;
              raw[i][j][h][v] = BF16 ? *(const oc::d_v4u_any*)((const uint16_t*)w + at)
                                     : *(const oc::d_v4u_any*)((const float*)w + at);
            }
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
          load4<BF16>(x, (row0 + (r < left ? r : 0)) * (int64_t)R + k + i * 4 * LK, xv[i][r]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float one[ROWS];
#pragma unroll
          for (int r = 0; r < ROWS; ++r) one[r] = xv[i][r][j];
#pragma unroll
          for (int h = 0; h < H; ++h) {
            float wv[8];
#pragma unroll
            for (int m = 0; m < 4; ++m) {
              if (BF16) {
                wv[2 * m] = oc::bf_up(raw[i][j][h][0][m] & 0xffffu);
                wv[2 * m + 1] = __builtin_bit_cast(float, raw[i][j][h][0][m] & 0xffff0000u);
              } else {  // (a bit cast of a vector's element would take the first one's bits)
                wv[m] = __builtin_bit_cast(oc::d_v4f, raw[i][j][h][0])[m];
                wv[4 + m] = __builtin_bit_cast(oc::d_v4f, raw[i][j][h][V - 1])[m];
              }
            }
            add(h, one, wv);
          }
        }
    };
    constexpr int G = BF16 && H == 1 ? 4 : 2, STEP = G * 4 * LK;
    int k0 = 0;
    for (; k0 + STEP <= Rv; k0 += STEP) group(std::integral_constant<int, G>{}, k0 + kl * 4);
    for (int k = k0 + kl * 4; k < Rv; k += LK * 4) group(std::integral_constant<int, 1>{}, k);
    for (int k = Rv + kl; k < R; k += LK) {
      float one[ROWS], wv[8];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) one[r] = oc::load1(x, BF16, (row0 + (r < left ? r : 0)) * (int64_t)R + k);
#pragma unroll
      for (int h = 0; h < H; ++h) {
        oc::load8n(w, BF16, (int64_t)k * Q + h * e.n + c, 8, all, wv);
        add(h, one, wv);
      }
    }
  }
  for (int m = 32; m >= CL; m >>= 1)
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[h][r][j] += __shfl_xor(acc[h][r][j], m);
  const int lane = tid & 63;
  if (lane < CL)
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j) red[tid >> 6][h][r][lane][j] = acc[h][r][j];
  __syncthreads();
  const int r = tid / CL;
  if (r >= left || c >= e.n) return;
  float z[1][8] = {}, u[1][8] = {};
#pragma unroll
  for (int v = 0; v < WAVES; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      z[0][j] += red[v][0][r][tc][j];
      if (GLU) u[0][j] += red[v][H - 1][r][tc][j];
    }
  float b0[8] = {}, b1[8] = {};
  if (e.bias) {
    oc::load8n(e.bias, false, c, e.n - c, Q, b0);
    if (GLU) oc::load8n(e.bias, false, e.n + c, e.n - c, Q, b1);
  }
  const int64_t m[1] = {row0 + r};
  oc::epilogue<1, GLU>(e, m, rows, c, b0, b1, z, u);
}

}  // namespace

namespace oc {

void gemm_rows(oc_dtype dt, int32_t rows, int32_t R, int32_t Q, const void* x, const void* w,
               const Epi& epi, hipStream_t s) {
  const int ROWS = rows < 3 ? rows : 4;
  const dim3 grid((unsigned)cdiv(epi.n, 8 * CL), (unsigned)cdiv(rows, ROWS));
  const auto run = [&](auto k) {
    launch_main(k, grid, dim3(TB), s, x, w, (int)rows, (int)R, (int)Q, epi);
  };
  const auto pick = [&](auto bf16, auto glu) {
    constexpr bool B = decltype(bf16)::value, G = decltype(glu)::value;
    if (rows == 1) run(k_dense_rows<B, 1, G>);
    else if (rows == 2) run(k_dense_rows<B, 2, G>);
    else run(k_dense_rows<B, 4, G>);
  };
  if (dt == OC_BF16) {
    if (epi.glu) pick(std::true_type{}, std::true_type{});
    else pick(std::true_type{}, std::false_type{});
  } else {
    if (epi.glu) pick(std::false_type{}, std::true_type{});
    else pick(std::false_type{}, std::false_type{});
  }
}

}  // namespace oc
