// Layer norm and the residual step on rows that fit in registers: TPR threads hold a row,
// NV vectors of eight channels each, so that each row is read once.  The next row's loads
// are started before the present one's sums.
//
// Bound by memory: each value is read and written once (the forward of 65536 x 4096 bf16
// writes 517 MiB, its backward 544 with the column sums).  That forward takes 205 us (5.2
// TB/s), its backward 326 (4.9); the residual step of 16384 x 8192 fp32 395 and 630 (5.4 and
// 5.1); a large copy reaches 4.7 to 5.3.  The backward of rows of 8193 to 16384 keeps no
// next row and reaches 2.2 to 4.5: the values of four vectors a thread do not fit its
// registers (scratch a lane: bf16 step 224 bytes, fp32 step 148, bf16 norm 28, fp32 norm
// none).
#include <algorithm>

#include "norm.h"

namespace {

using oc::cdiv;
using oc::cut;
using oc::hidden;
using oc::MOST_ADDED;
using oc::Norm;
using oc::NormBwd;
using oc::Place;
using oc::Raw;
using oc::row_store;
using oc::unpack;

// (A vector's element goes by value: __builtin_bit_cast of v[1] itself takes v[0].)
__device__ __forceinline__ float float_of(uint32_t u) { return __builtin_bit_cast(float, u); }

// v of another lane by data-parallel primitives (no trip through LDS).
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// The sum over groups of L lanes (a power of two up to 64), in each of them: pairs, then
// pairs of pairs, ...  Each step adds the same two values in both halves, so that the
// lanes agree in every bit.
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  if (L >= 2) v += dpp<0xB1>(v);   // quad_perm 1 0 3 2
  if (L >= 4) v += dpp<0x4E>(v);   // quad_perm 2 3 0 1
  if (L >= 8) v += dpp<0x141>(v);  // row_half_mirror: the other four of eight
  if (L >= 16) v += dpp<0x140>(v); // row_mirror: the other eight of sixteen
  if (L >= 32) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = float_of(r[0]) + float_of(r[1]);
  }
  if (L >= 64) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    v = float_of(r[0]) + float_of(r[1]);
  }
  return v;
}

// Threads of a workgroup.
constexpr int block_fwd(int tpr) { return tpr <= 64 ? 256 : tpr; }
constexpr int block_bwd(int tpr) { return tpr <= 512 ? 512 : tpr; }
// Waves that a SIMD holds of a forward kernel, by the registers it needs, or two fewer:
// bf16 norms and fp32 steps of 9 to 256 channels keep two registers in scratch (12 bytes a
// lane), the fp32 step of 1024 threads five.  (With one wave fewer and no scratch 2^27
// values of 64 channels take 98 us as with it for the bf16 norm, 426 us instead of 431 for
// the fp32 step.)  The forward has as many workgroups as the card holds at once (one more
// would be a round of its own: bf16 rows of 64 to 256 channels 4.6 TB/s instead of 5.4).
constexpr int waves_fwd(int tpr, int nv, bool step) {
  return nv == 1 ? (step ? 6 : 8) : step || tpr >= 512 ? 4 : 5;
}

// The row's h from what lies in memory.
template <bool BF, bool STEP>
__device__ __forceinline__ void form_h(const Raw<BF>& x, const Raw<BF>& res, bool has_res,
                                       const oc::Drop& drop, const oc::DropKey& key,
                                       uint64_t index, float (&v)[8], bool (&keep)[8]) {
  unpack(x, v);
  if (STEP) {
    if (drop.on) {
      oc::keep8(drop, key, index, keep);
      oc::drop8(drop, keep, v);
    }
    if (has_res) {
      float r[8];
      unpack(res, r);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += r[k];
    }
  }
}

// The lanes that share a row's index, as one number where a wave has one row.
template <int TPR>
__device__ __forceinline__ int group_of(int thread) {
  return TPR >= 64 ? __builtin_amdgcn_readfirstlane(thread / TPR) : thread / TPR;
}

// Rows of more than one wave add their waves' sums through `red`, wave by wave.  Rows in
// turn use its two halves: a wave that has passed a row's barrier has read the row before.
//
// Forward.  The lanes of a wave find their mean m by one sum, then delta = mean of v - m
// and the mean square of v - m by two more (each square is divided by the count before it
// is added, as the values of the mean are, so that the sum stays in range); waves are
// joined by Chan et al.'s formula for counts, means and mean squared deviations, relative
// to the first wave's mean.
template <bool BF, int TPR, int NV, bool STEP>
__global__ __launch_bounds__(block_fwd(TPR), waves_fwd(TPR, NV, STEP)) void
    k_ln_rows(Norm a) {
  constexpr int BLK = block_fwd(TPR), G = BLK / TPR, L = TPR < 64 ? TPR : 64, W = TPR / L;
  __shared__ float red[2][W > 1 ? W : 1][3];
  const int t = threadIdx.x % TPR, g = group_of<TPR>(threadIdx.x);
  const int nv = (a.c + 7) / 8;
  const int64_t n = a.rows * a.c, stride = (int64_t)gridDim.x * G;
  const oc::DropKey key = STEP && a.drop.on ? oc::drop_key(a.drop) : oc::DropKey{};
  const bool has_res = STEP && a.res;
  int cnt[NV];
  float gam[NV][8], bet[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (j * TPR + t) * 8;
    cnt[j] = a.c - col;
#pragma unroll
    for (int k = 0; k < 8; ++k) gam[j][k] = 1.f, bet[j][k] = 0.f;
    if (a.gamma && cnt[j] > 0) oc::load8n(a.gamma, false, col, cnt[j], a.c, gam[j]);
    if (a.beta && cnt[j] > 0) oc::load8n(a.beta, false, col, cnt[j], a.c, bet[j]);
  }
  const auto place = [&](int64_t at, int j) {
    return Place{at, (j * TPR + t) * 8, cnt[j], n - at};
  };
  // channels of a wave's part of a row
  const auto channels = [&](int w) {
    int have = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int left = a.c - (j * TPR + w * L) * 8;
      have += left < 0 ? 0 : left < L * 8 ? left : L * 8;
    }
    return (float)have;
  };
  const int w0 = t / L;
  const float own = channels(w0), r_own = own > 0.f ? 1.f / own : 0.f, rc = 1.f / (float)a.c;
  Raw<BF> x[NV], res[NV];
  const auto load = [&](int64_t at) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (cnt[j] > 0) {
        raw_load(x[j], a.x, place(at, j));
        if (has_res) raw_load(res[j], a.res, place(at, j));
      }
  };
  int64_t row = (int64_t)blockIdx.x * G + g;
  int64_t at = row * a.c;
  const int64_t on = stride * a.c;
  if (row < a.rows) load(at);
  for (int par = 0; row < a.rows; row += stride, at += on, par ^= 1) {
    float v[NV][8];
    bool keep[8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      form_h<BF, STEP>(x[j], res[j], has_res, a.drop, key, (uint64_t)row * nv + (j * TPR + t),
                       v[j], keep);
      cut(v[j], cnt[j]);
    }
    if (row + stride < a.rows) load(at + on);
    if (STEP) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (cnt[j] > 0) row_store<BF>(a.h, place(at, j), v[j]);
    }
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) m = fmaf(v[j][k], r_own, m);
    m = lanes_sum<L>(m);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[j][k] -= m;
      cut(v[j], cnt[j]);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        s1 += v[j][k];
        s2 = fmaf(v[j][k] * r_own, v[j][k], s2);
      }
    }
    s1 = lanes_sum<L>(s1);
    s2 = lanes_sum<L>(s2);
    float delta = s1 * r_own, var = fmaf(-delta, delta, s2), mean = m + delta;
    if (W > 1) {
      if ((t & 63) == 0) {
        red[par][w0][0] = m;
        red[par][w0][1] = delta;
        red[par][w0][2] = var;
      }
      __syncthreads();
      const float m0 = red[par][0][0];
      float far = 0.f;  // the row's mean - m0
#pragma unroll
      for (int w = 0; w < W; ++w)
        far = fmaf(channels(w) * rc, (red[par][w][0] - m0) + red[par][w][1], far);
      var = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float d = ((red[par][w][0] - m0) + red[par][w][1]) - far, share = channels(w) * rc;
        var += share > 0.f ? share * fmaf(d, d, red[par][w][2]) : 0.f;
      }
      delta = far - (m - m0);  // of this wave's deviations
      mean = m0 + far;
    }
    if (var < 0.f) var = 0.f;  // (NaN stays NaN)
    const float invstd = 1.f / sqrtf(var + a.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (cnt[j] <= 0) continue;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[j][k] = fmaf((v[j][k] - delta) * invstd, gam[j][k], bet[j][k]);
      row_store<BF>(a.y, place(at, j), v[j]);
    }
    if (t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.invstd) a.invstd[row] = invstd;
    }
  }
}

// Backward: one reduction of three sums a row (of g, g d and d, with d = (h - mean)
// invstd: the deviations themselves times g can be past fp32 where dx is not), of a
// thread's one vector up to 4096 channels (two vectors: 16 waves of 128 registers spill),
// two up to 8192 (512 threads of up to 256 registers: fp32 residual step 630 us for 16384
// x 8192, with 1024 threads of one vector 850), four above; bf16 rows that leave a quarter
// of the lanes of one vector without work have three (2^27 values in rows of 768: 174 us
// instead of 215, of 1536 177 instead of 202).  dgamma's and dbeta's sums stay in
// registers over the group's rows, at most MOST_ADDED; the workgroup's groups are then
// added in double through LDS, and its sums written for the sum over the workgroups.
template <bool BF, int TPR, int NV, bool STEP>
__global__ __launch_bounds__(block_bwd(TPR), NV == 1 ? 4 : 2) void
    k_ln_rows_bwd(NormBwd a, float* part) {
  constexpr int BLK = block_bwd(TPR), G = BLK / TPR, L = TPR < 64 ? TPR : 64, W = TPR / L;
  __shared__ float red[2][W > 1 ? BLK / 64 : 1][3];
  __shared__ float cols[G > 1 ? 2 : 1][G > 1 ? 8 : 1][G > 1 ? BLK : 1];
  const int t = threadIdx.x % TPR, g = group_of<TPR>(threadIdx.x);
  const int nv = (a.c + 7) / 8;
  const int64_t n = a.rows * a.c, nb = gridDim.x, b = blockIdx.x;
  const int64_t r0 = a.rows * b / nb, r1 = a.rows * (b + 1) / nb;
  const oc::DropKey key = STEP && a.drop.on ? oc::drop_key(a.drop) : oc::DropKey{};
  const bool has_res = STEP && a.res, has_dh = STEP && a.dh;
  const float rc = 1.f / (float)a.c;
  int cnt[NV];
  // Four vectors a thread leave no registers for the next row's loads and gamma.
  constexpr bool AHEAD = NV <= 3;
  float gam[AHEAD ? NV : 1][8], sg[NV][8], sb[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    cnt[j] = a.c - (j * TPR + t) * 8;
#pragma unroll
    for (int k = 0; k < 8; ++k) sg[j][k] = sb[j][k] = 0.f;
  }
  const auto load_gamma = [&](int j, float(&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 1.f;
    if (a.gamma && cnt[j] > 0)
      oc::load8n(a.gamma, false, (j * TPR + t) * 8, hidden(cnt[j]), a.c, v);
  };
  if (AHEAD)
#pragma unroll
    for (int j = 0; j < NV; ++j) load_gamma(j, gam[j]);
  const auto place = [&](int64_t at, int j) {
    return Place{at, (j * TPR + t) * 8, cnt[j], n - at};
  };
  // (of four fp32 vectors one is loaded at a time)
  constexpr int RAWS = AHEAD || BF ? NV : 1;
  // d is held times invstd, but for four fp32 vectors, where g d is formed as (g invstd) d:
  // the step's backward of 8192 x 16384 takes 734 us, with d held times invstd 758.
  constexpr bool SCALED = RAWS == NV;
  Raw<BF> x[RAWS], res[RAWS], dy[RAWS], dh[AHEAD ? NV : 1];
  float mean = 0.f, invstd = 0.f;
  const auto load_at = [&](int64_t at, int j, Raw<BF>& rx, Raw<BF>& rdy, Raw<BF>& rres) {
    if (cnt[j] <= 0) return;
    raw_load(rx, a.x, place(at, j));
    raw_load(rdy, a.dy, place(at, j));
    if (has_res) raw_load(rres, a.res, place(at, j));
  };
  const auto load = [&](int64_t row, int64_t at) {
    mean = a.mean[row];
    invstd = a.invstd[row];
    if (RAWS == NV)
#pragma unroll
      for (int j = 0; j < NV; ++j) load_at(at, j, x[j % RAWS], dy[j % RAWS], res[j % RAWS]);
  };
  // (groups that share a workgroup's barriers make the same number of steps)
  int64_t at = (r0 + g) * a.c;
  const int64_t on = (int64_t)G * a.c;
  if (AHEAD && r0 + g < r1) load(r0 + g, at);
  for (int64_t first = r0, par = 0; first < r1; first += G, at += on, par ^= 1) {
    const int64_t row = first + g;
    const bool here = W == 1 || G == 1 || row < r1;
    if (W == 1 && row >= r1) break;
    if (!AHEAD && here) load(row, at);
    float d[NV][8], e[NV][8];
    bool keep[AHEAD ? NV : 1][8];
    uint32_t kept = 0;  // (bits for bools, of which each takes two scalar registers)
    const float m = mean, r = invstd;
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int i = AHEAD ? j : 0;
      const int l = j % RAWS;
      if (RAWS < NV && here) load_at(at, j, x[l], dy[l], res[l]);
      form_h<BF, STEP>(x[l], res[l], has_res, a.drop, key, (uint64_t)row * nv + (j * TPR + t),
                       d[j], keep[i]);
      unpack(dy[l], e[j]);
#pragma unroll
      for (int k = 0; k < 8; ++k) d[j][k] = SCALED ? (d[j][k] - m) * r : d[j][k] - m;
      cut(d[j], here ? cnt[j] : 0);
      cut(e[j], here ? cnt[j] : 0);
      if (!AHEAD) {
        load_gamma(j, gam[i]);
        if (STEP && a.drop.on)
#pragma unroll
          for (int k = 0; k < 8; ++k) kept |= (keep[i][k] ? 1u : 0u) << (j * 8 + k);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float q = e[j][k] * gam[i][k];
        s[0] += q;
        s[1] = fmaf(SCALED ? q : q * r, d[j][k], s[1]);
        s[2] += d[j][k];
      }
      // (the next vector's loads stay behind this one's use: their registers are the same)
      if (RAWS < NV) asm volatile("" ::: "memory");
    }
    // needed behind the sums only: loaded while they are formed
    if (AHEAD) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (has_dh && here && cnt[j] > 0) raw_load(dh[AHEAD ? j : 0], a.dh, place(at, j));
      if (row + G < r1) load(row + G, at + on);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k] = lanes_sum<L>(s[k]);
    if (W > 1) {
      if ((t & 63) == 0) {
#pragma unroll
        for (int k = 0; k < 3; ++k) red[par][threadIdx.x / 64][k] = s[k];
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        s[k] = red[par][g * W][k];
#pragma unroll
        for (int w = 1; w < W; ++w) s[k] += red[par][g * W + w][k];
      }
    }
    const float delta = s[2] * rc, gm = s[0] * rc;
    const float zm = fmaf(SCALED ? -delta : -delta * r, s[0], s[1]) * rc;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int i = AHEAD ? j : 0;
      float u[8] = {};
      if (!AHEAD) {
        if (has_dh && here && cnt[j] > 0) raw_load(dh[i], a.dh, place(at, j));
        load_gamma(j, gam[i]);
      }
      if (has_dh && here && cnt[j] > 0) unpack(dh[i], u);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float z = SCALED ? d[j][k] - delta : (d[j][k] - delta) * r;
        sg[j][k] = fmaf(e[j][k], z, sg[j][k]);
        sb[j][k] += e[j][k];
        e[j][k] = r * fmaf(-z, zm, fmaf(e[j][k], gam[i][k], -gm));
        if (has_dh) e[j][k] += u[k];
      }
      if (!here || cnt[j] <= 0) continue;
      if (a.dres) row_store<BF>(a.dres, place(at, j), e[j]);
      if (STEP && a.dx) {
        if (a.drop.on) {
          if (!AHEAD)
#pragma unroll
            for (int k = 0; k < 8; ++k) keep[i][k] = kept >> (j * 8 + k) & 1;
          oc::drop8(a.drop, keep[i], e[j]);
        }
        row_store<BF>(a.dx, place(at, j), e[j]);
      }
      if (RAWS < NV) asm volatile("" ::: "memory");
    }
  }
  if (!part) return;
  if (G == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (cnt[j] <= 0) continue;
      const int col = (j * TPR + t) * 8;
      oc::store8n(part + b * 2 * a.c, false, col, cnt[j], sg[j]);
      oc::store8n(part + (b * 2 + 1) * a.c, false, col, cnt[j], sb[j]);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      cols[0][k][threadIdx.x] = sg[j][k];
      cols[G > 1][k][threadIdx.x] = sb[j][k];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < TPR * 16; i += BLK) {
      const int h = i / (TPR * 8), q = i % (TPR * 8), col = j * TPR * 8 + q;
      if (col >= a.c) continue;
      double sum = 0.0;
#pragma unroll
      for (int w = 0; w < G; ++w) sum += (double)cols[h][q & 7][w * TPR + (q >> 3)];
      part[(b * 2 + h) * a.c + col] = (float)sum;
    }
  }
}

// Threads of a row of c channels with v vectors each, at least as many as a power of two
// up to a wave takes.
int threads_of(int c, int v) {
  const int nv = (int)cdiv(c, 8);
  int t = 1;
  while (t < 64 && t < nv) t *= 2;
  while (v * t < nv) t *= 2;
  return t;
}
int threads_bwd(int c) { return threads_of(c, c <= 4096 ? 1 : c <= 8192 ? 2 : 4); }

// f(threads of a row, vectors of a thread), both as constants.
template <int V>
using Int = std::integral_constant<int, V>;
template <typename F>
void with_small(int t, F&& f) {
  switch (t) {
    case 1: return f(Int<1>{}, Int<1>{});
    case 2: return f(Int<2>{}, Int<1>{});
    case 4: return f(Int<4>{}, Int<1>{});
    case 8: return f(Int<8>{}, Int<1>{});
    case 16: return f(Int<16>{}, Int<1>{});
    case 32: return f(Int<32>{}, Int<1>{});
    default: return f(Int<64>{}, Int<1>{});
  }
}
template <typename F>
void with_fwd(int c, F&& f) {
  const int t = threads_of(c, 2);
  if (c <= 512) return with_small(t, f);
  switch (t) {
    case 64: return f(Int<64>{}, Int<2>{});
    case 128: return f(Int<128>{}, Int<2>{});
    case 256: return f(Int<256>{}, Int<2>{});
    case 512: return f(Int<512>{}, Int<2>{});
    default: return f(Int<1024>{}, Int<2>{});
  }
}
template <typename F>
void with_bwd(int c, bool three, F&& f) {
  const int t = threads_bwd(c);
  if (three)
    return t == 128 ? f(Int<32>{}, Int<3>{})
           : t == 256 ? f(Int<64>{}, Int<3>{}) : f(Int<128>{}, Int<3>{});
  if (c <= 512) return with_small(t, f);
  if (c > 8192) return f(Int<512>{}, Int<4>{});
  if (c > 4096) return f(Int<512>{}, Int<2>{});
  switch (t) {
    case 128: return f(Int<128>{}, Int<1>{});
    case 256: return f(Int<256>{}, Int<1>{});
    default: return f(Int<512>{}, Int<1>{});
  }
}

}  // namespace

namespace oc {

void norm_rows_fwd(const Norm& a, hipStream_t s) {
  with_fwd(a.c, [&](auto t, auto v) {
    constexpr int TPR = decltype(t)::value, NV = decltype(v)::value, BLK = block_fwd(TPR);
    const auto go = [&](auto kernel, int waves) {
      const int64_t most = waves * 256 / BLK * (int64_t)cu_count();
      launch_main(kernel, dim3((unsigned)std::min(cdiv(a.rows, BLK / TPR), most)), dim3(BLK), s,
                  a);
    };
    constexpr int PLAIN = waves_fwd(TPR, NV, false), STEP = waves_fwd(TPR, NV, true);
    if (a.h)
      a.bf16 ? go(k_ln_rows<true, TPR, NV, true>, STEP) : go(k_ln_rows<false, TPR, NV, true>, STEP);
    else
      a.bf16 ? go(k_ln_rows<true, TPR, NV, false>, PLAIN)
             : go(k_ln_rows<false, TPR, NV, false>, PLAIN);
  });
}

int64_t norm_rows_blocks(int64_t rows, int32_t c) {
  const int tpr = threads_bwd(c), g = block_bwd(tpr) / tpr;
  // (twice as many workgroups as CUs where every group then has two rows or more and a
  // workgroup four: 1000 x 4096 fp32 takes 21 us with two rows a workgroup, 16 with four)
  return std::max(std::min<int64_t>(cdiv(rows, std::max(2 * g, 4)), 512),
                  cdiv(rows, MOST_ADDED * g));
}

void norm_rows_bwd(const NormBwd& a, float* part, hipStream_t s) {
  const int64_t blocks = norm_rows_blocks(a.rows, a.c);
  // three vectors a thread: a quarter of the threads, and each group needs some rows (4096
  // x 768: 17.5 us, with one vector 13)
  const int one = threads_bwd(a.c);
  const bool three = a.bf16 && one >= 128 && a.c <= 4096 && cdiv(a.c, 8) * 4 <= 3 * one &&
                     a.rows >= blocks * 4 * (4 * 512 / one);
  with_bwd(a.c, three, [&](auto t, auto v) {
    constexpr int TPR = decltype(t)::value, NV = decltype(v)::value;
    const auto go = [&](auto kernel) {
      launch_main(kernel, dim3((unsigned)blocks), dim3(block_bwd(TPR)), s, a, part);
    };
    if (a.drop.on || a.res || a.dx || a.dh)
      a.bf16 ? go(k_ln_rows_bwd<true, TPR, NV, true>)
             : go(k_ln_rows_bwd<NV == 3, TPR, NV, true>);  // (three: bf16 only)
    else
      a.bf16 ? go(k_ln_rows_bwd<true, TPR, NV, false>)
             : go(k_ln_rows_bwd<NV == 3, TPR, NV, false>);
  });
}

}  // namespace oc
