// Dense layers over rows: the matrix products of oc_dense_* and oc_glu_* and
// what their epilogues do.
#pragma once

#include "common.h"

namespace oc {

typedef float d_v4f __attribute__((ext_vector_type(4)));
typedef uint32_t d_v4u __attribute__((ext_vector_type(4)));
typedef uint32_t d_v2u __attribute__((ext_vector_type(2)));
// Vectors at any element's address: global memory takes them at any alignment.
typedef d_v4f d_v4f_any __attribute__((aligned(4)));
typedef d_v4u d_v4u_any __attribute__((aligned(2)));

// What becomes of the product z [M][nz] (nz = n, or 2 n when glu):
//   glu 0: y[m][c] = act(z[m][c] + bias[c]) + res[m][c]
//   glu 1: y[m][c] = act(z[m][c] + bias[c]) (z[m][n + c] + bias[n + c])
// pre (if any) receives z + bias in fp32, or with pre_bits the bits [z + bias > 0],
// eight columns a byte, (n + 7) / 8 bytes a row.  y and res are bf16 when y_bf16, else
// fp32.  A residual may be y itself: a lane reads its elements before it writes them.
struct Epi {
  int32_t act, glu, n;
  int32_t y_bf16, pre_bits;
  const float* bias;
  const void* res;
  void* y;
  void* pre;
  // The backward's dz from a product formed again instead (dy given; type y_bf16):
  // y receives dz = dy act'(z) (gated [dy u act'(g) | dy act(g)]) in rows of ldz
  // elements, zero past the columns, and colsum [row tiles][nz], if any, its column sums.
  const void* dy;
  int64_t ldz;
  float* colsum;
};

// out [P][Q] = sum over r < R of A(p, r) B(r, q), then `epi` (M = P, nz = Q).
//   a_rs 0: A is stored [P][R], 1: [R][P].  b_rs 1: B is stored [R][Q], 0: [Q][R].
//   lda, ldb: elements from row to row; columns between a row's end and there hold
//   zeros where they lie in its last 16-byte vector.  half: with glu, B's column of
//   the other half's first.  dt: type of A and B.
struct Gemm {
  oc_dtype dt;
  int64_t P, R;
  int32_t Q;
  const void *a, *b;
  int64_t lda, ldb;
  int32_t half;
  bool a_rs, b_rs;
  Epi epi;
};

// Whether a layer's bf16 operands are copied to rows of whole 16-byte vectors first:
// where they are not, and the product is large enough to gain from it (8383 x 513 ->
// 1027: the forward takes 48 us on rows of any length through registers, in 64 x 64
// tiles, and 37 with the copies; a product of 2 GFLOP takes some 10 either way).
inline bool pads(oc_dtype dt, int64_t rows, int64_t cin, int64_t cout, bool glu) {
  return dt == OC_BF16 && (cin % 8 || cout % 8) &&
         2.0 * rows * cin * cout * (glu ? 2 : 1) >= 2e9;
}
inline int64_t pad8(int64_t n) { return (n + 7) / 8 * 8; }

// The forward product of few rows: out [rows][Q] = x [rows][R] times w [R][Q], no workspace.
// Few: where it is faster than the tiles, that is for up to 4 (fp32: 8) rows, and for
// more while its workgroups (4 rows, 16 columns) have a CU each and the reduction is
// not long.  With tiles in brackets: fp32 1024 -> 1024, 8 rows 6.1 us (10.5), 16 rows 6.3
// (10.9); 4096 -> 4096, 8 rows 24 (28), 16 rows 49 (28); bf16 1024 -> 1024, 4 rows 5.7
// (7.7), 8 rows 5.9 (7.6); 4096 -> 4096, 4 rows 11.7 (13.4), 8 rows 17.0 (13.7).
inline bool few_rows(oc_dtype dt, int64_t rows, int64_t cin, int64_t cout) {
  return rows <= (dt == OC_F32 ? 8 : 4) ||
         (rows <= 64 && cdiv(cout, 16) * cdiv(rows, 4) <= 256 && cin <= 2048);
}
void gemm_rows(oc_dtype dt, int32_t rows, int32_t R, int32_t Q, const void* x, const void* w,
               const Epi& epi, hipStream_t s);

// Row tiles of a product that forms dz.
int64_t gemm_dz_tiles(oc_dtype dt, bool direct, int64_t P, int64_t Q, int64_t R, bool glu);
// Whether its operands go straight to LDS.
bool gemm_direct(oc_dtype dt, const void* a, int64_t lda, const void* b, int64_t ldb, bool glu,
                 int64_t half);

// Bytes of workspace the product needs (partial sums of a split reduction);
// a function of the type and the sizes alone.
size_t gemm_ws(oc_dtype dt, int64_t P, int64_t Q, int64_t R, bool glu);
// Likewise of gemm2.
size_t gemm2_ws(oc_dtype dt, int64_t rows, int64_t cin, int64_t nz);
// Enqueue it.  main: its kernel does the call's main arithmetic (profiling).
void gemm(const Gemm& g, void* ws, bool main, hipStream_t s);
// Both products of a backward: dx [rows][cin] over nz terms, dw [cin][nz] over the rows.
void gemm2(const Gemm& dx, const Gemm& dw, void* ws, hipStream_t s);

// --- device side ---------------------------------------------------------

// The place of block i of `total` in an order of tiles or columns: each XCD (blocks are
// dealt out to the eight in turn) takes a contiguous range.
__device__ __forceinline__ uint32_t xcd_order(uint32_t i, uint32_t total) {
  const uint32_t x = i & 7, per = total >> 3, rem = total & 7;
  return x * per + (x < rem ? x : rem) + (i >> 3);
}

__device__ __forceinline__ float bf_up(uint32_t h) {
  return __builtin_bit_cast(float, h << 16);
}
// Two values rounded to bf16 (nearest, ties to even), the first in the low half.
__device__ __forceinline__ uint32_t bf_pair(float a, float b) {
  typedef float v2f __attribute__((ext_vector_type(2)));
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){a, b}, v2bf));
}

// Activations and their gradients in fp32.  SiLU is z s, s = 1 / (1 + e^-z), of
// slope s (1 + z (1 - s)); GELU is z Phi(z), of slope Phi(z) + z phi(z), Phi
// and phi the normal distribution and its density.  The exponential and the
// reciprocal are the hardware's (one ulp of 2^x; x = z log2 e is off by |z| ulp,
// where e^z itself is small): some 20 instructions a value instead of 40 for erff,
// which took 40 of the 107 us of a 35472 x 256 -> 1024 GELU layer.
__device__ __forceinline__ float exp_fast(float x) {
  return __builtin_amdgcn_exp2f(x * 1.44269504088896341f);
}
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + exp_fast(-z));
}
// Phi(-|z|), that is half of 1 - erf(|z| / sqrt(2)); e receives e^(-z^2 / 2).  Phi(-|z|)
// / e is a smooth function of t = 1 / (1 + 0.3 |z|), here t times a polynomial of degree
// 7, fitted to the least largest relative error over |z| <= 14 (beyond, e is 0): 1.7e-7.
// With its roundings and those of e the result is off by at most (22 + 1.5 z^2) 2^-24 of
// itself, so that GELU's small values at negative z keep their digits too.
__device__ __forceinline__ float normal_tail(float z, float& e) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, fabsf(z), 1.f));
  float p = fmaf(0.0356747732f, t, -0.157203063f);
  p = fmaf(p, t, 0.206353441f);
  p = fmaf(p, t, -0.0536835864f);
  p = fmaf(p, t, 0.128561601f);
  p = fmaf(p, t, 0.0999135002f);
  p = fmaf(p, t, 0.120753959f);
  p = fmaf(p, t, 0.119629301f);
  e = exp_fast(-0.5f * z * z);
  return p * t * e;
}
__device__ __forceinline__ float act_value(int act, float z) {
  if (act == OC_ACT_RELU) return z < 0.f ? 0.f : z;  // (NaN stays NaN)
  if (act == OC_ACT_SILU) return z * sigmoid(z);
  if (act == OC_ACT_GELU) {
    // z Phi(z) = max(z, 0) - |z| Phi(-|z|); the tail is 0 well before |z| = 16
    float e;
    return fmaf(-fminf(fabsf(z), 16.f), normal_tail(z, e), fmaxf(z, 0.f));
  }
  return z;
}
// d act'(z).  A ReLU's is a mask, as the convolutions' is: where z is not positive it is 0
// whatever d holds (an infinity times 0 would be NaN).
__device__ __forceinline__ float act_grad(int act, float d, float z) {
  if (act == OC_ACT_RELU) return z > 0.f ? d : 0.f;
  if (act == OC_ACT_SILU) {
    const float s = sigmoid(z);
    return d * (s * fmaf(z, 1.f - s, 1.f));
  }
  if (act == OC_ACT_GELU) {
    float e;
    const float q = normal_tail(z, e);
    return d * fmaf(z * e, 0.39894228040143268f, z < 0.f ? q : 1.f - q);
  }
  return d;
}

// Eight consecutive elements i .. i + 7 of an fp32 or bf16 array.
__device__ __forceinline__ void load8(const void* p, bool bf16, int64_t i, float (&v)[8]) {
  if (bf16) {
    const d_v4u u = *(const d_v4u_any*)((const uint16_t*)p + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = bf_up(u[k] & 0xffffu);
      v[2 * k + 1] = __builtin_bit_cast(float, u[k] & 0xffff0000u);
    }
  } else {
    const d_v4f a = *(const d_v4f_any*)((const float*)p + i);
    const d_v4f b = *(const d_v4f_any*)((const float*)p + i + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = a[k], v[4 + k] = b[k];
  }
}
__device__ __forceinline__ void store8(void* p, bool bf16, int64_t i, const float (&v)[8]) {
  if (bf16) {
    *(d_v4u_any*)((uint16_t*)p + i) = d_v4u{bf_pair(v[0], v[1]), bf_pair(v[2], v[3]),
                                            bf_pair(v[4], v[5]), bf_pair(v[6], v[7])};
  } else {
    *(d_v4f_any*)((float*)p + i) = d_v4f{v[0], v[1], v[2], v[3]};
    *(d_v4f_any*)((float*)p + i + 4) = d_v4f{v[4], v[5], v[6], v[7]};
  }
}
__device__ __forceinline__ float load1(const void* p, bool bf16, int64_t i) {
  return bf16 ? bf_up(((const uint16_t*)p)[i]) : ((const float*)p)[i];
}
__device__ __forceinline__ void store1(void* p, bool bf16, int64_t i, float v) {
  if (bf16)
    ((uint16_t*)p)[i] = (uint16_t)bf_pair(v, v);
  else
    ((float*)p)[i] = v;
}
// The first cnt (1..8) of them; the others read as zero.  n: elements in all.  What
// lies behind them in the array is read and dropped: one vector load, where eight
// loads under a mask each wait for the one before.
__device__ __forceinline__ void load8n(const void* p, bool bf16, int64_t i, int cnt, int64_t n,
                                       float (&v)[8]) {
  if (i + 8 <= n) {
    load8(p, bf16, i, v);
    if (cnt < 8) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = k < cnt ? v[k] : 0.f;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < cnt && i + k < n ? load1(p, bf16, i + k) : 0.f;
  }
}
// The first cnt of them; the others are not written.
__device__ __forceinline__ void store8n(void* p, bool bf16, int64_t i, int cnt,
                                        const float (&v)[8]) {
  if (cnt >= 8) {
    store8(p, bf16, i, v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < cnt) store1(p, bf16, i + k, v[k]);
  }
}

// The epilogue of U rows m[] (those below M), columns c .. c + 7 (those below e.n):
// z the sums and b0 the bias there; with GLU z and b0 are the gate's, u and b1 the
// other half's.  z and u are used up.
template <int U, bool GLU>
__device__ __forceinline__ void epilogue(const Epi& e, const int64_t (&m)[U], int64_t M, int c,
                                         const float (&b0)[8], const float (&b1)[8],
                                         float (&z)[U][8], float (&u)[U][8]) {
  const int cnt = e.n - c;
  float r[U][8];
  if (!GLU && e.res) {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (m[i] < M) load8n(e.res, e.y_bf16, m[i] * e.n + c, cnt, M * e.n, r[i]);
  }
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      z[i][k] += b0[k];
      if (GLU) u[i][k] += b1[k];
    }
  if (e.pre) {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (m[i] < M) {
        const int64_t at = m[i] * (GLU ? 2 : 1) * e.n + c;
        if (!GLU && e.pre_bits) {
          uint32_t bits = 0;
#pragma unroll
          for (int k = 0; k < 8; ++k) bits |= (z[i][k] > 0.f ? 1u : 0u) << k;
          ((uint8_t*)e.pre)[m[i] * ((e.n + 7) / 8) + c / 8] = (uint8_t)bits;
        } else {
          store8n(e.pre, false, at, cnt, z[i]);
          if (GLU) store8n(e.pre, false, at + e.n, cnt, u[i]);
        }
      }
  }
  if (e.act == OC_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) z[i][k] = act_value(OC_ACT_RELU, z[i][k]);
  } else if (e.act == OC_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) z[i][k] = act_value(OC_ACT_SILU, z[i][k]);
  } else if (e.act == OC_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) z[i][k] = act_value(OC_ACT_GELU, z[i][k]);
  }
  if (GLU) {
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) z[i][k] *= u[i][k];
  } else if (e.res) {
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) z[i][k] += r[i][k];
  }
#pragma unroll
  for (int i = 0; i < U; ++i)
    if (m[i] < M) store8n(e.y, e.y_bf16, m[i] * e.n + c, cnt, z[i]);
}

// Likewise for dz: u and z become its halves (without GLU, z becomes dz).
template <int ACT, int U, bool GLU>
__device__ __forceinline__ void slopes(const float (&d)[U][8], float (&z)[U][8], float (&u)[U][8]) {
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float g = z[i][k];
      z[i][k] = act_grad(ACT, GLU ? d[i][k] * u[i][k] : d[i][k], g);
      if (GLU) u[i][k] = d[i][k] * act_value(ACT, g);
    }
}
template <int U, bool GLU>
__device__ __forceinline__ void epilogue_dz(const Epi& e, const int64_t (&m)[U], int64_t M, int c,
                                            const float (&b0)[8], const float (&b1)[8],
                                            float (&z)[U][8], float (&u)[U][8], float (&s0)[8],
                                            float (&s1)[8]) {
  const int cnt = e.n - c;
  float d[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (m[i] < M) load8n(e.dy, e.y_bf16, m[i] * e.n + c, cnt, M * e.n, d[i]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      z[i][k] += b0[k];
      if (GLU) u[i][k] += b1[k];
    }
  }
  if (e.act == OC_ACT_NONE) slopes<OC_ACT_NONE, U, GLU>(d, z, u);
  else if (e.act == OC_ACT_RELU) slopes<OC_ACT_RELU, U, GLU>(d, z, u);
  else if (e.act == OC_ACT_SILU) slopes<OC_ACT_SILU, U, GLU>(d, z, u);
  else slopes<OC_ACT_GELU, U, GLU>(d, z, u);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (m[i] >= M) continue;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (k >= cnt) z[i][k] = u[i][k] = 0.f;  // (of columns that are not there)
      s0[k] += z[i][k];
      if (GLU) s1[k] += u[i][k];
    }
    if (GLU) {
      store8n(e.y, e.y_bf16, m[i] * e.ldz + c, cnt, z[i]);
      store8n(e.y, e.y_bf16, m[i] * e.ldz + e.n + c, cnt, u[i]);
      if (cnt <= 8)
        for (int64_t k = 2 * e.n; k < e.ldz; ++k) store1(e.y, e.y_bf16, m[i] * e.ldz + k, 0.f);
    } else {
      store8n(e.y, e.y_bf16, m[i] * e.ldz + c, (int)(e.ldz - c), z[i]);
    }
  }
}

}  // namespace oc
