// Shared by the row operators (oc_ln_*, oc_dropout_rng, oc_drop_ln_*, oc_embed_*):
// the dropout mask, sums over the threads of a row, and checks of buffers.
#pragma once

#include <cmath>
#include <cstring>

#include "dense.h"

namespace oc {

// --- the dropout mask ---------------------------------------------------------

// a ^ b ^ c, one instruction.
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
  return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1,
// 2, 3", SC 2011): ten rounds of two 32 x 32 -> 64 bit products on a counter of four
// words under a key of two.
__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
    c[0] = xor3((uint32_t)(b >> 32), c[1], k0);
    c[2] = xor3((uint32_t)(a >> 32), c[3], k1);
    c[1] = (uint32_t)b;
    c[3] = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// A dropout call: a value is kept where its 32-bit number is below T = hi 2^16 + lo.
struct Drop {
  const uint64_t* rng;  // dev {seed, step}
  uint32_t hi, lo, site;
  float scale;
  int on;  // 0: everything is kept
};
struct DropKey {
  uint32_t k0, k1, c2, c3;
};
__device__ __forceinline__ DropKey drop_key(const Drop& d) {
  const uint64_t seed = d.rng[0], step = d.rng[1];
  return DropKey{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)step, (uint32_t)(step >> 32)};
}
// Which of the eight values of group `index` are kept.  One call of the generator gives
// the high halves of eight numbers, which decide all but one value in 65536; the low
// halves, from a second call, are formed only where a high half equals T's (16384 x 4096
// bf16 values in the last-level cache 39.0 us, with both calls always 42.2; from memory
// 208 either way).
__device__ __forceinline__ void keep8(const Drop& d, const DropKey& key, uint64_t index,
                                      bool (&k)[8]) {
  const uint32_t c1 = (uint32_t)(index >> 32) | d.site << 16;
  uint32_t w[4] = {(uint32_t)index, c1, key.c2, key.c3};
  philox(w, key.k0, key.k1);
  bool tie = false;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t half = j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu;
    k[j] = half < d.hi;
    tie |= half == d.hi;
  }
  if (tie && d.lo != 0) {
    uint32_t v[4] = {(uint32_t)index, c1 | 1u << 31, key.c2, key.c3};
    philox(v, key.k0, key.k1);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t half = j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu;
      const uint32_t low = j & 1 ? v[j >> 1] >> 16 : v[j >> 1] & 0xffffu;
      k[j] = k[j] || (half == d.hi && low < d.lo);
    }
  }
}
__device__ __forceinline__ void drop8(const Drop& d, const bool (&k)[8], float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = k[j] ? v[j] * d.scale : 0.f;
}

// --- eight values of a row ---------------------------------------------------------

// Eight values as they lie in memory, so that a load can be in flight while the row
// before is worked on.
template <bool BF>
struct Raw;
template <>
struct Raw<true> {
  d_v4u u;
};
template <>
struct Raw<false> {
  d_v4f a, b;
};
// A lane's number of values, behind the compiler's back: it would form the eight
// comparisons with it in front of the loop over the rows and keep them there in 16 scalar
// registers, which it then has to save and fetch.
__device__ __forceinline__ int hidden(int cnt) {
  asm("" : "+v"(cnt));
  return cnt;
}
// Zeros behind the row's end, in the lanes that have it.
__device__ __forceinline__ void cut(float (&v)[8], int cnt) {
  if (cnt < 8) {
    const int q = hidden(cnt);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < q ? v[k] : 0.f;
  }
}

// A row's place in an array: where a wave has one row (all but the shortest), the row's
// start is the same for its lanes and a lane's own part 32 bits.
struct Place {
  int64_t at;  // the row's first element
  int col, cnt;
  int64_t left;  // elements from there to the array's end
};
__device__ __forceinline__ void raw_load(Raw<true>& r, const void* p, const Place& w) {
  const uint16_t* q = (const uint16_t*)p + w.at;
  if (w.cnt >= 8 || w.col + 8 <= w.left) {
    r.u = *(const d_v4u_any*)(q + (uint32_t)w.col);
  } else {
    const int c = hidden(w.cnt);
    uint32_t h[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = k < c ? q[w.col + k] : 0;
    r.u = d_v4u{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
  }
}
__device__ __forceinline__ void raw_load(Raw<false>& r, const void* p, const Place& w) {
  const float* q = (const float*)p + w.at;
  if (w.cnt >= 8 || w.col + 8 <= w.left) {
    r.a = *(const d_v4f_any*)(q + (uint32_t)w.col);
    r.b = *(const d_v4f_any*)(q + (uint32_t)w.col + 4);
  } else {
    const int c = hidden(w.cnt);
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < c ? q[w.col + k] : 0.f;
    r.a = d_v4f{v[0], v[1], v[2], v[3]};
    r.b = d_v4f{v[4], v[5], v[6], v[7]};
  }
}
template <bool BF>
__device__ __forceinline__ void row_store(void* p, const Place& w, const float (&v)[8]) {
  void* q = BF ? (void*)((uint16_t*)p + w.at) : (void*)((float*)p + w.at);
  if (w.cnt >= 8)
    store8(q, BF, (uint32_t)w.col, v);
  else
    store8n(q, BF, (uint32_t)w.col, hidden(w.cnt), v);
}
__device__ __forceinline__ void unpack(const Raw<true>& r, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = bf_up(r.u[k] & 0xffffu);
    v[2 * k + 1] = __builtin_bit_cast(float, r.u[k] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const Raw<false>& r, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = r.a[k], v[4 + k] = r.b[k];
}

// --- the call's arguments ------------------------------------------------------------

// Host: the call's Drop, or why not.
inline oc_status make_drop(const char* who, double p, const uint64_t* rng, int32_t site,
                           Drop* out) {
  if (!(p >= 0.0 && p < 1.0)) return fail(OC_ERR_ARG, "%s: ratio %g not in [0, 1)", who, p);
  if (site < 0 || site > 32767) return fail(OC_ERR_ARG, "%s: site %d not in 0..32767", who, site);
  const uint64_t t = (uint64_t)std::nearbyint((1.0 - p) * 4294967296.0);
  if (t == 0) return fail(OC_ERR_ARG, "%s: a ratio of %g keeps nothing", who, p);
  *out = Drop{rng, (uint32_t)(t >> 16), (uint32_t)(t & 0xffffu), (uint32_t)site,
              (float)(4294967296.0 / (double)t), t < ((uint64_t)1 << 32)};
  if (out->on && !rng) return fail(OC_ERR_ARG, "%s: NULL generator state", who);
  if (out->on && (uintptr_t)rng % 8)
    return fail(OC_ERR_ARG, "%s: the generator state is not 8-byte aligned", who);
  return OC_OK;
}

// --- buffers ---------------------------------------------------------------------

// A call's buffers, for the check that no output overlaps another buffer; one of those
// named `same` may be an output's as a whole (each value is read before it is written).
struct Span {
  const char* name;
  const void* p;
  size_t bytes;
  bool out;
  const char* same;
};
template <int N>
inline oc_status check_spans(const char* who, const Span (&s)[N]) {
  for (int i = 0; i < N; ++i) {
    if (!s[i].p || !s[i].bytes || !s[i].out) continue;
    for (int j = 0; j < N; ++j) {
      if (j == i || !s[j].p || !s[j].bytes || (s[j].out && j < i)) continue;
      const uintptr_t a = (uintptr_t)s[i].p, b = (uintptr_t)s[j].p;
      if (a >= b + s[j].bytes || b >= a + s[i].bytes) continue;
      if (a == b && s[i].bytes == s[j].bytes && s[i].same && !std::strcmp(s[i].same, s[j].name))
        continue;
      return fail(OC_ERR_ARG, "%s: %s overlaps %s", who, s[i].name, s[j].name);
    }
  }
  return OC_OK;
}

inline oc_status check_row_ws(const char* who, const void* ws, size_t have, size_t need) {
  if (need && (!ws || have < need))
    return fail(OC_ERR_ARG, "%s: workspace %zu bytes < %zu", who, ws ? have : 0, need);
  if (need && (uintptr_t)ws % 16)
    return fail(OC_ERR_ARG, "%s: the workspace is not 16-byte aligned", who);
  return OC_OK;
}

constexpr int64_t ROWS_MOST = (int64_t)1 << 28;
constexpr int32_t COLS_MOST = 1 << 16;
inline oc_status check_rows(const char* who, oc_dtype dt, int64_t rows, int32_t c) {
  if (dt != OC_F32 && dt != OC_BF16) return fail(OC_ERR_ARG, "%s: dtype %d", who, (int)dt);
  if (rows < 0 || rows >= ROWS_MOST || c < 1 || c > COLS_MOST)
    return fail(OC_ERR_ARG, "%s: %lld rows of %d channels", who, (long long)rows, c);
  if (rows * c >= (int64_t)1 << 40)
    return fail(OC_ERR_UNSUPPORTED, "%s: %lld rows of %d channels are too many", who,
                (long long)rows, c);
  return OC_OK;
}
inline size_t value_bytes(oc_dtype dt) { return dt == OC_BF16 ? 2 : 4; }
#define OC_TRY(call)                    \
  do {                                  \
    const oc_status s_ = (call);        \
    if (s_ != OC_OK) return s_;         \
  } while (0)

}  // namespace oc
