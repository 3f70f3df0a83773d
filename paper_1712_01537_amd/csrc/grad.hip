// The global norm of many gradient tensors and clipping by it.
//
//   norm = sqrt(sum over tensors and elements of g^2)
//   c = norm <= max_norm ? 1 : max_norm / norm,   out = c g
//
// A first pass reads every gradient once and leaves one sum of squares per
// workgroup; squares and sums are in double, so that no gradient's square
// overflows or vanishes and the sum of 10^9 of them keeps its digits.  The
// clipping pass's workgroups each add those sums (at most MOST_SUMS doubles, in
// the same order, hence the same norm everywhere) before they scale their
// share: no launch in between, no atomics.  Both passes are bound by memory:
// 4 (2) bytes a value read in the first, then read again and written.
//
// Tensors come as a table in the kernel's arguments (so that a captured call
// keeps its own copy), MOST_TENSORS a launch, cut into chunks of CHUNK elements
// of one tensor; a workgroup takes every gridDim.x-th chunk.  The clipping pass
// goes backwards, so that it finds what the first pass read last in the last-level
// cache.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "dense.h"

namespace {

using oc::cdiv;

constexpr int TB = 256, MOST_TENSORS = 128, MOST_SUMS = 2048, MOST_BLOCKS = 2048;
constexpr int CHUNK = TB * 8 * 4;  // four vectors of eight per thread

struct Table {
  const void* in[MOST_TENSORS];
  void* out[MOST_TENSORS];
  int64_t count[MOST_TENSORS];
  uint32_t first[MOST_TENSORS + 1];  // first chunk of each tensor, the number of chunks
  uint8_t in_bf16[MOST_TENSORS], out_bf16[MOST_TENSORS];
  int32_t n;
};
static_assert(sizeof(Table) + 64 <= 4096, "kernel arguments");

// The tensor that holds chunk k.
__device__ __forceinline__ int tensor_of(const Table& t, uint32_t k) {
  int lo = 0, hi = t.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.first[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
}

// f(v, element, count) for the vectors of eight of this thread in the block's chunks.
// Back: from the last chunk to the first.
template <bool BACK, typename Load, typename F>
__device__ __forceinline__ void for_chunks(const Table& t, Load&& load, F&& f) {
  const uint32_t total = t.first[t.n];
  for (uint32_t j = blockIdx.x; j < total; j += gridDim.x) {
    const uint32_t k = BACK ? total - 1 - j : j;
    const int i = tensor_of(t, k);
    const int64_t e0 = (int64_t)(k - t.first[i]) * CHUNK + threadIdx.x * 8, n = t.count[i];
    float v[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j) load(i, e0 + j * TB * 8, n, v[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) f(i, e0 + j * TB * 8, n, v[j]);
  }
}

__device__ __forceinline__ void load_in(const Table& t, int i, int64_t e, int64_t n, float (&v)[8]) {
  const int cnt = (int)(n - e < 8 ? n - e : 8);
  if (cnt > 0) {
    oc::load8n(t.in[i], t.in_bf16[i], e, cnt, n, v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 0.f;
  }
}

// The sum of the block's threads' values, in every thread: a fixed tree.
__device__ __forceinline__ double block_sum(double a) {
  __shared__ double red[TB];
  red[threadIdx.x] = a;
  __syncthreads();
  for (int h = TB / 2; h > 0; h >>= 1) {
    if ((int)threadIdx.x < h) red[threadIdx.x] += red[threadIdx.x + h];
    __syncthreads();
  }
  return red[0];
}

__global__ __launch_bounds__(TB) void k_sq_sum(Table t, double* part) {
  double a[8] = {};
  for_chunks<false>(
      t, [&](int i, int64_t e, int64_t n, float(&v)[8]) { load_in(t, i, e, n, v); },
      [&](int, int64_t, int64_t, float(&v)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) a[k] = fma((double)v[k], (double)v[k], a[k]);
      });
  const double s = block_sum(((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7])));
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The sum of the n partial sums (of this block's threads, each every TB-th).
__device__ __forceinline__ double total_of(const double* part, int n) {
  double a = 0.0;
  for (int i = threadIdx.x; i < n; i += TB) a += part[i];
  return block_sum(a);
}

__global__ __launch_bounds__(TB) void k_sq_total(const double* part, int n, double* total,
                                                 float* norm) {
  const double s = total_of(part, n);
  if (threadIdx.x != 0) return;
  if (total) *total = s;
  if (norm) *norm = (float)sqrt(s);
}

__global__ __launch_bounds__(TB) void k_clip(Table t, const double* part, int n, double max_norm,
                                             float* norm) {
  const double r = sqrt(total_of(part, n));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)r;
  // The factor as c 2^e, 0.5 <= c < 1 (or 1, 0, NaN): one below fp32's normal numbers (a
  // norm of 10^37 clipped to 0.1) would have few bits or none as an fp32 value.
  const bool within = r <= max_norm;
  const double factor = max_norm / r;
  const int e2 = within ? 0 : __builtin_amdgcn_frexp_exp(factor);
  const float c = within ? 1.f : (float)__builtin_amdgcn_frexp_mant(factor);
  for_chunks<true>(
      t,
      [&](int i, int64_t e, int64_t cnt, float(&v)[8]) {
        // nothing changes: gradients scaled in place by one
        if (within && t.in[i] == t.out[i]) return;
        load_in(t, i, e, cnt, v);
      },
      [&](int i, int64_t e, int64_t cnt, float(&v)[8]) {
        if ((within && t.in[i] == t.out[i]) || e >= cnt) return;
        if (!within) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = __builtin_amdgcn_ldexpf(v[k] * c, e2);
        }
        oc::store8n(t.out[i], t.out_bf16[i], e, (int)(cnt - e < 8 ? cnt - e : 8), v);
      });
}

// Chunks of tensors i0 .. i0 + MOST_TENSORS - 1 (or to n), and the workgroups they get.
int64_t chunks_of(int32_t i0, int32_t n, const int64_t* counts) {
  int64_t c = 0;
  for (int32_t i = i0; i < n && i < i0 + MOST_TENSORS; ++i) c += cdiv(counts[i], CHUNK);
  return c;
}
int blocks_of(int64_t chunks) { return (int)std::min<int64_t>(chunks, MOST_BLOCKS); }

int64_t sums_of(int32_t n, const int64_t* counts) {
  int64_t s = 0;
  for (int32_t i = 0; i < n; i += MOST_TENSORS) s += blocks_of(chunks_of(i, n, counts));
  return s;
}

oc_status check_list(const char* who, int32_t n, const void* const* grads, const oc_dtype* dts,
                     const int64_t* counts) {
  if (n < 0 || (n > 0 && (!grads || !dts || !counts)))
    return oc::fail(OC_ERR_ARG, "%s: %d tensors", who, n);
  for (int32_t i = 0; i < n; ++i) {
    if (dts[i] != OC_F32 && dts[i] != OC_BF16)
      return oc::fail(OC_ERR_ARG, "%s: tensor %d has dtype %d", who, i, (int)dts[i]);
    if (counts[i] < 0 || counts[i] > (int64_t)1 << 40 || (counts[i] > 0 && !grads[i]))
      return oc::fail(OC_ERR_ARG, "%s: tensor %d is NULL or has a bad count", who, i);
  }
  for (int32_t i = 0; i < n; i += MOST_TENSORS)
    if (chunks_of(i, n, counts) > (int64_t)0x7fffffff)  // (indices step on by gridDim.x)
      return oc::fail(OC_ERR_ARG, "%s: too many values", who);
  return OC_OK;
}

template <typename F>
void for_tables(int32_t n, const void* const* grads, const oc_dtype* dts, const int64_t* counts,
                void* const* outs, const oc_dtype* out_dts, F&& f) {
  for (int32_t i0 = 0; i0 < n; i0 += MOST_TENSORS) {
    Table t{};
    int64_t chunks = 0;
    for (int32_t i = i0; i < n && i < i0 + MOST_TENSORS; ++i) {
      if (counts[i] == 0) continue;
      const int k = t.n++;
      t.in[k] = grads[i];
      t.in_bf16[k] = dts[i] == OC_BF16;
      t.out[k] = outs ? outs[i] : nullptr;
      t.out_bf16[k] = out_dts && out_dts[i] == OC_BF16;
      t.count[k] = counts[i];
      t.first[k] = (uint32_t)chunks;
      chunks += cdiv(counts[i], CHUNK);
    }
    t.first[t.n] = (uint32_t)chunks;
    if (t.n > 0) f(t, blocks_of(chunks));
  }
}

// One sum of squares per workgroup in part; their number.
int sq_sums(int32_t n, const void* const* grads, const oc_dtype* dts, const int64_t* counts,
            double* part, hipStream_t s) {
  int at = 0;
  for_tables(n, grads, dts, counts, nullptr, nullptr, [&](const Table& t, int blocks) {
    oc::launch(k_sq_sum, dim3(blocks), dim3(TB), 0, s, t, part + at);
    at += blocks;
  });
  return at;
}

// Every output apart from the other outputs and from every gradient, but for its own as a
// whole: a workgroup would read what another has written, or both would write.
oc_status check_outputs(int32_t n, const void* const* grads, const oc_dtype* dts,
                        const int64_t* counts, void* const* outs, const oc_dtype* out_dts) {
  struct Span {
    uintptr_t from, to;
    int32_t i;
  };
  const auto span = [&](const void* p, oc_dtype t, int32_t i) {
    return Span{(uintptr_t)p, (uintptr_t)p + (uintptr_t)counts[i] * (t == OC_BF16 ? 2 : 4), i};
  };
  const auto before = [](const Span& a, const Span& b) { return a.from < b.from; };
  const std::unique_ptr<Span[]> all(new (std::nothrow) Span[n > 0 ? n : 1]);
  if (!all) return oc::fail(OC_ERR_NOMEM, "oc_grad_clip: %d tensors", n);
  Span *const first = all.get(), *last = first;
  for (int32_t i = 0; i < n; ++i)
    if (counts[i] > 0) *last++ = span(outs[i], out_dts[i], i);
  if (!std::is_sorted(first, last, before)) std::sort(first, last, before);
  for (const Span* s = first; s + 1 < last; ++s)
    if (s[1].from < s->to)
      return oc::fail(OC_ERR_ARG, "oc_grad_clip: outputs %d and %d overlap", s->i, s[1].i);
  for (int32_t i = 0; i < n; ++i) {
    if (counts[i] == 0 || outs[i] == grads[i]) continue;
    const Span g = span(grads[i], dts[i], i);
    // the first output that ends behind the gradient's start (they are apart and in order)
    const Span* s = std::partition_point(first, last, [&](const Span& o) { return o.to <= g.from; });
    if (s < last && s->from < g.to)
      return oc::fail(OC_ERR_ARG, "oc_grad_clip: output %d overlaps gradient %d", s->i, i);
  }
  return OC_OK;
}

oc_status check_ws(const char* who, int32_t n, const int64_t* counts, const void* ws,
                   size_t have) {
  const size_t need = oc_grad_workspace(n, counts);
  if (!ws || have < need)
    return oc::fail(OC_ERR_ARG, "%s: workspace %zu bytes < %zu", who, ws ? have : 0, need);
  if ((uintptr_t)ws % 8)
    return oc::fail(OC_ERR_ARG, "%s: the workspace is not 8-byte aligned", who);
  return OC_OK;
}

}  // namespace

extern "C" {

size_t oc_grad_workspace(int32_t n, const int64_t* counts) {
  if (n < 0 || (n > 0 && !counts)) return 0;
  for (int32_t i = 0; i < n; ++i)
    if (counts[i] < 0) return 0;
  return oc::align256((size_t)(sums_of(n, counts) + 1) * sizeof(double));
}

oc_status oc_grad_norm(int32_t n, const void* const* grads, const oc_dtype* dts,
                       const int64_t* counts, float* norm, void* ws, size_t ws_bytes,
                       hipStream_t s) {
  oc_status st = check_list("oc_grad_norm", n, grads, dts, counts);
  if (st != OC_OK) return st;
  if (!norm) return oc::fail(OC_ERR_ARG, "oc_grad_norm: NULL buffer");
  st = check_ws("oc_grad_norm", n, counts, ws, ws_bytes);
  if (st != OC_OK) return st;
  double* part = (double*)ws;
  const int sums = sq_sums(n, grads, dts, counts, part, s);
  oc::launch(k_sq_total, dim3(1), dim3(TB), 0, s, (const double*)part, sums, (double*)nullptr,
             norm);
  OC_LAUNCH_CHECK();
  return OC_OK;
}

oc_status oc_grad_clip(int32_t n, const void* const* grads, const oc_dtype* dts,
                       const int64_t* counts, double max_norm, void* const* outs,
                       const oc_dtype* out_dts, float* norm, void* ws, size_t ws_bytes,
                       hipStream_t s) {
  oc_status st = check_list("oc_grad_clip", n, grads, dts, counts);
  if (st != OC_OK) return st;
  if (!(max_norm >= 0.0))
    return oc::fail(OC_ERR_ARG, "oc_grad_clip: max_norm must not be negative or NaN");
  if (n > 0 && (!outs || !out_dts)) return oc::fail(OC_ERR_ARG, "oc_grad_clip: NULL outputs");
  for (int32_t i = 0; i < n; ++i) {
    if (counts[i] > 0 && !outs[i])
      return oc::fail(OC_ERR_ARG, "oc_grad_clip: output %d is NULL", i);
    if (out_dts[i] != OC_F32 && out_dts[i] != dts[i])
      return oc::fail(OC_ERR_ARG, "oc_grad_clip: output %d has dtype %d", i, (int)out_dts[i]);
    if (counts[i] > 0 && outs[i] == grads[i] && out_dts[i] != dts[i])
      return oc::fail(OC_ERR_ARG, "oc_grad_clip: output %d is its gradient in another type", i);
  }
  st = check_outputs(n, grads, dts, counts, outs, out_dts);
  if (st != OC_OK) return st;
  st = check_ws("oc_grad_clip", n, counts, ws, ws_bytes);
  if (st != OC_OK) return st;
  double* part = (double*)ws;
  int sums = sq_sums(n, grads, dts, counts, part, s);
  if (sums == 0 || sums > MOST_SUMS) {
    oc::launch(k_sq_total, dim3(1), dim3(TB), 0, s, (const double*)part, sums, part + sums,
               sums == 0 ? norm : (float*)nullptr);
    part += sums;
    sums = 1;
  }
  for_tables(n, grads, dts, counts, outs, out_dts, [&](const Table& t, int blocks) {
    oc::launch_main(k_clip, dim3(blocks), dim3(TB), s, t, (const double*)part, sums, max_norm,
                    norm);
    norm = nullptr;  // written once
  });
  OC_LAUNCH_CHECK();
  return OC_OK;
}

}  // extern "C"
