// Dropout whose mask comes from a counter-based generator (oc_dropout_rng): y = keep ?
// x 2^32 / T : 0, the mask a function of the state {seed, step}, the site, the row and
// the column alone (rows.h), so that the backward forms it again instead of reading it.
#include <algorithm>

#include "rows.h"

namespace {

using oc::cdiv;
using oc::Drop;

constexpr int TB = 256;
constexpr int64_t MOST_BLOCKS = (int64_t)1 << 22;

// A thread has eight columns of a row.  d.on 0: a copy.
__global__ __launch_bounds__(TB) void k_drop_rng(Drop d, const void* x, bool bf16, int64_t rows,
                                                 int c, void* y) {
  const int nv = (c + 7) / 8;
  const int64_t groups = rows * nv, n = rows * c;
  const oc::DropKey key = d.on ? oc::drop_key(d) : oc::DropKey{};
  for (int64_t i = (int64_t)blockIdx.x * TB + threadIdx.x; i < groups;
       i += (int64_t)gridDim.x * TB) {
    const int64_t row = i / nv;
    const int col = (int)(i - row * nv) * 8;
    float v[8];
    oc::load8n(x, bf16, row * c + col, c - col, n, v);
    if (d.on) {
      bool k[8];
      oc::keep8(d, key, (uint64_t)i, k);
      oc::drop8(d, k, v);
    }
    oc::store8n(y, bf16, row * c + col, c - col, v);
  }
}

}  // namespace

extern "C" oc_status oc_dropout_rng(oc_dtype dt, int64_t rows, int32_t c, const void* x, double p,
                                    const uint64_t* rng, int32_t site, void* y, hipStream_t s) {
  const char* who = "oc_dropout_rng";
  OC_TRY(oc::check_rows(who, dt, rows, c));
  Drop drop;
  OC_TRY(oc::make_drop(who, p, rng, site, &drop));
  if (rows == 0) return OC_OK;
  if (!x || !y) return oc::fail(OC_ERR_ARG, "%s: NULL buffer", who);
  const size_t n = (size_t)rows * c * oc::value_bytes(dt);
  const oc::Span sp[] = {{"y", y, n, true, "x"},
                         {"x", x, n, false, nullptr},
                         {"rng", rng, drop.on ? (size_t)16 : 0, false, nullptr}};
  OC_TRY(oc::check_spans(who, sp));
  if (!drop.on && x == y) return OC_OK;
  const int64_t groups = rows * cdiv(c, 8);
  oc::launch_main(k_drop_rng, dim3((unsigned)std::min(cdiv(groups, TB), MOST_BLOCKS)), dim3(TB), s,
                  drop, x, dt == OC_BF16, rows, (int)c, y);
  OC_LAUNCH_CHECK();
  return OC_OK;
}
