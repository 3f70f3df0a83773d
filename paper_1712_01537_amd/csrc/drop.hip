// Dropout whose mask comes from a counter-based generator (oc_dropout_rng): y = keep ?
// x 2^32 / T : 0, the mask a function of the state {seed, step}, the site, the row and
// the column alone (rows.h), so that the backward forms it again instead of reading it.
// Bound by memory: 65536 x 4096 bf16 182 to 187 us (5.7 to 5.9 TB/s read and written), with
// one pair of buffers or six in turn (6 GiB, past the last-level cache), 211 in the first
// calls of a run; p = 0.1 as 0.5; 134 vector instructions for the 512 values of a wave.
#include <algorithm>

#include "rows.h"

namespace {

using oc::cdiv;
using oc::Drop;

constexpr int TB = 256;
constexpr int64_t MOST_BLOCKS = (int64_t)1 << 22;

// A thread has eight columns of a row.  d.on 0: a copy.  WHOLE: c is a multiple of eight,
// so that group i is elements 8 i on and no row has to be known.
template <bool BF, bool WHOLE>
__global__ __launch_bounds__(TB) void k_drop_rng(Drop d, const void* x, int64_t rows, int c,
                                                 void* y) {
  const int nv = (c + 7) / 8;
  const int64_t groups = rows * nv, n = rows * c;
  const oc::DropKey key = d.on ? oc::drop_key(d) : oc::DropKey{};
  for (int64_t i = (int64_t)blockIdx.x * TB + threadIdx.x; i < groups;
       i += (int64_t)gridDim.x * TB) {
    int64_t at = i * 8;
    int cnt = 8;
    if (!WHOLE) {
      const int64_t row =
          groups <= 0xffffffffll ? (int64_t)((uint32_t)i / (uint32_t)nv) : i / nv;
      const int col = (int)(i - row * nv) * 8;
      at = row * c + col;
      cnt = c - col;
    }
    float v[8];
    if (WHOLE)
      oc::load8(x, BF, at, v);
    else
      oc::load8n(x, BF, at, cnt, n, v);
    if (d.on) {
      bool k[8];
      oc::keep8(d, key, (uint64_t)i, k);
      oc::drop8(d, k, v);
    }
    if (WHOLE)
      oc::store8(y, BF, at, v);
    else
      oc::store8n(y, BF, at, cnt, v);
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
  const auto go = [&](auto kernel) {
    oc::launch_main(kernel, dim3((unsigned)std::min(cdiv(groups, TB), MOST_BLOCKS)), dim3(TB), s,
                    drop, x, rows, (int)c, y);
  };
  if (c % 8 == 0)
    dt == OC_BF16 ? go(k_drop_rng<true, true>) : go(k_drop_rng<false, true>);
  else
    dt == OC_BF16 ? go(k_drop_rng<true, false>) : go(k_drop_rng<false, false>);
  OC_LAUNCH_CHECK();
  return OC_OK;
}
