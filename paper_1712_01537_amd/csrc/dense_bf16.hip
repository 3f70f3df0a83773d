// The dense layers' tile kernel for bf16 operands.
#include "dense_tile.h"

namespace {

template <int SHAPE, bool ARS, bool BRS, bool GLU, bool DIRECT, bool DZ>
void go(bool main, const oc::TileArgs& t, hipStream_t s) {
  constexpr oc::TileInfo i = oc::tile_info<uint16_t>(SHAPE);
  constexpr int WGM = i.threads / 64 / (i.bn / 64);
  const auto k = oc::k_dense_tile<uint16_t, i.bm, i.bn, WGM, i.bk, i.nb, ARS, BRS, GLU, DIRECT, DZ>;
  const dim3 grid((unsigned)(t.whole + t.classes * t.members));
  if (main) oc::launch_main(k, grid, dim3(i.threads), s, t);
  else oc::launch(k, grid, dim3(i.threads), 0, s, t);
}

template <int SHAPE, bool DIRECT>
void pick(bool a_rs, bool b_rs, bool main, const oc::TileArgs& t, hipStream_t s) {
  if (a_rs) go<SHAPE, true, true, false, DIRECT, false>(main, t, s);
  else if (!b_rs) go<SHAPE, false, false, false, DIRECT, false>(main, t, s);
  else if (t.epi.dy && t.epi.glu) go<SHAPE, false, true, true, DIRECT, true>(main, t, s);
  else if (t.epi.dy) go<SHAPE, false, true, false, DIRECT, true>(main, t, s);
  else if (t.epi.glu) go<SHAPE, false, true, true, DIRECT, false>(main, t, s);
  else go<SHAPE, false, true, false, DIRECT, false>(main, t, s);
}

template <int SHAPE, bool DIRECT>
void go2(const oc::TileArgs& dx, const oc::TileArgs& dw, bool swapped, hipStream_t s) {
  constexpr oc::TileInfo i = oc::tile_info<uint16_t>(SHAPE);
  constexpr int WGM = i.threads / 64 / (i.bn / 64);
  const unsigned n = dx.whole + dx.classes * dx.members, m = dw.whole + dw.classes * dw.members;
  oc::launch_main(oc::k_dense_tiles2<uint16_t, i.bm, i.bn, WGM, i.bk, i.nb, DIRECT>, dim3(n + m),
                  dim3(i.threads), s, dx, dw, (uint32_t)(swapped ? n : m), swapped);
}

}  // namespace

namespace oc {

void tile_bf16(int shape, bool a_rs, bool b_rs, bool direct, bool main, const TileArgs& t,
               hipStream_t s) {
  if (!direct) return pick<TILE_SMALL, false>(a_rs, b_rs, main, t, s);  // (the only one planned)
  switch (shape) {
    case TILE_LARGE: return pick<TILE_LARGE, true>(a_rs, b_rs, main, t, s);
    case TILE_TWO: return pick<TILE_TWO, true>(a_rs, b_rs, main, t, s);
    case TILE_MEDIUM: return pick<TILE_MEDIUM, true>(a_rs, b_rs, main, t, s);
    default: return pick<TILE_SMALL, true>(a_rs, b_rs, main, t, s);
  }
}

void tiles2_bf16(int shape, bool direct, const TileArgs& dx, const TileArgs& dw, bool swapped,
                 hipStream_t s) {
  if (!direct) return go2<TILE_SMALL, false>(dx, dw, swapped, s);
  switch (shape) {
    case TILE_LARGE: return go2<TILE_LARGE, true>(dx, dw, swapped, s);
    case TILE_MEDIUM: return go2<TILE_MEDIUM, true>(dx, dw, swapped, s);
    default: return go2<TILE_SMALL, true>(dx, dw, swapped, s);
  }
}

}  // namespace oc
