// The dense layers' tile kernel for fp32 operands.
#include "dense_tile.h"

namespace {

template <int SHAPE, bool ARS, bool BRS, bool GLU, bool DZ>
void go(bool main, const oc::TileArgs& t, hipStream_t s) {
  constexpr oc::TileInfo i = oc::tile_info<float>(SHAPE);
  constexpr int WGM = i.threads / 64 / (i.bn / 64);
  const auto k = oc::k_dense_tile<float, i.bm, i.bn, WGM, i.bk, i.nb, ARS, BRS, GLU, false, DZ>;
  const dim3 grid((unsigned)(t.whole + t.classes * t.members));
  if (main) oc::launch_main(k, grid, dim3(i.threads), s, t);
  else oc::launch(k, grid, dim3(i.threads), 0, s, t);
}

template <int SHAPE>
void pick(bool a_rs, bool b_rs, bool main, const oc::TileArgs& t, hipStream_t s) {
  if (a_rs) go<SHAPE, true, true, false, false>(main, t, s);
  else if (!b_rs) go<SHAPE, false, false, false, false>(main, t, s);
  else if (t.epi.dy && t.epi.glu) go<SHAPE, false, true, true, true>(main, t, s);
  else if (t.epi.dy) go<SHAPE, false, true, false, true>(main, t, s);
  else if (t.epi.glu) go<SHAPE, false, true, true, false>(main, t, s);
  else go<SHAPE, false, true, false, false>(main, t, s);
}

template <int SHAPE>
void go2(const oc::TileArgs& dx, const oc::TileArgs& dw, bool swapped, hipStream_t s) {
  constexpr oc::TileInfo i = oc::tile_info<float>(SHAPE);
  constexpr int WGM = i.threads / 64 / (i.bn / 64);
  const unsigned n = dx.whole + dx.classes * dx.members, m = dw.whole + dw.classes * dw.members;
  oc::launch_main(oc::k_dense_tiles2<float, i.bm, i.bn, WGM, i.bk, i.nb, false>, dim3(n + m),
                  dim3(i.threads), s, dx, dw, (uint32_t)(swapped ? n : m), swapped);
}

}  // namespace

namespace oc {

void tile_f32(int shape, bool a_rs, bool b_rs, bool main, const TileArgs& t, hipStream_t s) {
  switch (shape) {
    case TILE_LARGE: return pick<TILE_LARGE>(a_rs, b_rs, main, t, s);
    case TILE_TWO: return pick<TILE_TWO>(a_rs, b_rs, main, t, s);
    case TILE_MEDIUM: return pick<TILE_MEDIUM>(a_rs, b_rs, main, t, s);
    default: return pick<TILE_SMALL>(a_rs, b_rs, main, t, s);
  }
}

void tiles2_f32(int shape, const TileArgs& dx, const TileArgs& dw, bool swapped, hipStream_t s) {
  switch (shape) {
    case TILE_LARGE: return go2<TILE_LARGE>(dx, dw, swapped, s);
    case TILE_TWO: return go2<TILE_TWO>(dx, dw, swapped, s);
    case TILE_MEDIUM: return go2<TILE_MEDIUM>(dx, dw, swapped, s);
    default: return go2<TILE_SMALL>(dx, dw, swapped, s);
  }
}

}  // namespace oc
