"""GPU parity of the row operators with the float64 oracle: layer norm, dropout
from a counter, the residual step, table rows, and all of them run together.

Tolerances.  u = 2^-24 is fp32's rounding, v the output type's (2^-8 for bf16,
0 beside u for fp32).  A sum over a row of c channels passes through at most A =
max(96, c / 256 + 16) additions (a thread's own, then the lanes' and waves'), each of
which rounds a partial sum of magnitudes by at most u; sums over rows pass
through at most 64 in fp32, are rounded once as a block's and once at the end
(66 u of the sum of magnitudes).

  z = (x - m - delta) r:  the mean's rounding is in delta, so its error is that
      of the mean of the deviations, A u of a mean |x - m| <= 1 / r; r's relative
      error is half the sum of squares' (A / 2 u) and some 6 roundings of its own.
      |z error| <= u ((A / 2 + 10) |z| + A + 4)
  y = z gamma + beta: |gamma| times that, and a rounding of each of the two
  dx = r (g - mean g - z mean(g z)): every term's error is at most (2 A + 20) u
      of the term with its sums taken over magnitudes.
"""
import numpy as np
import pytest
import torch

import paper_1712_01537_amd as oc
from oracle import rows as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
DT = pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])


def v_of(dt):
    return 2.0 ** -8 if dt == BF16 else U


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def make(shape, dt, seed, scale=1.0, shift=0):
    """N(0, scale^2) values, `shift` elements into their buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = int(np.prod(shape))
    buf = torch.empty(n + shift, device="cuda").normal_(generator=g).mul_(scale).to(dt)
    return buf[shift:shift + n].view(shape)


def near(got, want, tol, what):
    err = np.abs(_np(got) - want)
    bad = ~(err <= tol)  # (a NaN is bad)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, err - tol, -1)), err.shape)
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} off; at {i} got "
                             f"{_np(got)[i]!r}, want {want[i]!r} within {np.broadcast_to(tol, err.shape)[i]!r}")


def adds(h):
    return max(96, h.shape[1] // 256 + 16)


def z_tol(z):
    a = adds(z)
    return U * ((a / 2 + 10) * np.abs(z) + a + 4)


def check_y(y, h, gamma, beta, eps, dt, what, extra=0.0):
    """extra: how far z may be off by errors of h."""
    want, mean, r = R.ln_fwd(h, gamma, beta, eps)
    z = (h - mean[:, None]) * r[:, None]
    g = 1.0 if gamma is None else np.abs(gamma)
    tol = (z_tol(z) + extra) * g + U * (np.abs(z) * g + np.abs(want)) + v_of(dt) * np.abs(want)
    near(y, want, tol * 1.01 + 1e-38, what)
    return mean, r


def check_stats(mean, invstd, h, eps, what, err=0.0):
    m, r = R.stats(h, eps)
    dev = np.abs(h - m[:, None]).mean(1)
    near(mean, m, U * (2 * np.abs(m) + adds(h) * dev) + err + 1e-38, what + " mean")
    near(invstd, r, r * (U * (adds(h) / 2 + 8) + err * r), what + " invstd")


def check_bwd(h, dy, dh, gamma, invstd, dt, got, what, keep=None, q=1.0, herr=None):
    """got: dx behind dropout (or None), dres, dgamma, dbeta; invstd as read; herr: how far
    the values of h may be off that the kernel forms."""
    dx, dres, dg, db = got
    want, wg, wb = R.ln_bwd(h, dy, gamma, invstd)
    r = invstd[:, None]
    z = (h - h.mean(1, keepdims=True)) * r
    g = dy if gamma is None else dy * gamma
    mags = np.abs(g) + np.abs(g).mean(1, keepdims=True) + (1 + np.abs(z)) * (
        np.abs(g) * (1 + np.abs(z))).mean(1, keepdims=True)
    # a z off by e changes z mean(g z) by (e mean |g z| + |z| mean |g| e)
    ze = 0.0 if herr is None else r * 2 * herr.max(1, keepdims=True)
    tol = r * ((2 * adds(h) + 20) * U * mags + ze * (1 + np.abs(z)) * (
        np.abs(g) * (1 + np.abs(z))).mean(1, keepdims=True))
    if dh is not None:
        want = want + dh
        tol = tol + U * np.abs(want)
    if dres is not None:
        near(dres, want, 1.01 * (tol + v_of(dt) * np.abs(want)) + 1e-38, what + " dres")
    if dx is not None:
        w = want if keep is None else np.where(keep, want / q, 0.0)
        t = tol / q + (3 * U + v_of(dt)) * np.abs(w)
        near(dx, w, 1.01 * t + 1e-38, what + " dx")
        if keep is not None:
            assert (_np(dx)[~keep] == 0).all(), what
    if dg is not None:
        near(dg, wg, 1.01 * (np.abs(dy) * (z_tol(z) + ze + 68 * U * np.abs(z))).sum(0) + 1e-38,
             what + " dgamma")
    if db is not None:
        near(db, wb, 67 * U * np.abs(dy).sum(0) + 1e-38, what + " dbeta")


# one channel, one row, widths around every vector and lane count, many rows, long rows
SHAPES = [(1, 1), (5, 1), (3, 2), (7, 7), (1000, 3), (65, 8), (33, 9), (130, 15), (4, 16),
          (1, 63), (300, 64), (77, 65), (1, 127), (9000, 24), (35, 128), (50, 257), (3, 511),
          (64, 512), (17, 513), (129, 1000), (1, 1024), (6, 1025), (40, 2047), (3, 2048),
          (2, 2049), (70, 4096), (9, 5000), (2, 8192), (3, 8200), (1, 16384), (2, 16385), (4, 20001), (1, 65536)]


@DT
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_ln(i, dt):
    rows, c = SHAPES[i]
    print(f"[ln] {rows} x {c} {dt}", flush=True)
    shift = i % 4
    x = make((rows, c), dt, i, 3.0, shift)
    x += make((rows, 1), dt, i + 50, 5.0)
    dy = make((rows, c), dt, i + 100, 1.0, (i + 1) % 3)
    affine = i % 3 != 2
    gamma = make((c,), F32, i + 200, 1.0, i % 2) if affine else None
    beta = make((c,), F32, i + 300) if affine and i % 2 else None
    eps = 1e-5 if i % 2 else 0.5
    y, mean, invstd = oc.oc_ln_fwd(x, gamma, beta, eps, need_stats=True)
    check_y(y, _np(x), _np(gamma), _np(beta), eps, dt, "y")
    check_stats(mean, invstd, _np(x), eps, "stats")
    assert torch.equal(oc.oc_ln_fwd(x, gamma, beta, eps)[0], y)
    dx, dg, db = oc.oc_ln_bwd(x, dy, gamma, mean, invstd)
    check_bwd(_np(x), _np(dy), None, _np(gamma), _np(invstd), dt, (None, dx, dg, db), "bwd")
    one = oc.oc_ln_bwd(x, dy, gamma, mean, invstd, need_dgamma=False, need_dbeta=False)
    assert torch.equal(one[0], dx) and one[1] is None and one[2] is None
    two = oc.oc_ln_bwd(x, dy, gamma, mean, invstd, need_dx=False, need_dbeta=False)
    assert two[0] is None and torch.equal(two[1], dg)


@DT
@pytest.mark.parametrize("c", [17, 1024, 4096])
def test_ln_means_far_from_zero(c, dt):
    """A mean 4096 (fp32) or 64 (bf16, whose values are then multiples of 1/4) times
    the deviations costs no digits of y or of the gradients."""
    far = 4096.0 if dt == F32 else 64.0
    x = (make((50, c), F32, c) + far).to(dt)
    dy = make((50, c), dt, c + 1)
    y, mean, invstd = oc.oc_ln_fwd(x, None, None, 1e-5, need_stats=True)
    check_y(y, _np(x), None, None, 1e-5, dt, "y")
    check_bwd(_np(x), _np(dy), None, None, _np(invstd), dt,
              (None, *oc.oc_ln_bwd(x, dy, None, mean, invstd)), "bwd")


@DT
@pytest.mark.parametrize("c", [5, 64, 1000, 4097])
def test_ln_constant_rows_are_beta(c, dt):
    x = torch.full((9, c), 3.0, device="cuda", dtype=dt)
    x[4] = 0
    beta = make((c,), F32, c)
    y, mean, invstd = oc.oc_ln_fwd(x, make((c,), F32, 1), beta, 1e-5, need_stats=True)
    near(y, np.broadcast_to(_np(beta), (9, c)), 1e-4 + 2.0 ** -8 * np.abs(_np(beta)), "y")
    assert torch.equal(mean, x[:, 0].float())
    dx, dg, _ = oc.oc_ln_bwd(x, make((9, c), dt, 2), None, mean, invstd)
    assert torch.isfinite(dx).all() and (dg.abs() <= 1e-4).all()


@DT
@pytest.mark.parametrize("c", [7, 128, 1024, 5000, 17000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_finite_stay_alone(c, dt, bad):
    x, dy = make((40, c), dt, 1), make((40, c), dt, 2)
    want = oc.oc_ln_fwd(x, need_stats=True)
    dwant = oc.oc_ln_bwd(x, dy, None, want[1], want[2])[0]
    xb = x.clone()
    xb[17, c // 2] = bad
    got = oc.oc_ln_fwd(xb, need_stats=True)
    dgot, dg, db = oc.oc_ln_bwd(xb, dy, None, got[1], got[2])
    rest = [r for r in range(40) if r != 17]
    assert torch.equal(got[0][rest], want[0][rest]) and torch.equal(dgot[rest], dwant[rest])
    assert got[0][17].isnan().all() and dgot[17].isnan().all() and dg.isnan().all()
    assert torch.isfinite(db).all()


def rng_of(seed, step):
    return torch.tensor([seed, step], dtype=torch.int64, device="cuda")


@DT
@pytest.mark.parametrize("i", range(len(SHAPES)))
@pytest.mark.parametrize("p", [0.5, 0.1, 0.0])
def test_dropout(i, p, dt):
    rows, c = SHAPES[i]
    print(f"[drop] {rows} x {c} {dt} {p}", flush=True)
    seed, step, site = -1234567890123456789 + i, (1 << 33) + i, (i * 1111) % 32768
    x = make((rows, c), dt, i, 1.0, i % 5)
    rng = rng_of(seed, step)
    y = oc.oc_dropout_rng(x, p, rng, site=site)
    keep, q = R.mask(rows, c, p, seed, step, site)
    want = np.where(keep, _np(x) / q, 0.0)
    near(y, want, (2.1 * U + v_of(dt)) * np.abs(want) if p else 0.0, "y")
    ones = oc.oc_dropout_rng(torch.ones_like(x), p, rng, site=site)
    assert np.array_equal(_np(ones) != 0, keep)
    z = x.clone()
    assert oc.oc_dropout_rng(z, p, rng, site=site, y=z) is z and torch.equal(z, y)  # in place
    assert rng.tolist() == [seed, step]


@pytest.mark.parametrize("p", [1e-5, 2.0 ** -16, 0.3, 0.9, 1 - 2.0 ** -20])
def test_dropout_low_halves_decide_ties(p):
    """Of 2^23 values some 128 have a high half equal to T's: each side of it."""
    rows, c, seed, step, site = 8192, 1024, 99, 12, 32767
    t = R.threshold(p)
    num = R.numbers(rows, c, seed, step, site)
    assert (num >> np.uint64(16) == t >> 16).sum() > 50
    ones = torch.ones(rows, c, device="cuda")
    assert np.array_equal(_np(oc.oc_dropout_rng(ones, p, rng_of(seed, step), site=site)) != 0,
                          num < t)


def test_dropout_masks_what_is_not_finite():
    x = torch.full((64, 100), float("nan"), device="cuda")
    x[::2] = float("inf")
    y = _np(oc.oc_dropout_rng(x, 0.5, rng_of(1, 2)))
    keep, _ = R.mask(64, 100, 0.5, 1, 2)
    assert (y[~keep] == 0).all() and not np.isfinite(y[keep]).any()


# p, residual, upstream dh, affine
STEPS = [(0.1, True, True, True), (0.5, False, False, True), (0.0, True, True, False),
         (0.0, False, False, True), (0.25, True, False, False)]


@DT
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_drop_ln(i, dt):
    rows, c = SHAPES[i]
    p, with_res, with_dh, affine = STEPS[i % len(STEPS)]
    print(f"[drop_ln] {rows} x {c} {dt} {STEPS[i % len(STEPS)]}", flush=True)
    seed, step, site = 7 + i, 3, 9
    x = make((rows, c), dt, i, 2.0, i % 3)
    res = make((rows, c), dt, i + 10, 1.0, i % 4) if with_res else None
    dy, dh = make((rows, c), dt, i + 20), make((rows, c), dt, i + 30, 1.0, 1)
    dh = dh if with_dh else None
    gamma = make((c,), F32, i + 40) if affine else None
    beta = make((c,), F32, i + 50, 1.0, 1) if affine else None
    rng, eps = rng_of(seed, step), 1e-2
    keep, q = (None, 1.0) if p == 0 else R.mask(rows, c, p, seed, step, site)
    xd = _np(x) if p == 0 else np.where(keep, _np(x) / q, 0.0)
    hw = xd if res is None else xd + _np(res)
    h, y, mean, invstd = oc.oc_drop_ln_fwd(x, res, p, rng, gamma, beta, site=site, eps=eps,
                                           need_stats=True)
    herr = U * (3 * np.abs(xd) * (p > 0) + np.abs(hw) * (res is not None))
    near(h, hw, 1.01 * herr + v_of(dt) * np.abs(hw), "h")
    _, r = R.stats(hw, eps)
    z = np.abs(R.ln_fwd(hw, None, None, eps)[0])
    most = herr.max(1, keepdims=True)
    check_y(y, hw, _np(gamma), _np(beta), eps, dt, "y", extra=r[:, None] * (2 + z) * most)
    check_stats(mean, invstd, hw, eps, "stats", err=most[:, 0])
    got = oc.oc_drop_ln_bwd(x, res, dy, p, rng, gamma, mean, invstd, dh=dh, site=site)
    check_bwd(hw, _np(dy), _np(dh), _np(gamma), _np(invstd), dt, got, "bwd", keep, q, herr)
    few = oc.oc_drop_ln_bwd(x, res, dy, p, rng, gamma, mean, invstd, dh=dh, site=site, need_dres=False,
                            need_dgamma=False, need_dbeta=False)
    assert torch.equal(few[0], got[0]) and few[1:] == (None, None, None)
    if res is not None:  # in the residual's place
        again = oc.oc_drop_ln_fwd(x, res, p, rng, gamma, beta, site=site, eps=eps, h=res)
        assert again[0] is res and torch.equal(res, h) and torch.equal(again[1], y)


@pytest.mark.parametrize("rows,c", [(33_000, 520), (32_800, 768), (17_000, 1100), (8300, 2304)])
def test_many_bf16_rows(rows, c):
    """Widths whose backward has three vectors a thread from so many rows on."""
    dt, p, seed, step, site = BF16, 0.25, 5, 6, 7
    x, res = make((rows, c), dt, 1, 2.0, 1), make((rows, c), dt, 2)
    dy, dh = make((rows, c), dt, 3, 1.0, 3), make((rows, c), dt, 4)
    gamma, rng = make((c,), F32, 5), rng_of(seed, step)
    y, mean, invstd = oc.oc_ln_fwd(x, gamma, need_stats=True)
    got = oc.oc_ln_bwd(x, dy, gamma, mean, invstd)
    check_bwd(_np(x), _np(dy), None, _np(gamma), _np(invstd), dt, (None, *got), "ln")
    keep, q = R.mask(rows, c, p, seed, step, site)
    xd = np.where(keep, _np(x) / q, 0.0)
    hw = xd + _np(res)
    herr = U * (3 * np.abs(xd) + np.abs(hw))
    h, y, mean, invstd = oc.oc_drop_ln_fwd(x, res, p, rng, gamma, site=site, need_stats=True)
    got = oc.oc_drop_ln_bwd(x, res, dy, p, rng, gamma, mean, invstd, dh=dh, site=site)
    check_bwd(hw, _np(dy), _np(dh), _np(gamma), _np(invstd), dt, got, "drop_ln", keep, q, herr)


def test_drop_ln_is_dropout_then_layer_norm():
    """fp32: the fused step's mask, sums and norm are the separate calls'."""
    x, res = make((500, 384), F32, 1), make((500, 384), F32, 2)
    gamma, beta, rng = make((384,), F32, 3), make((384,), F32, 4), rng_of(5, 6)
    h, y, mean, invstd = oc.oc_drop_ln_fwd(x, res, 0.3, rng, gamma, beta, site=2, need_stats=True)
    near(oc.oc_dropout_rng(x, 0.3, rng, site=2) + res, _np(h), 2 * U * np.abs(_np(h)) + 3 * U * 2 * np.abs(_np(x)), "h")
    want = oc.oc_ln_fwd(h, gamma, beta, need_stats=True)
    assert torch.equal(y, want[0]) and torch.equal(mean, want[1])


EMBEDS = [(0, 5, 8), (1, 1, 1), (3, 7, 5), (64, 40, 128), (65, 40, 128), (64, 1000, 3),
          (500, 1, 64), (1000, 4, 33), (3000, 257, 100), (5000, 4096, 16), (5000, 4097, 8),
          (70, 100_000, 9), (20_000, 30_000, 24), (2500, 300, 1024), (700, 11, 2049),
          (40_000, 3, 7), (100_000, 5000, 8), (9000, 1, 513), (300, 70_000_000, 1),
          (70, 5, 65536)]


def ids_of(rows, num, kind, seed):
    rng = np.random.default_rng(seed)
    if kind == "same":
        ids = np.full(rows, num - 1)
    elif kind == "skewed":
        ids = (rng.random(rows) ** 4 * num).astype(np.int64)
    elif kind == "outside":
        ids = rng.integers(-3, num + 3, rows)
        ids[rng.random(rows) < 0.1] = -2 ** 31
        ids[rng.random(rows) < 0.1] = 2 ** 31 - 1
    elif kind == "none":
        ids = np.full(rows, -1)
    else:
        ids = rng.integers(0, num, rows)
    return ids.astype(np.int32)


@DT
@pytest.mark.parametrize("i", range(len(EMBEDS)))
@pytest.mark.parametrize("kind", ["even", "same", "skewed", "outside", "none"])
def test_embed(i, kind, dt):
    rows, num, c = EMBEDS[i]
    print(f"[embed] {rows} of {num} x {c} {kind} {dt}", flush=True)
    ids = ids_of(rows, num, kind, i)
    d = torch.as_tensor(ids).cuda()
    table = make((num, c), dt, i, 1.0, i % 3)
    dy = make((rows, c), dt, i + 1, 1.0, (i + 1) % 3)
    scale = 1.0 if i % 2 else 5.3
    y = oc.oc_embed_fwd(d, table, scale=scale)
    there = (ids >= 0) & (ids < num)
    # (rows of the table that no id names are not formed on the host: the largest has 70 M)
    used, at = np.unique(ids[there], return_inverse=True)
    short = _np(table[torch.as_tensor(used, device="cuda").long()])
    local = np.full(rows, -1)
    local[there] = at
    want = R.embed_fwd(local, short, np.float32(scale).astype(np.float64))
    near(y, want, (1.01 * U + v_of(dt)) * np.abs(want), "y")
    for out in (F32, dt):
        buf = torch.full((num * c + 16,), 7.0, device="cuda", dtype=out)
        got = buf[8:8 + num * c].view(num, c)
        assert oc.oc_embed_bwd(d, dy, num, scale=scale, dtable=got) is got
        assert (buf[:8] == 7).all() and (buf[8 + num * c:] == 7).all()
        w = R.embed_bwd(local, _np(dy), len(used), np.float32(scale).astype(np.float64))
        m = R.embed_bwd(local, np.abs(_np(dy)), len(used), abs(scale))
        rows_at = torch.as_tensor(used, device="cuda").long()
        near(got[rows_at], w, 68 * U * m + v_of(out) * np.abs(w), "dtable")
        if len(used) < num:
            others = torch.ones(num, dtype=torch.bool, device="cuda")
            others[rows_at] = False
            assert not got[others].any()
        assert torch.equal(oc.oc_embed_bwd(d, dy, num, scale=scale, dtype=out), got)


@DT
@pytest.mark.parametrize("rows,c", [(70_000, 520), (40_001, 1000), (2_100_000, 5)])
def test_embed_forward_of_many_rows(rows, c, dt):
    """Several rows in flight a group of lanes, ids outside the table among them."""
    num = 3000
    d = torch.as_tensor(ids_of(rows, num, "outside", 9)).cuda()
    table = make((num, c), dt, 8, 1.0, 1)
    y = oc.oc_embed_fwd(d, table, scale=3.0)
    there = ((d >= 0) & (d < num)).unsqueeze(1)
    want = torch.where(there, table.float()[d.clamp(0, num - 1).long()] * 3.0,
                       torch.zeros((), device="cuda"))
    assert torch.equal(y, want.to(dt))  # (one product, rounded once)


def test_embed_order_of_equal_ids_is_the_rows():
    """Sums whose value depends on the order: 1, then 2^24 and its negative, in fp32."""
    dy = torch.tensor([[2.0 ** 24], [1.0], [-(2.0 ** 24)], [1.0]], device="cuda").repeat(20, 1)
    ids = torch.arange(20, dtype=torch.int32, device="cuda").repeat_interleave(4)
    perm = torch.randperm(80, generator=torch.Generator().manual_seed(1))
    # rows of one id keep their order among themselves
    order = torch.sort(perm // 4, stable=True)[1]
    ids2, dy2 = torch.empty_like(ids), torch.empty_like(dy)
    ids2[order.cuda()], dy2[order.cuda()] = ids, dy
    assert torch.equal(oc.oc_embed_bwd(ids2, dy2, 20), oc.oc_embed_bwd(ids, dy, 20))


@DT
def test_embed_of_an_octrees_places(dt):
    """Shuffle keys as ids: the places of a batch's octants at depth 4."""
    g = torch.Generator().manual_seed(3)
    pts = torch.rand(6000, 3, generator=g).cuda()
    nrm = torch.nn.functional.normalize(torch.randn(6000, 3, generator=g), dim=1).cuda()
    tree = oc.oc_build(pts, nrm, np.array([0, 1000, 3500, 6000], np.int32), 4, 2)
    keys = tree.keys(4)
    place = _np(keys).astype(np.int64) & 0xFFFFFF
    assert (_np(keys).astype(np.int64) >> 24).max() == 2 and place.max() < 4096
    table, dy = make((4096, 48), dt, 1), make((len(place), 48), dt, 2)
    want = R.embed_fwd(place, _np(table))
    near(oc.oc_embed_fwd(keys, table, keys=True), want, v_of(dt) * np.abs(want), "y")
    # shapes from 128 on make the key's sign bit
    far = (keys.long() + (200 << 24)).to(torch.int32)
    assert int(far.min()) < 0
    assert torch.equal(oc.oc_embed_fwd(far, table, keys=True),
                       oc.oc_embed_fwd(keys, table, keys=True))
    w, m = R.embed_bwd(place, _np(dy), 4096), R.embed_bwd(place, np.abs(_np(dy)), 4096)
    near(oc.oc_embed_bwd(keys, dy, 4096, keys=True), w, 68 * U * m, "dtable")


@DT
def test_nothing_behind_the_rows_is_written(dt):
    for rows, c in ((7, 5), (33, 100), (9, 1027), (5, 4099), (3, 8195), (2, 16391)):
        n = rows * c

        def room(m=n, t=dt):
            return torch.full((m + 40,), 9.0, device="cuda", dtype=t)

        x, res, dy = (make((rows, c), dt, i, 1.0, i) for i in (1, 2, 3))
        rng, L = rng_of(1, 1), oc.load()
        code = 1 if dt == BF16 else 0
        bufs = [room() for _ in range(5)] + [room(rows, F32) for _ in range(2)] + [
            room(c, F32) for _ in range(2)]
        h, y, dx, dres, d, mean, invstd, dg, db = (b[13:13 + len(b) - 40] for b in bufs)
        ws = torch.full((L.oc_ln_bwd_workspace(rows, c) + 64,), 3, dtype=torch.uint8,
                        device="cuda")
        P = lambda t: t.data_ptr()  # noqa: E731
        st = torch.cuda.current_stream().cuda_stream
        assert L.oc_drop_ln_fwd(code, rows, c, P(x), P(res), 0.5, P(rng), 0, None, None, 1e-5,
                                P(h), P(y), P(mean), P(invstd), st) == 0
        assert L.oc_drop_ln_bwd(code, rows, c, P(x), P(res), P(dy), None, 0.5, P(rng), 0, None, P(mean),
                                P(invstd), P(dx), P(dres), P(dg), P(db), P(ws),
                                ws.numel() - 64, st) == 0
        assert L.oc_dropout_rng(code, rows, c, P(x), 0.5, P(rng), 0, P(d), st) == 0
        for b in bufs:
            assert (b[:13] == 9).all() and (b[-27:] == 9).all()
            assert torch.isfinite(b).all()
        assert (ws[-64:] == 3).all()


def test_offsets_past_32_bits():
    """More than 2^32 bytes and 2^31 values of a feature map: the last rows are the
    short call's."""
    rows, c = 2_200_000, 1024
    x = torch.empty((rows, c), dtype=BF16, device="cuda")
    for r in range(0, rows, 200_000):
        x[r:r + 200_000] = make((200_000, c), BF16, r)
    y, mean, invstd = oc.oc_ln_fwd(x, need_stats=True)
    tail = x[-1000:].clone()
    short = oc.oc_ln_fwd(tail, need_stats=True)
    assert torch.equal(y[-1000:], short[0]) and torch.equal(mean[-1000:], short[1])
    dx, _, db = oc.oc_ln_bwd(x, y, None, mean, invstd)
    assert torch.equal(dx[-1000:], oc.oc_ln_bwd(tail, short[0], None, short[1], short[2])[0])
    near(db[:64], y[:, :64].double().sum(0).cpu().numpy(),
         67 * U * y[:, :64].double().abs().sum(0).cpu().numpy(), "dbeta")
    del dx, y
    rng = rng_of(3, 4)
    d = oc.oc_dropout_rng(x, 0.5, rng)
    # the last row's groups
    first = (rows - 1) * (c // 8)
    i = np.arange(first, first + c // 8, dtype=np.uint64)
    w = R.philox(np.stack([i, i * 0, i * 0 + np.uint64(4), i * 0], -1), (3, 0))
    high = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(-1)
    assert np.array_equal(_np(d[-1]) != 0, (high < 32768) & (_np(x[-1]) != 0))
    del d
    ids = torch.arange(rows, dtype=torch.int32, device="cuda").flip(0)
    e = oc.oc_embed_fwd(ids, x)
    assert torch.equal(e[:1000], x[-1000:].flip(0))
    g = oc.oc_embed_bwd(ids, e, rows, dtype=BF16)
    assert torch.equal(g, x)


def test_calls_repeat_their_bits_on_every_stream():
    x, dy = make((5000, 700), BF16, 1), make((5000, 700), BF16, 2)
    ids = torch.as_tensor(ids_of(5000, 90, "skewed", 1)).cuda()
    rng = rng_of(5, 5)

    def all_of():
        h, y, mean, invstd = oc.oc_drop_ln_fwd(x, dy, 0.2, rng, need_stats=True)
        return [h, y, *oc.oc_drop_ln_bwd(x, dy, dy, 0.2, rng, None, mean, invstd),
                *oc.oc_ln_bwd(x, dy, None, mean, invstd), oc.oc_embed_bwd(ids, dy, 90)]

    want = all_of()
    torch.cuda.synchronize()
    outs = []
    for _ in range(3):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append(all_of())
    torch.cuda.synchronize()
    for got in outs:
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_states_and_sizes_that_do_not_fit_are_refused():
    x = make((4, 16), F32, 1)
    good = rng_of(1, 2)
    for rng in (None, good[:1], good.to(torch.int32), good.cpu(), torch.tensor([1, 2])):
        with pytest.raises(oc.OcError):
            oc.oc_dropout_rng(x, 0.5, rng)
    for call in (lambda: oc.oc_ln_fwd(x.t()), lambda: oc.oc_ln_fwd(x, x[0, :8]),
                 lambda: oc.oc_ln_fwd(x.half()), lambda: oc.oc_ln_fwd(x[0]),
                 lambda: oc.oc_drop_ln_fwd(x, x.bfloat16(), 0.5, good),
                 lambda: oc.oc_ln_bwd(x, x[:3], None, x[:, 0], x[:, 0]),
                 lambda: oc.oc_dropout_rng(x, 0.5, good, y=x[:2]),
                 lambda: oc.oc_embed_fwd(torch.zeros(3, dtype=torch.int64, device="cuda"), x),
                 lambda: oc.oc_embed_bwd(torch.zeros(3, dtype=torch.int32, device="cuda"), x, 5),
                 lambda: oc.oc_embed_bwd(torch.zeros(4, dtype=torch.int32, device="cuda"), x, 5,
                                         dtype=torch.float16)):
        with pytest.raises(oc.OcError):
            call()


@DT
@pytest.mark.parametrize("rows,num,c,kind", [
    (4096, 300, 24, "skewed"), (4097, 300, 24, "skewed"), (131_073, 513, 16, "even"),
    (1_048_577, 70_000, 3, "outside"), (1_048_576, 2, 9, "even"), (300_000, 1 << 20, 5, "even"),
    (600_000, 5, 520, "skewed"), (35_000_000, 3, 1, "even"), (65_536, 1 << 18, 2, "skewed")])
def test_embed_sizes_of_every_plan(rows, num, c, kind, dt):
    """Around the sort's limits and in pieces longer than fp32 sums go; against torch's
    float64 sums on the GPU."""
    d = torch.as_tensor(ids_of(rows, num, kind, 3)).cuda()
    dy = make((rows, c), dt, 4)
    got = oc.oc_embed_bwd(d, dy, num)
    there = (d >= 0) & (d < num)
    at, g = d[there].long(), dy[there].double()

    def sums(t):
        if num <= 8:
            return torch.stack([t[at == v].sum(0) for v in range(num)])
        return torch.zeros((num, c), dtype=torch.float64, device="cuda").index_add_(0, at, t)

    want, mags = sums(g), sums(g.abs())
    err = (got.double() - want).abs() - 68 * U * mags
    assert float(err.max()) <= 0, float(err.max())
    assert torch.equal(oc.oc_embed_bwd(d, dy, num), got)


@DT
def test_no_rows(dt):
    for c in (1, 64, 1000, 5000, 9000, 20000):
        x = torch.empty((0, c), device="cuda", dtype=dt)
        y, mean, invstd = oc.oc_ln_fwd(x, need_stats=True)
        assert y.shape == (0, c) and mean.shape == (0,)
        dx, dg, db = oc.oc_ln_bwd(x, x, None, mean, invstd)
        assert dx.shape == (0, c) and not dg.any() and not db.any()
        rng = rng_of(1, 2)
        h, y, mean, invstd = oc.oc_drop_ln_fwd(x, x.clone(), 0.5, rng, need_stats=True)
        got = oc.oc_drop_ln_bwd(x, x.clone(), x, 0.5, rng, None, mean, invstd)
        assert not got[2].any() and not got[3].any()
        assert oc.oc_dropout_rng(x, 0.5, rng).shape == (0, c)
        assert oc.oc_embed_fwd(torch.empty(0, dtype=torch.int32, device="cuda"),
                               torch.ones((4, c), device="cuda", dtype=dt)).shape == (0, c)


@DT
@pytest.mark.parametrize("rows,c", [(33, 8), (70, 127), (40, 1024), (9, 5001), (3, 17000)])
def test_in_place(rows, c, dt):
    """Where the header lets an output be an input, the bits are the separate call's."""
    L, code, st = oc.load(), 1 if dt == BF16 else 0, torch.cuda.current_stream().cuda_stream
    x, res, rng = make((rows, c), dt, 1), make((rows, c), dt, 2), rng_of(3, 4)
    P = lambda t: t.data_ptr()  # noqa: E731
    y, _, _ = oc.oc_ln_fwd(x)
    a = x.clone()
    assert L.oc_ln_fwd(code, rows, c, P(a), None, None, 1e-5, P(a), None, None, st) == 0
    assert torch.equal(a, y)
    h, y, _, _ = oc.oc_drop_ln_fwd(x, res, 0.4, rng)
    a, b = x.clone(), res.clone()
    assert L.oc_drop_ln_fwd(code, rows, c, P(a), P(b), 0.4, P(rng), 0, None, None, 1e-5, P(b),
                            P(a), None, None, st) == 0
    assert torch.equal(b, h) and torch.equal(a, y)


def test_two_streams_at_once():
    """Calls in flight together share nothing: each has the bits of the call alone."""
    torch.manual_seed(0)
    xs = [make((20_000, 512), BF16, i) for i in range(2)]
    ids = [torch.as_tensor(ids_of(20_000, 700, "skewed", i)).cuda() for i in range(2)]
    rngs = [rng_of(i, i) for i in range(2)]

    def run(i):
        h, y, m, r = oc.oc_drop_ln_fwd(xs[i], None, 0.3, rngs[i], need_stats=True)
        return [h, y, *oc.oc_drop_ln_bwd(xs[i], None, y, 0.3, rngs[i], None, m, r),
                oc.oc_embed_bwd(ids[i], xs[i], 700), oc.oc_dropout_rng(y, 0.3, rngs[i], site=1)]

    want = [run(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(run(i))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))


class Block:
    """What a user builds of them: places from a table, a residual step, a gated layer, a
    residual step and a head, with the loss, clipping and the update."""

    P, CLASSES = 0.25, 6

    def __init__(self, rows, c, dt, seed=1):
        self.dt, self.rows, self.c = dt, rows, c
        w = lambda shape, i, s: make(shape, F32, seed + i, s)  # noqa: E731
        self.w = dict(table=w((40, c), 0, 1.0), g1=w((c,), 1, 0.1) + 1, b1=w((c,), 2, 0.1),
                      wg=w((c, 4 * c), 3, c ** -0.5), wd=w((2 * c, c), 4, (2 * c) ** -0.5),
                      g2=w((c,), 5, 0.1) + 1, b2=w((c,), 6, 0.1),
                      wh=w((c, self.CLASSES), 7, c ** -0.5))
        self.ids = torch.as_tensor(ids_of(rows, 40, "outside", seed)).cuda()
        self.labels = (torch.arange(rows, device="cuda") % self.CLASSES).to(torch.int32)
        self.rng = rng_of(11, 0)

    def step(self):
        """(loss, gradients) in fp32 or bf16 features; gradients fp32."""
        dt, p = self.dt, self.w
        v = {k: t.to(dt) if t.dim() == 2 else t for k, t in p.items()}
        e = oc.oc_embed_fwd(self.ids, v["table"], scale=2.0)
        h1, y1, m1, r1 = oc.oc_drop_ln_fwd(e, None, self.P, self.rng, v["g1"], v["b1"], site=0,
                                           need_stats=True)
        u, pre = oc.oc_glu_fwd(y1, v["wg"], need_pre=True)
        f, _ = oc.oc_dense_fwd(u, v["wd"])
        h2, y2, m2, r2 = oc.oc_drop_ln_fwd(f, h1, self.P, self.rng, v["g2"], v["b2"], site=1,
                                           need_stats=True)
        d2 = oc.oc_dropout_rng(y2, self.P, self.rng, site=2)
        z, _ = oc.oc_dense_fwd(d2, v["wh"])
        loss, dz = oc.oc_softmax_ce(z.float(), self.labels)
        g = {}
        dd2, g["wh"], _ = oc.oc_dense_bwd(d2, v["wh"], dz.to(dt), need_db=False)
        dy2 = oc.oc_dropout_rng(dd2, self.P, self.rng, site=2)
        df, dh1, g["g2"], g["b2"] = oc.oc_drop_ln_bwd(f, h1, dy2, self.P, self.rng, v["g2"], m2,
                                                      r2, site=1)
        du, g["wd"], _ = oc.oc_dense_bwd(u, v["wd"], df, need_db=False)
        dy1, g["wg"], _ = oc.oc_glu_bwd(y1, v["wg"], du, pre, need_db=False)
        de, _, g["g1"], g["b1"] = oc.oc_drop_ln_bwd(e, None, dy1, self.P, self.rng, v["g1"], m1,
                                                    r1, dh=dh1, site=0, need_dres=False)
        g["table"] = oc.oc_embed_bwd(self.ids, de, 40, scale=2.0)
        return loss, g

    def plain(self, w, step=0):
        """The loss in float64 torch, differentiable."""
        ids = self.ids.cpu().long()
        there = ((ids >= 0) & (ids < 40)).unsqueeze(1)
        masks = [R.mask(self.rows, self.c, self.P, 11, step, s) for s in range(3)]
        drop = lambda x, i: x * torch.as_tensor(masks[i][0] / masks[i][1])  # noqa: E731
        ln = torch.nn.functional.layer_norm
        e = torch.where(there, w["table"][ids.clamp(0, 39)] * 2.0, torch.zeros((), dtype=torch.float64))
        h1 = drop(e, 0)
        y1 = ln(h1, (self.c,), w["g1"], w["b1"], 1e-5)
        a, b = (y1 @ w["wg"]).chunk(2, 1)
        h2 = h1 + drop((torch.nn.functional.silu(a) * b) @ w["wd"], 1)
        y2 = ln(h2, (self.c,), w["g2"], w["b2"], 1e-5)
        return torch.nn.functional.cross_entropy(drop(y2, 2) @ w["wh"], self.labels.cpu().long())


@pytest.mark.parametrize("rows,c", [(64, 32), (300, 72)])
def test_block_matches_autograd(rows, c):
    """fp32: chains of eight operators, whose errors (some 100 u each, relative to the
    largest values) are passed on by slopes of order 1: 1e-4 of each gradient's largest."""
    b = Block(rows, c, F32)
    loss, g = b.step()
    w = {k: t.detach().double().cpu().requires_grad_() for k, t in b.w.items()}
    want = b.plain(w)
    grads = torch.autograd.grad(want, list(w.values()))
    assert abs(float(loss) - float(want.detach())) < 1e-4
    for k, e in zip(w, grads):
        near(g[k], e.numpy(), 1e-4 * float(e.abs().max()), k)


def test_block_matches_differences():
    """The operators' gradient along itself, against the float64 loss's differences."""
    b = Block(50, 24, F32, seed=3)
    _, g = b.step()
    w = {k: t.detach().double().cpu() for k, t in b.w.items()}
    for k in ("table", "g1", "b2", "wd"):
        d = g[k].double().cpu()
        step = 1e-4 / float(d.norm())
        hi, lo = ({**w, k: w[k] + s * step * d} for s in (1, -1))
        slope = float(b.plain(hi) - b.plain(lo)) / (2 * step)
        assert abs(slope - float(d.square().sum())) < 1e-3 * float(d.square().sum()), k


@DT
def test_block_in_a_graph_draws_new_masks(dt):
    """A captured step, replayed with another step of the generator's state each time and
    eager work between, equals the eager step's bits, clipping and update included."""
    def train(b, vel):
        loss, g = b.step()
        names = sorted(g)
        oc.oc_grad_clip([g[k] for k in names], 1.0)
        for k in names:
            oc.oc_sgd(b.w[k], g[k], vel[k], 0.1, 0.9, 1e-4)
        b.rng[1] += 1
        return loss

    a, b = Block(200, 64, dt), Block(200, 64, dt)
    va, vb = ({k: torch.zeros_like(t) for k, t in m.w.items()} for m in (a, b))
    for _ in range(2):  # warm up both alike
        train(a, va)
        train(b, vb)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        lb = train(b, vb)
    losses = []
    for _ in range(4):
        la = train(a, va)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        losses.append(float(lb))
        assert float(la) == float(lb)
        assert all(torch.equal(a.w[k], b.w[k]) for k in a.w)
    assert len(set(losses)) == 4 and int(b.rng[1]) == 6
