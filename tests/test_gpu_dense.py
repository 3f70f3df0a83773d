"""GPU parity of the dense layers (oc_dense_*, oc_glu_*) with the float64 oracle.

Tolerances (u = 2^-24): a sum of R products in fp32, in any order, is off by at
most (R + 4) u S, S the sum of the products' absolute values; the 4 covers what
each product itself may be off by.  An activation adds a few ulp of its own (8 u
of |z| + |y|) and stretches z's error by its largest slope, 1.13; its slope
changes by at most 0.8 per unit of z.  bf16 results are rounded once more, by
2^-8 relative, and so is dz in bf16.  Beside these bounds for each element, the
2-norm of the fp32 errors stays below u (2 + sqrt(R)) of the result's scale:
errors of either sign add up as a random walk, while a lost part of an operand
(2^-17) would not pass.
"""
import numpy as np
import pytest
import torch

import paper_1712_01537_amd as oc
from oracle import dense as D

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = 2.0 ** -8
ACT = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _abs(x):
    return np.abs(np.asarray(x, np.float64))


def make(rows, cin, cout, dt, act, glu, seed=0, bias=True, res=True):
    """Inputs on the GPU.  Before a ReLU they lie on a grid whose sums are exact
    in fp32, so that no rounding decides the sign of z."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 7919 * rows + 31 * cin + cout)
    nz = 2 * cout if glu else cout

    def rnd(shape, scale, t, grid=act == "relu"):
        v = torch.empty(shape, device="cuda").normal_(generator=g)
        v = (v * 8).round() / 8 if grid else v
        return (v * scale).to(t)

    s = 2.0 ** -round(0.5 * np.log2(cin))
    return dict(x=rnd((rows, cin), 1.0, DT[dt]), w=rnd((cin, nz), s, DT[dt]),
                b=rnd((nz,), 0.125, torch.float32) if bias else None,
                res=rnd((rows, cout), 1.0, DT[dt], False) if res and not glu else None,
                dy=rnd((rows, cout), 1.0, DT[dt], False))


def check(got, ref, tol, what):
    got, ref = _np(got), np.asarray(ref)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert np.isfinite(got).all(), what
    bad = np.abs(got - ref) > tol
    if bad.any():
        i = np.unravel_index(np.argmax(np.abs(got - ref) - tol), ref.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} outside; worst at {i}: got "
                             f"{got[i]!r} ref {ref[i]!r} tol {np.broadcast_to(tol, ref.shape)[i]!r}")


def check_norm(got, ref, scale, R, what):
    """2-norm of the error against that of the terms' root of squares."""
    err = np.linalg.norm(_np(got) - ref)
    most = U * (2 + np.sqrt(R)) * (np.linalg.norm(scale) + np.linalg.norm(ref))
    assert err <= most, (what, err, most)


def run_and_check(c, act, glu, dt, bwd=True, dw_dtype=None, again=False):
    a = ACT[act]
    x, w = _np(c["x"]), _np(c["w"])
    rows, cin = x.shape
    f32 = dt == "f32"
    rnd = 0.0 if f32 else BF
    b = _np(c["b"])
    S = _abs(x) @ _abs(w) + (0 if b is None else _abs(b))
    tz = (cin + 4) * U * S + 1e-38
    if glu:
        y, pre = oc.oc_glu_fwd(c["x"], c["w"], c["b"], act=a, need_pre=True, again=again)
        yr, z = D.glu_fwd(x, w, b, act)
        n = z.shape[1] // 2
        g, u = z[:, :n], z[:, n:]
        ag = D.act(g, act)
        tag = 1.13 * tz[:, :n] + 8 * U * (_abs(g) + _abs(ag))
        ty = tag * (_abs(u) + tz[:, n:]) + _abs(ag) * tz[:, n:] + 2 * U * _abs(yr)
    else:
        y, pre = oc.oc_dense_fwd(c["x"], c["w"], c["b"], res=c["res"], act=a, need_pre=True,
                                 again=again)
        yr, z = D.dense_fwd(x, w, b, _np(c["res"]), act)
        r = 0.0 if c["res"] is None else _abs(_np(c["res"]))
        ty = 1.13 * tz + 8 * U * (_abs(z) + r + _abs(yr))
    check(y, yr, ty + rnd * (_abs(yr) + ty), "y")
    if again:
        assert isinstance(pre, oc.Again)
    elif act == "relu" and not glu:  # signs, eight columns a byte
        bits = np.unpackbits(pre.cpu().numpy(), axis=1, bitorder="little")
        np.testing.assert_array_equal(bits[:, :z.shape[1]], z > 0)
    else:
        check(pre, z, tz, "pre")
        check_norm(pre, z, np.sqrt(np.square(x) @ np.square(w)), cin, "pre")
    if not bwd:
        return
    if glu:
        outs = oc.oc_glu_bwd(c["x"], c["w"], c["dy"], pre, act=a, dw_dtype=dw_dtype)
        dy = _np(c["dy"])
        dz = D.glu_dz(dy, z, act)
        tg = _abs(dy) * ((_abs(u) + tz[:, n:]) * (0.8 * tz[:, :n] + 8 * U * (1 + _abs(g)))
                         + 1.13 * tz[:, n:]) + 4 * U * _abs(dz[:, :n])
        tu = _abs(dy) * tag + 4 * U * _abs(dz[:, n:])
        tdz = np.concatenate([tg, tu], 1)
    else:
        outs = oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=a, pre=pre, dw_dtype=dw_dtype)
        dy = _np(c["dy"])
        dz = D.dense_dz(dy, z, act)
        exact = act in ("none", "relu")
        tdz = 0 * dy if exact else (_abs(dy) * (0.8 * tz + 8 * U * (1 + _abs(z))) + 2 * U * _abs(dz))
    dx, dw, db = outs
    dxr, dwr, dbr = D.layer_bwd(x, w, dz)
    top = tdz if f32 or (not glu and act in ("none", "relu")) else tdz + BF * (_abs(dz) + tdz)
    nz = dz.shape[1]
    Sx = (_abs(dz) + top) @ _abs(w).T
    check(dx, dxr, top @ _abs(w).T + (nz + 4) * U * Sx + rnd * (_abs(dxr) + Sx * U * nz + top @ _abs(w).T),
          "dx")
    tw = _abs(x).T @ top + (rows + 4) * U * (_abs(x).T @ (_abs(dz) + top))
    check(dw, dwr, tw + (BF * (_abs(dwr) + tw) if dw.dtype == torch.bfloat16 else 0), "dw")
    check(db, dbr, tdz.sum(0) + (rows + 4) * U * (_abs(dz) + tdz).sum(0), "db")
    if f32 and act in ("none", "relu") and not glu:
        check_norm(dx, dxr, np.sqrt(np.square(dz) @ np.square(w).T), nz, "dx")
        check_norm(dw, dwr, np.sqrt(np.square(x).T @ np.square(dz)), rows, "dw")


SIZES = [(1, 1, 1), (1, 8, 8), (1, 129, 40), (2, 7, 3), (3, 1024, 130), (5, 64, 1), (8, 40, 257),
         (9, 96, 64), (16, 16, 16), (17, 33, 65), (31, 130, 72), (32, 1024, 128), (64, 64, 64),
         (65, 3, 16), (100, 520, 24), (127, 100, 136), (128, 128, 128), (257, 1, 129),
         (300, 344, 88), (513, 72, 200), (1000, 16, 8), (1025, 31, 33), (2500, 256, 264)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_dense(i, dt):
    rows, cin, cout = SIZES[i]
    acts = list(ACT)
    for act in (acts[i % 4], acts[(i + 1 + i // 4) % 4]):
        print(f"[dense] {dt} {rows}x{cin}->{cout} {act}", flush=True)
        run_and_check(make(rows, cin, cout, dt, act, False, bias=i % 3 != 0, res=i % 2 == 0), act,
                      False, dt, dw_dtype=torch.bfloat16 if dt == "bf16" and i % 2 else None)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_glu(i, dt):
    rows, cin, cout = SIZES[i]
    act = list(ACT)[(i + 2) % 4]
    print(f"[glu] {dt} {rows}x{cin}->{cout} {act}", flush=True)
    run_and_check(make(rows, cin, cout, dt, act, True, bias=i % 2 == 0), act, True, dt,
                  dw_dtype=torch.bfloat16 if dt == "bf16" and i % 2 else None)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_formed_again(i, glu, dt):
    """The backward from x and w alone: within the same bounds."""
    rows, cin, cout = SIZES[i]
    act = list(ACT)[1 + i % 3]
    print(f"[again] {dt} glu {glu} {rows}x{cin}->{cout} {act}", flush=True)
    run_and_check(make(rows, cin, cout, dt, act, glu, bias=i % 3 != 1), act, glu, dt, again=True)


def test_which_is_formed_again():
    """Left to the rule: 32768 x 64 -> 2 x 1024 would keep 256 MB, the last-level
    cache's size, and is formed again; 8 rows fewer are kept.  The gradients agree."""
    g = torch.Generator().manual_seed(5)
    w = (torch.randn(64, 2048, generator=g) / 8).bfloat16().cuda()
    x = torch.randn(32768, 64, generator=g).bfloat16().cuda()
    dy = torch.randn(32768, 1024, generator=g).bfloat16().cuda()
    assert isinstance(oc.oc_glu_fwd(x[8:], w, need_pre=True)[1], torch.Tensor)
    assert oc.oc_glu_fwd(x, w)[1] is None
    got = []
    for again in (None, False):
        y, pre = oc.oc_glu_fwd(x, w, need_pre=True, again=again)
        assert isinstance(pre, oc.Again if again is None else torch.Tensor)
        got.append((y,) + tuple(oc.oc_glu_bwd(x, w, dy, pre)))
    assert torch.equal(got[0][0], got[1][0])
    # The slopes may be contracted differently, so that a dz now and then rounds to the
    # neighbouring bf16 value (2^-7 of it apart), and dx and dw (2^-7 apart) after it:
    # with the terms' signs at random, at most twice 2^-7 of the root of the squares.
    for a, b in zip(got[0][1:], got[1][1:]):
        assert (a.double() - b.double()).norm() <= 2.0**-6 * b.double().norm()


LARGE = [(70_000, 72, 520, "relu"), (9000, 1032, 2056, "silu"), (40_001, 264, 1000, "gelu"),
         (5000, 520, 4104, "none"), (33_000, 515, 260, "silu"), (6000, 2051, 777, "gelu")]


@pytest.mark.parametrize("again", [False, True])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(LARGE)))
def test_large(i, dt, glu, again):
    """Sizes of the large tiles, aligned and not.  The error's 2-norm against that
    of the result: 2^-9 for each rounding to bf16 (its mean square is below a third
    of half a step's), and a random walk of fp32 roundings of the root of the
    terms' squares."""
    rows, cin, cout, act = LARGE[i]
    print(f"[large] {dt} glu {glu} {rows}x{cin}->{cout} {act}", flush=True)
    c = make(rows, cin, cout, dt, act, glu)
    a = ACT[act]
    x, w, dy = c["x"].double(), c["w"].double(), c["dy"].double()
    for v in (x, w):
        v.requires_grad_()
    b = c["b"].double().requires_grad_()
    fn = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu,
          "gelu": torch.nn.functional.gelu}[act]
    z = x @ w + b
    if glu:
        y, pre = oc.oc_glu_fwd(c["x"], c["w"], c["b"], act=a, need_pre=True, again=again)
        got = oc.oc_glu_bwd(c["x"], c["w"], c["dy"], pre, act=a, dw_dtype=DT[dt])
        yr = fn(z[:, :cout]) * z[:, cout:]
    else:
        y, pre = oc.oc_dense_fwd(c["x"], c["w"], c["b"], res=c["res"], act=a, need_pre=True,
                                 again=again)
        got = oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=a, pre=pre, dw_dtype=DT[dt])
        yr = fn(z) + c["res"].double()
    ref = torch.autograd.grad(yr, (x, w, b), dy)
    nz = w.shape[1]
    for what, p, r, terms, rounds in (("y", y, yr.detach(), cin, 1), ("dx", got[0], ref[0], nz, 2),
                                      ("dw", got[1], ref[1], rows, 2), ("db", got[2], ref[2], rows, 0)):
        most = U * (4 + 2 * terms ** 0.5) + (rounds * 2.0 ** -9 if dt == "bf16" else 0.0)
        err = float((p.double() - r).norm() / r.norm())
        assert err <= most, (what, err, most)
        # no single value far off: 64 times the mean error
        far = float((p.double() - r).abs().max() / (r.abs() + r.square().mean().sqrt()).max())
        assert far <= 64 * most, (what, far, most)


# Backwards whose two products share a launch: the tile shapes and, of either product,
# whole and split reductions, in both orders (on a card of 256 CUs).
TOGETHER = [("bf16", 26680, 1968, 3664), ("bf16", 20680, 960, 2272), ("bf16", 2137, 1200, 1672),
            ("bf16", 934, 1744, 1480), ("bf16", 2597, 976, 96), ("bf16", 6055, 360, 208),
            ("bf16", 71, 936, 2288), ("bf16", 4612, 120, 2776), ("bf16", 35, 8, 88),
            ("bf16", 718, 8, 72), ("bf16", 35, 96, 624), ("bf16", 33, 1656, 1648),
            ("bf16", 2125, 8, 1040), ("bf16", 2177, 24, 2936), ("bf16", 1500, 203, 77),
            ("f32", 4151, 920, 3288), ("f32", 1355, 1504, 1640), ("f32", 1640, 1992, 264),
            ("f32", 1296, 2000, 216), ("f32", 221, 880, 3200), ("f32", 155, 1960, 1704),
            ("f32", 1168, 200, 1824), ("f32", 1467, 240, 2176), ("f32", 801, 1760, 592),
            ("f32", 426, 1904, 920), ("f32", 3092, 456, 8), ("f32", 1731, 784, 416),
            ("f32", 242, 1168, 1136), ("f32", 405, 80, 1760), ("f32", 1178, 1872, 728),
            ("f32", 895, 1808, 80), ("f32", 1428, 848, 216), ("f32", 116, 1632, 1096),
            ("f32", 625, 224, 1384), ("f32", 2071, 504, 1288), ("f32", 33, 8, 104),
            ("f32", 238, 24, 40), ("f32", 35, 448, 3640), ("f32", 678, 24, 1152),
            ("f32", 397, 33, 205)]


@pytest.mark.parametrize("dt,rows,cin,cout", TOGETHER)
def test_both_products(dt, rows, cin, cout):
    """test_large's bounds, one rounding of each result (dz is dy)."""
    c = make(rows, cin, cout, dt, "none", False)
    x, w, dy = c["x"].double(), c["w"].double(), c["dy"].double()
    got = oc.oc_dense_bwd(c["x"], c["w"], c["dy"], dw_dtype=DT[dt])
    for p, r, terms in ((got[0], dy @ w.T, cout), (got[1], x.T @ dy, rows),
                        (got[2], dy.sum(0), 0)):
        most = U * (4 + 2 * (terms or rows) ** 0.5) + (2.0 ** -9 if dt == "bf16" and terms else 0.0)
        assert float((p.double() - r).norm() / r.norm()) <= most
        far = float((p.double() - r).abs().max() / (r.abs() + r.square().mean().sqrt()).max())
        assert far <= 64 * most


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cin,cout,glu", [(70, 65536, 3, False), (70, 3, 65536, False),
                                               (3, 65536, 5, False), (2, 5, 65536, False),
                                               (9, 4, 32768, True), (1, 12, 32768, True)])
def test_longest_rows(rows, cin, cout, glu, dt):
    for again in (False, True):
        run_and_check(make(rows, cin, cout, dt, "silu", glu), "silu", glu, dt, again=again)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("glu", [False, True])
def test_gradients_against_differences(glu, act):
    """Central differences of the kernels' own forward along random directions.
    With h = 2^-7 a direction of unit mean square changes z by some h; the third
    derivative's term is h^2 / 6 < 1.1e-5 of the slope's, a few times more where
    products of two changes enter; fp32 outputs of size 1 are off by some 2^-23 each,
    so a sum of n of them by 2^-23 sqrt(n), over 2 h 2^-17 sqrt(n), while a derivative
    is of size sqrt(n): 1e-3 of the gradient's norm covers both."""
    c = make(90, 40, 48, "f32", act, glu, res=False)
    a, f = ACT[act], oc.oc_glu_fwd if glu else oc.oc_dense_fwd
    _, pre = f(c["x"], c["w"], c["b"], act=a, need_pre=True)
    grads = (oc.oc_glu_bwd(c["x"], c["w"], c["dy"], pre, act=a) if glu
             else oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=a, pre=pre))
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    h = 2.0 ** -7
    for k, grad in zip("xwb", grads):
        v = torch.empty_like(grad).normal_(generator=g)
        scale = 1.0 if k != "w" else 40 ** -0.5
        ends = []
        for s in (h * scale, -h * scale):
            t = {q: c[q] + s * v if q == k else c[q] for q in "xwb"}
            ends.append(float((f(t["x"], t["w"], t["b"], act=a)[0].double() * c["dy"].double()).sum()))
        num = (ends[0] - ends[1]) / (2 * h * scale)
        want = float((grad.double() * v.double()).sum())
        assert abs(num - want) <= 1e-3 * float(grad.double().norm()), (k, num, want)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_a_row_does_not_depend_on_the_others(dt):
    """The same row among few, some and many: within the bounds of its own sums
    (other kernels and orders), whatever the rest holds."""
    c = make(700, 136, 72, dt, "gelu", False)
    z = D.product(_np(c["x"]), _np(c["w"]), _np(c["b"]))
    S = _abs(_np(c["x"])) @ _abs(_np(c["w"])) + _abs(_np(c["b"]))
    for rows in (1, 3, 4, 5, 8, 9, 16, 17, 64, 65, 130, 700):
        pre = oc.oc_dense_fwd(c["x"][:rows].contiguous(), c["w"], c["b"], act=3, need_pre=True)[1]
        check(pre, z[:rows], (136 + 4) * U * S[:rows], rows)


def _view(t, shift):
    """A contiguous copy of t whose first element is `shift` elements into its buffer."""
    buf = torch.full((t.numel() + 16,), 7.0, dtype=t.dtype, device=t.device)
    v = buf[shift:shift + t.numel()].view(t.shape)
    v.copy_(t)
    return v


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("rows", [1, 6, 300])
def test_any_alignment(rows, glu, dt):
    """Buffers at any element's address give what aligned ones give."""
    c = make(rows, 72, 40, dt, "gelu", glu)
    for again in (False, True):
        run_and_check({k: None if v is None else _view(v, 1 + i)
                       for i, (k, v) in enumerate(c.items())}, "gelu", glu, dt, again=again)


def test_relu_backward_takes_the_output():
    for dt in DT:
        c = make(130, 64, 72, dt, "relu", False, res=False)
        y, pre = oc.oc_dense_fwd(c["x"], c["w"], c["b"], act=1, need_pre=True)
        for p, q in zip(oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=1, pre=pre),
                        oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=1, pre=y)):
            assert torch.equal(p, q)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_parts_asked_for(dt):
    """Each gradient alone is that of the whole call, but for the order of its sums
    (of at most 200 terms: each side within test_large's bound of the exact value);
    none of them asked for touches nothing."""
    most = 2 * (U * (4 + 2 * 200 ** 0.5) + (2.0 ** -9 if dt == "bf16" else 0.0))
    c = make(200, 48, 80, dt, "silu", False)
    for again in (False, True):
        _, pre = oc.oc_dense_fwd(c["x"], c["w"], c["b"], act=2, need_pre=True, again=again)
        every = oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=2, pre=pre)
        for k in range(3):
            need = [j == k for j in range(3)]
            got = oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=2, pre=pre, need_dx=need[0],
                                  need_dw=need[1], need_db=need[2])
            assert sum(g is not None for g in got) == 1
            assert (got[k].double() - every[k].double()).norm() <= most * every[k].double().norm()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_no_rows(dt):
    e = torch.empty((0, 24), dtype=DT[dt], device="cuda")
    for glu in (False, True):
        w = torch.ones((24, 10), dtype=DT[dt], device="cuda")
        dw = torch.full((24, 10), 3.0, dtype=DT[dt], device="cuda")
        n = 5 if glu else 10
        dy = torch.empty((0, n), dtype=DT[dt], device="cuda")
        pre = torch.empty((0, 10), dtype=torch.float32, device="cuda")
        if glu:
            assert oc.oc_glu_fwd(e, w)[0].shape == (0, n)
            dx, dw, db = oc.oc_glu_bwd(e, w, dy, pre, dw=dw)
        else:
            assert oc.oc_dense_fwd(e, w, act=3)[0].shape == (0, n)
            dx, dw, db = oc.oc_dense_bwd(e, w, dy, act=3, pre=pre, dw=dw)
        assert dx.shape == (0, 24) and not dw.any() and not db.any()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cin,cout", [(1, 64, 72), (33, 40, 65), (300, 72, 24)])
def test_what_is_behind_stays(rows, cin, cout, dt):
    """Nothing is written behind any output, and the residual may be the output."""
    c = make(rows, cin, cout, dt, "gelu", False)
    L, code = oc.load(), 1 if dt == "bf16" else 0

    def guarded(n, t):
        v = torch.full((n + 64,), 11.0, dtype=t, device="cuda")
        return v, v[:n]

    want, wpre = oc.oc_dense_fwd(c["x"], c["w"], c["b"], res=c["res"], act=3, need_pre=True)
    yb, y = guarded(rows * cout, DT[dt])
    pb, pre = guarded(rows * cout, torch.float32)
    y.copy_(c["res"].view(-1))
    ws = torch.full((int(L.oc_dense_fwd_workspace(code, rows, cin, cout)) + 256,), 5,
                    dtype=torch.uint8, device="cuda")
    assert L.oc_dense_fwd(code, 3, rows, cin, cout, c["x"].data_ptr(), c["w"].data_ptr(),
                          c["b"].data_ptr(), y.data_ptr(), y.data_ptr(), pre.data_ptr(),
                          ws.data_ptr(), ws.numel() - 256, oc._stream()) == 0
    assert torch.equal(y.view(rows, cout), want) and torch.equal(pre.view(rows, cout), wpre)
    dxb, dx = guarded(rows * cin, DT[dt])
    dwb, dw = guarded(cin * cout, torch.float32)
    dbb, db = guarded(cout, torch.float32)
    ws2 = torch.full((int(L.oc_dense_bwd_workspace(code, 3, rows, cin, cout)) + 256,), 5,
                     dtype=torch.uint8, device="cuda")
    assert L.oc_dense_bwd(code, 3, rows, cin, cout, c["x"].data_ptr(), c["w"].data_ptr(),
                          None, pre.data_ptr(), None, c["dy"].data_ptr(), dx.data_ptr(), 0,
                          dw.data_ptr(), db.data_ptr(), ws2.data_ptr(), ws2.numel() - 256,
                          oc._stream()) == 0
    for buf, v in ((yb, y), (pb, pre), (dxb, dx), (dwb, dw), (dbb, db)):
        assert (buf[v.numel():] == 11.0).all()
    assert (ws[-256:] == 5).all() and (ws2[-256:] == 5).all()
    for p, q in zip((dx.view(rows, cin), dw.view(cin, cout), db),
                    oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=3, pre=pre.view(rows, cout))):
        assert torch.equal(p, q)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cin,cout", [(2, 96, 40), (70, 160, 72), (600, 520, 264)])
def test_infinities_and_nan_stay_in_their_rows(rows, cin, cout, dt):
    """A row of x that holds an infinity or NaN gives what IEEE sums give there and
    leaves every other row's bits as they were; the same in dx and, by columns,
    in dw.  There fp32 values are split two neighbours at a time, so the partner of
    an infinite one is formed again in fp32 too: another order of the same sum,
    each within (rows + 4) u S of it."""
    c = make(rows, cin, cout, dt, "none", False, res=False, bias=False)
    y0 = oc.oc_dense_fwd(c["x"], c["w"])[0]
    dx0, dw0, _ = oc.oc_dense_bwd(c["x"], c["w"], c["dy"])
    x, dy = c["x"].clone(), c["dy"].clone()
    r, k, n = rows - 1, cin // 2, cout - 1
    x[r, k] = float("inf")
    dy[r, n] = float("nan")
    w64 = c["w"].double().cpu()
    y = oc.oc_dense_fwd(x, c["w"])[0]
    want = torch.sign(w64[k]) * float("inf")
    assert torch.equal(y[r].double().cpu(), want)
    keep = torch.arange(rows, device="cuda") != r
    assert torch.equal(y[keep], y0[keep])
    dx, dw, db = oc.oc_dense_bwd(x, c["w"], dy)
    assert torch.isnan(dx[r]).all() and torch.equal(dx[keep], dx0[keep])
    assert torch.isnan(db[n]) and torch.isfinite(db[:-1]).all()
    assert torch.isnan(dw[:, n]).all()
    assert torch.equal(dw[k, :-1].double().cpu(), torch.sign(dy[r, :-1].double().cpu()) * float("inf"))
    rest, cols = torch.arange(cin, device="cuda"), torch.arange(cout, device="cuda")
    S = c["x"].double().abs().t() @ c["dy"].double().abs()
    off = (dw.double() - dw0.double()).abs() <= 2 * (rows + 4) * U * S
    assert off[rest != k][:, cols != n].all()
    same = (rest // 2 != k // 2)[:, None] & (cols // 2 != n // 2)[None, :]
    assert torch.equal(dw[same], dw0[same])


@pytest.mark.parametrize("scale", [1e-36, 1e-18, 1e18, 3e31, 1e37])
def test_f32_range(scale):
    """Operands far from 1 keep fp32's precision; sums above 2^80 as well."""
    rows, cin, cout = 150, 72, 88
    c = make(rows, cin, cout, "f32", "none", False, res=False, bias=False)
    x = c["x"] * scale
    y = oc.oc_dense_fwd(x, c["w"])[0]
    S = _abs(_np(x)) @ _abs(_np(c["w"]))
    check(y, _np(x) @ _np(c["w"]), (cin + 4) * U * S + 1e-43, "y")
    dx, dw, _ = oc.oc_dense_bwd(x, c["w"], c["dy"])
    Sw = _abs(_np(x)).T @ _abs(_np(c["dy"]))
    if Sw.max() < 3.4e38:  # else a partial sum may pass fp32's largest value, in some order
        check(dw, _np(x).T @ _np(c["dy"]), (rows + 4) * U * Sw + 1e-43, "dw")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_same_bits_again(dt):
    for rows, cin, cout in ((1, 1024, 640), (40, 512, 72), (3000, 128, 264)):
        for glu in (False, True):
            c = make(rows, cin, cout, dt, "silu", glu)
            def once(again):
                if glu:
                    y, pre = oc.oc_glu_fwd(c["x"], c["w"], c["b"], need_pre=True, again=again)
                    return (y,) + tuple(oc.oc_glu_bwd(c["x"], c["w"], c["dy"], pre))
                y, pre = oc.oc_dense_fwd(c["x"], c["w"], c["b"], act=2, need_pre=True, again=again)
                return (y,) + tuple(oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=2, pre=pre))
            for again in (False, True):
                for p, q in zip(once(again), once(again)):
                    assert torch.equal(p, q)


@pytest.mark.parametrize("again", [False, True])
def test_other_stream_and_graphs(again):
    """On a stream of its own, and in two captured graphs replayed in turn with
    eager work between, each with new inputs: the eager call's bits."""
    cs = [make(150, 64, 72, dt, "gelu", glu, seed=k)
          for k, (dt, glu) in enumerate([("f32", False), ("bf16", True)])]

    def step(c, glu):
        if glu:
            y, pre = oc.oc_glu_fwd(c["x"], c["w"], c["b"], act=3, need_pre=True, again=again)
            return (y,) + tuple(oc.oc_glu_bwd(c["x"], c["w"], c["dy"], pre, act=3))
        y, pre = oc.oc_dense_fwd(c["x"], c["w"], c["b"], res=c["res"], act=3, need_pre=True,
                                 again=again)
        return (y,) + tuple(oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=3, pre=pre))

    side = torch.cuda.Stream()
    want = [step(c, g) for c, g in zip(cs, (False, True))]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = [step(c, g) for c, g in zip(cs, (False, True))]
    side.synchronize()
    for p, q in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(p, q))
    graphs, outs = [], []
    for c, g in zip(cs, (False, True)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(c, g))
        graphs.append(graph)
    for rep in range(4):
        for c in cs:
            c["x"].copy_(torch.roll(c["x"], 1, 0))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for c, g, out in zip(cs, (False, True), outs):
            for p, q in zip(step(c, g), out):
                assert torch.equal(p, q), rep


def test_more_than_4_gib():
    """Rows whose output, saved values and gradient pass 2^32 bytes."""
    rows, cin, cout = 1_100_003, 8, 1024
    c = make(rows, cin, cout, "f32", "relu", False, res=False)
    y, pre = oc.oc_dense_fwd(c["x"], c["w"], c["b"], act=1, need_pre=True)
    at = torch.tensor([0, 1, 131071, 524287, 524288, 1048575, 1048576, rows - 1], device="cuda")
    z = c["x"][at].double() @ c["w"].double() + c["b"].double()
    assert torch.equal(y[at].double(), torch.relu(z))
    bit = torch.arange(cout, device="cuda")
    assert torch.equal((pre[at][:, bit // 8] >> (bit % 8) & 1).bool(), z > 0)
    dx, dw, db = oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=1, pre=y)
    for p, q in zip(oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=1, pre=pre), (dx, dw, db)):
        assert torch.equal(p, q)
    dz = c["dy"][at].double() * (z > 0)
    w = c["w"].double()
    tol = (cout + 4) * U * (dz.abs() @ w.abs().t())
    assert ((dx[at].double() - dz @ w.t()).abs() <= tol).all()
    dwr = torch.zeros((cin, cout), dtype=torch.float64, device="cuda")
    dbr, S = torch.zeros(cout, dtype=torch.float64, device="cuda"), torch.zeros_like(dwr)
    for i in range(0, rows, 100_000):
        x, d = c["x"][i:i + 100_000].double(), c["dy"][i:i + 100_000].double()
        d = d * (y[i:i + 100_000] > 0)
        dwr += x.t() @ d
        S += x.abs().t() @ d.abs()
        dbr += d.sum(0)
    # Roundings are of either sign, so T of them on a running sum of size s leave
    # an error of U / sqrt(3) sqrt(T) s; the sum itself is a random walk of size
    # S / sqrt(rows).  Six products for every 32 rows: T <= 6 rows / 32, however
    # the rows are dealt out (64 steps were too few for long shares).  Five of
    # these, for 8192 values.
    walk = 5 * U * (6 * rows / 32 / 3) ** 0.5
    assert ((dw.double() - dwr).abs() <= walk * (S.max() / rows ** 0.5 + dwr.abs())).all()
    assert ((db.double() - dbr).abs() <= 64 * U * (dbr.abs() + rows ** 0.5)).all()


def test_refusals_of_tensors():
    c = make(4, 8, 16, "f32", "none", False)
    bad = torch.zeros((8, 32), device="cuda")
    for call in (lambda: oc.oc_dense_fwd(c["x"], c["w"].to(torch.bfloat16)),
                 lambda: oc.oc_dense_fwd(c["x"], bad[:, ::2]),
                 lambda: oc.oc_dense_fwd(c["x"], torch.zeros((7, 16), device="cuda")),
                 lambda: oc.oc_dense_fwd(c["x"], c["w"], res=c["res"][:3]),
                 lambda: oc.oc_dense_fwd(c["x"], c["w"], b=c["b"].double()),
                 lambda: oc.oc_dense_fwd(c["x"], c["w"], act=7),
                 lambda: oc.oc_dense_fwd(c["x"].half(), c["w"].half()),
                 lambda: oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=2),
                 lambda: oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=1),
                 lambda: oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=2, pre=c["dy"].byte()),
                 lambda: oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=1, pre=c["dy"].byte()),
                 lambda: oc.oc_dense_bwd(c["x"], c["w"], c["dy"][:2]),
                 lambda: oc.oc_dense_bwd(c["x"], c["w"], c["dy"], dw_dtype=torch.bfloat16),
                 lambda: oc.oc_glu_fwd(c["x"], c["w"][:, :15].contiguous()),
                 lambda: oc.oc_glu_bwd(c["x"], c["w"], c["dy"], c["dy"])):
        with pytest.raises(oc.OcError):
            call()
