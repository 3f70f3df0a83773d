"""Pins of the dense-layer oracle (oracle/dense.py): against float64 torch and
its autograd, and its gradients against central differences; argument errors of
the entry points, which are found before any device work."""
import ctypes as C
import math

import numpy as np
import pytest
import torch
import torch.nn.functional as F

import paper_1712_01537_amd as oc
from oracle import dense as D

TORCH_ACT = {"none": lambda z: z, "relu": torch.relu, "silu": F.silu, "gelu": F.gelu}


@pytest.mark.parametrize("name", D.ACTS)
def test_dense_matches_torch(name):
    rng = np.random.default_rng(5)
    x, w, b = rng.standard_normal((9, 6)), rng.standard_normal((6, 5)), rng.standard_normal(5)
    r, dy = rng.standard_normal((9, 5)), rng.standard_normal((9, 5))
    y, z = D.dense_fwd(x, w, b, r, name)
    t = [torch.tensor(v, requires_grad=True) for v in (x, w, b)]
    yt = TORCH_ACT[name](t[0] @ t[1] + t[2]) + torch.tensor(r)
    np.testing.assert_allclose(y, yt.detach().numpy(), rtol=1e-12, atol=1e-13)
    want = torch.autograd.grad(yt, t, torch.tensor(dy))
    for got, ref in zip(D.layer_bwd(x, w, D.dense_dz(dy, z, name)), want):
        np.testing.assert_allclose(got, ref.numpy(), rtol=1e-11, atol=1e-12)


@pytest.mark.parametrize("name", D.ACTS)
def test_glu_matches_torch(name):
    rng = np.random.default_rng(6)
    x, w, b = rng.standard_normal((7, 4)), rng.standard_normal((4, 10)), rng.standard_normal(10)
    dy = rng.standard_normal((7, 5))
    y, z = D.glu_fwd(x, w, b, name)
    t = [torch.tensor(v, requires_grad=True) for v in (x, w, b)]
    g, u = (t[0] @ t[1] + t[2]).chunk(2, dim=1)
    yt = TORCH_ACT[name](g) * u
    np.testing.assert_allclose(y, yt.detach().numpy(), rtol=1e-12, atol=1e-13)
    want = torch.autograd.grad(yt, t, torch.tensor(dy))
    for got, ref in zip(D.layer_bwd(x, w, D.glu_dz(dy, z, name)), want):
        np.testing.assert_allclose(got, ref.numpy(), rtol=1e-11, atol=1e-12)


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_gradients_against_differences(name):
    rng = np.random.default_rng(7)
    x, w, b = rng.standard_normal((3, 4)), rng.standard_normal((4, 6)), rng.standard_normal(6)
    dy, dyg = rng.standard_normal((3, 6)), rng.standard_normal((3, 3))

    def loss(glu, *v):
        y = D.glu_fwd(*v, name=name)[0] if glu else D.dense_fwd(*v, name=name)[0]
        return float((y * (dyg if glu else dy)).sum())

    for glu in (False, True):
        z = D.product(x, w, b)
        dz = D.glu_dz(dyg, z, name) if glu else D.dense_dz(dy, z, name)
        got = D.layer_bwd(x, w, dz)
        h = 1e-6  # truncation h^2 f''' / 6 ~ 1e-12, rounding 1e-16 / h ~ 1e-10
        for k, v in enumerate((x, w, b)):
            num = np.empty_like(v)
            for i in np.ndindex(v.shape):
                keep, ends = v[i], []
                for d in (h, -h):
                    v[i] = keep + d
                    ends.append(loss(glu, x, w, b))
                v[i] = keep
                num[i] = (ends[0] - ends[1]) / (2 * h)
            np.testing.assert_allclose(got[k], num, rtol=1e-6, atol=1e-7)


def test_clip_matches_torch():
    rng = np.random.default_rng(8)
    gs = [rng.standard_normal(s) for s in (3, 100, (5, 7), 0)]
    for most in (0.0, 0.5, 5.0, 1e9, math.inf):
        n, out = D.grad_clip(gs, most)
        ps = [torch.nn.Parameter(torch.zeros(g.shape, dtype=torch.float64)) for g in map(np.asarray, gs)]
        for p, g in zip(ps, gs):
            p.grad = torch.tensor(g)
        nt = torch.linalg.vector_norm(torch.cat([p.grad.flatten() for p in ps]))
        assert abs(n - float(nt)) <= 1e-12 * float(nt)
        for o, g in zip(out, gs):
            np.testing.assert_allclose(o, g * min(1.0, most / n), rtol=1e-12)


# --- refusals (no device work) ------------------------------------------------

P = C.c_void_p(256)  # never read: every call below is refused before


def _fwd(dt=0, act=0, rows=4, cin=3, cout=5, x=P, w=P, y=P, ws=None, n=0):
    return oc.load().oc_dense_fwd(dt, act, rows, cin, cout, x, w, None, None, y, None, ws, n, None)


def test_dense_refusals():
    L = oc.load()
    for bad in (dict(dt=2), dict(dt=-1), dict(act=4), dict(act=-1), dict(rows=-1),
                dict(rows=1 << 28), dict(cin=0), dict(cin=65537), dict(cout=0),
                dict(cout=65537), dict(x=None), dict(w=None), dict(y=None)):
        assert _fwd(**bad) == 1, bad
        assert b"oc_dense_fwd" in L.oc_last_error()
    assert _fwd(rows=0, x=None, w=None, y=None) == 0  # nothing to do
    assert _fwd(rows=1 << 24, cout=4096) == 5 and _fwd(rows=1 << 24, cin=4096) == 5
    assert L.oc_dense_fwd_workspace(0, 1 << 24, 3, 4096) == 0
    for bad in ((2, 4, 3, 5), (0, 0, 3, 5), (0, 4, 0, 5), (0, 4, 3, 65537)):
        assert L.oc_dense_fwd_workspace(*bad) == 0
        assert L.oc_dense_bwd_workspace(bad[0], 0, *bad[1:]) == 0

    def bwd(dt=0, act=2, rows=4, pre=P, y=None, dy=P, dx=P, dw_dt=0, dw=P, db=P, x=P, w=P, ws=P,
            n=1 << 30):
        return L.oc_dense_bwd(dt, act, rows, 3, 5, x, w, None, pre, y, dy, dx, dw_dt, dw, db, ws, n,
                              None)

    assert bwd(act=1, y=P) == 1  # both pre and y
    assert bwd(pre=None, x=None, dw=None) == 1 and bwd(pre=None, w=None, dx=None) == 1
    assert bwd(dy=None) == 1 and bwd(w=None) == 1 and bwd(x=None) == 1
    assert bwd(dw_dt=1) == 1 and bwd(dw_dt=7) == 1 and bwd(dt=1, dw_dt=7) == 1
    assert bwd(act=9) == 1 and bwd(rows=-2) == 1
    need = L.oc_dense_bwd_workspace(0, 2, 4, 3, 5)
    assert bwd(ws=C.c_void_p(264)) == 1 and b"aligned" in L.oc_last_error()
    assert need > 0 and bwd(n=need - 1) == 1 and bwd(ws=None) == 1
    assert b"workspace" in L.oc_last_error()
    assert bwd(dx=None, dw=None, db=None) == 0  # nothing asked for


def test_glu_refusals():
    L = oc.load()

    def fwd(dt=0, act=2, rows=4, cin=3, cout=5, x=P, w=P, y=P):
        return L.oc_glu_fwd(dt, act, rows, cin, cout, x, w, None, y, None, None, 0, None)

    for bad in (dict(dt=3), dict(act=5), dict(rows=-1), dict(cout=32769), dict(x=None),
                dict(w=None), dict(y=None)):
        assert fwd(**bad) == 1, bad
        assert b"oc_glu_fwd" in L.oc_last_error()
    assert fwd(rows=0) == 0
    assert L.oc_glu_fwd_workspace(0, 4, 3, 32769) == 0
    assert L.oc_glu_bwd_workspace(0, 4, 3, 32769) == 0
    need = L.oc_glu_bwd_workspace(0, 4, 3, 5)
    for x, pre, dy, n in ((None, None, P, need), (P, P, None, need), (P, P, P, need - 1)):
        assert L.oc_glu_bwd(0, 2, 4, 3, 5, x, P, None, pre, dy, P, 0, None, P, P, n, None) == 1


def test_grad_refusals():
    L = oc.load()
    ptrs, dts, counts = (C.c_void_p * 2)(256, 512), (C.c_int * 2)(0, 1), (C.c_int64 * 2)(5, 6)
    need = L.oc_grad_workspace(2, counts)
    assert need >= 24

    def clip(n=2, g=ptrs, d=dts, c=counts, most=1.0, o=ptrs, od=dts, ws=P, nb=need):
        return L.oc_grad_clip(n, g, d, c, most, o, od, None, ws, nb, None)

    assert clip(n=-1) == 1 and clip(g=None) == 1 and clip(d=None) == 1 and clip(c=None) == 1
    assert clip(d=(C.c_int * 2)(0, 2)) == 1 and clip(c=(C.c_int64 * 2)(5, -1)) == 1
    assert clip(g=(C.c_void_p * 2)(256, None)) == 1 and clip(o=(C.c_void_p * 2)(256, None)) == 1
    assert clip(most=-0.5) == 1 and clip(most=math.nan) == 1
    assert clip(o=None) == 1 and clip(od=None) == 1
    assert clip(od=(C.c_int * 2)(1, 1)) == 1   # fp32 into bf16
    assert clip(od=(C.c_int * 2)(0, 0)) == 1   # in place, in another type
    assert clip(ws=C.c_void_p(260)) == 1 and clip(ws=None) == 1 and clip(nb=need - 1) == 1
    # more chunks (of 8192 values) in a launch's 128 tensors than an index counts
    many = (C.c_void_p * 128)(*[256] * 128), (C.c_int * 128)(), (C.c_int64 * 128)(*[1 << 37] * 128)
    assert L.oc_grad_norm(128, *many, P, P, 1 << 40, None) == 1
    assert b"too many values" in L.oc_last_error()
    assert L.oc_grad_norm(2, ptrs, dts, counts, None, P, need, None) == 1
    assert L.oc_grad_norm(2, ptrs, dts, counts, P, P, need - 1, None) == 1
    assert L.oc_grad_workspace(-1, counts) == 0 and L.oc_grad_workspace(1, None) == 0


def test_binding_refuses_host_tensors():
    x, w = torch.zeros(4, 3), torch.zeros(3, 6)
    for call in (lambda: oc.oc_dense_fwd(x, w), lambda: oc.oc_dense_bwd(x, w, x),
                 lambda: oc.oc_glu_fwd(x, w), lambda: oc.oc_glu_bwd(x, w, x, x),
                 lambda: oc.oc_grad_norm([x]), lambda: oc.oc_grad_clip([x], 1.0)):
        with pytest.raises(oc.OcError):
            call()
