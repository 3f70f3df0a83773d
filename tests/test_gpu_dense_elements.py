"""Every value of the dense layers' large and shared-launch bf16 cases against 64 bits.

Bounds (u = 2^-24; S the sum of a sum's products' absolute values, Q of their squares):
a sum of R products in fp32 is off by at most (R + 4) u S; a bf16 result is rounded by at
most 2^-8 of itself.  dz is rounded to bf16 (unless it is dy or 0), so each term of dx and
dw is off by up to 2^-8 of itself, uniformly and of either sign: a standard deviation of
2^-8 sqrt(Q / 3), of which 6 2^-8 sqrt(Q) is more than ten."""
import pytest
import torch

import paper_1712_01537_amd as oc
import test_gpu_dense as T

pytestmark = pytest.mark.gpu

U, BF = 2.0 ** -24, 2.0 ** -8


def within(got, ref, tol, what):
    off = (got.double() - ref).abs() - tol
    assert torch.isfinite(got).all() and float(off.max()) <= 0.0, (what, int((off > 0).sum()))


def gradients(got, x, w, dz, rounded, tdz):
    """dx, dw and db for dz, itself off by tdz before its rounding."""
    ax, aw, az = x.abs(), w.abs(), dz.abs() + tdz
    rows, nz = dz.shape
    for g, a, b, aa, ab, terms, err, what in (
            (got[0], dz, w.t().contiguous(), az, aw.t().contiguous(), nz,
             lambda: tdz @ aw.t().contiguous(), "dx"),
            (got[1], x.t().contiguous(), dz, ax.t().contiguous(), az, rows,
             lambda: ax.t().contiguous() @ tdz, "dw")):
        ref = a @ b
        tol = (terms + 4) * U * (aa @ ab) + err()
        if rounded:
            tol += 6 * BF * ((aa * aa) @ (ab * ab)).sqrt()
        within(g, ref, tol + BF * (ref.abs() + tol), what)
    within(got[2], dz.sum(0), 70 * U * az.sum(0) + tdz.sum(0), "db")


def slope(act, z):
    z = z.clone().requires_grad_()
    y = {"none": lambda v: v * 1.0, "relu": torch.relu, "silu": torch.nn.functional.silu,
         "gelu": torch.nn.functional.gelu}[act](z)
    return y.detach(), torch.autograd.grad(y.sum(), z)[0]


@pytest.mark.parametrize("again", [False, True])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("i", range(len(T.LARGE)))
def test_large(i, glu, again):
    rows, cin, cout, act = T.LARGE[i]
    print(f"[elements] glu {glu} {rows}x{cin}->{cout} {act}", flush=True)
    c, a = T.make(rows, cin, cout, "bf16", act, glu), T.ACT[act]
    x, w, dy = c["x"].double(), c["w"].double(), c["dy"].double()
    z = x @ w + c["b"].double()
    tz = (cin + 4) * U * (x.abs() @ w.abs() + c["b"].double().abs())
    if glu:
        y, pre = oc.oc_glu_fwd(c["x"], c["w"], c["b"], act=a, need_pre=True, again=again)
        got = oc.oc_glu_bwd(c["x"], c["w"], c["dy"], pre, act=a, dw_dtype=torch.bfloat16)
        g, u, tg, tu = z[:, :cout], z[:, cout:], tz[:, :cout], tz[:, cout:]
        ag, sg = slope(act, g)
        tag = 1.13 * tg + 8 * U * (g.abs() + ag.abs())
        ref = ag * u
        ty = tag * (u.abs() + tu) + ag.abs() * tu + 2 * U * ref.abs()
        dz = torch.cat([dy * u * sg, dy * ag], 1)
        tdz = torch.cat([dy.abs() * ((u.abs() + tu) * (0.8 * tg + 8 * U * (1 + g.abs())) + 1.13 * tu),
                         dy.abs() * tag], 1) + 4 * U * dz.abs()
    else:
        y, pre = oc.oc_dense_fwd(c["x"], c["w"], c["b"], res=c["res"], act=a, need_pre=True,
                                 again=again)
        got = oc.oc_dense_bwd(c["x"], c["w"], c["dy"], act=a, pre=pre, dw_dtype=torch.bfloat16)
        az, sz = slope(act, z)
        r = c["res"].double()
        ref = az + r
        ty = 1.13 * tz + 8 * U * (z.abs() + r.abs() + ref.abs())
        dz = dy * sz
        tdz = (torch.zeros_like(dz) if act in ("none", "relu")
               else dy.abs() * (0.8 * tz + 8 * U * (1 + z.abs())) + 2 * U * dz.abs())
    within(y, ref, ty + BF * (ref.abs() + ty), "y")
    gradients(got, x, w, dz, glu or act not in ("none", "relu"), tdz)


@pytest.mark.parametrize("dt,rows,cin,cout", [c for c in T.TOGETHER if c[0] == "bf16"])
def test_both_products(dt, rows, cin, cout):
    c = T.make(rows, cin, cout, dt, "none", False)
    x, w, dy = c["x"].double(), c["w"].double(), c["dy"].double()
    got = oc.oc_dense_bwd(c["x"], c["w"], c["dy"], dw_dtype=torch.bfloat16)
    gradients(got, x, w, dy, False, torch.zeros_like(dy))
