"""GPU parity of the global gradient norm and of clipping with the float64
oracle, and of the operators run together: layers, loss, clipping and update.

Squares and their sum are in double, so the norm is off by its own rounding to
fp32 (2^-24) and the double sum's (2^-53 per term, nothing beside it); a clipped
value is off by the rounding of the factor and of the product (2 x 2^-24)."""
import math

import numpy as np
import pytest
import torch

import paper_1712_01537_amd as oc
from oracle import dense as D
from oracle import train as T

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _np(t):
    return t.detach().double().cpu().numpy()


def make(sizes, seed, kinds=(torch.float32,), shift=0):
    """Gradients as views into one buffer a type, `shift` elements in."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = kinds[i % len(kinds)]
        buf = torch.empty(n + shift, device="cuda").normal_(generator=g).mul_(10.0 ** (i % 5 - 2))
        out.append(buf.to(t)[shift:shift + n])
    return out


def check(grads, most, outs=None):
    ref = [_np(g) for g in grads]
    n, clipped = D.grad_clip(ref, most)
    assert abs(float(oc.oc_grad_norm(grads)) - n) <= 1.01 * U * n
    norm = oc.oc_grad_clip(grads, most, outs=outs)
    assert abs(float(norm) - n) <= 1.01 * U * n
    for i, (o, r) in enumerate(zip(grads if outs is None else outs, clipped)):
        rnd = 2.0 ** -8 if o.dtype == torch.bfloat16 else 0.0
        err = np.abs(_np(o) - r)
        assert (err <= (2.1 * U + rnd) * np.abs(r) + 1e-45).all(), (i, err.max())
    return norm


SIZES = [[1], [0], [7], [5, 0, 3], [8192], [8193, 8191, 1], [100_003], list(range(1, 140)),
         [3 * 7] * 300, [4_000_037, 2, 65]]


@pytest.mark.parametrize("i", range(len(SIZES)))
@pytest.mark.parametrize("kinds", [(torch.float32,), (torch.bfloat16,),
                                   (torch.float32, torch.bfloat16)])
def test_clip(i, kinds):
    sizes = SIZES[i]
    for most in (0.25, 1e30):
        print(f"[clip] {sizes[:6]} max {most}", flush=True)
        grads = make(sizes, i, kinds, shift=i % 3)
        outs = [torch.full((n + 3,), 9.0, device="cuda")[1:n + 1] for n in sizes]
        kept = [g.clone() for g in grads]
        check(grads, most, outs)
        assert all(torch.equal(g, k) for g, k in zip(grads, kept))  # inputs stay
        check(grads, most)  # in place


def test_nothing_behind_is_written():
    big = torch.full((1000,), 4.0, device="cuda")
    g = big[10:900]
    oc.oc_grad_clip([g], 1.0)
    assert (big[:10] == 4.0).all() and (big[900:] == 4.0).all() and (g != 4.0).all()


def test_no_tensors_and_zero_gradients():
    assert float(oc.oc_grad_norm([])) == 0.0
    assert float(oc.oc_grad_clip([], 1.0)) == 0.0
    z = [torch.zeros(100, device="cuda")]
    assert float(oc.oc_grad_clip(z, 0.0)) == 0.0 and not z[0].any()
    one = [torch.ones(100, device="cuda")]
    assert float(oc.oc_grad_clip(one, 0.0)) == 10.0 and not one[0].any()


def test_squares_outside_the_range_of_fp32():
    for s in (1e-30, 1e30):
        g = [torch.full((4096,), s, device="cuda"), torch.full((3,), -s, device="cuda")]
        check(g, 0.5 * s)
    # the gradient at the border is left alone, bit for bit
    g = [torch.full((4,), 0.5, device="cuda")]
    assert float(oc.oc_grad_clip(g, 1.0)) == 1.0 and (g[0] == 0.5).all()


def test_infinity_and_nan():
    g = [torch.ones(3000, device="cuda"), torch.ones(5, device="cuda")]
    g[0][17] = -math.inf
    assert float(oc.oc_grad_clip(g, 1.0)) == math.inf
    assert torch.isnan(g[0][17]) and int(torch.isnan(g[0]).sum()) == 1 and not g[1].any()
    g = [torch.ones(3000, device="cuda"), torch.ones(5, device="cuda")]
    g[1][0] = math.nan
    assert math.isnan(float(oc.oc_grad_clip(g, 1.0)))
    assert all(torch.isnan(t).all() for t in g)


def test_many_partial_sums():
    """More tensors and workgroups than one table and one pass over the sums take."""
    grads = make([400_003] * 150, 3)
    check(grads, 1.0, [torch.empty_like(g) for g in grads])


def test_same_bits_streams_and_graphs():
    grads = make([70_001, 5, 900_000], 9, (torch.float32, torch.bfloat16))
    outs = [torch.empty(g.numel(), device="cuda") for g in grads]
    n0 = oc.oc_grad_clip(grads, 1.0, outs=outs)
    first = [o.clone() for o in outs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        n1 = oc.oc_grad_clip(grads, 1.0, outs=outs)
    side.synchronize()
    assert torch.equal(n0, n1) and all(torch.equal(a, b) for a, b in zip(first, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = oc.oc_grad_clip(grads, 1.0, outs=outs)
    for rep in range(4):
        grads[0].mul_(1.5)
        want = [torch.empty_like(o) for o in outs]
        n = oc.oc_grad_clip(grads, 1.0, outs=want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(n, norm) and all(torch.equal(a, b) for a, b in zip(want, outs)), rep


def test_outputs_among_the_gradients():
    """Gradients may be their own outputs beside others that are not; empty tensors
    share an address (or none); another tensor's gradient is refused."""
    g, h, o = (torch.full((10,), v, device="cuda") for v in (1.0, 2.0, 0.0))
    e = [torch.empty(0, device="cuda") for _ in range(4)]
    with pytest.raises(oc.OcError):
        oc.oc_grad_clip([g, h], 1.0, outs=[h, g])
    with pytest.raises(oc.OcError):
        oc.oc_grad_clip([g, h], 1.0, outs=[o, g])
    n = oc.oc_grad_clip([g, e[0], h, e[1]], 1.0, outs=[o, e[2], h, e[3]])
    norm = math.sqrt(50.0)
    assert abs(n.item() - norm) <= 2.0**-23 * norm
    for t, v in ((g, 1.0), (o, 1.0 / norm), (h, 2.0 / norm)):
        assert (t - v).abs().max().item() <= 2.0**-22 * v


def test_refusals_of_tensors():
    g = torch.ones(10, device="cuda")
    for call in (lambda: oc.oc_grad_norm([g.double()]), lambda: oc.oc_grad_norm([g[::2]]),
                 lambda: oc.oc_grad_clip([g], -1.0), lambda: oc.oc_grad_clip([g], math.nan),
                 lambda: oc.oc_grad_clip([g, g], 1.0), lambda: oc.oc_grad_clip([g, g[:3]], 1.0),
                 lambda: oc.oc_grad_clip([g], 1.0, outs=[]),
                 lambda: oc.oc_grad_clip([g], 1.0, outs=[g[:5]]),
                 lambda: oc.oc_grad_clip([g], 1.0, outs=[g.to(torch.bfloat16)])):
        with pytest.raises(oc.OcError):
            call()
    assert (g == 1.0).all()


def test_run_together():
    """A classifier over octant features, one training iteration: dense (ReLU),
    gated block, dense with a residual, softmax loss, the backward of each,
    clipping, SGD; against the oracle's own iteration in float64."""
    rng = np.random.default_rng(11)
    rows, c0, c1, nc = 700, 24, 56, 11
    x = rng.standard_normal((rows, c0))
    shapes = [(c0, c1), (c1,), (c1, 2 * 40), (80,), (40, c1), (c1,), (c1, nc), (nc,)]
    par = [rng.standard_normal(s) * (s[0] ** -0.5 if len(s) == 2 else 0.1) for s in shapes]
    x, par = np.float32(x), [np.float32(p) for p in par]
    labels = rng.integers(0, nc, rows).astype(np.int32)
    X, W = torch.as_tensor(x).cuda(), [torch.as_tensor(p).cuda() for p in par]
    V = [torch.zeros_like(w) for w in W]

    h, _ = oc.oc_dense_fwd(X, W[0], W[1], act=oc.OC_ACT_GELU, need_pre=False)
    h, p0 = oc.oc_dense_fwd(X, W[0], W[1], act=oc.OC_ACT_GELU, need_pre=True)
    m, p1 = oc.oc_glu_fwd(h, W[2], W[3], act=oc.OC_ACT_SILU, need_pre=True)
    y, _ = oc.oc_dense_fwd(m, W[4], W[5], res=h)
    z, _ = oc.oc_dense_fwd(y, W[6], W[7])
    loss, dz = oc.oc_softmax_ce(z, torch.as_tensor(labels).cuda())
    dy, g6, g7 = oc.oc_dense_bwd(y, W[6], dz)
    dm, g4, g5 = oc.oc_dense_bwd(m, W[4], dy)
    dh, g2, g3 = oc.oc_glu_bwd(h, W[2], dm, p1)
    dh = dh + dy
    _, g0, g1 = oc.oc_dense_bwd(X, W[0], dh, act=oc.OC_ACT_GELU, pre=p0, need_dx=False)
    grads = [g0, g1, g2, g3, g4, g5, g6, g7]
    raw = [g.clone() for g in grads]
    norm = oc.oc_grad_clip(grads, 0.05)
    for w, g, v in zip(W, grads, V):
        oc.oc_sgd(w, g, v, 0.1, 0.9, 5e-4)

    hr, z0 = D.dense_fwd(x, par[0], par[1], None, "gelu")
    mr, z1 = D.glu_fwd(hr, par[2], par[3], "silu")
    yr, _ = D.dense_fwd(mr, par[4], par[5], hr)
    zr, _ = D.dense_fwd(yr, par[6], par[7])
    lr, dzr = T.softmax_ce(zr, labels)
    dyr, r6, r7 = D.layer_bwd(yr, par[6], dzr)
    dmr, r4, r5 = D.layer_bwd(mr, par[4], dyr)
    dhr, r2, r3 = D.layer_bwd(hr, par[2], D.glu_dz(dmr, z1, "silu"))
    _, r0, r1 = D.layer_bwd(x, par[0], D.dense_dz(dhr + dyr, z0, "gelu"))
    ref = [r0, r1, r2, r3, r4, r5, r6, r7]
    assert abs(float(loss) - lr) <= 1e-5 * lr
    # four layers of at most 100 terms and one sum over 700 rows in fp32: each
    # adds some 2^-24 sqrt(terms) of the scale, 1e-5 of it covers them all
    for k, (g, r) in enumerate(zip(raw, ref)):
        assert np.linalg.norm(_np(g) - r) <= 1e-5 * np.linalg.norm(r), k
    n, clipped = D.grad_clip(ref, 0.05)
    assert n > 0.05 and abs(float(norm) - n) <= 1e-5 * n
    for w, p, g in zip(W, par, clipped):
        wr, _ = T.sgd_step(p, g, np.zeros_like(g), 0.1, 0.9, 5e-4)
        assert np.abs(_np(w) - wr).max() <= 1e-6 * (1 + np.abs(wr).max())
