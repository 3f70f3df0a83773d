"""GPU tests of the dense layers and of clipping at their edges: operands that are not
finite or far from 1, small results, long sums, overlapping outputs, calls from two threads.

Bounds as in test_gpu_dense.py (u = 2^-24): a sum of R products in fp32, in any order, is
off by at most (R + 4) u S, S the sum of the products' absolute values."""
import math

import pytest
import torch

import paper_1712_01537_amd as oc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def normal(shape, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(generator=g) * scale


def product_check(got, a, b, what):
    """got against a b in 64 bits: NaN and infinities where those are, else within the
    bound."""
    ref = a.double() @ b.double()
    tol = (a.shape[1] + 4) * U * (a.double().abs() @ b.double().abs())
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what
    inf = torch.isinf(ref)
    assert torch.equal(got[inf].double(), ref[inf]), what
    fin = torch.isfinite(ref)
    assert ((got.double() - ref)[fin].abs() <= tol[fin]).all(), what


# Sizes of every tile shape, with whole and shared reductions and ragged edges.
ODD = [(70, 37, 50), (300, 72, 65), (517, 130, 259), (2100, 96, 200), (1300, 520, 1031),
       (9000, 48, 130), (12000, 515, 260)]


@pytest.mark.parametrize("rows,cin,cout", ODD)
def test_fp32_operands_that_no_parts_hold(rows, cin, cout):
    """Infinities, NaN and values of 2^110 here and there: each result is what its own
    sum is in fp32, in y, dx and dw."""
    x, w = normal((rows, cin), 1), normal((cin, cout), 2, cin ** -0.5)
    dy = normal((rows, cout), 3)
    for t, big in ((x, 2.0 ** 110), (w, 2.0 ** -12), (dy, -(2.0 ** 12))):
        at = torch.randint(0, t.numel(), (3,), generator=torch.Generator().manual_seed(rows))
        t.view(-1)[at[0]] = big
        t.view(-1)[at[1]] = -math.inf
        t.view(-1)[at[2]] = math.nan
    x[rows - 1, cin - 1] = 2.0 ** 110
    y, _ = oc.oc_dense_fwd(x, w)
    product_check(y, x, w, "y")
    dx, dw, _ = oc.oc_dense_bwd(x, w, dy)
    product_check(dx, dy, w.t().contiguous(), "dx")
    product_check(dw, x.t().contiguous(), dy, "dw")
    if cout % 2 == 0:  # gated: y = g u with no activation
        z = x.double() @ w.double()
        ref = z[:, :cout // 2] * z[:, cout // 2:]
        got = oc.oc_glu_fwd(x, w, act=oc.OC_ACT_NONE)[0]
        # (a product of two sums of 2^110 and more passes fp32's largest value)
        ref = torch.where(ref.abs() > 3.4e38, ref.sign() * math.inf, ref)
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        assert torch.equal(torch.isinf(got), torch.isinf(ref))


def micros(f):
    f()
    best = math.inf
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3)
    return best


def test_one_nan_weight_does_not_hold_up_a_layer():
    """Forming a column's results again is a few times the layer's work at most (one
    lane a result took 40 times the forward and 30 times the backward)."""
    x, w, dy = normal((8192, 256), 1), normal((256, 512), 2, 0.0625), normal((8192, 512), 3)
    for f in (lambda: oc.oc_dense_fwd(x, w), lambda: oc.oc_dense_bwd(x, w, dy)):
        w[3, 5] = 0.5
        plain = micros(f)
        w[3, 5] = math.nan
        assert micros(f) <= 10 * plain


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [6, 40_000])
def test_gelu_keeps_the_digits_of_small_values(rows, dt):
    """z Phi(z) and its slope relative to themselves at negative z.  One channel of weight
    1 makes z exactly x, and dx exactly dz = dy act'(z) with dy = 1.

    Phi(-|z|) is off by at most (22 + 1.5 z^2) u of itself: the reciprocal and its operand
    3 u, stretched by at most 0.8 / 0.3; the fit 3 u; eight steps of a polynomial whose
    terms sum to at most twice its value 5 u; e^(-z^2/2) 2 u and 3 u of z^2 / 2; products
    2 u.  y adds one more rounding, the slope's two terms two each."""
    x = -torch.linspace(0.02, 12.0, rows, device="cuda")[:, None].to(dt)
    one, dy = torch.ones((1, 1), device="cuda", dtype=dt), torch.ones_like(x)
    z = x.double()
    phi = torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    tail = 0.5 * torch.special.erfc(-z * math.sqrt(0.5))
    rnd = 2.0 ** -8 if dt == torch.bfloat16 else 0.0
    rel = (24 + 2 * z * z) * U
    y, pre = oc.oc_dense_fwd(x, one, act=oc.OC_ACT_GELU, need_pre=True, again=False)
    ref = z * tail
    assert ((y.double() - ref).abs() <= (rel + rnd + rel * rnd) * ref.abs()).all()
    for kept in (pre, oc.Again(None)):
        dx, dw, db = oc.oc_dense_bwd(x, one, dy, act=oc.OC_ACT_GELU, pre=kept)
        ref = tail + z * phi
        off = rel * (tail + z.abs() * phi)
        # (bf16: dz is rounded, dx holds it)
        assert ((dx.double() - ref).abs() <= off + rnd * (ref.abs() + off)).all()


@pytest.mark.parametrize("most", [0.1, 1e-6, 1e-20])
@pytest.mark.parametrize("size", [1e37, 1e38, 3e38])
def test_clipping_of_huge_gradients(size, most):
    """max_norm / norm lies below fp32's normal numbers, or below all of its numbers,
    while the clipped values are ordinary: off by the rounding of the factor and of the
    product (in fp32 by 2 u, in double by 1)."""
    n = 10_007
    g = torch.Generator("cuda").manual_seed(1)
    base = [torch.empty(n, device="cuda").uniform_(-1, 1, generator=g) * size,
            normal(300, 2, size / 8).to(torch.bfloat16), torch.full((3,), size, device="cuda")]
    norm = torch.cat([g.double() for g in base]).norm()
    for place in (False, True):
        grads = [g.clone() for g in base]
        outs = grads if place else [torch.empty(g.numel(), device="cuda") for g in grads]
        oc.oc_grad_clip(grads, most, outs=None if place else outs)
        for g, o in zip(base, outs):
            ref = g.double() * (most / norm)
            rnd = 2.0 ** -8 if o.dtype == torch.bfloat16 else 0.0
            # (values below fp32's normal numbers are off by half of its smallest one)
            assert ((o.double() - ref).abs() <= (2.1 * U + rnd) * ref.abs() + 1e-45).all()


def test_dbias_of_very_many_rows():
    """At most 64 values are added up in fp32 (63 roundings), the rest in double (each
    partial sum and the result rounded once).  The value is one whose sum in fp32 loses
    2^-16 with every term from the 256th on: 500 in a row are off by 125 u."""
    rows = 500 * 2048 * 256
    v = 1.0 + 2.0 ** -16 - 2.0 ** -23
    x = torch.zeros((rows, 1), device="cuda")
    dy = torch.full((rows, 1), v, device="cuda")
    db = oc.oc_dense_bwd(x, x[:1], dy, need_dx=False, need_dw=False)[2]
    assert abs(float(db.double()) - rows * v) <= 65 * U * rows * v


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cin,cout", [(3, 16, 24), (300, 40, 72), (1100, 33, 65)])
def test_relu_masks_what_is_not_finite(rows, cin, cout, dt):
    """Infinities and NaN in dy where the unit is not active leave the bits of zeros
    there, from the forward's bits, its output or x w + b formed again."""
    x, w = normal((rows, cin), 1).to(dt), normal((cin, cout), 2, cin ** -0.5).to(dt)
    dy = normal((rows, cout), 3).to(dt)
    y, bits = oc.oc_dense_fwd(x, w, act=oc.OC_ACT_RELU, need_pre=True, again=False)
    off = y == 0
    zero, bad = dy.masked_fill(off, 0.0), dy.masked_fill(off, math.inf)
    bad[off & (torch.arange(cout, device="cuda") % 3 == 0)] = math.nan
    for pre in (bits, y, oc.Again(None)):
        want = oc.oc_dense_bwd(x, w, zero, act=oc.OC_ACT_RELU, pre=pre)
        got = oc.oc_dense_bwd(x, w, bad, act=oc.OC_ACT_RELU, pre=pre)
        assert all(torch.isfinite(p).all() and torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cin,cout", [(3, 16, 24), (300, 40, 72), (1100, 33, 65)])
def test_gated_relu_masks_what_is_not_finite(rows, cin, cout, dt):
    """A dy u that passes the largest value, where the gate is not active."""
    x, w = normal((rows, cin), 1).to(dt), normal((cin, 2 * cout), 2, cin ** -0.5).to(dt)
    w[:, cout:] *= 2.0 ** 65
    dy = normal((rows, cout), 3).to(dt)
    pre = oc.oc_glu_fwd(x, w, act=oc.OC_ACT_RELU, need_pre=True, again=False)[1]
    off = pre[:, :cout] < -0.01  # (formed again, a value next to 0 may change sides)
    dy = torch.where(off, dy * 2.0 ** 75, torch.zeros_like(dy))
    assert torch.isinf(dy.float() * pre[:, cout:]).any()
    for kept in (pre, oc.Again(None)):
        for g in oc.oc_glu_bwd(x, w, dy, kept, act=oc.OC_ACT_RELU):
            assert (g == 0).all()


def test_clipping_into_views():
    """Views that overlap are refused and untouched; views end to end and a gradient
    listed twice are not."""
    buf = torch.full((1000,), 2.0, device="cuda")
    for grads, outs in (([buf[:600], buf[599:]], None), ([buf[:500]], [buf[1:501]]),
                        ([buf[:10], buf[500:510]], [buf[20:30], buf[29:39]]),
                        ([buf[:10], buf[500:510]], [buf[505:515], buf[20:30]])):
        with pytest.raises(oc.OcError):
            oc.oc_grad_clip(grads, 1.0, outs=outs)
    assert (buf == 2.0).all()
    out = torch.zeros(600, device="cuda")
    norm = oc.oc_grad_clip([buf[:300], buf[:300]], 1.0, outs=[out[:300], out[300:]])
    want = math.sqrt(600 * 4.0)
    assert abs(float(norm) - want) <= 1.01 * U * want
    assert ((out.double() - 2.0 / want).abs() <= 2.1 * U * 2.0 / want).all()
    assert (buf == 2.0).all()
    oc.oc_grad_clip([buf[:600], buf[600:]], 1.0)
    want = 2.0 / math.sqrt(4000.0)
    assert ((buf.double() - want).abs() <= 2.1 * U * want).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cin,cout", [(2, 96, 40), (70, 160, 72), (600, 520, 264),
                                           (5000, 520, 1032), (300, 75, 67)])
def test_what_is_not_finite_stays_in_its_row_and_column(rows, cin, cout, dt):
    """Values are split in parts one by one: next to an infinity or NaN every other row's
    and column's bits are as they were, its neighbours' too."""
    x, w = normal((rows, cin), 1).to(dt), normal((cin, cout), 2, cin ** -0.5).to(dt)
    dy = normal((rows, cout), 3).to(dt)
    y0, (dx0, dw0, db0) = oc.oc_dense_fwd(x, w)[0], oc.oc_dense_bwd(x, w, dy)
    r, k, n = rows - 1, cin // 2, cout - 1
    x[r, k], dy[r, n] = math.inf, math.nan
    y, (dx, dw, db) = oc.oc_dense_fwd(x, w)[0], oc.oc_dense_bwd(x, w, dy)
    i, j, m = (torch.arange(v, device="cuda") for v in (rows, cin, cout))
    assert torch.equal(y[i != r], y0[i != r]) and torch.equal(dx[i != r], dx0[i != r])
    assert torch.equal(db[m != n], db0[m != n])
    assert torch.equal(dw[j != k][:, m != n], dw0[j != k][:, m != n])
    assert torch.isnan(dx[r]).all() and torch.isnan(dw[:, n]).all() and torch.isnan(db[n])
    assert torch.isinf(y[r]).all() and torch.isinf(dw[k, m != n]).all()


def test_two_threads():
    """Calls from two threads at once, each on a stream of its own, over sizes whose plans
    both threads work out: the bits of a single thread."""
    import threading

    sizes = [(300 + 64 * i, 40 + 24 * (i % 5), 96 + 8 * i) for i in range(12)]
    data = [(normal((r, k), i).to(t), normal((k, 2 * n), i + 50, k ** -0.5).to(t), normal((r, n), i + 99).to(t))
            for t in (torch.float32, torch.bfloat16) for i, (r, k, n) in enumerate(sizes)]

    def step(x, w, dy):
        y, pre = oc.oc_glu_fwd(x, w, need_pre=True)
        dx, dw, db = oc.oc_glu_bwd(x, w, dy, pre)
        outs = [torch.empty_like(g) for g in (dw, db)]
        return (y, dx, dw, db, oc.oc_grad_clip([dw, db], 0.5, outs=outs), *outs)

    want = [step(*d) for d in data]
    torch.cuda.synchronize()
    failed = []

    def work(order):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(5):
                    got = [(i, step(*data[i])) for i in order]
                    torch.cuda.current_stream().synchronize()
                    for i, g in got:
                        if not all(torch.equal(p, q) for p, q in zip(want[i], g)):
                            failed.append(i)
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=(o,))
               for o in (list(range(len(data))), list(reversed(range(len(data)))))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
