"""The row operators' oracle against published values, torch in float64 and
differences; and the operators' refusals, which need no GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_1712_01537_amd as oc
from oracle import rows as R

# Known answers of Philox4x32-10, as published with the generator.
KNOWN = [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
]


@pytest.mark.parametrize("counter,key,words", KNOWN)
def test_philox_known_answers(counter, key, words):
    assert tuple(int(w) for w in R.philox(np.array(counter, np.uint64), key)) == words


def test_numbers_are_uniform_and_apart():
    a = R.numbers(512, 1000, 77, 3, 1).astype(np.float64)
    n = a.size
    # mean and variance of n uniform numbers, six deviations
    assert abs(a.mean() / 2 ** 32 - 0.5) < 6 * np.sqrt(1 / 12 / n)
    assert abs(np.square(a / 2 ** 32 - 0.5).mean() - 1 / 12) < 6 * np.sqrt(1 / 180 / n)
    for other in ((78, 3, 1), (77, 4, 1), (77, 3, 2), (77 + (1 << 32), 3, 1),
                  (77, 3 + (1 << 32), 1)):
        b = R.numbers(512, 1000, *other).astype(np.float64)
        assert abs(np.corrcoef(a.ravel(), b.ravel())[0, 1]) < 6 / np.sqrt(n)
    low = R.numbers(512, 1000, 77, 3, 1) & np.uint64(0xFFFF)
    assert abs(low.astype(np.float64).mean() / 65536 - 0.5) < 6 * np.sqrt(1 / 12 / n)


@pytest.mark.parametrize("p", [0.0, 1e-12, 0.1, 0.5, 0.99999])
def test_share_kept(p):
    keep, q = R.mask(700, 1001, p, 5, 6)
    assert abs(q - (1 - p)) <= 2.0 ** -33
    assert abs(keep.mean() - q) <= 6 * np.sqrt(q * (1 - q) / keep.size)


@pytest.mark.parametrize("rows,c", [(1, 1), (3, 2), (5, 17), (2, 300)])
@pytest.mark.parametrize("affine", [False, True])
def test_ln_matches_autograd(rows, c, affine):
    g = torch.Generator().manual_seed(rows * 1000 + c)
    x, dy = (torch.randn(rows, c, generator=g, dtype=torch.float64) for _ in range(2))
    w, b = (torch.randn(c, generator=g, dtype=torch.float64) for _ in range(2))
    leaves = [t.requires_grad_() for t in ((x, w, b) if affine else (x,))]
    y = torch.nn.functional.layer_norm(x, (c,), *(leaves[1:] or (None, None)), 1e-3)
    want = torch.autograd.grad(y, leaves, dy)
    gamma, beta = (w.detach().numpy(), b.detach().numpy()) if affine else (None, None)
    got, _, r = R.ln_fwd(x.detach().numpy(), gamma, beta, 1e-3)
    np.testing.assert_allclose(got, y.detach().numpy(), rtol=1e-12, atol=1e-12)
    grads = R.ln_bwd(x.detach().numpy(), dy.numpy(), gamma, r)
    for a, e in zip(grads, want):
        np.testing.assert_allclose(a, e.numpy(), rtol=1e-9, atol=1e-9 * float(r.max()))


def test_ln_matches_differences():
    rng = np.random.default_rng(3)
    x, dy, w = rng.normal(size=(4, 9)), rng.normal(size=(4, 9)), rng.normal(size=9)
    _, _, r = R.ln_fwd(x, w, None, 1e-2)
    dx = R.ln_bwd(x, dy, w, r)[0]
    step = 1e-6
    for i, j in ((0, 0), (1, 8), (3, 4)):
        hi, lo = x.copy(), x.copy()
        hi[i, j] += step
        lo[i, j] -= step
        d = ((R.ln_fwd(hi, w, None, 1e-2)[0] - R.ln_fwd(lo, w, None, 1e-2)[0]) * dy).sum()
        assert abs(d / (2 * step) - dx[i, j]) < 1e-8


def test_embed_matches_autograd():
    g = torch.Generator().manual_seed(4)
    table = torch.randn(7, 5, generator=g, dtype=torch.float64, requires_grad=True)
    ids = torch.tensor([3, 0, 3, -1, 6, 3, 7, 0])
    there = (ids >= 0) & (ids < 7)
    y = torch.where(there[:, None], table[ids.clamp(0, 6)] * 1.5, torch.zeros((), dtype=torch.float64))
    dy = torch.randn(8, 5, generator=g, dtype=torch.float64)
    (want,) = torch.autograd.grad(y, table, dy)
    np.testing.assert_allclose(R.embed_fwd(ids, table.detach(), 1.5), y.detach(), rtol=1e-14)
    np.testing.assert_allclose(R.embed_bwd(ids, dy, 7, 1.5), want, rtol=1e-13, atol=1e-13)


# --- refusals of the C entries: nothing is enqueued, so no GPU is needed ------

F32, BF16 = 0, 1
BASE = 1 << 40  # addresses that nothing reads


def _at(i):
    return C.c_void_p(BASE + i * (1 << 30))


def _ln_fwd(dt=F32, rows=4, c=8, x=1, gamma=2, beta=3, eps=1e-5, y=4, mean=5, invstd=6):
    a = [None if v is None else _at(v) for v in (x, gamma, beta, y, mean, invstd)]
    return oc.load().oc_ln_fwd(dt, rows, c, a[0], a[1], a[2], eps, a[3], a[4], a[5], None)


def _ln_bwd(dt=F32, rows=4, c=8, x=1, dy=2, gamma=3, mean=4, invstd=5, dx=6, dg=7, db=8, ws=9,
            ws_bytes=1 << 20):
    a = [None if v is None else _at(v) for v in (x, dy, gamma, mean, invstd, dx, dg, db, ws)]
    return oc.load().oc_ln_bwd(dt, rows, c, *a, ws_bytes, None)


def _drop(dt=F32, rows=4, c=8, x=1, p=0.5, rng=2, site=0, y=3):
    a = [None if v is None else _at(v) for v in (x, rng, y)]
    return oc.load().oc_dropout_rng(dt, rows, c, a[0], p, a[1], site, a[2], None)


def _drop_ln_fwd(dt=F32, rows=4, c=8, x=1, res=2, p=0.5, rng=3, site=0, gamma=4, beta=5,
                 eps=1e-5, h=6, y=7, mean=8, invstd=9):
    a = [None if v is None else _at(v) for v in (x, res, rng, gamma, beta, h, y, mean, invstd)]
    return oc.load().oc_drop_ln_fwd(dt, rows, c, a[0], a[1], p, a[2], site, a[3], a[4], eps,
                                    *a[5:], None)


def _drop_ln_bwd(dt=F32, rows=4, c=8, x=1, res=13, dy=2, dh=3, p=0.5, rng=4, site=0, gamma=5, mean=6,
                 invstd=7, dx=8, dres=9, dg=10, db=11, ws=12, ws_bytes=1 << 20):
    a = [None if v is None else _at(v)
         for v in (x, res, dy, dh, rng, gamma, mean, invstd, dx, dres, dg, db, ws)]
    return oc.load().oc_drop_ln_bwd(dt, rows, c, *a[:4], p, a[4], site, *a[5:],
                                    ws_bytes, None)


def _embed_fwd(dt=F32, flags=0, rows=4, num=3, c=8, ids=1, table=2, scale=1.0, y=3):
    a = [None if v is None else _at(v) for v in (ids, table, y)]
    return oc.load().oc_embed_fwd(dt, flags, rows, num, c, a[0], a[1], scale, a[2], None)


def _embed_bwd(dt=F32, flags=0, rows=100, num=3, c=8, ids=1, dy=2, scale=1.0, out_dt=F32, out=3,
               ws=4, ws_bytes=1 << 24):
    a = [None if v is None else _at(v) for v in (ids, dy, out, ws)]
    return oc.load().oc_embed_bwd(dt, flags, rows, num, c, a[0], a[1], scale, out_dt, a[2], a[3],
                                  ws_bytes, None)


NAN = float("nan")



REFUSED = [
    (_ln_fwd, dict(dt=2)), (_ln_fwd, dict(rows=-1)), (_ln_fwd, dict(rows=1 << 28)),
    (_ln_fwd, dict(c=0)), (_ln_fwd, dict(c=65537)), (_ln_fwd, dict(eps=0.0)),
    (_ln_fwd, dict(eps=NAN)), (_ln_fwd, dict(x=None)), (_ln_fwd, dict(y=None)),
    (_ln_fwd, dict(mean=1)), (_ln_fwd, dict(invstd=5)), (_ln_fwd, dict(y=2)),
    (_ln_bwd, dict(dt=-1)), (_ln_bwd, dict(x=None)), (_ln_bwd, dict(dy=None)),
    (_ln_bwd, dict(mean=None)), (_ln_bwd, dict(invstd=None)), (_ln_bwd, dict(ws=None)),
    (_ln_bwd, dict(ws_bytes=8)), (_ln_bwd, dict(dx=2)), (_ln_bwd, dict(dx=1)),
    (_ln_bwd, dict(dg=8)), (_ln_bwd, dict(ws=6)),
    (_drop, dict(dt=3)), (_drop, dict(c=0)), (_drop, dict(p=1.0)), (_drop, dict(p=-0.1)),
    (_drop, dict(p=NAN)), (_drop, dict(p=1 - 2.0 ** -40)), (_drop, dict(site=-1)),
    (_drop, dict(site=32768)), (_drop, dict(rng=None)), (_drop, dict(x=None)),
    (_drop, dict(y=None)), (_drop, dict(y=2)),
    (_drop_ln_fwd, dict(p=1.5)), (_drop_ln_fwd, dict(eps=-1.0)), (_drop_ln_fwd, dict(h=None)),
    (_drop_ln_fwd, dict(x=None)), (_drop_ln_fwd, dict(y=None)), (_drop_ln_fwd, dict(rng=None)),
    (_drop_ln_fwd, dict(h=1)), (_drop_ln_fwd, dict(y=2)), (_drop_ln_fwd, dict(h=7)),
    (_drop_ln_bwd, dict(p=1.0)), (_drop_ln_bwd, dict(x=None)), (_drop_ln_bwd, dict(dx=13)), (_drop_ln_bwd, dict(dx=9)),
    (_drop_ln_bwd, dict(dres=3)), (_drop_ln_bwd, dict(dx=2)), (_drop_ln_bwd, dict(rng=None)),
    (_drop_ln_bwd, dict(ws_bytes=0)), (_drop_ln_bwd, dict(site=1 << 20)),
    (_embed_fwd, dict(flags=2)), (_embed_fwd, dict(num=0)), (_embed_fwd, dict(num=1 << 28)),
    (_embed_fwd, dict(ids=None)), (_embed_fwd, dict(table=None)), (_embed_fwd, dict(y=2)),
    (_embed_bwd, dict(out_dt=BF16)), (_embed_bwd, dict(out=None)), (_embed_bwd, dict(ids=None)),
    (_embed_bwd, dict(dy=None)), (_embed_bwd, dict(ws=None)), (_embed_bwd, dict(ws_bytes=64)),
    (_embed_bwd, dict(out=2)), (_embed_bwd, dict(ws=3)), (_embed_bwd, dict(flags=-1)),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refused(i):
    call, change = REFUSED[i]
    assert call(**change) == 1, (call.__name__, change)
    assert oc.load().oc_last_error().decode()


def test_too_many_values_are_unsupported():
    assert _ln_fwd(rows=1 << 27, c=1 << 14) == 5
    assert _embed_fwd(num=1 << 27, c=1 << 14) == 5


def test_partial_overlaps_are_refused():
    L = oc.load()
    x = BASE
    for off in (4, 64, 4 * 31):  # y starts inside x
        assert L.oc_ln_fwd(F32, 4, 8, C.c_void_p(x), None, None, 1e-5, C.c_void_p(x + off), None,
                           None, None) == 1
        assert L.oc_dropout_rng(F32, 4, 8, C.c_void_p(x), 0.5, C.c_void_p(x + (1 << 30)), 0,
                                C.c_void_p(x + off), None) == 1
    assert L.oc_dropout_rng(F32, 4, 8, C.c_void_p(x), 0.5, C.c_void_p(x + (1 << 30) + 4), 0,
                            C.c_void_p(x + (1 << 29)), None) == 1  # state off 8 bytes


def test_no_rows_are_no_work():
    assert _ln_fwd(rows=0, x=None, y=None) == 0
    assert _drop(rows=0, x=None, y=None) == 0
    assert _drop_ln_fwd(rows=0, x=None, h=None, y=None) == 0
    assert _embed_fwd(rows=0, ids=None, y=None) == 0
    assert _ln_bwd(rows=0, dg=None, db=None) == 0
    assert _drop(p=1e-12, rng=None, x=1, y=1) == 0  # keeps everything, in place


def test_workspaces_grow_with_their_sizes():
    L = oc.load()
    assert L.oc_ln_bwd_workspace(-1, 8) == 0 and L.oc_ln_bwd_workspace(8, 0) == 0
    assert L.oc_embed_bwd_workspace(64, 8, 8) == 0  # few rows need none
    assert L.oc_embed_bwd_workspace(65, 8, 8) > 0
    # several digits need a second list; up to 4096 rows none is kept outside LDS
    assert L.oc_embed_bwd_workspace(10000, 1 << 20, 64) > L.oc_embed_bwd_workspace(10000, 4, 64)
    assert L.oc_embed_bwd_workspace(1000, 1 << 20, 64) == L.oc_embed_bwd_workspace(1000, 4, 64)


def test_binding_refuses_what_is_no_device_tensor():
    x = torch.zeros(2, 8)
    for call in (lambda: oc.oc_ln_fwd(x), lambda: oc.oc_dropout_rng(x, 0.5, None),
                 lambda: oc.oc_drop_ln_fwd(x, x, 0.0, None), lambda: oc.oc_ln_fwd([1.0]),
                 lambda: oc.oc_embed_fwd(torch.zeros(2, dtype=torch.int32), x),
                 lambda: oc.oc_embed_bwd(torch.zeros(2, dtype=torch.int32), x, 4),
                 lambda: oc.oc_ln_bwd(x, x, None, x[0], x[0]),
                 lambda: oc.oc_drop_ln_bwd(x, x, x, 0.0, None, None, x[0], x[0])):
        with pytest.raises(oc.OcError):
            call()
