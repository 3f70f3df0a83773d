"""Layer norm and the residual step with several rows a workgroup, and every option of
the step at every kernel variant, against the float64 oracle with the bounds of
test_gpu_rows."""
import numpy as np
import pytest
import torch

import paper_1712_01537_amd as oc
from oracle import rows as R
from test_gpu_rows import (BF16, DT, F32, STEPS, U, _np, check_bwd, check_stats, check_y, make,
                           near, rng_of, v_of)

pytestmark = pytest.mark.gpu


def check_step(rows, c, dt, p, with_res, with_dh, affine, seed):
    step, site, eps = 3, 9, 1e-2
    x = make((rows, c), dt, seed, 2.0, 1) + make((rows, 1), dt, seed + 1, 3.0)
    res = make((rows, c), dt, seed + 2) if with_res else None
    dy = make((rows, c), dt, seed + 3)
    dh = make((rows, c), dt, seed + 4, 1.0, 1) if with_dh else None
    gamma = make((c,), F32, seed + 5) if affine else None
    beta = make((c,), F32, seed + 6) if affine else None
    rng = rng_of(seed, step)
    keep, q = (None, 1.0) if p == 0 else R.mask(rows, c, p, seed, step, site)
    xd = _np(x) if p == 0 else np.where(keep, _np(x) / q, 0.0)
    hw = xd if res is None else xd + _np(res)
    h, y, mean, invstd = oc.oc_drop_ln_fwd(x, res, p, rng, gamma, beta, site=site, eps=eps,
                                           need_stats=True)
    # (as in test_gpu_rows: dropout's two roundings and its scale's, and the sum's)
    herr = U * (3 * np.abs(xd) * (p > 0) + np.abs(hw) * with_res)
    near(h, hw, 1.01 * herr + v_of(dt) * np.abs(hw), "h")
    _, r = R.stats(hw, eps)
    z = np.abs(R.ln_fwd(hw, None, None, eps)[0])
    most = herr.max(1, keepdims=True)
    check_y(y, hw, _np(gamma), _np(beta), eps, dt, "y", extra=r[:, None] * (2 + z) * most)
    check_stats(mean, invstd, hw, eps, "stats", err=most[:, 0])
    got = oc.oc_drop_ln_bwd(x, res, dy, p, rng, gamma, mean, invstd, dh=dh, site=site)
    check_bwd(hw, _np(dy), _np(dh), _np(gamma), _np(invstd), dt, got, "bwd", keep, q, herr)


# a width for each number of waves a row, and rows for three or more a workgroup of the
# forward on 256 CUs
MANY = [(8000, 1100), (4000, 2304), (1700, 4100), (800, 8200), (800, 16384), (600, 16385)]


@DT
@pytest.mark.parametrize("rows,c", MANY)
def test_ln_of_many_rows_is_that_of_few(rows, c, dt):
    """Against the oracle, and bit for bit against the same rows in calls that have a row
    a workgroup."""
    x, dy = make((rows, c), dt, 1, 2.0) + make((rows, 1), dt, 2, 3.0), make((rows, c), dt, 3)
    gamma, beta = make((c,), F32, 4), make((c,), F32, 5)
    y, mean, invstd = oc.oc_ln_fwd(x, gamma, beta, need_stats=True)
    check_y(y, _np(x), _np(gamma), _np(beta), 1e-5, dt, "y")
    check_stats(mean, invstd, _np(x), 1e-5, "stats")
    h, y2, mean2, invstd2 = oc.oc_drop_ln_fwd(x, dy, 0.0, None, gamma, beta, need_stats=True)
    for r in range(0, rows, 200):
        s = slice(r, r + 200)
        few = oc.oc_ln_fwd(x[s], gamma, beta, need_stats=True)
        assert all(torch.equal(a[s], b) for a, b in zip((y, mean, invstd), few)), r
        few = oc.oc_drop_ln_fwd(x[s], dy[s], 0.0, None, gamma, beta, need_stats=True)
        assert all(torch.equal(a[s], b) for a, b in zip((h, y2, mean2, invstd2), few)), r
    dx, dg, db = oc.oc_ln_bwd(x, dy, gamma, mean, invstd)
    check_bwd(_np(x), _np(dy), None, _np(gamma), _np(invstd), dt, (None, dx, dg, db), "bwd")
    for r in range(0, rows, 200):
        s = slice(r, r + 200)
        few = oc.oc_ln_bwd(x[s], dy[s], gamma, mean[s], invstd[s], need_dgamma=False,
                           need_dbeta=False)[0]
        assert torch.equal(dx[s], few), r


@DT
@pytest.mark.parametrize("rows,c", MANY)
def test_step_of_many_rows(rows, c, dt):
    check_step(rows, c, dt, 0.25, True, True, True, 11)


# 1 to 64 lanes, 2 to 8 waves, two and four vectors a thread, rows in no registers; rows
# for several a workgroup of the backward
VARIANTS = [(600, 5), (600, 24), (300, 130), (100, 500), (50, 1000), (50, 2000), (30, 4000),
            (9, 5000), (9, 8192), (9, 8200), (5, 12000), (5, 16384), (5, 17000)]


@DT
@pytest.mark.parametrize("rows,c", VARIANTS)
@pytest.mark.parametrize("i", range(len(STEPS)))
def test_every_option_at_every_variant(i, rows, c, dt):
    check_step(rows, c, dt, *STEPS[i], 20 + i)


@pytest.mark.parametrize("i", range(len(STEPS)))
def test_every_option_of_three_vectors_a_thread(i):
    """bf16 rows of 513 to 3000 channels that leave a quarter of one vector's lanes idle."""
    check_step(8300, 2100, BF16, *STEPS[i], 30 + i)
