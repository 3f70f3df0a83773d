"""Layer norm and the residual step on values far from 1, against the float64
oracle with the bounds of test_gpu_rows (counted from the roundings, relative to
each value: nothing in them depends on the rows' size)."""
import pytest
import torch

import paper_1712_01537_amd as oc
from test_gpu_rows import DT, F32, _np, check_bwd, check_stats, check_y, make, rng_of

pytestmark = pytest.mark.gpu

# every number of waves a row: lanes of one wave, 2 to 16 waves, rows in no registers
WIDTHS = [24, 512, 1000, 2048, 4096, 8200, 16384, 17000, 65536]


def far_rows(c, dt, power, seed):
    """Deviations up to 2^power: uniform ones, the two ends in turn, and one end in a
    row's first half, the other in its second (the waves' means differ most)."""
    x = make((6, c), F32, seed).remainder(2.0) - 1.0
    x[2:4] = 1.0
    x[2, ::2] = -1.0
    x[3, c // 2:] = -1.0
    return x.mul_(2.0 ** power).to(dt)


@DT
@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("power", [-40, 56, 58, 60, 62])
def test_deviations_up_to_the_stated_limit(c, dt, power):
    """The squares of a row's deviations are added as shares of their mean, which stays
    in range up to deviations of 2^63 however wide the row is (a plain sum of squares
    overflows from 2^64 / sqrt(c) on)."""
    eps = 1e-5 if power > 0 else 1e-26
    x, dy = far_rows(c, dt, power, c), make((6, c), dt, c + 1)
    gamma, beta = make((c,), F32, 3), make((c,), F32, 4)
    y, mean, invstd = oc.oc_ln_fwd(x, gamma, beta, eps, need_stats=True)
    check_y(y, _np(x), _np(gamma), _np(beta), eps, dt, "y")
    check_stats(mean, invstd, _np(x), eps, "stats")
    dx, dg, db = oc.oc_ln_bwd(x, dy, gamma, mean, invstd)
    check_bwd(_np(x), _np(dy), None, _np(gamma), _np(invstd), dt, (None, dx, dg, db), "bwd")
    # the residual step: the same rows as the sum of their halves
    rng, half = rng_of(1, 2), x * 0.5  # (exact)
    h, y2, mean2, invstd2 = oc.oc_drop_ln_fwd(half, half.clone(), 0.0, rng, gamma, beta, eps=eps,
                                              need_stats=True)
    assert torch.equal(h, x)
    check_y(y2, _np(x), _np(gamma), _np(beta), eps, dt, "step's y")
    check_stats(mean2, invstd2, _np(x), eps, "step's stats")
    got = oc.oc_drop_ln_bwd(half, half.clone(), dy, 0.0, rng, gamma, mean, invstd)
    check_bwd(_np(x), _np(dy), None, _np(gamma), _np(invstd), dt, got, "step's bwd")


@DT
@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("power,grad", [(62, 66), (62, -60), (-40, 80), (0, 110)])
def test_gradients_as_large_as_the_deviations(c, dt, power, grad):
    """dx is of the size of dy invstd; no sum on the way to it is of the size of dy times
    the deviations (2^62 2^66 is past fp32, dx itself some 2^4)."""
    eps = 1e-5 if power >= 0 else 1e-26
    x, dy = far_rows(c, dt, power, c), far_rows(c, dt, grad, c + 1).flip(0).contiguous()
    gamma = make((c,), F32, 3)
    _, mean, invstd = oc.oc_ln_fwd(x, gamma, None, eps, need_stats=True)
    dx, dg, db = oc.oc_ln_bwd(x, dy, gamma, mean, invstd)
    check_bwd(_np(x), _np(dy), None, _np(gamma), _np(invstd), dt, (None, dx, dg, db), "bwd")
    half, rng = x * 0.5, rng_of(1, 2)
    got = oc.oc_drop_ln_bwd(half, half.clone(), dy, 0.0, rng, gamma, mean, invstd)
    check_bwd(_np(x), _np(dy), None, _np(gamma), _np(invstd), dt, got, "step's bwd")
