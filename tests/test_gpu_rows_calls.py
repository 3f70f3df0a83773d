"""Calls of the row operators that the header allows, through the binding."""
import pytest
import torch

import paper_1712_01537_amd as oc
from test_gpu_rows import DT, F32, make, rng_of

pytestmark = pytest.mark.gpu


@DT
def test_a_ratio_that_keeps_everything_needs_no_state(dt):
    """Of T = (1 - p) 2^32 rounded, a ratio below 2^-33 leaves 2^32: no mask is drawn."""
    x, res, dy = (make((37, 130), dt, i) for i in range(3))
    for p in (0.0, 0, 1e-12, 2.0 ** -34):
        assert torch.equal(oc.oc_dropout_rng(x, p, None), x)
        want = oc.oc_drop_ln_fwd(x, res, 0.0, rng_of(1, 2), need_stats=True)
        got = oc.oc_drop_ln_fwd(x, res, p, None, need_stats=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        back = [oc.oc_drop_ln_bwd(x, res, dy, q, r, None, want[2], want[3])
                for q, r in ((0.0, rng_of(1, 2)), (p, None))]
        assert all(torch.equal(a, b) for a, b in zip(*back))
    for p in (2.0 ** -32, 0.5):
        for call in (lambda: oc.oc_dropout_rng(x, p, None),
                     lambda: oc.oc_drop_ln_fwd(x, res, p, None),
                     lambda: oc.oc_drop_ln_bwd(x, res, dy, p, None, None, want[2], want[3])):
            with pytest.raises(oc.OcError, match="generator state"):
                call()
