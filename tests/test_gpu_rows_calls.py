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


@DT
@pytest.mark.parametrize("rows,c", [(33, 8), (70, 127), (600, 1024), (9, 5001), (3, 17000)])
def test_outputs_where_the_caller_says(rows, c, dt):
    """y in a tensor of the caller's, and in x's place; h in res's."""
    x, res, rng = make((rows, c), dt, 1), make((rows, c), dt, 2), rng_of(3, 4)
    gamma = make((c,), F32, 5)
    y, mean, invstd = oc.oc_ln_fwd(x, gamma, need_stats=True)
    out = torch.empty_like(x)
    got = oc.oc_ln_fwd(x, gamma, need_stats=True, y=out)
    assert got[0] is out and torch.equal(out, y)
    assert torch.equal(got[1], mean) and torch.equal(got[2], invstd)
    a = x.clone()
    assert oc.oc_ln_fwd(a, gamma, y=a)[0] is a and torch.equal(a, y)
    h, y, _, _ = oc.oc_drop_ln_fwd(x, res, 0.4, rng, gamma)
    got = oc.oc_drop_ln_fwd(x, res, 0.4, rng, gamma, y=out)
    assert got[1] is out and torch.equal(out, y) and torch.equal(got[0], h)
    a, b = x.clone(), res.clone()
    got = oc.oc_drop_ln_fwd(a, b, 0.4, rng, gamma, h=b, y=a)
    assert got[0] is b and got[1] is a and torch.equal(b, h) and torch.equal(a, y)
    for call in (lambda: oc.oc_ln_fwd(x, gamma, y=out[:1, :c // 2]),
                 lambda: oc.oc_ln_fwd(x, gamma, y=out.float() if dt != F32 else out.bfloat16()),
                 lambda: oc.oc_ln_fwd(x, gamma, y=out.cpu()),
                 lambda: oc.oc_drop_ln_fwd(x, res, 0.4, rng, gamma, y=res),
                 lambda: oc.oc_drop_ln_fwd(x, res, 0.4, rng, gamma, y=out, h=out)):
        with pytest.raises(oc.OcError):
            call()


def test_sizes_of_a_table_that_no_call_takes():
    """Refused before the gradient's memory is asked for."""
    ids, dy = torch.zeros(100, dtype=torch.int32, device="cuda"), make((100, 8), F32, 1)
    for num in (0, -1, 1 << 28, 1 << 40):
        for rows in (4, 100):
            with pytest.raises(oc.OcError, match="a table of"):
                oc.oc_embed_bwd(ids[:rows], dy[:rows], num)


@DT
def test_a_key_of_minus_one_is_the_last_place_of_depth_8(dt):
    """A key's 24 place bits name each row of a table of 8^8 rows, so no key lies outside
    it: -1 is the last place, in shape 255.  Smaller tables do not have that place."""
    keys = torch.tensor([-1, 0, 5 << 24, 0xFFFFFF] * 20, dtype=torch.int32, device="cuda")
    dy = torch.ones((80, 1), dtype=dt, device="cuda")
    for depth in (8, 7):
        num, last = 8 ** depth, 1.0 if depth == 8 else 0.0
        table = torch.full((num, 1), 2.0, dtype=dt, device="cuda")
        y = oc.oc_embed_fwd(keys, table, keys=True)
        assert y[:4, 0].tolist() == [2.0 * last, 2.0, 2.0, 2.0 * last]
        g = oc.oc_embed_bwd(keys, dy, num, keys=True)
        assert float(g[0]) == 40 and float(g[-1]) == 40 * last
        assert float(g.sum()) == 40 + 40 * last
