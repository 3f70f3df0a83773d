"""The gradient of table rows adds the rows of one id in their order, whichever sort
brought them together."""
import pytest
import torch

import paper_1712_01537_amd as oc
from test_gpu_rows import DT

pytestmark = pytest.mark.gpu

# fp32 sums in this order are 1: 2^24 + 1 is 2^24 again.  In another order of the four, or
# of two neighbours, they are 0, 1 or 2.
FOUR = (2.0 ** 24, 1.0, -(2.0 ** 24), 1.0)


def spread(ids, dy, seed):
    """The rows at random places, those of one id in the same order."""
    g = torch.Generator().manual_seed(seed)
    ids2 = ids[torch.randperm(len(ids), generator=g)]
    at = torch.sort(ids2, stable=True)[1]
    dy2 = torch.empty_like(dy)
    dy2[at] = dy[torch.sort(ids, stable=True)[1]]
    return ids2, dy2


# ids with four rows each, the table's rows: the sort in LDS with one to three digits, and
# that of one to three digits over many workgroups
@DT
@pytest.mark.parametrize("used,num", [(100, 101), (1000, 1024), (1024, 70_000), (1000, 1 << 27),
                                      (1100, 500_000), (3000, 3000), (16_000, 16_384),
                                      (60_000, 1 << 20), (300_000, 300_000)])
def test_rows_of_an_id_keep_their_order(used, num, dt):
    step = num // used
    ids = (torch.arange(used, dtype=torch.int32) * step).repeat_interleave(4)
    dy = torch.tensor(FOUR).repeat(used).unsqueeze(1).repeat(1, 3).contiguous()
    ids2, dy2 = spread(ids, dy, used)
    c = 3 if num < 1 << 24 else 1
    got = oc.oc_embed_bwd(ids2.cuda(), dy2[:, :c].contiguous().to(dt).cuda(), num)
    assert (got[torch.arange(used, device="cuda") * step] == 1.0).all()
    assert float(got.sum(dtype=torch.float64)) == used * c  # (the others are 0)


@DT
@pytest.mark.parametrize("rows,num,c", [(4000, 3, 5), (9000, 700, 40), (50_000, 5, 9),
                                        (200_000, 1000, 64), (300_000, 2, 600)])
def test_long_runs_are_added_in_their_order(rows, num, c, dt):
    """The bits are those of the same rows sorted beforehand."""
    g = torch.Generator().manual_seed(rows)
    ids = (torch.rand(rows, generator=g) ** 3 * num).to(torch.int32).sort()[0]
    dy = (torch.randn(rows, c, generator=g) * torch.exp(4 * torch.randn(rows, 1, generator=g)))
    ids2, dy2 = spread(ids, dy, 1)
    a = oc.oc_embed_bwd(ids.cuda(), dy.to(dt).cuda(), num)
    b = oc.oc_embed_bwd(ids2.cuda(), dy2.to(dt).cuda(), num)
    assert torch.equal(a, b)
