"""Lists that oc_grad_norm and oc_grad_clip refuse before any device work: outputs that
overlap, and what is no list."""
import ctypes as C

import pytest

import paper_1712_01537_amd as oc

F32, BF16 = 0, 1


def clip(grads, outs, counts, dts=None, out_dts=None):
    n = len(counts)
    dts = (C.c_int * n)(*(dts or [F32] * n))
    out_dts = (C.c_int * n)(*(out_dts or dts))
    counts = (C.c_int64 * n)(*counts)
    # (no workspace: a call whose outputs are in order is refused for that)
    return oc.load().oc_grad_clip(n, (C.c_void_p * n)(*grads), dts, counts, 1.0,
                                  (C.c_void_p * n)(*outs), out_dts, None, None, 0, None)


@pytest.mark.parametrize("grads,outs,counts,dts,out_dts", [
    ([4096, 8192], [4096, 4096], [5, 6], None, None),              # one address twice
    ([4096, 8192], [512, 528], [5, 6], None, None),                # the first's last value
    ([4096, 8192], [528, 512], [6, 5], None, None),                # out of order
    ([4096, 4112], [4096, 4112], [5, 6], None, None),              # in place, overlapping views
    ([4096, 8192], [8192, 512], [5, 6], None, None),               # another's gradient
    ([4096, 8192], [512, 4100], [5, 6], None, None),               # a piece of another's
    ([4096], [4100], [5], None, None),                             # its own, moved on
    ([4096], [4080], [5], None, None),
    ([4096, 8192], [4096, 4090], [5, 6], [F32, BF16], [F32, BF16]),
    ([4096, 8192], [512, 530], [5, 6], [BF16, BF16], [F32, F32]),  # fp32 outputs of bf16
    ([64, 4096, 8192], [64, 8210, 512], [0, 5, 10], None, None),
])
def test_overlaps(grads, outs, counts, dts, out_dts):
    assert clip(grads, outs, counts, dts, out_dts) == 1
    assert b"overlap" in oc.load().oc_last_error()


@pytest.mark.parametrize("grads,outs,counts,dts,out_dts", [
    ([4096, 8192], [512, 532], [5, 6], None, None),                # end to end
    ([4096, 8192], [4096, 8192], [5, 6], None, None),              # in place
    ([4096, 4096], [512, 1024], [5, 5], None, None),               # one gradient twice
    ([4096, 8192], [4116, 8192], [5, 6], None, None),              # behind its gradient
    ([4096, 4096, 4096], [512, 512, 512], [0, 0, 5], None, None),  # empty tensors
    ([4096, 8192], [512, 522], [5, 6], [BF16, BF16], None),
])
def test_apart(grads, outs, counts, dts, out_dts):
    assert clip(grads, outs, counts, dts, out_dts) == 1
    assert b"workspace" in oc.load().oc_last_error()


@pytest.mark.parametrize("what", [iter([]), (t for t in ()), None, 3])
def test_no_list(what):
    for call in (lambda: oc.oc_grad_norm(what), lambda: oc.oc_grad_clip(what, 1.0)):
        with pytest.raises(oc.OcError, match="list of tensors"):
            call()
