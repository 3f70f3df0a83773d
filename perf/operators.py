"""The dense-layer operators and the gradient clipping this library is measured
on, with their plain forms.

A case is a dict of plain values.  Its op is one of

- dense: y = act(x w + bias) + residual; with train also dx, dw and dbias for
  an upstream gradient;
- glu:   y = act(x w_g + b_g) (x w_u + b_u), w = [w_g | w_u]; with train also
  dx, dw and dbias;
- clip:  the global norm of a list of gradients and the gradients scaled to at
  most max_norm, written as one fp32 buffer (the update's operand).

Rows are octants (or whole shapes for a head); features are N(0, 1), weights
N(0, 1 / cin), upstream gradients N(0, 1).  Before a ReLU features and weights
lie on a grid of 1/16 of their scale, as quantised ones do: sums are then exact
in fp32, and which side of zero a value is on is not a matter of rounding.
dtype is the type of x, w, the residual and every output but dbias, which is
fp32.
"""
import math
import random

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MOST_FLOPS = 2.0 * 65536 * 1024 * 4096  # of one product of the largest case
MOST_VALUES = 65536 * (1024 + 4096)     # of its input and output


def listed():
    return [
        # one feature row answered by a service: latency and the weights' bytes
        dict(name="dense_row_bf16", op="dense", dtype="bf16", rows=1, cin=1024, cout=1024,
             act="silu", bias=True, res=True, train=False),
        # the classification head's first layer on a batch of 32 shapes
        dict(name="dense_head_f32", op="dense", dtype="f32", rows=32, cin=1024, cout=128,
             act="relu", bias=True, res=False, train=True),
        # a pointwise layer over the octants of depth 5: few channels, many rows
        dict(name="dense_d5_f32", op="dense", dtype="f32", rows=139800, cin=32, cout=128,
             act="relu", bias=True, res=True, train=True),
        # sizes that are no multiple of anything
        dict(name="dense_odd_f32", op="dense", dtype="f32", rows=8383, cin=513, cout=1027,
             act="gelu", bias=True, res=False, train=True),
        # wide layers in full precision
        dict(name="dense_wide_f32", op="dense", dtype="f32", rows=35472, cin=512, cout=1024,
             act="silu", bias=True, res=True, train=True),
        # the expansion of a feed-forward block over the octants of depth 4
        dict(name="dense_d4_bf16", op="dense", dtype="bf16", rows=35472, cin=256, cout=1024,
             act="gelu", bias=True, res=False, train=True),
        # the largest layer
        dict(name="dense_large_bf16", op="dense", dtype="bf16", rows=65536, cin=1024, cout=4096,
             act="relu", bias=True, res=False, train=True),
        # one feature row through the gated block
        dict(name="glu_row_bf16", op="glu", dtype="bf16", rows=1, cin=1024, cout=4096,
             act="silu", bias=False, train=False),
        # a small gated block over the octants of depth 3, odd width
        dict(name="glu_d3_f32", op="glu", dtype="f32", rows=8384, cin=128, cout=341, act="gelu",
             bias=True, train=True),
        # a wide gated block
        dict(name="glu_large_bf16", op="glu", dtype="bf16", rows=32768, cin=1024, cout=2816,
             act="silu", bias=False, train=True),
        # the parameters of the O-CNN(6) classification network: latency
        dict(name="clip_ocnn_f32", op="clip", dtype="f32", tensors=19, values=0, layout=0,
             max_norm=0.5),
        # many ragged tensors, half of them bf16
        dict(name="clip_ragged_mixed", op="clip", dtype="mixed", tensors=201, values=200_000_000,
             layout=7, max_norm=1.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("dense", "dense", "glu", "glu", "clip"))
    if op == "clip":
        n = _log(rng, 1, 300)
        return dict(op=op, dtype=rng.choice(("f32", "bf16", "mixed")), tensors=n,
                    values=_log(rng, max(1000, 4 * n), 200_000_000),
                    layout=rng.randrange(1, 1 << 20), max_norm=rng.choice((0.1, 0.5, 1.0, 1e6)))
    cin, cout = _log(rng, 3, 4096), _log(rng, 3, 4096)
    for _ in range(2):  # half the sizes are multiples of 32, as networks have them
        if rng.random() < 0.5:
            cin = max(32, cin // 32 * 32)
        if rng.random() < 0.5:
            cout = max(32, cout // 32 * 32)
    wide = 2 * cout if op == "glu" else cout
    rows = _log(rng, 1, 300_000)
    rows = max(1, int(min(rows, MOST_FLOPS / (2.0 * cin * wide), MOST_VALUES / (cin + wide))))
    c = dict(op=op, dtype=rng.choice(("f32", "bf16")), rows=rows, cin=cin, cout=cout,
             act=rng.choice(("relu", "silu", "gelu") if op == "glu"
                            else ("none", "relu", "silu", "gelu")),
             bias=rng.random() < 0.7, train=rng.random() < 0.6)
    if op == "dense":
        c["res"] = rng.random() < 0.5
    return c


def _sizes(case):
    """Sizes of a clip case's tensors, a function of the case alone."""
    if case["layout"] == 0:  # conv weights, BN scales and shifts, the two FC layers
        ch = (3, 8, 16, 32, 64, 128)
        got = [27 * a * b for a, b in zip(ch, ch[1:])]
        got += [c for c in ch[1:] for _ in range(2)]
        return got + [1024 * 128, 128, 128 * 40, 40]
    r = random.Random(case["layout"])
    share = [math.exp(r.uniform(0.0, 9.0)) for _ in range(case["tensors"])]
    total = sum(share)
    return [max(1, int(case["values"] * s / total)) for s in share]


def _kinds(case):
    """Whether each tensor of a clip case is bf16."""
    n = len(_sizes(case))
    if case["dtype"] == "mixed":
        return [i % 2 == 1 for i in range(n)]
    return [case["dtype"] == "bf16"] * n


def work(case):
    """Each input read once, each output written once; two operations a product."""
    if case["op"] == "clip":
        b = sum(n * ((2 if k else 4) + 4) for n, k in zip(_sizes(case), _kinds(case)))
        return {"bytes": b + 4, "flops": 3.0 * sum(_sizes(case))}
    s = 2 if case["dtype"] == "bf16" else 4
    m, k, f = case["rows"], case["cin"], case["cout"]
    n = 2 * f if case["op"] == "glu" else f
    b = s * (m * k + k * n + m * f) + (4 * n if case["bias"] else 0)
    b += s * m * f if case.get("res") else 0
    if case["train"]:  # dy in; dx, dw, dbias out
        b += s * (m * f + m * k + k * n) + 4 * n
    return {"bytes": b, "flops": 2.0 * m * k * n * (3 if case["train"] else 1)}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))

    def normal(shape, scale, dtype):
        v = torch.empty(shape, dtype=torch.float32, device=DEV)
        return v.normal_(0.0, scale, generator=g).to(dtype)

    if case["op"] == "clip":
        sizes, kinds = _sizes(case), _kinds(case)
        # gradients are views of one flat buffer a type, as a training step keeps them
        flat = {k: normal(sum(n for n, q in zip(sizes, kinds) if q == k), 0.01, t)
                for k, t in ((False, torch.float32), (True, torch.bfloat16))}
        out = torch.empty(sum(sizes), dtype=torch.float32, device=DEV)
        at, o, grads, outs = {False: 0, True: 0}, 0, [], []
        r = random.Random(int(seed))
        for n, k in zip(sizes, kinds):
            v = flat[k][at[k]:at[k] + n]
            v.mul_(10.0 ** r.uniform(-1.0, 2.0))  # layers' gradients differ in size
            grads.append(v)
            outs.append(out[o:o + n])
            at[k] += n
            o += n
        return {"case": case, "grads": grads, "outs": outs, "flat": out}
    t = TYPES[case["dtype"]]
    m, k, f = case["rows"], case["cin"], case["cout"]
    n = 2 * f if case["op"] == "glu" else f
    if case["act"] == "relu":
        on_grid = lambda shape, scale, dtype: (  # noqa: E731
            normal(shape, 16.0, torch.float32).round_().mul_(scale / 16.0).to(dtype))
        w_scale = 2.0 ** -round(0.5 * math.log2(k))
    else:
        on_grid, w_scale = normal, k ** -0.5
    s = {"case": case, "x": on_grid((m, k), 1.0, t), "w": on_grid((k, n), w_scale, t),
         "b": on_grid((n,), 0.125, torch.float32) if case["bias"] else None,
         "res": normal((m, f), 1.0, t) if case.get("res") else None}
    if case["train"]:
        s["dy"] = normal((m, f), 1.0, t)
    return s


# --- the plain forms --------------------------------------------------------


def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
                + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi)))
    return torch.ones_like(z)


def _plain(s):
    c, t = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = x @ w
    if s["b"] is not None:
        z = z + s["b"]
    if c["op"] == "glu":
        f = c["cout"]
        gate, up = z[:, :f], z[:, f:]
        y = _act(gate, c["act"]) * up
    else:
        y = _act(z, c["act"])
        if s["res"] is not None:
            y = y + s["res"].float()
    if not c["train"]:
        return {"y": y.to(t)}
    dy = s["dy"].float()
    if c["op"] == "glu":
        dz = torch.cat([dy * up * _slope(gate, c["act"]), dy * _act(gate, c["act"])], dim=1)
    else:
        dz = dy * _slope(z, c["act"])
    return {"y": y.to(t), "dx": (dz @ w.t()).to(t), "dw": (x.t() @ dz).to(t), "db": dz.sum(0)}


def _plain_clip(s):
    c = s["case"]
    norm = torch.stack([g.float().square().sum(dtype=torch.float64)
                        for g in s["grads"]]).sum().sqrt()
    scale = torch.clamp(c["max_norm"] / norm, max=1.0).float()
    return {"norm": norm.float(),
            "grads": torch.cat([g.float() * scale for g in s["grads"]], out=s["flat"])}


# --- the framework's calls --------------------------------------------------


def _own(s):
    import paper_1712_01537_amd as oc

    c, x, w, b = s["case"], s["x"], s["w"], s["b"]
    act = {"none": oc.OC_ACT_NONE, "relu": oc.OC_ACT_RELU, "silu": oc.OC_ACT_SILU,
           "gelu": oc.OC_ACT_GELU}[c["act"]]
    if c["op"] == "glu":
        y, pre = oc.oc_glu_fwd(x, w, b, act=act, need_pre=c["train"])
        if not c["train"]:
            return {"y": y}
        dx, dw, db = oc.oc_glu_bwd(x, w, s["dy"], pre, act=act, dw_dtype=x.dtype)
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    # the backward of a ReLU needs signs only: the output itself, where nothing is added to it
    keep = c["train"] and c["act"] != "none" and not (c["act"] == "relu" and s["res"] is None)
    y, pre = oc.oc_dense_fwd(x, w, b, res=s["res"], act=act, need_pre=keep)
    if not c["train"]:
        return {"y": y}
    if c["act"] == "relu" and not keep:
        pre = y
    dx, dw, db = oc.oc_dense_bwd(x, w, s["dy"], act=act, pre=pre, dw_dtype=x.dtype)
    return {"y": y, "dx": dx, "dw": dw, "db": db}


def _own_clip(s):
    import paper_1712_01537_amd as oc

    norm = oc.oc_grad_clip(s["grads"], s["case"]["max_norm"], outs=s["outs"])
    return {"norm": norm, "grads": s["flat"]}


def run(state):
    if state["case"]["op"] == "clip":
        return _own_clip(state) if own else _plain_clip(state)
    return _own(state) if own else _plain(state)


# --- 64-bit values ----------------------------------------------------------


def exact(case, seed):
    """The gradients come from differentiating the definition in 64 bits."""
    s = prepare(case, seed)
    if case["op"] == "clip":
        g = torch.cat([v.double() for v in s["grads"]])
        norm = torch.linalg.vector_norm(g)
        return {"norm": norm, "grads": g if float(norm) <= case["max_norm"]
                else g.mul_(case["max_norm"] / norm)}
    fn = {"none": lambda z: z, "relu": torch.relu, "silu": torch.nn.functional.silu,
          "gelu": torch.nn.functional.gelu}[case["act"]]
    x, w = s["x"].double(), s["w"].double()
    n = w.shape[1]
    b = s["b"].double() if s["b"] is not None else torch.zeros(n, dtype=torch.float64, device=DEV)
    leaves = [v.requires_grad_(case["train"]) for v in (x, w, b)]
    z = torch.addmm(b, x, w)
    if case["op"] == "glu":
        gate, up = z.chunk(2, dim=1)
        y = fn(gate) * up
    else:
        y = fn(z)
        if s["res"] is not None:
            y = y + s["res"].double()
    if not case["train"]:
        return {"y": y}
    dx, dw, db = torch.autograd.grad(y, leaves, s["dy"].double())
    return {"y": y.detach(), "dx": dx, "dw": dw, "db": db}
