"""The row operators around dense layers that this library is measured on, with
their plain forms.  Rows are octants (or whole shapes), columns channels.

A case is a dict of plain values.  Its op is one of

- ln:      layer norm, y = (x - mean) / sqrt(var + eps) gamma + beta over the
           columns of each row; with train also dx, dgamma and dbeta for dy;
- drop:    dropout of ratio p whose mask comes from a counter-based generator;
           with train also the gradient of x for dy, the mask drawn once more;
- drop_ln: a residual step, h = res + dropout(x), y = layer norm of h (formed
           before h is rounded to its type); with train also the gradients of x,
           res, gamma and beta for dy and the gradient dh that reaches h by the
           residual path;
- embed:   y = scale table[id] for each row, 0 where the id is outside the
           table; with train also the table's gradient for dy.

dtype is the type of x, res, h, y, dy, dx and the table with its gradient;
gamma, beta and their gradients are fp32.

The mask.  Columns of a row are in groups of eight.  Group g of row r has the index
i = r ceil(cols / 8) + g; Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC 2011)
with the key {seed low, seed high} and the counter {i low, i high + 2^16 site, step
low, step high} gives four words, whose halves, low before high, are the high 16
bits of a number for each column; the same with 2^31 added to the counter's second
word gives the low 16 bits.  A value is kept where its 32-bit number is below
T = round((1 - p) 2^32), and scaled by 2^32 / T.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
# most values of x of a drawn case, by op, and of the table
MOST = {"ln": 1 << 28, "drop": 1 << 28, "drop_ln": 1 << 27, "embed": 1 << 26}
MOST_TABLE = 1 << 25


def listed():
    return [
        # one feature row answered by a service: latency
        dict(name="ln_row_bf16", op="ln", dtype="bf16", rows=1, cols=1024, affine=True,
             train=False),
        # the octants of depth 5, few channels
        dict(name="ln_d5_f32", op="ln", dtype="f32", rows=139800, cols=128, affine=True,
             train=True),
        # sizes that are no multiple of anything
        dict(name="ln_odd_f32", op="ln", dtype="f32", rows=8383, cols=513, affine=True,
             train=True),
        # the widest rows of a feed-forward block, the largest batch
        dict(name="ln_large_bf16", op="ln", dtype="bf16", rows=65536, cols=4096, affine=True,
             train=True),
        # the classification head on a batch of 32 shapes
        dict(name="drop_head_f32", op="drop", dtype="f32", rows=32, cols=1024, p=0.5, site=1,
             train=True),
        # the inner features of a large feed-forward block
        dict(name="drop_large_bf16", op="drop", dtype="bf16", rows=65536, cols=4096, p=0.1,
             site=3, train=True),
        # one row of a residual block in a service: no dropout, latency
        dict(name="drop_ln_row_bf16", op="drop_ln", dtype="bf16", rows=1, cols=1024, p=0.0,
             site=0, res=True, train=False),
        # the residual step over the octants of depth 4
        dict(name="drop_ln_d4_bf16", op="drop_ln", dtype="bf16", rows=35472, cols=1024, p=0.1,
             site=2, res=True, train=True),
        # wide rows in full precision
        dict(name="drop_ln_wide_f32", op="drop_ln", dtype="f32", rows=16384, cols=8192, p=0.2,
             site=5, res=True, train=True),
        # a category for each of 32 shapes: latency
        dict(name="embed_head_f32", op="embed", dtype="f32", rows=32, num=40, cols=128,
             scale=1.0, ids="even", pad=False, train=True),
        # the octants' places at depth 4, from their shuffle keys: ids ascend in each shape
        dict(name="embed_keys_d4_f32", op="embed", dtype="f32", rows=35472, num=4096, cols=256,
             scale=1.0, ids="keys", pad=False, train=True),
        # a large table whose first entries are met by thousands of rows, padded rows
        dict(name="embed_large_bf16", op="embed", dtype="bf16", rows=65536, num=32768, cols=1024,
             scale=32.0, ids="skewed", pad=True, train=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("ln", "drop", "drop_ln", "embed"))
    c = dict(op=op, dtype=rng.choice(("f32", "bf16")), rows=_log(rng, 1, 300_000))
    # (a norm over a handful of columns cancels nearly all of its gradient)
    cols = _log(rng, 16 if "ln" in op else 1, 4096 if op == "embed" else 16384)
    if rng.random() < 0.5:  # half the widths are multiples of 32, as networks have them
        cols = max(32, cols // 32 * 32)
    c["cols"] = cols
    c["rows"] = max(1, min(c["rows"], MOST[op] // cols))
    c["train"] = rng.random() < 0.7
    if op == "ln":
        c["affine"] = rng.random() < 0.8
    elif op == "embed":
        c["ids"] = rng.choice(("even", "skewed", "keys"))
        if c["ids"] == "keys":  # 8^depth places, up to 32 shapes
            depth = rng.randrange(1, 7)
            while depth > 1 and 8 ** depth * cols > MOST_TABLE:
                depth -= 1
            c["num"] = 8 ** depth
            c["rows"] = min(c["rows"], 32 * c["num"])
        else:
            c["num"] = max(1, min(_log(rng, 1, 200_000), MOST_TABLE // cols))
        c["pad"] = c["ids"] != "keys" and rng.random() < 0.5
        c["scale"] = rng.choice((1.0, float(cols) ** 0.5))
    else:
        c["p"] = rng.choice((0.0, 0.1, 0.25, 0.5, 0.9) if op == "drop_ln"
                            else (0.05, 0.1, 0.25, 0.5, 0.9))
        c["site"] = rng.randrange(0, 64)
        if op == "drop_ln":
            c["res"] = rng.random() < 0.8
    return c


def work(case):
    """Each input read once, each output written once."""
    s = 2 if case["dtype"] == "bf16" else 4
    m, n = case["rows"], case["cols"]
    train, op = case["train"], case["op"]
    if op == "embed":
        num = case["num"]
        used = min(m, num)  # rows of the table that are read, at most
        b = 4 * m + s * (used * n + m * n)
        return {"bytes": b + (s * (m * n + num * n) if train else 0),
                "flops": m * n * (3.0 if train else 1.0)}
    if op == "drop":
        return {"bytes": s * m * n * (4 if train else 2), "flops": m * n * (2.0 if train else 1.0)}
    b = s * m * n * 2  # x, y
    if op == "drop_ln":
        b += s * m * n * (2 if case["res"] else 1)  # res, h
    affine = case.get("affine", True)
    b += 8 * n if affine else 0
    if train:
        b += s * m * n * 2 + (8 * n if affine else 0)  # dy, dx; dgamma, dbeta
        if op == "drop_ln":
            b += s * m * n * (2 if case["res"] else 1)  # dh, dres
    return {"bytes": b, "flops": m * n * (20.0 if train else 8.0)}


def _ids(case, g):
    m, num = case["rows"], case["num"]
    if case["ids"] == "keys":
        shapes = max(1, min(32, m), -(-m // num))
        keys = []
        for b in range(shapes):
            n = m * (b + 1) // shapes - m * b // shapes
            place = torch.randperm(num, generator=g, device=DEV)[:n].sort()[0]
            keys.append(place + (b << 24))
        return torch.cat(keys).to(torch.int32)
    u = torch.rand(m, generator=g, device=DEV, dtype=torch.float64)
    if case["ids"] == "skewed":
        u = u ** 4
    ids = (u * num).to(torch.int64).clamp_(max=num - 1)
    if case["pad"]:
        ids[torch.rand(m, generator=g, device=DEV) < 1.0 / 16] = -1
    return ids.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    t = TYPES[case["dtype"]]
    m, n, op = case["rows"], case["cols"], case["op"]

    def normal(shape, dtype):
        return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=g).to(dtype)

    s = {"case": case}
    if op == "embed":
        s["table"] = normal((case["num"], n), t)
        s["ids"] = _ids(case, g)
    else:
        # rows' features differ in size and lie around a value of their own
        size = torch.exp(normal((m, 1), torch.float32) * 0.5)
        x = torch.empty((m, n), dtype=torch.float32, device=DEV).normal_(generator=g)
        s["x"] = x.add_(normal((m, 1), torch.float32)).mul_(size).to(t)
    if op in ("ln", "drop_ln"):
        affine = case.get("affine", True)
        s["gamma"] = normal((n,), torch.float32).mul_(0.1).add_(1.0) if affine else None
        s["beta"] = normal((n,), torch.float32).mul_(0.1) if affine else None
    if op in ("drop", "drop_ln"):
        s["rng"] = torch.randint(-(1 << 62), 1 << 62, (2,), generator=g, device=DEV)
        s["rng"][1] &= 0xFFFFF  # steps taken
    if op == "drop_ln":
        s["res"] = normal((m, n), t) if case["res"] else None
    if case["train"]:
        s["dy"] = normal((m, n), t)
        if op == "drop_ln":
            s["dh"] = normal((m, n), t)
    return s


# --- the plain forms --------------------------------------------------------

LOW = 0xFFFFFFFF


def _words(index, site, rng, second):
    """Philox4x32-10's four words for the group indices, as 64-bit integers."""
    k0, k1 = rng[0] & LOW, (rng[0] >> 32) & LOW
    c0 = index & LOW
    c1 = ((index >> 32) & 0xFFFF) | (site << 16) | ((1 << 31) if second else 0)
    c2, c3 = rng[1] & LOW, (rng[1] >> 32) & LOW
    for r in range(10):
        if r:
            k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # (64 bits, wrapped: all of them count)
        c0, c1, c2, c3 = (((b >> 32) & LOW) ^ c1 ^ k0, b & LOW, ((a >> 32) & LOW) ^ c3 ^ k1,
                          a & LOW)
    return c0, c1, c2, c3


def _threshold(p):
    return int(round((1.0 - p) * 4294967296.0))


def _kept(case, rng):
    """The mask, and the kept values' scale."""
    m, n = case["rows"], case["cols"]
    t = _threshold(case["p"])
    groups = -(-n // 8)
    index = torch.arange(m * groups, device=DEV)

    def halves(second):
        w = torch.stack(torch.broadcast_tensors(*_words(index, case["site"], rng, second)), 1)
        return torch.stack([w & 0xFFFF, w >> 16], 2).reshape(m, groups * 8)[:, :n]

    return (halves(False) << 16) + halves(True) < t, 4294967296.0 / t


def _norm(h, gamma, beta):
    """Layer norm of fp32 rows: y, the normalised rows and 1 / deviation."""
    d = h - h.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    z = d * r
    y = z if gamma is None else z * gamma + beta
    return y, z, r


def _norm_bwd(dy, z, r, gamma):
    g = dy if gamma is None else dy * gamma
    dh = r * (g - g.mean(1, keepdim=True) - z * (g * z).mean(1, keepdim=True))
    # (sums over all rows: 64 bits)
    return dh, (dy * z).sum(0, dtype=torch.float64).float(), dy.sum(0, dtype=torch.float64).float()


def _plain(s):
    c = s["case"]
    op, t = c["op"], TYPES[c["dtype"]]
    if op == "embed":
        ids = s["ids"].long()
        if c["ids"] == "keys":
            ids = ids & 0xFFFFFF
        there = ((ids >= 0) & (ids < c["num"])).unsqueeze(1)
        ids = ids.clamp(0, c["num"] - 1)
        zero = torch.zeros((), dtype=torch.float32, device=DEV)
        y = torch.where(there, s["table"][ids].float() * c["scale"], zero).to(t)
        if not c["train"]:
            return {"y": y}
        dy = torch.where(there, s["dy"].float(), zero).double()  # (long sums: 64 bits)
        dt = torch.zeros(s["table"].shape, dtype=torch.float64, device=DEV).index_add_(0, ids, dy)
        return {"y": y, "dtable": (dt * c["scale"]).to(t)}
    x = s["x"].float()
    if op == "ln":
        y, z, r = _norm(x, s["gamma"], s["beta"])
        if not c["train"]:
            return {"y": y.to(t)}
        dx, dg, db = _norm_bwd(s["dy"].float(), z, r, s["gamma"])
        out = {"y": y.to(t), "dx": dx.to(t)}
        return dict(out, dgamma=dg, dbeta=db) if c["affine"] else out
    if c["p"]:
        keep, scale = _kept(c, s["rng"])
        drop = lambda v: torch.where(keep, v * scale, torch.zeros_like(v))  # noqa: E731
    else:
        drop = lambda v: v  # noqa: E731
    if op == "drop":
        y = drop(x).to(t)
        return {"y": y, "dx": drop(s["dy"].float()).to(t)} if c["train"] else {"y": y}
    h = drop(x)
    if s["res"] is not None:
        h = h + s["res"].float()
    y, z, r = _norm(h, s["gamma"], s["beta"])
    out = {"h": h.to(t), "y": y.to(t)}
    if not c["train"]:
        return out
    dh, dg, db = _norm_bwd(s["dy"].float(), z, r, s["gamma"])
    dh = dh + s["dh"].float()
    out.update(dx=drop(dh).to(t), dgamma=dg, dbeta=db)
    return dict(out, dres=dh.to(t)) if c["res"] else out


# --- the framework's calls --------------------------------------------------


def _own(s):
    import paper_1712_01537_amd as oc

    c = s["case"]
    op, train = c["op"], c["train"]
    if op == "embed":
        keys = c["ids"] == "keys"
        y = oc.oc_embed_fwd(s["ids"], s["table"], scale=c["scale"], keys=keys)
        if not train:
            return {"y": y}
        dt = oc.oc_embed_bwd(s["ids"], s["dy"], c["num"], scale=c["scale"], keys=keys,
                             dtype=s["table"].dtype)
        return {"y": y, "dtable": dt}
    x = s["x"]
    if op == "ln":
        y, mean, invstd = oc.oc_ln_fwd(x, s["gamma"], s["beta"], eps=EPS, need_stats=train)
        if not train:
            return {"y": y}
        dx, dg, db = oc.oc_ln_bwd(x, s["dy"], s["gamma"], mean, invstd,
                                  need_dgamma=c["affine"], need_dbeta=c["affine"])
        out = {"y": y, "dx": dx}
        return dict(out, dgamma=dg, dbeta=db) if c["affine"] else out
    if op == "drop":
        y = oc.oc_dropout_rng(x, c["p"], s["rng"], site=c["site"])
        if not train:
            return {"y": y}
        return {"y": y, "dx": oc.oc_dropout_rng(s["dy"], c["p"], s["rng"], site=c["site"])}
    h, y, mean, invstd = oc.oc_drop_ln_fwd(x, s["res"], c["p"], s["rng"], s["gamma"], s["beta"],
                                           site=c["site"], eps=EPS, need_stats=train)
    out = {"h": h, "y": y}
    if not train:
        return out
    dx, dres, dg, db = oc.oc_drop_ln_bwd(x, s["res"], s["dy"], c["p"], s["rng"], s["gamma"], mean,
                                         invstd, dh=s["dh"], site=c["site"], need_dres=c["res"])
    out.update(dx=dx, dgamma=dg, dbeta=db)
    return dict(out, dres=dres) if c["res"] else out


def run(state):
    return _own(state) if own else _plain(state)


# --- 64-bit values ----------------------------------------------------------


def _product(a, m):
    """High and low words of a m, from products of 16-bit halves."""
    ah, al, mh, ml = a // 65536, a % 65536, m // 65536, m % 65536
    t = al * ml
    u = ah * ml + t // 65536
    v = al * mh + u % 65536
    return ah * mh + u // 65536 + v // 65536, (v % 65536) * 65536 + t % 65536


def _numbers(case, rng):
    """The 32-bit number of each value."""
    m, n = case["rows"], case["cols"]
    groups = (n + 7) // 8
    seed, step = (int(v) % (1 << 64) for v in rng.tolist())
    i = torch.arange(m * groups, device=DEV).view(m, groups)
    out = torch.zeros(m, groups, 8, dtype=torch.int64, device=DEV)
    for shift, mark in ((65536, 0), (1, 1 << 31)):
        a = [i % (1 << 32), i // (1 << 32) + case["site"] * 65536 + mark,
             torch.full_like(i, step % (1 << 32)), torch.full_like(i, step // (1 << 32))]
        for r in range(10):
            key = [(seed // (1 << 32 * j) + r * w) % (1 << 32)
                   for j, w in ((0, 0x9E3779B9), (1, 0xBB67AE85))]
            (ph, pl), (qh, ql) = _product(a[0], 0xD2511F53), _product(a[2], 0xCD9E8D57)
            a = [qh ^ a[1] ^ key[0], ql, ph ^ a[3] ^ key[1], pl]
        for j in range(8):
            out[:, :, j] += (a[j // 2] // (1 << 16 * (j % 2))) % 65536 * shift
    return out.view(m, groups * 8)[:, :n]


def _norm64(h, gamma, beta):
    centred = h - h.mean(1, keepdim=True)
    y = centred / (centred.square().mean(1, keepdim=True) + EPS).sqrt()
    return y if gamma is None else y * gamma + beta


def exact(case, seed):
    """The gradients come from differentiating the definition in 64 bits."""
    s = prepare(case, seed)
    op, train, n = case["op"], case["train"], case["cols"]
    dy = s["dy"].double() if train else None
    if op == "embed":
        ids = s["ids"].long()
        if case["ids"] == "keys":
            ids = ids % (1 << 24)
        # a row of zeros behind the table stands for every id outside it
        ids = torch.where((ids < 0) | (ids >= case["num"]), torch.full_like(ids, case["num"]), ids)
        table = torch.cat([s["table"].double(), torch.zeros(1, n, dtype=torch.float64, device=DEV)])
        y = table[ids] * case["scale"]
        if not train:
            return {"y": y}
        order = torch.argsort(ids, stable=True)
        ends = torch.cumsum(torch.bincount(ids, minlength=case["num"] + 1), 0)
        sums = torch.zeros(ids.numel() + 1, n, dtype=torch.float64, device=DEV)
        torch.cumsum(dy[order], 0, out=sums[1:])
        at = sums[ends]
        at[1:] -= at[:-1].clone()
        return {"y": y, "dtable": at[:-1] * case["scale"]}
    x = s["x"].double().requires_grad_(train)
    gamma, beta = (s[k].double().requires_grad_(train) if s.get(k) is not None else None
                   for k in ("gamma", "beta"))
    keep, q = None, 1.0
    if op != "ln" and case["p"] > 0:
        most = round((1.0 - case["p"]) * 2 ** 32)
        keep, q = _numbers(case, s["rng"]) < most, most / 2 ** 32
    if op == "ln":
        y = _norm64(x, gamma, beta)
        if not train:
            return {"y": y}
        leaves = [x] + ([gamma, beta] if case["affine"] else [])
        got = torch.autograd.grad(y, leaves, dy)
        return dict(zip(("y", "dx", "dgamma", "dbeta"), (y.detach(), *got)))
    u = x if keep is None else (x / q).masked_fill(~keep, 0.0)
    if op == "drop":
        if not train:
            return {"y": u}
        return {"y": u.detach(), "dx": torch.autograd.grad(u, x, dy)[0]}
    res = s["res"].double().requires_grad_(train) if s["res"] is not None else None
    h = u if res is None else u + res
    y = _norm64(h, gamma, beta)
    if not train:
        return {"h": h, "y": y}
    leaves = [x, gamma, beta] + ([res] if res is not None else [])
    got = torch.autograd.grad([y, h], leaves, [dy, s["dh"].double()])
    return dict(zip(("h", "y", "dx", "dgamma", "dbeta", "dres"), (h.detach(), y.detach(), *got)))
