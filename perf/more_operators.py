"""The operators that train a temporal attention layer, as timed cases.

Rows (nodes, edges, sampled slots) are of several types, each with weights of
its own.  Six kinds of pass:

* ``group``   rows sorted by their type (``group_rows``): types given row by
              row, or looked up for sampled slots, some of which are empty;
* ``linear``  rows times their type's weights (``linear_typed``);
* ``step``    the same and its gradients (``linear_typed_backward``): those of
              the rows, of every type's weights and of their biases;
* ``norm``    layer norm of rows (``layer_norm``);
* ``train``   residual's addition, layer norm and its gradients
              (``layer_norm_backward``), with a gradient that comes to the sum itself;
* ``layer``   all of it for one batch: slots are grouped by their nodes' type,
              projected, added to a residual, normed; then backward.

``order`` holds the rows of type 0, then those of type 1, and so on, rows of no
type last; ``offsets[g]`` is where those of type g begin.
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def listed():
    return [
        # one training batch: 600 edges x (source, destination, negative)
        dict(name="group_roots", kind="group", rows=1800, types=3, nodes=0, empty=0.0, skew=0.0),
        # the second hop of a super-batch of 64 batches: 768,000 roots x 10, looked up by node
        dict(name="group_slots", kind="group", rows=7_680_000, types=7, nodes=2_000_000, empty=0.1, skew=1.0),
        # one event arrives: its 768-dim row (MAG's node features) through a fused projection
        dict(name="linear_event", kind="linear", rows=1, k=768, out=2304, types=4, empty=0.0, skew=0.0, bias=True, dtype="bf16"),
        # one batch of roots: 4000 edges x (source, destination, negative), MAG's width
        dict(name="linear_batch", kind="linear", rows=12_000, k=768, out=1024, types=4, empty=0.0, skew=1.0, bias=True, dtype="bf16"),
        # the paper's hidden width in float32, an odd row count, a few empty slots
        dict(name="linear_hidden", kind="linear", rows=1801, k=272, out=100, types=3, empty=0.1, skew=0.0, bias=True, dtype="f32"),
        # the same width trained over many kinds of events, most of them rare
        dict(name="step_relations", kind="step", rows=40_000, k=272, out=100, types=200, empty=0.0, skew=1.0, bias=True, dtype="f32"),
        # roots and slots of one batch at MAG's width
        dict(name="step_slots", kind="step", rows=132_000, k=768, out=1024, types=4, empty=0.1, skew=1.0, bias=True, dtype="bf16"),
        # a wide feed-forward layer
        dict(name="step_wide", kind="step", rows=16_384, k=4096, out=4096, types=8, empty=0.0, skew=0.0, bias=False, dtype="bf16"),
        # one event's row
        dict(name="norm_event", kind="norm", rows=1, dim=768, dtype="bf16"),
        # roots and slots of one batch at MAG's width
        dict(name="train_slots", kind="train", rows=132_000, dim=768, dtype="bf16"),
        # roots of one batch at the paper's hidden width
        dict(name="train_hidden", kind="train", rows=12_001, dim=100, dtype="f32"),
        # slots of one batch: edge features and time encoding to a hidden width, in float32 as the paper trains
        dict(name="layer_batch", kind="layer", rows=120_000, k=272, out=128, types=3, nodes=2_000_000, empty=0.1, skew=1.0,
             dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: a multiple of 16 or 4 as most are, or any."""
    w = _log(rng, lo, hi)
    return max(lo, w // 16 * 16) if rng.random() < 0.4 else max(lo, w // 4 * 4) if rng.random() < 0.5 else w


def draw(rng):
    kind = rng.choice(["group", "linear", "linear", "step", "step", "norm", "train", "layer"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    skew, empty = rng.choice([0.0, 1.0, 2.0]), rng.choice([0.0, 0.0, 0.1, 0.6])
    if kind == "group":
        return dict(kind=kind, rows=_log(rng, 64, 7_680_000), types=_log(rng, 2, 1000), nodes=rng.choice([0, 1000, 2_000_000]),
                    empty=empty, skew=skew)
    if kind in ("norm", "train"):
        dim = _width(rng, 1, 8192)
        return dict(kind=kind, rows=_log(rng, 1, min(200_000, 100_000_000 // dim)), dim=dim, dtype=dtype)
    k, out = _width(rng, 16, 4096), _width(rng, 16, 4096)
    if kind == "layer":                 # float32: between its operators nothing is rounded to fewer bits
        k, out, dtype = min(k, 1024), min(out, 1024), "f32"
    most = (1 << 37 if dtype == "bf16" else 1 << 33) // (k * out)           # rows
    types = min(_log(rng, 1, 300), max(1, (1 << 26) // (k * out)))
    rows = _log(rng, 1, max(2, min(132_000, most)))
    case = dict(kind=kind, rows=rows, k=k, out=out, types=types, empty=empty if rows >= 16 else 0.0, skew=skew, dtype=dtype)
    if kind == "layer":
        case["nodes"] = rng.choice([1000, 2_000_000])
    else:
        case["bias"] = rng.random() < 0.5
    return case


class _Random:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape):
        return torch.randn(*shape, device="cuda", generator=self.g)

    def uniform(self, *shape):
        return torch.rand(*shape, device="cuda", generator=self.g)

    def ints(self, lo, hi, *shape, dtype=torch.int64):
        return torch.randint(lo, hi, shape, device="cuda", generator=self.g, dtype=dtype)

    def types(self, n, case, empty):
        """Types of n rows, type g's share falling as (g + 1)^-skew; -1 for the empty ones."""
        share = torch.arange(1, case["types"] + 1, device="cuda", dtype=torch.float64) ** -case["skew"]
        upto = (share.cumsum(0) / share.sum()).float()
        t = torch.searchsorted(upto, self.uniform(n)).clamp(max=case["types"] - 1).to(torch.int32)
        t[self.uniform(n) < empty] = -1
        return t


def prepare(case, seed):
    r = _Random(seed)
    s = dict(case)
    n = case["rows"]
    if case["kind"] in ("norm", "train"):
        s["type"] = TYPES[case["dtype"]]
        d = case["dim"]
        s["x"] = (3 * r.normal(n, d) + r.normal(n, 1)).to(s["type"])
        s["gamma"], s["beta"] = 1 + 0.1 * r.normal(d), 0.1 * r.normal(d)
        if case["kind"] == "train":
            s["res"] = r.normal(n, d).to(s["type"])
            s["dy"], s["dh"] = r.normal(n, d).to(s["type"]), r.normal(n, d).to(s["type"])
        return s
    if case.get("nodes"):               # types of nodes, looked up for slots that hold their ids
        s["of"] = r.types(case["nodes"], case, 0.0)
        s["ids"] = r.ints(0, case["nodes"], n, dtype=torch.int32)
        s["ids"][r.uniform(n) < case["empty"]] = -1
    else:
        s["of"], s["ids"] = r.types(n, case, case["empty"]), None
    if case["kind"] == "group":
        return s
    s["type"] = t = TYPES[case["dtype"]]
    k, out, types = case["k"], case["out"], case["types"]
    s["x"] = r.normal(n, k).to(t)
    s["w"] = (r.normal(types, out, k) / math.sqrt(k)).to(t)
    s["b"] = r.normal(types, out) if case.get("bias", True) else None
    if case["kind"] != "linear":
        s["dy"] = r.normal(n, out).to(t)
    if case["kind"] == "layer":
        s["res"] = r.normal(n, out).to(t)
        s["gamma"], s["beta"] = 1 + 0.1 * r.normal(out), 0.1 * r.normal(out)
        s["leaves"] = [s[name].requires_grad_() for name in ("x", "w", "b", "res", "gamma", "beta")]
    # kept by a program over the layer's projections, forward and backward
    order, offsets = _plain_group(s)
    s["order"], s["offsets"] = order, offsets
    s["ends"] = offsets.tolist()
    return s


# ---- the operators in their plain form --------------------------------------

def _plain_group(s):
    t = s["of"]
    if s["ids"] is not None:
        t = torch.where(s["ids"] < 0, -1, t[s["ids"].clamp(min=0)])
    t = torch.where((t < 0) | (t >= s["types"]), s["types"], t)
    t, order = torch.sort(t, stable=True)
    every = torch.arange(s["types"] + 1, device="cuda", dtype=t.dtype)
    return order.to(torch.int32), torch.searchsorted(t, every)


def _of_type(s, order, ends):
    """Each type with its rows."""
    return [(g, order[ends[g]:ends[g + 1]].long()) for g in range(s["types"]) if ends[g + 1] > ends[g]]


def _plain_linear(s, x, w, b, order, ends):
    y = torch.zeros(s["rows"], s["out"], device="cuda", dtype=s["type"])
    for g, rows in _of_type(s, order, ends):
        v = torch.matmul(x[rows].float(), w[g].float().t())
        y[rows] = (v if b is None else v + b[g]).to(s["type"])
    return y


def _plain_linear_backward(s, dy, x, w, order, ends, bias):
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    db = torch.zeros(s["types"], s["out"], device="cuda") if bias else None
    for g, rows in _of_type(s, order, ends):
        d = dy[rows].float()
        dx[rows] = torch.matmul(d, w[g].float()).to(s["type"])
        dw[g] = torch.matmul(d.t(), x[rows].float()).to(s["type"])
        if bias:
            db[g] = d.sum(0)
    return dx, dw, db


def _plain_norm(x, res, gamma, beta):
    kept = x if res is None else (x.float() + res.float()).to(x.dtype)
    h = kept.float()
    c = h - h.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(c.square().mean(1, keepdim=True) + EPS)
    return (c * rstd * gamma + beta).to(x.dtype), kept


def _plain_norm_backward(dy, h, gamma, dh):
    h, d = h.float(), dy.float()
    c = h - h.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(c.square().mean(1, keepdim=True) + EPS)
    xh, g = c * rstd, d * gamma
    dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * rstd
    if dh is not None:
        dx = dx + dh.float()
    return dx.to(dy.dtype), (d * xh).sum(0), d.sum(0)


def _plain(s):
    kind = s["kind"]
    if kind == "group":
        return _plain_group(s)
    if kind == "linear":
        return _plain_linear(s, s["x"], s["w"], s["b"], s["order"], s["ends"])
    if kind == "step":
        y = _plain_linear(s, s["x"], s["w"], s["b"], s["order"], s["ends"])
        return (y,) + _plain_linear_backward(s, s["dy"], s["x"], s["w"], s["order"], s["ends"], s["b"] is not None)
    if kind == "norm":
        return _plain_norm(s["x"], None, s["gamma"], s["beta"])[0]
    if kind == "train":
        y, h = _plain_norm(s["x"], s["res"], s["gamma"], s["beta"])
        return (y, h) + _plain_norm_backward(s["dy"], h, s["gamma"], s["dh"])
    with torch.no_grad():
        order, offsets = _plain_group(s)
        ends = offsets.tolist()
        x, w, b, res, gamma, beta = s["leaves"]
        y, h = _plain_norm(_plain_linear(s, x, w, b, order, ends), res, gamma, beta)
        dres, dgamma, dbeta = _plain_norm_backward(s["dy"], h, gamma, None)
        dx, dw, db = _plain_linear_backward(s, dres, x, w, order, ends, True)
    return y, dx, dw, db, dres, dgamma, dbeta


# ---- the framework's calls --------------------------------------------------

def _own(s):
    import paper_2203_14883_amd as tgl
    kind = s["kind"]
    if kind == "group":
        groups = tgl.group_rows(s["of"], s["types"], ids=s["ids"])
        return groups.order, groups.offsets
    if kind == "norm":
        return tgl.layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS)
    if kind == "train":
        y, h, stats = tgl.layer_norm(s["x"], s["gamma"], s["beta"], residual=s["res"], eps=EPS, return_stats=True)
        return (y, h) + tgl.layer_norm_backward(s["dy"], h, stats, s["gamma"], dh=s["dh"])
    if kind == "layer":
        groups = tgl.group_rows(s["of"], s["types"], ids=s["ids"])
        x, w, b, res, gamma, beta = s["leaves"]
        y, _ = tgl.layer_norm(tgl.linear_typed(x, w, groups, b), gamma, beta, residual=res, eps=EPS)
        dx, dw, db, dres, dgamma, dbeta = torch.autograd.grad(y, s["leaves"], s["dy"])
        return y.detach(), dx, dw, db, dres, dgamma, dbeta
    groups = tgl.RowGroups(s["offsets"], s["order"])
    y = tgl.linear_typed(s["x"], s["w"], groups, s["b"])
    if kind == "linear":
        return y
    return (y,) + tgl.linear_typed_backward(s["dy"], s["x"], s["w"], groups, bias=s["b"] is not None)


def run(state):
    return _own(state) if own else _plain(state)


def _shares(case):
    """Expected rows of each type."""
    share = [(g + 1) ** -case["skew"] for g in range(case["types"])]
    return [case["rows"] * (1 - case["empty"]) * v / sum(share) for v in share]


def work(case):
    n, kind = case["rows"], case["kind"]
    if kind == "group":
        return {"bytes": n * 4 + (n * 4 if case["nodes"] else 0) + n * 4 + 8 * (case["types"] + 1), "flops": 0}
    e = SIZE[case["dtype"]]
    if kind in ("norm", "train"):
        d = case["dim"]
        if kind == "norm":
            return {"bytes": 2 * n * d * e + 8 * d, "flops": 8 * n * d}
        # x, residual -> y, h; dy, dh (h once more) -> dx; the two gradients
        return {"bytes": 7 * n * d * e + 16 * d, "flops": 24 * n * d}
    k, out = case["k"], case["out"]
    rows = sum(_shares(case))                                               # that have a type
    used = sum(1 - math.exp(-v) for v in _shares(case))                     # types that have rows
    weights = used * out * k * e
    if kind == "linear":
        return {"bytes": rows * k * e + n * out * e + weights + 4 * n, "flops": 2 * rows * k * out}
    b = rows * k * e + 2 * n * out * e + n * k * e + weights + case["types"] * out * k * e + 4 * n
    if kind == "layer":                 # ids, residual and its gradient besides
        b += 8 * n + 2 * n * out * e
    return {"bytes": b, "flops": 6 * rows * k * out}


# ---- the operators' definitions in 64 bits ----------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    with torch.no_grad():
        if kind == "group":
            return _exact_group(case, s)
        if kind in ("norm", "train"):
            return _exact_norm(case, s)
        return _exact_linear(case, s)


def _exact_types(case, s):
    """The type of every row, -1 for none."""
    if s["ids"] is None:
        return s["of"]
    there = s["ids"] >= 0
    t = torch.full((case["rows"],), -1, device="cuda", dtype=torch.int32)
    t[there] = s["of"][s["ids"][there].long()]
    return t


def _exact_group(case, s):
    t = _exact_types(case, s)
    lists = [torch.nonzero(t == g)[:, 0] for g in range(case["types"])] + [torch.nonzero(t < 0)[:, 0]]
    begin = [0]
    for rows in lists[:-1]:
        begin.append(begin[-1] + len(rows))
    return torch.cat(lists).to(torch.int32), torch.tensor(begin, device="cuda")


def _normed(h, gamma, beta):
    sd = (h.var(1, unbiased=False, keepdim=True) + EPS).sqrt()
    xh = (h - h.mean(1, keepdim=True)) / sd
    return xh * gamma.double() + beta.double(), xh, sd


def _norm_gradients(dy, xh, sd, gamma):
    """Through the matrix of derivatives of a row, (I - 1 1'/d - xh xh'/d) / sd."""
    d = dy.shape[1]
    g = dy.double() * gamma.double()
    dx = (g - g.sum(1, keepdim=True) / d - xh * ((xh * g).sum(1, keepdim=True) / d)) / sd
    return dx, (dy.double() * xh).sum(0), dy.double().sum(0)


def _exact_norm(case, s):
    if case["kind"] == "norm":
        return _normed(s["x"].double(), s["gamma"], s["beta"])[0]
    h = s["x"].double() + s["res"].double()
    y, xh, sd = _normed(h.to(s["type"]).double(), s["gamma"], s["beta"])    # the norm is of the sum as it is kept
    dx, dgamma, dbeta = _norm_gradients(s["dy"], xh, sd, s["gamma"])
    return y, h, dx + s["dh"].double(), dgamma, dbeta


def _exact_linear(case, s):
    t = _exact_types(case, s)
    n, k, out, types = case["rows"], case["k"], case["out"], case["types"]
    x, w = s["x"].double(), s["w"].double()
    rows = [(g, torch.nonzero(t == g)[:, 0]) for g in range(types)]
    y = torch.zeros(n, out, dtype=torch.float64, device="cuda")
    for g, i in rows:
        y[i] = x[i] @ w[g].T + (0 if s["b"] is None else s["b"][g].double())
    if case["kind"] == "linear":
        return y
    d, first = s["dy"].double(), [y]
    if case["kind"] == "layer":
        z, xh, sd = _normed(y + s["res"].double(), s["gamma"], s["beta"])
        d, dgamma, dbeta = _norm_gradients(d, xh, sd, s["gamma"])
        first = [z]
        last = [d, dgamma, dbeta]
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros(types, out, dtype=torch.float64, device="cuda")
    for g, i in rows:
        dx[i], dw[g], db[g] = d[i] @ w[g], d[i].T @ x[i], d[i].sum(0)
    grads = [dx, dw, db if s["b"] is not None else None]
    return tuple(first + grads + (last if case["kind"] == "layer" else []))
