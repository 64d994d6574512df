"""The 8-bit serving operators of a temporal attention layer, as timed cases.

Five kinds of pass:

* ``project``  the layer's input: residual's addition, root-mean-square norm
               and rounding of the rows to 8 bits (``norm_quant``), then the
               8-bit product with the projection's weights (``linear_i8``);
* ``linear``   the 8-bit product alone (``linear_i8``), rows already rounded;
* ``write``    keys and values appended to the histories of an 8-bit cache
               (``cache_write``), and the touched pages read back
               (``cache_read``);
* ``read``     keys and values of sampled slots read back (``cache_read``);
* ``attend``   attention of roots over sampled slots, or over their histories
               (``cache_attend``).

A cache holds ``data`` int8 ``[pages, heads, 2, P, Dp]`` (keys, then values;
``Dp`` is the head's width rounded up to 16) and one float32 scale per page,
head and kind.  Position p of a sequence is row ``p % P`` of page
``table[seq, p // P]``; a negative page is padding.
"""
import math

import torch

own = False

EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
TINY = 2.0 ** -100


def listed():
    return [
        # one event arrives: its 768-dim row (MAG's node features) through a fused projection
        dict(name="project_event", kind="project", rows=1, dim=768, out=2304, dtype="bf16"),
        # one batch of roots: 4000 edges x (source, destination, negative), MAG's width
        dict(name="project_batch", kind="project", rows=12_000, dim=768, out=1024, dtype="bf16"),
        # the paper's hidden width in float32: 172-dim edge features + 100-dim time encoding, an odd row count
        dict(name="linear_hidden", kind="linear", rows=1801, k=272, out=100, bias=True, dtype="f32"),
        # a super-batch through a wide feed-forward layer
        dict(name="linear_wide", kind="linear", rows=16_384, k=4096, out=4096, bias=False, dtype="bf16"),
        # one new event for each of 4000 nodes, into histories of up to 512 events
        dict(name="append_events", kind="write", seqs=4000, lo=1, hi=1, kept=512, page=16, heads=2, dim=50, dtype="f32"),
        # whole histories written at once, as after a restart
        dict(name="write_histories", kind="write", seqs=300, lo=1, hi=2047, kept=0, page=32, heads=8, dim=128, dtype="bf16"),
        # keys and values of one batch's sampled slots: 12,000 roots x 10, a page per node
        dict(name="read_slots", kind="read", seqs=12_000, slots=10, nodes=2_000_000, heads=2, dim=50, dtype="f32"),
        # the paper's attention layer over those slots: 2 heads of 50, some roots without neighbours
        dict(name="attend_slots", kind="attend", seqs=12_000, q=1, lo=0, hi=10, window=0, page=1, heads=2, group=1,
             dim=50, nodes=2_000_000, dtype="f32"),
        # one root with one long history (GDELT's hot nodes): latency and a split of the long axis
        dict(name="attend_long", kind="attend", seqs=1, q=1, lo=1_000_003, hi=1_000_003, window=0, page=64, heads=8,
             group=4, dim=128, nodes=0, dtype="bf16"),
        # a serving batch with histories of every length up to 8192
        dict(name="attend_histories", kind="attend", seqs=64, q=1, lo=1, hi=8192, window=0, page=16, heads=8, group=4,
             dim=128, nodes=0, dtype="bf16"),
        # the same nodes' newest window only, few heads, small pages
        dict(name="attend_window", kind="attend", seqs=600, q=1, lo=1, hi=3000, window=1000, page=4, heads=2, group=2,
             dim=64, nodes=0, dtype="bf16"),
        # 256 new events of each of 4 nodes, every one over its past
        dict(name="attend_events", kind="attend", seqs=4, q=256, lo=2500, hi=4097, window=0, page=16, heads=8, group=4,
             dim=128, nodes=0, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["project", "linear", "write", "read", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "project":
        return dict(kind=kind, rows=_log(rng, 1, 12_000), dim=_log(rng, 64, 2048), out=_log(rng, 64, 2304), dtype=dtype)
    if kind == "linear":
        return dict(kind=kind, rows=_log(rng, 1, 16_384), k=_log(rng, 64, 4096), out=_log(rng, 64, 4096),
                    bias=rng.random() < 0.5, dtype=dtype)
    heads, dim = rng.choice([1, 2, 4, 8]), rng.choice([32, 50, 64, 96, 100, 128, 200, 256])
    if kind == "write":
        hi = _log(rng, 1, 2000)
        seqs = _log(rng, 1, max(2, min(4000, 600_000_000 // (hi * heads * dim * 2))))
        return dict(kind=kind, seqs=seqs, lo=1, hi=hi, kept=rng.choice([0, 100, 512]), page=rng.choice([1, 2, 4, 8, 16, 32, 64]),
                    heads=heads, dim=dim, dtype=dtype)
    if kind == "read":
        return dict(kind=kind, seqs=_log(rng, 1, 12_000), slots=rng.randint(1, 30), nodes=rng.choice([1000, 100_000, 1_000_000]),
                    heads=rng.choice([1, 2, 4]), dim=min(dim, 128), dtype=dtype)
    group = rng.choice([1, 1, 2, 4, 8])
    if rng.random() < 0.3:
        return dict(kind=kind, seqs=_log(rng, 1, 12_000), q=1, lo=0, hi=rng.randint(1, 30), window=0, page=1,
                    heads=min(heads, 4), group=group, dim=min(dim, 128), nodes=rng.choice([1000, 100_000, 1_000_000]), dtype=dtype)
    hi = _log(rng, 16, 100_000)
    seqs = _log(rng, 1, max(2, min(600, 400_000_000 // (hi * heads * dim * 2))))
    q = rng.choice([1, 1, 1, 2, 7, 64])
    if seqs * q * heads * group * hi > 1 << 27:
        q = 1
    return dict(kind=kind, seqs=seqs, q=q, lo=rng.choice([0, 1, hi]), hi=hi, window=rng.choice([0, 0, 100, 5000]),
                page=rng.choice([1, 2, 4, 8, 16, 32, 64, 128]), heads=heads, group=group, dim=dim, nodes=0, dtype=dtype)


def _spread(n, lo, hi):
    """n lengths spread evenly over [lo, hi]."""
    i = torch.arange(n)
    return lo + ((hi - lo + 1) * (2 * i + 1)) // (2 * n)


def _seen(lengths, q, window):
    """Positions that some query of each sequence sees."""
    return lengths.clamp(max=window + q - 1) if window else lengths


def _round16(d):
    return (d + 15) // 16 * 16


class _Random:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, *shape):
        return torch.randn(*shape, device="cuda", generator=self.g)

    def ints(self, lo, hi, *shape, dtype=torch.int64):
        return torch.randint(lo, hi, shape, device="cuda", generator=self.g, dtype=dtype)

    def order(self, n):
        return torch.randperm(n, device="cuda", generator=self.g)


def _int8_rows(r, rows, k):
    """Rows in 8 bits as a quantiser leaves them: 16-byte aligned, a scale each."""
    x = r.normal(rows, k)
    s = x.abs().amax(1) / 127
    q = torch.zeros(rows, _round16(k), device="cuda", dtype=torch.int8)[:, :k]
    q.copy_(torch.round(x / s[:, None]))
    return q, s


def _new_cache(r, pages, heads, page, dim):
    data = r.ints(-127, 128, pages, heads, 2, page, _round16(dim), dtype=torch.int8)
    data[..., dim:] = 0
    scales = torch.exp(0.5 * r.normal(pages, heads, 2)) / 64
    return data, scales


def _tables(r, lengths, page):
    """Every sequence its own pages, in no order; -1 past its end."""
    need = (lengths + page - 1) // page
    width = max(1, int(need.max()))
    pages = max(1, int(need.sum()))
    table = torch.full((len(lengths), width), -1, device="cuda", dtype=torch.int32)
    at = torch.arange(width, device="cuda")[None, :] < need.cuda()[:, None]
    table[at] = r.order(pages)[: int(need.sum())].to(torch.int32)
    return table, pages


def prepare(case, seed):
    r = _Random(seed)
    s = dict(case)
    s["type"] = TYPES[case["dtype"]]
    if case["kind"] in ("project", "linear"):
        k = case["dim"] if case["kind"] == "project" else case["k"]
        s["wq"], s["ws"] = _int8_rows(r, case["out"], k)
        s["ws"] /= math.sqrt(k)
        if case["kind"] == "project":
            s["x"] = r.normal(case["rows"], k).to(s["type"])
            s["r"] = (2 * r.normal(case["rows"], k)).to(s["type"])
            s["w"] = 1 + 0.1 * r.normal(k)
        else:
            s["xq"], s["xs"] = _int8_rows(r, case["rows"], k)
            s["b"] = r.normal(case["out"]) if case["bias"] else None
        return s
    heads, dim = case["heads"], case["dim"]
    if case["kind"] == "write":
        n = case["seqs"]
        kept = _spread(n, 0, case["kept"])[torch.randperm(n, generator=torch.Generator().manual_seed(int(seed)))]
        new = _spread(n, case["lo"], case["hi"])
        P = case["page"]
        s["table"], pages = _tables(r, kept + new, P)
        s["data"], s["scales"] = _new_cache(r, pages, heads, P, dim)
        s["start"] = kept.cuda()
        s["offsets"] = torch.nn.functional.pad(new.cumsum(0), (1, 0)).cuda()
        s["tokens"] = int(new.sum())
        # both as a fused projection leaves them: keys and values beside each other
        kv = (2 * r.normal(s["tokens"], 2, heads, dim)).to(s["type"])
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
        back = kept // P * P            # read back from the first touched page's start
        s["back"] = back.cuda()
        s["back_offsets"] = torch.nn.functional.pad((kept + new - back).cumsum(0), (1, 0)).cuda()
        s["back_tokens"] = int((kept + new - back).sum())
        return s
    if case["kind"] == "read":
        s["data"], s["scales"] = _new_cache(r, case["nodes"], heads, 1, dim)
        s["table"] = r.ints(0, case["nodes"], case["seqs"], case["slots"], dtype=torch.int32)
        s["table"][r.ints(0, 10, case["seqs"], case["slots"]) == 0] = -1
        return s
    n, T = case["seqs"], case["q"]
    lengths = _spread(n, case["lo"], case["hi"])[torch.randperm(n, generator=torch.Generator().manual_seed(int(seed)))]
    s["begin"] = s["end"] = None
    if case["nodes"]:                   # sampled slots: a page per node, empty slots are padding
        s["data"], s["scales"] = _new_cache(r, case["nodes"], heads, 1, dim)
        s["table"] = r.ints(0, case["nodes"], n, case["hi"], dtype=torch.int32)
        s["table"][torch.arange(case["hi"], device="cuda")[None, :] >= lengths.cuda()[:, None]] = -1
    else:
        s["table"], pages = _tables(r, lengths, case["page"])
        s["data"], s["scales"] = _new_cache(r, pages, heads, case["page"], dim)
        s["end"] = lengths.cuda()
        if case["window"]:
            s["begin"] = (s["end"] - case["window"] - (T - 1)).clamp(min=0)
    # keys are near 73 x scale in size: queries that give scores of a few units
    s["query"] = (r.normal(n, T, heads * case["group"], dim) * 1.5).to(s["type"])
    return s


# ---- the operators in their plain form --------------------------------------

def _plain_norm(x, res, w):
    h = x.float() + res.float()
    t = h * w
    a = t.abs().amax(1, keepdim=True)
    s = torch.where(a < TINY, torch.zeros_like(a), a / 127)
    q = torch.round(t * torch.where(a < TINY, torch.zeros_like(a), 1 / s))
    return q, s / torch.sqrt(h.square().mean(1, keepdim=True) + EPS), h.to(x.dtype)


def _plain_linear(q, s, wq, ws, b, dtype):
    y = torch.matmul(q, wq.float().t()) * s * ws
    return (y if b is None else y + b).to(dtype)


def _places(table, start, offsets, tokens, P):
    """Page (or -1) and row of each of the tokens' places, and its sequence."""
    t = torch.arange(tokens, device="cuda")
    seq = torch.searchsorted(offsets, t, right=True) - 1
    pos = start[seq] + t - offsets[seq]
    return table[seq, pos // P].long(), pos % P, seq


def _plain_write(s):
    data, scales, P, D = s["data"], s["scales"], s["page"], s["dim"]
    page, row, _ = _places(s["table"], s["start"], s["offsets"], s["tokens"], P)
    x = torch.stack([s["k"], s["v"]], 2).float()                        # [tokens, heads, 2, dim]
    top = torch.zeros_like(scales)
    top.scatter_reduce_(0, page[:, None, None].expand(-1, *scales.shape[1:]), x.abs().amax(-1), "amax")
    new = torch.where(top < TINY, torch.zeros_like(top), top / 127)
    some = s["start"] % P > 0                                           # histories that end inside a page
    first = s["table"].gather(1, (s["start"] // P).clamp(max=s["table"].shape[1] - 1)[:, None])[:, 0][some].long()
    old = scales[first]
    new[first] = torch.maximum(new[first], old)
    inv = torch.where(new == 0, torch.zeros_like(new), 1 / new)
    kept = torch.arange(P, device="cuda")[None, :] < (s["start"][some] % P)[:, None]
    was = data[first]
    again = torch.round(was.float() * (old * inv[first])[..., None, None]).to(torch.int8)
    data[first] = torch.where(kept[:, None, None, :, None], again, was)
    data[page, :, :, row, :D] = torch.round(x * inv[page][..., None]).to(torch.int8)
    scales[page] = new[page]


def _plain_read(data, scales, page, row, D, dtype):
    ok = (page >= 0) & (page < data.shape[0])
    at = page.clamp(0, data.shape[0] - 1)
    x = data[at, :, :, row, :D].float() * scales[at][..., None]
    x = torch.where(ok[:, None, None, None], x, torch.zeros_like(x)).to(dtype)
    return x[:, :, 0], x[:, :, 1]


def _plain_attend(s):
    data, scales, table, q = s["data"], s["scales"], s["table"].long(), s["query"]
    n, T, H, D = q.shape
    heads, P = data.shape[1], data.shape[3]
    L = table.shape[1] * P
    at = table.clamp(0, data.shape[0] - 1)
    kv = (data[at][..., :D].float() * scales[at][..., None, None]).permute(3, 0, 2, 1, 4, 5).reshape(2, n, heads, L, D)
    pos = torch.arange(L, device="cuda")
    seen = (table >= 0).repeat_interleave(P, 1)[:, None, :].expand(n, T, L)
    if s["end"] is not None:
        last = s["end"][:, None] - (T - 1) + torch.arange(T, device="cuda")
        seen = seen & (pos < last[..., None])
    if s["begin"] is not None:
        seen = seen & (pos >= s["begin"][:, None, None])
    seen = seen[:, None, None]                                          # [n, 1, 1, T, L]
    g = H // heads
    qh = q.float().reshape(n, T, heads, g, D).permute(0, 2, 3, 1, 4).reshape(n, heads, g * T, D)
    score = torch.matmul(qh, kv[0].transpose(-1, -2)).reshape(n, heads, g, T, L) * (1 / math.sqrt(D))
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    den = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(n, heads, g * T, L), kv[1]).reshape(n, heads, g, T, D)
    o = torch.where(den > 0, o / den, torch.zeros_like(o))
    return o.permute(0, 3, 1, 2, 4).reshape(n, T, H, D).to(q.dtype)


def _plain(s):
    if s["kind"] == "project":
        q, scale, h = _plain_norm(s["x"], s["r"], s["w"])
        return h, _plain_linear(q, scale, s["wq"], s["ws"], None, s["type"])
    if s["kind"] == "linear":
        return _plain_linear(s["xq"].float(), s["xs"][:, None], s["wq"], s["ws"], s["b"], s["type"])
    if s["kind"] == "write":
        _plain_write(s)
        page, row, _ = _places(s["table"], s["back"], s["back_offsets"], s["back_tokens"], s["page"])
        return _plain_read(s["data"], s["scales"], page, row, s["dim"], s["type"])
    if s["kind"] == "read":
        page = s["table"].reshape(-1).long()
        return _plain_read(s["data"], s["scales"], page, torch.zeros_like(page), s["dim"], s["type"])
    return _plain_attend(s)


# ---- the framework's calls --------------------------------------------------

def _own(s):
    import paper_2203_14883_amd as tgl
    if s["kind"] == "project":
        q, scale, h = tgl.norm_quant(s["x"], s["w"], residual=s["r"], eps=EPS)
        return h, tgl.linear_i8(q, scale, s["wq"], s["ws"], out_dtype=s["type"])
    if s["kind"] == "linear":
        return tgl.linear_i8(s["xq"], s["xs"], s["wq"], s["ws"], bias=s["b"], out_dtype=s["type"])
    cache = tgl.HistoryCache(s["data"], s["scales"], s["dim"])
    if s["kind"] == "write":
        tgl.cache_write(cache, s["k"], s["v"], s["table"], start=s["start"], offsets=s["offsets"])
        return tgl.cache_read(cache, s["table"], start=s["back"], offsets=s["back_offsets"], n=s["back_tokens"],
                              out_dtype=s["type"])
    if s["kind"] == "read":
        return tgl.cache_read(cache, s["table"], n=s["table"].numel(), out_dtype=s["type"])
    return tgl.cache_attend(cache, s["query"], s["table"], begin=s["begin"], end=s["end"])


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    e = SIZE[case["dtype"]]
    if case["kind"] in ("project", "linear"):
        m, n = case["rows"], case["out"]
        k = case["dim"] if case["kind"] == "project" else case["k"]
        b = n * k + 4 * n + m * n * e + (3 * m * k * e + 4 * k if case["kind"] == "project" else m * k + 4 * m + 4 * n * case["bias"])
        return {"bytes": b, "flops": 2 * m * n * k}
    row = case["heads"] * case["dim"] * 2               # values of one token: keys and values
    if case["kind"] == "write":
        n, P = case["seqs"], case["page"]
        kept = _spread(n, 0, case["kept"])
        new = int(_spread(n, case["lo"], case["hi"]).sum())
        back = new + int((kept % P).sum())
        return {"bytes": new * row * (e + 1) + back * row * (e + 1), "flops": 3 * new * row + back * row}
    if case["kind"] == "read":
        t = case["seqs"] * case["slots"]
        return {"bytes": t * (row * e + 4) + 0.9 * t * (row + 8 * case["heads"]), "flops": t * row}
    n, T = case["seqs"], case["q"]
    lengths = _spread(n, case["lo"], case["hi"])
    read = int(_seen(lengths, T, case["window"]).sum())
    H = case["heads"] * case["group"]
    io = 2 * n * T * H * case["dim"] * e
    back = T - 1 - torch.arange(T)
    end = (lengths[:, None] - back).clamp(min=0)
    pairs = int((end - (lengths[:, None] - case["window"] - (T - 1)).clamp(min=0)).clamp(min=0).sum() if case["window"] else end.sum())
    return {"bytes": read * (row + 8 * case["heads"] / case["page"] + 4 / case["page"]) + io, "flops": 4 * pairs * H * case["dim"]}


# ---- the operators' definitions in 64 bits ----------------------------------

def _steps(x, dims):
    """The step of the 8-bit values that hold x, by the largest magnitude over dims."""
    return x.abs().amax(dims, keepdim=True) / 127


def _held(x, step):
    """The values that stand for x at a step, 0 where the step is 0."""
    return torch.where(step > 0, torch.round(x / torch.where(step > 0, step, torch.ones_like(step))), torch.zeros_like(x)) * step


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("project", "linear"):
        W = s["wq"].double() * s["ws"].double()[:, None]
        if kind == "linear":
            y = (s["xq"].double() * s["xs"].double()[:, None]) @ W.T
            return y + s["b"].double() if case["bias"] else y
        h = s["x"].double() + s["r"].double()
        y = h * s["w"].double() * (h.pow(2).mean(1, keepdim=True) + EPS).rsqrt()
        return h, _held(y, _steps(y, 1)) @ W.T
    if kind == "read":
        table = s["table"].reshape(-1).long()
        got = s["data"].double()[..., : case["dim"]][:, :, :, 0] * s["scales"].double()[..., None]
        got = torch.cat([got, torch.zeros_like(got[:1])])[torch.where(table < 0, got.shape[0], table)]
        return got[:, :, 0], got[:, :, 1]
    if kind == "write":
        return _exact_write(case, s)
    return _exact_attend(case, s)


def _exact_write(case, s):
    """Page by page: all rows of a touched page in one block, rows that are not there held at 0."""
    P, H, D = case["page"], case["heads"], case["dim"]
    start, offsets, table = s["start"].cpu(), s["offsets"].cpu(), s["table"].cpu()
    counts = offsets[1:] - offsets[:-1]
    first, last = start // P, (start + counts - 1) // P
    per = last - first + 1                                             # pages that each sequence touches
    seq = torch.repeat_interleave(torch.arange(len(per)), per)
    slot = torch.arange(len(seq)) - (per.cumsum(0) - per)[seq] + first[seq]
    pages = table[seq, slot].long().cuda()
    pos = slot[:, None] * P + torch.arange(P)
    is_new = (pos >= start[seq][:, None]) & (pos < (start + counts)[seq][:, None])
    is_kept = pos < start[seq][:, None]
    token = (offsets[:-1][seq][:, None] + pos - start[seq][:, None]).clamp(0, max(0, s["tokens"] - 1)).cuda()
    both = torch.stack([s["k"], s["v"]], 2)[token].double().permute(0, 2, 3, 1, 4)    # [pages, H, 2, P, D]
    new, kept = (m.cuda()[:, None, None, :, None] for m in (is_new, is_kept))
    fresh = torch.where(new, both, torch.zeros_like(both))
    old = s["scales"][pages].double()[..., None, None]
    there = torch.where(kept, s["data"][pages][..., :D].double() * old, torch.zeros_like(both))
    step = torch.maximum(_steps(fresh, (-2, -1)), old * kept.any(3, keepdim=True))
    got = _held(torch.where(new, fresh, there), step).permute(0, 3, 1, 2, 4)          # [pages, P, H, 2, D]
    got = got[(is_new | is_kept).cuda()]                               # in the order of reading back
    return got[:, :, 0], got[:, :, 1]


def _exact_attend(case, s):
    n, T, H, D = s["query"].shape
    heads, P, g = case["heads"], case["page"], case["group"]
    width = s["table"].shape[1]
    o = torch.zeros(n, T, H, D, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 31) // (width * P * heads * max(D, g * T)))    # sequences at a time
    for a in range(0, n, step):
        table = s["table"][a : a + step].long()
        m = len(table)
        pages = s["data"][table.clamp(min=0)][..., :D].double() * s["scales"][table.clamp(min=0)].double()[..., None, None]
        keys = pages[:, :, :, 0].transpose(1, 2).reshape(m, heads, width * P, D)
        values = pages[:, :, :, 1].transpose(1, 2).reshape(m, heads, width * P, D)
        at = torch.arange(width * P, device="cuda")
        t = torch.arange(T, device="cuda")[None, :, None]
        hide = table.lt(0)[:, at // P][:, None, :]
        if s["end"] is not None:
            hide = hide | (at >= s["end"][a : a + step, None, None] - (T - 1 - t))
        if s["begin"] is not None:
            hide = hide | (at < s["begin"][a : a + step, None, None])
        hide = hide.expand(m, T, -1)
        query = s["query"][a : a + step].double().view(m, T, heads, g, D) / math.sqrt(D)
        for j in range(g):
            x = query[:, :, :, j].transpose(1, 2) @ keys.transpose(2, 3)
            x = x.masked_fill(hide[:, None], float("-inf"))
            w = (x - torch.logsumexp(x, -1, keepdim=True)).exp()
            w = torch.where(hide[:, None], torch.zeros_like(w), w)
            o[a : a + step, :, j::g] = (w @ values).transpose(1, 2)
    return o
