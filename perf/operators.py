"""What a decode step needs between its linear layers, as cases that can be timed.

The linear layers stream their weights (``perf/cases.py``); these are the operators next to them:

* ``attention``: one new token per sequence attends to the paged cache of keys and values (grouped heads,
  binary16 or 8-bit pages with a scale per token and head, an optional sliding window).
* ``append``: the new tokens' queries and keys are rotated, keys and values are written to the pages of their
  sequences: one token each in a decode step, thousands in packed prompts.
* ``fork`` / ``compact`` / ``turnover``: the pages of the cache: sequences that share a parent's pages, a pool
  squeezed to its lowest pages, finished sequences freed and room reserved for new ones.
* ``norm``: the residual stream takes a block's output (normed, gated, scaled) and is normed for the next block.

Head counts and widths are those of the 7B-, 8B-, 13B- and 70B-class blocks of ``perf/cases.py`` and generic
ones around them.  With ``own`` the framework's entry points run; without, elementary torch operations in
32 bits compute the same outputs, rounded once at the end.
"""
import math
from types import SimpleNamespace

import torch

own = False   # (the framework is imported where it is called: a tree without the operators can load this file)

DEV = "cuda"


# ---- the cases ----------------------------------------------------------------------------------------------

def _attention(seqs, lo, hi, q_heads, kv_heads, dim, page, int8=False, window=0):
    return {"kind": "attention", "seqs": seqs, "lo": lo, "hi": hi, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "page": page, "int8": int8, "window": window}


def _append(seqs, tokens, step, q_heads, kv_heads, dim, page, int8, rot, interleaved):
    return {"kind": "append", "seqs": seqs, "tokens": tokens, "step": step, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "page": page, "int8": int8, "rot": rot, "interleaved": interleaved}


def _fork(parents, children, length, layers, kv_heads, dim, page, pages, int8=False):
    return {"kind": "fork", "parents": parents, "children": children, "length": length, "layers": layers, "kv_heads": kv_heads,
            "dim": dim, "page": page, "pages": pages, "int8": int8}


def _compact(seqs, live, layers, kv_heads, dim, page, pages, int8=False):
    return {"kind": "compact", "seqs": seqs, "live": live, "layers": layers, "kv_heads": kv_heads, "dim": dim, "page": page,
            "pages": pages, "int8": int8}


def _turnover(seqs, leave, length, page, pages):
    return {"kind": "turnover", "seqs": seqs, "leave": leave, "length": length, "page": page, "pages": pages}


def _norm(rows, cols, layer, post, gate, wide, scale):
    return {"kind": "norm", "rows": rows, "cols": cols, "layer": layer, "post": post, "gate": gate, "wide": wide, "scale": scale}


def listed():
    return [
        # one user, a short chat, an 8B-class model: the smallest call, launch and latency
        dict(_attention(1, 512, 512, 32, 8, 128, 16), name="attention_1seq_512"),
        # a decode batch of sixteen users at all lengths, the same model
        dict(_attention(16, 1, 8192, 32, 8, 128, 16), name="attention_16seq_8b"),
        # five sequences of a 7B-class model, every query head its own keys
        dict(_attention(5, 701, 3001, 32, 32, 128, 32), name="attention_5seq_7b_mha"),
        # many short sequences with narrow heads and small pages: a serving batch at its start
        dict(_attention(200, 1, 600, 64, 8, 64, 8), name="attention_200seq_short"),
        # sixteen long documents of a 70B-class model in an 8-bit cache: the largest pass
        dict(_attention(16, 32768, 131072, 64, 8, 128, 64, int8=True), name="attention_16seq_70b_long"),
        # one decode step of sixteen sequences: latency
        dict(_append(16, 16, True, 32, 8, 128, 16, False, 128, False), name="append_step_16"),
        # five packed prompts of a 70B-class model into an 8-bit cache
        dict(_append(5, 8192, False, 64, 8, 128, 64, True, 128, False), name="append_prompt_int8"),
        # four prompts continued four times each: pages shared, the last page of each child copied in every layer
        dict(_fork(4, 4, 3001, 16, 8, 128, 64, 240), name="fork_4x4"),
        # a fragmented pool, 40 % of it live, squeezed before a long prompt is taken
        dict(_compact(24, 0.4, 8, 8, 128, 16, 4096), name="compact_4096"),
        # sixteen of 256 sequences end, sixteen prompts take their rows: bookkeeping only
        dict(_turnover(256, 16, 3500, 16, 65536), name="turnover_256"),
        # the step between two blocks for one token of a 7B-class model
        dict(_norm(1, 4096, False, False, "none", False, 1.0), name="norm_1x4096"),
        # the same for a prompt of a 70B-class model, both norms, a gate per channel, the residual stream in 32 bits
        dict(_norm(8192, 8192, False, True, "channel", True, 0.5), name="norm_8192x8192"),
    ]


def _log(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def draw(rng):
    kind = rng.choice(("attention", "attention", "attention", "append", "append", "fork", "compact", "turnover", "norm", "norm"))
    page = rng.choice((8, 16, 32, 64, 128))
    dim = rng.choice((64, 80, 96, 128, 128, 192, 256))
    kv_heads = rng.choice((1, 2, 5, 8, 8, 32))
    int8 = rng.random() < 0.4
    if kind == "attention":
        group = rng.choice((1, 2, 3, 4, 7, 8, 12, 16, 20)) if kv_heads <= 8 else rng.choice((1, 2))
        seqs = int(_log(rng, 1, 256))
        most = 2.4e9 / (seqs * kv_heads * dim * 4)   # tokens per sequence: a bound on the plain form's memory
        hi = max(1, int(min(131072, most, _log(rng, 16, 131072))))
        lo = rng.choice((0, 1, hi // 2, hi))
        window = rng.choice((0, 0, 0, 1 + int(_log(rng, 8, 8192))))
        return _attention(seqs, lo, hi, kv_heads * group, kv_heads, dim, page, int8, window)
    if kind == "append":
        step = rng.random() < 0.5
        seqs = int(_log(rng, 1, 64))
        group = rng.choice((1, 2, 4, 5, 8)) if kv_heads <= 8 else 1
        tokens = seqs if step else max(seqs, int(_log(rng, 64, 8192)))
        rot = rng.choice((0, dim, dim, 16 * (dim // 32)))
        return _append(seqs, tokens, step, kv_heads * group, kv_heads, dim, page, int8, rot, rng.random() < 0.4)
    if kind in ("fork", "compact"):
        layers = rng.choice((1, 2, 5, 8))
        pages = max(96, int(min(4096, 2.5e8 / (layers * kv_heads * dim * page)) * rng.uniform(0.3, 1.0)))
        if kind == "compact":
            return _compact(int(_log(rng, 1, 64)), rng.uniform(0.1, 0.95), layers, kv_heads, dim, page, pages, int8)
        parents, children = rng.choice((1, 2, 3, 4)), rng.choice((1, 2, 3, 5))
        length = 1 + int(rng.random() * (page * (pages - parents * children) // parents - page))
        return _fork(parents, children, length, layers, kv_heads, dim, page, pages, int8)
    if kind == "turnover":
        seqs = int(_log(rng, 2, 512))
        pages = int(_log(rng, 1024, 100000))
        return _turnover(seqs, rng.randint(1, max(1, seqs // 4)), max(1, int(0.6 * pages * page / seqs)), page, pages)
    cols = rng.choice((4096, 8192, 1 + int(_log(rng, 63, 16384)), 8 * int(_log(rng, 16, 2048))))
    rows = int(min(_log(rng, 1, 16384), 6.7e7 / cols)) or 1
    return _norm(rows, cols, rng.random() < 0.4, rng.random() < 0.5, rng.choice(("none", "channel", "element")), rng.random() < 0.5,
                 rng.choice((1.0, 0.25, 1.4)))


# ---- what a program has in hand -----------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(0x5EED0 + int(seed))
    return g


def _half(g, *shape, sigma=1.0):
    t = torch.empty(shape, dtype=torch.float16, device=DEV)
    return t.normal_(0.0, sigma, generator=g)


def _ints(g, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=g, device=DEV, dtype=torch.int32)


def _lengths(g, c):
    """Lengths over the case's range, both ends among them."""
    n = _ints(g, c["lo"], c["hi"] + 1, c["seqs"])
    n[-1] = c["hi"]
    if c["seqs"] > 1:
        n[0] = c["lo"]
    return n


def _pool(g, int8, *shape):
    """Keys or values of `shape` (..., page, heads, tokens, dim): binary16, or 8-bit integers and a scale per row."""
    if not int8:
        return _half(g, *shape), None
    ints = torch.empty(shape, dtype=torch.int8, device=DEV)
    ints.random_(-127, 128, generator=g)
    return ints, torch.empty(shape[:-1], dtype=torch.float32, device=DEV).uniform_(0.005, 0.03, generator=g)


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = SimpleNamespace(c=c)
    if c["kind"] == "norm":
        n, m = c["rows"], c["cols"]
        s.x = _half(g, n, m, sigma=2.0)
        s.x = s.x.float() if c["wide"] else s.x
        s.y = _half(g, n, m)
        ones = lambda sigma: (1 + _half(g, m, sigma=sigma).float()).half()  # noqa: E731
        s.post_w, s.pre_w = ones(0.1) if c["post"] else None, ones(0.2)
        s.post_b = _half(g, m, sigma=0.1) if c["post"] and c["layer"] else None
        s.pre_b = _half(g, m, sigma=0.1) if c["layer"] else None
        s.gate = {"none": None, "channel": _half(g, m, sigma=0.5)}.get(c["gate"], None)
        if c["gate"] == "element":
            s.gate = _half(g, n, m, sigma=0.5)
        s.x_out, s.h = torch.empty_like(s.x), torch.empty(n, m, dtype=torch.float16, device=DEV)
        return s
    page = c["page"]
    if c["kind"] == "attention":
        s.len = _lengths(g, c)
        stride = -(-c["hi"] // page)
        pages = c["seqs"] * stride
        s.table = torch.randperm(pages, generator=g, device=DEV).int().view(c["seqs"], stride)
        s.k, s.ks = _pool(g, c["int8"], pages, c["kv_heads"], page, c["dim"])
        s.v, s.vs = _pool(g, c["int8"], pages, c["kv_heads"], page, c["dim"])
        s.scale = c["dim"] ** -0.5
        # as the projections give it: queries, keys and values of a token in one row
        s.q = _half(g, c["seqs"], (c["q_heads"] + 2 * c["kv_heads"]) * c["dim"], sigma=1.5)
        s.out = torch.empty(c["seqs"], c["q_heads"], c["dim"], dtype=torch.float16, device=DEV)
        s.lse = torch.empty(c["seqs"], c["q_heads"], dtype=torch.float32, device=DEV)
        return s
    if c["kind"] == "append":
        n = c["seqs"]
        if c["step"]:
            new = torch.ones(n, dtype=torch.int32, device=DEV)
            before = _ints(g, 0, 4 * page, n)
        else:   # packed prompts of different lengths, each of one token at least
            cuts = torch.randperm(c["tokens"] - 1, generator=g, device=DEV)[:n - 1].sort().values.int() + 1
            ends = torch.cat([cuts, torch.tensor([c["tokens"]], dtype=torch.int32, device=DEV)])
            new = torch.diff(ends, prepend=torch.zeros(1, dtype=torch.int32, device=DEV))
            before = _ints(g, 0, page, n)
        s.starts = torch.nn.functional.pad(new.cumsum(0), (1, 0)).int()
        s.len = (before + new).int()
        need = -(-s.len // page)
        stride = 5 if c["step"] else -(-c["tokens"] // page) + 1
        pages = n * 5 + 3 if c["step"] else -(-c["tokens"] // page) + 2 * n + 3
        s.table = torch.zeros(n, stride, dtype=torch.int32, device=DEV)
        order = torch.randperm(pages, generator=g, device=DEV).int()
        s.table[torch.arange(stride, device=DEV)[None] < need[:, None]] = order[:int(need.sum())]
        s.k, s.ks = _pool(g, c["int8"], pages, c["kv_heads"], page, c["dim"])
        s.v, s.vs = _pool(g, c["int8"], pages, c["kv_heads"], page, c["dim"])
        s.qkv = _half(g, c["tokens"], (c["q_heads"] + 2 * c["kv_heads"]) * c["dim"])
        s.q_out = torch.empty(c["tokens"], c["q_heads"] * c["dim"], dtype=torch.float16, device=DEV)
        s.q_out.copy_(s.qkv[:, :c["q_heads"] * c["dim"]])
        if c["int8"]:   # room for the values that the cache stands for
            s.read_k, s.read_v = (torch.empty(s.k.shape, dtype=torch.float16, device=DEV) for _ in range(2))
        # the far end of a long context too: the table's rows are the positions from an offset on
        at = torch.arange(stride * page, device=DEV, dtype=torch.float64) + 50000
        freq = 500000.0 ** (-torch.arange(c["rot"] // 2, device=DEV, dtype=torch.float64) / max(1, c["rot"] // 2))
        angle = at[:, None] * freq[None]
        s.rope = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
        return s
    # pages of a cache: one block of whole numbers holds the table, the lengths and the reference counts
    if c["kind"] == "fork":
        rows = c["parents"] * (1 + c["children"])
        stride = -(-c["length"] // page) + 1
    else:
        rows = c["seqs"]
        stride = c["pages"] if c["kind"] == "compact" else 2 * (-(-c["length"] // page)) + 2
    pages = c["pages"]
    s.rows, s.stride = rows, stride
    table, length = torch.zeros(rows, stride, dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    order = torch.randperm(pages, generator=g, device=DEV).int()
    if c["kind"] == "fork":
        n = c["parents"]
        length[:n] = torch.clamp(c["length"] - _ints(g, 0, page, n), min=1)
        length[0] = c["length"]
        pairs = torch.stack([torch.arange(n, device=DEV).repeat_interleave(c["children"]),
                             torch.arange(n * c["children"], device=DEV) + n], 1)
        s.pairs = pairs[torch.randperm(pairs.shape[0], generator=g, device=DEV)].int().contiguous()
    elif c["kind"] == "compact":
        total = max(rows, int(c["live"] * pages)) - rows   # every sequence has a page, the rest as it falls
        share = torch.bincount(torch.randint(0, rows, (total,), generator=g, device=DEV), minlength=rows) + 1
        length[:] = share.int() * page - _ints(g, 0, page, rows)
    else:
        length[:] = torch.clamp(_ints(g, c["length"] // 2, c["length"] + 1, rows), min=1)
        s.leave = torch.randperm(rows, generator=g, device=DEV)[:c["leave"]].int().sort().values.int()
        s.new = torch.ones(rows, dtype=torch.int32, device=DEV)   # a token for those that stay, a prompt for those that come
        s.new[s.leave.long()] = _ints(g, 1, c["length"] + 1, c["leave"])
    need = -(-length // page)
    mask = torch.arange(stride, device=DEV)[None] < need[:, None]
    table[mask] = order[:int(need.sum())]
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    refs[table[mask].long()] = 1
    s.first = torch.cat([table.reshape(-1), length, refs])
    s.books = s.first.clone()
    s.table = s.books[:rows * stride].view(rows, stride)
    s.len = s.books[rows * stride:rows * stride + rows]
    s.refs = s.books[rows * stride + rows:]
    s.status = torch.zeros(2, dtype=torch.int32, device=DEV)
    s.most = int(length.max())
    if c["kind"] != "turnover":
        s.kv, s.scales = _pool(g, c["int8"], c["layers"], 2, pages, c["kv_heads"], page, c["dim"])
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------

def _plain_attention(s):
    c = s.c
    n, hq, hk, d, page = c["seqs"], c["q_heads"], c["kv_heads"], c["dim"], c["page"]
    q = s.q[:, :hq * d].view(n, hk, hq // hk, d).float()
    at = s.table.long()

    def rows(pool, scale):
        x = pool[at].float()                                          # [n][pages][heads][tokens][dim]
        x = x if scale is None else x * scale[at][..., None]
        return x.permute(0, 2, 1, 3, 4).reshape(n, hk, -1, d)

    score = torch.matmul(q, rows(s.k, s.ks).transpose(-1, -2)) * s.scale   # [n][hk][group][t]
    t = torch.arange(score.shape[-1], device=DEV)[None]
    keep = t < s.len[:, None]
    if c["window"]:
        keep = keep & (t >= s.len[:, None] - c["window"])
    score = score.masked_fill(~keep[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = (score - top).exp()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, rows(s.v, s.vs)) / torch.where(total > 0, total, torch.ones_like(total))
    return out.reshape(n, hq, d).half(), (total.log() + top).reshape(n, hq)


def _rotate(x, cs, rot, interleaved):
    if not rot:
        return x
    cos, sin = cs[..., 0][:, None], cs[..., 1][:, None]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_append(s):
    c = s.c
    hq, hk, d, page, n = c["q_heads"], c["kv_heads"], c["dim"], c["page"], c["tokens"]
    j = torch.arange(n, device=DEV)
    seq = torch.searchsorted(s.starts[1:].contiguous(), j.int(), right=True)
    pos = (s.len[seq] - s.starts[seq + 1] + j).long()
    where, slot = s.table[seq, pos // page].long(), pos % page
    x = s.qkv.float().view(n, hq + 2 * hk, d)
    turned = _rotate(x[:, :hq + hk], s.rope[pos], c["rot"], c["interleaved"])

    def put(pool, scale, rows):
        if scale is None:
            pool[where, :, slot] = rows.half()
            return
        top = rows.abs().amax(-1)
        step = top / 127
        pool[where, :, slot] = (rows / torch.where(step > 0, step, torch.ones_like(step))[..., None]).round().to(torch.int8)
        scale[where, :, slot] = step

    put(s.k, s.ks, turned[:, hq:])
    put(s.v, s.vs, x[:, hq + hk:])
    s.q_out.copy_(turned[:, :hq].reshape(n, hq * d))


def _free_pages(refs):
    """Page numbers, the free ones first and in order."""
    return torch.argsort((refs != 0).to(torch.int8), stable=True)


def _plain_fork(s):
    c, page = s.c, s.c["page"]
    parent, child = s.pairs[:, 0].long(), s.pairs[:, 1].long()
    length = s.len[parent]
    full, rest = length // page, length % page
    needs = rest > 0
    fresh = _free_pages(s.refs)[needs.cumsum(0) - needs.long()]
    j = torch.arange(s.stride, device=DEV)[None]
    above = s.table[parent]
    last = above.gather(1, torch.clamp(full, max=s.stride - 1)[:, None].long())[:, 0].long()
    row = torch.where(j < full[:, None], above, s.table[child])
    row = torch.where((j == full[:, None]) & needs[:, None], fresh[:, None].int(), row)
    s.table[child] = row
    s.len[child] = length
    shared = (j < full[:, None]).int()
    s.refs.scatter_add_(0, above.reshape(-1).long(), shared.reshape(-1))
    s.refs.scatter_add_(0, fresh, needs.int())
    s.status.zero_()
    to = torch.where(needs, fresh, last)
    keep = (torch.arange(page, device=DEV)[None] < rest[:, None])[None, None, :, None, :]
    for pool, mask in ((s.kv, keep[..., None]), (s.scales, keep)):
        if pool is not None:
            pool[:, :, to] = torch.where(mask, pool[:, :, last], pool[:, :, to])


def _plain_compact(s):
    live = s.refs > 0
    count = live.sum()
    at = torch.arange(s.refs.numel(), device=DEV)
    src, dst = (live & (at >= count)).nonzero()[:, 0], (~live & (at < count)).nonzero()[:, 0]
    to = at.clone()
    to[src] = dst
    used = torch.arange(s.stride, device=DEV)[None] < (-(-s.len // s.c["page"]))[:, None]
    s.table.copy_(torch.where(used, to[s.table.long()].int(), s.table))
    s.refs[dst] = s.refs[src]
    s.refs[src] = 0
    s.status.copy_(torch.stack([count, torch.tensor(src.numel(), device=DEV)]))
    s.kv[:, :, dst] = s.kv[:, :, src]
    if s.scales is not None:
        s.scales[:, :, dst] = s.scales[:, :, src]


def _plain_turnover(s):
    page = s.c["page"]
    gone = s.leave.long()
    j = torch.arange(s.stride, device=DEV)[None]
    used = (j < (-(-s.len[gone] // page))[:, None]).int()
    s.refs.scatter_add_(0, s.table[gone].reshape(-1).long(), -used.reshape(-1))
    s.len[gone] = 0
    have = -(-s.len // page)
    s.len.add_(s.new)
    need = -(-s.len // page) - have
    first = need.cumsum(0) - need
    rank = first[:, None] + j - have[:, None]
    mine = (j >= have[:, None]) & (j < (have + need)[:, None])
    order = _free_pages(s.refs)
    pages = order[torch.where(mine, rank, torch.zeros_like(rank)).long()].int()
    s.table.copy_(torch.where(mine, pages, s.table))
    s.refs.scatter_add_(0, pages.reshape(-1).long(), mine.reshape(-1).int())
    s.status.zero_()


def _unit(x, layer, weight, bias, eps):
    if layer:
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * weight
    return x if bias is None else x + bias


EPS = 1e-5


def _plain_norm(s):
    c = s.c
    f = lambda t: None if t is None else t.float()  # noqa: E731
    u = f(s.y)
    if c["post"]:
        u = _unit(u, c["layer"], f(s.post_w), f(s.post_b), EPS)
    if s.gate is not None:
        u = u * f(s.gate)
    x = f(s.x) + c["scale"] * u
    s.x_out.copy_(x)
    s.h.copy_(_unit(x, c["layer"], f(s.pre_w), f(s.pre_b), EPS))


# ---- the framework's calls ----------------------------------------------------------------------------------

def _own_attention(s):
    import paper_2402_15319_b200 as vq
    c = s.c
    if not hasattr(s, "fmt"):   # what a program keeps for its cache
        s.fmt = vq.VQKVFormat(s.k.shape[0], c["page"], c["kv_heads"], c["dim"], vq.VQ_KV_INT8 if c["int8"] else vq.VQ_KV_FP16)
        s.pool, s.seqs = vq.KVPool(s.k, s.v, s.ks, s.vs), vq.KVSeqs(s.table, s.len)
        s.ws = torch.zeros(vq.vq_kv_attention_workspace_bytes(s.fmt), dtype=torch.uint8, device=DEV)
    vq.vq_kv_attention(s.fmt, s.pool, s.seqs, c["q_heads"], s.q, s.q.stride(0), s.out, c["q_heads"] * c["dim"], s.lse, s.scale, c["window"],
                       s.ws)
    return s.out, s.lse


def _own_append(s):
    import paper_2402_15319_b200 as vq
    c = s.c
    if not hasattr(s, "fmt"):
        s.fmt = vq.VQKVFormat(s.k.shape[0], c["page"], c["kv_heads"], c["dim"], vq.VQ_KV_INT8 if c["int8"] else vq.VQ_KV_FP16)
        s.pool, s.seqs = vq.KVPool(s.k, s.v, s.ks, s.vs), vq.KVSeqs(s.table, s.len)
        hq, hk, d = c["q_heads"], c["kv_heads"], c["dim"]
        s.new_k, s.new_v = s.qkv[:, hq * d:], s.qkv[:, (hq + hk) * d:]
        s.rotary = vq.KVRotary(s.rope, s.rope.shape[0], c["rot"], c["interleaved"], hq, s.qkv, s.qkv.stride(0), s.q_out, hq * d) if c["rot"] else None
    vq.vq_kv_append(s.fmt, s.pool, s.seqs, None if c["step"] else s.starts, c["tokens"], s.new_k, s.qkv.stride(0), s.new_v, s.qkv.stride(0),
                    s.rotary)


def _own_pages(s):
    import paper_2402_15319_b200 as vq
    c = s.c
    if not hasattr(s, "fmt"):
        kind = vq.VQ_KV_INT8 if c.get("int8") else vq.VQ_KV_FP16
        s.fmt = vq.VQKVFormat(c["pages"], c["page"], c.get("kv_heads", 8), c.get("dim", 128), kind)
        s.seqs = vq.KVSeqs(s.table, s.len)
        if c["kind"] != "turnover":
            sc = s.scales
            s.pools = [vq.KVPool(s.kv[i, 0], s.kv[i, 1], *((None, None) if sc is None else (sc[i, 0], sc[i, 1]))) for i in range(c["layers"])]
        s.ws = torch.zeros(vq.vq_kv_pages_workspace_bytes(s.fmt, s.rows), dtype=torch.uint8, device=DEV)
    if c["kind"] == "fork":
        vq.vq_kv_fork(s.fmt, s.pools, s.seqs, s.refs, s.pairs, s.pairs.shape[0], s.status, s.ws)
    elif c["kind"] == "compact":
        vq.vq_kv_compact(s.fmt, s.pools, s.seqs, s.refs, s.status, s.ws)
    else:
        vq.vq_kv_free(s.fmt, s.seqs, s.refs, s.leave, s.leave.numel())
        vq.vq_kv_reserve(s.fmt, s.seqs, s.refs, s.new, s.status, s.ws)


def _own_norm(s):
    import paper_2402_15319_b200 as vq
    c = s.c
    if not hasattr(s, "norm"):
        gate = {"none": vq.VQ_GATE_NONE, "channel": vq.VQ_GATE_CHANNEL, "element": vq.VQ_GATE_ELEMENT}[c["gate"]]
        m = c["cols"]
        s.norm = vq.VQNorm(c["rows"], m, vq.VQ_NORM_LAYER if c["layer"] else vq.VQ_NORM_RMS, vq.VQ_RESIDUAL_FP32 if c["wide"] else vq.VQ_RESIDUAL_FP16,
                           gate, EPS, c["scale"], m, m, m, m, m)
    vq.vq_residual_norm(s.norm, s.x, s.y, s.gate, s.post_w, s.post_b, s.pre_w, s.pre_b, s.x_out, s.h)


def run(s):
    kind = s.c["kind"]
    if kind == "attention":
        return _own_attention(s) if own else _plain_attention(s)
    if kind == "append":
        _own_append(s) if own else _plain_append(s)
        if s.ks is None:
            return s.k, s.v, s.q_out
        # the values the cache stands for
        return torch.mul(s.k, s.ks[..., None], out=s.read_k), torch.mul(s.v, s.vs[..., None], out=s.read_v), s.q_out
    if kind == "norm":
        _own_norm(s) if own else _plain_norm(s)
        return s.x_out, s.h
    s.books.copy_(s.first)   # the books as they are before the call: the same call can be made again
    if own:
        _own_pages(s)
    else:
        {"fork": _plain_fork, "compact": _plain_compact, "turnover": _plain_turnover}[kind](s)
    return [s.table, s.len, s.refs, s.status] + ([] if kind == "turnover" else [s.kv]) + ([] if getattr(s, "scales", None) is None else [s.scales])


# ---- what a pass cannot do without --------------------------------------------------------------------------

def work(case):
    c = case
    kind = c["kind"]
    if kind == "norm":
        per = (4 if c["wide"] else 2) * 2 + 2 + 2 + (2 if c["gate"] == "element" else 0)
        return {"bytes": c["rows"] * c["cols"] * per + 2 * c["cols"], "flops": 12 * c["rows"] * c["cols"]}
    row = c.get("kv_heads", 0) * (c["dim"] + 4 if c["int8"] else 2 * c["dim"]) if "kv_heads" in c else 0   # bytes of one token's keys
    if kind == "attention":
        mean = (c["lo"] + c["hi"]) / 2
        if c["window"]:
            lo, hi, w = c["lo"], c["hi"], c["window"]
            mean = sum(min(w, lo + (hi - lo) * i / 64) for i in range(65)) / 65
        tokens = c["seqs"] * mean
        return {"bytes": 2 * row * tokens + c["seqs"] * c["q_heads"] * (4 * c["dim"] + 4), "flops": 4 * tokens * c["q_heads"] * c["dim"]}
    if kind == "append":
        turned = 4 * c["q_heads"] * c["dim"] if c["rot"] else 0
        return {"bytes": c["tokens"] * (turned + 2 * row + 4 * c["kv_heads"] * c["dim"] + 4 * c["rot"]),
                "flops": 3 * c["tokens"] * (c["q_heads"] + c["kv_heads"]) * c["rot"]}
    if kind == "fork":
        n = c["parents"] * c["children"]
        half = c["page"] / 2
        return {"bytes": n * half * c["layers"] * row * 4 + 4 * c["pages"] + 8 * n * (c["length"] // c["page"]), "flops": 0}
    if kind == "compact":
        moved = c["live"] * (1 - c["live"]) * c["pages"]
        return {"bytes": moved * c["page"] * c["layers"] * row * 4 + 4 * c["pages"] + 8 * c["live"] * c["pages"], "flops": 0}
    cells = c["leave"] * c["length"] // c["page"]
    return {"bytes": 4 * c["pages"] + 16 * cells + 12 * c["seqs"], "flops": 0}


# ---- the same in 64 bits, from the definitions --------------------------------------------------------------

def _rows64(s, pool, scale, i, count):
    """The first `count` keys or values of sequence i, [heads][count][dim] in 64 bits."""
    page = s.c["page"]
    at = torch.arange(count, device=DEV)
    where, slot = s.table[i][at // page].long(), at % page
    x = pool[where, :, slot].double()
    if scale is not None:
        x = x * scale[where, :, slot].double()[..., None]
    return x.transpose(0, 1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "attention":
        hq, hk, d = c["q_heads"], c["kv_heads"], c["dim"]
        out = torch.zeros(c["seqs"], hq, d, dtype=torch.float64, device=DEV)
        lse = torch.full((c["seqs"], hq), -math.inf, dtype=torch.float64, device=DEV)
        for i, n in enumerate(s.len.tolist()):
            first = max(0, n - c["window"]) if c["window"] else 0
            if n == first:
                continue
            q = s.q[i, :hq * d].double().view(hk, hq // hk, d)
            k, v = (_rows64(s, p, z, i, n)[:, first:] for p, z in ((s.k, s.ks), (s.v, s.vs)))
            score = (q @ k.transpose(1, 2)) * s.scale
            lse[i] = torch.logsumexp(score, -1).reshape(-1)
            out[i] = (torch.softmax(score, -1) @ v).reshape(hq, d)
        return out, lse
    if c["kind"] == "append":
        hq, hk, d, page, rot = c["q_heads"], c["kv_heads"], c["dim"], c["page"], c["rot"]
        x = s.qkv.double().view(c["tokens"], hq + 2 * hk, d)
        starts, lens = s.starts.tolist(), s.len.tolist()
        pos = torch.cat([torch.arange(lens[i] - (starts[i + 1] - starts[i]), lens[i], device=DEV) for i in range(c["seqs"])])
        seq = torch.cat([torch.full((starts[i + 1] - starts[i],), i, device=DEV) for i in range(c["seqs"])])
        if rot:
            turn = torch.view_as_complex(s.rope.double())[pos][:, None]
            part = x[:, :hq + hk, :rot]
            z = torch.view_as_complex(part.reshape(*part.shape[:2], rot // 2, 2)) if c["interleaved"] else torch.complex(part[..., :rot // 2], part[..., rot // 2:])
            z = z * turn
            done = torch.view_as_real(z).reshape(part.shape) if c["interleaved"] else torch.cat([z.real, z.imag], -1)
            x = torch.cat([torch.cat([done, x[:, :hq + hk, rot:]], -1), x[:, hq + hk:]], 1)
        k, v = (p.double() if z is None else p.double() * z.double()[..., None] for p, z in ((s.k, s.ks), (s.v, s.vs)))
        where, slot = s.table[seq, pos // page].long(), pos % page
        for pool, new in ((k, x[:, hq:hq + hk]), (v, x[:, hq + hk:])):
            if c["int8"]:
                step = new.abs().amax(-1, keepdim=True) / 127
                new = torch.where(step > 0, (new / step).round() * step, torch.zeros_like(new))
            pool[where, :, slot] = new
        return k, v, x[:, :hq].reshape(c["tokens"], hq * d)
    if c["kind"] == "norm":
        def unit(x, w, b):
            if c["layer"]:
                x = x - x.mean(1, keepdim=True)
            x = x / (x.square().mean(1, keepdim=True) + EPS).sqrt() * w.double()
            return x if b is None else x + b.double()
        u = s.y.double()
        u = unit(u, s.post_w, s.post_b) if c["post"] else u
        u = u if s.gate is None else u * s.gate.double()
        x = s.x.double() + c["scale"] * u
        return x, unit(x, s.pre_w, s.pre_b)
    return None   # whole numbers, and values that are copied
