"""Plain 64-bit definitions of the cache's operators, on host tensors, and the books' rules in Python integers."""
from __future__ import annotations

import math

import torch


def cache_rows(pool, scale, table_row, head, tokens, page_tokens, n_pages):
    """Keys (or values) of the listed tokens of one head in 64 bits, and which of them lie on a page of the pool."""
    at = torch.tensor(list(tokens), dtype=torch.int64)
    page = table_row[at // page_tokens].long()
    ok = (page >= 0) & (page < n_pages)
    page = torch.where(ok, page, torch.zeros_like(page))
    x = pool[page, head, at % page_tokens].double()
    if scale is not None:
        x = x * scale[page, head, at % page_tokens].double()[:, None]
    return x, ok


def attention(q, k, v, ks, vs, table, lens, page_tokens, scale, window):
    """(out, lse, bound of |v| weighted by the softmax, bound of a score's rounding) per sequence and query head."""
    n, hq, d = q.shape
    n_pages, hk = k.shape[0], k.shape[1]
    out = torch.zeros(n, hq, d, dtype=torch.float64)
    mag = torch.zeros(n, hq, d, dtype=torch.float64)
    ds = torch.zeros(n, hq, dtype=torch.float64)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64)
    for s in range(n):
        length = min(max(int(lens[s]), 0), table.shape[1] * page_tokens)
        first = max(0, length - window) if window else 0
        tokens = range(first, length)
        for h in range(hk):
            kk, ok = cache_rows(k, ks, table[s], h, tokens, page_tokens, n_pages)
            vv, _ = cache_rows(v, vs, table[s], h, tokens, page_tokens, n_pages)
            kk, vv = kk[ok], vv[ok]
            if not len(kk):
                continue
            for i in range(h * (hq // hk), (h + 1) * (hq // hk)):
                sc = kk @ q[s, i].double() * scale
                p = torch.softmax(sc, 0)
                out[s, i], mag[s, i] = p @ vv, p @ vv.abs()
                lse[s, i] = torch.logsumexp(sc, 0)
                ds[s, i] = (kk.abs() @ q[s, i].double().abs()).max() * abs(scale)
    return out, lse, mag, ds


def rotate(x, cs, rot, interleaved):
    """x: [..., dim] in 64 bits, cs: [rot / 2, 2]."""
    y = x.clone()
    cos, sin = cs[:, 0].double(), cs[:, 1].double()
    if rot:
        ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        a, b = x[..., ia], x[..., ib]
        y[..., ia], y[..., ib] = a * cos - b * sin, b * cos + a * sin
    return y


class Books:
    """Table, lengths and reference counts by the rules of the header, one entry after the other."""

    def __init__(self, n_pages, page, n_seqs, stride):
        self.n_pages, self.page, self.stride = n_pages, page, stride
        self.table = [[0] * stride for _ in range(n_seqs)]
        self.len = [0] * n_seqs
        self.refs = [0] * n_pages

    def pages(self, n):
        return -(-n // self.page)

    def free_pages(self):
        return [p for p in range(self.n_pages) if self.refs[p] == 0]

    def reserve(self, grow):
        grow = [max(0, g) for g in grow]
        long = sum(n + g > self.stride * self.page for n, g in zip(self.len, grow))
        if long:
            return 0, long
        need = [self.pages(n + g) - self.pages(n) for n, g in zip(self.len, grow)]
        free = self.free_pages()
        if len(free) < sum(need):
            return sum(need) - len(free), 0
        for s, c in enumerate(need):
            for _ in range(c):
                p = free.pop(0)
                self.table[s][self.pages(self.len[s])] = p
                self.refs[p] = 1
                self.len[s] += self.page   # (whole pages here, the true length below)
            self.len[s] -= c * self.page
            at = self.pages(self.len[s])
            assert at + c <= self.stride
        for s, c in enumerate(need):
            self.len[s] += grow[s]
        return 0, 0

    def fork(self, pairs):
        """Status, and the copies (source page, destination page, tokens)."""
        seen, good = set(), []
        for p, c in pairs:
            ok = 0 <= p < len(self.len) and 0 <= c < len(self.len) and self.len[c] <= 0 and c not in seen
            seen.add(c)
            if ok:
                good.append((p, c))
        free = self.free_pages()
        need = sum(self.len[p] % self.page > 0 for p, _ in good)
        if len(free) < need:
            return (need - len(free), len(pairs) - len(good)), []
        before, copies = list(self.len), []
        for p, c in good:
            full, rest = before[p] // self.page, before[p] % self.page
            for j in range(full):
                self.table[c][j] = self.table[p][j]
                self.refs[self.table[p][j]] += 1
            if rest:
                new = free.pop(0)
                self.table[c][full] = new
                self.refs[new] = 1
                copies.append((self.table[p][full], new, rest))
            self.len[c] = before[p]
        return (0, len(pairs) - len(good)), copies

    def free(self, slots):
        for s in slots:
            if 0 <= s < len(self.len):
                for j in range(self.pages(self.len[s])):
                    self.refs[self.table[s][j]] -= 1
                self.len[s] = 0

    def compact(self):
        used = sum(r != 0 for r in self.refs)
        src = [p for p in range(used, self.n_pages) if self.refs[p]]
        dst = [p for p in range(used) if not self.refs[p]]
        to = dict(zip(src, dst))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        for s, n in enumerate(self.len):
            for j in range(self.pages(n)):
                self.table[s][j] = to.get(self.table[s][j], self.table[s][j])
        return (used, len(src)), [(a, b, self.page) for a, b in to.items()]
