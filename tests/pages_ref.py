"""The pages' bookkeeping and the beam search's choice from their definitions, on the CPU: lists of pages, one row after the other, and
candidates in 64 bits."""
import math

import torch


class Table:
    def __init__(self, n, width):
        self.width, self.rows, self.len = width, [[] for _ in range(n)], [0] * n

    def entries(self):
        return [r + [-1] * (self.width - len(r)) for r in self.rows]


class Book:
    """pool: [layer][page][kv head][K or V .. fp32: 2, bf16: 1][groups of 32 positions][values], any type"""

    def __init__(self, n_pages, page, pool=None):
        self.n, self.page, self.pool, self.status = n_pages, page, pool, 0
        self.tables = []

    def refs(self):
        out = [0] * self.n
        for t in self.tables:
            for r in t.rows:
                for p in r:
                    out[p] += 1
        return out

    def table(self, n, width):
        self.tables.append(Table(n, width))
        return self.tables[-1]

    def grow(self, t, new=None):
        n, ps = len(t.rows), self.page
        new = [1] * n if new is None else list(new)
        for i in range(n):
            if new[i] < 0 or t.len[i] + new[i] > t.width * ps:
                self.status |= 8
                new[i] = 0
        refs = self.refs()
        last = [t.rows[i][t.len[i] // ps] if new[i] and t.len[i] % ps else None for i in range(n)]
        copies = [p is not None and refs[p] > 1 and (refs[p] > last.count(p) or last.index(p) != i) for i, p in enumerate(last)]
        need = sum(copies) + sum(-(-(t.len[i] + new[i]) // ps) - -(-t.len[i] // ps) for i in range(n))
        free = [p for p in range(self.n) if refs[p] == 0]
        if need > len(free):
            self.status |= 4
            return
        for i in range(n):
            if copies[i]:
                p, at = free.pop(0), t.len[i] // ps
                g = (t.len[i] % ps + 31) // 32
                if self.pool is not None:
                    self.pool[:, p, :, :, :g] = self.pool[:, t.rows[i][at], :, :, :g]
                t.rows[i][at] = p
            while len(t.rows[i]) * ps < t.len[i] + new[i]:
                t.rows[i].append(free.pop(0))
            t.len[i] += new[i]

    def fork(self, t, parent, source=None, keep=None, group=0, rows=()):
        source = source or t
        limit = group or len(source.rows)
        old = [(list(r), l) for r, l in zip(source.rows, source.len)]
        before = [x.clone() for x in rows]
        for i, p in enumerate(parent):
            k = 1 << 40 if keep is None else keep[i]
            if p < -1 or p >= limit or k < 0:
                self.status |= 8
                continue
            if p < 0:
                t.rows[i], t.len[i] = [], 0
                continue
            at = p + (i // group * group if group else 0)
            t.len[i] = min(old[at][1], k)
            t.rows[i] = old[at][0][:-(-t.len[i] // self.page)]
            for x, b in zip(rows, before):
                x[i] = b[at]

    def compact(self):
        refs = self.refs()
        used = sum(r > 0 for r in refs)
        name = dict(zip([p for p in range(used, self.n) if refs[p]], [p for p in range(used) if not refs[p]]))
        for t in self.tables:
            t.rows = [[name.get(p, p) for p in r] for r in t.rows]
        if self.pool is not None:
            for old, p in name.items():
                self.pool[:, p] = self.pool[:, old]


def choose(logits, score, n_beams, keep, done=None, end=-1):
    """(score in 64 bits, parent, token, done), lists of lists"""
    out = [], [], [], []
    vocab = logits.shape[1]
    for g in range(len(logits) // n_beams):
        found = []
        for b in range(n_beams):
            row = g * n_beams + b
            s, z = float(score[row]), logits[row].double()
            if not math.isfinite(s):
                continue
            if done is not None and done[row]:
                found.append((-s, b, end, 1))
                continue
            top = float(z.max())
            if torch.isnan(z).any() or not math.isfinite(top):
                continue
            log = math.log(float(torch.exp(z - top).sum()))
            # in a beam the order is that of the logits, equal ones by their place
            for v in torch.sort(z, descending=True, stable=True).indices[:keep].tolist():
                if float(z[v]) > -math.inf:
                    found.append((-(s - log + (float(z[v]) - top)), b, v, int(v == end)))
        found.sort(key=lambda c: (c[0], c[1] * vocab + c[2]))
        found = found[:keep] + [(math.inf, -1, -1, 0)] * max(0, keep - len(found))
        for o, k in zip(out, range(4)):
            o.append([-c[0] if k == 0 else c[k] for c in found])
    return out
