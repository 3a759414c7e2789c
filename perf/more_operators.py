"""Beam search over the paged cache as cases that can be timed and compared: the choice of the beams that go on, and the pages that
they share, own, copy and give back without the host.

Head layouts are those of the repository's workloads (`synth.CONFIGS`) and a few generic ones; vocabularies are theirs (2048 and
32000) or generic, odd ones among them.  Values follow the repository's recipe for synthetic inputs: logits N(0, (0.02 sqrt(d))^2)
times a scale of the row that is log-uniform in 0.5 .. 8, cached keys and values N(0, (0.02 sqrt(d))^2).

A case is one call, or the calls that a step makes one after the other:
  select   beams.select: of each request's beams, the `keep` best continuations over beams and vocabulary
  beams    what follows a choice, for requests whose beams share the pages of their prompt: Pages.fork in place (each row becomes a
           child of the row that was chosen, its tokens and its hidden state go with it, and it is cut to the length that all of
           them have), then Pages.grow by one position (a page that others hold too is copied before it is written)
  arrive   new requests on cached prefixes: Pages.fork from a store's table (the rows give back what they held before), then
           Pages.grow by the rest of the prompts
  copy     copy_pages: whole pages of one pool into another one
  compact  requests take pages, others end, and what is left moves to the low pages: Pages.grow, Pages.fork, Pages.compact; every
           other pass serves the other half of the requests

A page is allotted in the order of (row, place in the row), the lowest free one first.  A row that writes into a page which other rows
hold gets a copy of it; where every row that holds it writes in the same call, the first of them keeps it.  Copied are the groups
of 32 positions that hold any.

The pool is [layer][page][kv head][block]; a block of fp32 is K[page_size][hd], then V[page_size][hd]; a block of bf16 is groups of
32 positions, 64 * hd values each.
"""
import math
import random

import numpy as np
import torch

own = False

STD = 0.02

# key/value heads, head width, type; d: width of the model
FAMILIES = {
    "7b": dict(dtype="bf16", d=4096, hkv=32, hd=128),
    "70b": dict(dtype="bf16", d=8192, hkv=8, hd=128),
    "narrow": dict(dtype="bf16", d=1024, hkv=5, hd=64),
    "one_kv": dict(dtype="bf16", d=2048, hkv=1, hd=96),
    "fp32": dict(dtype="f32", d=256, hkv=4, hd=64),
    "fp32_grouped": dict(dtype="f32", d=512, hkv=2, hd=84),
}
HISTORY = 128                                               # tokens of a row that go with it


def _select(dtype, d, groups, beams, vocab, keep, done=False):
    return dict(kind="select", dtype=dtype, d=d, groups=groups, beams=beams, vocab=vocab, keep=keep, done=done)


def _beams(family, layers, page, groups, beams, ctx_lo, ctx_hi):
    return dict(FAMILIES[family], kind="beams", layers=layers, page=page, groups=groups, beams=beams, ctx_lo=ctx_lo, ctx_hi=ctx_hi)


def _arrive(family, layers, page, rows, stored, ctx_lo, ctx_hi, q_lo, q_hi):
    return dict(FAMILIES[family], kind="arrive", layers=layers, page=page, rows=rows, stored=stored, ctx_lo=ctx_lo, ctx_hi=ctx_hi, q_lo=q_lo,
                q_hi=q_hi)


def _copy(family, layers, page, n):
    return dict(FAMILIES[family], kind="copy", layers=layers, page=page, n=n)


def _compact(family, layers, page, rows, ctx_lo, ctx_hi):
    return dict(FAMILIES[family], kind="compact", layers=layers, page=page, rows=rows, ctx_lo=ctx_lo, ctx_hi=ctx_hi)


def listed():
    cases = {
        # the fp32 workload's vocabulary, two requests of four beams: launches and latency
        "select_fp32_b8": _select("f32", 256, 2, 4, 2048, 4),
        # one request of five beams, twice as many candidates as beams, as a search that puts ended ones aside asks for
        "select_one_request": _select("f32", 4096, 1, 5, 32000, 10),
        # a batch of 64 requests of four beams on logits of 16 bits, some of the beams at their end
        "select_batch_bf16": _select("bf16", 8192, 64, 4, 32000, 4, done=True),
        # many wide searches over a large vocabulary of odd size
        "select_wide": _select("f32", 4096, 32, 16, 131071, 32),
        # the fp32 workload: two requests of four beams over 64 positions
        "beams_fp32_b8": _beams("fp32", 4, 32, 2, 4, 64, 64),
        # a step of 64 requests of four beams, eight layers of the largest shape
        "beams_70b_b256": _beams("70b", 8, 64, 64, 4, 512, 1024),
        # requests whose system prompts are cached, taken to the end of their own prompts
        "arrive_70b_b57": _arrive("70b", 4, 64, 57, 5, 300, 1500, 40, 450),
        # questions about one long document
        "arrive_7b_document": _arrive("7b", 1, 64, 16, 1, 30000, 30000, 100, 300),
        # one page of the fp32 workload to another pool
        "copy_fp32_1": _copy("fp32", 4, 32, 1),
        # a pool's pages in use to another pool
        "copy_7b_173": _copy("7b", 4, 64, 173),
        # a handful of short requests
        "compact_fp32_b8": _compact("fp32", 4, 32, 8, 20, 100),
        # a large batch, a third of whose requests end
        "compact_70b_b96": _compact("70b", 8, 64, 96, 300, 1500),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _spread(rng, lo, hi):
    """whole number from lo .. hi, even over its logarithm"""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("select", "select", "beams", "arrive", "copy", "compact"))
    if kind == "select":
        vocab, beams = _spread(rng, 256, 131071), _spread(rng, 1, 32)
        groups = _spread(rng, 1, max(1, min(64, (1 << 25) // (vocab * beams))))
        keep = rng.choice((beams, beams, 2 * beams, _spread(rng, 1, 2 * beams)))
        return _select(rng.choice(("f32", "bf16")), rng.choice((256, 1024, 4096, 8192)), groups, beams, vocab, keep, done=rng.random() < 0.4)
    family = rng.choice(tuple(FAMILIES))
    f = FAMILIES[family]
    layers, page = rng.randint(1, 6), rng.choice((32, 64, 64, 96, 128))
    per_page = layers * page * 2 * f["hkv"] * f["hd"] * (2 if f["dtype"] == "bf16" else 4)
    most = max(4, min(4000, (1 << 30) // per_page))         # pages in use at a time
    if kind == "copy":
        return _copy(family, layers, page, _spread(rng, 1, max(1, most // 2)))
    hi = _spread(rng, 8, max(16, min(8000, most * page // 8)))
    lo = rng.randint(1, hi)
    rows = max(1, min(256, most // (hi // page + 4)))
    if kind == "beams":
        beams = _spread(rng, 1, min(12, rows))
        return _beams(family, layers, page, _spread(rng, 1, max(1, rows // beams)), beams, lo, hi)
    if kind == "arrive":
        q_hi = _spread(rng, 1, max(1, min(2000, hi)))
        return _arrive(family, layers, page, _spread(rng, 1, max(1, rows // 2)), rng.randint(1, 3), lo, hi, rng.randint(1, q_hi), q_hi)
    return _compact(family, layers, page, _spread(rng, 3, max(3, rows)), lo, hi)


# ------------------------------------------------------------------ what the inputs are
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed((seed * 7919 + what * 104729) % (1 << 62))


def _int32(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def _logits(case, seed):
    """logits [groups * beams][vocab], running scores, rows at their end (0 or 1)"""
    rows = case["groups"] * case["beams"]
    scale = torch.exp(torch.empty(rows, 1, device="cuda").uniform_(math.log(0.5), math.log(8.0), generator=_gen(seed, 1)))
    z = torch.empty(rows, case["vocab"], device="cuda").normal_(0.0, STD * math.sqrt(case["d"]), generator=_gen(seed, 2)).mul_(scale)
    score = torch.empty(rows, device="cuda").normal_(0.0, 2.0, generator=_gen(seed, 3)).abs_().mul_(-1.0)
    done = (torch.empty(rows, device="cuda").uniform_(generator=_gen(seed, 4)) < 0.15) if case["done"] else None
    return z.to(_type(case)), score, None if done is None else done.to(torch.uint8)


def _block(case):
    return 2 * case["page"] * case["hd"]


def _pool_values(case, seed, what, n_pages):
    n = case["layers"] * n_pages * case["hkv"] * _block(case)
    return torch.empty(n, dtype=_type(case), device="cuda").normal_(0.0, STD * math.sqrt(case["d"]), generator=_gen(seed, what))


def _states(case, seed, rows):
    """tokens and hidden states that go with a row"""
    tokens = torch.randint(0, 32000, (rows, HISTORY), dtype=torch.int32, device="cuda", generator=_gen(seed, 6))
    return [tokens, torch.empty(rows, case["d"], device="cuda").normal_(generator=_gen(seed, 7))]


def _pages_of(n, page):
    return (n + page - 1) // page


def _plan(case):
    """what belongs to a case whatever the seed, so that its pool has one size: rows, width of the table, pages of the pool, lengths,
    and the rows that go on"""
    r, page = random.Random(17), case["page"]
    if case["kind"] == "beams":
        g, b = case["groups"], case["beams"]
        length = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(g)]
        prompt = [max(1, n - r.randint(0, 2 * page)) for n in length]
        need = sum(_pages_of(p, page) + b * (_pages_of(n + 1, page) - p // page + 1) for n, p in zip(length, prompt))
        parent = [r.randrange(b) for _ in range(g * b)]
        return dict(rows=g * b, width=_pages_of(max(length) + 1, page), n_pages=need + 3, length=length, prompt=prompt, parent=parent)
    if case["kind"] == "arrive":
        stored = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["stored"])]
        parent = [r.randrange(case["stored"]) for _ in range(case["rows"])]
        keep = [r.randint((stored[p] + 1) // 2, stored[p]) for p in parent]
        new = [r.randint(case["q_lo"], case["q_hi"]) for _ in parent]
        need = sum(_pages_of(s, page) for s in stored) + sum(_pages_of(n, page) + 1 for n in new)
        width = _pages_of(max(max(stored), max(k + n for k, n in zip(keep, new))), page)
        return dict(rows=case["rows"], width=width, n_pages=need + 3, stored=stored, parent=parent, keep=keep, new=new)
    length = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["rows"])]
    return dict(rows=case["rows"], width=_pages_of(max(length), page), n_pages=sum(_pages_of(n, page) for n in length) + 3, length=length)


def _copied_pages(case):
    """the pages of a copy: which, whereto, and how many each pool has"""
    n = case["n"]
    a, b = list(range(n + n // 3 + 1)), list(range(n + n // 5 + 2))
    random.Random(29).shuffle(a)
    random.Random(31).shuffle(b)
    return a[:n], b[:n], len(a), len(b)


class _PlainPages:
    """who holds which page, in torch operations: tables [rows][width] of page numbers (-1: none), refs [pages]"""

    def __init__(self, case, n_pages, pool):
        self.case, self.page, self.n = case, case["page"], n_pages
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.pool = pool.view(case["layers"], n_pages, -1)

    def table(self, rows, width):
        return dict(pages=torch.full((rows, width), -1, dtype=torch.int32, device="cuda"), kv_len=torch.zeros(rows, dtype=torch.int32, device="cuda"))

    def _count(self, entries, sign):
        held = entries[entries >= 0].long()
        self.refs.index_add_(0, held, torch.full_like(held, sign, dtype=torch.int32))

    def fork(self, table, parent, source=None, keep=None, group=0, rows=()):
        source = source or table
        n, width = table["pages"].shape
        base = torch.arange(n, device="cuda") // group * group if group else 0
        none, at = parent < 0, base + parent.clamp(min=0).long()
        pages, length = source["pages"][at], source["kv_len"][at]
        if keep is not None:
            length = torch.minimum(length, keep)
            pages = torch.where(torch.arange(width, device="cuda") < ((keep + self.page - 1) // self.page)[:, None], pages, -1)
        pages, length = torch.where(none[:, None], -1, pages), torch.where(none, 0, length)
        self._count(pages, 1)
        self._count(table["pages"], -1)
        table["pages"].copy_(pages)
        table["kv_len"].copy_(length)
        for x in rows:
            x.copy_(torch.where(none[:, None], x, x[at]))

    def grow(self, table, new=None):
        pages, length, page = table["pages"], table["kv_len"], self.page
        n, width = pages.shape
        new = torch.ones_like(length) if new is None else new
        part, last = length % page, (length // page).clamp(max=width - 1).long()
        held = pages.gather(1, last[:, None])[:, 0].long().clamp(min=0)
        shared = (new > 0) & (part > 0) & (self.refs[held] > 1)
        same = (held[:, None] == held) & shared & shared[:, None]
        earlier = (same & torch.ones(n, n, dtype=torch.bool, device="cuda").tril(-1)).any(1)
        copies = shared & (earlier | (self.refs[held] > same.sum(1)))
        have, want = (length + page - 1) // page, (length + new + page - 1) // page
        need = copies + want - have
        first = need.cumsum(0) - need
        free = torch.nonzero(self.refs == 0)[:, 0]
        src, dst = held[copies], free[first[copies]]
        self._copy_groups(src, dst, (part[copies] + 31) // 32)
        self.refs.index_add_(0, src, torch.full_like(src, -1, dtype=torch.int32))
        pages[copies, last[copies]] = dst.int()
        at = torch.arange(width, device="cuda")[None] - have[:, None]                 # of a new page among the row's new ones
        fresh = (at >= 0) & (at < (want - have)[:, None])
        pages[fresh] = free[((first + copies)[:, None] + at)[fresh]].int()
        self.refs[pages[fresh].long()] = 1
        self.refs[dst] = 1
        length += new

    def _copy_groups(self, src, dst, groups):
        """the first `groups` groups of 32 positions of each page"""
        c = self.case
        g = torch.arange(self.page // 32, device="cuda") < groups[:, None]             # [copies][groups]
        if c["dtype"] == "f32":
            pool, g = self.pool.view(c["layers"], self.n, c["hkv"], 2, self.page // 32, 32 * c["hd"]), g[None, :, None, None, :, None]
        else:
            pool, g = self.pool.view(c["layers"], self.n, c["hkv"], self.page // 32, 64 * c["hd"]), g[None, :, None, :, None]
        pool[:, dst] = torch.where(g, pool[:, src], pool[:, dst])

    def compact(self, table):
        used = self.refs > 0
        n_used = used.sum()
        low = torch.arange(self.n, device="cuda") < n_used
        src, dst = torch.nonzero(used & ~low)[:, 0], torch.nonzero(~used & low)[:, 0]
        self.pool[:, dst] = self.pool[:, src]
        name = torch.arange(self.n, dtype=torch.int32, device="cuda")
        name[src] = dst.int()
        table["pages"].copy_(torch.where(table["pages"] >= 0, name[table["pages"].clamp(min=0).long()], table["pages"]))
        self.refs[dst] = self.refs[src]
        self.refs[src] = 0


def _bookkeeping(case, seed, n_pages):
    """the pool and who holds its pages, and a function that makes a table"""
    if own:
        from paper_2504_10724_amd import paged
        kv = paged.PagedCache(n_layers=case["layers"], n_pages=n_pages, n_kv_heads=case["hkv"], head_dim=case["hd"], page_size=case["page"],
                              dtype=case["dtype"])
        kv.pool.copy_(_pool_values(case, seed, 5, n_pages))
        pages = paged.Pages(kv, max_seqs=4096)
        return kv.pool, pages, lambda rows, width: paged.PageTable(kv, rows, width)
    pool = _pool_values(case, seed, 5, n_pages)
    pages = _PlainPages(case, n_pages, pool)
    return pool, pages, pages.table


def prepare(case, seed):
    state = dict(case=case)
    if case["kind"] == "select":
        z, score, done = _logits(case, seed)
        state.update(logits=z, score=score, done=done, end=case["vocab"] // 2 if case["done"] else -1)
        if own:
            from paper_2504_10724_amd import beams
            state["out"] = beams.selection(case["groups"], case["keep"], done=case["done"])
            state["workspace"] = beams.workspace(case["groups"], case["beams"], case["vocab"], case["keep"])
        return state
    if case["kind"] == "copy":
        src, dst, n_from, n_to = _copied_pages(case)
        state.update(src=_int32(src), dst=_int32(dst))
        if own:
            from paper_2504_10724_amd import paged
            for name, what, n in (("a", 5, n_from), ("b", 8, n_to)):
                state[name] = paged.PagedCache(n_layers=case["layers"], n_pages=n, n_kv_heads=case["hkv"], head_dim=case["hd"],
                                               page_size=case["page"], dtype=case["dtype"])
                state[name].pool.copy_(_pool_values(case, seed, what, n))
        else:
            state.update(a=_pool_values(case, seed, 5, n_from).view(case["layers"], n_from, -1),
                         b=_pool_values(case, seed, 8, n_to).view(case["layers"], n_to, -1))
        return state
    p = _plan(case)
    state["pool"], pages, make = _bookkeeping(case, seed, p["n_pages"])
    state.update(pages=pages, table=make(p["rows"], p["width"]))
    rows = np.arange(p["rows"])
    if case["kind"] == "beams":
        b = case["beams"]
        length, prompt = np.repeat(p["length"], b), np.repeat(p["prompt"], b)
        pages.grow(state["table"], _int32(np.where(rows % b == 0, prompt, 0)))
        pages.fork(state["table"], _int32(rows * 0), group=b)
        pages.grow(state["table"], _int32(length - prompt))
        state.update(parent=_int32(p["parent"]), keep=_int32(length), rows=_states(case, seed, p["rows"]))
    elif case["kind"] == "arrive":
        state["store"] = make(case["stored"], p["width"])
        pages.grow(state["store"], _int32(p["stored"]))
        state.update(parent=_int32(p["parent"]), keep=_int32(p["keep"]), new=_int32(p["new"]))
    else:
        # rows 0, 3, 6, .. stay; of the others every second one is there
        length = np.asarray(p["length"])
        there = [rows % 3 == 0, rows % 3 == 1, rows % 3 == 2]
        pages.grow(state["table"], _int32(np.where(there[0] | there[2], length, 0)))
        state["turn"] = 0
        state["new"] = [_int32(np.where(there[1 + k], length, 0)) for k in (0, 1)]
        state["left"] = [_int32(np.where(there[2 - k], -1, rows)) for k in (0, 1)]
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if case["kind"] == "select":
        return _run_select(state)
    if case["kind"] == "copy":
        if own:
            from paper_2504_10724_amd import paged
            paged.copy_pages(state["a"], state["b"], state["src"], state["dst"])
            return state["b"].pool
        state["b"][:, state["dst"].long()] = state["a"][:, state["src"].long()]
        return state["b"].view(-1)
    pages, table = state["pages"], state["table"]
    more = {}
    if case["kind"] == "beams":
        pages.fork(table, state["parent"], keep=state["keep"], group=case["beams"], rows=state["rows"])
        pages.grow(table)
        more = dict(tokens=state["rows"][0], hidden=state["rows"][1])
    elif case["kind"] == "arrive":
        pages.fork(table, state["parent"], source=state["store"], keep=state["keep"])
        pages.grow(table, state["new"])
    else:
        k = state["turn"]
        state["turn"] = 1 - k
        pages.grow(table, state["new"][k])
        pages.fork(table, state["left"][k])
        pages.compact(table)
    if own:
        return dict(more, pages=table.pages, kv_len=table.kv_len, refs=pages.refs, pool=state["pool"])
    return dict(more, pages=table["pages"], kv_len=table["kv_len"], refs=pages.refs, pool=state["pool"])


def _run_select(state):
    case = state["case"]
    if own:
        from paper_2504_10724_amd import beams
        got = beams.select(state["logits"], state["score"], case["beams"], keep=case["keep"], done=state["done"], end_token=state["end"],
                           out=state["out"], workspace=state["workspace"])
        return dict(score=got.score, parent=got.parent, token=got.token, **({} if got.done is None else dict(done=got.done)))
    # in 64 bits: which of two beams' candidates is the better one is often a matter of the last places
    z, score, vocab = state["logits"].double(), state["score"].double()[:, None], case["vocab"]
    top = z.amax(1, keepdim=True)
    key = score + (z - top) - torch.log(torch.exp(z - top).sum(1, keepdim=True))
    if case["done"]:
        key = torch.where(state["done"].bool()[:, None], torch.where(torch.arange(vocab, device="cuda") == state["end"], score, -math.inf), key)
    key, at = torch.sort(key.view(case["groups"], -1), dim=1, descending=True, stable=True)
    short = case["keep"] - key.shape[1]
    key, at = key[:, :case["keep"]], at[:, :case["keep"]]
    if short > 0:                                           # fewer candidates than are asked for
        key, at = torch.nn.functional.pad(key, (0, short), value=-math.inf), torch.nn.functional.pad(at, (0, short))
    found = key > -math.inf
    out = dict(score=key.float(), parent=torch.where(found, at // vocab, -1).int(), token=torch.where(found, at % vocab, -1).int())
    if case["done"]:
        before = state["done"].view(case["groups"], -1).gather(1, out["parent"].clamp(min=0).long())
        out["done"] = torch.where(found, before | (out["token"] == state["end"]), 0).to(torch.uint8)
    return out


# ------------------------------------------------------------------ what a pass cannot do without
class _Book:
    """who holds which page, one row and one page after the other (lists); what is copied is kept in `moved`"""

    def __init__(self, page, n_pages):
        self.page, self.refs, self.moved, self.taken = page, [0] * n_pages, [], 0

    def _take(self):
        p = self.refs.index(0, self.low)
        self.refs[p], self.low, self.taken = 1, p + 1, self.taken + 1
        return p

    def grow(self, rows, new):
        """rows: [pages, length] of each"""
        writers = {}
        for i, (pages, length) in enumerate(rows):
            if new[i] and length % self.page:
                writers.setdefault(pages[length // self.page], []).append(i)
        held = list(self.refs)
        self.low = 0
        for i, (pages, length) in enumerate(rows):
            if not new[i]:
                continue
            at, part = divmod(length, self.page)
            if part:
                old, w = pages[at], writers[pages[at]]
                if held[old] > 1 and (held[old] > len(w) or i != w[0]):
                    pages[at] = self._take()
                    self.moved.append((old, pages[at], _pages_of(part, 32)))
            while len(pages) * self.page < length + new[i]:
                pages.append(self._take())
            rows[i][1] = length + new[i]
        for old, _, _ in self.moved:
            self.refs[old] -= 1

    def fork(self, rows, parents, keep):
        """rows become copies of the rows `parents`, [pages, length] or None each, cut to `keep`"""
        made = [[[], 0] if p is None else [list(p[0][:_pages_of(min(k, p[1]), self.page)]), min(k, p[1])] for p, k in zip(parents, keep)]
        for pages, _ in made:
            for p in pages:
                self.refs[p] += 1
        for pages, _ in rows:
            for p in pages:
                self.refs[p] -= 1
        rows[:] = made

    def compact(self, rows):
        n = sum(r > 0 for r in self.refs)
        high = [p for p in range(n, len(self.refs)) if self.refs[p]]
        name = dict(zip(high, (p for p in range(n) if not self.refs[p])))
        for old, p in name.items():
            self.refs[p], self.refs[old] = self.refs[old], 0
            self.moved.append((old, p, self.page // 32))
        for r in rows:
            r[0] = [name.get(p, p) for p in r[0]]


def _book_pass(case, passes=1):
    """the case's preparation and passes on a _Book, the book with what the last pass copied, and what the rows hold"""
    p = _plan(case)
    book = _Book(case["page"], p["n_pages"])
    rows = [[[], 0] for _ in range(p["rows"])]
    moved = []

    def step(f, *a):
        book.moved, book.taken = [], 0
        f(*a)
        moved.extend(book.moved)
    if case["kind"] == "beams":
        b, n = case["beams"], p["rows"]
        step(book.grow, rows, [p["prompt"][i // b] if i % b == 0 else 0 for i in range(n)])
        step(book.fork, rows, [rows[i // b * b] for i in range(n)], [1 << 30] * n)
        step(book.grow, rows, [p["length"][i // b] - p["prompt"][i // b] for i in range(n)])
    elif case["kind"] == "arrive":
        store = [[[], 0] for _ in p["stored"]]
        step(book.grow, store, p["stored"])
    else:
        step(book.grow, rows, [n if i % 3 != 1 else 0 for i, n in enumerate(p["length"])])
    before = len(moved)
    for k in range(passes):
        before = len(moved)
        if case["kind"] == "beams":
            step(book.fork, rows, [rows[i // b * b + p["parent"][i]] for i in range(n)], [p["length"][i // b] for i in range(n)])
            step(book.grow, rows, [1] * n)
        elif case["kind"] == "arrive":
            step(book.fork, rows, [store[i] for i in p["parent"]], p["keep"])
            step(book.grow, rows, p["new"])
        else:
            step(book.grow, rows, [n if i % 3 == 1 + k % 2 else 0 for i, n in enumerate(p["length"])])
            step(book.fork, rows, [None if i % 3 == 2 - k % 2 else r for i, r in enumerate(rows)], [1 << 30] * len(rows))
            step(book.compact, rows)
    return book, rows, moved, before


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "select":
        rows = case["groups"] * case["beams"]
        return dict(bytes=float(size * rows * case["vocab"] + 4 * rows + 12 * case["groups"] * case["keep"]), flops=4.0 * rows * case["vocab"])
    group = 64.0 * case["layers"] * case["hkv"] * case["hd"] * size                     # of 32 positions
    if case["kind"] == "copy":
        return dict(bytes=2.0 * case["n"] * case["page"] / 32 * group + 8 * case["n"], flops=0.0)
    book, rows, moved, before = _book_pass(case, 2)
    entries = sum(len(pages) for pages, _ in rows)
    states = 2.0 * len(rows) * (4 * HISTORY + 4 * case["d"]) if case["kind"] == "beams" else 0.0
    return dict(bytes=2.0 * group * sum(g for _, _, g in moved[before:]) + 8.0 * entries + 16.0 * len(rows) + states, flops=0.0)


# ------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    if case["kind"] == "select":
        z, score, done = _logits(case, seed)
        best = []
        for g in range(case["groups"]):
            mine = slice(g * case["beams"], (g + 1) * case["beams"])
            p = torch.log_softmax(z[mine].double(), 1) + score[mine].double()[:, None]
            if done is not None:
                for b in range(case["beams"]):
                    if done[mine][b]:
                        p[b] = -math.inf
                        p[b, case["vocab"] // 2] = score[mine][b].double()
            s = torch.topk(p.flatten(), min(case["keep"], p.numel())).values
            best.append(torch.cat([s, torch.full((case["keep"] - len(s),), -math.inf, dtype=torch.float64, device="cuda")]))
        return dict(score=torch.stack(best), parent=None, token=None, **({} if done is None else dict(done=None)))
    if case["kind"] == "copy":
        src, dst, n_from, n_to = _copied_pages(case)
        a = _pool_values(case, seed, 5, n_from).view(case["layers"], n_from, -1)
        b = _pool_values(case, seed, 8, n_to).view(case["layers"], n_to, -1).double()
        for i, j in zip(src, dst):
            b[:, j] = a[:, i].double()
        return b.view(-1)
    p = _plan(case)
    book, rows, moved, _ = _book_pass(case)
    pool = _pool_values(case, seed, 5, p["n_pages"]).double()
    split = (2, case["page"] // 32) if case["dtype"] == "f32" else (1, case["page"] // 32)
    view = pool.view(case["layers"], p["n_pages"], case["hkv"], *split, -1)
    for old, to, groups in moved:
        view[:, to, :, :, :groups] = view[:, old, :, :, :groups]
    out = dict(pages=None, kv_len=None, refs=None, pool=pool)
    if case["kind"] == "beams":
        hidden = _states(case, seed, p["rows"])[1].double()
        b = case["beams"]
        out.update(tokens=None, hidden=torch.stack([hidden[i // b * b + p["parent"][i]] for i in range(p["rows"])]))
    return out
