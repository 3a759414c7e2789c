"""The operators of the paged cache as cases that can be timed and compared: rotary positions, appending keys and values
to a paged cache with the rotation on the way, and attention of new tokens over that cache.

Head layouts are those of the repository's workloads (`synth.CONFIGS`) and a few generic ones; row counts, lengths and
page sizes are the ranges such caches are served with.  Values follow the repository's recipe for synthetic inputs: what
leaves a projection, and what is cached, is N(0, (0.02 sqrt(d))^2); page numbers are a random order, as a pool that has been
in use for a while hands them out.

A case is one call:
  rope     ee_rope_apply on the query and key heads of n projected rows (`back`: the inverse rotation, a gradient's)
  append   ee_paged_append of a batch's new tokens: queries rotated, keys rotated into their pages, values into theirs
  attend   ee_paged_attention of a batch's new tokens
A batch is `chunks` sequences that bring q_lo .. q_hi tokens each and `singles` sequences that bring one, all over
ctx_lo .. ctx_hi positions that are cached already.

The pool is [layer][page][kv head][block]; a block of fp32 is K[page_size][hd], then V[page_size][hd]; a block of bf16 is
groups of 32 positions, each the keys [2][hd / 32][4][16 positions][8 features] and then the values
[hd / 16][4 quads][16 features][2][4 positions].
"""
import math
import random

import numpy as np
import torch

own = False

STD = 0.02

# query heads, key/value heads, head width and type; d: width of the model (sets the values' spread)
FAMILIES = {
    "7b": dict(dtype="bf16", d=4096, hq=32, hkv=32, hd=128),
    "34b": dict(dtype="bf16", d=8192, hq=64, hkv=8, hd=128),
    "70b": dict(dtype="bf16", d=8192, hq=64, hkv=8, hd=128),
    "small": dict(dtype="bf16", d=2048, hq=16, hkv=4, hd=128),
    "off_grid": dict(dtype="bf16", d=576, hq=4, hkv=2, hd=128),
    "narrow": dict(dtype="bf16", d=1024, hq=15, hkv=5, hd=64),
    "one_kv": dict(dtype="bf16", d=2048, hq=20, hkv=1, hd=96),
    "wide": dict(dtype="bf16", d=4096, hq=16, hkv=2, hd=256),
    "fp32": dict(dtype="f32", d=256, hq=4, hkv=4, hd=64),
    "fp32_grouped": dict(dtype="f32", d=512, hq=6, hkv=2, hd=84),
}

PLAIN = dict(pairing="half", rot=0, scaling="none", factor=1.0)       # rot 0: the whole head


def _case(family, kind, **more):
    return dict(FAMILIES[family], kind=kind, **more)


def _rope(family, n, max_pos, back=False, **more):
    return _case(family, "rope", n=n, max_pos=max_pos, back=back, **dict(PLAIN, **more))


def _append(family, chunks, q_lo, q_hi, singles, ctx_lo, ctx_hi, page, **more):
    return _case(family, "append", chunks=chunks, q_lo=q_lo, q_hi=q_hi, singles=singles, ctx_lo=ctx_lo, ctx_hi=ctx_hi, page=page,
                 **dict(PLAIN, **more))


def _attend(family, chunks, q_lo, q_hi, singles, ctx_lo, ctx_hi, page, window=0):
    return _case(family, "attend", chunks=chunks, q_lo=q_lo, q_hi=q_hi, singles=singles, ctx_lo=ctx_lo, ctx_hi=ctx_hi, page=page,
                 window=window)


def listed():
    cases = {
        # the fp32 workload as it stands: one token for each of 8 rows (launches and latency)
        "rope_fp32_b8": _rope("fp32", 8, 128),
        # a long document's chunk, an odd number of tokens, on a model that rotates neighbours in half of the head and whose
        # frequencies are scaled for long contexts
        "rope_34b_4097_long": _rope("34b", 4097, 131072, pairing="interleaved", rot=64, scaling="bands", factor=8.0),
        # the gradient of the same for an ordinary training batch's rows, whole heads, a scaled base
        "rope_70b_1999_back": _rope("70b", 1999, 16384, back=True, scaling="base", factor=4.0),
        # the paper's default, one request, its next token
        "append_7b_b1": _append("7b", 0, 0, 0, 1, 512, 1024, 64),
        # the next token of a large batch on the largest shape
        "append_70b_b256": _append("70b", 0, 0, 0, 256, 128, 1024, 64),
        # prompts taken in chunks beside requests that decode
        "append_34b_mixed": _append("34b", 7, 100, 450, 57, 0, 2048, 128),
        # the fp32 workload: 8 rows over 64 positions
        "attend_fp32_b8": _attend("fp32", 0, 0, 0, 8, 64, 64, 32),
        # one request with a long context: few rows, one long axis
        "attend_7b_b1_long": _attend("7b", 0, 0, 0, 1, 32767, 32767, 64),
        # a decode step of the largest batch: 512 to 2048 cached positions a row
        "attend_70b_b256": _attend("70b", 0, 0, 0, 256, 512, 2048, 64),
        # two chunks of prompts beside 62 requests that decode
        "attend_34b_mixed": _attend("34b", 2, 300, 700, 62, 256, 2048, 128),
        # prompts from their first token: four of about 2000
        "attend_70b_prompts": _attend("70b", 4, 1900, 2048, 0, 0, 0, 64),
        # a chunk late in a long document
        "attend_7b_late_chunk": _attend("7b", 1, 1023, 1023, 0, 30000, 30000, 64),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _spread(rng, lo, hi):
    """whole number from lo .. hi, even over its logarithm"""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("rope", "append", "attend", "attend", "attend"))
    family = rng.choice(tuple(FAMILIES))
    f = FAMILIES[family]
    small = f["dtype"] == "f32"
    rot = rng.choice((0, 0, f["hd"] // 2, f["hd"] // 4 * 2))
    turn = dict(pairing=rng.choice(("half", "interleaved")), rot=rot, scaling=rng.choice(("none", "none", "linear", "base", "bands")))
    turn["factor"] = 1.0 if turn["scaling"] == "none" else round(rng.uniform(1.5, 16.0), 2)
    if kind == "rope":
        return _rope(family, _spread(rng, 1, 4097), _spread(rng, 4097, 131072), back=rng.random() < 0.4, **turn)
    page = rng.choice((32, 64, 64, 96, 128, 256))
    form = rng.choice(("singles", "singles", "chunks", "mixed"))
    budget = 1 << (18 if small else 21)                # cached positions x key/value heads of the batch
    hi = _spread(rng, 16, 4096 if small else 32768)
    lo = rng.randint(1, hi)
    most = max(1, min(256, budget // (hi * f["hkv"])))
    singles = 0 if form == "chunks" else _spread(rng, 1, most)
    chunks = 0 if form == "singles" else rng.randint(1, min(4, most))
    q_hi = _spread(rng, 2, 512 if small else 1500) if chunks else 0
    if kind == "attend":
        # (new token, position) pairs x query heads: no more than about half of the largest listed case's
        while chunks and chunks * q_hi * (hi + q_hi) * f["hq"] > 5e8:
            q_hi = max(2, q_hi // 2)
            hi, lo = max(16, hi // 2), max(1, lo // 2)
    q_lo = rng.randint(1, q_hi) if chunks else 0
    lo = min(lo, hi)
    if kind == "append":
        return _append(family, chunks, q_lo, q_hi, singles, min(lo, 2048), min(hi, 2048), page, **turn)
    return _attend(family, chunks, q_lo, q_hi, singles, 0 if rng.random() < 0.15 else lo, hi, page,
                   window=_spread(rng, 1, hi) if rng.random() < 0.25 else 0)


# ------------------------------------------------------------------ what the inputs are
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed((seed * 7919 + what * 104729) % (1 << 62))


def _values(case, seed, what, shape):
    return torch.empty(shape, dtype=_type(case), device="cuda").normal_(0.0, STD * math.sqrt(case["d"]), generator=_gen(seed, what))


def _int32(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def _sequences(case):
    """(new tokens, positions in the cache with them) of each sequence: a mix that belongs to the case, so that its cache
    has one size"""
    r = random.Random(17)
    new = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["chunks"])] + [1] * case["singles"]
    r.shuffle(new)
    return [(n, n + r.randint(case["ctx_lo"], case["ctx_hi"])) for n in new]


def _pages(case):
    """pages of the pool, and the page numbers of each sequence, one row of a rectangular table each"""
    need = [(length + case["page"] - 1) // case["page"] for _, length in _sequences(case)]
    total = sum(need) + 3
    order = list(range(total))
    random.Random(29).shuffle(order)
    table, at = np.full((len(need), max(need)), -1, np.int32), 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return total, table


def _rot(case):
    return case["rot"] or case["hd"]


def _frequencies(case):
    """of each pair, in 64 bits (numpy)"""
    r, s, theta = _rot(case), case["factor"], 10000.0
    j = np.arange(r // 2, dtype=np.float64)
    if case["scaling"] == "base":
        theta *= s ** (r / (r - 2.0))
    f = theta ** (-2.0 * j / r)
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "bands":
        w = np.clip((4096.0 * f / (2.0 * math.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = f * (w + (1.0 - w) / s)
    return f


def _max_pos(case):
    return case["max_pos"] if case["kind"] == "rope" else max(length for _, length in _sequences(case))


def _rope_positions(case, seed):
    return torch.randint(0, case["max_pos"], (case["n"],), dtype=torch.int32, device="cuda", generator=_gen(seed, 2))


def _rows(case, seed):
    """projected rows [n][query heads, key heads, value heads][hd]"""
    n = case["n"] if case["kind"] == "rope" else sum(q for q, _ in _sequences(case))
    return _values(case, seed, 1, (n, case["hq"] + 2 * case["hkv"], case["hd"]))


def _pool_shape(case):
    return (_pages(case)[0] * case["hkv"] * 2 * case["page"] * case["hd"],)


def prepare(case, seed):
    state = dict(case=case)
    rows = _rows(case, seed) if case["kind"] != "attend" else None
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    if own:
        from paper_2504_10724_amd import paged
    if case["kind"] != "attend":
        if own:
            state["rope"] = paged.Rope(hd, _max_pos(case), rot_dim=_rot(case), pairing=case["pairing"], theta=10000.0,
                                       scaling=case["scaling"], factor=case["factor"], trained_pos=4096, low=1.0, high=4.0)
        else:
            a = torch.arange(_max_pos(case), dtype=torch.float64, device="cuda")[:, None] * torch.tensor(_frequencies(case), device="cuda")
            state["cos"], state["sin"] = torch.cos(a).float(), torch.sin(a).float()
    if case["kind"] == "rope":
        x = rows[:, :hq + hkv]
        return dict(state, x=x, pos=_rope_positions(case, seed), y=torch.empty(x.shape, dtype=x.dtype, device="cuda"))
    seqs, (n_pages, table) = _sequences(case), _pages(case)
    start = np.concatenate([[0], np.cumsum([q for q, _ in seqs])])
    n, lengths = int(start[-1]), [length for _, length in seqs]
    tables = dict(q_start=_int32(start), kv_len=_int32(lengths), pages=_int32(table))
    if own:
        kv = paged.PagedCache(n_layers=1, n_pages=n_pages, n_kv_heads=hkv, head_dim=hd, page_size=case["page"], dtype=case["dtype"])
        kv.pool.copy_(_values(case, seed, 3, _pool_shape(case)))
        state.update(kv=kv, pool=kv.pool, step=paged.PagedStep(tables["q_start"], tables["kv_len"], tables["pages"], n_tokens=n,
                                                               max_q_len=max(q for q, _ in seqs), max_kv_len=max(lengths)))
    else:
        state.update(pool=_values(case, seed, 3, _pool_shape(case)), seqs=seqs, starts=start.tolist(), pages=tables["pages"])
        if case["kind"] == "append":
            state["seq"] = torch.tensor(np.repeat(np.arange(len(seqs)), [q for q, _ in seqs]), device="cuda")
            state["pos"] = torch.tensor(np.concatenate([np.arange(length - q, length) for q, length in seqs]), device="cuda")
    if case["kind"] == "append":
        state.update(q=rows[:, :hq], k=rows[:, hq:hq + hkv], v=rows[:, hq + hkv:],
                     q_out=torch.empty((n, hq, hd), dtype=rows.dtype, device="cuda"))
    else:
        q = _values(case, seed, 4, (n, hq, hd))
        state.update(q=q, out=torch.empty_like(q))
        if own:
            state["workspace"] = state["kv"].workspace(state["step"], hq)
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if own:
        from paper_2504_10724_amd import paged
        if case["kind"] == "rope":
            return state["rope"].apply(state["x"], state["pos"], out=state["y"], inverse=case["back"])
        if case["kind"] == "append":
            paged.append(state["kv"], 1, state["step"], state["k"], state["v"], rope=state["rope"], q=state["q"], q_out=state["q_out"])
            return dict(q=state["q_out"], pool=state["pool"])
        return paged.attend(state["kv"], 1, state["step"], state["q"], out=state["out"], window=case["window"],
                            workspace=state["workspace"])
    if case["kind"] == "rope":
        state["y"].copy_(_plain_rotate(state, state["x"], state["pos"].long(), case["back"]))
        return state["y"]
    if case["kind"] == "append":
        return _plain_append(state)
    return _plain_attend(state)


def _plain_rotate(state, x, pos, back):
    case, r = state["case"], _rot(state["case"])
    c, s = state["cos"][pos][:, None], state["sin"][pos][:, None]
    if back:
        s = -s
    x = x.float()
    if case["pairing"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_places(case, page, at):
    """elements of the pool where position `at` of page `page` keeps its keys and values: [n][hkv][hd] each"""
    hkv, hd, ps = case["hkv"], case["hd"], case["page"]
    g, i = torch.arange(hkv, device="cuda")[None, :, None], torch.arange(hd, device="cuda")[None, None, :]
    base, at = (page[:, None, None] * hkv + g) * (2 * ps * hd), at[:, None, None]
    if case["dtype"] == "f32":
        return base + at * hd + i, base + (ps + at) * hd + i
    r, base = at % 32, base + at // 32 * (64 * hd)
    k = (((r // 16 * (hd // 32) + i // 32) * 4 + i % 32 // 8) * 16 + r % 16) * 8 + i % 8
    v = ((i // 16 * 4 + r % 16 // 4) * 16 + i % 16) * 8 + r // 16 * 4 + r % 4
    return base + k, base + 32 * hd + v


def _plain_append(state):
    case, pool, pos = state["case"], state["pool"], state["pos"]
    page = state["pages"][state["seq"], pos // case["page"]].long()
    k_at, v_at = _plain_places(case, page, pos % case["page"])
    pool[k_at] = _plain_rotate(state, state["k"], pos, False).to(pool.dtype)
    pool[v_at] = state["v"].to(pool.dtype)
    state["q_out"].copy_(_plain_rotate(state, state["q"], pos, False))
    return dict(q=state["q_out"], pool=pool)


def _plain_gather(case, pool, pages, n):
    """first n positions of a sequence, [2][hkv][n][hd] in 32 bits"""
    hkv, hd, ps = case["hkv"], case["hd"], case["page"]
    b = pool.view(-1, hkv, 2 * ps * hd)[pages].float()
    if case["dtype"] == "f32":
        b = b.view(-1, hkv, 2, ps, hd).permute(2, 1, 0, 3, 4)
    else:
        b = b.view(-1, hkv, ps // 32, 2, 32 * hd)
        k = b[:, :, :, 0].reshape(-1, hkv, ps // 32, 2, hd // 32, 4, 16, 8).permute(1, 0, 2, 3, 6, 4, 5, 7)
        v = b[:, :, :, 1].reshape(-1, hkv, ps // 32, hd // 16, 4, 16, 2, 4).permute(1, 0, 2, 6, 4, 7, 3, 5)
        b = torch.stack([k.reshape(hkv, -1, hd), v.reshape(hkv, -1, hd)])
    return b.reshape(2, hkv, -1, hd)[:, :, :n]


def _plain_attend(state):
    case, out = state["case"], state["out"]
    hq, hkv, hd, w, ps = case["hq"], case["hkv"], case["hd"], case["window"], case["page"]
    for s, (n, length) in enumerate(state["seqs"]):
        at = state["starts"][s]
        k, v = _plain_gather(case, state["pool"], state["pages"][s, :(length + ps - 1) // ps], length)
        q = state["q"][at:at + n].float().view(n, hkv, hq // hkv, hd).permute(1, 2, 0, 3).reshape(hkv, -1, hd)
        pos = torch.arange(length - n, length, device="cuda")[:, None]
        j = torch.arange(length, device="cuda")[None]
        hide = j > pos if w == 0 else (j > pos) | (j <= pos - w)
        step = max(1, (1 << 28) // (q.shape[1] * length))            # key/value heads at a time
        for g in range(0, hkv, step):
            x = torch.matmul(q[g:g + step], k[g:g + step].transpose(1, 2).contiguous()) * (1.0 / math.sqrt(hd))
            x = x.view(-1, n, length).masked_fill_(hide, -math.inf)
            x = torch.exp(x - x.amax(-1, keepdim=True))
            x = (x / x.sum(-1, keepdim=True)).view(-1, hq // hkv * n, length)
            y = torch.matmul(x, v[g:g + step].contiguous()).view(-1, n, hd)
            out[at:at + n, g * (hq // hkv):g * (hq // hkv) + len(y)] = y.transpose(0, 1)
    return out


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rope":
        n, r = case["n"], _rot(case)
        return dict(bytes=2.0 * size * n * (hq + hkv) * hd + 4.0 * n * (r + 1), flops=3.0 * n * (hq + hkv) * r)
    seqs, w = _sequences(case), case.get("window", 0)
    n = sum(q for q, _ in seqs)
    tables = 4.0 * (2 * len(seqs) + sum((length + case["page"] - 1) // case["page"] for _, length in seqs))
    if case["kind"] == "append":
        return dict(bytes=2.0 * size * n * (hq + 2 * hkv) * hd + 4.0 * n * _rot(case) + tables, flops=3.0 * n * (hq + hkv) * _rot(case))
    pairs = keys = 0
    for q, length in seqs:
        pairs += sum(min(p + 1, w or p + 1) for p in range(length - q, length))
        keys += min(length, q + w - 1) if w else length
    return dict(bytes=2.0 * size * (keys * hkv * hd + n * hq * hd) + tables, flops=4.0 * pairs * hq * hd)


# ------------------------------------------------------------------ the same in 64 bits
def _exact_rotate(case, x, pos, back=False):
    """element by element from its pair's partner: y_i = x_i cos + (partner) sin, minus for the first of a pair"""
    r = _rot(case)
    i = torch.arange(r, device="cuda")
    if case["pairing"] == "half":
        pair, partner, first = i % (r // 2), (i + r // 2) % r, i < r // 2
    else:
        pair, partner, first = i // 2, i + 1 - i % 2 * 2, i % 2 == 0
    a = pos.double()[:, None] * torch.tensor(_frequencies(case), device="cuda")[pair]
    sign = torch.where(first, -1.0, 1.0).double() * (-1.0 if back else 1.0)
    y = x.double().clone()
    y[..., :r] = x[..., :r].double() * torch.cos(a)[:, None] + x[..., partner].double() * (torch.sin(a) * sign)[:, None]
    return y


def _exact_split(case, block):
    """keys and values [n][hkv][page][hd] of pages [n][hkv][2 page hd], by the place of each element"""
    hd, ps = case["hd"], case["page"]
    p, i = torch.arange(ps, device="cuda")[:, None], torch.arange(hd, device="cuda")[None]
    if case["dtype"] == "f32":
        k, v = p * hd + i, (ps + p) * hd + i
    else:
        half, quad, in_quad, group = p % 32 // 16, p % 16 // 4, p % 4, p // 32 * 64 * hd
        k = group + half * 16 * hd + i // 8 * 128 + p % 16 * 8 + i % 8
        v = group + 32 * hd + i // 16 * 512 + quad * 128 + i % 16 * 8 + half * 4 + in_quad
    return block[..., k], block[..., v], k, v


def exact(case, seed):
    if case["kind"] == "rope":
        x = _rows(case, seed)[:, :case["hq"] + case["hkv"]]
        return _exact_rotate(case, x, _rope_positions(case, seed), case["back"])
    hq, hkv, hd, ps = case["hq"], case["hkv"], case["hd"], case["page"]
    seqs, table = _sequences(case), _pages(case)[1]
    blocks = _values(case, seed, 3, _pool_shape(case)).view(-1, hkv, 2 * ps * hd)
    if case["kind"] == "append":
        rows, pool = _rows(case, seed), blocks.double()
        pos = torch.tensor([p for q, length in seqs for p in range(length - q, length)], device="cuda")
        page = torch.tensor([int(table[s, p // ps]) for s, (q, length) in enumerate(seqs) for p in range(length - q, length)], device="cuda")
        _, _, k_at, v_at = _exact_split(case, pool[:1])
        g = torch.arange(hkv, device="cuda")[None, :, None]
        pool[page[:, None, None], g, k_at[pos % ps][:, None]] = _exact_rotate(case, rows[:, hq:hq + hkv], pos)
        pool[page[:, None, None], g, v_at[pos % ps][:, None]] = rows[:, hq + hkv:].double()
        return dict(q=_exact_rotate(case, rows[:, :hq], pos), pool=pool.view(-1))
    n = sum(q for q, _ in seqs)
    q_all, out, at = _values(case, seed, 4, (n, hq, hd)), torch.empty((n, hq, hd), dtype=torch.float64, device="cuda"), 0
    for s, (new, length) in enumerate(seqs):
        mine = blocks[torch.tensor(table[s, :(length + ps - 1) // ps].astype(np.int64), device="cuda")]
        behind = torch.arange(length - new, length, device="cuda")[:, None] - torch.arange(length, device="cuda")[None]
        seen = (behind >= 0) & (behind < (case["window"] or length + 1))
        hidden = torch.zeros(seen.shape, dtype=torch.float64, device="cuda").masked_fill_(~seen, -math.inf)
        few = max(1, (1 << 26) // (new * length)) if new > 1 else hq   # query heads at a time
        for g in range(hkv):
            k, v, _, _ = _exact_split(case, mine[:, g])
            k, v = k.reshape(-1, hd)[:length].double(), v.reshape(-1, hd)[:length].double()
            kt = k.T.contiguous() / math.sqrt(hd)
            h, end = g * (hq // hkv), (g + 1) * (hq // hkv)
            while h < end:
                m = min(few, end - h)
                z = (q_all[at:at + new, h:h + m].double().reshape(-1, hd) @ kt).view(new, m, length) + hidden[:, None]
                out[at:at + new, h:h + m] = (torch.softmax(z, -1).view(-1, length) @ v).view(new, m, hd)
                h += m
        at += new
    return out
