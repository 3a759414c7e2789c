"""Rotary positions, the append to the paged cache and the attention over it against their definitions in 64 bits.

Tolerances.  bf16 results carry one rounding (an 8-bit significand: 2^-8 of the value); the attention's probabilities another (2^-8
of each, which moves a result by at most 2^-8 sum_j p_j |v_j| =: 2^-8 A, and |result| <= A): 2^-7 A on top of what fp32 gives.  fp32 results: a rotation is two products and a sum of values rounded once each, and a table entry rounded
once (4 x 2^-24 of |a| + |b|); a score's error is at most (hd + 2) 2^-24 D, D = max_j sum_i |q_i k_ji| scale, a probability's relative
error twice that (its own score and the largest) and a few roundings, the sums over n positions add n 2^-24 at most."""
import ctypes as C

import pytest
import torch

import paged_ref as R
from paper_2504_10724_amd import capi as ee
from paper_2504_10724_amd import paged as P

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _randn(shape, dtype, seed, std=1.3):
    return (torch.randn(shape, generator=_gen(seed)) * std).to(dtype)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32)


def _strided(x, token_pad, head_pad, shift):
    """x [n][h][hd] on the device as a view of a larger tensor: rows further apart, heads further apart, base shifted"""
    n, h, hd = x.shape
    ts = h * (hd + head_pad) + token_pad
    base = torch.full((n * ts + shift + hd,), 7.0, dtype=x.dtype, device="cuda")
    v = base.as_strided((n, h, hd), (ts, hd + head_pad, 1), shift)
    v.copy_(x)
    return v


# ------------------------------------------------------------------ rotary positions
ROPES = [
    # dtype, hd, rot, pairing, scaling, factor, (token pad, head pad, shift)
    ("bf16", 128, 128, "half", "none", 1.0, (0, 0, 0)),
    ("bf16", 128, 128, "interleaved", "linear", 4.0, (0, 0, 0)),
    ("bf16", 128, 64, "half", "base", 8.0, (16, 0, 0)),
    ("bf16", 96, 24, "interleaved", "bands", 8.0, (8, 8, 8)),
    ("bf16", 96, 24, "half", "bands", 2.5, (0, 0, 0)),               # 12 pairs: no whole 16-byte items
    ("bf16", 80, 80, "half", "none", 1.0, (0, 0, 1)),                # not aligned
    ("bf16", 64, 64, "interleaved", "none", 1.0, (3, 1, 0)),
    ("bf16", 6, 2, "half", "none", 1.0, (0, 0, 0)),
    ("f32", 64, 64, "half", "bands", 8.0, (0, 0, 0)),
    ("f32", 64, 32, "interleaved", "linear", 0.5, (4, 4, 4)),
    ("f32", 84, 42, "half", "none", 1.0, (0, 0, 0)),
    ("f32", 84, 42, "interleaved", "base", 3.0, (0, 0, 2)),
    ("f32", 2, 2, "interleaved", "none", 1.0, (1, 0, 0)),
]


@pytest.mark.parametrize("case", ROPES, ids=lambda c: "-".join(str(x) for x in c[:5]) + "-" + ".".join(str(x) for x in c[6]))
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_against_its_definition(case, inverse):
    dtype, hd, rot, pairing, scaling, factor, pads = case
    print(f"[case] rope {case} inverse {inverse}", flush=True)
    max_pos, n, heads = 70001, 37, 5
    rope = P.Rope(hd, max_pos, rot_dim=rot, pairing=pairing, theta=500.0, scaling=scaling, factor=factor, trained_pos=300, low=1.0, high=4.0,
                  magnitude=1.25)
    x = _randn((n, heads, hd), DT[dtype], 3)
    pos = torch.randint(0, max_pos, (n,), generator=_gen(4), dtype=torch.int32)
    pos[0], pos[1] = 0, max_pos - 1
    xd = _strided(x, *pads)
    got = rope.apply(xd, pos.cuda(), inverse=inverse)
    want = R.rotate(x, pos, rot, pairing, 1.25, inverse, theta=500.0, scaling=scaling, factor=factor, trained_pos=300)
    size = R.rotate(x.abs(), torch.zeros_like(pos), rot, pairing, 1.25).abs()          # |a| of each element; its partner's:
    both = size.clone()
    for j in range(rot // 2):
        a, b = (j, j + rot // 2) if pairing == "half" else (2 * j, 2 * j + 1)
        both[..., a] = both[..., b] = size[..., a] + size[..., b]
    tol = 4 * U * both + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
    assert ((got.cpu().double() - want).abs() <= tol).all()
    assert torch.equal(got[..., rot:].cpu(), x[..., rot:])
    rope.apply(xd, pos.cuda(), out=xd, inverse=inverse)                                # in place: the same bits
    assert torch.equal(xd, got)
    if pads != (0, 0, 0):                                                              # what lies between the rows stays
        whole = torch.as_strided(xd, (xd.stride(0) * n,), (1,), 0).cpu()
        keep = torch.ones(len(whole), dtype=torch.bool)
        at = pads[2] + torch.arange(n)[:, None, None] * xd.stride(0) + torch.arange(heads)[None, :, None] * xd.stride(1) + torch.arange(hd)
        keep[at[at < len(whole)]] = False
        assert (whole[keep] == 7.0).all()


@pytest.mark.parametrize("n,heads", [(1, 1), (1, 72), (2, 3), (1001, 9), (5, 200)])
def test_rope_sizes(n, heads):
    print(f"[case] rope {n} rows of {heads} heads", flush=True)
    rope = P.Rope(128, 4096)
    x = _randn((n, heads, 128), torch.bfloat16, 6)
    pos = torch.randint(0, 4096, (n,), generator=_gen(7), dtype=torch.int32)
    want = R.rotate(x, pos, 128)
    tol = 2.0 ** -8 * want.abs() + 8 * U * x.abs().double().amax()
    assert ((rope.apply(x.cuda(), pos.cuda()).cpu().double() - want).abs() <= tol).all()


def test_rope_inverse_is_the_gradient():
    """sum(w * rope(x)) differs by w . rope(e) along e: against differences of the operator itself, which is linear"""
    print("[case] rope gradient", flush=True)
    for pairing in ("half", "interleaved"):
        rope = P.Rope(24, 500, rot_dim=16, pairing=pairing, magnitude=0.75)
        x, w = _randn((3, 2, 24), torch.float32, 8).cuda(), _randn((3, 2, 24), torch.float32, 9).cuda()
        pos = _i32([0, 17, 499]).cuda()
        grad = rope.apply(w, pos, inverse=True).double()
        for t in range(3):
            for i in range(24):
                e = torch.zeros_like(x)
                e[t, 1, i] = 0.5
                up, down = rope.apply(x + e, pos).double(), rope.apply(x - e, pos).double()
                diff = ((up - down) * w.double()).sum()
                # x + e and x - e are rounded once, and so are the products: up to 40 values of size 6 times 2^-24
                assert abs(diff - grad[t, 1, i]) <= 40 * 6 * 6 * U, (pairing, t, i)


def test_rope_positions_outside_the_table_are_refused():
    print("[case] rope refusals", flush=True)
    rope = P.Rope(64, 100)
    x = _randn((5, 2, 64), torch.float32, 10).cuda()
    out, status = torch.full_like(x, 9.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    rope.apply(x, _i32([5, -1, 99, 100, 0]).cuda(), out=out, status=status)
    assert status.item() == 1
    assert (out[1] == 9.0).all() and (out[3] == 9.0).all() and (out[[0, 2, 4]] != 9.0).all()
    rope.apply(x, _i32([5, -1, 99, 100, 0]).cuda(), out=out)                           # nowhere to report: still not written
    assert (out[1] == 9.0).all()
    assert rope.apply(x[:0], _i32([]).cuda()).shape == (0, 2, 64)


# ------------------------------------------------------------------ batches over a paged cache
class Batch:
    """seqs: (new rows, positions with them) of each sequence; pages in a random order, three to spare"""

    def __init__(self, seqs, hq, hkv, hd, ps, dtype, *, n_layers=1, seed=1, drop=()):
        self.seqs, self.hq, self.hkv, self.hd, self.ps, self.dt = seqs, hq, hkv, hd, ps, DT[dtype]
        need = [max(0, (length + ps - 1) // ps) for _, length in seqs]
        self.n_pages, self.n_layers = sum(need) + 3, n_layers
        order = torch.randperm(self.n_pages, generator=_gen(seed)).tolist()
        self.pages, at = [], 0
        for n in need:
            self.pages.append(order[at:at + n])
            at += n
        for s, i, value in drop:
            self.pages[s][i] = value
        width = max(1, max(need))
        table = torch.full((len(seqs), width), -1, dtype=torch.int32)
        for s, p in enumerate(self.pages):
            table[s, :len(p)] = _i32(p)
        start = [0]
        for n, _ in seqs:
            start.append(start[-1] + n)
        self.n, self.start = start[-1], start
        self.kv = P.PagedCache(n_layers, self.n_pages, hkv, hd, ps, dtype)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.step = P.PagedStep(_i32(start).cuda(), _i32([length for _, length in seqs]).cuda(), table.cuda(), n_tokens=self.n,
                                max_q_len=max(n for n, _ in seqs), max_kv_len=max(0, max(length for _, length in seqs)), status=self.status)
        self.seed = seed

    def fill(self, std=1.3):
        """random keys and values in every page; returns them as [2][layer][page][hkv][ps][hd]"""
        x = _randn((2, self.n_layers, self.n_pages, self.hkv, self.ps, self.hd), self.dt, self.seed + 50, std)
        self.put(x)
        return x

    def put(self, x):
        self.kv.pool.copy_(R.write_pool(x, self.dt))

    def get(self):
        return R.read_pool(self.kv.pool.cpu(), self.n_layers, self.n_pages, self.hkv, self.hd, self.ps)

    def queries(self, std=1.3):
        return _randn((self.n, self.hq, self.hd), self.dt, self.seed + 60, std)

    def check_attention(self, x, q, layer=1, window=0, scale=None, got=None):
        s = self.hd ** -0.5 if scale is None else scale
        want, size, dots = R.attend(q, x[:, layer - 1], self.seqs, self.pages, window, s)
        if got is None:
            got = P.attend(self.kv, layer, self.step, q.cuda(), scale=scale, window=window)
        tol = U * size * (2 * (self.hd + 4) * dots + max(length for _, length in self.seqs) + 64)
        if self.dt == torch.bfloat16:
            tol = tol + 2.0 ** -7 * size
        err = (got.cpu().double() - want).abs()
        bad = ~(err <= tol)
        assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), float((err / tol.clamp_min(1e-30)).max()))
        return got


def _append_reference(b, x, k, v, rope_args, n_max, layer):
    """the pool after the append, and which (2, page, head, position) entries it wrote"""
    want, wrote = x.double().clone(), torch.zeros(x.shape[:-1], dtype=torch.bool)
    row = 0
    for (rows, length), table in zip(b.seqs, b.pages):
        for j in range(rows):
            p = length - rows + j
            if 0 <= p < n_max and 0 <= table[p // b.ps] < b.n_pages:
                kk = R.rotate(k[row][None], _i32([p]), **rope_args)[0] if rope_args else k[row].double()
                want[0, layer - 1, table[p // b.ps], :, p % b.ps] = kk
                want[1, layer - 1, table[p // b.ps], :, p % b.ps] = v[row].double()
                wrote[:, layer - 1, table[p // b.ps], :, p % b.ps] = True
            row += 1
    return want, wrote


APPENDS = [
    # dtype, hq, hkv, hd, page, rot, pairing, seqs
    ("bf16", 8, 2, 128, 64, 128, "half", [(1, 1), (1, 64), (1, 65), (1, 200)]),
    ("bf16", 4, 4, 128, 32, 64, "interleaved", [(1, 33), (0, 40), (1, 7)]),
    ("bf16", 8, 2, 128, 96, 128, "half", [(70, 70), (1, 97), (33, 64), (5, 101), (2, 130), (0, 0)]),
    ("bf16", 3, 1, 96, 64, 48, "half", [(31, 62), (32, 64), (33, 65), (1, 300)]),
    ("bf16", 0, 5, 64, 128, 0, "half", [(100, 131), (17, 17)]),
    ("bf16", 2, 1, 256, 64, 24, "half", [(40, 41)]),                  # 12 pairs: element by element
    ("bf16", 12, 3, 192, 32, 192, "interleaved", [(2, 33), (2, 2), (1, 64)]),
    ("f32", 4, 4, 64, 64, 64, "half", [(1, 65)] * 8),
    ("f32", 6, 2, 84, 32, 42, "half", [(50, 99), (1, 1), (3, 40)]),
    ("f32", 2, 2, 4, 96, 4, "interleaved", [(100, 100)]),
]


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: "-".join(str(x) for x in c[:7]))
@pytest.mark.parametrize("layout", ["qkv", "apart", "odd"])
def test_append_against_its_definition(case, layout):
    dtype, hq, hkv, hd, ps, rot, pairing, seqs = case
    print(f"[case] append {case} {layout}", flush=True)
    b = Batch(seqs, hq, hkv, hd, ps, dtype, n_layers=2)
    x = b.fill()
    rows = _randn((b.n, hq + 2 * hkv, hd), b.dt, 11)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    max_pos = 400
    rope = P.Rope(hd, max_pos, rot_dim=rot, pairing=pairing) if rot else None
    if layout == "qkv":
        dev = rows.cuda()
        dq, dk, dv = dev[:, :hq], dev[:, hq:hq + hkv], dev[:, hq + hkv:]
    elif layout == "apart":
        dq, dk, dv = q.cuda(), k.transpose(0, 1).contiguous().cuda().transpose(0, 1), v.contiguous().cuda()
    else:
        dq, dk, dv = _strided(q, 0, 8, 0) if hq else None, _strided(k, 1, 0, 3), _strided(v, 5, 2, 1)
    q_out = P.append(b.kv, 2, b.step, dk, dv, rope=rope, q=dq if hq else None)
    want, wrote = _append_reference(b, x, k, v, dict(rot=rot, pairing=pairing) if rot else None, max_pos, 2)
    got = b.get()
    assert torch.equal(got[~wrote], x[~wrote])                         # nothing else moved, the other layer included
    assert torch.equal(got[1], want[1].to(b.dt))
    near = 2.0 ** -8 if dtype == "bf16" else 0.0
    assert ((got[0].double() - want[0]).abs() <= near * want[0].abs() + 8 * U * 8).all()
    if hq:
        pos = _i32([length - n + j for n, length in seqs for j in range(n)])
        wq = R.rotate(q, pos, rot, pairing) if rot else q.double()
        assert ((q_out.cpu().double() - wq).abs() <= near * wq.abs() + 8 * U * 8).all()
    assert b.status.item() == 0


def test_append_refuses_row_by_row():
    print("[case] append refusals", flush=True)
    # a sequence with more new rows than positions, one past the rotary table, one with a page that does not exist, one that is fine
    b = Batch([(5, 3), (4, 102), (40, 100), (2, 34)], 2, 1, 128, 32, "bf16", drop=[(2, 2, -1), (3, 0, 99)])
    x = b.fill()
    rows = _randn((b.n, 4, 128), b.dt, 12)
    dev = rows.cuda()
    q_out = torch.full((b.n, 2, 128), 9.0, dtype=b.dt, device="cuda")
    P.append(b.kv, 1, b.step, dev[:, 2:3], dev[:, 3:], rope=P.Rope(128, 100), q=dev[:, :2], q_out=q_out)
    assert b.status.item() == 1
    _, wrote = _append_reference(b, x, rows[:, 2:3], rows[:, 3:], dict(rot=128), 100, 1)
    got = b.get()
    assert torch.equal(got[~wrote], x[~wrote])
    assert not torch.equal(got[wrote], x[wrote])
    untouched = (q_out == 9.0).all(-1).all(-1).cpu().tolist()
    pos = [length - n + j for n, length in b.seqs for j in range(n)]
    assert untouched == [not 0 <= p < 100 for p in pos]


def test_sequences_outside_the_hosts_figures_are_left_out():
    print("[case] figures", flush=True)
    b = Batch([(3, 40), (2, 90), (4, 20)], 4, 2, 128, 32, "bf16")
    x, q = b.fill(), b.queries()
    for q_start, kv_len, bad in (([0, 3, 5, 9], [40, 97, 20], 1), ([0, 3, 8, 9], [40, 90, 20], 1), ([0, 3, 2, 9], [40, 90, 20], None),
                                 ([0, 3, 5, 10], [40, 90, 20], 2), ([0, 3, 5, 9], [-1, 90, 20], 0)):
        b.status.zero_()
        step = P.PagedStep(_i32(q_start).cuda(), _i32(kv_len).cuda(), b.step.tensors[2], n_tokens=9, max_q_len=4, max_kv_len=96,
                           status=b.status)
        out = torch.full((9, 4, 128), 9.0, dtype=b.dt, device="cuda")
        P.attend(b.kv, 1, step, q.cuda(), out=out)
        assert b.status.item() & 2, (q_start, kv_len)
        b.put(x)
        rows = torch.zeros((9, 2, 128), dtype=b.dt, device="cuda")
        P.append(b.kv, 1, step, rows, rows)
        torch.cuda.synchronize()
        if bad is not None:
            lo, hi = (0, 3, 5)[bad], (3, 5, 9)[bad]
            assert (out[lo:hi] == 9.0).all()


# ------------------------------------------------------------------ attention
ATTENDS = [
    # dtype, hq, hkv, hd, page, window, seqs
    ("bf16", 4, 4, 128, 64, 0, [(1, 1)]),
    ("bf16", 8, 1, 128, 32, 0, [(1, 1), (1, 31), (1, 32), (1, 33), (1, 64), (1, 257), (0, 9), (1, 1000)]),
    ("bf16", 6, 2, 64, 96, 0, [(1, 95), (1, 96), (1, 97), (1, 500)]),
    ("bf16", 16, 1, 96, 32, 0, [(1, 200), (1, 3)]),
    ("bf16", 20, 1, 128, 64, 0, [(1, 200), (1, 3), (1, 700)]),         # more query heads a kv head than a block of 16
    ("bf16", 71, 1, 64, 128, 0, [(1, 300), (2, 5)]),
    ("bf16", 4, 2, 192, 64, 0, [(1, 130), (3, 130)]),
    ("bf16", 4, 2, 256, 32, 0, [(1, 130), (17, 130), (1, 1)]),
    ("bf16", 8, 2, 128, 64, 0, [(4, 70), (4, 4), (4, 300), (4, 129)]),  # every sequence the same few rows
    ("bf16", 8, 2, 128, 64, 0, [(70, 70), (1, 200), (33, 133), (0, 0), (1, 1), (16, 300)]),
    ("bf16", 4, 4, 128, 32, 0, [(130, 130), (1, 77)]),
    ("bf16", 3, 1, 96, 64, 0, [(129, 200), (64, 64)]),
    ("bf16", 4, 1, 256, 64, 0, [(70, 100), (1, 20)]),
    ("bf16", 8, 2, 64, 64, 0, [(150, 170)]),
    ("bf16", 4, 2, 192, 96, 0, [(50, 199)]),
    ("bf16", 8, 2, 128, 64, 1, [(40, 90), (1, 33)]),                   # a row sees itself alone
    ("bf16", 8, 2, 128, 64, 37, [(40, 90), (1, 300), (3, 3)]),
    ("bf16", 8, 2, 128, 32, 64, [(100, 400), (1, 64), (1, 65)]),
    ("bf16", 8, 2, 128, 64, 1 << 30, [(40, 90), (1, 300)]),
    ("bf16", 8, 2, 128, 64, 0, [(9, 4), (1, 0), (40, 10), (2, 70)]),   # rows before position 0 see nothing
    ("f32", 4, 4, 64, 64, 0, [(1, 65)] * 8),
    ("f32", 6, 2, 84, 32, 0, [(50, 99), (1, 1), (3, 40), (1, 600)]),
    ("f32", 2, 1, 4, 96, 0, [(100, 100)]),
    ("f32", 10, 1, 256, 32, 0, [(7, 150), (1, 33)]),
    ("f32", 20, 1, 36, 32, 17, [(70, 150), (1, 33), (5, 2)]),
    ("f32", 4, 2, 128, 64, 0, [(1, 1500)]),
]


@pytest.mark.parametrize("case", ATTENDS, ids=lambda c: "-".join(str(x) for x in c[:6]) + f"-{sum(n for n, _ in c[6])}rows")
def test_attention_against_its_definition(case):
    dtype, hq, hkv, hd, ps, window, seqs = case
    print(f"[case] attend {case}", flush=True)
    b = Batch(seqs, hq, hkv, hd, ps, dtype, n_layers=2)
    x, q = b.fill(), b.queries()
    got = b.check_attention(x, q, layer=2, window=window)
    assert b.status.item() == 0
    # rows and results anywhere in memory
    for pads in ((8, 0, 8), (1, 3, 1)):
        qd, out = _strided(q, *pads), _strided(torch.zeros_like(q), *pads)
        P.attend(b.kv, 2, b.step, qd, out=out, window=window)
        assert torch.equal(out, got), pads


@pytest.mark.parametrize("dtype,rows", [("bf16", 1), ("bf16", 8), ("bf16", 100), ("f32", 1), ("f32", 40)])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, rows):
    """infinities and NaN at later positions, before the window, in unused parts of the pages and in other pages"""
    for value in (float("inf"), float("nan"), -3.0e38):
        print(f"[case] unseen {dtype} {rows} rows {value}", flush=True)
        b = Batch([(rows, 250), (rows, rows), (rows, 129)], 8, 2, 128, 64, dtype)
        x, q = b.fill(), b.queries()
        ref = b.check_attention(x, q, window=100)
        y = torch.full_like(x, value)
        for (n, length), table in zip(b.seqs, b.pages):
            for p in range(max(0, length - n - 99), length):
                y[:, 0, table[p // 64], :, p % 64] = x[:, 0, table[p // 64], :, p % 64]
        b.put(y)
        assert torch.equal(P.attend(b.kv, 1, b.step, q.cuda(), window=100), ref)
        if rows > 1:                                                   # the last position: every earlier row is as before
            for (n, length), table in zip(b.seqs, b.pages):
                y[:, 0, table[(length - 1) // 64], :, (length - 1) % 64] = value
            b.put(y)
            got = P.attend(b.kv, 1, b.step, q.cuda(), window=100)
            last = [e - 1 for e in b.start[1:]]
            keep = [i for i in range(b.n) if i not in last]
            assert torch.equal(got[keep], ref[keep])


@pytest.mark.parametrize("dtype,rows", [("bf16", 1), ("bf16", 100), ("f32", 1), ("f32", 40)])
def test_non_finite_values_reach_the_rows_that_see_them(dtype, rows):
    print(f"[case] seen {dtype} {rows} rows", flush=True)
    b = Batch([(rows, 250), (rows, rows + 3)], 4, 2, 128, 64, dtype)
    x, q = b.fill(), b.queries()
    ref = b.check_attention(x, q)
    at = 250 - rows                                                    # of the first row: all rows of sequence 0 see it
    for value in (float("inf"), float("nan")):
        y = x.clone()
        y[1, 0, b.pages[0][at // 64], 1, at % 64, 5] = value           # one feature of a value of kv head 1
        b.put(y)
        got = P.attend(b.kv, 1, b.step, q.cuda())
        assert torch.equal(got[rows:], ref[rows:]) and torch.equal(got[:rows, :2], ref[:rows, :2])
        other = [i for i in range(128) if i != 5]
        assert torch.equal(got[:rows, 2:][..., other], ref[:rows, 2:][..., other])
        hit = got[:rows, 2:, 5].float()
        assert (hit.isnan() if value != value else hit == value).all()
        y = x.clone()
        y[0, 0, b.pages[0][at // 64], 1, at % 64, 5] = float("nan")    # a key: the whole row
        b.put(y)
        got = P.attend(b.kv, 1, b.step, q.cuda())
        assert got[:rows, 2:].isnan().all() and torch.equal(got[rows:], ref[rows:])


def test_scores_of_any_size():
    """keys of the type's lowest value and scores far apart: the softmax's maximum carries them; all scores -inf is 0/0"""
    print("[case] score sizes", flush=True)
    for dtype in ("bf16", "f32"):
        for rows in (1, 70):
            b = Batch([(rows, 200)], 2, 1, 64, 32, dtype)
            x, q = b.fill(), b.queries()
            x[0, 0] *= 64.0                                            # scores of several hundred
            b.put(x)
            b.check_attention(x, q)
            x[0, 0] = torch.finfo(b.dt).min                            # finite keys, infinite scores: -inf for q of positive sum
            b.put(x)
            q1 = torch.ones_like(q)
            got = P.attend(b.kv, 1, b.step, q1.cuda(), scale=1.0)
            assert got.isnan().all()
            x[0, 0, b.pages[0][0], 0, 0] = 0.0                         # one finite score: it takes all
            b.put(x)
            got = P.attend(b.kv, 1, b.step, q1.cuda(), scale=1.0)
            assert torch.equal(got[:, 0].cpu(), x[1, 0, b.pages[0][0], 0, 0].expand(rows, -1))


def test_scales_and_large_contexts():
    print("[case] scale, long", flush=True)
    b = Batch([(3, 3000), (1, 2049)], 2, 1, 64, 32, "bf16")
    x, q = b.fill(), b.queries()
    for scale in (0.0, -0.2, 0.5):
        b.check_attention(x, q, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_unmapped_pages_are_left_out(dtype):
    print(f"[case] unmapped {dtype}", flush=True)
    for rows in (1, 60):
        b = Batch([(rows, 200), (rows, 100), (rows, 300)], 8, 2, 64, 32, dtype, drop=[(0, 2, -1), (0, 6, 9999), (2, 0, -5)] +
                  [(1, i, -1) for i in range(4)])
        x, q = b.fill(), b.queries()
        got = b.check_attention(x, q)
        assert b.status.item() == 1
        assert (got[rows:2 * rows] == 0).all()                         # nothing left of sequence 1


def test_offsets_beyond_32_bits():
    """a pool of more than 2^32 elements: the last pages, by append and attention"""
    print("[case] 64-bit offsets", flush=True)
    n_pages, ps, hkv, hd = 4200, 4096, 1, 128                          # 2^32.03 elements
    b = Batch([(40, 300), (1, 130)], 2, hkv, hd, 32, "bf16")
    kv = P.PagedCache(1, n_pages, hkv, hd, ps, "bf16")
    assert kv.pool.numel() > 1 << 32
    pages = _i32([[n_pages - 1], [n_pages - 2]]).cuda()
    step = P.PagedStep(b.step.tensors[0], b.step.tensors[1], pages, n_tokens=41, max_q_len=40, max_kv_len=300)
    hist = P.PagedStep(_i32([0, 300, 430]).cuda(), b.step.tensors[1], pages, n_tokens=430, max_q_len=300, max_kv_len=300)
    k, v = _randn((430, 1, hd), torch.bfloat16, 31), _randn((430, 1, hd), torch.bfloat16, 32)
    P.append(kv, 1, hist, k.cuda(), v.cuda())
    q = b.queries()
    got = P.attend(kv, 1, step, q.cuda())
    x = torch.zeros(2, 2, 1, 4096, hd, dtype=torch.bfloat16)
    x[0, 0, 0, :300], x[1, 0, 0, :300], x[0, 1, 0, :130], x[1, 1, 0, :130] = k[:300, 0], v[:300, 0], k[300:, 0], v[300:, 0]
    want, size, _ = R.attend(q, x, b.seqs, [[0], [1]], 0, hd ** -0.5)
    assert ((got.cpu().double() - want).abs() <= 2.0 ** -7 * 1.01 * size).all()


def test_chunks_and_single_tokens_build_the_same_cache_and_the_same_answers():
    """a prompt in one call, in chunks, token by token: the pools are equal, the answers close"""
    print("[case] chunks", flush=True)
    hq, hkv, hd, ps, n = 4, 2, 128, 32, 75
    rows = _randn((n, hq + 2 * hkv, hd), torch.bfloat16, 40).cuda()
    rope = P.Rope(hd, 128)
    table = _i32([[4, 1, 3]]).cuda()
    results = []
    for cuts in ([0, 75], [0, 31, 32, 60, 75], list(range(76))):
        kv = P.PagedCache(1, 5, hkv, hd, ps, "bf16")
        kv.pool.zero_()
        out = torch.empty(n, hq, hd, dtype=torch.bfloat16, device="cuda")
        for a, e in zip(cuts, cuts[1:]):
            step = P.PagedStep(_i32([0, e - a]).cuda(), _i32([e]).cuda(), table, n_tokens=e - a, max_q_len=e - a, max_kv_len=96)
            part = rows[a:e]
            q = P.append(kv, 1, step, part[:, hq:hq + hkv], part[:, hq + hkv:], rope=rope, q=part[:, :hq])
            P.attend(kv, 1, step, q, out=out[a:e])
        results.append((kv.pool.clone(), out))
    for pool, out in results[1:]:
        assert torch.equal(pool, results[0][0])
        assert (out.float() - results[0][1].float()).abs().max() <= 2.0 ** -6 * rows.float().abs().max()      # each within 2^-7 A


def test_host_figures_above_the_devices():
    """one set of figures for every step of a server: rows, sequences and lengths below them"""
    print("[case] figures above", flush=True)
    b = Batch([(1, 70), (0, 0), (1, 200), (20, 30), (0, 5)], 8, 2, 128, 64, "bf16")
    x, q = b.fill(), b.queries()
    b.check_attention(x, q)
    width = torch.cat([b.step.tensors[2], torch.full((5, 60), -1, dtype=torch.int32, device="cuda")], 1)
    step = P.PagedStep(b.step.tensors[0], b.step.tensors[1], width, n_tokens=b.n, max_q_len=b.n, max_kv_len=4000, status=b.status)
    ws = b.kv.workspace(P.PagedStep(b.step.tensors[0], b.step.tensors[1], width, n_tokens=64, max_q_len=64, max_kv_len=4032), 8)
    got = P.attend(b.kv, 1, step, q.cuda(), workspace=ws)
    b.check_attention(x, q, got=got)
    assert b.status.item() == 0


def test_many_sequences():
    """more than 64 and more than 64 x 64 sequences, most without rows"""
    print("[case] many sequences", flush=True)
    for n_seqs in (65, 1000, 4500):
        lens = [(0, 0)] * n_seqs
        for s, n in ((0, 2), (63, 1), (64, 40), (n_seqs // 2, 3), (n_seqs - 1, 33)):
            lens[s] = (n, n + 20)
        b = Batch(lens, 2, 1, 64, 32, "bf16")
        x, q = b.fill(), b.queries()
        b.check_attention(x, q)
        k = _randn((b.n, 1, 64), b.dt, 70)
        P.append(b.kv, 1, b.step, k.cuda(), k.cuda())
        want, wrote = _append_reference(b, x, k, k, None, 1 << 30, 1)
        assert torch.equal(b.get().double(), want)


def test_repeated_calls_give_the_same_bits_on_any_stream():
    print("[case] streams", flush=True)
    b = Batch([(1, 2000), (1, 300), (30, 900)], 8, 2, 128, 64, "bf16")
    x, q = b.fill(), b.queries().cuda()
    ref = P.attend(b.kv, 1, b.step, q)
    ws = [b.kv.workspace(b.step, 8).fill_(255) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(P.attend(b.kv, 1, b.step, q, workspace=ws[i % 2]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs)


def test_a_recorded_step_follows_the_device_arrays():
    """append and attention in a graph; lengths and inputs change between the replays"""
    print("[case] graph", flush=True)
    hq, hkv, hd, ps = 8, 2, 128, 32
    rope, kv = P.Rope(hd, 512), P.PagedCache(1, 40, hkv, hd, ps, "bf16")
    kv.pool.normal_()
    start, table = _i32([0, 1, 2]).cuda(), torch.arange(32, dtype=torch.int32, device="cuda").view(2, 16)
    length = _i32([100, 30]).cuda()
    step = P.PagedStep(start, length, table, n_tokens=2, max_q_len=1, max_kv_len=512)
    rows = torch.zeros(2, hq + 2 * hkv, hd, dtype=torch.bfloat16, device="cuda")
    q, out, ws = torch.empty(2, hq, hd, dtype=torch.bfloat16, device="cuda"), torch.empty(2, hq, hd, dtype=torch.bfloat16, device="cuda"), kv.workspace(step, hq)

    def go():
        P.append(kv, 1, step, rows[:, hq:hq + hkv], rows[:, hq + hkv:], rope=rope, q=rows[:, :hq], q_out=q)
        P.attend(kv, 1, step, q, out=out, workspace=ws)
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for i in range(5):
        rows.copy_(_randn(tuple(rows.shape), torch.bfloat16, 80 + i))
        length.copy_(_i32([100 + 83 * i, 30 + i]))
        pool = kv.pool.clone()
        graph.replay()
        torch.cuda.synchronize()
        got, got_pool = out.clone(), kv.pool.clone()
        kv.pool.copy_(pool)
        go()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(got_pool, kv.pool), i


def test_wrapper_refusals():
    print("[case] wrapper refusals", flush=True)
    b = Batch([(2, 40)], 4, 2, 64, 32, "bf16")
    b.fill()
    q = b.queries().cuda()
    k = torch.zeros(2, 2, 64, dtype=b.dt, device="cuda")
    for bad in (q.float(), q[:1], q[..., :32], q.cpu(), q.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ee.EEError):
            P.attend(b.kv, 1, b.step, bad)
    with pytest.raises(ee.EEError):
        P.attend(b.kv, 1, b.step, q[:, :3])                            # 3 query heads of 2 kv heads
    with pytest.raises(ee.EEError):
        P.attend(b.kv, 2, b.step, q)
    with pytest.raises(ee.EEError):
        P.attend(b.kv, 1, b.step, q, out=q)
    with pytest.raises(ee.EEError):
        P.attend(b.kv, 1, b.step, q, window=-1)
    with pytest.raises(ee.EEError):
        P.append(b.kv, 1, b.step, k, k[:, :1])
    with pytest.raises(ee.EEError):
        P.append(b.kv, 1, b.step, k, k, rope=P.Rope(128, 100))
    with pytest.raises(ee.EEError):
        P.PagedStep(b.step.tensors[0].long(), b.step.tensors[1], b.step.tensors[2], n_tokens=2, max_q_len=2, max_kv_len=40)
    with pytest.raises(ee.EEError):
        P.PagedCache(1, 4, 2, 64, 48)
    with pytest.raises(ee.EEError):
        P.Rope(64, 100, pairing="both")
    n = ee.load().ee_paged_attention_workspace(b.kv.h, 4, C.byref(b.step.c))
    if n > 0:
        with pytest.raises(ee.EEError):
            P.attend(b.kv, 1, b.step, q, workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))


def test_rope_settings_keep_all_their_bits():
    """a factor that fp32 would round moves the angle of a late position by thousandths"""
    print("[case] rope settings", flush=True)
    x, pos = _randn((64, 3, 64), torch.float32, 90), torch.arange(64, dtype=torch.int32) * 2000 + 3000
    for scaling, factor in (("linear", 3.17), ("base", 7.53), ("bands", 1.23)):
        rope = P.Rope(64, 131072, scaling=scaling, factor=factor, theta=9999.7, trained_pos=4096, low=1.1, high=3.7, magnitude=1.07)
        got = rope.apply(x.cuda(), pos.cuda()).cpu().double()
        want = R.rotate(x, pos, 64, "half", 1.07, theta=9999.7, scaling=scaling, factor=factor, trained_pos=4096, low=1.1, high=3.7)
        # an angle of up to 1.3e5 in fp64 (2^-36 off at most), a table entry, two products and a sum
        assert ((got - want).abs() <= 4 * U * 1.07 * 2 * x.abs().amax() + 2.0 ** -35 * 8).all(), scaling


SPLITS = [
    # dtype, hq, hkv, hd, page, window, (rows, positions) of each sequence: lengths that are split and ones that are not, more
    # sequences than a tile has columns, tiles and single rows together
    ("f32", 4, 1, 64, 64, 0, [(1, 1600 + 7 * s) for s in range(21)]),
    ("f32", 2, 1, 84, 32, 0, [(3, 1700), (1, 40), (20, 1900), (1, 2200)]),
    ("bf16", 4, 1, 64, 64, 0, [(1, 1600 + 7 * s) for s in range(21)]),
    ("bf16", 4, 1, 64, 32, 0, [(9, 1700 + s) for s in range(9)]),              # 36 columns each: one tile a sequence
    ("bf16", 3, 1, 96, 64, 0, [(50, 1800), (1, 1700), (1, 30), (60, 2100)]),
    ("bf16", 4, 2, 128, 64, 1600, [(45, 2500), (1, 2400), (1, 1590)]),
    ("bf16", 8, 1, 192, 64, 0, [(10, 1900), (1, 1700), (3, 100)]),
]


@pytest.mark.parametrize("case", SPLITS, ids=lambda c: "-".join(str(x) for x in c[:6]) + f"-{len(c[6])}seqs")
def test_long_positions_in_shares(case):
    """at most 48 groups of 32 positions are never split: these are longer"""
    dtype, hq, hkv, hd, ps, window, seqs = case
    print(f"[case] shares {case[:6]} {len(seqs)} sequences", flush=True)
    b = Batch(seqs, hq, hkv, hd, ps, dtype)
    x, q = b.fill(), b.queries()
    assert ee.load().ee_paged_attention_workspace(b.kv.h, hq, C.byref(b.step.c)) > 0
    got = b.check_attention(x, q, window=window)
    ws = b.kv.workspace(b.step, hq).fill_(255)                         # whatever the workspace holds
    assert torch.equal(P.attend(b.kv, 1, b.step, q.cuda(), window=window, workspace=ws), got)


STEPS = [
    # heads of one and of two groups a step; windows that start in the first and in the second of two groups; lengths of an odd number of groups
    (128, 8, 2, 0, [(130, 607), (70, 70), (33, 993)]),
    (128, 4, 4, 301, [(140, 500), (65, 1300)]),
    (64, 6, 2, 333, [(90, 675), (64, 96)]),
    (96, 20, 1, 0, [(7, 650), (40, 161)]),
    (256, 4, 1, 270, [(50, 390), (17, 608)]),
]


@pytest.mark.parametrize("case", STEPS, ids=lambda c: "-".join(str(x) for x in c[:4]))
def test_tiles_whose_scores_rise_with_the_position(case):
    """the reference of the exponents moves many times, in groups that all columns see and in others; pages of one group are missing here
    and there"""
    hd, hq, hkv, window, seqs = case
    print(f"[case] rising {case}", flush=True)
    for drop in ((), [(0, 3, -1), (0, 8, -1), (0, 9, 1 << 20), (1, 1, -1)]):
        b = Batch(seqs, hq, hkv, hd, 32, "bf16", drop=drop)
        x, q = b.fill(), b.queries()
        for (n, length), table in zip(b.seqs, b.pages):
            for i, page in enumerate(table):
                if 0 <= page < b.n_pages:
                    x[0, 0, page] *= 0.5 + 0.75 * i                    # scores of a few at first, of a hundred at the end
        b.put(x)
        b.check_attention(x, q, window=window)
        assert b.status.item() == (1 if drop else 0)


@pytest.mark.parametrize("hd", [64, 128, 192])
def test_tiles_that_begin_with_scores_of_minus_infinity(hd):
    """positions whose score is -inf weigh nothing, also where nothing else has been seen yet: as if their pages were not there"""
    print(f"[case] -inf first {hd}", flush=True)
    seqs, low = [(100, 500)], 5
    b = Batch(seqs, 4, 2, hd, 32, "bf16")
    x, q = b.fill(), b.queries().abs()
    y = x.clone()
    for page in b.pages[0][:low]:
        y[0, 0, page] = torch.finfo(b.dt).min
    b.put(y)
    got = P.attend(b.kv, 1, b.step, q.cuda())
    gone = Batch(seqs, 4, 2, hd, 32, "bf16", drop=[(0, i, -1) for i in range(low)])
    gone.check_attention(x, q, got=got)
