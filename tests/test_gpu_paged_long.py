"""Attention over the paged cache where one workgroup takes many groups of 32 positions, where a row has many shares of them, and in
fp32 heads wider than 128; against 64 bits, with test_gpu_paged.py's tolerances.

Page numbers are looked up for 64 groups at a time (of a tile, of a wave of the other kernels: 256 groups of its workgroup), and the
statistics of 64 shares: the cases cross those limits, once and several times, with pages missing around them."""
import pytest
import torch

from paper_2504_10724_amd import paged as P
from test_gpu_paged import U, Batch

pytestmark = pytest.mark.gpu


def _attend64(b, x, q, window, scale):
    """test_gpu_paged.py's reference, a sequence at a time: result, sum_j p_j |v_j|, max_j sum_i |q_i k_ji| scale over what a row sees"""
    G = b.hq // b.hkv
    out, size, dots = torch.zeros(b.n, b.hq, b.hd).double(), torch.zeros(b.n, b.hq, b.hd).double(), torch.zeros(b.n, b.hq, 1).double()
    for (n, length), table, at in zip(b.seqs, b.pages, b.start):
        if n == 0:
            continue
        pages = torch.tensor(table)
        there = (pages >= 0) & (pages < b.n_pages)
        p, j = torch.arange(length - n, length)[:, None], torch.arange(length)[None]
        seen = (j <= p) & (j > p - (window or length)) & there.repeat_interleave(b.ps)[None, :length]
        kv = x[:, 0, pages.clamp(0, b.n_pages - 1)].double()           # [2][page][kv head][ps][hd]
        for g in range(b.hkv):
            k, v = kv[0, :, g].reshape(-1, b.hd)[:length], kv[1, :, g].reshape(-1, b.hd)[:length]
            for h in range(g * G, (g + 1) * G):
                qh = q[at:at + n, h].double()
                s = (qh @ k.T * scale).masked_fill(~seen, float("-inf"))
                w = torch.softmax(s, -1).nan_to_num(0.0)               # rows that see nothing
                out[at:at + n, h], size[at:at + n, h] = w @ v, w @ v.abs()
                dots[at:at + n, h, 0] = (qh.abs() @ k.abs().T * scale).masked_fill(~seen, 0.0).amax(-1)
    return out, size, dots


def _check(b, x, q, window=0):
    scale = b.hd ** -0.5
    got = P.attend(b.kv, 1, b.step, q.cuda(), scale=scale, window=window)
    want, size, dots = _attend64(b, x, q, window, scale)
    tol = U * size * (2 * (b.hd + 4) * dots + max(length for _, length in b.seqs) + 64)
    if b.dt == torch.bfloat16:
        tol = tol + 2.0 ** -7 * size
    bad = ~((got.cpu().double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())
    ws = b.kv.workspace(b.step, b.hq).fill_(255)                       # whatever the workspace holds
    assert torch.equal(P.attend(b.kv, 1, b.step, q.cuda(), scale=scale, window=window, workspace=ws), got)
    return got


# from 512 workgroups on nothing is split: the listed sequences stand among 520, the others of which bring no row
WHOLE = [
    # dtype, query heads, kv heads, hd, page, window, (rows, positions)
    ("bf16", 4, 1, 64, 32, 0, [(100, 9001), (1, 17000), (40, 4170), (1, 8193)]),
    ("bf16", 2, 1, 64, 64, 0, [(30, 4231), (1, 8400)]),                # one tile a sequence
    ("bf16", 3, 1, 96, 32, 5000, [(70, 12000), (1, 14001)]),
    ("bf16", 2, 1, 128, 32, 0, [(100, 8321), (1, 16500)]),
    ("bf16", 1, 1, 128, 32, 4300, [(50, 9000), (1, 8200)]),
    ("bf16", 2, 1, 128, 32, 0, [(1, 17000), (1, 8191), (1, 8192)]),    # single rows by themselves
    ("bf16", 2, 1, 192, 32, 0, [(40, 4300), (1, 16500)]),
    ("bf16", 2, 1, 256, 32, 2200, [(20, 6500), (1, 9000)]),
    ("bf16", 2, 1, 256, 64, 0, [(70, 4200), (1, 9000)]),
    ("f32", 2, 1, 64, 32, 0, [(40, 8500), (1, 17000)]),
    ("f32", 1, 1, 36, 32, 9000, [(10, 17000), (1, 8200)]),
    ("f32", 2, 1, 128, 32, 0, [(10, 8300), (1, 16500)]),
    ("f32", 2, 1, 84, 32, 0, [(10, 8300), (1, 9000)]),
    ("f32", 2, 1, 256, 32, 0, [(9, 8300)]),
    ("f32", 2, 1, 200, 32, 0, [(9, 16500)]),
]


def _missing(seqs, ps):
    """pages of the first two sequences around the 64th, 128th and 256th group, some more than one long"""
    drop = []
    for s, (_, length) in enumerate(seqs[:2]):
        for first, last in ((0, 0), (62, 65), (127, 129), (191, 191), (253, 262), (511, 512)):
            for i in range(first * 32 // ps, last * 32 // ps + 1):
                if i < (length + ps - 1) // ps:
                    drop.append((s, i, -1 if i % 2 else 1 << 20))
    return drop


@pytest.mark.parametrize("case", WHOLE, ids=lambda c: "-".join(str(x) for x in c[:6]) + f"-{c[6][0][0]}rows")
@pytest.mark.parametrize("missing", [False, True])
def test_workgroups_of_many_groups(case, missing):
    dtype, hq, hkv, hd, ps, window, seqs = case
    print(f"[case] whole {case} missing {missing}", flush=True)
    b = Batch(seqs + [(0, 0)] * (520 - len(seqs)), hq, hkv, hd, ps, dtype, drop=_missing(seqs, ps) if missing else ())
    x, q = b.fill(), b.queries()
    _check(b, x, q, window)
    assert b.status.item() == (1 if missing else 0)


# a few workgroups split the positions into as many shares as the rules allow
SHARES = [
    ("bf16", 2, 1, 64, 0, [(1, 36000)]),                               # 67 shares of 17 groups
    ("bf16", 4, 2, 128, 0, [(1, 36000)]),
    ("bf16", 2, 1, 256, 0, [(1, 15000)]),                              # 67 of 7
    ("bf16", 2, 1, 128, 0, [(40, 19000)]),                             # a tile: 66 of 9
    ("bf16", 2, 1, 192, 0, [(20, 15000)]),
    ("bf16", 1, 1, 64, 20000, [(1, 36000), (50, 30000)]),
    ("f32", 2, 1, 64, 0, [(1, 10500)]),                                # 66 of 5
    ("f32", 2, 1, 64, 0, [(20, 21000)]),                               # 132 of 5 for two tiles
    ("f32", 2, 1, 84, 0, [(1, 21000)]),
    ("f32", 2, 1, 200, 0, [(3, 10500)]),
    ("f32", 2, 1, 256, 0, [(1, 21000)]),
]


@pytest.mark.parametrize("case", SHARES, ids=lambda c: "-".join(str(x) for x in c[:5]) + f"-{c[5][0][0]}rows")
@pytest.mark.parametrize("missing", [False, True])
def test_rows_of_many_shares(case, missing):
    """with `missing`, whole shares see nothing: the first ones, some in the middle, the last but one"""
    dtype, hq, hkv, hd, window, seqs = case
    print(f"[case] shares {case} missing {missing}", flush=True)
    n = (seqs[0][1] + 31) // 32
    gone = [*range(0, 40), *range(n // 2 - 30, n // 2 + 30), *range(n - 39, n - 2)]
    b = Batch(seqs, hq, hkv, hd, 32, dtype, drop=[(0, i, -1) for i in gone] if missing else ())
    x, q = b.fill(), b.queries()
    _check(b, x, q, window)
    assert b.status.item() == (1 if missing else 0)


@pytest.mark.parametrize("hd", [132, 200, 252])
@pytest.mark.parametrize("window", [0, 45])
def test_fp32_heads_wider_than_128(hd, window):
    for seqs in ([(1, 1), (1, 33), (1, 400)], [(70, 70), (5, 200), (1, 31)], [(40, 1500), (1, 1300)]):
        print(f"[case] fp32 {hd} window {window} {seqs}", flush=True)
        b = Batch(seqs, 6, 2, hd, 32, "f32")
        x, q = b.fill(), b.queries()
        _check(b, x, q, window)
        # what no row sees does not reach one, beyond the last position as before the window
        y = torch.full_like(x, float("nan"))
        for (n, length), table in zip(b.seqs, b.pages):
            for p in range(max(0, length - n + 1 - window) if window else 0, length):
                y[:, 0, table[p // 32], :, p % 32] = x[:, 0, table[p // 32], :, p % 32]
        b.put(y)
        _check(b, x, q, window)
