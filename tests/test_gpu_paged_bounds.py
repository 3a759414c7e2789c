"""What the paged cache's calls may touch: their workspace and no byte beside it, and of a batch in which some sequences lie outside the
host's figures, the others' places and rows."""
import pytest
import torch

import paged_ref as R
from paper_2504_10724_amd import capi as ee
from paper_2504_10724_amd import paged as P
from test_gpu_paged import U, Batch, _i32, _randn

pytestmark = pytest.mark.gpu

WORKSPACES = [
    # dtype, query heads, kv heads, hd, (rows, positions)
    ("bf16", 4, 2, 64, [(1, 3000), (1, 2500)]),
    ("bf16", 20, 1, 128, [(9, 2000), (1, 1700)]),
    ("bf16", 4, 2, 128, [(90, 2000), (1, 1900)]),
    ("bf16", 4, 1, 256, [(40, 1200), (1, 1500)]),
    ("bf16", 4, 1, 192, [(1, 1200)] * 7),
    ("f32", 4, 2, 64, [(40, 1500), (1, 900)]),
    ("f32", 4, 2, 84, [(1, 2000)]),
    ("f32", 2, 1, 256, [(7, 1000)]),
]


@pytest.mark.parametrize("case", WORKSPACES, ids=lambda c: "-".join(str(x) for x in c[:4]) + f"-{c[4][0][0]}rows")
def test_a_call_stays_inside_its_workspace(case):
    dtype, hq, hkv, hd, seqs = case
    print(f"[case] workspace {case}", flush=True)
    b = Batch(seqs, hq, hkv, hd, 32, dtype)
    x, q = b.fill(), b.queries()
    need = ee.load().ee_paged_attention_workspace(b.kv.h, hq, b.step.ref)
    assert need > 0
    memory = torch.full((need + 8192,), 171, dtype=torch.uint8, device="cuda")
    got = P.attend(b.kv, 1, b.step, q.cuda(), workspace=memory[4096:4096 + need])
    b.check_attention(x, q, got=got)
    assert (memory[:4096] == 171).all() and (memory[4096 + need:] == 171).all() and not (memory[4096:4096 + need] == 171).all()
    with pytest.raises(ee.EEError):
        P.attend(b.kv, 1, b.step, q.cuda(), workspace=memory[4096:4095 + need])
    with pytest.raises(ee.EEError):
        P.attend(b.kv, 1, b.step, q.cuda(), workspace=memory[128:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 20])                                 # rows of a few and of many columns
def test_sequences_outside_the_figures_keep_to_themselves(dtype, m):
    """refused sequences: status bit 2 of either call, nothing of theirs written; the others: as if they were alone"""
    seqs, hd, scale = [(3 * m, 100), (2 * m, 150), (4 * m, 80)], 64, 0.125
    b = Batch(seqs, 4, 2, hd, 32, dtype)
    x, q = b.fill(), b.queries()
    k, v = _randn((b.n, 2, hd), b.dt, 91), _randn((b.n, 2, hd), b.dt, 92)
    for start, length, refused in (([0, 3, 5, 9], [100, 161, 80], {1}),              # more positions than the host's figure
                                   ([0, 3, 8, 9], [100, 150, 80], {1}),              # more rows
                                   ([0, 3, 5, 10], [100, 150, 80], {2}),             # rows past the end of the call
                                   ([0, 3, 5, 9], [-1, 150, 80], {0}),
                                   ([0, 3, 3, 9], [100, 150, 80], {2})):             # one without rows, then too many
        start = [m * a for a in start]
        print(f"[case] figures {dtype} {m} {start} {length}", flush=True)
        step = P.PagedStep(_i32(start).cuda(), _i32(length).cuda(), b.step.tensors[2], n_tokens=9 * m, max_q_len=4 * m, max_kv_len=160, status=b.status)
        served = [(s, start[s], start[s + 1], length[s]) for s in range(3) if s not in refused]
        b.put(x)
        b.status.zero_()
        out = torch.full((9 * m, 4, hd), 9.0, dtype=b.dt, device="cuda")
        P.attend(b.kv, 1, step, q.cuda(), out=out)
        assert b.status.item() == 2
        mine = torch.zeros(9 * m, dtype=torch.bool)
        for s, a, e, n in served:
            want, size, dots = R.attend(q[a:e], x[:, 0], [(e - a, n)], [b.pages[s]], 0, scale)
            tol = U * size * (2 * (hd + 4) * dots + n + 64) + (2.0 ** -7 * size if dtype == "bf16" else 0.0)
            assert ((out[a:e].cpu().double() - want).abs() <= tol).all()
            mine[a:e] = True
        assert (out[~mine.cuda()] == 9.0).all()
        b.status.zero_()
        P.append(b.kv, 1, step, k.cuda(), v.cuda())
        assert b.status.item() == 2
        want = x.clone()
        for s, a, e, n in served:
            for i in range(a, e):
                p = n - (e - i)
                want[0, 0, b.pages[s][p // 32], :, p % 32], want[1, 0, b.pages[s][p // 32], :, p % 32] = k[i], v[i]
        assert torch.equal(b.get(), want)
