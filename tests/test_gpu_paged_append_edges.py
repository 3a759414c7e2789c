"""The append to the paged cache where rows run past the rotary table, and calls that move more than the caches hold."""
import pytest
import torch

import paged_ref as R
from paper_2504_10724_amd import paged as P
from test_gpu_paged import U, Batch, _append_reference, _randn, _strided

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("odd", [False, True])
def test_rows_that_all_lie_past_the_rotary_table(dtype, odd):
    """a group of 32 positions whose new rows are all at the table's end or beyond it: nothing of them is written, the others are"""
    max_pos = 100
    for seqs in ([(1, 101), (1, 100), (1, 30)],                        # single rows: at max_pos, the last inside, well inside
                 [(1, 170), (1, 129)],                                 # nothing inside
                 [(4, 104), (40, 140), (33, 129), (7, 99)],            # whole chunks beyond, chunks that cross the end
                 [(60, 228), (2, 102)]):
        print(f"[case] append past the table {dtype} odd {odd} {seqs}", flush=True)
        b = Batch(seqs, 4, 2, 64, 32, dtype)
        x = b.fill()
        rows = _randn((b.n, 8, 64), b.dt, 21)
        q, k, v = rows[:, :4], rows[:, 4:6], rows[:, 6:]
        pads = (1, 3, 1) if odd else (0, 0, 0)
        q_out = torch.full((b.n, 4, 64), 9.0, dtype=b.dt, device="cuda")
        P.append(b.kv, 1, b.step, _strided(k, *pads), _strided(v, *pads), rope=P.Rope(64, max_pos), q=_strided(q, *pads), q_out=q_out)
        want, wrote = _append_reference(b, x, k, v, dict(rot=64), max_pos, 1)
        got = b.get()
        assert torch.equal(got[~wrote], x[~wrote])
        assert torch.equal(got[1], want[1].to(b.dt))
        near = 2.0 ** -8 if dtype == "bf16" else 0.0
        assert ((got[0].double() - want[0]).abs() <= near * want[0].abs() + 8 * U * 8).all()
        pos = torch.tensor([length - n + j for n, length in seqs for j in range(n)])
        inside = pos < max_pos
        wq = R.rotate(q[inside], pos[inside], 64)
        assert ((q_out.cpu()[inside].double() - wq).abs() <= near * wq.abs() + 8 * U * 8).all()
        assert (q_out.cpu()[~inside] == 9.0).all()
        assert b.status.item() == 1
