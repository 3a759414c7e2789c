"""Numerics of the attention over the paged cache that test_gpu_paged.py's tolerances do not tell apart, against 64 bits.

fp32 terms as there: e = U A (2 (hd + 4) D + n + 64), with A = sum_j p_j |v_j| and D = max_j sum_i |q_i k_ji| scale.  A bf16 result
carries one rounding of 2^-8 of the value."""
import pytest
import torch

import paged_ref as R
from paper_2504_10724_amd import paged as P
from test_gpu_paged import U, Batch

pytestmark = pytest.mark.gpu

SINGLES = [
    # hd, query heads, kv heads, window, (rows, positions) of each sequence
    (64, 6, 2, 0, [(1, 95), (1, 500), (1, 1)]),
    (96, 8, 1, 0, [(1, 700), (1, 33)]),
    (128, 8, 2, 0, [(1, 64), (1, 257), (1, 1000)]),
    (128, 8, 2, 37, [(1, 90), (1, 300)]),
    (128, 4, 2, 0, [(4, 300), (4, 70)]),                               # four rows of two heads: eight columns
    (128, 8, 2, 0, [(70, 300), (1, 200), (1, 611)]),                   # beside a chunk, in its launch
    (192, 4, 2, 0, [(1, 400), (17, 30), (1, 900)]),                    # beside a chunk, in a launch of their own
    (256, 4, 2, 0, [(1, 130), (1, 800)]),                              # in shares
]


@pytest.mark.parametrize("case", SINGLES, ids=lambda c: "-".join(str(x) for x in c[:4]) + f"-{len(c[4])}seqs")
def test_few_columns_keep_the_probabilities_bits(case):
    """sequences of up to 16 columns: a probability enters the second product as a pair of bf16, 2^-8 x 2^-8 of it off at most, so
    all that a result has lost beside fp32's terms is its own rounding"""
    hd, hq, hkv, window, seqs = case
    print(f"[case] precision {case}", flush=True)
    b = Batch(seqs, hq, hkv, hd, 64, "bf16")
    x, q = b.fill(), b.queries()
    got = P.attend(b.kv, 1, b.step, q.cuda(), window=window).cpu().double()
    want, size, dots = R.attend(q, x[:, 0], b.seqs, b.pages, window, hd ** -0.5)
    e = size * (2.0 ** -16 + U * (2 * (hd + 4) * dots + max(length for _, length in seqs) + 64))
    for (n, _), at in zip(seqs, b.start):
        if n * (hq // hkv) <= 16:
            rows = slice(at, at + n)
            err = (got[rows] - want[rows]).abs()
            tol = 2.0 ** -8 * (want[rows].abs() + e[rows]) + e[rows]
            assert (err <= tol).all(), (n, float((err / tol).max()))


@pytest.mark.parametrize("at", [50, 178])                              # in the second group, in the second of one of four waves
@pytest.mark.parametrize("dtype,rows", [("bf16", 1), ("bf16", 8), ("bf16", 100), ("f32", 1), ("f32", 40)])
def test_large_values_average_whatever_the_order_of_the_scores(dtype, rows, at):
    """the average of equal finite values is that value, also where a later score is a hundred times as likely as the first ones"""
    print(f"[case] large values {dtype} {rows} rows, {at}", flush=True)
    b = Batch([(rows, rows + 200), (rows, rows + 189)], 4, 2, 64, 32, dtype)
    x, q = torch.zeros(2, 1, b.n_pages, 2, 32, 64, dtype=b.dt), torch.zeros(b.n, 4, 64, dtype=b.dt)
    x[1] = 4e36
    q[..., 0] = 1.0
    for table in b.pages:
        x[0, 0, table[at // 32], :, at % 32, 0] = 4.84                 # 2^6.98 times the weight of a score of zero
    b.put(x)
    got = P.attend(b.kv, 1, b.step, q.cuda(), scale=1.0).cpu().double()
    value = float(x[1, 0, 0, 0, 0, 0])
    # weights add up to one within 300 roundings each; the probabilities' and the result's rounding in bf16
    assert ((got - value).abs() <= value * (600 * U + (2.0 ** -7 if dtype == "bf16" else 0.0))).all(), got.flatten()[:4]


@pytest.mark.parametrize("dtype,rows", [("bf16", 1), ("bf16", 100), ("f32", 1), ("f32", 40)])
def test_a_scale_of_zero_does_not_hide_what_the_queries_hold(dtype, rows):
    """0 x NaN and 0 x inf are NaN: so are the row's weights"""
    print(f"[case] scale zero {dtype} {rows} rows", flush=True)
    b = Batch([(rows, 150), (rows, rows)], 4, 2, 64, 32, dtype)
    x, q = b.fill(), b.queries()
    ref = b.check_attention(x, q, scale=0.0)
    for value in (float("nan"), float("inf")):
        y = q.clone()
        y[0, 1, 3] = value
        got = P.attend(b.kv, 1, b.step, y.cuda(), scale=0.0)
        assert got[0, 1].isnan().all()
        keep = torch.ones(b.n, 4, dtype=torch.bool)
        keep[0, 1] = False
        assert torch.equal(got[keep.cuda()], ref[keep.cuda()])


@pytest.mark.parametrize("rows,n_seqs", [(1, 64), (40, 3)])
def test_fp32_weights_of_scores_close_together(rows, n_seqs):
    """Values are rows of the identity, so that a result is the row's weights.  Scores of one product, at most 0.07 in log2 units: an
    exponent is off by a few hundredths of a rounding, the hardware's 2^x and 1/x by one unit in the last place each (2 U; as a random
    rounding 2 U / sqrt 3), the sum of 64 weights by its seven levels of U / sqrt 3 at most, the last product by one: root mean square
    sqrt(2 * 4/3 + 8/3) U = 2.31 U.  An exponent that was rounded at a size of 8 would add 2^-21 ln 2 / sqrt 3 = 3.2 U."""
    print(f"[case] close scores {rows} rows", flush=True)
    b = Batch([(rows, 64)] * n_seqs, 4, 2, 64, 32, "f32")
    x, q = torch.zeros(2, 1, b.n_pages, 2, 32, 64), torch.zeros(b.n, 4, 64)
    gen = torch.Generator().manual_seed(7)
    q[..., 0] = torch.rand(b.n, 4, generator=gen) * 0.2 - 0.1
    for table in b.pages:
        for i, page in enumerate(table):
            x[0, 0, page, :, :, 0] = torch.rand(2, 32, generator=gen) - 0.5
            x[1, 0, page] = torch.eye(64)[32 * i:32 * i + 32]
    b.put(x)
    got = P.attend(b.kv, 1, b.step, q.cuda(), scale=1.0).cpu().double()
    want, _, _ = R.attend(q, x[:, 0], b.seqs, b.pages, 0, 1.0)
    seen = want > 0
    assert (got[~seen] == 0).all()
    off = (got[seen] / want[seen] - 1).square().mean().sqrt()
    assert off <= 2.31 * U, float(off / U)
