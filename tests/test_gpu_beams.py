"""The choice of a beam search's next beams against its definition in 64 bits.

Scores: the key is computed in 64 bits from sums whose terms are off by less than 1e-11 of themselves, so that the logarithm is off by
2e-11 at most, and rounded once to fp32: 2^-24 of it.  Parents and tokens have to be equal: the inputs' keys differ by more than
that, or are equal by construction."""
import math

import pytest
import torch

import pages_ref as R
from paper_2504_10724_amd import beams as B
from paper_2504_10724_amd import capi as ee

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _check(got, want):
    score, parent, token, done = want
    assert got.parent.tolist() == parent and got.token.tolist() == token
    want = torch.tensor(score, dtype=torch.float64)
    have = got.score.double().cpu()
    gone = want == -math.inf
    assert (have[gone] == -math.inf).all()
    assert ((have - want).abs()[~gone] <= 2.0 ** -24 * want.abs()[~gone] + 1e-10).all()
    if got.done is not None:
        assert got.done.tolist() == done


def _inputs(groups, beams, vocab, dtype, seed, spread=2.0):
    z = torch.randn(groups * beams, vocab, generator=_gen(seed)) * spread
    return z.to(DT[dtype]), -(torch.randn(groups * beams, generator=_gen(seed + 1)) * 2).abs()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups,beams,vocab,keep", [
    (1, 1, 1, 1), (1, 1, 1, 5), (3, 2, 1, 2), (2, 4, 2048, 4), (1, 5, 32000, 10), (5, 3, 4097, 7), (2, 2, 8193, 128), (1, 64, 333, 128),
    (2, 7, 12289, 64), (3, 1, 4095, 1), (1, 3, 70001, 33), (65, 4, 130, 8), (1, 12, 100, 100), (2, 64, 4200, 64),
    # what one workgroup has at most, and one more
    (2, 1, 16384, 32), (2, 1, 16385, 32), (3, 4, 4096, 32), (3, 4, 4097, 32), (1, 9, 1024, 18), (1, 9, 1025, 18), (2, 64, 1024, 32), (2, 2, 8192, 33),
    (1, 3, 3, 9), (2, 5, 7, 4), (1, 2, 8, 16)])
def test_against_the_definition(groups, beams, vocab, keep, dtype):
    print(f"[case] select {groups} x {beams} of {vocab}, {keep} kept, {dtype}", flush=True)
    z, score = _inputs(groups, beams, vocab, dtype, 7 * vocab + keep)
    _check(B.select(z.cuda(), score.cuda(), beams, keep=keep), R.choose(z, score, beams, keep))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_beams_that_have_ended(dtype):
    print(f"[case] ended {dtype}", flush=True)
    z, score = _inputs(6, 4, 5000, dtype, 3)
    done = (torch.rand(24, generator=_gen(4)) < 0.4).to(torch.uint8)
    done[:4] = 1                                             # a request that is through
    z[done.bool()] = math.nan                                # of an ended beam nothing is read
    z[5, 77] = 30.0                                          # one that ends now
    got = B.select(z.cuda(), score.cuda(), 4, done=done.cuda(), end_token=77)
    want = R.choose(z, score, 4, 4, done, 77)
    _check(got, want)
    assert got.done[0].tolist() == [1, 1, 1, 1] and 1 in want[3][1]
    _check(B.select(z.cuda(), score.cuda(), 4, keep=9, done=done.cuda(), end_token=77), R.choose(z, score, 4, 9, done, 77))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (8, 8)])
def test_rows_at_any_stride_and_alignment(dtype, offset, pad):
    """what lies between the rows is NaN"""
    print(f"[case] strides {dtype} {offset} {pad}", flush=True)
    vocab = 9001
    z, score = _inputs(2, 3, vocab, dtype, 11)
    wide = torch.full((6, offset + vocab + pad), math.nan, dtype=DT[dtype], device="cuda")
    wide[:, offset:offset + vocab] = z.cuda()
    _check(B.select(wide[:, offset:offset + vocab], score.cuda(), 3, keep=6), R.choose(z, score, 3, 6))
    same = wide[:1, offset:offset + vocab].expand(6, vocab)  # one row for all beams
    _check(B.select(same, score.cuda(), 3, keep=6), R.choose(z[:1].expand(6, vocab), score, 3, 6))


@pytest.mark.parametrize("vocab", [6000, 1500])
def test_values_that_are_no_numbers(vocab):
    """masks of -inf and of the type's lowest value, rows that leave nothing, infinities and NaN, scores that are none"""
    print(f"[case] no numbers {vocab}", flush=True)
    last = vocab * 3 // 4
    for dtype in ("f32", "bf16"):
        low = torch.finfo(DT[dtype]).min
        z, score = _inputs(9, 3, vocab, dtype, 21)
        z[0, 1:] = -math.inf                                 # one token left
        z[1] = -math.inf                                     # none
        z[3] = math.nan
        z[4, last] = math.nan
        z[6, 17] = math.inf
        z[9, 10:] = low                                      # ten tokens that matter; the others are candidates
        z[10] = low                                          # all equal
        z[11] = -math.inf
        z[12:15, 3:] = -math.inf                             # nine candidates of a request
        z[15, :last], z[15, last + 1:] = -math.inf, -math.inf          # one token, far behind
        z[18:21] = -math.inf                                 # a request that has no candidate
        score[21], score[22], score[24] = -math.inf, math.nan, math.inf
        score[25] = -3e38
        for keep in (3, 20):
            want = R.choose(z, score, 3, keep)
            assert want[1][6] == [-1] * keep
            _check(B.select(z.cuda(), score.cuda(), 3, keep=keep), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,keep", [(40, 8), (700, 20), (700, 128), (4000, 32), (4000, 1), (20000, 5), (20000, 128)])
def test_equal_candidates_go_by_their_place(dtype, vocab, keep):
    """logits of few values, a row of one value, zeros of both signs, beams that are alike"""
    print(f"[case] ties {dtype} {vocab} {keep}", flush=True)
    z = torch.randint(0, 3, (12, vocab), generator=_gen(5)).to(DT[dtype])
    score = torch.zeros(12)
    z[3] = 1.0
    z[4] = z[5]
    z[6:9] = torch.where(torch.rand(3, vocab, generator=_gen(6)) < 0.5, 0.0, -0.0).to(DT[dtype])
    score[6:9] = torch.tensor([-0.0, 0.0, -0.0])
    z[9:] = 0.0
    _check(B.select(z.cuda(), score.cuda(), 3, keep=keep), R.choose(z, score, 3, keep))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_order_between_beams_is_that_of_64_bits(dtype):
    """two beams with the same distribution, one of them moved by a whole number (the logarithm moves along), at scores that differ in the
    last place of fp32: every candidate of the better one goes before its twin"""
    print(f"[case] order {dtype}", flush=True)
    vocab, keep = 10000, 32
    steps = torch.randint(0, 64, (vocab,), generator=_gen(9)).float()
    z = torch.stack([steps * 0.25, steps * 0.25 + 16.0, steps * 0.25 - 8.0]).to(DT[dtype])
    assert (z[1].float() - z[0].float() == 16.0).all() and (z[2].float() - z[0].float() == -8.0).all()
    score = torch.tensor([-5.0, -5.0 + 2.0 ** -21, -5.0 - 2.0 ** -21])
    got = B.select(z.cuda(), score.cuda(), 3, keep=keep)
    assert got.parent.tolist() == R.choose(z, score, 3, keep)[1]
    best = steps == steps.max()
    assert int(best.sum()) * 3 > keep
    assert got.parent[0].tolist() == sorted(got.parent[0].tolist(), key=[1, 0, 2].index)


def test_results_in_place_and_in_given_buffers():
    print("[case] in place", flush=True)
    z, score = _inputs(4, 5, 3000, "f32", 31)
    done = torch.zeros(20, dtype=torch.uint8)
    done[3] = done[11] = 1
    want = R.choose(z, score, 5, 5, done, 9)
    s, d = score.cuda(), done.cuda()
    out = B.selection(4, 5, done=True)._replace(score=s.view(4, 5), done=d.view(4, 5))
    ws = B.workspace(4, 5, 3000, 5)
    ws.fill_(255)
    assert B.select(z.cuda(), s, 5, done=d, end_token=9, out=out, workspace=ws) is out
    _check(out, want)


def test_many_steps_are_the_same_every_time():
    print("[case] repeated", flush=True)
    z, score = _inputs(16, 8, 20011, "bf16", 41)
    z, score = z.cuda(), score.cuda()
    first = B.select(z, score, 8, keep=16)
    for _ in range(5):
        again = B.select(z, score, 8, keep=16)
        assert all(torch.equal(a, b) for a, b in zip(first[:3], again[:3]))


def test_rows_beyond_32_bits_of_elements():
    """the last rows of logits of more than 2^31 values"""
    print("[case] large", flush=True)
    vocab, rows = 131072, 17000
    z = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    score = -torch.rand(rows, device="cuda")
    got = B.select(z, score, 4)
    assert z.numel() > 2 ** 31
    for g in (0, 2100, rows // 4 - 1):
        at = slice(4 * g, 4 * g + 4)
        _check(B.Selection(*(x[g:g + 1] for x in got[:3]), None), R.choose(z[at].cpu(), score[at].cpu(), 4, 4))


def test_no_requests():
    print("[case] none", flush=True)
    got = B.select(torch.empty(0, 50, device="cuda"), torch.empty(0, device="cuda"), 4)
    assert got.score.shape == (0, 4)


def test_refusals():
    print("[case] refusals", flush=True)
    z, score = torch.zeros(8, 100, device="cuda"), torch.zeros(8, device="cuda")
    done = torch.zeros(8, dtype=torch.uint8, device="cuda")
    ws = B.workspace(2, 4, 100, 4)
    bad = [lambda: B.select(z, score, 3), lambda: B.select(z, score, 0), lambda: B.select(z, score, -4), lambda: B.select(z[0], score, 4),
           lambda: B.select(z.half(), score, 4), lambda: B.select(z.double(), score, 4), lambda: B.select(z.t(), score, 4),
           lambda: B.select(z, score.double(), 4), lambda: B.select(z, score[:4], 4), lambda: B.select(z, score.cpu(), 4),
           lambda: B.select(z.cpu(), score.cpu(), 4), lambda: B.select(z, torch.zeros(16, device="cuda")[::2], 4),
           lambda: B.select(z, score, 4, keep=0), lambda: B.select(z, score, 4, keep=129), lambda: B.select(z, score, 4, keep=2 ** 32 + 1),
           lambda: B.select(z, score, 4, end_token=100), lambda: B.select(z, score, 4, end_token=-2), lambda: B.select(z, score, 4, done=done),
           lambda: B.select(z, score, 4, done=done.bool(), end_token=1), lambda: B.select(z, score, 4, done=done.cpu(), end_token=1),
           lambda: B.select(z[:, :0], score, 4), lambda: B.select(z, score, 4, out=B.selection(2, 5)),
           lambda: B.select(z, score, 4, keep=2, out=B.selection(2, 2)._replace(score=score[:4].view(2, 2))),
           lambda: B.select(z, score, 4, workspace=ws[:-256]), lambda: B.select(z, score, 4, workspace=ws.cpu()),
           lambda: B.select(z, score, 4, workspace=torch.empty(ws.numel() + 16, dtype=torch.uint8, device="cuda")[16:]),
           lambda: B.select(z.clone().requires_grad_(), score, 4), lambda: B.workspace(2 ** 33, 4, 100, 4)]
    for i, call in enumerate(bad):
        with pytest.raises(ee.EEError):
            print(f"[refusal] {i}", flush=True)
            call()
    with torch.no_grad():
        B.select(z.clone().requires_grad_(), score, 4, workspace=ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("groups,beams,vocab", [(600, 2, 3), (1025, 1, 1), (300, 4, 7), (270, 4, 8), (70, 16, 50)])
def test_many_rows_of_few_tokens(groups, beams, vocab, dtype):
    z, score = _inputs(groups, beams, vocab, dtype, vocab)
    _check(B.select(z.cuda(), score.cuda(), beams), R.choose(z, score, beams, beams))


def test_rows_that_are_one():
    """a stride of 0: all beams have the same logits, and their candidates differ by the scores alone"""
    z, score = _inputs(1, 1, 5000, "f32", 11)
    score = torch.tensor([-1.0, -0.5, -0.5, -3.0])
    _check(B.select(z.cuda().expand(4, 5000), score.cuda(), 4, keep=20), R.choose(z.expand(4, 5000), score, 4, 20))


def _choose_by_logits(logits, score, n_beams, keep, done=None, end=-1):
    """(parents, tokens): keys in 64 bits, and where they are equal the smaller beam, in a beam the larger logit, then the smaller token"""
    out = [], []
    for g in range(len(logits) // n_beams):
        found = []
        for b in range(n_beams):
            s, z = float(score[g * n_beams + b]), logits[g * n_beams + b].double()
            if not math.isfinite(s):
                continue
            if done is not None and done[g * n_beams + b]:
                found.append((-s, b, 0.0, end))
                continue
            top, log = float(z.max()), math.log(float(torch.exp(z - z.max()).sum()))
            found += [(-(s - log + (v - top)), b, -v, t) for t, v in enumerate(z.tolist())]
        found = sorted(found)[:keep]
        out[0].append([f[1] for f in found] + [-1] * (keep - len(found)))
        out[1].append([f[3] for f in found] + [-1] * (keep - len(found)))
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,keep", [(8192, 4), (8192, 40), (8192, 128), (300, 5), (300, 128), (4097, 9)])
def test_a_beam_whose_score_swallows_its_logits(vocab, keep, dtype):
    """its candidates' keys are all equal in 64 bits, and it goes on with its largest logits, alone as in a batch, whose slices are wider"""
    print(f"[case] swallowed {dtype} {vocab} {keep}", flush=True)
    z, _ = _inputs(1, 4, vocab, dtype, vocab + keep)
    score = torch.tensor([-math.inf, -3e38, math.nan, -math.inf])
    want = torch.sort(z[1].double(), descending=True, stable=True).indices[:keep].tolist()
    for groups in (1, 1200):
        got = B.select(z.repeat(groups, 1).cuda(), score.repeat(groups).cuda(), 4, keep=keep)
        at = torch.tensor([0, groups // 2, groups - 1], device="cuda")
        assert got.token[at].tolist() == [want] * 3 and got.parent[at].tolist() == [[1] * keep] * 3
        assert (got.score == score[1].cuda()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,keep", [(20, 50), (700, 128), (5000, 20), (20000, 128)])
def test_logits_that_differ_by_less_than_keys_can(vocab, keep, dtype):
    """of 1e-30 and less, zeros of both signs among them: every sum is the vocabulary's size, two beams tie, one is ahead, one has ended"""
    print(f"[case] tiny logits {dtype} {vocab} {keep}", flush=True)
    z = (torch.randn(8, vocab, generator=_gen(vocab)) * 1e-30).to(DT[dtype])
    z[:, ::7], z[:, 3::7] = 0.0, -0.0
    score = torch.tensor([-5.0, -5.0, -4.5, -9.0, -math.inf, -2.0, -2.0, -2.0])
    done = torch.tensor([0, 0, 0, 1, 0, 0, 0, 0], dtype=torch.uint8)
    got = B.select(z.cuda(), score.cuda(), 4, keep=keep, done=done.cuda(), end_token=7)
    parent, token = _choose_by_logits(z, score, 4, keep, done, 7)
    assert got.parent.tolist() == parent and got.token.tolist() == token


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [9, 3000])
def test_a_chosen_candidate_has_a_finite_score(vocab, dtype):
    """a mask of the type's lowest value taken twice: the key is beyond fp32, the score is fp32's lowest finite number, and the beam goes on"""
    print(f"[case] finite scores {dtype} {vocab}", flush=True)
    low, lowest = torch.finfo(DT[dtype]).min, -torch.finfo(torch.float32).max
    z = torch.zeros(4, vocab, dtype=DT[dtype])
    z[:, 1:] = low                                           # one token is allowed
    score = torch.tensor([0.0, -math.inf, -math.inf, -math.inf])
    for aside, want_score in ((1, [0.0, low, low, low]), (3, [low, low, low, lowest]), (0, [lowest] * 4)):
        got = B.select(z.cuda(), score.cuda(), 4)
        parent, token = _choose_by_logits(z, score, 4, 4)
        assert min(parent[0]) >= 0 and got.parent.tolist() == parent and got.token.tolist() == token
        assert got.score[0].tolist() == want_score
        score = got.score[0].cpu()
        score[:aside] = -math.inf                            # the better ones are put aside
    none = B.select(z[:, :1].cuda(), score.cuda(), 4, keep=6)              # places that no candidate is left for
    assert none.score[0].tolist() == [lowest] * 4 + [-math.inf] * 2 and none.parent[0].tolist() == [0, 1, 2, 3, -1, -1]


def test_tangents_are_not_lost():
    """tensors of forward-mode derivatives, which no call computes, under no_grad too"""
    print("[case] tangents", flush=True)
    from torch.autograd import forward_ad
    z, score = torch.zeros(8, 100, device="cuda"), torch.zeros(8, device="cuda")
    with forward_ad.dual_level():
        for call in (lambda: B.select(forward_ad.make_dual(z, torch.ones_like(z)), score, 4),
                     lambda: B.select(z, forward_ad.make_dual(score, torch.ones_like(score)), 4)):
            with pytest.raises(ee.EEError, match="gradient"):
                call()
            with torch.no_grad(), pytest.raises(ee.EEError, match="gradient"):
                call()
        dual = forward_ad.make_dual(z, torch.ones_like(z))
        B.select(dual.detach(), score, 4)
        B.select(z, score, 4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("keep", [1, 20, 128])
@pytest.mark.parametrize("values", ["normal", "equal", "scores"])
def test_more_lists_than_are_collected(values, keep, dtype):
    """640 slices of one request: all of them in the running, or those of some beams; some beams have ended"""
    print(f"[case] many lists {values} {keep} {dtype}", flush=True)
    beams, vocab = 64, 40000
    z, score = _inputs(1, beams, vocab, dtype, keep)
    done = (torch.arange(beams) % 9 == 5).to(torch.uint8)
    if values != "normal":
        z.zero_()
    if values == "equal":
        score = torch.full((beams,), -3.0)
        score[done.bool()] = -3.0 - 20.0                     # behind all others
    want = R.choose(z, score, beams, keep, done, 11)
    _check(B.select(z.cuda(), score.cuda(), beams, keep=keep, done=done.cuda(), end_token=11), want)
