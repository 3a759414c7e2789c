"""A beam search on the paged cache as a program runs it: choice, forks and growth together, eager and recorded into a graph."""
import importlib.util
import os

import pytest
import torch

import pages_ref as R
from paper_2504_10724_amd import beams as B
from paper_2504_10724_amd import paged as P

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "beam_search.py")


def _example():
    spec = importlib.util.spec_from_file_location("beam_search", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


@pytest.mark.parametrize("beams,requests", [(4, 3), (1, 2), (6, 5)])
def test_scores_agree_with_those_without_a_cache(beams, requests):
    print(f"[case] example, {requests} requests of {beams}", flush=True)
    # per block: probabilities, attention output, projection and residual each rounded to bf16 (2^-8), on both sides, two blocks; the logits of
    # such states are off by as much of theirs, and the tokens' log-probabilities, of 1.5 and more, by less than the logits' rms (3) of that
    assert _example().main(["--beams", str(beams), "--requests", str(requests)]) <= 16 * 2.0 ** -8


def _search(e, beams, weights, rope):
    gen = torch.Generator(device="cuda").manual_seed(5)
    return e.Search([torch.randint(8, e.VOCAB, (n,), generator=gen, device="cuda") for n in (31, 70, 5)], beams, 40, weights, rope)


def test_a_recorded_step_does_what_the_calls_do():
    """every replay, with other work and waits between, against the same search step by step; then the pages of all beams are given back"""
    print("[case] graph", flush=True)
    e = _example()
    weights, rope = e.make_weights(2, torch.Generator(device="cuda").manual_seed(2)), P.Rope(e.HD, 256)
    eager, recorded = (_search(e, 5, weights, rope) for _ in range(2))
    eager.advance()
    recorded.advance()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded.advance()
    for i in range(37):
        graph.replay()
        if i % 3 == 0:
            torch.cuda.synchronize()
            torch.randn(1 << 20, device="cuda").sum()
        eager.advance()
        for name, a, b in (("tokens", eager.tokens, recorded.tokens), ("scores", eager.score, recorded.score), ("done", eager.done, recorded.done),
                           ("pages", eager.table.pages, recorded.table.pages), ("lengths", eager.table.kv_len, recorded.table.kv_len),
                           ("refs", eager.pages.refs, recorded.pages.refs)):
            assert torch.equal(a, b), (i, name)
    assert int(eager.status.item()) == 0 and int(recorded.status.item()) == 0
    entries = torch.bincount(recorded.table.pages[recorded.table.pages >= 0], minlength=recorded.cache.cfg.n_pages)
    assert torch.equal(entries.int(), recorded.pages.refs)
    recorded.pages.fork(recorded.table, torch.full_like(recorded.table.kv_len, -1))
    assert not recorded.pages.refs.any() and not recorded.table.kv_len.any() and (recorded.table.pages == -1).all()


def test_two_searches_at_once():
    """on streams of their own, each with its own cache and workspace"""
    print("[case] two searches", flush=True)
    e = _example()
    weights, rope = e.make_weights(2, torch.Generator(device="cuda").manual_seed(2)), P.Rope(e.HD, 256)
    alone, *both = (_search(e, 4, weights, rope) for _ in range(3))
    for _ in range(12):
        alone.advance()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for _ in range(12):
        for s, stream in zip(both, streams):
            with torch.cuda.stream(stream):
                s.advance()
    torch.cuda.synchronize()
    for s in both:
        assert torch.equal(s.tokens, alone.tokens) and torch.equal(s.score, alone.score) and torch.equal(s.table.pages, alone.table.pages)


def test_chosen_beams_and_their_pages():
    """choices with ended beams and requests without a candidate, whose rows become empty; every step against lists"""
    print("[case] choices and pages", flush=True)
    groups, beams, vocab, page = 5, 3, 50, 32
    n = groups * beams
    kv = P.PagedCache(2, 90, 1, 64, page, "bf16")
    kv.pool.copy_(torch.randint(-128, 128, kv.pool.shape, device="cuda"))
    pages, table = P.Pages(kv, n), P.PageTable(kv, n, 6)
    book = R.Book(90, page, kv.pool.cpu().view(2, 90, 1, 1, 1, -1))
    t = book.table(n, 6)
    gen = torch.Generator().manual_seed(3)
    new = [30 if i % beams == 0 else 0 for i in range(n)]
    score, done = torch.where(torch.arange(n) % beams == 0, 0.0, -torch.inf), torch.zeros(n, dtype=torch.uint8)
    history = torch.randint(0, 99, (n, 7), generator=gen, dtype=torch.int32)
    s, d, h = score.cuda(), done.cuda(), history.cuda()
    pages.grow(table, torch.tensor(new, dtype=torch.int32, device="cuda"))
    book.grow(t, new)
    out = B.selection(groups, beams, done=True)._replace(score=s.view(groups, beams), done=d.view(groups, beams))
    for step in range(40):
        z = torch.randn(n, vocab, generator=gen) * 2
        if step == 20:
            z[3:6] = -torch.inf                              # a request that ends here
        got = B.select(z.cuda(), s, beams, done=d, end_token=4, out=out)
        want = R.choose(z, score, beams, beams, done, 4)
        assert got.parent.tolist() == want[1] and got.token.tolist() == want[2] and got.done.tolist() == want[3], step
        score, done = got.score.flatten().cpu(), got.done.flatten().cpu()      # the rounded scores
        parent = [p for g in want[1] for p in g]
        pages.fork(table, got.parent.view(-1), group=beams, rows=[h])
        book.fork(t, parent, group=beams, rows=[history])
        grow = [0 if p < 0 or bool(e) else 1 for p, e in zip(parent, done)]
        pages.grow(table, torch.tensor(grow, dtype=torch.int32, device="cuda"))
        book.grow(t, grow)
        assert table.kv_len.tolist() == t.len and table.pages.tolist() == t.entries() and pages.refs.tolist() == book.refs(), step
        assert torch.equal(h.cpu(), history) and torch.equal(kv.pool.cpu(), book.pool.reshape(-1)), step
    assert t.len[3:6] == [0, 0, 0]
