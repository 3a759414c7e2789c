"""Beam search on the paged cache without the host in the loop: each step's choice, the pages that the chosen beams share, copy or give back,
and the next step's attention all stay on the device, so that the step is recorded once into a graph and replayed.

Per step: `paged.append` and `paged.attend` (per layer), a projection onto the vocabulary, `beams.select`, `Pages.fork` (each row becomes a
child of the row that was chosen; its tokens go with it) and `Pages.grow` (room for the next position; a page that other beams hold
too is copied).  The model is random-weight attention blocks in plain torch.  At the end every beam is scored once more without a cache.

    python examples/beam_search.py [--requests 3] [--beams 4] [--new 24]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2504_10724_amd import beams, paged  # noqa: E402

HQ, HKV, HD, PAGE, D, VOCAB, END = 8, 2, 128, 32, 512, 1000, 7


def make_weights(layers, gen):
    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * shape[0] ** -0.5 * scale).to(torch.bfloat16)
    blocks = [dict(qkv=normal(D, (HQ + 2 * HKV) * HD), out=normal(HQ * HD, D)) for _ in range(layers)]
    return dict(blocks=blocks, embed=torch.randn(VOCAB, D, generator=gen, device="cuda").to(torch.bfloat16), head=normal(D, VOCAB, scale=3.0))


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5)).to(torch.bfloat16)


def project(x, w):
    y = (norm(x) @ w["qkv"]).view(len(x), HQ + 2 * HKV, HD)
    return y[:, :HQ], y[:, HQ:HQ + HKV], y[:, HQ + HKV:]


class Search:
    """requests of n_beams beams each; row r * n_beams + b of every array is beam b of request r"""

    def __init__(self, prompts, n_beams, new, weights, rope):
        n, longest = len(prompts) * n_beams, max(len(p) for p in prompts) + new
        self.prompts, self.n_beams, self.w, self.rope = prompts, n_beams, weights, rope
        width = (longest + PAGE - 1) // PAGE
        self.cache = paged.PagedCache(len(weights["blocks"]), n * (width + 1), HKV, HD, PAGE, "bf16")
        self.pages, self.table = paged.Pages(self.cache, n), paged.PageTable(self.cache, n, width)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")       # noqa: E731
        self.status = i32([0])
        # the beams of a request start as one: the others are there from the first choice on
        self.score = torch.where(torch.arange(n, device="cuda") % n_beams == 0, 0.0, -torch.inf)
        self.done = torch.zeros(n, dtype=torch.uint8, device="cuda")
        self.tokens = torch.full((n, new), -1, dtype=torch.int32, device="cuda")
        self.chosen = beams.selection(len(prompts), n_beams, done=True)._replace(score=self.score.view(-1, n_beams), done=self.done.view(-1, n_beams))
        self.column = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.room = beams.workspace(len(prompts), n_beams, VOCAB, n_beams)
        starts = i32(list(range(n + 1)))
        self.step = paged.PagedStep(starts, self.table.kv_len, self.table.pages, n_tokens=n, max_q_len=1, max_kv_len=longest, status=self.status)
        self.attention_room = self.cache.workspace(self.step, HQ)
        self.prefill(i32)

    def blocks(self, x, step, workspace=None):
        for layer, w in enumerate(self.w["blocks"], 1):
            q, k, v = project(x, w)
            q = paged.append(self.cache, layer, step, k, v, rope=self.rope, q=q)
            x = x + paged.attend(self.cache, layer, step, q, workspace=workspace).reshape(len(x), -1) @ w["out"]
        return x

    def prefill(self, i32):
        """the prompts into the first beam's pages, which the other beams share from then on"""
        b, lengths = self.n_beams, [len(p) for p in self.prompts]
        self.pages.grow(self.table, i32([lengths[i // b] if i % b == 0 else 0 for i in range(len(lengths) * b)]), status=self.status)
        starts = [0]
        for i in range(len(lengths) * b):
            starts.append(starts[-1] + (lengths[i // b] if i % b == 0 else 0))
        step = paged.PagedStep(i32(starts), self.table.kv_len, self.table.pages, n_tokens=starts[-1], max_q_len=max(lengths), max_kv_len=max(lengths),
                               status=self.status)
        x = self.blocks(torch.cat([self.w["embed"][p] for p in self.prompts]), step)
        ends = torch.tensor(starts, device="cuda")[b::b] - 1
        self.choose(x[ends].repeat_interleave(b, 0))
        self.pages.grow(self.table, status=self.status)

    def choose(self, x):
        logits = norm(x) @ self.w["head"]
        beams.select(logits, self.score, self.n_beams, done=self.done, end_token=END, out=self.chosen, workspace=self.room)
        self.pages.fork(self.table, self.chosen.parent.view(-1), group=self.n_beams, rows=[self.tokens], status=self.status)
        self.tokens.index_copy_(1, self.column, self.chosen.token.view(-1, 1))
        self.column += 1

    def advance(self):
        """one token for every beam"""
        self.choose(self.blocks(self.w["embed"][self.chosen.token.view(-1).clamp(min=0).long()], self.step, self.attention_room))
        self.pages.grow(self.table, status=self.status)


def rescore(prompt, tokens, weights, rope):
    """sum of the tokens' log-probabilities up to the end token, over the whole sequence at once and without a cache"""
    cut = (tokens == END).nonzero()
    tokens = tokens[:int(cut[0]) + 1] if len(cut) else tokens
    x = weights["embed"][torch.cat([prompt, tokens[:-1].long()])]
    pos = torch.arange(len(x), dtype=torch.int32, device="cuda")
    hide = torch.triu(torch.ones(len(x), len(x), dtype=torch.bool, device="cuda"), 1)
    for w in weights["blocks"]:
        q, k, v = project(x, w)
        q, k = rope.apply(q, pos).float(), rope.apply(k, pos).float()
        k, v = (t.float().repeat_interleave(HQ // HKV, 1).transpose(0, 1).contiguous() for t in (k, v))
        s = torch.matmul(q.transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) * HD ** -0.5
        o = torch.matmul(torch.softmax(s.masked_fill(hide, float("-inf")), -1), v).transpose(0, 1)
        x = x + o.reshape(len(x), -1).to(torch.bfloat16) @ w["out"]
    p = torch.log_softmax((norm(x[len(prompt) - 1:]) @ weights["head"]).double(), -1)
    return float(p.gather(1, tokens.long()[:, None]).sum())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=3)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--new", type=int, default=24)
    a = ap.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(1)
    weights = make_weights(a.layers, gen)
    rope = paged.Rope(HD, 1024)
    prompts = [torch.randint(8, VOCAB, (17 + 61 * i % 90,), generator=gen, device="cuda") for i in range(a.requests)]
    search = Search(prompts, a.beams, a.new, weights, rope)
    search.advance()                                         # once by hand, then recorded
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        search.advance()
    for _ in range(a.new - 2):
        graph.replay()
    torch.cuda.synchronize()
    assert int(search.status.item()) == 0
    worst = 0.0
    for r in range(a.requests):
        for b in range(a.beams):
            row = r * a.beams + b
            want, got = rescore(prompts[r], search.tokens[row], weights, rope), float(search.score[row])
            worst = max(worst, abs(got - want) / abs(want))
    held = int((search.pages.refs > 0).sum())
    print(f"{a.requests} requests of {a.beams} beams, {a.new} tokens each, {held} pages held by {int(search.pages.refs.sum())} entries; scores differ by "
          f"{worst:.4f} of theirs from those without a cache")
    return worst


if __name__ == "__main__":
    main()
