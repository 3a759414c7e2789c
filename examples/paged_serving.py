"""A small server loop on the paged cache: requests arrive while others decode, prompts are taken in chunks beside single tokens,
every sequence owns the pages its length needs and gives them back when it is done.

Per layer and step, what libee does is two calls: `paged.append` (keys rotated into the pages, values beside them, queries rotated)
and `paged.attend`.  The rest of the model here is random-weight attention blocks in plain torch, enough to feed one token into the
next.  At the end every request is computed once more without a cache, with `Rope.apply` and dense attention, and compared.

    python examples/paged_serving.py [--requests 6] [--layers 2] [--chunk 48]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2504_10724_amd import paged  # noqa: E402

HQ, HKV, HD, PAGE, D = 8, 2, 128, 64, 512


class Pages:
    """which pages are free, and which belong to whom"""

    def __init__(self, n):
        self.free, self.of = list(range(n)), {}

    def grow(self, request, length):
        mine = self.of.setdefault(request, [])
        while len(mine) * PAGE < length:
            mine.append(self.free.pop())

    def give_back(self, request):
        self.free += self.of.pop(request)


def make_weights(layers, gen):
    def normal(*shape):
        return (torch.randn(shape, generator=gen, device="cuda") * shape[0] ** -0.5).to(torch.bfloat16)
    return [dict(qkv=normal(D, (HQ + 2 * HKV) * HD), out=normal(HQ * HD, D)) for _ in range(layers)]


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5)).to(torch.bfloat16)


def project(x, w):
    y = (norm(x) @ w["qkv"]).view(len(x), HQ + 2 * HKV, HD)
    return y[:, :HQ], y[:, HQ:HQ + HKV], y[:, HQ + HKV:]


def serve(prompts, n_new, weights, rope, chunk, n_pages, width):
    """prompts: [tokens][D] tensors.  Returns each request's hidden states, position by position; a new token's input is the last output."""
    cache = paged.PagedCache(len(weights), n_pages, HKV, HD, PAGE, "bf16")
    pages, states, waiting, running = Pages(n_pages), {}, list(range(len(prompts))), {}
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    while waiting or running:
        if waiting:                                          # one request joins a step
            r = waiting.pop(0)
            running[r], states[r] = 0, []
        rows, starts, lengths, table = [], [0], [], []
        for r, done in running.items():
            n = min(chunk, len(prompts[r]) - done) if done < len(prompts[r]) else 1
            rows.append(prompts[r][done:done + n] if done < len(prompts[r]) else states[r][-1][-1:])
            running[r] = done + n
            pages.grow(r, done + n)
            starts.append(starts[-1] + n)
            lengths.append(done + n)
            table.append(pages.of[r] + [-1] * (width - len(pages.of[r])))
        dev = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (starts, lengths, table)]
        step = paged.PagedStep(*dev, n_tokens=starts[-1], max_q_len=max(b - a for a, b in zip(starts, starts[1:])), max_kv_len=max(lengths),
                               status=status)
        x = torch.cat(rows)
        for layer, w in enumerate(weights, 1):
            q, k, v = project(x, w)
            q = paged.append(cache, layer, step, k, v, rope=rope, q=q)
            x = x + paged.attend(cache, layer, step, q).reshape(len(x), -1) @ w["out"]
        for (r, done), a, b in zip(list(running.items()), starts, starts[1:]):
            states[r].append(x[a:b])
            if done == len(prompts[r]) + n_new - 1:
                del running[r]
                pages.give_back(r)
    assert int(status.item()) == 0 and len(pages.free) == n_pages
    return [torch.cat(states[r]) for r in range(len(prompts))]


def dense(x, weights, rope):
    """the same blocks over a whole sequence, without a cache"""
    pos = torch.arange(len(x), dtype=torch.int32, device="cuda")
    hide = torch.triu(torch.ones(len(x), len(x), dtype=torch.bool, device="cuda"), 1)
    for w in weights:
        q, k, v = project(x, w)
        q, k = rope.apply(q, pos).float(), rope.apply(k, pos).float()
        k, v = (t.float().repeat_interleave(HQ // HKV, 1).transpose(0, 1).contiguous() for t in (k, v))
        s = torch.matmul(q.transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) * HD ** -0.5
        o = torch.matmul(torch.softmax(s.masked_fill(hide, float("-inf")), -1), v).transpose(0, 1)
        x = x + o.reshape(len(x), -1).to(torch.bfloat16) @ w["out"]
    return x


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=6)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--chunk", type=int, default=48)
    ap.add_argument("--new", type=int, default=20)
    a = ap.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(1)
    weights = make_weights(a.layers, gen)
    rope = paged.Rope(HD, 1024, rot_dim=64, pairing="interleaved", scaling="bands", factor=4.0, trained_pos=256)
    lengths = [17 + 61 * i % 190 for i in range(a.requests)]
    prompts = [torch.randn(n, D, generator=gen, device="cuda").to(torch.bfloat16) for n in lengths]
    width = (max(lengths) + a.new + PAGE - 1) // PAGE
    out = serve(prompts, a.new, weights, rope, a.chunk, width * a.requests, width)
    worst = 0.0
    for p, got in zip(prompts, out):
        inputs = torch.cat([p, got[len(p) - 1:-1]])          # each new token's input was the output before it
        want = dense(inputs, weights, rope)
        worst = max(worst, float((got.float() - want.float()).abs().max() / want.float().abs().max()))
    print(f"{a.requests} requests, {sum(len(s) for s in out)} positions, largest difference from dense attention {worst:.4f} of the largest value")
    return worst


if __name__ == "__main__":
    main()
