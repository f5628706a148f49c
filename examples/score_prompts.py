"""Outlier scores of prompts while a language model serves them.

A small decoder (random weights; the point is the calls) serves requests over a paged cache and
hands the mean hidden state of every request's tokens to the kNN detector, fitted on the prompts of
a first batch.  The rows that the detector scores come out of the sequence operators:

  tod_attn_prompt   whole packed prompts (the fitting batch)
  tod_page_map      pages and slots of a step's new tokens from the requests' lengths
  tod_page_append   their queries and keys rotated by position, keys and values into the pages
  tod_attn_paged    chunks of new prompts and single tokens over the pages
  tod_knn_decision  the scores of the new requests

With --four the cache holds 4-bit rows, a quarter of the memory: tod_page_append4 and
tod_attn_paged4.

Usual prompts draw their tokens from a small part of the vocabulary, odd ones from the rest.
Run: python examples/score_prompts.py [--four]
"""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

from paper_2110_14007_amd import tod  # noqa: E402


class Decoder:
    """Pre-norm decoder blocks with grouped heads and rotary positions."""

    def __init__(self, vocab=512, layers=2, heads=8, kv_heads=2, dim=64, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.layers = heads, kv_heads, dim, layers
        width = heads * dim

        def weight(a, b):
            return (torch.randn(a, b, generator=gen, device="cuda") / a ** 0.5).half()

        self.embed = torch.randn(vocab, width, generator=gen, device="cuda").half()
        self.qkv = [weight(width, (heads + 2 * kv_heads) * dim) for _ in range(layers)]
        self.proj = [weight(width, width) for _ in range(layers)]
        self.up = [weight(width, 2 * width) for _ in range(layers)]
        self.down = [weight(2 * width, width) for _ in range(layers)]
        self.rates = 10000.0 ** (-torch.arange(dim // 2, device="cuda") / (dim // 2))

    @staticmethod
    def norm(x):
        return torch.nn.functional.rms_norm(x.float(), x.shape[-1:]).half()

    def rotate(self, x, pos):
        a = pos[:, None, None] * self.rates
        lo, hi = x.float().chunk(2, -1)
        return torch.cat([lo * a.cos() - hi * a.sin(), lo * a.sin() + hi * a.cos()], -1).half()

    def forward(self, tokens, attend):
        """Hidden states [tokens, width]; attend(layer, q, k, v) -> [tokens, heads, dim] rotates
        queries and keys by position."""
        x = self.embed[tokens]
        h, g, d = self.heads, self.kv_heads, self.dim
        for i in range(self.layers):
            qkv = (self.norm(x) @ self.qkv[i]).view(-1, h + 2 * g, d)
            o = attend(i, qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:])
            x = x + o.reshape(x.shape) @ self.proj[i]
            x = x + torch.nn.functional.gelu(self.norm(x) @ self.up[i]) @ self.down[i]
        return self.norm(x)


def whole_prompts(model, prompts):
    """Mean hidden state of every prompt's tokens, all prompts packed."""
    lens = torch.tensor([len(p) for p in prompts], device="cuda")
    row_start = torch.nn.functional.pad(torch.cumsum(lens, 0), (1, 0)).to(torch.int32)
    pos = torch.cat([torch.arange(len(p), device="cuda") for p in prompts])
    ws = tod.Workspace()
    h = model.forward(torch.cat(prompts), lambda i, q, k, v: tod.tod_attn_prompt(
        model.rotate(q, pos), model.rotate(k, pos), v, row_start, workspace=ws))
    return sums_of(h, lens) / lens[:, None]


def sums_of(h, lens):
    """Sums of the rows of h over sequences of the given lengths."""
    owner = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), lens)
    out = torch.zeros(len(lens), h.shape[1], device="cuda")
    return out.index_add_(0, owner, h.float())


class Server:
    """Requests over a paged cache, of 4-bit rows with `four`, served in steps that mix chunks of
    prompts and single tokens."""

    def __init__(self, model, prompts, page=16, chunk=48, four=False):
        self.model, self.prompts, self.page, self.chunk = model, prompts, page, chunk
        n, cols = len(prompts), max(-(-len(p) // page) for p in prompts)
        pages = sum(-(-len(p) // page) for p in prompts)
        shape = (pages, model.kv_heads, page, model.dim)
        self.four = four
        if four:
            self.caches = [tod.Cache4.zeros(*shape) for _ in range(model.layers)]
        else:
            self.caches = [[torch.zeros(shape, dtype=torch.float16, device="cuda")
                            for _ in range(2)] for _ in range(model.layers)]
        self.table = torch.full((n, cols), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(pages, device="cuda").to(torch.int32)
        self.done = [0] * n
        self.sums = torch.zeros(n, model.heads * model.dim, device="cuda")
        self.ws = tod.Workspace()

    def step(self):
        """Serves the next tokens of every unfinished request; False when all are done."""
        fresh = [min(self.chunk if i % 3 else 1 + self.chunk * (d == 0), len(p) - d)
                 for i, (p, d) in enumerate(zip(self.prompts, self.done))]
        if not any(fresh):
            return False
        cached = torch.tensor(self.done, dtype=torch.int32, device="cuda")
        new = torch.tensor(fresh, dtype=torch.int32, device="cuda")
        tokens = torch.cat([p[d:d + f] for p, d, f in zip(self.prompts, self.done, fresh)])
        row_start, slot, pos, used = tod.tod_page_map(cached, new, self.free, self.table,
                                                      self.page, sum(fresh))

        def attend(i, q, k, v):
            cache, where = self.caches[i], (self.table, row_start, cached)
            if self.four:
                q = tod.tod_page_append4(q, k, v, pos, slot, self.model.rates, cache)
                return tod.tod_attn_paged4(q, cache, *where, max_fresh=max(fresh),
                                           workspace=self.ws)
            q = tod.tod_page_append(q, k, v, pos, slot, self.model.rates, *cache)
            return tod.tod_attn_paged(q, *cache, *where, max_fresh=max(fresh), workspace=self.ws)

        h = self.model.forward(tokens, attend)
        taken, lacking = used.tolist()
        if lacking:
            raise RuntimeError("the cache has no page left for %d tokens" % lacking)
        self.free = self.free[taken:]
        self.sums += sums_of(h, new.long())
        self.done = [d + f for d, f in zip(self.done, fresh)]
        return True

    def states(self):
        return self.sums / torch.tensor(self.done, device="cuda")[:, None]


def make_prompts(n, lo, hi, seed, part):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = torch.randint(lo, hi, (n,), generator=gen, device="cuda").tolist()
    return [torch.randint(part[0], part[1], (m,), generator=gen, device="cuda") for m in lens]


def main(four=False):
    model = Decoder()
    fitted = whole_prompts(model, make_prompts(200, 80, 200, 1, (0, 64)))
    usual, odd = make_prompts(24, 80, 200, 2, (0, 64)), make_prompts(6, 80, 200, 3, (64, 512))
    server = Server(model, usual + odd, four=four)
    steps = 0
    while server.step():
        steps += 1
    score = tod.tod_knn_decision(server.states(), fitted, 5)
    drift = (server.states() - whole_prompts(model, usual + odd)).abs().max()
    print("%d requests in %d steps; scores of usual prompts %.2f to %.2f, of odd ones %.2f to %.2f"
          % (len(server.prompts), steps, float(score[:24].min()), float(score[:24].max()),
             float(score[24:].min()), float(score[24:].max())))
    print("largest difference between served and whole-prompt states: %.4f" % float(drift))
    return score, float(drift)


if __name__ == "__main__":
    main(four="--four" in sys.argv[1:])
