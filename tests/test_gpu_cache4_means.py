"""Attention over a 4-bit cache whose outputs are of the values' size also over many keys, and not what is
left of a sum around zero: a piece of a sequence that is lost, joined with the wrong weight or read from
another's rows shows.

means: the values' means differ by column, by sequence and along the keys.  heavy: some keys along a
sequence share nearly all of its weight, with values of their own.

Error of an element, derived: each weight is rounded to the input type (u = 2^-11 for fp16, 2^-8 for
bf16, half a step), u sum p|v|; the output too, u |out|; everything between is fp32, and fp32 scores
move the weights by less than 1e-4 and the sum of the weights as much: 2e-4 sum p|v|.  Log sums:
1e-4 + 1e-6 |lse|.  The test says itself that this is less than a fiftieth (heavy: a tenth) of the mean
output, and less than a quarter of what a heavy key adds to it in the mean.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


CASES = {
    "one_new": dict(cached=[20000, 9], fresh=[1, 1], hq=4, hk=1, d=128, page=16),
    "one_new_d256": dict(cached=[9000, 9], fresh=[1, 1], hq=2, hk=2, d=256, page=32),
    "one_new_odd_page": dict(cached=[7001, 4000], fresh=[1, 1], hq=2, hk=1, d=64, page=7),
    "one_new_wide_group": dict(cached=[9000, 900], fresh=[1, 1], hq=24, hk=1, d=96, page=16),
    "one_new_many": dict(cached=[(397 * i) % 4000 for i in range(40)], fresh=[1] * 40, hq=8, hk=2,
                         d=128, page=16),
    "four_new": dict(cached=[30000, 63], fresh=[4, 3], hq=8, hk=2, d=128, page=32),
    "four_new_d64": dict(cached=[9000, 12000], fresh=[4, 2], hq=4, hk=1, d=64, page=16),
    "chunk": dict(cached=[20000], fresh=[70], hq=8, hk=2, d=128, page=16),
    "chunk_d32": dict(cached=[8000], fresh=[90], hq=2, hk=1, d=32, page=16),
    "chunk_d64": dict(cached=[12345], fresh=[90], hq=4, hk=2, d=64, page=64),
    "chunk_d192": dict(cached=[5000], fresh=[50], hq=4, hk=2, d=192, page=16),
    "chunk_d256": dict(cached=[9000], fresh=[40], hq=4, hk=2, d=256, page=16),
    "chunk_odd_page": dict(cached=[5000], fresh=[90], hq=2, hk=1, d=96, page=7),
    "long_beside_short": dict(cached=[30000, 3, 3, 3], fresh=[17, 17, 1, 33], hq=8, hk=1, d=128,
                              page=64),
    "prompts": dict(cached=[0, 0, 0], fresh=[700, 1, 333], hq=4, hk=2, d=128, page=16),
    "mixed": dict(cached=[6000, 9000, 3, 12000], fresh=[60, 1, 140, 1], hq=4, hk=2, d=128, page=16),
    "mixed_group_of_24": dict(cached=[9000, 90, 10000], fresh=[1, 50, 1], hq=24, hk=1, d=128,
                              page=24),
}
HEAVY = 11  # heavy keys of a sequence


@pytest.mark.parametrize("kind", ["means", "heavy"])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_outputs_of_the_values_size(env, name, dtype, kind):
    torch, tod = env
    c, dt = CASES[name], getattr(torch, dtype)
    hq, hk, d, page, n = c["hq"], c["hk"], c["d"], c["page"], len(c["cached"])
    gen = torch.Generator(device="cuda").manual_seed(41)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    lens = [a + b for a, b in zip(c["cached"], c["fresh"])]
    need = [-(-m // page) for m in lens]
    pages = sum(need) + 3
    ids = torch.randperm(pages, generator=gen, device="cuda")
    table = torch.full((n, max(need)), -1, dtype=torch.int32, device="cuda")
    q = normal(sum(c["fresh"]), hq, d)
    k, v = normal(pages * page, hk, d), normal(pages * page, hk, d)
    if kind == "heavy":  # scores of 24, and of about 0
        q *= 0.5
        q[..., 0] = 4 * math.sqrt(d)
        k[..., 0] = 0
    rows, heavy, used = [], [], 0
    for r in range(n):
        mine = ids[used:used + need[r]]
        table[r, :need[r]] = mine.to(torch.int32)
        j = torch.arange(lens[r], device="cuda")
        rows.append(mine[j // page] * page + j % page)
        used += need[r]
        sign = 2.0 * torch.sign(normal(hk, d))
        # (The first key is one of them: every row sees a heavy key.)
        heavy.append(torch.arange(min(HEAVY, lens[r]), device="cuda") * lens[r] // HEAVY
                     if lens[r] >= HEAVY else j)
        if kind == "means":
            v[rows[r]] = 0.5 * v[rows[r]] + sign * (1 + j / lens[r])[:, None, None]
        else:
            at = rows[r][heavy[r]]
            k[at, :, 0] = 6.0
            v[at] = torch.sign(v[at]) * (2 + v[at].abs().clamp(max=2))
    q, k, v = q.to(dt), k.to(dt), v.to(dt)
    cache = tod.Cache4.zeros(pages, hk, page, d)
    every = torch.arange(pages * page, device="cuda")
    tod.tod_page_append4(k, k, v, every.int(), every, torch.zeros(0, device="cuda"), cache)
    k, v = (x.double() for x in tod.tod_page_read4(cache, every, dt))
    starts = torch.tensor([sum(c["fresh"][:i]) for i in range(n + 1)], dtype=torch.int32,
                          device="cuda")
    cached = torch.tensor(c["cached"], dtype=torch.int32, device="cuda")
    for hint in (None, max(c["fresh"])):
        out, lse = tod.tod_attn_paged4(q, cache, table, starts, cached, max_fresh=hint,
                                       return_lse=True)
        first = 0
        for r in range(n):
            f, m = c["fresh"][r], lens[r]
            pos = torch.arange(m, device="cuda")
            hidden = pos[None, :] > pos[m - f:, None]
            for h in range(hq):
                kh, vh = k[rows[r], h * hk // hq], v[rows[r], h * hk // hq]
                s = q[first:first + f, h].double() @ kh.T.contiguous() / math.sqrt(d)
                s = s.masked_fill(hidden, -math.inf)
                z = torch.logsumexp(s, dim=1)
                p = torch.exp(s - z[:, None])
                want, size = p @ vh, p @ vh.abs()
                bound = (U[dtype] + 2e-4) * size + U[dtype] * want.abs()
                assert float(bound.max()) < float(want.abs().mean()) / (
                    50 if kind == "means" else 10)
                if kind == "heavy":
                    seen = (~hidden[:, heavy[r]]).sum(1)
                    share = (p[:, heavy[r]].sum(1) / seen).min()
                    assert float(bound.max()) < float(share * vh[heavy[r]].abs().mean()) / 4
                off = (out[first:first + f, h].double() - want).abs() - bound
                assert float(off.max()) <= 0, (r, h, float(off.max()))
                off = (lse[first:first + f, h].double() - z).abs() - 1e-6 * z.abs()
                assert float(off.max()) <= 1e-4, (r, h)
            first += f
