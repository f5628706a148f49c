"""Attention over a 4-bit cache of unusual contents: blocks that are not finite, seen and unseen, very
many small weights, scores far beyond what a softmax needs, and values near the largest of the type.

Cases, expectations and derivations are those of the same tests over 16-bit pages.  Output: the
weights and the output are rounded to the input type (u = 2^-11 for fp16, 2^-8 for bf16, half an ulp)
and everything between is fp32: 2 u max|v| + 2e-4 max|v|; log sums: 1e-4 + 1e-6 |lse|.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


def filled(torch, tod, k, v, page):
    """A cache whose slots 0, 1, .. hold the rows k, v [rows, heads, dim]."""
    rows, heads, dim = k.shape
    cache = tod.Cache4.zeros(-(-rows // page), heads, page, dim)
    slot = torch.arange(rows, device="cuda")
    tod.tod_page_append4(k, k, v, torch.zeros(rows, dtype=torch.int32, device="cuda"), slot,
                         torch.zeros(0, device="cuda"), cache)
    return cache


# at: positions of the first sequence whose block holds what is not finite.
CASES = {
    "only_token": dict(cached=[0], fresh=[1], hq=4, hk=2, d=64, page=16, at=[0]),
    "one_new_at_itself": dict(cached=[100, 30], fresh=[1, 1], hq=8, hk=2, d=128, page=16, at=[100]),
    "one_new_cached": dict(cached=[100, 30], fresh=[1, 1], hq=8, hk=2, d=128, page=16, at=[3]),
    "one_new_odd_page": dict(cached=[300, 30], fresh=[1, 1], hq=2, hk=1, d=64, page=7, at=[3, 290]),
    "one_new_pieces": dict(cached=[20000, 9], fresh=[1, 1], hq=4, hk=1, d=128, page=16,
                           at=[64, 15000]),
    "one_new_pieces_d256": dict(cached=[9000, 9], fresh=[1, 1], hq=2, hk=2, d=256, page=32,
                                at=[7777]),
    "one_new_wide_group": dict(cached=[900, 9], fresh=[1, 1], hq=24, hk=1, d=96, page=16, at=[500]),
    "four_new_cached": dict(cached=[130, 63], fresh=[4, 1], hq=4, hk=2, d=96, page=32, at=[17]),
    "four_new_both": dict(cached=[130, 63], fresh=[4, 3], hq=8, hk=2, d=128, page=32,
                          at=[17, 132]),
    "four_new_pieces": dict(cached=[9000], fresh=[4], hq=4, hk=1, d=64, page=16, at=[40, 9002]),
    "many_pairs": dict(cached=[900] + [70] * 79, fresh=[1] * 80, hq=4, hk=2, d=64, page=16,
                       at=[500]),
    "chunk": dict(cached=[150, 0], fresh=[100, 77], hq=4, hk=2, d=128, page=16, at=[20, 200]),
    "chunk_odd_page": dict(cached=[61], fresh=[90], hq=2, hk=1, d=96, page=7, at=[5]),
    "chunk_d32": dict(cached=[61, 5], fresh=[90, 1], hq=2, hk=1, d=32, page=16, at=[5, 100]),
    "chunk_d256": dict(cached=[150], fresh=[100], hq=4, hk=2, d=256, page=16, at=[20, 201]),
    "split_chunk": dict(cached=[3000], fresh=[40], hq=8, hk=2, d=128, page=16, at=[1, 2500]),
    "mixed": dict(cached=[700, 900, 3], fresh=[60, 1, 40], hq=4, hk=2, d=128, page=16,
                  at=[650, 720]),
}


@pytest.mark.parametrize("kind", ["nan", "inf", "last_inf"])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_values_that_are_not_finite(env, name, dtype, kind):
    """nan: a block of NaN (scale byte 255); inf: scale bytes for which the block's codes are
    infinite numbers of the type.  Rows that see the key get the sum in the block's columns; other
    columns and rows keep their finite results.  last_inf: in the last key's block."""
    torch, tod = env
    c, dt = CASES[name], getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(23)
    hq, hk, d, page, n = c["hq"], c["hk"], c["d"], c["page"], len(c["cached"])
    lens = [a + b for a, b in zip(c["cached"], c["fresh"])]
    need = [-(-m // page) for m in lens]
    pages = sum(need) + 3
    at = c["at"] if kind != "last_inf" else [lens[0] - 1]
    q = torch.randn(sum(c["fresh"]), hq, d, generator=gen, device="cuda").to(dt)
    k, v = (torch.randn(pages * page, hk, d, generator=gen, device="cuda").to(dt) for _ in range(2))
    cache = filled(torch, tod, k, v, page)
    ids = torch.randperm(pages, generator=gen, device="cuda")
    table = torch.full((n, max(need)), -1, dtype=torch.int32, device="cuda")
    rows, used = [], 0
    for r in range(n):
        mine = ids[used:used + need[r]]
        table[r, :need[r]] = mine.to(torch.int32)
        j = torch.arange(lens[r], device="cuda")
        rows.append(mine[j // page] * page + j % page)
        used += need[r]
    every = torch.arange(pages * page, device="cuda")
    k, clean = tod.tod_page_read4(cache, every, dt)
    spoilt = []
    for p in at:  # the block's last columns' scale: of a NaN, or beyond the type
        slot = int(rows[0][p])
        cache.v_scales[slot // page, :, slot % page, d // 32 - 1] = {
            "nan": 255, "inf": 254, "last_inf": 254}[kind]
        cache.v_codes[slot // page, :, slot % page, d // 2 - 16:] = 0x7f
        spoilt.append(slot)
    # Rows behind the sequence's last, in its last page, and pages of nobody hold NaN as well.
    own = torch.cat(rows)
    other = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    other[own] = False
    for x in (cache.k_scales, cache.v_scales):
        flat = x.transpose(1, 2).reshape(pages * page, hk, d // 32).clone()
        flat[other] = 255
        x.copy_(flat.view(pages, page, hk, d // 32).transpose(1, 2))
    _, held = tod.tod_page_read4(cache, every, dt)
    clean = clean.double()
    for slot in spoilt:
        bad = held[slot, :, d - 32:]
        assert not torch.isfinite(bad).any()
        clean[slot, :, d - 32:] = 0.0
    clean[other] = 0.0
    v_max = float(clean.abs().max())
    starts = torch.tensor([sum(c["fresh"][:i]) for i in range(n + 1)], dtype=torch.int32,
                          device="cuda")
    cached = torch.tensor(c["cached"], dtype=torch.int32, device="cuda")
    for hint in (None, max(c["fresh"])):
        out, lse = tod.tod_attn_paged4(q, cache, table, starts, cached, max_fresh=hint,
                                       return_lse=True)
        bound, first = (2 * U[dtype] + 2e-4) * v_max, 0
        for r in range(n):
            f, m = c["fresh"][r], lens[r]
            pos = torch.arange(m, device="cuda")
            hidden = pos[None, :] > pos[m - f:, None]
            for h in range(hq):
                g = h * hk // hq
                s = q[first:first + f, h].double() @ k[rows[r], g].double().T / math.sqrt(d)
                s = s.masked_fill(hidden, -INF)
                z = torch.logsumexp(s, dim=1)
                want = torch.exp(s - z[:, None]) @ clean[rows[r], g]
                got = out[first:first + f, h].double()
                if r == 0:
                    total = torch.zeros(f, 32, dtype=torch.float64, device="cuda")
                    for p, slot in zip(at, spoilt):
                        total += torch.where(hidden[:, p, None], 0.0,
                                             held[slot, g, d - 32:].double())
                    odd = ~torch.isfinite(total)
                    tail = got[:, d - 32:]
                    assert torch.equal(tail[odd].isnan(), total[odd].isnan()), h
                    real = odd & ~total.isnan()
                    assert torch.equal(tail[real], total[real]), h
                    got[:, d - 32:] = torch.where(odd, want[:, d - 32:], tail)
                assert float((got - want).abs().max()) <= bound, (r, h)
                off = (lse[first:first + f, h].double() - z).abs() - 1e-6 * z.abs()
                assert float(off.max()) <= 1e-4, (r, h)
            first += f


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("fresh", [1, 4, 40])
def test_keys_that_are_not_finite(env, fresh, dtype):
    """Rows that see a key of NaN are NaN, and those before it are as they were without it."""
    torch, tod = env
    dt, n, d, page = getattr(torch, dtype), 500, 128, 16
    gen = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(fresh, 4, d, generator=gen, device="cuda").to(dt)
    k, v = (torch.randn(512, 2, d, generator=gen, device="cuda").to(dt) for _ in range(2))
    cache = filled(torch, tod, k, v, page)
    table = torch.arange(32, dtype=torch.int32, device="cuda")[None]
    args = (table, torch.tensor([0, fresh], dtype=torch.int32, device="cuda"),
            torch.tensor([n - fresh], dtype=torch.int32, device="cuda"))
    want, want_lse = tod.tod_attn_paged4(q, cache, *args, return_lse=True)
    at = n - (fresh + 1) // 2
    cache.k_scales[at // page, 0, at % page, 1] = 255
    out, lse = tod.tod_attn_paged4(q, cache, *args, return_lse=True)
    sees = torch.arange(n - fresh, n, device="cuda") >= at
    assert out[sees, :2].isnan().all() and lse[sees, :2].isnan().all()
    assert torch.equal(out[~sees], want[~sees]) and torch.equal(lse[~sees], want_lse[~sees])
    assert torch.equal(out[:, 2:], want[:, 2:]) and torch.equal(lse[:, 2:], want_lse[:, 2:])


# A key that outweighs each of very many others by e^gap: together they still count.  All other keys
# have the same score, so that with N of them
#   out = (v0 + N e^-gap v1) / (1 + N e^-gap),  lse = gap + ln(1 + N e^-gap).
# Log sums: 1e-4 allowed, a few roundings of numbers up to 35 expected.  Outputs: the weights are
# rounded all alike, u |out|, and the output, u |out| or 2^-25; weights below fp16's normal range are
# off by at most 2^-35 each; fp32 scores move the weights by 3e-6:
# (2 u + 3e-6) |out| + 2^-25 + N 2^-35.  (Keys and values here are values of the codes.)
SMALL = {
    "one_new": dict(keys=131072, fresh=1, at=0),
    "one_new_late": dict(keys=131072, fresh=1, at=130000),
    "one_new_whole": dict(keys=131072, fresh=1, at=0, shared=3100),
    "four_new": dict(keys=120011, fresh=4, at=70000),
    "four_new_whole": dict(keys=100000, fresh=4, at=3, shared=3100),
    "chunk": dict(keys=131072, fresh=60, at=5),
    "chunk_late": dict(keys=110003, fresh=60, at=90000),
    "chunk_whole": dict(keys=100000, fresh=128, at=5, shared=800),
}


@pytest.mark.parametrize("gap", [16.0, 24.0])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("name", sorted(SMALL))
def test_small_weights(env, name, dtype, gap):
    torch, tod = env
    c, d, dt, page = SMALL[name], 64, getattr(torch, dtype), 64
    n, f, s = c["keys"], c["fresh"], c.get("shared", 1)
    k = torch.zeros(n, 1, d, dtype=dt, device="cuda")
    k[c["at"], 0, 0] = gap
    q = torch.zeros(f * s, 1, d, dtype=dt, device="cuda")
    q[:, :, 0] = 8.0  # the scale is 1 / 8
    table = torch.arange(-(-n // page), dtype=torch.int32, device="cuda").repeat(s, 1)
    starts = torch.arange(0, f * s + 1, f, dtype=torch.int32, device="cuda")
    cached = torch.full((s,), n - f, dtype=torch.int32, device="cuda")
    seen = torch.arange(n - f + 1, n + 1, dtype=torch.float64, device="cuda").repeat(s)
    others = (seen - 1) * math.exp(-gap)
    for v0 in (0.0, 1.0):
        v = torch.ones(n, 1, d, dtype=dt, device="cuda")
        v[c["at"]] = v0
        cache = filled(torch, tod, k, v, page)
        out, lse = tod.tod_attn_paged4(q, cache, table, starts, cached, max_fresh=f,
                                       return_lse=True)
        assert (out == out[:, :, :1]).all()
        out = out[:, 0, 0].double()
        assert float((lse[:, 0].double() - gap - torch.log1p(others)).abs().max()) <= 1e-4
        want = (v0 + others) / (1 + others)
        allowed = (2 * U[dtype] + 3e-6) * want + 2.0 ** -25 + seen * 2.0 ** -35
        worst = int(((out - want).abs() - allowed).argmax())
        assert ((out - want).abs() <= allowed).all(), (float(out[worst]), float(want[worst]))


KEYS = 700


def pattern(torch, name):
    """The keys' first element: with 8192 in the queries, a 1,024th of the score."""
    i = torch.arange(KEYS, device="cuda", dtype=torch.float64)
    top = 48 * 1024.0
    return {
        "level": torch.full_like(i, top),
        "level_low": torch.full_like(i, -top),
        "rising": top * i / KEYS,
        "falling": top * (KEYS - i) / KEYS,
        "rising_through_0": top * (2 * i / KEYS - 1),
        "falling_through_0": top * (1 - 2 * i / KEYS),
        "saw": top * ((i * 37) % 101) / 101,
        "small_then_large": torch.where(i < 400, 0.0, top),
        "large_then_small": torch.where(i < 400, top, 0.0),
    }[name]


@pytest.mark.parametrize("fresh", [3, 90])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("name", ["level", "level_low", "rising", "falling", "rising_through_0",
                                  "falling_through_0", "saw", "small_then_large",
                                  "large_then_small"])
def test_large_scores(env, name, dtype, fresh):
    """Scores of up to 5e7.  Those that differ, differ by thousands, so that the largest take all of
    the weight, in equal parts: 2 u max|v|.  Log sums: 4 2^-24 of a score, and 1e-4."""
    torch, tod = env
    dt, d, n, f = getattr(torch, dtype), 64, KEYS, fresh
    gen = torch.Generator(device="cuda").manual_seed(3)
    v = torch.randn(n, 1, d, generator=gen, device="cuda").to(dt)
    k = torch.zeros(n, 1, d, dtype=dt, device="cuda")
    k[:, 0, 0] = pattern(torch, name).to(dt)
    cache = filled(torch, tod, k, v, 20)
    k, v = (x.double() for x in tod.tod_page_read4(cache, torch.arange(n, device="cuda"), dt))
    q = torch.zeros(f, 1, d, dtype=dt, device="cuda")
    q[:, 0, 0] = 8192.0  # the scale is 1 / 8
    out, lse = tod.tod_attn_paged4(
        q, cache, torch.arange(n // 20, dtype=torch.int32, device="cuda")[None],
        torch.tensor([0, f], dtype=torch.int32, device="cuda"),
        torch.tensor([n - f], dtype=torch.int32, device="cuda"), max_fresh=f, return_lse=True)
    pos = torch.arange(n, device="cuda")
    s = (1024.0 * k[:, 0, 0]).expand(f, n).masked_fill(pos[None, :] > pos[n - f:, None], -INF)
    z = torch.logsumexp(s, 1)
    want = torch.softmax(s, 1) @ v[:, 0]
    err = float((out[:, 0].double() - want).abs().max())
    assert err <= 2 * U[dtype] * float(v.abs().max()), err
    assert ((lse[:, 0].double() - z).abs() <= 1e-4 + 2.0 ** -22 * z.abs()).all()


@pytest.mark.parametrize("kind", ["chunk", "split_chunk", "tokens"])
@pytest.mark.parametrize("rise", [2.0, 6.0, 12.0, 24.0])
def test_large_values(env, kind, rise):
    """bf16 values near the largest that a cache holds, of one magnitude: the output is theirs,
    within 2 u and 1e-4 for the scores.  One key of score 0 among many that do not count, and later
    one that outweighs it by e^rise."""
    torch, tod = env
    n, d, page, large = (4000 if kind == "split_chunk" else 400), 64, 16, 2.0 ** 126
    k = torch.zeros(n, 1, d, dtype=torch.bfloat16, device="cuda")
    k[:, 0, 0] = -48.0
    k[3, 0, 0], k[n // 2, 0, 0] = 0.0, rise
    v = torch.full((n, 1, d), large, dtype=torch.bfloat16, device="cuda")
    v[:, :, 1] = -large
    cache = filled(torch, tod, k, v, page)
    f = {"chunk": 60, "split_chunk": 40, "tokens": 2}[kind]
    q = torch.zeros(f, 1, d, dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = 8.0  # the scale is 1 / 8
    out = tod.tod_attn_paged4(q, cache, torch.arange(n // page, dtype=torch.int32, device="cuda")[None],
                              torch.tensor([0, f], dtype=torch.int32, device="cuda"),
                              torch.tensor([n - f], dtype=torch.int32, device="cuda"), max_fresh=f)
    assert torch.isfinite(out).all()
    assert ((out[:, 0].double() - v[:f, 0].double()).abs() <= (2.0 ** -7 + 1e-4) * large).all()
