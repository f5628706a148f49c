"""The sequence operators on the GPU against plain implementations in 64 bits: page map,
page write, attention over packed prompts and over pages.

Tolerances of attention, derived: the weights p are rounded to the input type (u = 2^-11 for
fp16, 2^-8 / 2 = 2^-9 for bf16, half an ulp) and so is the output, everything between is fp32.
The output is sum p v / sum p with |rounding of p| <= u p (fp16: plus 2^-25 where p is
subnormal; the largest p is at least 1), so the product is off by at most u max|v| over the
visible keys and rounding the output adds u |out| <= u max|v|: 2 u max|v| and 2^-25 n max|v|.
fp32 scores: a product of d terms of magnitude |q| |k| scale is off by at most
d 2^-24 |q| |k| scale, which moves every weight by that factor: with rows of about sqrt(d)
length times 1.5 that is under 1e-4 here.  The tests allow 2.5 u max|v| + 2e-4 max|v| and, for the log sums,
1e-4 + 1e-6 |lse|.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -9}


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


def dtype_of(torch, name):
    return {"fp16": torch.float16, "bf16": torch.bfloat16}[name]


# ---------------------------------------------------------------------------
# plain implementations, numpy fp64
# ---------------------------------------------------------------------------

def plain_map(cached, fresh, free, table, page, tokens):
    table = table.copy()
    n, cols = table.shape
    starts, slots, poss, used, lost, total = [], [], [], 0, 0, 0
    for r in range(n):
        starts.append(min(total, tokens))
        c, f = max(int(cached[r]), 0), max(int(fresh[r]), 0)
        take = max(0, min(f, tokens - total))
        total += f
        lost += f - take
        have = min(-(-c // page), cols)
        want = min(-(-(c + take) // page), cols)
        for j in range(have, want):
            table[r, j] = free[used] if used < len(free) else -1
            used += 1
        for i in range(take):
            p = c + i
            col = p // page
            s = -1
            if col < cols and table[r, col] >= 0:
                s = int(table[r, col]) * page + p % page
            lost += s < 0
            slots.append(s)
            poss.append(p)
    starts.append(min(total, tokens))
    pad = tokens - len(slots)
    return (np.array(starts), np.array(slots + [-1] * pad), np.array(poss + [-1] * pad),
            np.array([used, lost]), table)


def plain_attention(q, k, v, first, causal, scale=None):
    """q [n, hq, d], k, v [len, hk, d] fp64; query i stands at position first + i."""
    n, hq, d = q.shape
    length, hk, _ = k.shape
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = np.zeros((n, hq, d))
    lse = np.full((n, hq), -np.inf)
    for h in range(hq):
        kh, vh = k[:, h // (hq // hk)], v[:, h // (hq // hk)]
        for i in range(n):
            seen = min(length, first + i + 1) if causal else length
            if seen <= 0:
                continue
            s = scale * (kh[:seen] @ q[i, h])
            top = s.max()
            p = np.exp(s - top)
            out[i, h] = (p @ vh[:seen]) / p.sum()
            lse[i, h] = top + math.log(p.sum())
    return out, lse


def check(name, out, lse, want, want_lse, v_max):
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.isfinite(out).all()
    err = np.abs(out - want).max()
    bound = (2.5 * U[name] + 2e-4) * v_max
    assert err <= bound, "out off by %.3g, allowed %.3g" % (err, bound)
    seen = np.isfinite(want_lse)
    assert (lse[~seen] == -np.inf).all() and (out[~seen] == 0).all()
    off = np.abs(lse[seen] - want_lse[seen]) - 1e-6 * np.abs(want_lse[seen])
    assert seen.sum() == 0 or off.max() <= 1e-4, "lse off by %.3g" % off.max()


def rows(torch, gen, name, *shape, spread=1.0):
    return (spread * torch.randn(*shape, generator=gen, device="cuda")).to(dtype_of(torch, name))


def starts_of(torch, lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------
# page map and page write
# ---------------------------------------------------------------------------

MAPS = {
    "one": dict(cached=[0], fresh=[1], page=16, cols=4, free=3),
    "single_tokens": dict(cached=list(range(0, 70)), fresh=[1] * 70, page=16, cols=8, free=90),
    "page_of_one": dict(cached=[0, 3, 5], fresh=[4, 0, 2], page=1, cols=9, free=20),
    "odd_page": dict(cached=[0, 7, 13, 14, 27], fresh=[5, 9, 1, 0, 30], page=7, cols=20, free=20),
    "long": dict(cached=[100, 0, 5], fresh=[3000, 2500, 4000], page=32, cols=200, free=400),
    "free_ends": dict(cached=[15, 16, 0, 31], fresh=[40, 40, 40, 40], page=16, cols=6, free=5),
    "no_free": dict(cached=[15, 16], fresh=[3, 3], page=16, cols=6, free=0),
    "table_ends": dict(cached=[10, 40, 33], fresh=[60, 9, 1], page=16, cols=2, free=20),
    "all_idle": dict(cached=[4, 9, 0], fresh=[0, 0, 0], page=8, cols=4, free=4, tokens=5),
    "negative": dict(cached=[-3, 5], fresh=[2, -4], page=8, cols=4, free=4, tokens=3),
    "padded": dict(cached=[4, 9], fresh=[3, 2], page=8, cols=4, free=4, tokens=40),
    "cut": dict(cached=[4, 9, 2], fresh=[30, 20, 9], page=8, cols=9, free=40, tokens=37),
    "many": dict(cached=[(37 * i) % 200 for i in range(3001)],
                 fresh=[(i * i) % 9 for i in range(3001)], page=16, cols=14, free=6000),
    "begun_page_missing": dict(cached=[12, 20], fresh=[9, 1], page=8, cols=4, free=9, hole=True),
}


@pytest.mark.parametrize("name", sorted(MAPS))
def test_page_map(env, name):
    torch, tod = env
    c = MAPS[name]
    rng = np.random.default_rng(7)
    n, page, cols = len(c["cached"]), c["page"], c["cols"]
    ids = rng.permutation(n * cols + c["free"]).astype(np.int32)
    table = np.full((n, cols), -1, np.int32)
    for r in range(n):
        have = min(-(-max(c["cached"][r], 0) // page), cols)
        table[r, :have] = ids[r * cols:r * cols + have]
    if c.get("hole"):
        table[0, 1] = -1
    free = ids[n * cols:].copy()
    tokens = c.get("tokens", sum(c["fresh"]))
    want = plain_map(c["cached"], c["fresh"], free, table, page, tokens)
    t = torch.from_numpy(table).cuda()
    args = (torch.tensor(c["cached"], dtype=torch.int32, device="cuda"),
            torch.tensor(c["fresh"], dtype=torch.int32, device="cuda"),
            torch.from_numpy(free).cuda(), t, page, tokens)
    for _ in range(2):  # the call may be repeated on its own result
        row_start, slot, pos, used = tod.tod_page_map(*args)
        for got, ref in zip((row_start, slot, pos, used, t), want):
            np.testing.assert_array_equal(got.cpu().numpy(), ref)


@pytest.mark.parametrize("name", ["fp16", "bf16"])
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 8, 1), (5, 3, 72, 7), (130, 2, 64, 16),
                                                   (1025, 8, 128, 32), (33, 1, 256, 64)])
def test_page_write(env, name, tokens, heads, dim, page):
    torch, tod = env
    gen = torch.Generator(device="cuda").manual_seed(3)
    n_pages = tokens // page + 3
    kv = rows(torch, gen, name, tokens, 2 * heads, dim)
    k, v = kv[:, :heads], kv[:, heads:]
    slot = torch.randperm(n_pages * page, generator=gen, device="cuda")[:tokens].contiguous()
    if tokens > 4:  # no page, and slots outside the cache
        slot[1], slot[2], slot[3] = -1, n_pages * page, -(1 << 40)
    kp, vp = (rows(torch, gen, name, n_pages, heads, page, dim) for _ in range(2))
    want_k, want_v = kp.clone(), vp.clone()
    for t, s in enumerate(slot.cpu().tolist()):
        if 0 <= s < n_pages * page:
            want_k[s // page, :, s % page] = k[t]
            want_v[s // page, :, s % page] = v[t]
    tod.tod_page_write(k, v, slot, kp, vp)
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)


# ---------------------------------------------------------------------------
# attention over packed prompts
# ---------------------------------------------------------------------------

PROMPTS = {
    "one_token": dict(lens=[1], hq=4, hk=2, d=64),
    "short": dict(lens=[3, 0, 1, 17, 0], hq=2, hk=2, d=64),
    "stage_edges": dict(lens=[63, 64, 65, 31, 33], hq=2, hk=1, d=64),
    "tile_edges": dict(lens=[127, 128, 129, 1, 255], hq=3, hk=3, d=64),
    "group_4": dict(lens=[40, 0, 77, 200], hq=8, hk=2, d=128),
    "group_6": dict(lens=[50, 130], hq=6, hk=1, d=96),
    "group_7": dict(lens=[90], hq=7, hk=1, d=80),
    "dim_8": dict(lens=[70, 5], hq=2, hk=1, d=8),
    "dim_72": dict(lens=[70, 65], hq=2, hk=2, d=72),
    "dim_256": dict(lens=[150, 20], hq=4, hk=2, d=256),
    "dim_200": dict(lens=[100], hq=1, hk=1, d=200),
    "longer": dict(lens=[700], hq=2, hk=1, d=128),
    "many": dict(lens=[(i * 7) % 12 for i in range(150)], hq=2, hk=1, d=64),
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("name", sorted(PROMPTS))
def test_attn_prompt(env, name, dt, causal):
    torch, tod = env
    c = PROMPTS[name]
    gen = torch.Generator(device="cuda").manual_seed(11)
    lens, hq, hk, d = c["lens"], c["hq"], c["hk"], c["d"]
    t = sum(lens)
    qkv = rows(torch, gen, dt, t, hq + 2 * hk, d)
    q, k, v = (1.5 * qkv[:, :hq]).to(qkv.dtype), qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    out, lse = tod.tod_attn_prompt(q, k, v, starts_of(torch, lens), causal=causal,
                                   return_lse=True)
    q64, k64, v64 = (x.double().cpu().numpy() for x in (q, k, v))
    want, want_lse, at = np.zeros((t, hq, d)), np.zeros((t, hq)), 0
    for n in lens:
        r = slice(at, at + n)
        want[r], want_lse[r] = plain_attention(q64[r], k64[r], v64[r], 0, causal)
        at += n
    check(dt, out, lse, want, want_lse, np.abs(v64).max())


def test_attn_prompt_padding_rows_are_empty(env):
    torch, tod = env
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (rows(torch, gen, "bf16", 300, 2, 64) for _ in range(3))
    k[200:], v[200:] = float("nan"), float("inf")
    out, lse = tod.tod_attn_prompt(q, k, v, starts_of(torch, [150, 50]), return_lse=True)
    assert (out[200:] == 0).all() and (lse[200:] == -math.inf).all()
    assert torch.isfinite(out).all()


def test_attn_prompt_scale_strides_and_out(env):
    torch, tod = env
    gen = torch.Generator(device="cuda").manual_seed(6)
    base = rows(torch, gen, "fp16", 4, 90, 64)  # heads outermost
    q, k, v = base[:2].transpose(0, 1), base[2:3].transpose(0, 1), base[3:].transpose(0, 1)
    buf = torch.empty(90, 2, 64, dtype=q.dtype, device="cuda")
    out, lse = tod.tod_attn_prompt(q, k, v, starts_of(torch, [90]), scale=0.31, out=buf,
                                   return_lse=True)
    assert out.data_ptr() == buf.data_ptr()
    want, want_lse = plain_attention(*(x.double().cpu().numpy() for x in (q, k, v)), 0, True, 0.31)
    check("fp16", out, lse, want, want_lse, float(v.abs().max()))


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
def test_attn_prompt_spiked_scores(env, dt):
    # Maxima that keep growing along the keys, by more than one rescaling step.
    torch, tod = env
    gen = torch.Generator(device="cuda").manual_seed(8)
    n, d = 400, 64
    q, k, v = (rows(torch, gen, dt, n, 1, d) for _ in range(3))
    q[:, :, 0], k[:, :, 0] = 8.0, torch.linspace(0, 60, n, device="cuda").to(k.dtype)[:, None]
    out, lse = tod.tod_attn_prompt(q, k, v, starts_of(torch, [n]), causal=False, return_lse=True)
    q64, k64, v64 = (x.double().cpu().numpy() for x in (q, k, v))
    want, want_lse = plain_attention(q64, k64, v64, 0, False)
    check(dt, out, lse, want, want_lse, np.abs(v64).max())


# ---------------------------------------------------------------------------
# attention over pages
# ---------------------------------------------------------------------------

PAGED = {
    "first_token": dict(cached=[0], fresh=[1], hq=4, hk=2, d=64, page=16),
    "single_tokens": dict(cached=[0, 1, 15, 16, 17, 200, 333], fresh=[1] * 7, hq=8, hk=2, d=128,
                          page=16),
    "idle": dict(cached=[50, 20, 0, 90], fresh=[1, 0, 0, 2], hq=4, hk=4, d=64, page=16),
    "page_of_one": dict(cached=[9, 70], fresh=[3, 1], hq=2, hk=1, d=64, page=1),
    "odd_page": dict(cached=[100, 13, 64], fresh=[5, 30, 1], hq=4, hk=2, d=64, page=7),
    "big_page": dict(cached=[100, 300], fresh=[1, 20], hq=4, hk=2, d=128, page=256),
    "few_new": dict(cached=[130, 63, 257], fresh=[2, 4, 3], hq=8, hk=1, d=128, page=32),
    "chunk": dict(cached=[200], fresh=[150], hq=8, hk=2, d=128, page=32),
    "whole_prompt": dict(cached=[0, 0], fresh=[130, 70], hq=4, hk=2, d=64, page=16),
    "mixed": dict(cached=[300, 10, 0, 77, 500], fresh=[1, 90, 40, 1, 1], hq=6, hk=2, d=96,
                  page=16),
    "group_1": dict(cached=[150, 40], fresh=[1, 1], hq=12, hk=12, d=64, page=8),
    "group_16": dict(cached=[150, 40], fresh=[1, 3], hq=16, hk=1, d=128, page=64),
    "group_40": dict(cached=[150, 40], fresh=[1, 2], hq=40, hk=1, d=64, page=64),
    "dim_256": dict(cached=[90, 222], fresh=[1, 33], hq=4, hk=1, d=256, page=16),
    "dim_80": dict(cached=[90, 222], fresh=[1, 33], hq=4, hk=4, d=80, page=16),
    "long": dict(cached=[5000, 40, 3000], fresh=[1, 1, 1], hq=2, hk=1, d=64, page=16),
    "long_chunk": dict(cached=[2500], fresh=[20], hq=4, hk=1, d=64, page=16),
}


def paged_case(torch, c, dt, seed=13):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    hq, hk, d, page = c["hq"], c["hk"], c["d"], c["page"]
    n = len(c["cached"])
    have = [-(-(a + b) // page) for a, b in zip(c["cached"], c["fresh"])]
    ids = rng.permutation(sum(have) + 5).astype(np.int32)
    table = np.full((n, max(have) + 2), -1, np.int32)
    at = 0
    for r in range(n):
        table[r, :have[r]] = ids[at:at + have[r]]
        at += have[r]
    kp, vp = (rows(torch, gen, dt, len(ids), hk, page, d) for _ in range(2))
    q = rows(torch, gen, dt, sum(c["fresh"]), hq, d, spread=1.5)
    return q, kp, vp, table


def paged_want(c, q, kp, vp, table):
    q64, k64, v64 = (x.double().cpu().numpy() for x in (q, kp, vp))
    want, want_lse, at = np.zeros(q64.shape), np.zeros(q64.shape[:2]), 0
    for r, (a, n) in enumerate(zip(c["cached"], c["fresh"])):
        j = np.arange(a + n)
        pg, row = table[r, j // c["page"]], j % c["page"]
        rr = slice(at, at + n)
        want[rr], want_lse[rr] = plain_attention(q64[rr], k64[pg, :, row], v64[pg, :, row], a,
                                                 True)
        at += n
    return want, want_lse


@pytest.mark.parametrize("hint", [True, False])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("name", sorted(PAGED))
def test_attn_paged(env, name, dt, hint):
    torch, tod = env
    c = PAGED[name]
    q, kp, vp, table = paged_case(torch, c, dt)
    want, want_lse = paged_want(c, q, kp, vp, table)
    # rows of the pages past the sequences' ends hold anything
    for r, (a, n) in enumerate(zip(c["cached"], c["fresh"])):
        if (a + n) % c["page"]:
            pg = int(table[r, (a + n) // c["page"]])
            kp[pg, :, (a + n) % c["page"]:] = float("nan")
            vp[pg, :, (a + n) % c["page"]:] = float("inf")
    out, lse = tod.tod_attn_paged(
        q, kp, vp, torch.from_numpy(table).cuda(), starts_of(torch, c["fresh"]),
        torch.tensor(c["cached"], dtype=torch.int32, device="cuda"),
        max_fresh=max(c["fresh"]) if hint else None, return_lse=True)
    check(dt, out, lse, want, want_lse, float(vp[torch.isfinite(vp)].abs().max()))


def test_attn_paged_entries_that_are_no_page(env):
    # Such an entry counts as a page of zeros, whatever it holds.
    torch, tod = env
    c = dict(cached=[100, 70], fresh=[1, 30], hq=4, hk=2, d=64, page=16)
    q, kp, vp, table = paged_case(torch, c, "bf16")
    bad = table.copy()
    bad[0, 2], bad[1, 1], bad[1, 3] = -1, 1 << 30, -(1 << 31)
    zk, zv = (torch.cat([x, torch.zeros_like(x[:1])]) for x in (kp, vp))
    zero = table.copy()
    zero[0, 2] = zero[1, 1] = zero[1, 3] = kp.shape[0]
    want, want_lse = paged_want(c, q, zk, zv, zero)
    out, lse = tod.tod_attn_paged(
        q, kp, vp, torch.from_numpy(bad).cuda(), starts_of(torch, c["fresh"]),
        torch.tensor(c["cached"], dtype=torch.int32, device="cuda"), return_lse=True)
    check("bf16", out, lse, want, want_lse, float(vp.abs().max()))


# ---------------------------------------------------------------------------
# infinities and NaN in places that a row does not see
# ---------------------------------------------------------------------------

HIDDEN = {
    "prompt": dict(cached=[0], fresh=[200], hq=4, hk=2, d=64),
    "prompt_long_d128": dict(cached=[0, 0], fresh=[330, 75], hq=2, hk=2, d=128),
    "prompt_d256": dict(cached=[0], fresh=[90], hq=2, hk=1, d=256),
    "pages": dict(cached=[150, 0], fresh=[100, 77], hq=4, hk=2, d=128, page=16),
    "pages_odd": dict(cached=[61], fresh=[90], hq=2, hk=1, d=80, page=7),
    "few_new": dict(cached=[130, 63], fresh=[4, 3], hq=8, hk=2, d=128, page=32),
    "few_new_long": dict(cached=[9000], fresh=[5], hq=4, hk=1, d=64, page=16),
    "split_chunk": dict(cached=[3000], fresh=[40], hq=8, hk=2, d=128, page=16),
}


@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("name", sorted(HIDDEN))
def test_attn_hidden_nonfinite(env, name, dt):
    # One of the new tokens has keys that are NaN and values with infinities and NaN.  The rows
    # before it do not see them; the rows from it on have NaN weights.  Then finite keys with such
    # values: the rows from it on get infinities and NaN in those columns and no others.
    torch, tod = env
    c = HIDDEN[name]
    paged = "page" in c
    gen = torch.Generator(device="cuda").manual_seed(19)
    hq, hk, d, t = c["hq"], c["hk"], c["d"], sum(c["fresh"])
    starts = starts_of(torch, c["fresh"])
    at = 2 * c["fresh"][0] // 3  # the token, of the first sequence
    if paged:
        q, kp, vp, table = paged_case(torch, c, dt)
        p = c["cached"][0] + at
        where = (int(table[0, p // c["page"]]), slice(None), p % c["page"])
        want, want_lse = paged_want(c, q, kp, vp, table)

        def run(kx, vx):
            return tod.tod_attn_paged(
                q, kx, vx, torch.from_numpy(table).cuda(), starts,
                torch.tensor(c["cached"], dtype=torch.int32, device="cuda"),
                max_fresh=max(c["fresh"]), return_lse=True)
    else:
        q, kp, vp = (rows(torch, gen, dt, t, n, d) for n in (hq, hk, hk))
        where = (at,)
        q64, k64, v64 = (x.double().cpu().numpy() for x in (q, kp, vp))
        want, want_lse, b = np.zeros(q64.shape), np.zeros(q64.shape[:2]), 0
        for n in c["fresh"]:
            r = slice(b, b + n)
            want[r], want_lse[r] = plain_attention(q64[r], k64[r], v64[r], 0, True)
            b += n

        def run(kx, vx):
            return tod.tod_attn_prompt(q, kx, vx, starts, return_lse=True)

    v_max = float(vp.abs().max())
    kx, vx = kp.clone(), vp.clone()
    vx[where + (Ellipsis, 1)] = float("nan")
    vx[where + (Ellipsis, 4)] = float("inf")
    vx[where + (Ellipsis, d - 1)] = -float("inf")
    out, lse = run(kx, vx)
    hit = np.zeros(t, bool)
    hit[at:c["fresh"][0]] = True
    hit = torch.from_numpy(hit).cuda()
    o = out.float()
    assert torch.isnan(o[hit][..., 1]).all()
    assert (o[hit][..., 4] == math.inf).all() and (o[hit][..., d - 1] == -math.inf).all()
    fine = o.clone()
    w = torch.from_numpy(want).cuda()
    for col in (1, 4, d - 1):
        fine[hit, ..., col] = w[hit][..., col].float()
    check(dt, fine, lse, want, want_lse, v_max)
    kx[where] = float("nan")
    out, lse = run(kx, vx)
    assert torch.isnan(out[hit].float()).all() and torch.isnan(lse[hit]).all()
    check(dt, out[~hit], lse[~hit], want[~hit.cpu().numpy()], want_lse[~hit.cpu().numpy()], v_max)


# ---------------------------------------------------------------------------
# larger calls, against fp64 on the GPU
# ---------------------------------------------------------------------------

LARGE = {
    "prompts_d128": dict(cached=[0] * 5, fresh=[4001, 1, 900, 0, 2333], hq=32, hk=8, d=128),
    "prompts_d64": dict(cached=[0] * 3, fresh=[3000, 2999, 511], hq=24, hk=24, d=64),
    "prompts_d96": dict(cached=[0] * 2, fresh=[5003, 640], hq=16, hk=16, d=96),
    "prompts_d256": dict(cached=[0], fresh=[2100], hq=16, hk=4, d=256),
    "prompts_one_head": dict(cached=[0], fresh=[9000], hq=1, hk=1, d=64),
    "pages_d128": dict(cached=[3000, 10, 200], fresh=[1700, 1, 2900], hq=32, hk=8, d=128, page=16),
    "pages_odd": dict(cached=[300, 777], fresh=[2000, 2500], hq=28, hk=4, d=80, page=12),
    "pages_big": dict(cached=[1000], fresh=[4100], hq=32, hk=8, d=64, page=256),
    "one_chunk": dict(cached=[20011], fresh=[130], hq=16, hk=2, d=128, page=32),
    "tokens": dict(cached=[20000, 0, 511, 30001], fresh=[1, 3, 1, 2], hq=8, hk=2, d=128, page=16),
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dt", ["fp16", "bf16"])
@pytest.mark.parametrize("name", sorted(LARGE))
def test_attn_large(env, name, dt, causal):
    torch, tod = env
    c = LARGE[name]
    paged = "page" in c
    if paged and not causal:
        pytest.skip("attention over pages is causal")
    gen = torch.Generator(device="cuda").manual_seed(17)
    hq, hk, d, t = c["hq"], c["hk"], c["d"], sum(c["fresh"])
    starts = starts_of(torch, c["fresh"])
    if paged:
        q, kp, vp, table = paged_case(torch, c, dt)
        out, lse = tod.tod_attn_paged(
            q, kp, vp, torch.from_numpy(table).cuda(), starts,
            torch.tensor(c["cached"], dtype=torch.int32, device="cuda"),
            max_fresh=max(c["fresh"]), return_lse=True)
        v_max = float(vp.abs().max())
    else:
        qkv = rows(torch, gen, dt, t, hq + 2 * hk, d)
        q, k, v = (1.5 * qkv[:, :hq]).to(qkv.dtype), qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        out, lse = tod.tod_attn_prompt(q, k, v, starts, causal=causal, return_lse=True)
        v_max = float(v.abs().max())
    bound, at = (2.5 * U[dt] + 2e-4) * v_max, 0
    for r, (a, n) in enumerate(zip(c["cached"], c["fresh"])):
        for h in range(0, hq, max(1, hq // 4)):
            if paged:
                j = np.arange(a + n)
                pg = torch.from_numpy(table[r, j // c["page"]].astype(np.int64)).cuda()
                row = torch.from_numpy(j % c["page"]).cuda()
                kh, vh = (x[pg, h // (hq // hk), row].double() for x in (kp, vp))
            else:
                kh, vh = (x[at:at + n, h // (hq // hk)].double() for x in (k, v))
            s = q[at:at + n, h].double() @ kh.T / math.sqrt(d)
            if causal:
                pos = torch.arange(a + n, device="cuda")
                s = s.masked_fill(pos[None, :] > pos[a:a + n, None], -math.inf)
            z = torch.logsumexp(s, dim=1)
            want = torch.exp(s - z[:, None]) @ vh
            if n:
                err = float((out[at:at + n, h].double() - want).abs().max())
                assert err <= bound, (r, h, err, bound)
                off = float((lse[at:at + n, h].double() - z).abs().max())
                assert off <= 1e-4, (r, h, off)
        at += n
