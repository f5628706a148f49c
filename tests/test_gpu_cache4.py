"""The rotating appends and the 4-bit cache on the GPU against plain implementations in 64 bits.

Tolerances, derived.  Rotated 16-bit rows: x cos - y sin with cos and sin right to 2^-23 (the angle
is reduced in 64 bits and rounded to 32, the series is one of 32 bits), products and their sum rounded
(2^-24 each): off by at most 2^-22 (|x| + |y|), then rounded to the type: half a step of the value, and
half of its smallest step.  With no element larger than m the tests allow u |want| + 2^-21 m + tiny.
What a 4-bit cache holds is compared for
equality: scales and codes come from 64-bit arithmetic, and of the few thousand blocks here none lies
within 2^-50 of a border but those that lie on it exactly.

Attention: as derived for 16-bit pages, whose weights are rounded the same way, with the values that
the cache stands for: the weights p are rounded to the input type (u), the output too, everything
between is fp32: 2 u max|v|; fp32 scores move the weights by less than 1e-4.  Allowed:
(2.5 u + 2e-4) max|v| and, for the log sums, 1e-4 + 1e-6 |lse|.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}  # half a step, relative to the value
TINY = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -134}
LIMITS = {"fp16": (-23, 13), "bf16": (-125, 125)}
VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


def dtype_of(torch, name):
    return {"fp16": torch.float16, "bf16": torch.bfloat16}[name]


def f64(x):
    return x.detach().cpu().double().numpy()


# ---------------------------------------------------------------------------
# plain implementations, numpy fp64
# ---------------------------------------------------------------------------

def plain_rotate(x, pos, rates, interleaved):
    """x [tokens, heads, dim] fp64, rates fp32."""
    out, half = x.copy(), len(rates)
    a = np.outer(pos.astype(np.float64), rates.astype(np.float64))[:, None, :]
    i = np.arange(half)
    lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    out[..., lo] = x[..., lo] * np.cos(a) - x[..., hi] * np.sin(a)
    out[..., hi] = x[..., lo] * np.sin(a) + x[..., hi] * np.cos(a)
    return out


def plain_encode(x, name):
    """(codes uint8 [.., dim / 2], scales uint8 [.., dim / 32]) of x [.., dim] fp64."""
    lo, hi = LIMITS[name]
    b = x.reshape(x.shape[:-1] + (-1, 32))
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(-1)
    e = np.full(top.shape, lo)
    for k in range(lo, hi):  # the smallest exponent that holds the block
        e = np.where(top > 7.0 * 2.0 ** k, k + 1, e)
    mag = np.minimum(np.abs(b) / np.exp2(e.astype(np.float64))[..., None], 6.0)
    dist = np.abs(mag[..., None] - VALUES)
    near = dist == dist.min(-1, keepdims=True)
    even = near & (np.arange(8) % 2 == 0)  # of two as near, the even code
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = (code + 8 * (b < 0)).astype(np.uint8)
    code[bad] = 0
    code = code.reshape(x.shape)
    return code[..., ::2] | code[..., 1::2] << 4, np.where(bad, 255, e + 127).astype(np.uint8)


def plain_decode(codes, scales, name=None):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    v = np.where(c & 8, -1.0, 1.0) * VALUES[c & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    v = v * np.repeat(s, 32, axis=-1)
    if name == "fp16":  # numbers of the type
        with np.errstate(over="ignore"):
            v = v.astype(np.float16).astype(np.float64)
    return v


def plain_attention(q, k, v, first, scale):
    """q [n, hq, d], k, v [len, hk, d] fp64; query i stands at position first + i."""
    n, hq, d = q.shape
    length, hk, _ = k.shape
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    for h in range(hq):
        kh, vh = k[:, h // (hq // hk)], v[:, h // (hq // hk)]
        s = scale * (q[:, h] @ kh.T)
        for i in range(n):
            seen = min(length, first + i + 1)
            if seen <= 0:
                continue
            top = s[i, :seen].max()
            p = np.exp(s[i, :seen] - top)
            out[i, h] = (p @ vh[:seen]) / p.sum()
            lse[i, h] = top + math.log(p.sum())
    return out, lse


# ---------------------------------------------------------------------------
# appends and reads
# ---------------------------------------------------------------------------

APPENDS = {
    "step": dict(tokens=5, heads=8, kv=2, dim=128, r=128, page=16),
    "pairs": dict(tokens=37, heads=4, kv=4, dim=64, r=64, page=16, interleaved=True),
    "part": dict(tokens=19, heads=6, kv=2, dim=96, r=48, page=7),
    "pairs_part": dict(tokens=9, heads=3, kv=1, dim=64, r=22, page=3, interleaved=True),
    "odd_half": dict(tokens=23, heads=2, kv=1, dim=64, r=36, page=5),
    "one_pair": dict(tokens=3, heads=1, kv=1, dim=32, r=2, page=1),
    "none": dict(tokens=11, heads=2, kv=2, dim=32, r=0, page=4),
    "wide": dict(tokens=70, heads=5, kv=1, dim=256, r=256, page=48),
    "one_token": dict(tokens=1, heads=8, kv=8, dim=160, r=160, page=16),
    "far": dict(tokens=64, heads=4, kv=2, dim=128, r=128, page=16, pos=2 ** 31 - 1),
    "missing": dict(tokens=300, heads=2, kv=2, dim=64, r=64, page=16, missing=0.4),
    "many": dict(tokens=2500, heads=2, kv=1, dim=64, r=32, page=64),
}


def append_case(torch, case, name, dim=None):
    c = dict(dict(pos=200000, interleaved=False, missing=0.0), **case)
    dim = dim or c["dim"]
    g = torch.Generator(device="cuda").manual_seed(5)
    t, hq, hk, page = c["tokens"], c["heads"], c["kv"], c["page"]
    spread = torch.exp(2 * torch.randn(t, hq + 2 * hk, 1, generator=g, device="cuda"))
    x = (spread * torch.randn(t, hq + 2 * hk, dim, generator=g, device="cuda")).to(
        dtype_of(torch, name))
    pages = -(-t // page) + 3
    slot = torch.randperm(pages * page, generator=g, device="cuda")[:t].contiguous()
    slot[torch.rand(t, generator=g, device="cuda") < c["missing"]] = -1
    pos = torch.randint(-3, c["pos"], (t,), generator=g, device="cuda", dtype=torch.int32)
    if t > 3:
        pos[1], slot[2] = 0, pages * page  # no turn at all; a slot past the cache
    r = c["r"]
    rates = 10000.0 ** (-torch.arange(r // 2, device="cuda").float() / max(1, r // 2))
    return c, x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:], pos, slot, rates, pages


def check_rotated(name, got, x, want, r):
    off = np.abs(f64(got) - want)
    size = np.abs(x).max(-1, keepdims=True)
    bound = U[name] * np.abs(want) + 2.0 ** -21 * size + TINY[name]
    assert (off <= bound).all(), "off by %.3g" % (off - bound).max()
    assert np.array_equal(f64(got)[..., r:], x[..., r:])


@pytest.mark.parametrize("name", ["fp16", "bf16"])
@pytest.mark.parametrize("case", sorted(APPENDS))
def test_append(env, case, name):
    torch, tod = env
    for dim in (None, 72) if case == "odd_half" else (None,):
        c, q, k, v, pos, slot, rates, pages = append_case(torch, APPENDS[case], name, dim)
        shape = (pages, k.shape[1], c["page"], k.shape[2])
        kp = torch.full(shape, 7.0, dtype=k.dtype, device="cuda")
        vp = torch.full(shape, 9.0, dtype=k.dtype, device="cuda")
        out = tod.tod_page_append(q, k, v, pos, slot, rates, kp, vp, interleaved=c["interleaved"])
        torch.cuda.synchronize()
        turn = (pos.cpu().numpy(), rates.cpu().numpy(), c["interleaved"])
        check_rotated(name, out, f64(q), plain_rotate(f64(q), *turn), c["r"])
        at = slot.cpu().numpy()
        ok = (at >= 0) & (at < pages * c["page"])
        rows = kp.transpose(1, 2).reshape(-1, *k.shape[1:])
        check_rotated(name, rows[at[ok]], f64(k)[ok], plain_rotate(f64(k), *turn)[ok], c["r"])
        vrows = vp.transpose(1, 2).reshape(-1, *k.shape[1:])
        assert torch.equal(vrows[at[ok]], v[torch.from_numpy(ok).cuda()])
        left = np.setdiff1d(np.arange(len(rows)), at[ok])
        assert (f64(rows)[left] == 7.0).all() and (f64(vrows)[left] == 9.0).all()


@pytest.mark.parametrize("name", ["fp16", "bf16"])
@pytest.mark.parametrize("case", sorted(APPENDS))
def test_append4_and_read4(env, case, name):
    torch, tod = env
    c, q, k, v, pos, slot, rates, pages = append_case(torch, APPENDS[case], name)
    cache = tod.Cache4.zeros(pages, k.shape[1], c["page"], k.shape[2])
    cache.k_codes.fill_(0x5a)
    cache.v_scales.fill_(77)
    out = tod.tod_page_append4(q, k, v, pos, slot, rates, cache, interleaved=c["interleaved"])
    torch.cuda.synchronize()
    turn = (pos.cpu().numpy(), rates.cpu().numpy(), c["interleaved"])
    check_rotated(name, out, f64(q), plain_rotate(f64(q), *turn), c["r"])
    at = slot.cpu().numpy()
    ok = (at >= 0) & (at < pages * c["page"])
    held = [plain_encode(plain_rotate(f64(k), *turn), name), plain_encode(f64(v), name)]
    got = [[x.cpu().numpy().swapaxes(1, 2).reshape(-1, k.shape[1], x.shape[3]) for x in pair]
           for pair in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales))]
    for (codes, scales), (have_codes, have_scales) in zip(held, got):
        assert np.array_equal(scales[ok], have_scales[at[ok]])
        assert np.array_equal(codes[ok], have_codes[at[ok]])
    left = np.setdiff1d(np.arange(pages * c["page"]), at[ok])
    assert (got[0][0][left] == 0x5a).all() and (got[1][1][left] == 77).all()
    for kind in ("fp16", "bf16") if name == "fp16" else ("bf16",):
        rk, rv = tod.tod_page_read4(cache, slot, dtype_of(torch, kind))
        torch.cuda.synchronize()
        for x, (codes, scales) in zip((rk, rv), held):
            want = plain_decode(codes, scales)
            want[~ok] = 0
            assert np.array_equal(f64(x), want)


@pytest.mark.parametrize("name", ["fp16", "bf16"])
def test_append4_borders(env, name):
    """Every border of two codes and of two scales, each type's largest and smallest values, and
    values that are not finite."""
    torch, tod = env
    big = 65504.0 if name == "fp16" else 3.3895e38
    small = 2.0 ** -24 if name == "fp16" else 2.0 ** -133
    rows = []
    for top in (7.0, 7.03125, 6.0, 3.5, 1.75, 1.765625):
        for sign in (1, -1):
            marks = [0, .25, .25 + 2 ** -8, .75, .75 - 2 ** -8, 1.25, 1.75, 2.5, 3.5, 5, 5.0625, 6, 7]
            rows.append([top] + [sign * m * (1 if top > 3.5 else top / 7) for m in marks])
    rows += [[big], [-big, big / 2, 1.0], [small, -small, 3 * small], [0.0], [-0.0],
             [big, big * 0.75, big * 0.4], [float("inf"), 1.0], [float("nan"), 2.0], [-float("inf")]]
    x = torch.zeros(len(rows), 1, 32)
    for i, r in enumerate(rows):
        x[i, 0, :len(r)] = torch.tensor(r)
    x = x.to(dtype_of(torch, name)).cuda()
    n = len(rows)
    cache = tod.Cache4.zeros(n, 1, 1, 32)
    slot = torch.arange(n, device="cuda")
    zero = torch.zeros(n, dtype=torch.int32, device="cuda")
    tod.tod_page_append4(x, x, x, zero, slot, torch.ones(16, device="cuda"), cache)
    codes, scales = plain_encode(f64(x), name)
    for c, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)):
        if c is cache.k_codes:  # a turn by nothing: 0 times an infinity of the pair is a NaN
            keep = np.isfinite(f64(x)).all((1, 2))
        else:
            keep = np.ones(n, bool)
        assert np.array_equal(s.cpu().numpy()[keep, 0], scales[keep])
        assert np.array_equal((c.cpu().numpy()[keep, 0] & 0x77), codes[keep] & 0x77)
    assert (cache.k_scales.cpu().numpy()[~np.isfinite(f64(x)).all((1, 2))] == 255).all()
    k, v = tod.tod_page_read4(cache, slot, x.dtype)
    want = plain_decode(codes, scales)
    got = f64(v)
    assert np.array_equal(got, want, equal_nan=True)
    finite = np.isfinite(f64(x)).all((1, 2))
    assert np.isnan(got[~finite]).all() and np.isfinite(got[finite]).all()


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

PAGED = {
    "one_token": dict(cached=[0], fresh=[1], heads=1, kv=1, dim=64, page=16),
    "tokens": dict(cached=[0, 5, 31, 32, 33, 63, 64, 65, 500], fresh=[1] * 9, heads=8, kv=2, dim=128,
                   page=16),
    "wide_group": dict(cached=[0, 100, 257], fresh=[1] * 3, heads=80, kv=2, dim=64, page=16),
    "group_of_nine": dict(cached=[3, 100, 257], fresh=[1] * 3, heads=18, kv=2, dim=96, page=48),
    "group_of_16": dict(cached=[3, 1000, 257], fresh=[1] * 3, heads=32, kv=2, dim=128, page=16),
    "group_of_17": dict(cached=[64, 127], fresh=[1] * 2, heads=17, kv=1, dim=128, page=32),
    "narrow": dict(cached=[1, 40, 200], fresh=[1, 2, 1], heads=6, kv=3, dim=32, page=5),
    "dim_96": dict(cached=[10, 130], fresh=[1, 3], heads=4, kv=1, dim=96, page=16),
    "dim_160": dict(cached=[10, 130, 0], fresh=[1, 5, 50], heads=4, kv=2, dim=160, page=7),
    "dim_256": dict(cached=[70, 300, 0], fresh=[1, 7, 40], heads=4, kv=2, dim=256, page=16),
    "page_of_one": dict(cached=[3, 40, 0], fresh=[1, 2, 40], heads=4, kv=2, dim=64, page=1),
    "few_new": dict(cached=[100, 0, 33, 7], fresh=[2, 8, 5, 1], heads=4, kv=1, dim=128, page=16),
    "chunk": dict(cached=[37], fresh=[150], heads=8, kv=2, dim=128, page=16),
    "chunk_split": dict(cached=[1800], fresh=[40], heads=4, kv=1, dim=128, page=32),
    "chunk_narrow": dict(cached=[0, 70], fresh=[90, 33], heads=2, kv=2, dim=32, page=16),
    "chunk_64": dict(cached=[0, 600], fresh=[200, 33], heads=4, kv=2, dim=64, page=16),
    "mixed": dict(cached=[0, 200, 90, 500, 0, 31], fresh=[70, 1, 60, 1, 1, 0], heads=8, kv=2, dim=128,
                  page=16),
    "idle": dict(cached=[0, 20, 4, 9], fresh=[0, 1, 0, 0], heads=4, kv=2, dim=64, page=16, pad=3),
    "padded": dict(cached=[9, 20], fresh=[3, 1], heads=4, kv=2, dim=64, page=8, pad=70),
    "long": dict(cached=[9000, 20], fresh=[1, 1], heads=8, kv=1, dim=128, page=64),
    "many": dict(cached=[(37 * i) % 300 for i in range(150)], fresh=[1] * 150, heads=2, kv=1, dim=64,
                 page=16),
    "holes": dict(cached=[100, 200], fresh=[2, 60], heads=4, kv=2, dim=128, page=16, holes=True),
    "short_table": dict(cached=[100, 37], fresh=[2, 60], heads=4, kv=2, dim=64, page=16, cols=4),
    "negative": dict(cached=[-5, 9], fresh=[4, 1], heads=4, kv=2, dim=64, page=16),
    "scaled": dict(cached=[50], fresh=[2], heads=4, kv=2, dim=64, page=16, scale=0.7),
}


class Paged:
    """A case's tensors; rows of the cache filled by encoding normal rows."""

    def __init__(self, torch, tod, case, name, seed=3, no_fresh=False):
        c = dict(dict(pad=0, holes=False, scale=None, cols=0), **case)
        self.case, self.name, self.torch = c, name, torch
        rng = np.random.default_rng(seed)
        page, hk, d = c["page"], c["kv"], c["dim"]
        ends = [max(a, 0) + b for a, b in zip(c["cached"], c["fresh"])]
        need = [-(-e // page) for e in ends]
        cols = c["cols"] or max(need) + 2
        n_pages = sum(need) + 3
        ids = rng.permutation(n_pages)
        self.table = np.full((len(need), cols), -1, np.int32)
        at = 0
        for r, n in enumerate(need):
            self.table[r, :min(n, cols)] = ids[at:at + min(n, cols)]
            at += n
        if c["holes"]:
            self.table[0, 1], self.table[1, 3], self.table[1, 0] = -1, n_pages, 2 ** 31 - 1
        codes = [plain_encode(rng.standard_normal((n_pages, hk, page, d)), name) for _ in range(2)]
        self.codes = codes
        self.cache = tod.Cache4(*[torch.from_numpy(np.ascontiguousarray(x)).cuda()
                                  for pair in codes for x in pair])
        t = sum(c["fresh"]) + c["pad"]
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.q = (1.5 * torch.randn(t, c["heads"], d, generator=g, device="cuda")).to(
            dtype_of(torch, name))
        self.start = np.concatenate([[0], np.cumsum(c["fresh"])])
        dev = dict(dtype=torch.int32, device="cuda")
        self.args = (torch.tensor(self.table, **dev), torch.tensor(self.start, **dev),
                     torch.tensor(c["cached"], **dev))

    def rows(self, r, length):
        """k, v [length, kv, dim] of a request, in 64 bits."""
        page, out = self.case["page"], []
        for codes, scales in self.codes:
            x = plain_decode(codes, scales, self.name)
            flat = np.zeros((length,) + (x.shape[1], x.shape[3]))
            for j in range(length):
                id = self.table[r, j // page]
                if 0 <= id < len(x):
                    flat[j] = x[id, :, j % page]
            out.append(flat)
        return out

    def want(self):
        c, q = self.case, f64(self.q)
        out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
        scale = c["scale"] or 1 / math.sqrt(c["dim"])
        v_max = 0.0
        for r, (a, n) in enumerate(zip(c["cached"], c["fresh"])):
            room = self.table.shape[1] * c["page"]
            first = min(max(a, 0), room)
            length = min(first + n, room)
            k, v = self.rows(r, length)
            s = slice(self.start[r], self.start[r] + n)
            out[s], lse[s] = plain_attention(q[s], k, v, first, scale)
            if length:
                v_max = max(v_max, np.abs(v).max())
        return out, lse, v_max


def check(name, out, lse, want, want_lse, v_max):
    out, lse = f64(out), f64(lse)
    assert np.isfinite(out).all()
    err = np.abs(out - want).max()
    assert err <= (2.5 * U[name] + 2e-4) * v_max, "out off by %.3g" % err
    seen = np.isfinite(want_lse)
    assert (lse[~seen] == -np.inf).all() and (out[~seen] == 0).all()
    off = np.abs(lse[seen] - want_lse[seen]) - 1e-6 * np.abs(want_lse[seen])
    assert seen.sum() == 0 or off.max() <= 1e-4, "lse off by %.3g" % off.max()


@pytest.mark.parametrize("name", ["fp16", "bf16"])
@pytest.mark.parametrize("case", sorted(PAGED))
def test_attn_paged4(env, case, name):
    torch, tod = env
    p = Paged(torch, tod, PAGED[case], name)
    ws = tod.Workspace()
    for fresh in (None, max(1, max(PAGED[case]["fresh"]))):
        out, lse = tod.tod_attn_paged4(p.q, p.cache, *p.args, max_fresh=fresh, workspace=ws,
                                       scale=p.case["scale"], return_lse=True)
        torch.cuda.synchronize()
        check(name, out, lse, *p.want())


def test_attn_paged4_strided_queries(env):
    torch, tod = env
    p = Paged(torch, tod, PAGED["mixed"], "bf16")
    wide = torch.zeros(p.q.shape[0], p.q.shape[1] + 4, p.q.shape[2], dtype=p.q.dtype, device="cuda")
    wide[:, 2:-2] = p.q
    out = tod.tod_attn_paged4(wide[:, 2:-2], p.cache, *p.args)
    assert torch.equal(out, tod.tod_attn_paged4(p.q, p.cache, *p.args))


def test_attn_paged4_repeats_itself(env):
    torch, tod = env
    p = Paged(torch, tod, PAGED["mixed"], "fp16")
    first = tod.tod_attn_paged4(p.q, p.cache, *p.args, return_lse=True)
    for _ in range(5):
        again = tod.tod_attn_paged4(p.q, p.cache, *p.args, return_lse=True)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
