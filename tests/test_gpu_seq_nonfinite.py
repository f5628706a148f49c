"""Infinite values that a row sees: out = sum p v / sum p is their sum in that column, since every
p = exp(s) is positive, wherever the key lies and however small its weight is.  Other columns, and
rows that do not see the key, keep their finite results.

Tolerance of the finite results as derived for random rows: the weights and the output are rounded
to the input type (u = 2^-11 for fp16, 2^-8 for bf16, half an ulp at the most) and everything between
is fp32, so that an output is off by at most 2 u max|v| plus the scores' own 1e-4 max|v|; allowed are
2 u max|v| + 2e-4 max|v|.  The log sums: 1e-4 + 1e-6 |lse|.
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


# at: the positions of the first sequence that hold such values.
CASES = {
    "only_token": dict(cached=[0], fresh=[1], hq=4, hk=2, d=64, page=16, at=[0]),
    "one_new_at_itself": dict(cached=[100, 30], fresh=[1, 1], hq=8, hk=2, d=128, page=16, at=[100]),
    "one_new_cached": dict(cached=[100, 30], fresh=[1, 1], hq=8, hk=2, d=128, page=16, at=[3]),
    "one_new_two": dict(cached=[300, 30], fresh=[1, 1], hq=2, hk=2, d=64, page=7, at=[3, 290]),
    "one_new_pieces": dict(cached=[20000, 9], fresh=[1, 1], hq=4, hk=1, d=128, page=16,
                           at=[64, 15000]),
    "one_new_pieces_d256": dict(cached=[9000, 9], fresh=[1, 1], hq=2, hk=2, d=256, page=32,
                                at=[7777]),
    "four_new_cached": dict(cached=[130, 63], fresh=[4, 1], hq=4, hk=2, d=80, page=32, at=[17]),
    "four_new_both": dict(cached=[130, 63], fresh=[4, 3], hq=8, hk=2, d=128, page=32,
                          at=[17, 132]),
    "four_new_pieces": dict(cached=[9000], fresh=[4], hq=4, hk=1, d=64, page=16, at=[40, 9002]),
    "many_pairs": dict(cached=[900] + [70] * 79, fresh=[1] * 80, hq=4, hk=2, d=64, page=16,
                       at=[500]),
    "chunk": dict(cached=[150, 0], fresh=[100, 77], hq=4, hk=2, d=128, page=16, at=[20, 200]),
    "chunk_odd_page": dict(cached=[61], fresh=[90], hq=2, hk=1, d=80, page=7, at=[5]),
    "split_chunk": dict(cached=[3000], fresh=[40], hq=8, hk=2, d=128, page=16, at=[1, 2500]),
    "prompt": dict(cached=[0, 0], fresh=[330, 75], hq=4, hk=2, d=128, at=[2, 200]),
    "prompt_d256": dict(cached=[0], fresh=[190], hq=2, hk=1, d=256, at=[33]),
    "prompt_split": dict(cached=[0], fresh=[1500], hq=1, hk=1, d=64, at=[10, 900]),
    "open_prompt": dict(cached=[0, 0], fresh=[330, 75], hq=4, hk=2, d=64, at=[300], open=True),
    "open_prompt_split": dict(cached=[0], fresh=[1500], hq=1, hk=1, d=96, at=[900], open=True),
}


# The key's score against the others': usual, so low that an fp16 weight is 0, and so low that an
# fp32 weight is.
@pytest.mark.parametrize("low", [0, 40, 1000])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_visible_infinities(env, name, dtype, low):
    torch, tod = env
    c = CASES[name]
    dt = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(23)
    hq, hk, d, page, n = c["hq"], c["hk"], c["d"], c.get("page"), len(c["cached"])
    t, causal = sum(c["fresh"]), not c.get("open")
    lens = [a + b for a, b in zip(c["cached"], c["fresh"])]

    def rows(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(dt)

    q = rows(t, hq, d)
    k, v = [rows(m, hk, d) for m in lens], [rows(m, hk, d) for m in lens]
    if low:  # an element of every query that the key answers with -low nats
        q[:, :, 0] = 4.0
        for x in k:
            x[:, :, 0] = 0.0
        for p in c["at"]:
            k[0][p] = 0.0
            k[0][p, :, 0] = -low * math.sqrt(d) / 4.0
    clean = [x.clone() for x in v]
    cols = {1: [INF] * len(c["at"]), d - 1: [-INF] * len(c["at"]),
            4: [INF, -INF] if len(c["at"]) == 2 else [NAN]}
    for col, values in cols.items():
        for p, x in zip(c["at"], values):
            v[0][p, :, col] = x
            clean[0][p, :, col] = 0.0
    v_max = max(float(x.abs().max()) for x in clean)
    starts = torch.tensor([sum(c["fresh"][:i]) for i in range(n + 1)], dtype=torch.int32,
                          device="cuda")
    if page:
        need = [-(-m // page) for m in lens]
        ids = torch.randperm(sum(need) + 3, generator=gen, device="cuda")
        kp, vp = rows(len(ids), hk, page, d), rows(len(ids), hk, page, d)
        table = torch.full((n, max(need)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for r in range(n):
            mine = ids[at:at + need[r]]
            table[r, :need[r]] = mine.to(torch.int32)
            j = torch.arange(lens[r], device="cuda")
            kp[mine[j // page], :, j % page] = k[r]
            vp[mine[j // page], :, j % page] = v[r]
            at += need[r]
        cached = torch.tensor(c["cached"], dtype=torch.int32, device="cuda")
        out, lse = tod.tod_attn_paged(q, kp, vp, table, starts, cached, max_fresh=max(c["fresh"]),
                                      return_lse=True)
    else:
        out, lse = tod.tod_attn_prompt(q, torch.cat(k), torch.cat(v), starts, causal=causal,
                                       return_lse=True)
    bound, at = (2 * U[dtype] + 2e-4) * v_max, 0
    for r in range(n):
        f, m = c["fresh"][r], lens[r]
        pos = torch.arange(m, device="cuda")
        hidden = pos[None, :] > pos[m - f:, None] if causal else torch.zeros(
            f, m, dtype=torch.bool, device="cuda")
        for h in range(hq):
            s = q[at:at + f, h].double() @ k[r][:, h * hk // hq].double().T / math.sqrt(d)
            s = s.masked_fill(hidden, -INF)
            z = torch.logsumexp(s, dim=1)
            want = torch.exp(s - z[:, None]) @ clean[r][:, h * hk // hq].double()
            got = out[at:at + f, h].double()
            if r == 0:
                for col, values in cols.items():
                    total = torch.zeros(f, dtype=torch.float64, device="cuda")
                    for p, x in zip(c["at"], values):
                        total += torch.where(hidden[:, p], 0.0, x)
                    odd = ~torch.isfinite(total)
                    assert torch.equal(got[odd, col].isnan(), total[odd].isnan()), (h, col)
                    real = odd & ~total.isnan()
                    assert torch.equal(got[real, col], total[real]), (h, col)
                    got[odd, col] = want[odd, col]
            assert float((got - want).abs().max()) <= bound, (r, h)
            off = (lse[at:at + f, h].double() - z).abs() - 1e-6 * z.abs()
            assert float(off.max()) <= 1e-4, (r, h)
        at += f
