"""Attention over pages for batches: more sequences than a wave has lanes, runs of idle ones, pairs of
a sequence and a head that are cut over several waves, chunks whose keys are split beside single
tokens, and rows past the last sequence.  Against 64 bits.

Tolerance, derived: u = 2^-11 for fp16 and 2^-8 for bf16 (half an ulp at the most).  The weights and
the output are rounded to the input type, each by u of itself at most, and everything between is
fp32 with scores off by less than 1e-4: (2 u + 2e-4) max|v|.  The log sums: 1e-4.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


def mixed(n, top, fresh, idle=()):
    """n sequences of up to top cached tokens; idle: ranges without new tokens."""
    cached = [(i * 7919 + 13) % (top + 1) for i in range(n)]
    new = [fresh[i % len(fresh)] for i in range(n)]
    for a, b in idle:
        new[a:b] = [0] * (b - a)
    return cached, new


CASES = {
    # sequences: 64 and 65, with idle ones between; a segment of several a lane
    "seqs_64": dict(lens=mixed(64, 300, [1]), hq=4, hk=2, d=64, page=16),
    "seqs_65": dict(lens=mixed(65, 300, [1, 0, 2]), hq=4, hk=2, d=64, page=16),
    "seqs_130": dict(lens=mixed(130, 200, [1, 1, 3], [(5, 80)]), hq=4, hk=1, d=128, page=32),
    "seqs_1000": dict(lens=mixed(1000, 150, [1, 2, 0, 1], [(100, 190), (400, 640)]), hq=2, hk=1,
                      d=64, page=16),
    "all_but_last_idle": dict(lens=mixed(300, 90, [1], [(0, 299)]), hq=2, hk=2, d=64, page=8),
    "all_but_first_idle": dict(lens=mixed(300, 90, [1], [(1, 300)]), hq=2, hk=2, d=64, page=8),
    "all_idle_but_padding": dict(lens=mixed(90, 90, [0]), hq=2, hk=2, d=64, page=8, pad=7),
    # pairs: 65 and more, cut over several waves, of fewer and more rows than a join has waves
    "pairs_65": dict(lens=mixed(65, 2500, [1]), hq=1, hk=1, d=64, page=64),
    "pairs_260_rows_2": dict(lens=mixed(130, 1500, [1]), hq=4, hk=2, d=64, page=16),
    "pairs_130_rows_24": dict(lens=mixed(65, 2000, [1, 5, 6]), hq=8, hk=2, d=128, page=32),
    "pairs_72_rows_32": dict(lens=mixed(72, 1800, [2, 1]), hq=16, hk=1, d=80, page=16),
    "pairs_80_d256": dict(lens=mixed(40, 1200, [1, 3]), hq=8, hk=2, d=256, page=16),
    "pairs_33_d256_rows_1": dict(lens=mixed(33, 900, [1]), hq=1, hk=1, d=256, page=16),
    # rows past the last sequence in a call of single tokens
    "padded_tokens": dict(lens=mixed(10, 200, [1]), hq=4, hk=2, d=64, page=16, pad=1500),
    "padded_seqs": dict(lens=mixed(100, 100, [1, 0]), hq=6, hk=2, d=72, page=16, pad=31),
    "padded_chunks": dict(lens=mixed(5, 200, [1, 50]), hq=4, hk=2, d=64, page=16, pad=300),
    # chunks of several sequences over long caches, split, beside single tokens that are read
    "split_two": dict(lens=([3000, 2000], [40, 33]), hq=8, hk=2, d=128, page=16),
    "split_three_and_tokens": dict(lens=([3000, 900, 0, 2500, 77, 4000, 1800],
                                         [40, 1, 1, 70, 2, 45, 1]), hq=8, hk=2, d=128, page=16),
    "split_uneven": dict(lens=([5000, 600, 40, 3100], [33, 130, 90, 1]), hq=4, hk=1, d=64, page=32),
    "split_d256": dict(lens=([2600, 1900, 50], [40, 36, 1]), hq=4, hk=1, d=256, page=16),
    "split_odd": dict(lens=([2600, 0, 1900, 50], [50, 0, 60, 1]), hq=7, hk=1, d=96, page=7),
    "many_tokens_one_chunk": dict(lens=([3000] + [(i * 37) % 400 for i in range(70)],
                                        [64] + [1] * 70), hq=8, hk=2, d=64, page=16),
}


@pytest.mark.parametrize("hint", [True, False])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_batches(env, name, dtype, hint):
    torch, tod = env
    c, dt = CASES[name], getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(31)
    (cached, fresh), hq, hk, d, page = c["lens"], c["hq"], c["hk"], c["d"], c["page"]
    n, t = len(cached), sum(fresh)
    lens = [a + b for a, b in zip(cached, fresh)]
    need = [-(-m // page) for m in lens]

    def rows(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(dt)

    q = rows(t + c.get("pad", 0), hq, d)
    kp, vp = rows(sum(need) + 3, hk, page, d), rows(sum(need) + 3, hk, page, d)
    ids = np.random.default_rng(31).permutation(sum(need) + 3).astype(np.int32)
    table = np.full((n, max(need) + 1), -1, np.int32)
    at = 0
    for r in range(n):
        table[r, :need[r]] = ids[at:at + need[r]]
        at += need[r]
    table = torch.from_numpy(table).cuda()

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    starts = np.concatenate([[0], np.cumsum(fresh)]).tolist()
    room = torch.full((q.numel() + 2048,), 7.0, dtype=dt, device="cuda")
    out = room[1024:-1024].view(q.shape)
    got, lse = tod.tod_attn_paged(q, kp, vp, table, ints(starts), ints(cached),
                                  max_fresh=max(max(fresh), 1) if hint else None, out=out,
                                  return_lse=True)
    assert got.data_ptr() == out.data_ptr()
    assert (room[:1024] == 7).all() and (room[-1024:] == 7).all()
    assert (out[t:] == 0).all() and (lse[t:] == -math.inf).all()
    if t == 0:
        return
    # All sequences at once: keys as [n, longest], new tokens as [n, most].
    longest, most = max(lens), max(fresh)
    j = torch.arange(longest, device="cuda")
    page_of = table.long().gather(1, (j // page).expand(n, longest).clamp(max=table.shape[1] - 1))
    page_of = page_of.clamp(min=0)
    row_of = (j % page).expand(n, longest)
    i = torch.arange(most, device="cuda").expand(n, most)
    first, f, past = (torch.tensor(x, device="cuda")[:, None] for x in (starts[:-1], fresh, cached))
    real = i < f
    token = torch.where(real, first + i, 0)
    hidden = j[None, None, :] > (past + i)[:, :, None]
    v_max = float(vp.abs().max())
    for h in range(hq):
        g = h * hk // hq
        k, v = kp[page_of, g, row_of].double(), vp[page_of, g, row_of].double()
        s = (q[token, h].double() @ k.transpose(1, 2).contiguous()) / math.sqrt(d)
        s = s.masked_fill(hidden, -math.inf)
        z = torch.logsumexp(s, 2)
        want = torch.exp(s - z[:, :, None]) @ v
        err = float((out[token, h].double() - want)[real].abs().max())
        assert err <= (2 * U[dtype] + 2e-4) * v_max, (h, err)
        assert float((lse[token, h].double() - z)[real].abs().max()) <= 1e-4, h
