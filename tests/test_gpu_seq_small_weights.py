"""A key that outweighs each of very many others by e^16 to e^24: together they still count.

All other keys have the same score, gap below the key's, so that with N of them
  out = (v0 + N e^-gap v1) / (1 + N e^-gap),  lse = gap + ln(1 + N e^-gap).

Log sums, derived: they are sums of fp32 weights in which no addition loses more than it must
(additions of weights near 2^-24 to 1, one by one, would lose up to all of them: 8e-3 here), so that
what is left are a few roundings of numbers up to 35: 35 2^-22 = 1e-5; allowed are 1e-4.

Outputs, derived with u = 2^-11 for fp16 and 2^-8 for bf16 (half an ulp at the most): the output is
rounded, u |out| or, below fp16's normal range, 2^-25.  With v0 = 0 the weights are rounded all
alike, u |out|.  With v0 = v1 that hardly counts, but an accumulator that is near 1 from the start
takes N / 16 additions of 2^-24 at most, N 2^-28 <= 2^-11.  Weights below fp16's normal range are
rounded to a multiple of 2^-24; the kernels take them times 2^10 at least where the largest is 1, so
that each is off by at most 2^-35 and the sum by N 2^-35.  fp32 scores of up to 24 are off by
24 2^-23, the weights by that factor: 3e-6.  Together (2 u + 3e-6) |out| + 2^-25 + N 2^-35.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

# Keys, new tokens (0: a whole prompt) and the position of the key.  shared: as many sequences over
# the same pages, so that a wave reads all of a sequence's keys.
CASES = {
    "one_new": dict(keys=131072, fresh=1, at=0),
    "one_new_late": dict(keys=131072, fresh=1, at=130000),
    "one_new_whole": dict(keys=131072, fresh=1, at=0, shared=1024),
    "one_new_whole_late": dict(keys=120000, fresh=1, at=60001, shared=1024),
    "four_new": dict(keys=120011, fresh=4, at=70000),
    "four_new_whole": dict(keys=100000, fresh=4, at=3, shared=1024),
    "chunk": dict(keys=131072, fresh=60, at=5),
    "chunk_late": dict(keys=110003, fresh=60, at=90000),
    "prompt": dict(keys=100003, fresh=0, at=50000),
    "prompt_first": dict(keys=120000, fresh=0, at=0),
}
U = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
GAPS = [16.0, 17.4, 18.0, 24.0]


def attend(name, dtype, gap, v0):
    """(out [rows], lse [rows], keys that a row sees [rows], the gap as the type holds it)."""
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    c, d, dt = CASES[name], 64, getattr(torch, dtype)
    n, f, s = c["keys"], c["fresh"], c.get("shared", 1)
    k = torch.zeros(n, 1, d, dtype=dt, device="cuda")
    v = torch.ones(n, 1, d, dtype=dt, device="cuda")
    k[c["at"], 0, 0], v[c["at"]] = gap, v0
    gap = float(k[c["at"], 0, 0])
    q = torch.zeros(f * s if f else n, 1, d, dtype=dt, device="cuda")
    q[:, :, 0] = 8.0  # the scale is 1 / 8
    if f:
        page = 64
        pages = -(-n // page)
        room = torch.zeros(2, pages * page, d, dtype=dt, device="cuda")
        room[0, :n], room[1, :n] = k[:, 0], v[:, 0]
        kp, vp = room.view(2, pages, 1, page, d)
        table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(s, 1)
        starts = torch.arange(0, f * s + 1, f, dtype=torch.int32, device="cuda")
        cached = torch.full((s,), n - f, dtype=torch.int32, device="cuda")
        out, lse = tod.tod_attn_paged(q, kp, vp, table, starts, cached, max_fresh=f,
                                      return_lse=True)
        seen = torch.arange(n - f + 1, n + 1, dtype=torch.float64, device="cuda").repeat(s)
    else:
        out, lse = tod.tod_attn_prompt(
            q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), return_lse=True)
        seen = torch.arange(1, n + 1, dtype=torch.float64, device="cuda")
    assert (out == out[:, :, :1]).all()
    return out[:, 0, 0].double(), lse[:, 0].double(), seen, gap


@pytest.mark.parametrize("gap", GAPS)
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_log_sums(name, dtype, gap):
    import torch
    _, lse, seen, gap = attend(name, dtype, gap, 1.0)
    want = torch.where(seen > CASES[name]["at"],
                       gap + torch.log1p((seen - 1) * math.exp(-gap)), torch.log(seen))
    assert float((lse - want).abs().max()) <= 1e-4


@pytest.mark.parametrize("v0", [0.0, 1.0])
@pytest.mark.parametrize("gap", GAPS)
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_outputs(name, dtype, gap, v0):
    import torch
    out, _, seen, gap = attend(name, dtype, gap, v0)
    has = seen > CASES[name]["at"]  # the key is among those that the row sees
    others = (seen - 1) * math.exp(-gap)
    want = torch.where(has, (v0 + others) / (1 + others), 1.0)
    off = (out - want).abs()
    allowed = (2 * U[dtype] + 3e-6) * want + 2.0 ** -25 + torch.where(has, seen, 0.0) * 2.0 ** -35
    worst = int((off - allowed).argmax())
    assert (off <= allowed).all(), (worst, float(out[worst]), float(want[worst]))
