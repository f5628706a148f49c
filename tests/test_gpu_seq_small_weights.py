"""A key that outweighs each of very many others by e^16 to e^24: together they still count.

All other keys have the same score, gap below the key's, so that with N of them
  out = (v0 + N e^-gap v1) / (1 + N e^-gap).
Tolerance, derived: the weights and the output are rounded to the input type (u = 2^-11 for fp16,
2^-9 for bf16), which is at worst the same relative error of all N: 2 u |out| with v0 = 0 or
v0 = v1.  Weights below fp16's normal range are rounded to a multiple of 2^-24; the kernels take
them times 2^10 at least where the largest is 1, so that each is off by at most 2^-35 and the sum
by N 2^-35 |v1|.  fp32 scores of up to 24 are off by 24 2^-23, the weights by that factor: 3e-6.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -9}

# The last position of the sequence, the new tokens, and the position of the key.
CASES = {
    "one_new": dict(keys=131072, fresh=1, at=0),
    "one_new_late": dict(keys=131072, fresh=1, at=130000),
    "four_new": dict(keys=120011, fresh=4, at=70000),
    "chunk": dict(keys=131072, fresh=60, at=5),
    "chunk_late": dict(keys=110003, fresh=60, at=90000),
    "prompt": dict(keys=100003, fresh=0, at=50000),
    "prompt_first": dict(keys=120000, fresh=0, at=0),
}


@pytest.mark.parametrize("v0", [0.0, 1.0])
@pytest.mark.parametrize("gap", [16.0, 17.4, 18.0, 24.0])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_many_small_weights(name, dtype, gap, v0):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    c, d, dt = CASES[name], 64, getattr(torch, dtype)
    n, f = c["keys"], c["fresh"]
    k = torch.zeros(n, 1, d, dtype=dt, device="cuda")
    v = torch.ones(n, 1, d, dtype=dt, device="cuda")
    k[c["at"], 0, 0], v[c["at"]] = gap, v0
    gap = float(k[c["at"], 0, 0])  # as the type holds it
    q = torch.zeros(f if f else n, 1, d, dtype=dt, device="cuda")
    q[:, :, 0] = 8.0  # the scale is 1 / 8
    if f:
        page = 64
        pages = -(-n // page)
        room = torch.zeros(2, pages * page, d, dtype=dt, device="cuda")
        room[0, :n], room[1, :n] = k[:, 0], v[:, 0]
        kp, vp = room.view(2, pages, 1, page, d)
        out, lse = tod.tod_attn_paged(
            q, kp, vp, torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages),
            torch.tensor([0, f], dtype=torch.int32, device="cuda"),
            torch.tensor([n - f], dtype=torch.int32, device="cuda"), max_fresh=f, return_lse=True)
        seen = torch.arange(n - f + 1, n + 1, dtype=torch.float64, device="cuda")
    else:
        out, lse = tod.tod_attn_prompt(
            q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), return_lse=True)
        seen = torch.arange(1, n + 1, dtype=torch.float64, device="cuda")
    small = math.exp(-gap)
    has = seen > c["at"]  # the key among them
    others = torch.where(has, seen - 1, 0.0) * small
    want = torch.where(has, (v0 + others) / (1 + others), 1.0)
    want_lse = torch.where(has, gap + torch.log1p(others), torch.log(seen))
    off = (out[:, 0].double() - want[:, None]).abs().amax(1)
    allowed = (2 * U[dtype] + 3e-6) * want + torch.where(has, seen, 0.0) * 2.0 ** -35
    worst = int((off - allowed).argmax())
    assert (off <= allowed).all(), (worst, float(out[worst, 0, 0]), float(want[worst]))
    assert float((lse[:, 0].double() - want_lse).abs().max()) <= 1e-4
