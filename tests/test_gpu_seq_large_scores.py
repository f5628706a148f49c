"""Scores of up to 5e7 in magnitude, rising, falling and level along the keys: far beyond what a
softmax needs, but what fp16 and bf16 tensors hold.

Scores that differ, differ by thousands, so that the largest that a row sees takes all of its weight;
level ones share it.  Tolerance, derived: the weights of a row are equal but for their roundings (u =
2^-11 for fp16, 2^-8 for bf16), and so is the output: 2 u max|v|.  Log sums: a score's roundings,
4 2^-24 of it, and 1e-4.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
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
        "steps": top * torch.floor(i / 100) / 7,
        "small_then_large": torch.where(i < 400, 0.0, top),
        "large_then_small": torch.where(i < 400, top, 0.0),
        "low_then_small": torch.where(i < 400, -top, 0.0),
    }[name]


NAMES = ["level", "level_low", "rising", "falling", "rising_through_0", "falling_through_0", "saw",
         "steps", "small_then_large", "large_then_small", "low_then_small"]


@pytest.mark.parametrize("kind", ["prompt", "open_prompt", "chunk", "tokens"])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("name", NAMES)
def test_large_scores(name, dtype, kind):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    dt, d, n = getattr(torch, dtype), 64, KEYS
    gen = torch.Generator(device="cuda").manual_seed(3)
    v = torch.randn(n, 1, d, generator=gen, device="cuda").to(dt)
    k = torch.zeros(n, 1, d, dtype=dt, device="cuda")
    k[:, 0, 0] = pattern(torch, name).to(dt)
    f = {"chunk": 90, "tokens": 3}.get(kind, n)
    q = torch.zeros(f, 1, d, dtype=dt, device="cuda")
    q[:, 0, 0] = 8192.0  # the scale is 1 / 8
    starts = torch.tensor([0, f], dtype=torch.int32, device="cuda")
    if kind in ("chunk", "tokens"):
        kp, vp = k.view(-1, 1, 20, d).contiguous(), v.view(-1, 1, 20, d).contiguous()
        out, lse = tod.tod_attn_paged(
            q, kp, vp, torch.arange(n // 20, dtype=torch.int32, device="cuda")[None],
            starts, torch.tensor([n - f], dtype=torch.int32, device="cuda"), max_fresh=f,
            return_lse=True)
    else:
        out, lse = tod.tod_attn_prompt(q, k, v, starts, causal=kind == "prompt", return_lse=True)
    s = (1024.0 * k[:, 0, 0].double()).expand(f, n)
    if kind != "open_prompt":
        pos = torch.arange(n, device="cuda")
        s = s.masked_fill(pos[None, :] > pos[n - f:, None], -math.inf)
    z = torch.logsumexp(s, 1)
    want = torch.softmax(s, 1) @ v[:, 0].double()
    err = float((out[:, 0].double() - want).abs().max())
    assert err <= 2 * U[dtype] * float(v.abs().max()), err
    assert ((lse[:, 0].double() - z).abs() <= 1e-4 + 2.0 ** -22 * z.abs()).all()
