"""bf16 values near the type's largest: out = sum p v / sum p is no larger than they are, and with
weights of at most 1 of which few count, their sum stays in range too.

Tolerance, derived: all values that a row sees have the same magnitude and sign, so that the output
is that value; the weights' roundings (u = 2^-8 each at the most) and its own: 2 u v, and 1e-4 v for
the scores'.
"""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["prompt", "open_prompt", "chunk", "split_chunk", "tokens"])
@pytest.mark.parametrize("rise", [2.0, 5.0, 5.5, 9.0, 20.0])
def test_large_values(kind, rise):
    # One key of score 0 among many that do not count, and later one that outweighs it by e^rise.
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    n, d, page, large = (4000 if kind == "split_chunk" else 400), 64, 16, 1.0e38
    k = torch.full((n, 1, d), 0.0, dtype=torch.bfloat16, device="cuda")
    k[:, 0, 0] = -40.0
    k[3, 0, 0], k[n // 2, 0, 0] = 0.0, rise
    v = torch.full((n, 1, d), large, dtype=torch.bfloat16, device="cuda")
    v[:, :, 1] = -large
    f = {"chunk": 60, "split_chunk": 40, "tokens": 2}.get(kind, n)
    q = torch.zeros(f, 1, d, dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = 8.0  # the scale is 1 / 8
    starts = torch.tensor([0, f], dtype=torch.int32, device="cuda")
    if "prompt" in kind:
        # (the first rows see keys of -40 alone, up to 3 of them, all alike)
        out = tod.tod_attn_prompt(q, k, v, starts, causal=kind == "prompt")
    else:
        kp, vp = k.view(-1, 1, page, d), v.view(-1, 1, page, d)
        table = torch.arange(n // page, dtype=torch.int32, device="cuda")[None]
        cached = torch.tensor([n - f], dtype=torch.int32, device="cuda")
        out = tod.tod_attn_paged(q, kp, vp, table, starts, cached, max_fresh=f)
    want = v[:f, 0].double()
    assert torch.isfinite(out).all()
    assert ((out[:, 0].double() - want).abs() <= (2.0 ** -7 + 1e-4) * large).all()
