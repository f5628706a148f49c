"""Row layouts of the attention operators: widths between those that the kernels are made for, and
strides whose offsets pass 32 bits within a stage."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("d,wide", [(8, 64), (24, 64), (72, 128), (96, 128), (104, 128),
                                    (136, 256), (200, 256)])
@pytest.mark.parametrize("page", [0, 2, 16])
def test_narrow_rows_equal_padded_ones(env, page, d, wide, dtype):
    # Zeros behind q, k and v change no score and no output (they add exact zeros), so that the
    # results are the same bit by bit.  page 0: whole prompts.
    torch, tod = env
    gen = torch.Generator(device="cuda").manual_seed(d + page)
    dt = getattr(torch, dtype)
    hq, hk, n, past = 6, 2, 150, 171
    scale = 1 / math.sqrt(d)
    pad = lambda x: torch.nn.functional.pad(x, (0, wide - d)).contiguous()
    q = torch.randn(n, hq, d, generator=gen, device="cuda").to(dt)
    starts = torch.tensor([0, 1, n], dtype=torch.int32, device="cuda")
    if page == 0:
        k, v = (torch.randn(n, hk, d, generator=gen, device="cuda").to(dt) for _ in range(2))
        call = lambda q, k, v: tod.tod_attn_prompt(q, k, v, starts, scale=scale, return_lse=True)
    else:
        cols = -(-(past + n) // page)
        k, v = (torch.randn(2 * cols, hk, page, d, generator=gen, device="cuda").to(dt)
                for _ in range(2))
        table = torch.randperm(2 * cols, generator=gen, device="cuda").to(torch.int32).view(2, cols)
        cached = torch.tensor([100, past], dtype=torch.int32, device="cuda")
        call = lambda q, k, v: tod.tod_attn_paged(q, k, v, table, starts, cached, max_fresh=n,
                                                  scale=scale, return_lse=True)
    out, lse = call(q, k, v)
    want, want_lse = call(pad(q), pad(k), pad(v))
    assert out.shape == (n, hq, d)
    assert torch.isfinite(out).all()
    assert torch.equal(out, want[:, :, :d]) and torch.equal(lse, want_lse)


def test_row_strides_past_32_bits(env):
    # Rows of k that lie 2^30 bytes apart: eight of them are one load's.
    torch, tod = env
    n, d, apart = 40, 64, 1 << 29
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(n, 1, d, generator=gen, device="cuda").to(torch.float16)
               for _ in range(3))
    starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    want = tod.tod_attn_prompt(q, k, v, starts)
    room = torch.empty((n - 1) * apart + d, dtype=torch.float16, device="cuda")
    far = room.as_strided((n, 1, d), (apart, d, 1))
    for r in range(n):
        far[r] = k[r]
    got = tod.tod_attn_prompt(q, far, v, starts)
    got_v = tod.tod_attn_prompt(q, k, far, starts)
    want_v = tod.tod_attn_prompt(q, k, k, starts)
    assert torch.equal(got, want) and torch.equal(got_v, want_v)
