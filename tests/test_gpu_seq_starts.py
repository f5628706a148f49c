"""Row starts that do not ascend: such a call stays inside its buffers, whatever it computes, and
the next call with starts in order is right."""
import pytest

pytestmark = pytest.mark.gpu

STARTS = {
    "back_to_zero": [0, 500, 600, 0, 700],
    "descending": [700, 600, 400, 130, 0],
    "negative": [0, -5, 300, -(1 << 31), 700],
    "past_the_end": [0, 1 << 30, 200, (1 << 31) - 1, 100],
    "all_at_the_end": [700] * 150,
    "zigzag": [(i * 389) % 701 for i in range(200)],
}


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


@pytest.mark.parametrize("heads", [1, 4, 40])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("name", sorted(STARTS))
def test_starts_that_do_not_ascend(env, name, paged, heads):
    torch, tod = env
    gen = torch.Generator(device="cuda").manual_seed(2)
    tokens, d, page, guard = 700, 64, 16, 4096
    n = len(STARTS[name]) - 1

    def rows(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(torch.float16)

    q = rows(tokens, heads, d)
    if paged:
        cols = 60
        kp, vp = rows(n * cols, 1, page, d), rows(n * cols, 1, page, d)
        table = torch.arange(n * cols, dtype=torch.int32, device="cuda").view(n, cols)
        cached = torch.full((n,), 30, dtype=torch.int32, device="cuda")
    else:
        k, v = rows(tokens, 1, d), rows(tokens, 1, d)
    room = torch.full((tokens * heads * d + 2 * guard,), 7.0, dtype=torch.float16, device="cuda")
    out = room[guard:-guard].view(tokens, heads, d)

    def run(starts):
        row_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        if paged:
            return tod.tod_attn_paged(q, kp, vp, table, row_start, cached, out=out)
        return tod.tod_attn_prompt(q, k, v, row_start, out=out)

    fine = [min(tokens, i * (tokens // n + 1)) for i in range(n + 1)]
    want = run(fine).clone()
    run(STARTS[name])
    torch.cuda.synchronize()
    assert (room[:guard] == 7).all() and (room[-guard:] == 7).all()
    assert torch.isfinite(out).all()
    assert torch.equal(run(fine), want)
