"""Sequence operators on a stream of the caller's while the current stream is still busy: their
outputs and workspace are not memory that the current stream's work has yet to use."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


def _calls(torch, tod):
    gen = torch.Generator(device="cuda").manual_seed(9)

    def rows(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    n, hq, hk, d, page = 300, 8, 2, 64, 16
    q, k, v = rows(n, hq, d), rows(n, hk, d), rows(n, hk, d)
    starts = ints([0, n])
    kp, vp = rows(300, hk, page, d), rows(300, hk, page, d)
    table = torch.arange(300, dtype=torch.int32, device="cuda").view(1, 300)
    cached, fresh, free = ints([4000]), ints([n]), ints(list(range(300, 400)))
    one, own = ints([0, 1]), table.clone()
    return {
        "prompt": lambda **kw: tod.tod_attn_prompt(q, k, v, starts, return_lse=True, **kw),
        "paged": lambda **kw: tod.tod_attn_paged(q, kp, vp, table, starts, cached,
                                                 return_lse=True, **kw),
        "token": lambda **kw: tod.tod_attn_paged(q[:1], kp, vp, table, one, cached,
                                                 max_fresh=1, return_lse=True, **kw),
        "page_map": lambda **kw: tod.tod_page_map(cached, fresh, free, own, page, n, **kw),
    }


@pytest.mark.parametrize("name", ["prompt", "paged", "token", "page_map"])
def test_while_the_current_stream_is_busy(env, name):
    torch, tod = env
    call = _calls(torch, tod)[name]
    want = [x.clone() for x in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    # Tensors of many sizes that the current stream fills later, freed while that is still to come.
    sizes = [x.numel() * x.element_size() for x in want] + [1 << k for k in range(6, 26)]
    late = [torch.empty(max(s, 1), dtype=torch.uint8, device="cuda") for s in sizes * 3]
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)  # about 0.1 s
    for x in late:
        x.fill_(0x5a)
    del x, late
    got = call(stream=side)
    side.synchronize()
    early = [x.clone() for x in got]
    torch.cuda.synchronize()
    for a, b, c in zip(early, got, want):
        assert torch.equal(b, c), "written by the current stream's work"
        assert torch.equal(a, c)
