"""A step without new tokens: the sequence operators return empty results and touch nothing."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


@pytest.mark.parametrize("own_stream", [False, True])
@pytest.mark.parametrize("n_seq", [0, 1, 5])
def test_no_new_tokens(env, n_seq, own_stream):
    torch, tod = env
    stream = torch.cuda.Stream() if own_stream else None
    gen = torch.Generator(device="cuda").manual_seed(4)

    def rows(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(torch.float16)

    cached = torch.arange(10, 10 + n_seq, dtype=torch.int32, device="cuda")
    fresh = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
    free = torch.arange(4, dtype=torch.int32, device="cuda")
    table = torch.arange(3 * n_seq, dtype=torch.int32, device="cuda").view(n_seq, 3)
    kp, vp = rows(20, 2, 8, 64), rows(20, 2, 8, 64)
    before = [x.clone() for x in (table, kp, vp)]
    torch.cuda.synchronize()
    row_start, slot, pos, used = tod.tod_page_map(cached, fresh, free, table, 8, 0, stream=stream)
    q, k = rows(0, 4, 64), rows(0, 2, 64)
    tod.tod_page_write(k, k, slot, kp, vp, stream=stream)
    outs = [tod.tod_attn_prompt(q, k, k, row_start, return_lse=True, stream=stream),
            tod.tod_attn_paged(q, kp, vp, table, row_start, cached, return_lse=True,
                               stream=stream),
            (tod.tod_attn_prompt(q, k, k, row_start, causal=False, out=q.clone(), stream=stream),
             None)]
    torch.cuda.synchronize()
    assert row_start.dtype == torch.int32 and row_start.tolist() == [0] * (n_seq + 1)
    assert slot.dtype == torch.int64 and slot.shape == (0,)
    assert pos.dtype == torch.int32 and pos.shape == (0,)
    assert used.dtype == torch.int64 and used.tolist() == [0, 0]
    for out, lse in outs:
        assert out.shape == (0, 4, 64) and out.dtype == q.dtype
        assert lse is None or (lse.shape == (0, 4) and lse.dtype == torch.float32)
    for a, b in zip((table, kp, vp), before):
        assert torch.equal(a, b)


def test_no_room_for_new_tokens(env):
    # Lengths that do not fit into 0 tokens are left out, as they are with any other number.
    torch, tod = env
    cached = torch.tensor([3, 9], dtype=torch.int32, device="cuda")
    fresh = torch.tensor([4, -2], dtype=torch.int32, device="cuda")
    free = torch.arange(4, dtype=torch.int32, device="cuda")
    table = torch.full((2, 3), -1, dtype=torch.int32, device="cuda")
    row_start, _, _, used = tod.tod_page_map(cached, fresh, free, table, 8, 0)
    assert row_start.tolist() == [0, 0, 0] and used.tolist() == [0, 4]
    assert (table == -1).all()


def test_arguments_are_still_checked(env):
    torch, tod = env
    q = torch.zeros(0, 4, 64, dtype=torch.float16, device="cuda")
    rs = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        tod.tod_attn_prompt(q, q.float(), q, rs)
    with pytest.raises(ValueError):
        tod.tod_attn_prompt(q, q[:, :2], q, rs)
    with pytest.raises(tod.TodError):
        tod.tod_page_map(rs, rs, rs, rs.view(2, 1), 8, -1)
