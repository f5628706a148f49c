"""The sequence operators compute forward results only: with gradients enabled they refuse tensors
that require one, whose gradient would be lost without a word."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def calls():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    gen = torch.Generator(device="cuda").manual_seed(1)

    def rows(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    q, k, v, kp, vp = rows(5, 4, 64), rows(5, 2, 64), rows(5, 2, 64), rows(3, 2, 8, 64), rows(3, 2, 8, 64)
    starts, table, cached = ints([0, 5]), ints([[2, 0]]), ints([4])
    slot = torch.arange(5, device="cuda")
    return torch, {
        "prompt": (lambda t: tod.tod_attn_prompt(t["q"], t["k"], t["v"], starts, out=t["out"]),
                   dict(q=q, k=k, v=v, out=torch.empty_like(q))),
        "paged": (lambda t: tod.tod_attn_paged(t["q"], t["kp"], t["vp"], table, starts, cached),
                  dict(q=q, kp=kp, vp=vp)),
        "write": (lambda t: tod.tod_page_write(t["k"], t["v"], slot, t["kp"], t["vp"]),
                  dict(k=k, v=v, kp=kp, vp=vp)),
    }


@pytest.mark.parametrize("name,which", [
    ("prompt", "q"), ("prompt", "k"), ("prompt", "v"), ("prompt", "out"), ("paged", "q"),
    ("paged", "kp"), ("paged", "vp"), ("write", "k"), ("write", "v"), ("write", "kp"),
    ("write", "vp")])
def test_refused_with_gradients(calls, name, which):
    torch, table = calls
    call, tensors = table[name]
    mine = {n: x.clone() for n, x in tensors.items()}
    mine[which].requires_grad_()
    with pytest.raises(ValueError, match="requires a gradient"):
        call(mine)
    mine = {n: x.clone() for n, x in tensors.items()}
    want = call(mine)
    mine = {n: x.clone() for n, x in tensors.items()}
    mine[which].requires_grad_()
    with torch.no_grad():
        got = call(mine)
    assert want is None or torch.equal(got, want)
