"""The page map at the largest number of tokens that its entry point takes: 2^31 - 1."""
import pytest

pytestmark = pytest.mark.gpu


def test_page_map_of_most_tokens():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    tokens, page, cols = (1 << 31) - 1, 65536, 32767  # the table ends 65,535 positions early
    fresh = [tokens - 70000, 69000]                   # and 1,000 rows are past the last sequence

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    cached, new = ints([0, 5]), ints(fresh)
    table = torch.full((2, cols), -1, dtype=torch.int32, device="cuda")
    table[1, 0] = 40000
    free = torch.arange(cols + 3, dtype=torch.int32, device="cuda")
    starts, used = ints([7] * 3), torch.full((2,), 7, dtype=torch.int64, device="cuda")
    slot = torch.full((tokens,), 7, dtype=torch.int64, device="cuda")
    pos = torch.full((tokens,), 7, dtype=torch.int32, device="cuda")
    st = tod.raw_library().tod_page_map(
        cached.data_ptr(), new.data_ptr(), 2, free.data_ptr(), free.numel(), page,
        table.data_ptr(), cols, tokens, torch.cuda.current_stream().cuda_stream,
        starts.data_ptr(), slot.data_ptr(), pos.data_ptr(), used.data_ptr())
    assert st == tod.TOD_OK
    torch.cuda.synchronize()
    pages = -(-fresh[0] // page)
    assert starts.tolist() == [0, fresh[0], sum(fresh)]
    assert used.tolist() == [pages + 1, 0]
    assert table[0].tolist() == list(range(pages)) + [-1] * (cols - pages)
    assert table[1, :3].tolist() == [40000, pages, -1]
    step = 1 << 28
    for a in range(0, fresh[0], step):  # the first sequence's slots are its positions
        want = torch.arange(a, min(a + step, fresh[0]), device="cuda")
        assert torch.equal(slot[a:a + len(want)], want)
        assert torch.equal(pos[a:a + len(want)].long(), want)
    at = torch.arange(5, 5 + fresh[1], device="cuda")
    want = torch.where(at < page, 40000 * page, (pages - 1) * page) + at
    assert torch.equal(slot[fresh[0]:sum(fresh)], want)
    assert torch.equal(pos[fresh[0]:sum(fresh)].long(), at)
    assert (slot[sum(fresh):] == -1).all() and (pos[sum(fresh):] == -1).all()
