"""One Workspace for calls that do not wait: on two streams at once, and in a graph that is replayed
after the Workspace has grown."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


class Case:
    """n new tokens of every sequence over a cache, whose partial results lie in the workspace."""

    def __init__(self, torch, tod, seed, cached, n, hq=8, hk=2, d=128, page=32):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def rows(*shape):
            return torch.randn(*shape, generator=gen, device="cuda").to(torch.float16)

        def ints(values):
            return torch.tensor(values, dtype=torch.int32, device="cuda")

        cols = -(-(max(cached) + n) // page)
        self.q = rows(n * len(cached), hq, d)
        self.kp, self.vp = (rows(len(cached) * cols, hk, page, d) for _ in range(2))
        self.table = torch.randperm(len(cached) * cols, generator=gen,
                                    device="cuda").to(torch.int32).view(len(cached), cols)
        self.starts = ints([n * i for i in range(len(cached) + 1)])
        self.cached, self.n, self.tod = ints(cached), n, tod

    def run(self, **kw):
        return self.tod.tod_attn_paged(self.q, self.kp, self.vp, self.table, self.starts,
                                       self.cached, max_fresh=self.n, return_lse=True, **kw)


def test_two_streams_at_once(env):
    torch, tod = env
    cases = [Case(torch, tod, 1, [20000], 40), Case(torch, tod, 2, [17000], 40)]
    want = [[x.clone() for x in c.run()] for c in cases]
    ws = tod.Workspace()
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, (c, s) in enumerate(zip(cases, streams)):
            got[i].append(c.run(workspace=ws, stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
    with torch.cuda.stream(streams[0]):
        first = ws.get_queued(256, cases[0].q.device)
    with torch.cuda.stream(streams[1]):
        second = ws.get_queued(256, cases[0].q.device)
    assert first.data_ptr() != second.data_ptr()


@pytest.mark.parametrize("warm", [True, False])
def test_graph_outlives_growth(env, warm):
    torch, tod = env
    small, large = Case(torch, tod, 3, [9000], 20), Case(torch, tod, 4, [9000] * 3, 60)
    want = [x.clone() for x in small.run()]
    ws = tod.Workspace()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        if warm:  # the buffer is there before the capture
            small.run(workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        got = small.run(workspace=ws)
    size = tod.tod_attn_workspace_size(8, 2, 128, 20, 1, 20)
    with torch.cuda.stream(s):
        large.run(workspace=ws)
        torch.cuda.synchronize()
        # whoever gets memory now keeps it to itself
        junk = [torch.full((size,), 0x5a, dtype=torch.uint8, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    for _ in range(3):
        for x in got:
            x.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all((x == 0x5a).all() for x in junk)


def test_waiting_calls_share_one_buffer(env):
    # The detectors wait for their work: one buffer, whatever the stream.
    torch, tod = env
    ws = tod.Workspace()
    dev = torch.device("cuda:0")
    a = ws.get(1 << 16, dev)
    with torch.cuda.stream(torch.cuda.Stream()):
        assert ws.get(1 << 10, dev).data_ptr() == a.data_ptr()
