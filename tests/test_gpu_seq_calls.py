"""How the sequence operators are called: captured into a HIP graph, on another stream than the
tensors', twice with the same result, inside the workspace that they ask for, and what the binding
refuses."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


class Step:
    """One serving step of a small cache: lengths, table, new queries, keys and values."""

    def __init__(self, torch, cached, fresh, hq=4, hk=2, d=64, page=16, seed=1,
                 dtype="bfloat16"):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        dt = getattr(torch, dtype)
        n, t = len(cached), sum(fresh)
        need = [-(-(c + f) // page) for c, f in zip(cached, fresh)]
        have = [-(-c // page) for c in cached]
        total = sum(need) + 4
        ids = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
        self.table = torch.full((n, max(need) + 1), -1, dtype=torch.int32, device="cuda")
        at = 0
        for r in range(n):
            self.table[r, :have[r]] = ids[at:at + have[r]]
            at += have[r]
        self.free = ids[at:].contiguous()
        self.cached = torch.tensor(cached, dtype=torch.int32, device="cuda")
        self.fresh = torch.tensor(fresh, dtype=torch.int32, device="cuda")
        self.page, self.tokens, self.max_fresh = page, t, max(fresh)
        self.q, self.k, self.v = (
            torch.randn(t, h, d, generator=gen, device="cuda").to(dt) for h in (hq, hk, hk))
        self.kp, self.vp = (
            torch.randn(total, hk, page, d, generator=gen, device="cuda").to(dt)
            for _ in range(2))

    def run(self, tod, stream=None, workspace=None):
        row_start, slot, pos, used = tod.tod_page_map(self.cached, self.fresh, self.free,
                                                      self.table, self.page, self.tokens,
                                                      stream=stream)
        tod.tod_page_write(self.k, self.v, slot, self.kp, self.vp, stream=stream)
        out, lse = tod.tod_attn_paged(self.q, self.kp, self.vp, self.table, row_start, self.cached,
                                      max_fresh=self.max_fresh, stream=stream,
                                      workspace=workspace, return_lse=True)
        return out, lse, slot, pos, used


CASES = {
    "tokens": dict(cached=[100, 3, 77, 1500], fresh=[1, 1, 1, 1]),
    "mixed": dict(cached=[100, 0, 77, 900], fresh=[1, 60, 1, 33]),
    "split_chunk": dict(cached=[2000], fresh=[50], hq=8),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_graph_replays(env, name):
    torch, tod = env
    s = Step(torch, **CASES[name])
    ws = tod.Workspace()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(2):
            s.run(tod, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = s.run(tod, workspace=ws)
    for i in range(4):  # new contents each time, eager work and waits in between
        gen = torch.Generator(device="cuda").manual_seed(50 + i)
        for x in (s.q, s.k, s.v):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in got]
        want = s.run(tod)
        torch.cuda.synchronize()
        for a, b in zip(replayed, want):
            assert torch.equal(a, b)


def test_on_another_stream(env):
    torch, tod = env
    s = Step(torch, [100, 0, 77, 900], [1, 60, 1, 33])
    want = [x.clone() for x in s.run(tod)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        got = s.run(tod, stream=side)  # its workspace is released while the work is under way
        junk = [torch.full((1 << 20,), 7.0, device="cuda") for _ in range(8)]
        side.synchronize()
        del junk
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("name", sorted(CASES))
def test_same_result_twice(env, name):
    torch, tod = env
    s = Step(torch, **CASES[name])
    first = [x.clone() for x in s.run(tod)]
    for _ in range(3):
        for a, b in zip(s.run(tod), first):
            assert torch.equal(a, b)


@pytest.mark.parametrize("name", sorted(CASES))
def test_keeps_to_its_workspace(env, name):
    torch, tod = env
    s = Step(torch, **CASES[name])
    want = [x.clone() for x in s.run(tod)]

    class Guarded:
        def get(self, nbytes, device):
            self.n = nbytes
            self.buf = torch.full((nbytes + 4096,), 0x5a, dtype=torch.uint8, device=device)
            return self.buf[:nbytes]

    ws = Guarded()
    got = s.run(tod, workspace=ws)  # begun on 0x5a bytes: nothing in it is taken as zero
    torch.cuda.synchronize()
    assert (ws.buf[ws.n:] == 0x5a).all()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_prompt_equals_pages(env):
    # A whole prompt, and the same tokens in chunks of a growing cache.
    torch, tod = env
    gen = torch.Generator(device="cuda").manual_seed(4)
    n, hq, hk, d, page = 150, 4, 2, 64, 16
    q, k, v = (torch.randn(n, h, d, generator=gen, device="cuda").to(torch.float16)
               for h in (hq, hk, hk))
    starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    want = tod.tod_attn_prompt(q, k, v, starts).float()
    kp, vp = (torch.zeros(12, hk, page, d, dtype=torch.float16, device="cuda") for _ in range(2))
    table = torch.full((1, 11), -1, dtype=torch.int32, device="cuda")
    free = torch.arange(12, dtype=torch.int32, device="cuda").flip(0).contiguous()
    done, got = 0, []
    for step in (40, 1, 1, 60, 17, 1, 30):
        c = torch.tensor([done], dtype=torch.int32, device="cuda")
        f = torch.tensor([step], dtype=torch.int32, device="cuda")
        row_start, slot, pos, used = tod.tod_page_map(c, f, free, table, page, step)
        free = free[int(used[0]):]
        assert int(used[1]) == 0 and pos.tolist() == list(range(done, done + step))
        r = slice(done, done + step)
        tod.tod_page_write(k[r], v[r], slot, kp, vp)
        got.append(tod.tod_attn_paged(q[r], kp, vp, table, row_start, c, max_fresh=step))
        done += step
    # two roundings of fp16 weights and outputs of values up to 5
    assert float((torch.cat(got).float() - want).abs().max()) <= 5 * 4 * 2.0 ** -11


def test_long_offsets(env):
    # A cache whose rows pass 2^31 elements: its last pages.
    torch, tod = env
    page, hk, d, n_pages = 128, 8, 128, 17000  # 2.2 * 10^9 elements each
    kp = torch.zeros(n_pages, hk, page, d, dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    gen = torch.Generator(device="cuda").manual_seed(6)
    n = 200
    k, v = (torch.randn(n, hk, d, generator=gen, device="cuda").to(kp.dtype) for _ in range(2))
    q = torch.randn(1, 2 * hk, d, generator=gen, device="cuda").to(kp.dtype)
    pages = torch.tensor([n_pages - 1, n_pages - 3], dtype=torch.int64, device="cuda")
    j = torch.arange(n, device="cuda")
    tod.tod_page_write(k, v, pages[j // page] * page + j % page, kp, vp)
    out, lse = tod.tod_attn_paged(q, kp, vp, pages.to(torch.int32).view(1, 2),
                                  torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
                                  torch.tensor([n - 1], dtype=torch.int32, device="cuda"),
                                  max_fresh=1, return_lse=True)
    for h in range(2 * hk):
        s = (k[:, h // 2].double() @ q[0, h].double()) / math.sqrt(d)
        want = torch.softmax(s, 0) @ v[:, h // 2].double()
        assert float((out[0, h].double() - want).abs().max()) <= 2.5 * 2.0 ** -9 * 5
        assert abs(float(lse[0, h]) - float(torch.logsumexp(s, 0))) <= 1e-4


def test_lengths_that_lie(env):
    # Lengths and starts out of range stay inside the buffers and leave other rows right.
    torch, tod = env
    s = Step(torch, [100, 40], [3, 2])
    want = [x.clone() for x in s.run(tod)]
    row_start = torch.tensor([0, 3, 1 << 30], dtype=torch.int32, device="cuda")
    out, lse = tod.tod_attn_paged(s.q, s.kp, s.vp, s.table, row_start, s.cached,
                                  max_fresh=s.max_fresh, return_lse=True)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    wild = torch.tensor([100, (1 << 31) - 1], dtype=torch.int32, device="cuda")
    row_start = torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda")
    out, _ = tod.tod_attn_paged(s.q, s.kp, s.vp, s.table, row_start, wild, max_fresh=s.max_fresh,
                                return_lse=True)
    assert torch.equal(out[:3], want[0][:3]) and torch.isfinite(out).all()


def test_binding_refusals(env):
    torch, tod = env
    q = torch.zeros(6, 4, 64, dtype=torch.float16, device="cuda")
    k = torch.zeros(6, 2, 64, dtype=torch.float16, device="cuda")
    rs = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    ok = tod.tod_attn_prompt(q, k, k, rs)
    assert (ok == 0).all()
    for bad in (lambda: tod.tod_attn_prompt(q.float(), k.float(), k.float(), rs),
                lambda: tod.tod_attn_prompt(q, k.to(torch.bfloat16), k, rs),
                lambda: tod.tod_attn_prompt(q, k, k, rs.long()),
                lambda: tod.tod_attn_prompt(q, k, k, rs.cpu()),
                lambda: tod.tod_attn_prompt(torch.zeros_like(q).view(6, 64, 4).transpose(1, 2), k, k,
                                            rs)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: tod.tod_attn_prompt(q, k[:5], k[:5], rs),
                lambda: tod.tod_attn_prompt(q, k[:1].expand(6, 2, 64), k, rs),
                lambda: tod.tod_attn_prompt(q, k, k, rs, scale=0.0),
                lambda: tod.tod_attn_prompt(q, k, k, rs, out=torch.zeros_like(k))):
        with pytest.raises(ValueError):
            bad()
    wide = torch.zeros(6, 4, 68, dtype=torch.float16, device="cuda")
    with pytest.raises(tod.TodError) as e:  # a stride of 68 elements
        tod.tod_attn_prompt(wide[..., :64], k, k, rs)
    assert e.value.status == tod.TOD_ERR_UNSUPPORTED and "strides" in str(e.value)
    with pytest.raises(tod.TodError) as e:  # 8 bytes into an allocation
        buf = torch.zeros(6 * 2 * 64 + 4, dtype=torch.float16, device="cuda")
        tod.tod_attn_prompt(q, buf[4:].view(6, 2, 64), k, rs)
    assert e.value.status == tod.TOD_ERR_INVALID_ARG and "aligned" in str(e.value)
    with pytest.raises(tod.TodError) as e:
        Step(torch, [100, 3], [1, 1]).run(tod, workspace=tod.FixedWorkspace(256))
    assert e.value.status == tod.TOD_ERR_WORKSPACE


def test_one_row_tensors_of_any_stride(env):
    # torch leaves the stride of a dimension of size 1 to chance.
    torch, tod = env
    q = torch.randn(1, 2, 64, device="cuda").half().as_strided((1, 2, 64), (3, 64, 1))
    k = torch.randn(1, 1, 64, device="cuda").half().as_strided((1, 1, 64), (5, 7, 1))
    rs = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    out = tod.tod_attn_prompt(q, k, k, rs)
    assert torch.equal(out, k.expand(1, 2, 64))


def test_example(env):
    torch, _ = env
    from examples import score_prompts
    score, drift = score_prompts.main()
    # every odd prompt lies farther from the fitted ones than any usual prompt
    assert float(score[24:].min()) > float(score[:24].max())
    # normed fp16 states of two layers, up to 4 or so: a few roundings apart
    assert drift <= 0.1
