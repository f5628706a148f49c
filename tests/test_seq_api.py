"""CPU checks of the sequence operators' entry points: what they refuse, on the host and before
any HIP call, and their workspace sizes."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def tod():
    from paper_2110_14007_amd import tod
    return tod


FAKE = ctypes.c_void_p(0x100000)  # never dereferenced: validation rejects first
OFF4, OFF2 = ctypes.c_void_p(0x100004), ctypes.c_void_p(0x100002)
OFF8 = ctypes.c_void_p(0x100008)


def _map(tod, cached=FAKE, fresh=FAKE, n_seq=4, free=FAKE, n_free=8, page=16, table=FAKE, cols=4,
         tokens=9, row_start=FAKE, slot=FAKE, pos=FAKE, used=FAKE):
    return tod.raw_library().tod_page_map(cached, fresh, n_seq, free, n_free, page, table, cols,
                                          tokens, None, row_start, slot, pos, used)


@pytest.mark.parametrize("kw,status", [
    (dict(cached=None), 1), (dict(fresh=None), 1), (dict(table=None), 1),
    (dict(row_start=None), 1), (dict(slot=None), 1), (dict(free=None), 1),
    (dict(n_seq=0), 1), (dict(tokens=0), 1), (dict(cols=0), 1), (dict(n_free=-1), 1),
    (dict(page=0), 1), (dict(page=65537), 1), (dict(cached=OFF2), 1), (dict(slot=OFF4), 1),
    (dict(used=OFF4), 1), (dict(tokens=1 << 31), 4), (dict(n_seq=1 << 31), 4),
    (dict(cols=1 << 28), 4),
])
def test_page_map_refusals(tod, kw, status):
    assert _map(tod, **kw) == status
    assert tod.last_error() != ""


def _write(tod, k=FAKE, v=FAKE, tokens=5, heads=2, dim=64, kr=0, kh=0, vr=0, vh=0, slot=FAKE,
           kp=FAKE, vp=FAKE, pages=4, page=16):
    return tod.raw_library().tod_page_write(k, v, tokens, heads, dim, kr, kh, vr, vh, slot, kp, vp,
                                            pages, page, None)


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(slot=None), 1), (dict(kp=None), 1),
    (dict(vp=None), 1), (dict(tokens=0), 1), (dict(heads=0), 1), (dict(dim=0), 1),
    (dict(dim=12), 4), (dict(kr=-8), 1), (dict(vh=-64), 1), (dict(kr=132), 4), (dict(vh=4), 4),
    (dict(pages=0), 1), (dict(page=0), 1), (dict(pages=1 << 30), 4), (dict(tokens=1 << 31), 4),
    (dict(k=OFF8), 1), (dict(vp=OFF8), 1), (dict(slot=OFF4), 1),
])
def test_page_write_refusals(tod, kw, status):
    assert _write(tod, **kw) == status
    assert tod.last_error() != ""


def attn(tod, heads=8, kv_heads=2, dim=64, precision=2, **kw):
    a = tod.tod_attn()
    tod.raw_library().tod_default_attn(ctypes.byref(a), heads, kv_heads, dim, precision)
    for name, v in kw.items():
        setattr(a, name, v)
    return a


def _prompt(tod, a, q=FAKE, k=FAKE, v=FAKE, tokens=50, row_start=FAKE, n_seq=3, ws=FAKE,
            ws_bytes=1 << 40, out=FAKE, lse=FAKE):
    return tod.raw_library().tod_attn_prompt(ctypes.byref(a) if a is not None else None, q, k, v,
                                             tokens, row_start, n_seq, ws, ws_bytes, None, out, lse)


def _paged(tod, a, q=FAKE, kp=FAKE, vp=FAKE, pages=9, page=16, table=FAKE, cols=4, row_start=FAKE,
           cached=FAKE, n_seq=3, tokens=50, fresh=50, ws=FAKE, ws_bytes=1 << 40, out=FAKE,
           lse=FAKE):
    return tod.raw_library().tod_attn_paged(ctypes.byref(a) if a is not None else None, q, kp, vp,
                                            pages, page, table, cols, row_start, cached, n_seq,
                                            tokens, fresh, ws, ws_bytes, None, out, lse)


BOTH = [
    (dict(struct_size=8), 1), (dict(precision=0), 4), (dict(precision=1), 4),
    (dict(precision=7), 1), (dict(heads=0), 1), (dict(kv_heads=0), 1), (dict(dim=0), 1),
    (dict(kv_heads=3), 1), (dict(dim=20), 4), (dict(dim=264), 4), (dict(heads=65538), 4),
    (dict(causal=2), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(q_row=-8), 1), (dict(q_row=4), 4), (dict(k_head=100), 4),
]


@pytest.mark.parametrize("kw,status", BOTH)
def test_attention_options_refused(tod, kw, status):
    a = attn(tod, **kw)
    for call in (_prompt, _paged):
        assert call(tod, a) == status
        assert tod.last_error() != ""
    assert tod.raw_library().tod_attn_workspace_size(ctypes.byref(a), 50, 3, 50) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(row_start=None), 1),
    (dict(ws=None), 1), (dict(out=None), 1), (dict(tokens=0), 1), (dict(n_seq=0), 1),
    (dict(tokens=1 << 31), 4), (dict(n_seq=1 << 30), 4), (dict(q=OFF8), 1), (dict(k=OFF8), 1),
    (dict(out=OFF8), 1), (dict(row_start=OFF2), 1), (dict(lse=OFF2), 1),
    (dict(ws=ctypes.c_void_p(0x100010)), 3), (dict(ws_bytes=16), 3),
])
def test_attn_prompt_refusals(tod, kw, status):
    assert _prompt(tod, attn(tod), **kw) == status
    assert tod.last_error() != ""


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(kp=None), 1), (dict(vp=None), 1), (dict(table=None), 1),
    (dict(row_start=None), 1), (dict(cached=None), 1), (dict(ws=None), 1), (dict(out=None), 1),
    (dict(tokens=0), 1), (dict(n_seq=0), 1), (dict(cols=0), 1), (dict(fresh=0), 1),
    (dict(pages=0), 1), (dict(page=0), 1), (dict(page=65537), 1), (dict(pages=1 << 30), 4),
    (dict(cols=1 << 28), 4), (dict(kp=OFF8), 1), (dict(table=OFF2), 1), (dict(cached=OFF2), 1),
    (dict(ws=ctypes.c_void_p(0x100010)), 3), (dict(ws_bytes=16), 3),
])
def test_attn_paged_refusals(tod, kw, status):
    assert _paged(tod, attn(tod), **kw) == status
    assert tod.last_error() != ""


def test_attn_paged_is_causal(tod):
    assert _paged(tod, attn(tod, causal=0)) == tod.TOD_ERR_UNSUPPORTED


def test_null_options(tod):
    assert _prompt(tod, None) == 1 and _paged(tod, None) == 1
    tod.raw_library().tod_default_attn(None, 1, 1, 8, 2)


def test_workspace_sizes(tod):
    size = tod.tod_attn_workspace_size
    one = size(32, 8, 128, 1, 1)
    assert one > 0 and one % 256 == 0
    # single tokens: rows of the four heads of a group, for each worker's two pieces
    assert size(32, 8, 128, 64, 64, 1) >= 2 * 1024 * 4 * 128 * 4
    assert size(32, 8, 128, 64, 64, 1) < size(32, 8, 128, 64, 64, 8)
    for bad in ((32, 8, 128, 0, 1), (32, 8, 128, 1, 0), (32, 5, 128, 1, 1), (32, 8, 130, 1, 1),
                (32, 8, 128, 1, 1, 0)):
        assert size(*bad) == 0


def test_binding_refuses_host_tensors(tod):
    torch = pytest.importorskip("torch")
    i = torch.zeros(3, dtype=torch.int32)
    q = torch.zeros(4, 2, 64, dtype=torch.float16)
    pages = torch.zeros(2, 2, 16, 64, dtype=torch.float16)
    for call in (lambda: tod.tod_page_map(i, i, i, i.view(3, 1), 16, 4),
                 lambda: tod.tod_page_write(q, q, i.long(), pages, pages),
                 lambda: tod.tod_attn_prompt(q, q, q, i),
                 lambda: tod.tod_attn_paged(q, pages, pages, i.view(3, 1), i, i)):
        with pytest.raises(TypeError):
            call()
