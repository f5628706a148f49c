"""CPU checks of the entry points around a 4-bit cache and of the rotating appends: what they refuse,
on the host and before any HIP call, and their workspace sizes."""
import ctypes
import os
import re

import pytest


@pytest.fixture(scope="module")
def tod():
    from paper_2110_14007_amd import tod
    return tod


def at(offset=0):
    """A pointer of its own, never dereferenced: validation rejects first."""
    at.next += 1 << 32
    return ctypes.c_void_p(at.next + offset)


at.next = 1 << 40
INVALID, WORKSPACE, UNSUPPORTED = 1, 3, 4


def cache(tod, **kw):
    f = dict(struct_size=ctypes.sizeof(tod.tod_cache4), page_rows=16, n_pages=9, k_codes=at(),
             v_codes=at(), k_scales=at(), v_scales=at())
    f.update(kw)
    c = tod.tod_cache4()
    for name, v in f.items():
        setattr(c, name, v)
    return c


def append(tod, heads=8, kv_heads=2, dim=64, precision=2, **kw):
    a = tod.tod_append()
    tod.raw_library().tod_default_append(ctypes.byref(a), heads, kv_heads, dim, precision)
    for name, v in kw.items():
        setattr(a, name, v)
    return a


def ref(x):
    return ctypes.byref(x) if x is not None else None


def _append(tod, a, q=None, k=None, v=None, tokens=50, pos=None, rates=None, slot=None, kp=None,
            vp=None, pages=9, page=16, out=None):
    f = [x if x is not None else at() for x in (q, k, v, pos, rates, slot, kp, vp, out)]
    q, k, v, pos, rates, slot, kp, vp, out = (None if x is NULL else x for x in f)
    return tod.raw_library().tod_page_append(ref(a), q, k, v, tokens, pos, rates, slot, kp, vp,
                                             pages, page, None, out)


def _append4(tod, a, c, q=None, k=None, v=None, tokens=50, pos=None, rates=None, slot=None,
             out=None):
    f = [x if x is not None else at() for x in (q, k, v, pos, rates, slot, out)]
    q, k, v, pos, rates, slot, out = (None if x is NULL else x for x in f)
    return tod.raw_library().tod_page_append4(ref(a), q, k, v, tokens, pos, rates, slot, ref(c),
                                              None, out)


NULL = object()


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), INVALID), (dict(precision=0), UNSUPPORTED),
    (dict(precision=1), UNSUPPORTED), (dict(precision=7), INVALID), (dict(heads=0), INVALID),
    (dict(kv_heads=0), INVALID), (dict(dim=0), INVALID), (dict(dim=36, rotary=0), UNSUPPORTED),
    (dict(dim=264), UNSUPPORTED), (dict(rotary=-2), INVALID), (dict(rotary=66), INVALID),
    (dict(rotary=15), INVALID), (dict(interleaved=2), INVALID), (dict(q_row=-8), INVALID),
    (dict(q_head=12), UNSUPPORTED), (dict(v_row=4), UNSUPPORTED),
    (dict(heads=65534, kv_heads=2), UNSUPPORTED),
])
def test_append_options_refused(tod, kw, status):
    a = append(tod, **kw)
    assert _append(tod, a) == status
    assert tod.last_error() != ""
    assert _append4(tod, a, cache(tod)) == status
    assert tod.last_error() != ""


@pytest.mark.parametrize("kw,status", [
    (dict(q=NULL), INVALID), (dict(k=NULL), INVALID), (dict(v=NULL), INVALID),
    (dict(pos=NULL), INVALID), (dict(rates=NULL), INVALID), (dict(slot=NULL), INVALID),
    (dict(out=NULL), INVALID), (dict(tokens=0), INVALID), (dict(tokens=1 << 31), UNSUPPORTED),
    (dict(q=at(8)), INVALID), (dict(k=at(2)), INVALID), (dict(v=at(4)), INVALID),
    (dict(out=at(8)), INVALID), (dict(pos=at(2)), INVALID), (dict(rates=at(1)), INVALID),
    (dict(slot=at(4)), INVALID),
])
def test_append_refusals(tod, kw, status):
    assert _append(tod, append(tod), **kw) == status
    assert tod.last_error() != ""
    assert _append4(tod, append(tod), cache(tod), **kw) == status
    assert tod.last_error() != ""


@pytest.mark.parametrize("kw,status", [
    (dict(kp=NULL), INVALID), (dict(vp=NULL), INVALID), (dict(kp=at(8)), INVALID),
    (dict(pages=0), INVALID), (dict(page=0), INVALID), (dict(page=65537), INVALID),
    (dict(pages=1 << 30), UNSUPPORTED),
])
def test_append_pages_refused(tod, kw, status):
    assert _append(tod, append(tod), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), INVALID), (dict(k_codes=None), INVALID), (dict(v_codes=None), INVALID),
    (dict(k_scales=None), INVALID), (dict(v_scales=None), INVALID), (dict(k_codes=at(8)), INVALID),
    (dict(k_scales=at(4)), INVALID), (dict(v_scales=at(1)), INVALID),
    (dict(n_pages=0), INVALID), (dict(page_rows=0), INVALID), (dict(page_rows=65537), INVALID),
    (dict(n_pages=1 << 30), UNSUPPORTED),
])
def test_cache_refused(tod, kw, status):
    c = cache(tod, **kw)
    assert _append4(tod, append(tod), c) == status
    assert tod.last_error() != ""
    assert _read4(tod, c) == status
    assert _attn(tod, attn(tod), c) == status


def test_symbols_declared_and_exported(tod):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "tod.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(tod_\w*4\w*)\s*\(", text))
    assert names == set(tod.SYMBOLS4)
    for n in names:
        assert hasattr(tod.raw_library(), n), n


def test_null_structs(tod):
    assert _append(tod, None) == INVALID
    assert _append4(tod, None, cache(tod)) == INVALID
    assert _append4(tod, append(tod), None) == INVALID
    assert _read4(tod, None) == INVALID
    assert _attn(tod, None, cache(tod)) == INVALID and _attn(tod, attn(tod), None) == INVALID
    tod.raw_library().tod_default_append(None, 1, 1, 8, 2)


@pytest.mark.parametrize("which", ["q", "k", "v"])
def test_append_output_apart_from_inputs(tod, which):
    x = at()
    last = ctypes.c_void_p(x.value + (49 * 1024 + 64) * 2 - 16)  # the strides' last 16 bytes
    strides = {which + "_row": 1024, which + "_head": 8}
    heads = dict(heads=1, kv_heads=1, **strides)
    for out in (x, last):
        assert _append(tod, append(tod, **heads), out=out, **{which: x}) == INVALID
        assert "memory" in tod.last_error()
        assert _append4(tod, append(tod, **heads), cache(tod), out=out, **{which: x}) == INVALID


def test_rows_of_four_bits_come_in_blocks(tod):
    assert _append4(tod, append(tod, dim=72), cache(tod)) == UNSUPPORTED
    assert _read4(tod, cache(tod), dim=48) == UNSUPPORTED
    assert _attn(tod, attn(tod, dim=80), cache(tod)) == UNSUPPORTED
    assert tod.tod_attn_paged4_workspace_size(8, 2, 80, 4, 1) == 0


def _read4(tod, c, kv_heads=2, dim=64, precision=2, slot=None, tokens=5, k=None, v=None):
    f = [x if x is not None else at() for x in (slot, k, v)]
    slot, k, v = (None if x is NULL else x for x in f)
    return tod.raw_library().tod_page_read4(ref(c), kv_heads, dim, precision, slot, tokens, None,
                                            k, v)


@pytest.mark.parametrize("kw,status", [
    (dict(slot=NULL), INVALID), (dict(k=NULL), INVALID), (dict(v=NULL), INVALID),
    (dict(kv_heads=0), INVALID), (dict(dim=0), INVALID), (dict(dim=288), UNSUPPORTED),
    (dict(precision=1), UNSUPPORTED), (dict(precision=9), INVALID), (dict(tokens=0), INVALID),
    (dict(tokens=1 << 31), UNSUPPORTED), (dict(kv_heads=1 << 27), UNSUPPORTED),
    (dict(k=at(8)), INVALID), (dict(v=at(4)), INVALID), (dict(slot=at(4)), INVALID),
])
def test_read4_refusals(tod, kw, status):
    assert _read4(tod, cache(tod), **kw) == status
    assert tod.last_error() != ""


def attn(tod, heads=8, kv_heads=2, dim=64, precision=2, **kw):
    a = tod.tod_attn()
    tod.raw_library().tod_default_attn(ctypes.byref(a), heads, kv_heads, dim, precision)
    for name, v in kw.items():
        setattr(a, name, v)
    return a


def _attn(tod, a, c, q=None, table=None, cols=4, row_start=None, cached=None, n_seq=3, tokens=50,
          fresh=50, ws=None, ws_bytes=1 << 40, out=None, lse=None):
    f = [x if x is not None else at() for x in (q, table, row_start, cached, ws, out, lse)]
    q, table, row_start, cached, ws, out, lse = (None if x is NULL else x for x in f)
    return tod.raw_library().tod_attn_paged4(ref(a), q, ref(c), table, cols, row_start, cached,
                                             n_seq, tokens, fresh, ws, ws_bytes, None, out, lse)


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), INVALID), (dict(precision=0), UNSUPPORTED), (dict(heads=0), INVALID),
    (dict(kv_heads=3), INVALID), (dict(dim=20), UNSUPPORTED), (dict(dim=288), UNSUPPORTED),
    (dict(causal=0), UNSUPPORTED), (dict(scale=-1.0), INVALID), (dict(q_row=4), UNSUPPORTED),
])
def test_attention_options_refused(tod, kw, status):
    a = attn(tod, **kw)
    assert _attn(tod, a, cache(tod)) == status
    assert tod.last_error() != ""


@pytest.mark.parametrize("kw,status", [
    (dict(q=NULL), INVALID), (dict(table=NULL), INVALID), (dict(row_start=NULL), INVALID),
    (dict(cached=NULL), INVALID), (dict(ws=NULL), INVALID), (dict(out=NULL), INVALID),
    (dict(tokens=0), INVALID), (dict(n_seq=0), INVALID), (dict(cols=0), INVALID),
    (dict(fresh=0), INVALID), (dict(cols=1 << 27), UNSUPPORTED), (dict(tokens=1 << 31), UNSUPPORTED),
    (dict(q=at(8)), INVALID), (dict(out=at(8)), INVALID), (dict(table=at(2)), INVALID),
    (dict(cached=at(2)), INVALID), (dict(lse=at(2)), INVALID), (dict(ws=at(16)), WORKSPACE),
    (dict(ws_bytes=16), WORKSPACE),
])
def test_attn_paged4_refusals(tod, kw, status):
    assert _attn(tod, attn(tod), cache(tod), **kw) == status
    assert tod.last_error() != ""


def test_workspace_sizes(tod):
    size = tod.tod_attn_paged4_workspace_size
    assert size(32, 8, 128, 1, 1) > 0 and size(32, 8, 128, 1, 1) % 256 == 0
    for bad in ((32, 8, 128, 0, 1), (32, 8, 128, 1, 0), (32, 5, 128, 1, 1), (32, 8, 120, 1, 1),
                (32, 8, 128, 1, 1, 0)):
        assert size(*bad) == 0


def test_binding_refuses_host_tensors(tod):
    torch = pytest.importorskip("torch")
    i = torch.zeros(4, dtype=torch.int32)
    q = torch.zeros(4, 2, 64, dtype=torch.float16)
    pages = torch.zeros(2, 2, 16, 64, dtype=torch.float16)
    rates = torch.zeros(32)
    codes = torch.zeros(2, 2, 16, 32, dtype=torch.uint8)
    for call in (lambda: tod.tod_page_append(q, q, q, i, i.long(), rates, pages, pages),
                 lambda: tod.Cache4(codes, codes, codes, codes)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        tod.Cache4.zeros(2, 2, 16, 40, device="cpu")


def test_most_sequences(tod):
    # The join has 512 threads for every sequence and key / value head, beside the tiles' own.
    def room(n):
        return tod.tod_attn_paged4_workspace_size(8, 1, 64, 100, n, 100)

    assert room(8_000_000) > 0
    assert room((1 << 23) - 1000) == 0 and room(1 << 23) == 0
