"""CPU checks of the sizes that the sequence operators' entry points refuse: what a launch or 32-bit
positions cannot hold.  The workspace given is too small, so that nothing is ever launched."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def tod():
    from paper_2110_14007_amd import tod
    return tod


FAKE = ctypes.c_void_p(0x100000)  # never dereferenced
UNSUPPORTED, WORKSPACE = 4, 3


def _attn(tod, heads, kv_heads, dim=8):
    a = tod.tod_attn()
    tod.raw_library().tod_default_attn(ctypes.byref(a), heads, kv_heads, dim, 2)
    return a


def _prompt(tod, heads, kv_heads, tokens, n_seq):
    a = _attn(tod, heads, kv_heads)
    return tod.raw_library().tod_attn_prompt(ctypes.byref(a), FAKE, FAKE, FAKE, tokens, FAKE, n_seq,
                                             FAKE, 16, None, FAKE, None)


def _paged(tod, heads, kv_heads, tokens, n_seq, fresh, cols=4, page=16):
    a = _attn(tod, heads, kv_heads)
    return tod.raw_library().tod_attn_paged(ctypes.byref(a), FAKE, FAKE, FAKE, 9, page, FAKE, cols,
                                            FAKE, FAKE, n_seq, tokens, fresh, FAKE, 16, None, FAKE,
                                            None)


def _size(tod, heads, kv_heads, tokens, n_seq, fresh):
    a = _attn(tod, heads, kv_heads)
    return tod.raw_library().tod_attn_workspace_size(ctypes.byref(a), tokens, n_seq, fresh)


# A launch has fewer than 2^32 threads: 256 for every tile slot (tokens * group / 128 + n_seq + 1 a
# key / value head), 64 for each of up to 8 packed rows of every sequence and head whose tokens are
# joined.
@pytest.mark.parametrize("heads,kv_heads,tokens,n_seq,status", [
    (2, 2, 1, 1 << 23, UNSUPPORTED), (8, 8, 5, 1 << 21, UNSUPPORTED),
    (32, 32, 1 << 26, 1, UNSUPPORTED), (8, 8, 1 << 28, 7, UNSUPPORTED),
    (2, 2, 1, (1 << 23) - 4096, WORKSPACE), (8, 8, 5, (1 << 21) - 1024, WORKSPACE),
    (32, 32, (1 << 26) - (1 << 20), 1, WORKSPACE),
])
def test_prompt_launches(tod, heads, kv_heads, tokens, n_seq, status):
    assert _prompt(tod, heads, kv_heads, tokens, n_seq) == status
    assert tod.last_error() != ""


@pytest.mark.parametrize("heads,kv_heads,tokens,n_seq,fresh,status", [
    (1, 1, 1, 1 << 25, 1, WORKSPACE), (8, 2, 9, 1 << 22, 2, UNSUPPORTED),
    (8, 2, 9, 1 << 22, 1, WORKSPACE), (64, 8, 9, 1 << 20, 1, UNSUPPORTED),
    (64, 1, 9, 1 << 24, 2, UNSUPPORTED),
    (8, 2, 9, (1 << 22) - 1, 2, WORKSPACE), (64, 1, 9, (1 << 24) - 2000, 2, WORKSPACE),
])
def test_paged_launches(tod, heads, kv_heads, tokens, n_seq, fresh, status):
    assert _paged(tod, heads, kv_heads, tokens, n_seq, fresh) == status
    assert tod.last_error() != ""


def test_workspace_sizes_of_what_fits(tod):
    assert _size(tod, 64, 8, 9, 1 << 21, 1) == 0  # neither call takes it
    assert _size(tod, 64, 8, 9, 1 << 20, 1) > 0  # a prompt call does
    assert _size(tod, 1, 1, 1, 1 << 25, 1) > 0  # a paged call does


# Positions are 32 bits, with room for the call's tokens and the 64 positions that the stage after
# the last key names.
@pytest.mark.parametrize("page,cols,tokens,status", [
    (1, (1 << 31) - 2, 1, UNSUPPORTED), (1, (1 << 31) - 1 - 64, 1, UNSUPPORTED),
    (1, (1 << 31) - 1 - 64 - 1, 1, WORKSPACE), (2, (1 << 30) - 33, 3, UNSUPPORTED),
    (2, (1 << 30) - 35, 3, WORKSPACE), (65536, 32767, 1000, WORKSPACE),
    (65536, 32767, 65536, UNSUPPORTED),
])
def test_paged_positions(tod, page, cols, tokens, status):
    assert _paged(tod, 1, 1, tokens, 1, tokens, cols, page) == status
    assert tod.last_error() != ""
