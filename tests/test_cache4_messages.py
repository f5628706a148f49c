"""CPU check: a workspace that is too small is refused with the name of the function that gives its size."""
import ctypes

import pytest

from test_cache4_api import WORKSPACE, _attn, at, attn, cache


@pytest.fixture(scope="module")
def tod():
    from paper_2110_14007_amd import tod
    return tod


def test_names_the_size_of_its_own_workspace(tod):
    assert _attn(tod, attn(tod), cache(tod), ws_bytes=16) == WORKSPACE
    assert "tod_attn_paged4_workspace_size" in tod.last_error()
    status = tod.raw_library().tod_attn_paged(
        ctypes.byref(attn(tod)), at(), at(), at(), 9, 16, at(), 4, at(), at(), 3, 50, 50, at(), 16,
        None, at(), None)
    assert status == WORKSPACE
    assert "tod_attn_workspace_size" in tod.last_error()
