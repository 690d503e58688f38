"""Callers built before tl_kv_append_args, tl_attend_args and tl_pages had their
last member: the smaller structs are taken, and what lies behind them is not read (no
GPU: calls that have nothing to do, or are refused for what comes later)."""
import ctypes

import pytest

from paper_2408_05235_amd import _lib

from test_cache_refusals import D16, append, attend, pages, view


def size(cls):
    return getattr(cls, "granted").offset


@pytest.mark.parametrize("smaller", [0, 1])
def test_sizes(smaller):
    L = _lib.lib()
    v = view(n_seqs=0)
    calls = [
        lambda: L.tl_attend(ctypes.byref(attend(v, n_tokens=0, struct_size=size(_lib.AttendArgs) - smaller)), None),
        lambda: L.tl_kv_append(ctypes.byref(append(v, n_tokens=0, struct_size=size(_lib.KvAppendArgs) - smaller)), None),
        lambda: L.tl_pages_free(ctypes.byref(pages(struct_size=size(_lib.Pages) - smaller)), 0, D16, None),
    ]
    for call in calls:
        assert call() == (_lib.TL_EINVAL if smaller else _lib.TL_OK)
        if smaller:
            assert "struct_size" in _lib.lib().tl_last_error().decode()


def test_layouts():
    """The members as tl.h has them, the new ones behind all others."""
    for cls in (_lib.AttendArgs, _lib.KvAppendArgs, _lib.Pages):
        assert size(cls) + 8 == ctypes.sizeof(cls)
        assert cls._fields_[-1][0] == "granted"
