"""The norm's outputs (tl_norm) in each other's place are refused, on the host (no GPU:
pointers are never reached)."""
import ctypes

import pytest

from paper_2408_05235_amd import _lib

from test_step_refusals import norm

BASE = dict(x=1 << 20, residual=2 << 20, weight=3 << 20, out=4 << 20, scale=5 << 20, sum=6 << 20)


@pytest.mark.parametrize("kw", [
    dict(group=-1, sum=4 << 20), dict(group=-1, sum=(4 << 20) + 2 * 4 * 64 - 2), dict(group=-1, out=(6 << 20) + 2),
    dict(group=0, sum=(4 << 20) + 4 * 64 - 2), dict(group=0, scale=(4 << 20) + 4 * 64 - 4),
    dict(group=0, scale=(6 << 20) + 4), dict(group=16, out=(5 << 20) + 4 * 4 * 4 - 1),
])
def test_refused(kw):
    L = _lib.lib()
    a = norm(**{**BASE, **kw})
    assert L.tl_norm(ctypes.byref(a), None) == _lib.TL_EINVAL
    assert b"overlap" in L.tl_last_error()
