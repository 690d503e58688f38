"""What the entry points of the paged cache refuse, on the host and before
anything is enqueued (no GPU)."""
import ctypes
import math

import pytest

from paper_2408_05235_amd import _lib

D16 = ctypes.c_void_p(16)      # never dereferenced: the call is refused first


def view(**kw):
    v = _lib.KvView(ctypes.sizeof(_lib.KvView), _lib.BF16, 2, 64, 16, 4, 10, 3, 2048, 1024, 64, 16, 16, 16, 16)
    for k, x in kw.items():
        setattr(v, k, x)
    return v


VIEW = [
    (dict(struct_size=8), "struct_size"), (dict(dtype=0), "dtype"), (dict(dtype=3), "dtype"),
    (dict(n_kv_heads=0), "n_kv_heads"), (dict(head_dim=0), "head_dim"), (dict(head_dim=12), "head_dim"),
    (dict(head_dim=264), "head_dim"), (dict(page_tokens=0), "page_tokens"), (dict(page_tokens=65537), "page_tokens"),
    (dict(table_width=-1), "table_width"), (dict(n_pages=-1), "n_pages"), (dict(n_pages=2 ** 31), "n_pages"),
    (dict(n_seqs=-1), "n_seqs"), (dict(n_seqs=4), "without q_offset"), (dict(page_stride=-8), "strides"),
    (dict(head_stride=4), "strides"), (dict(token_stride=63), "strides"), (dict(length=None), "NULL"),
    (dict(page_table=None), "NULL"), (dict(key_pages=None), "NULL pages"), (dict(value_pages=24), "aligned"),
]


def attend(v=None, **kw):
    a = _lib.AttendArgs(ctypes.sizeof(_lib.AttendArgs), 4, v or view(), 3, None, 16, 256, 64, 0.125, 0, 0, 0, 16,
                        None, None, 0)
    for k, x in kw.items():
        setattr(a, k, x)
    return a


def append(v=None, **kw):
    a = _lib.KvAppendArgs(ctypes.sizeof(_lib.KvAppendArgs), 0, v or view(), 3, None, 16, 16, 128, 64, 128, 64)
    for k, x in kw.items():
        setattr(a, k, x)
    return a


def refused(call, needle, status=_lib.TL_EINVAL):
    assert call() == status
    assert needle in _lib.lib().tl_last_error().decode()


@pytest.mark.parametrize("kw,needle", VIEW)
def test_views(kw, needle):
    L = _lib.lib()
    refused(lambda: L.tl_attend(ctypes.byref(attend(view(**kw))), None), needle)
    refused(lambda: L.tl_kv_append(ctypes.byref(append(view(**kw))), None), needle)
    assert L.tl_attend_workspace_bytes(ctypes.byref(attend(view(**kw)))) == 0


@pytest.mark.parametrize("kw,needle", [
    (dict(struct_size=4), "struct_size"), (dict(n_heads=0), "n_heads"), (dict(n_heads=5), "n_heads"),
    (dict(n_tokens=-1), "n_tokens"), (dict(n_tokens=2), "without q_offset"), (dict(scale=0.0), "scale"),
    (dict(scale=-1.0), "scale"), (dict(scale=math.nan), "scale"), (dict(scale=math.inf), "scale"),
    (dict(window=-1), "window"), (dict(sinks=-1), "sinks"), (dict(max_length=-1), "max_length"),
    (dict(query=None), "NULL"), (dict(out=None), "NULL"), (dict(query=8), "aligned"), (dict(out=8), "aligned"),
    (dict(workspace=8), "aligned"), (dict(query_token_stride=4), "strides"), (dict(query_head_stride=-8), "strides"),
])
def test_attend(kw, needle):
    L = _lib.lib()
    refused(lambda: L.tl_attend(ctypes.byref(attend(**kw)), None), needle)
    assert L.tl_attend(None, None) == _lib.TL_EINVAL
    assert L.tl_attend_workspace_bytes(None) == 0


def test_attend_of_too_many_rows_is_beyond_the_library():
    L = _lib.lib()
    v = view(n_seqs=2 ** 30)
    refused(lambda: L.tl_attend(ctypes.byref(attend(v, n_tokens=2 ** 30)), None), "2^31", _lib.TL_EUNSUPPORTED)


@pytest.mark.parametrize("kw,needle", [
    (dict(struct_size=4), "struct_size"), (dict(key=None), "NULL"), (dict(value=None), "NULL"),
    (dict(key=24), "aligned"), (dict(value=24), "aligned"), (dict(key_token_stride=1), "strides"),
    (dict(value_head_stride=-8), "strides"), (dict(n_tokens=5), "without q_offset"),
])
def test_append(kw, needle):
    L = _lib.lib()
    refused(lambda: L.tl_kv_append(ctypes.byref(append(**kw)), None), needle)
    assert L.tl_kv_append(None, None) == _lib.TL_EINVAL


def test_nothing_to_do_is_no_error():
    L = _lib.lib()
    v = view(n_seqs=0)
    assert L.tl_attend(ctypes.byref(attend(v, n_tokens=0)), None) == _lib.TL_OK
    assert L.tl_kv_append(ctypes.byref(append(v, n_tokens=0)), None) == _lib.TL_OK


def pages(**kw):
    g = _lib.Pages(ctypes.sizeof(_lib.Pages), 16, 10, 3, 4, 0, 16, 16, 16)
    for k, x in kw.items():
        setattr(g, k, x)
    return g


@pytest.mark.parametrize("kw,needle", [
    (dict(struct_size=8), "struct_size"), (dict(page_tokens=0), "page_tokens"), (dict(page_tokens=65537), "page_tokens"),
    (dict(n_pages=-1), "n_pages"), (dict(n_slots=-1), "n_slots"), (dict(n_slots=2 ** 31), "n_slots"),
    (dict(table_width=-1), "table_width"), (dict(ref=None), "NULL"), (dict(page_table=None), "NULL"),
    (dict(length=None), "NULL"),
])
def test_pools(kw, needle):
    L = _lib.lib()
    g = ctypes.byref(pages(**kw))
    refused(lambda: L.tl_pages_extend(g, D16, D16, D16, None), needle)
    refused(lambda: L.tl_pages_fork(g, 1, *[D16] * 6, None), needle)
    refused(lambda: L.tl_pages_free(g, 1, D16, None), needle)
    refused(lambda: L.tl_pages_compact(g, *[D16] * 6, None), needle)
    assert L.tl_pages_work_words(g) == 0


def test_pool_calls():
    L = _lib.lib()
    g = ctypes.byref(pages())
    assert L.tl_pages_work_words(g) >= 10
    for i in range(3):
        a = [D16] * 3
        a[i] = None
        refused(lambda: L.tl_pages_extend(g, *a, None), "NULL")
    for i in range(6):
        a = [D16] * 6
        a[i] = None
        refused(lambda: L.tl_pages_fork(g, 1, *a, None), "NULL")
        refused(lambda: L.tl_pages_compact(g, *a, None), "NULL")
    refused(lambda: L.tl_pages_fork(g, -1, *[D16] * 6, None), "n_forks")
    refused(lambda: L.tl_pages_fork(g, 4, *[D16] * 6, None), "n_forks")
    refused(lambda: L.tl_pages_free(g, -1, D16, None), "n_free")
    refused(lambda: L.tl_pages_free(g, 1, None, None), "NULL")
    refused(lambda: L.tl_pages_free(None, 1, D16, None), "NULL")
    assert L.tl_pages_fork(g, 0, *[None] * 6, None) == _lib.TL_OK
    assert L.tl_pages_free(g, 0, None, None) == _lib.TL_OK


@pytest.mark.parametrize("args,needle", [
    ((D16, -1, 64, 64, 1, 640, D16, D16, 1), "n_pages"), ((D16, 10, 64, 64, 1, 640, D16, D16, -1), "n_pairs"),
    ((D16, 10, 64, 64, -1, 640, D16, D16, 1), "n_planes"), ((D16, 10, 8, 64, 1, 640, D16, D16, 1), "16 bytes"),
    ((D16, 10, 64, 72, 1, 640, D16, D16, 1), "16 bytes"), ((D16, 10, 64, 64, 1, 8, D16, D16, 1), "16 bytes"),
    ((ctypes.c_void_p(8), 10, 64, 64, 1, 640, D16, D16, 1), "16 bytes"), ((None, 10, 64, 64, 1, 640, D16, D16, 1), "NULL"),
    ((D16, 10, 64, 64, 1, 640, None, D16, 1), "NULL"), ((D16, 10, 64, 64, 1, 640, D16, None, 1), "NULL"),
])
def test_copy(args, needle):
    L = _lib.lib()
    refused(lambda: L.tl_pages_copy(*args, None, None), needle)


def test_python_checks():
    import torch
    from paper_2408_05235_amd import api
    t = torch.zeros(1, 1, 16, 64, dtype=torch.float32)
    i = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(ValueError, match="bfloat16"):
        api.tl_attend(t[0], t, t, i, i[0])
    with pytest.raises(ValueError, match="device"):
        api.tl_attend(t[0].bfloat16(), t.bfloat16(), t.bfloat16(), i, i[0])
    with pytest.raises(ValueError, match="device"):
        api.tl_pages_extend(i[0], i, i[0], i[0], 16)
    with pytest.raises(ValueError, match="device"):
        api.tl_pages_copy(t, i[0], i[0])
    with pytest.raises(ValueError, match="dtype"):
        api.KVCache(1, 1, 1, 16, 64, 1, 16, dtype=torch.float32)
