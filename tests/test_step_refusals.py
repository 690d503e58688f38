"""What the norm, the sampling and the selection of pages refuse, on the host
and before anything is enqueued (no GPU: pointers are never reached, tensors of other
devices are torch's fakes)."""
import ctypes
import math

import pytest
import torch

from paper_2408_05235_amd import _lib, api

from test_cache_refusals import VIEW, refused, view

EU = _lib.TL_EUNSUPPORTED


def args(cls, base, kw):
    a = cls(ctypes.sizeof(cls))
    for k, x in {**base, **kw}.items():
        setattr(a, k, x)
    return a


def norm(**kw):
    return args(_lib.NormArgs, dict(dtype=_lib.BF16, n_rows=4, n_cols=64, group=0, eps=1e-6, x=16, residual=16, weight=16,
                                    x_stride=64, residual_stride=64, out=16, scale=16, sum=16), kw)


def sample(**kw):
    return args(_lib.SampleArgs, dict(dtype=_lib.F32, n_rows=4, n_cols=64, logits=16, stride=64, u=16, token=16), kw)


def bounds(v=None, **kw):
    return args(_lib.PageBoundsArgs, dict(cache=v or view(), n_tokens=3, bounds=16, scale=16, scale_stride=2), kw)


def select(v=None, **kw):
    return args(_lib.SelectPagesArgs, dict(n_heads=4, cache=v or view(), n_tokens=3, query=16, query_token_stride=256,
                                           query_head_stride=64, bounds=16, scale=16, scale_stride=2, n_select=8, first=1,
                                           last=2, selected=16, workspace=16, workspace_bytes=1 << 20), kw)


def attend(v=None, inner=(), **kw):
    a = _lib.AttendArgs(ctypes.sizeof(_lib.AttendArgs), 4, v or view(), 3, None, 16, 256, 64, 0.125, 0, 0, 0, 16, None,
                        None, 0)
    for k, x in dict(inner).items():
        setattr(a, k, x)
    return args(_lib.AttendPagesArgs, dict(n_select=8, attend=a, selected=16), kw)


CASES = {
    "tl_norm": (norm, [
        (dict(struct_size=8), "struct_size"), (dict(dtype=0), "dtype"), (dict(dtype=4), "dtype"),
        (dict(n_rows=-1), "n_rows"), (dict(n_rows=2 ** 31), "n_rows"), (dict(n_cols=0), "n_cols"),
        (dict(n_cols=(1 << 22) + 1), "n_cols"), (dict(group=-2), "group"), (dict(group=8), "group"),
        (dict(group=48), "group"), (dict(group=1024), "group"), (dict(eps=-1.0), "eps"), (dict(eps=math.nan), "eps"),
        (dict(eps=math.inf), "eps"), (dict(x_stride=-64), "strides"), (dict(residual_stride=-1), "strides"),
        (dict(x=None), "NULL"), (dict(weight=None), "NULL"), (dict(out=None), "NULL"), (dict(scale=None), "NULL"),
        (dict(residual=None), "sum without residual"), (dict(x=17), "aligned"), (dict(dtype=_lib.F32, weight=18), "aligned"),
        (dict(scale=18), "aligned"), (dict(group=-1, out=17), "aligned"),
    ]),
    "tl_sample": (sample, [
        (dict(struct_size=8), "struct_size"), (dict(dtype=0), "dtype"), (dict(n_rows=-1), "n_rows"),
        (dict(n_cols=0), "n_cols"), (dict(n_cols=(1 << 22) + 1), "n_cols"), (dict(stride=-1), "stride"),
        (dict(logits=None), "NULL"), (dict(u=None), "NULL"), (dict(token=None), "NULL"), (dict(logits=18), "aligned"),
    ]),
    "tl_page_bounds": (bounds, [
        (dict(struct_size=8), "struct_size"), (dict(n_tokens=-1), "n_tokens"), (dict(n_tokens=2), "without q_offset"),
        (dict(bounds=None), "NULL"), (dict(scale=None), "NULL"), (dict(bounds=24), "aligned"),
        (dict(scale_stride=-1), "scale_stride"),
    ]),
    "tl_select_pages": (select, [
        (dict(struct_size=8), "struct_size"), (dict(n_heads=5), "n_heads"), (dict(n_heads=0), "n_heads"),
        (dict(query=None), "NULL"), (dict(query=8), "aligned"), (dict(query_token_stride=4), "strides"),
        (dict(n_select=0), "n_select"), (dict(n_select=4097), "n_select", EU), (dict(first=-1), "first"),
        (dict(last=-1), "last"), (dict(first=5, last=4), "together"), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), "together"),
        (dict(n_heads=2 * 129), "query heads per KV head", EU), (dict(selected=None), "NULL"), (dict(bounds=None), "NULL"),
        (dict(bounds=8), "aligned"), (dict(scale=None), "NULL"), (dict(scale_stride=-1), "scale_stride"),
        (dict(workspace=8), "aligned"), (dict(workspace=None), "workspace"), (dict(workspace_bytes=31), "at least 32"),
    ]),
    "tl_attend_pages": (attend, [
        (dict(struct_size=8), "struct_size"), (dict(n_select=0), "n_select"), (dict(n_select=4097), "n_select", EU),
        (dict(selected=None), "NULL"), (dict(inner=dict(window=1)), "window"), (dict(inner=dict(sinks=1)), "sinks"),
        (dict(inner=dict(scale=0.0)), "scale"), (dict(inner=dict(out=None)), "NULL"),
        (dict(inner=dict(struct_size=4)), "struct_size"),
    ]),
}


@pytest.mark.parametrize("name,i", [(n, i) for n, (_, cases) in CASES.items() for i in range(len(cases))])
def test_arguments(name, i):
    make, cases = CASES[name]
    kw, needle, *status = cases[i]
    call = getattr(_lib.lib(), name)
    refused(lambda: call(ctypes.byref(make(**kw)), None), needle, *status)
    if name + "_workspace_bytes" in _lib.EXPORTED and not needle.startswith(("at least", "workspace")):
        assert getattr(_lib.lib(), name + "_workspace_bytes")(ctypes.byref(make(**kw))) == 0


@pytest.mark.parametrize("name", list(CASES))
def test_null(name):
    assert getattr(_lib.lib(), name)(None, None) == _lib.TL_EINVAL
    if name + "_workspace_bytes" in _lib.EXPORTED:
        assert getattr(_lib.lib(), name + "_workspace_bytes")(None) == 0


@pytest.mark.parametrize("kw,needle", VIEW)
def test_views(kw, needle):
    L = _lib.lib()
    pages = any(k.endswith("_pages") and k != "n_pages" for k in kw)
    if "value_pages" not in kw or needle == "aligned":
        refused(lambda: L.tl_page_bounds(ctypes.byref(bounds(view(**kw))), None), needle)
    if not pages or needle == "aligned":
        refused(lambda: L.tl_select_pages(ctypes.byref(select(view(**kw))), None), needle)
    refused(lambda: L.tl_attend_pages(ctypes.byref(attend(view(**kw))), None), needle)


def test_nothing_to_do():
    """Calls without rows are fine, without pointers."""
    L = _lib.lib()
    none = view(n_seqs=0, length=None, page_table=None, key_pages=None, value_pages=None)
    empty = view(n_pages=0, key_pages=None, value_pages=None)
    for call, a in ((L.tl_norm, norm(n_rows=0, x=None, weight=None, out=None, scale=None)),
                    (L.tl_sample, sample(n_rows=0, logits=None, u=None, token=None)),
                    (L.tl_page_bounds, bounds(none, n_tokens=0, bounds=None, scale=None)),
                    (L.tl_page_bounds, bounds(empty, bounds=None, scale=None)),
                    (L.tl_select_pages, select(none, n_tokens=0, query=None, selected=None, workspace=None)),
                    (L.tl_attend_pages, attend(none, inner=dict(n_tokens=0, query=None, out=None), selected=None))):
        assert call(ctypes.byref(a), None) == _lib.TL_OK, L.tl_last_error()


def test_workspaces():
    L = _lib.lib()
    # 4 bytes a token, KV head and table entry; of many tokens 256 MiB
    assert L.tl_select_pages_workspace_bytes(ctypes.byref(select())) == 3 * 2 * 4 * 4
    v = view(n_seqs=1 << 20, table_width=4096)
    assert L.tl_select_pages_workspace_bytes(ctypes.byref(select(v, n_tokens=1 << 20))) == 256 << 20
    assert L.tl_attend_pages_workspace_bytes(ctypes.byref(attend())) == 0       # 128 tokens at most: one part
    v = view(n_seqs=1, table_width=4096)
    assert L.tl_attend_pages_workspace_bytes(ctypes.byref(attend(v, inner=dict(n_tokens=1), n_select=128))) > 0


# ---------------------------------------------------------------- the Python entry points

def tensors(device="cpu", moved=None, grad=()):
    dev = lambda name: "cuda:1" if name == moved else device
    T = {}

    def add(name, dtype, *shape):
        T[name] = torch.zeros(shape, dtype=dtype, device=dev(name), requires_grad=name in grad)

    b, i, f = torch.bfloat16, torch.int32, torch.float32
    for name, dtype, *shape in (
            ("x", b, 3, 64), ("weight", b, 64), ("residual", b, 3, 64), ("out", b, 3, 64), ("sum_out", b, 3, 64),
            ("logits", f, 3, 50), ("u", f, 3), ("temperature", f, 3), ("top_k", i, 3), ("top_p", f, 3), ("min_p", f, 3),
            ("token", i, 3), ("query", b, 3, 2, 64), ("key_pages", b, 4, 1, 16, 64), ("value_pages", b, 4, 1, 16, 64),
            ("bounds", torch.int8, 4, 1, 2, 64), ("scale", f, 4, 1), ("page_table", i, 3, 2), ("length", i, 3),
            ("q_offset", torch.int64, 4), ("granted", i, 4), ("selected", i, 3, 1, 2), ("attended", b, 3, 2, 64),
            ("workspace", torch.uint8, 4096)):
        add(name, dtype, *shape)
    return T


CALLS = [
    (lambda t: api.tl_norm(t["x"], t["weight"], 1e-6, t["residual"], None, t["out"], t["sum_out"]),
     ("x", "weight", "residual", "out", "sum_out"), ("x", "weight", "residual")),
    (lambda t: api.tl_sample(t["logits"], t["u"], t["temperature"], t["top_k"], t["top_p"], t["min_p"], True, t["token"]),
     ("logits", "u", "temperature", "top_k", "top_p", "min_p", "token"), ("logits",)),
    (lambda t: api.tl_page_bounds(t["key_pages"], t["bounds"], t["scale"], t["page_table"], t["length"], 3, t["q_offset"],
                                  t["granted"]),
     ("key_pages", "bounds", "scale", "page_table", "length", "q_offset", "granted"), ("key_pages",)),
    (lambda t: api.tl_select_pages(t["query"], t["bounds"], t["scale"], t["page_table"], t["length"], 16, 2, t["q_offset"],
                                   1, 1, t["selected"], t["workspace"], t["granted"]),
     ("query", "bounds", "scale", "page_table", "length", "q_offset", "selected", "workspace", "granted"), ("query",)),
    (lambda t: api.tl_attend_pages(t["query"], t["key_pages"], t["value_pages"], t["page_table"], t["length"],
                                   t["selected"], t["q_offset"], None, t["attended"], True, t["workspace"], t["granted"]),
     ("query", "key_pages", "value_pages", "page_table", "length", "selected", "q_offset", "attended", "workspace",
      "granted"), ("query", "key_pages", "value_pages")),
]


@pytest.mark.parametrize("call,names,grads", CALLS)
def test_gradients_are_not_lost_without_a_word(call, names, grads):
    for name in grads:
        with pytest.raises(ValueError, match="gradient"):
            call(tensors(grad=(name,)))
        with torch.no_grad(), pytest.raises(ValueError, match="device"):      # the next check
            call(tensors(grad=(name,)))


@pytest.mark.parametrize("call,names,grads", CALLS)
def test_tensors_of_two_devices(monkeypatch, call, names, grads):
    from torch._subclasses.fake_tensor import FakeTensorMode
    monkeypatch.setattr(api, "_raw_device", lambda: 0)
    monkeypatch.setattr(api, "_raw_stream", lambda d: 0)

    class Refuses:
        def __getattr__(self, name):
            def call(*a):
                assert name.endswith("_workspace_bytes"), f"{name} was called"
                return 16
            return call

    monkeypatch.setattr(api, "lib", lambda: Refuses())
    monkeypatch.setattr(torch._subclasses.fake_tensor.FakeTensor, "data_ptr", lambda self: 16)
    with FakeTensorMode():
        for name in names:
            with pytest.raises(ValueError, match="cuda:1"):
                call(tensors("cuda:0", name))
        with pytest.raises(ValueError, match="current device"):
            call(tensors("cuda:1"))
        with pytest.raises(AssertionError, match="was called"):        # all of them right
            call(tensors("cuda:0"))


@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32 + 5, -2 ** 32, 10 ** 30])
def test_numbers_beyond_32_bits(value):
    t = tensors()
    base = dict(page_tokens=16, n_select=2, first=1, last=1)
    for name in base:
        with pytest.raises(ValueError, match=name):
            api.tl_select_pages(t["query"], t["bounds"], t["scale"], t["page_table"], t["length"], **{**base, name: value})
    with pytest.raises(ValueError, match="group|device"):
        api.tl_norm(t["x"], t["weight"], group=value)


def test_shapes_and_types(monkeypatch):
    from torch._subclasses.fake_tensor import FakeTensorMode
    monkeypatch.setattr(api, "_raw_device", lambda: 0)
    monkeypatch.setattr(api, "_raw_stream", lambda d: 0)
    with FakeTensorMode():
        t = tensors("cuda:0")
        z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda:0")
        norm = lambda x=t["x"], w=t["weight"], **kw: api.tl_norm(x, w, **kw)
        draw = lambda x=t["logits"], u=t["u"], **kw: api.tl_sample(x, u, **kw)
        pages = (t["key_pages"], t["value_pages"], t["page_table"], t["length"])
        bad = [
            (lambda: norm(z(3, 64, dtype=torch.float64)), "x must be"), (lambda: norm(z(64)), "columns"),
            (lambda: norm(z(64, 3).T), "contiguous rows"), (lambda: norm(w=z(63)), "weight"),
            (lambda: norm(w=z(64, dtype=torch.float16)), "weight"), (lambda: norm(residual=z(3, 65)), "residual"),
            (lambda: norm(residual=z(64, 3).T), "contiguous rows"), (lambda: norm(group=-1), "group"),
            (lambda: norm(sum_out=z(3, 64)), "residual"), (lambda: norm(out=z(3, 64), group=0), "float8"),
            (lambda: norm(out=z(3, 128)[:, :64]), "contiguous"), (lambda: draw(z(3, 50, dtype=torch.int32)), "logits"),
            (lambda: draw(u=z(4, dtype=torch.float32)), "shape"), (lambda: draw(top_k=z(3, dtype=torch.int64)), "top_k"),
            (lambda: draw(top_p=z(3, dtype=torch.float64)), "top_p"), (lambda: draw(z(50, 3, dtype=torch.float32).T), "contiguous"),
            (lambda: api.tl_attend_pages(t["query"], *pages, z(3, 2, 2, dtype=torch.int32)), "selected"),
            (lambda: api.tl_attend_pages(t["query"], *pages, z(2, 1, 2, dtype=torch.int32)), "selected"),
            (lambda: api.tl_page_bounds(t["key_pages"], z(4, 1, 2, 65, dtype=torch.int8), t["scale"], *pages[2:], 3), "bounds"),
            (lambda: api.tl_page_bounds(t["key_pages"], t["bounds"], z(4, 2, dtype=torch.float32), *pages[2:], 3), "scale"),
            (lambda: api.tl_page_bounds(t["key_pages"], t["bounds"], z(4, 1), *pages[2:], 3), "scale"),
            (lambda: api.tl_select_pages(t["query"].float(), t["bounds"], t["scale"], *pages[2:], 16, 2), "query"),
        ]
        for call, needle in bad:
            with pytest.raises(ValueError, match=needle):
                call()


def test_sizes_beyond_32_bits(monkeypatch):
    """Sizes whose low 32 bits would pass are refused, not cut to them."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    monkeypatch.setattr(api, "_raw_device", lambda: 0)
    monkeypatch.setattr(api, "_raw_stream", lambda d: 0)
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: reached.append(name) or 0
    monkeypatch.setattr(api, "lib", Library)
    far = (1 << 32) + 64
    with FakeTensorMode():
        t = tensors("cuda:0")
        z = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda:0")
        ints = lambda *s: z(*s, dtype=torch.int32)
        calls = [
            lambda: api.tl_norm(z(1, far), z(far)), lambda: api.tl_norm(z(1, far), z(far), group=0),
            lambda: api.tl_sample(z(1, far), z(1, dtype=torch.float32)),
            lambda: api.tl_attend_pages(t["query"], t["key_pages"], t["value_pages"], t["page_table"], t["length"],
                                        ints(3, t["key_pages"].shape[1], far)),
            lambda: api.tl_select_pages(t["query"][:, :1].expand(3, far, 64), t["bounds"], t["scale"], t["page_table"],
                                        t["length"], 16, 2),
            lambda: api.tl_select_pages(t["query"], t["bounds"], t["scale"], ints(t["page_table"].shape[0], far),
                                        t["length"], 16, 2),
            lambda: api.tl_attend_pages(t["query"][:, :1].expand(3, far, 64), t["key_pages"], t["value_pages"],
                                        t["page_table"], t["length"], ints(3, t["key_pages"].shape[1], 2)),
        ]
        for call in calls:
            with pytest.raises(ValueError, match="32 bits"):
                call()
    assert not [n for n in reached if "workspace" not in n], reached
