"""What the Python entry points of the paged cache refuse before they look at
pointers (no GPU: tensors of other devices are torch's fakes)."""
import pytest
import torch

from paper_2408_05235_amd import api


def cpu(heads=2, kv=1, dim=64, tokens=3, grad=()):
    t = dict(query=torch.zeros(tokens, heads, dim), key=torch.zeros(tokens, kv, dim), value=torch.zeros(tokens, kv, dim),
             key_pages=torch.zeros(4, kv, 16, dim), value_pages=torch.zeros(4, kv, 16, dim))
    t = {k: x.bfloat16().requires_grad_(k in grad) for k, x in t.items()}
    t.update(page_table=torch.zeros(tokens, 2, dtype=torch.int32), length=torch.zeros(tokens, dtype=torch.int32))
    return t


def attend(t, **kw):
    return api.tl_attend(*(t[k] for k in ("query", "key_pages", "value_pages", "page_table", "length")), **kw)


def append(t, **kw):
    return api.tl_kv_append(*(t[k] for k in ("key", "value", "key_pages", "value_pages", "page_table", "length")), **kw)


@pytest.mark.parametrize("call,names", [(attend, ("query", "key_pages", "value_pages")),
                                        (append, ("key", "value", "key_pages", "value_pages"))])
def test_gradients_are_not_lost_without_a_word(call, names):
    for name in names:
        with pytest.raises(ValueError, match="gradient"):
            call(cpu(grad=(name,)))
        with torch.no_grad(), pytest.raises(ValueError, match="device"):      # the next check
            call(cpu(grad=(name,)))
    with pytest.raises(ValueError, match="gradient"):
        attend(cpu(), out=torch.zeros(3, 2, 64, dtype=torch.bfloat16, requires_grad=True))


def fakes(cls_device, moved):
    """The arguments of every call on ``cls_device``, one of them on another."""
    dev = lambda name: "cuda:1" if name == moved else cls_device
    i32 = lambda name, *s: torch.empty(s, dtype=torch.int32, device=dev(name))
    b16 = lambda name, *s: torch.empty(s, dtype=torch.bfloat16, device=dev(name))
    t = dict(query=b16("query", 3, 2, 64), key=b16("key", 3, 1, 64), value=b16("value", 3, 1, 64),
             out=b16("out", 3, 2, 64), key_pages=b16("key_pages", 4, 1, 16, 64),
             value_pages=b16("value_pages", 4, 1, 16, 64), pages=b16("pages", 2, 4, 1, 16, 64))
    for name, shape in (("page_table", (3, 2)), ("length", (3,)), ("granted", (4,)), ("ref", (4,)), ("add", (3,)),
                        ("status", (3,)), ("parent", (1,)), ("child", (1,)), ("slots", (1,)), ("work", (4096,)),
                        ("copy_src", (2,)), ("copy_dst", (2,)), ("n_copies", (1,))):
        t[name] = i32(name, *shape)
    t["q_offset"] = torch.empty(4, dtype=torch.int64, device=dev("q_offset"))
    t["workspace"] = torch.empty(64, dtype=torch.uint8, device=dev("workspace"))
    return t


CALLS = [
    (lambda t: attend(t, q_offset=t["q_offset"], out=t["out"], workspace=t["workspace"], granted=t["granted"]),
     ("query", "key_pages", "value_pages", "page_table", "length", "q_offset", "out", "workspace", "granted")),
    (lambda t: append(t, q_offset=t["q_offset"], granted=t["granted"]),
     ("key", "value", "key_pages", "value_pages", "page_table", "length", "q_offset", "granted")),
    (lambda t: api.tl_pages_extend(t["ref"], t["page_table"], t["length"], t["add"], 16, t["status"], t["work"], t["granted"]),
     ("ref", "page_table", "length", "add", "status", "work", "granted")),
    (lambda t: api.tl_pages_fork(t["ref"], t["page_table"], t["length"], t["parent"], t["child"], 16, t["work"], t["granted"]),
     ("ref", "page_table", "length", "parent", "child", "work", "granted")),
    (lambda t: api.tl_pages_free(t["ref"], t["page_table"], t["length"], t["slots"], 16),
     ("ref", "page_table", "length", "slots")),
    (lambda t: api.tl_pages_compact(t["ref"], t["page_table"], t["length"], 16,
                                    {k: t[k] for k in ("ref", "page_table", "copy_src", "copy_dst", "n_copies")}, t["work"]),
     ("ref", "page_table", "length", "copy_src", "copy_dst", "n_copies", "work")),
    (lambda t: api.tl_pages_copy(t["pages"], t["copy_src"], t["copy_dst"], t["n_copies"]),
     ("pages", "copy_src", "copy_dst", "n_copies")),
]


@pytest.mark.parametrize("call,names", CALLS)
def test_tensors_of_two_devices(monkeypatch, call, names):
    """Each argument in turn on another device; and all on one that is not the
    current one.  No pointer of a fake may be reached."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    monkeypatch.setattr(api, "_raw_device", lambda: 0)
    monkeypatch.setattr(api, "_raw_stream", lambda d: 0)

    class Refuses:
        def __getattr__(self, name):
            def call(*a):
                assert name in ("tl_attend_workspace_bytes", "tl_pages_work_words"), f"{name} was called"
                return 16
            return call

    monkeypatch.setattr(api, "lib", lambda: Refuses())
    monkeypatch.setattr(torch._subclasses.fake_tensor.FakeTensor, "data_ptr", lambda self: 16)
    with FakeTensorMode():
        for name in names:
            with pytest.raises(ValueError, match="cuda:1"):
                call(fakes("cuda:0", name))
        with pytest.raises(ValueError, match="current device"):
            call(fakes("cuda:1", None))
        with pytest.raises(AssertionError, match="was called"):        # all of them right
            call(fakes("cuda:0", None))


@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32 + 5, -2 ** 32, 10 ** 30])
def test_numbers_beyond_32_bits(value):
    """They were cut to their low bits: a window of 2^32 + 5 tokens was one of 5."""
    for name in ("window", "sinks", "max_length"):
        with pytest.raises(ValueError, match=name):
            attend(cpu(), **{name: value})
    i = torch.zeros(3, dtype=torch.int32)
    for call in (lambda: api.tl_pages_extend(i, i[None], i, i, value), lambda: api.tl_pages_fork(i, i[None], i, i, i, value),
                 lambda: api.tl_pages_free(i, i[None], i, i, value), lambda: api.tl_pages_compact(i, i[None], i, value)):
        with pytest.raises(ValueError, match="page_tokens"):
            call()
