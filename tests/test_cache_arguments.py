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
