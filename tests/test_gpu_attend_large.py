"""Attention with more workgroups than a launch takes."""
import numpy as np
import pytest
import torch

import cache_cases as cc

pytestmark = pytest.mark.gpu


def few_lengths(n, most):
    return (torch.arange(n, device="cuda") % most + 1).to(torch.int32)


def page_of(heads, tokens, dim, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(1, heads, tokens, dim, generator=g, device="cuda").bfloat16() for _ in range(2)]


def exact_rows(q, k, v, most):
    """Query q [heads, dim] over the first 1 .. most tokens of one KV head."""
    res = []
    for n in range(1, most + 1):
        s = (q.double() @ k[0, 0, :n].double().T.contiguous()) * q.shape[1] ** -0.5
        res.append(torch.softmax(s, 1) @ v[0, 0, :n].double())
    return torch.stack(res)


def test_many_sequences_of_one_token(gpu):
    """More workgroups than a launch takes, of two parts each."""
    from paper_2408_05235_amd import api
    n, heads, dim, most = 2 ** 24 + 5, 1, 8, 3
    k, v = page_of(1, 65536, dim)
    q = torch.randn(heads, dim, device="cuda").bfloat16()
    length = few_lengths(n, most)
    table = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    out = torch.full((n, heads, dim), 9.0, dtype=torch.bfloat16, device="cuda")
    query = q[None].expand(n, heads, dim).contiguous()
    api.tl_attend(query, k, v, table, length, out=out)
    want = exact_rows(q, k, v, most)
    for i in range(most):
        # (the output and the weights rounded to 8 bits, values of up to 4)
        assert bool(((out[i::most].double() - want[i]).abs() <= 2.0 ** -5).all())


def test_many_chunks(gpu):
    """The same where every sequence has rows for the tiles."""
    from paper_2408_05235_amd import api
    n, new, heads, dim = 2 ** 18 + 3, 17, 32, 8
    k, v = page_of(heads, 32, dim)
    q = torch.randn(new, heads, dim, device="cuda").bfloat16()
    table = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    length = torch.full((n,), new, dtype=torch.int32, device="cuda")
    off = torch.arange(n + 1, device="cuda") * new
    query = q[None].expand(n, new, heads, dim).reshape(n * new, heads, dim)
    out = torch.full(query.shape, 9.0, dtype=torch.bfloat16, device="cuda")
    api.tl_attend(query, k, v, table, length, off, out=out)
    got = out.view(n, new, heads, dim)
    assert bool((got == got[:1]).all())
    dense = [tuple(x[0].transpose(0, 1)[:new] for x in (k, v))]
    cc.check(dict(q=q, dense=dense, before=np.asarray([0]), new=np.asarray([new]), window=0, sinks=0, dtype="bf16"),
             got[0], None)
