"""Calls on the paged cache with more workgroups than a launch takes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_append_of_many_tokens(gpu):
    from paper_2408_05235_amd import api
    n, dim, page = 2 ** 28 + 4099, 8, 65536
    pages = -(-n // page)
    key = torch.randint(-30000, 30000, (n, 1, dim), dtype=torch.int16, device="cuda").view(torch.bfloat16)
    value = key.flip(0)
    k = torch.zeros(pages, 1, page, dim, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    length = torch.tensor([n], dtype=torch.int32, device="cuda")
    api.tl_kv_append(key, value, k, v, table, length, torch.tensor([0, n], device="cuda"))
    for got, want in ((k, key), (v, value)):
        flat = got.view(torch.int16).view(-1, dim)
        assert torch.equal(flat[:n], want.view(torch.int16).view(-1, dim)) and not bool(flat[n:].any())


def test_many_slots_leave(gpu):
    from paper_2408_05235_amd import api
    n = 2 ** 26 + 1000
    table = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    length = torch.ones(n, dtype=torch.int32, device="cuda")
    ref = torch.tensor([n], dtype=torch.int32, device="cuda")
    api.tl_pages_free(ref, table, length, torch.arange(n, dtype=torch.int32, device="cuda"), 16)
    assert int(ref) == 0 and not bool(length.any())
