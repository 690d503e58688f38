"""How much workspace the attention asks for (no GPU: nothing is enqueued)."""
import ctypes

import pytest

from paper_2408_05235_amd import _lib

from test_cache_refusals import attend, view


def workspace(n_seqs, table_width, offsets, n_heads=32, n_kv_heads=8, dim=128, **kw):
    v = view(n_kv_heads=n_kv_heads, head_dim=dim, table_width=table_width, n_seqs=n_seqs, page_stride=16 * 8 * dim,
             head_stride=16 * dim, token_stride=dim)
    a = attend(v, n_heads=n_heads, n_tokens=n_seqs, q_offset=16 if offsets else None, query_token_stride=n_heads * dim,
               query_head_stride=dim, **kw)
    return _lib.lib().tl_attend_workspace_bytes(ctypes.byref(a))


@pytest.mark.parametrize("offsets", [False, True])
def test_many_sequences_in_wide_tables(offsets):
    """Tables for a million tokens do not ask for more than a card has: parts
    that only even out long sequences take up to 1 GiB (and a part of a gigabyte for
    the statistics of small heads)."""
    for n_seqs in (64, 512, 4096, 65536, 2 ** 20):
        for dim in (8, 128, 256):
            assert workspace(n_seqs, 65536, offsets, dim=dim) <= 1.3 * 2 ** 30, (n_seqs, dim)


def test_few_long_sequences_still_have_parts():
    assert workspace(4, 2304, False, n_heads=64) > 2 ** 20
    assert workspace(96, 2304, False) >= 96 * 32 * 4 * 128 * 4
    assert workspace(1, 65536, False) > 2 ** 20
