"""How large the calls with many query rows per sequence may be, found on the host before anything is launched.  Addresses here are made up and never
dereferenced: calls that are taken stop at a workspace that is too small."""
import pytest

from paper_2506_18226_b200 import binding as B
from test_prompt_cpu import _chunk, _kv, _packed  # noqa: F401

MOST = 2 ** 31 - 8449           # numbers of tokens 32 items of 256 past the last one, and of rows a tile past it, fit 32 bits


@pytest.mark.parametrize("n", [MOST + 1, 2 ** 31 - 8192, 2 ** 31 - 256])
def test_tokens_and_rows_that_32_bits_do_not_number(n):
    one = dict(heads=1, kv=1, d=2, wsb=0)
    assert _packed(n_q=n, n_k=0, **one) == B.EINVAL
    assert _packed(n_q=0x100, n_k=n, **one) == B.EINVAL
    assert _chunk(kv=dict(n_kv_heads=1), n=n, heads=1, wsb=0) == B.EINVAL
    assert _packed(n_q=MOST, n_k=0, **one) == B.ENOMEM                    # (taken, but for the workspace)


def test_rows_of_a_table_and_its_prefix_together():
    rows = 16
    most = MOST // rows
    for own, pre, want in ((most, 1, B.EINVAL), (1, most, B.EINVAL), (most // 2 + 1, most // 2 + 1, B.EINVAL), (most // 2, most // 2, B.ENOMEM)):
        assert _chunk(kv=dict(page_rows=rows, n_kv_heads=1), batch=1, n=1, heads=1, max_pages=own, mpp=pre, wsb=0) == want
    # without a prefix the width of its table does not count
    assert _chunk(kv=dict(page_rows=rows, n_kv_heads=1), batch=1, n=1, heads=1, max_pages=most, mpp=10 ** 9, groups=0, wsb=0) == B.ENOMEM


@pytest.mark.parametrize("heads,kv,batch,tokens", [(32, 8, 1024, 1024), (64, 64, 700, 1000), (8, 8, 4000, 32768), (32, 1, 2, 2 ** 24)])
def test_many_tokens_of_many_sequences_are_taken(heads, kv, batch, tokens):
    """(What a call's work is depends on the lengths, which lie on the device: tokens times rows of all sequences together say little.)"""
    n = batch * tokens
    assert _packed(heads=heads, kv=kv, batch=batch, n_q=n, n_k=n, d=16, qt=heads * 16, qh=16, kt=kv * 16, kh=16, vt=kv * 16, vh=16, wsb=0) == B.ENOMEM
    assert _chunk(kv=dict(n_kv_heads=kv), heads=heads, batch=batch, n=n, max_pages=2 ** 20, mpp=1, wsb=0) == B.ENOMEM
