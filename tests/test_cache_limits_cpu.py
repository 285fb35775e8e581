"""What the paged cache's calls take and refuse at large sizes, on the CPU: launches,
workspaces, integers."""
import ctypes

import pytest

from paper_2604_02945_amd import binding as B
from test_cache_cpu import OK, UNSUP, cache, chunk, message


def attention_workspace(n_seqs, capacity, n_rows, max_new, heads=32, kv_heads=8, flags=1, dim=128, page=64, dtype=B.BF16):
    per = -(-capacity // page)
    c = cache(n_seqs=n_seqs, kv_heads=kv_heads, head_dim=dim, page_size=page, pages_per_seq=per, table_stride=per,
              weight_stride=per * page, dtype=dtype)
    ch = chunk(n_rows=n_rows, max_new=max_new)
    n = ctypes.c_size_t()
    return B.lib().msao_cache_attention_workspace(B._addr(c), B._addr(ch), heads, flags, ctypes.byref(n)), n.value


@pytest.mark.parametrize("flags", [0, 1, 3], ids=["all", "causal", "weight"])
@pytest.mark.parametrize("n_seqs,capacity,n_rows,max_new", [
    (256, 4096, 255 + 2048, 2048),    # generating requests, one with a chunk of its prompt
    (128, 16384, 127 + 8192, 8192),
    (64, 8192, 64 * 8192 // 2, 8192),  # prompts as they arrive
    (512, 8192, 512 * 5, 6)])
def test_ordinary_batches_are_taken(n_seqs, capacity, n_rows, max_new, flags):
    assert attention_workspace(n_seqs, capacity, n_rows, max_new, flags=flags)[0] == OK, message()


@pytest.mark.parametrize("flags", [1, 3], ids=["causal", "weight"])
def test_more_workgroups_than_a_launch_takes(flags):
    assert attention_workspace(1 << 14, 4096, 1 << 20, 1 << 14, flags=flags)[0] == UNSUP
    assert attention_workspace(1 << 22, 64, 1 << 22, 1, flags=flags)[0] == UNSUP


@pytest.mark.parametrize("flags", [1, 3], ids=["causal", "weight"])
@pytest.mark.parametrize("n_seqs,kv_heads,n_rows,max_new", [(1 << 27, 1 << 15, 1000, 1000), (2 ** 31 - 1, 65535, 100, 100),
                                                            (1 << 26, 1 << 15, 10, 1), (511, 1 << 15, 60000, 60000)])
def test_counts_whose_products_pass_64_bits_are_refused(n_seqs, kv_heads, n_rows, max_new, flags):
    got = attention_workspace(n_seqs, 1 << 29, n_rows, max_new, heads=kv_heads, kv_heads=kv_heads, flags=flags, page=65536)
    assert got[0] == UNSUP, message()
