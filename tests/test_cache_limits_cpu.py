"""What the paged cache's calls take and refuse at large sizes, on the CPU: launches,
workspaces, integers."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2604_02945_amd import binding as B
from test_cache_cpu import INVALID, OK, ROOT, UNSUP, append, cache, chunk, message


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


MIB = 1 << 20


@pytest.mark.parametrize("dtype", [B.BF16, B.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,heads,kv_heads,new", [(256, 32, 8, 6), (256, 64, 8, 6), (64, 64, 8, 1), (48, 128, 8, 8), (1024, 32, 8, 1)])
@pytest.mark.parametrize("capacity", [1 << 17, 1 << 20])
def test_the_workspace_of_wide_tables_is_bounded(n_seqs, heads, kv_heads, new, capacity, dtype):
    """Parts of at least pairs * capacity / 16,384 tokens: at most 16,384 / pairs and one for the
    rounding, with 128 channels and two sums in 32 bits for each row."""
    rc, n = attention_workspace(n_seqs, capacity, n_seqs * new, new, heads, kv_heads, dtype=dtype)
    assert rc == OK, message()
    assert n <= (16384 / (n_seqs * kv_heads) + 1) * n_seqs * new * heads * 130 * 4 + 512 and n < 1200 * MIB


def test_a_wider_table_needs_no_more_once_every_workgroup_has_its_part():
    sizes = [attention_workspace(256, 1 << e, 256 * 6, 6)[1] for e in range(10, 21)]
    assert sizes[0] < sizes[3] and max(sizes) == max(sizes[:5]) and sizes[-1] < 512 * MIB


def test_rows_that_share_memory(tmp_path):
    exe = str(tmp_path / "rows_check")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2604_02945_amd", "csrc"),
                           os.path.join(ROOT, "tests", "c", "cache_rows_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


ROW = 32 * 128


@pytest.mark.parametrize("q_out,stride,rows,code", [
    (0, ROW, 10, OK), (0, ROW + 64, 1, OK), (10 * ROW, ROW, 10, OK), (-10 * ROW, ROW, 10, OK), (10 * ROW, 3 * ROW, 10, OK),
    (0, ROW + 64, 10, INVALID), (0, 2 * ROW, 2, INVALID), (ROW, ROW, 10, INVALID), (-ROW, ROW, 10, INVALID), (9 * ROW, ROW, 10, INVALID),
    (8, ROW, 10, INVALID), (-8, ROW, 1, INVALID), (ROW - 8, 5 * ROW, 10, INVALID)])
def test_append_into_part_of_the_queries(q_out, stride, rows, code):
    """(q_out and strides in bf16 elements from q; the header's forms: q itself, or memory apart)"""
    base = 1 << 30
    a = append(q=base, q_out=base + 2 * q_out, q_stride=ROW, q_out_stride=stride)
    c, ch = cache(), chunk(n_rows=rows, max_new=min(rows, 4))  # (held: the call has their addresses)
    rc = B.lib().msao_cache_append(None, B._addr(c), B._addr(ch), B._addr(a), None)
    assert rc == INVALID and ("overlaps" in message()) == (code == INVALID), message()


def test_queries_and_outputs_as_parts_of_one_array():
    base = 1 << 30
    a = append(q=base, q_out=base + 2 * ROW, q_stride=2 * ROW, q_out_stride=2 * ROW)
    c, ch = cache(), chunk()
    assert B.lib().msao_cache_append(None, B._addr(c), B._addr(ch), B._addr(a), None) == INVALID
    assert message() == "ctx is NULL"  # the arguments pass


def host_cache(n_seqs=3, per=2, **kw):
    k = torch.zeros(6, 2, 16, 64)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return B.KvCache(k, k.clone(), kw.get("pages", i32(n_seqs, per)), kw.get("length", i32(n_seqs)))


@pytest.mark.parametrize("max_new", [11, 2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 63, 2 ** 70])
def test_a_bound_past_an_integer_is_the_number_of_rows(max_new):
    """max_new beyond n_rows counts as n_rows, whatever its low bits are."""
    c, start = host_cache(per=200), torch.zeros(4, dtype=torch.int32)
    ch = B._chunk(c, start, 10, max_new)
    assert (ch.n_rows, ch.max_new) == (10, 10)
    assert B.cache_attention_workspace(c, start, 10, max_new, 4) == B.cache_attention_workspace(c, start, 10, 10, 4) > 0


@pytest.mark.parametrize("n_rows,max_new,heads", [(2 ** 31, 1, 4), (2 ** 32 + 10, 4, 4), (10, -2 ** 32, 4), (-2 ** 32, 1, 4),
                                                  (10, 4, 2 ** 32 + 4), (-1, 1, 4), (10, -1, 4), (10, 4, 0), (10, 4, -4)])
def test_counts_past_an_integer_are_refused(n_rows, max_new, heads):
    small = all(abs(x) < 2 ** 31 for x in (n_rows, max_new, heads))
    with pytest.raises(B.MsaoError if small else ValueError, match="negative|positive" if small else "out of range"):
        B.cache_attention_workspace(host_cache(), torch.zeros(4, dtype=torch.int32), n_rows, max_new, heads)


def test_a_workspace_has_the_bytes_it_says():
    ws = torch.zeros(1024, dtype=torch.uint8)
    assert B._bytes_of(ws) == B._bytes_of(ws.view(torch.float32)) == 1024 and B._bytes_of(ws[512:]) == 512
    assert B._bytes_of(ws[:0]) == 0
    for bad in (ws[:1].expand(1 << 30), ws[::2], ws.view(32, 32).t(), torch.as_strided(ws, (64, 64), (4, 1))):
        with pytest.raises(ValueError, match="contiguous"):
            B._bytes_of(bad)


def test_single_entries_at_any_distance():
    """One sequence of a table whose columns hold what others need: torch says any stride of one entry."""
    table = torch.zeros(4, 7, dtype=torch.int32)
    c = host_cache(n_seqs=1, pages=table[:1, :3], length=table[:1, 5])
    assert c.n_seqs == 1 and c.struct.length == table.data_ptr() + 20
    c = host_cache(n_seqs=4, pages=torch.zeros(1, 4, dtype=torch.int32).t(), length=table.view(-1)[:4])
    assert (c.pages_per_seq, c.struct.table_stride) == (1, 1)
    for bad in (dict(n_seqs=4, length=table[:, 0]), dict(n_seqs=4, pages=table.t()[:4, :3])):
        with pytest.raises(ValueError, match="contiguous"):
            host_cache(**bad)
