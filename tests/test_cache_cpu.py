"""The paged cache's entry points on the CPU: refusals before any device is
touched, workspace sizes, the binding's checks, and the indexing that the
kernels share with the host (tests/c/cache_check.cpp)."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2604_02945_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, ALIGN, WS, UNSUP, HIP = range(6)
FAKE = 0x10000  # validation never dereferences


def cache(**kw):
    c = B.MsaoKvCache()
    c.k, c.v, c.pages, c.length, c.weight = FAKE, FAKE, FAKE, FAKE, FAKE
    dim, page, heads = kw.get("head_dim", 128), kw.get("page_size", 64), kw.get("kv_heads", 8)
    for st in (c.k_stride, c.v_stride):
        st[0], st[1], st[2] = heads * page * dim, page * dim, dim
    c.dtype, c.head_dim, c.kv_heads, c.page_size = B.BF16, dim, heads, page
    c.n_pages, c.n_seqs, c.pages_per_seq, c.table_stride = 100, 4, 20, 20
    c.weight_stride = 20 * page
    for name, v in kw.items():
        if name in ("k_stride", "v_stride"):
            for i, x in enumerate(v):
                getattr(c, name)[i] = x
        else:
            setattr(c, name, v)
    return c


def chunk(**kw):
    ch = B.MsaoChunk(FAKE, 10, 4)
    for name, v in kw.items():
        setattr(ch, name, v)
    return ch


def append(**kw):
    a = B.MsaoAppend()
    a.q = a.q_out = a.k = a.v = a.inv_freq = a.positions = FAKE
    a.q_stride = a.q_out_stride = 32 * 128
    a.k_stride = a.v_stride = 8 * 128
    a.eps, a.heads, a.rot_dim, a.n_axes, a.position_stride = 1e-6, 32, 128, 1, 10
    a.sections[0] = 64
    for name, v in kw.items():
        if name == "sections":
            for i, x in enumerate(v):
                a.sections[i] = x
        else:
            setattr(a, name, v)
    return a


def message():
    return B.lib().msao_last_error_global().decode()


def validate(c, ch=None):
    return B.lib().msao_cache_validate(B._addr(c), B._addr(ch) if ch is not None else None)


def test_struct_layouts_match_the_header(tmp_path):
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "msao.h"\nint main(void) { printf("%zu %zu %zu\\n", '
                   'sizeof(msao_kv_cache), sizeof(msao_chunk), sizeof(msao_append)); return 0; }\n')
    exe = str(tmp_path / "s")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    sizes = [int(x) for x in subprocess.check_output([exe]).split()]
    assert sizes == [ctypes.sizeof(x) for x in (B.MsaoKvCache, B.MsaoChunk, B.MsaoAppend)]


@pytest.mark.parametrize("kw,code", [
    ({}, OK), ({"weight": None}, OK), ({"n_seqs": 0, "pages": None, "length": None}, OK), ({"n_pages": 0, "k": None, "v": None}, OK),
    ({"dtype": 2}, INVALID), ({"head_dim": 0}, INVALID), ({"head_dim": 12}, INVALID), ({"head_dim": 264}, INVALID),
    ({"kv_heads": 0}, INVALID), ({"kv_heads": 65536}, INVALID),
    ({"page_size": 8}, INVALID), ({"page_size": 48}, INVALID), ({"page_size": 131072}, INVALID), ({"page_size": 0}, INVALID),
    ({"n_pages": -1}, INVALID), ({"n_seqs": -1}, INVALID), ({"pages_per_seq": -1}, INVALID),
    ({"pages_per_seq": (1 << 23) + 1, "table_stride": 1 << 25}, UNSUP), ({"table_stride": 19}, INVALID),
    ({"weight_stride": 20 * 64 - 1}, INVALID), ({"k": None}, INVALID), ({"v": None}, INVALID), ({"pages": None}, INVALID),
    ({"length": None}, INVALID), ({"k": FAKE + 8}, ALIGN), ({"v": FAKE + 2}, ALIGN), ({"length": FAKE + 2}, ALIGN),
    ({"weight": FAKE + 1}, ALIGN), ({"k_stride": (65536, 8192, 127)}, ALIGN), ({"k_stride": (65536, 8192, 120)}, INVALID),
    ({"v_stride": (-8, 8192, 128)}, INVALID), ({"v_stride": (1 << 41, 8192, 128)}, INVALID),
    ({"v_stride": (65536, 8192, 1 << 25)}, UNSUP)])
def test_cache_refusals(kw, code):
    assert validate(cache(**kw)) == code, message()


@pytest.mark.parametrize("kw,code", [
    ({}, OK), ({"max_new": 0}, OK), ({"n_rows": 0, "max_new": 0}, OK), ({"n_rows": -1}, INVALID), ({"max_new": -1}, INVALID),
    ({"max_new": 11}, OK), ({"start": None}, INVALID), ({"start": FAKE + 2}, ALIGN)])
def test_chunk_refusals(kw, code):
    assert validate(cache(), chunk(**kw)) == code, message()


@pytest.mark.parametrize("kw,code", [
    ({}, OK), ({"heads": 0, "q": None, "q_out": None}, OK), ({"rot_dim": 0, "inv_freq": None, "n_axes": 0}, OK),
    ({"positions": None}, OK), ({"q_norm": FAKE, "k_norm": FAKE}, OK), ({"n_axes": 3, "sections": (16, 16, 32)}, OK),
    ({"q": None}, INVALID), ({"q_out": None}, INVALID), ({"k": None}, INVALID), ({"v": None}, INVALID),
    ({"heads": -1}, INVALID), ({"q_stride": 32 * 128 - 8}, INVALID), ({"k_stride": 8 * 128 - 8}, INVALID),
    ({"v_stride": 8 * 128 + 4}, ALIGN), ({"q": FAKE + 8}, ALIGN), ({"k_norm": FAKE + 4}, ALIGN),
    ({"eps": -1e-9}, INVALID), ({"eps": float("nan")}, INVALID), ({"eps": float("inf")}, INVALID),
    ({"rot_dim": 24, "sections": (12,)}, INVALID), ({"rot_dim": 144, "sections": (72,)}, INVALID), ({"rot_dim": -16}, INVALID),
    ({"inv_freq": None}, INVALID), ({"n_axes": 0}, INVALID), ({"n_axes": 5}, INVALID), ({"sections": (63,)}, INVALID),
    ({"n_axes": 2, "sections": (65, -1)}, INVALID), ({"n_axes": 2, "sections": (32, 32), "positions": None}, INVALID),
    ({"position_stride": 9}, INVALID), ({"positions": FAKE + 1}, ALIGN), ({"flags": 2}, INVALID)])
def test_append_refusals(kw, code):
    c, ch, a = cache(), chunk(), append(**kw)
    rc = B.lib().msao_cache_append(None, B._addr(c), B._addr(ch), B._addr(a), None)
    if code == OK:  # the arguments pass; without a context nothing is enqueued
        assert rc == INVALID and message() == "ctx is NULL"
    else:
        assert rc == code and message() != "ctx is NULL", message()


def attention(c=None, ch=None, q=FAKE, q_stride=32 * 128, heads=32, scale=0.1, flags=1, out=FAKE, out_stride=32 * 128, lse=FAKE,
              ws=FAKE, ws_bytes=1 << 40):
    c, ch = c or cache(), ch or chunk()
    return B.lib().msao_cache_attention(None, B._addr(c), B._addr(ch), q, q_stride, heads, scale, flags, out, out_stride, lse, ws,
                                        ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    ({}, OK), ({"flags": 3}, OK), ({"flags": 0}, OK), ({"lse": None}, OK), ({"scale": 0.0}, OK), ({"scale": -1.0}, OK),
    ({"heads": 0}, INVALID), ({"heads": 30}, INVALID), ({"scale": float("nan")}, INVALID), ({"scale": float("inf")}, INVALID), ({"scale": 3e38}, INVALID),
    ({"flags": 4}, INVALID), ({"q": None}, INVALID), ({"out": None}, INVALID), ({"q": FAKE + 4}, ALIGN),
    ({"q_stride": 1 << 24}, UNSUP), ({"q_stride": (1 << 24) - 8, "out_stride": 1 << 30}, OK),
    ({"out_stride": 32 * 128 + 2}, ALIGN), ({"out_stride": 31 * 128}, INVALID), ({"lse": FAKE + 2}, ALIGN),
    ({"ws": None}, WS), ({"ws": FAKE + 16}, WS), ({"ws_bytes": 0}, WS)])
def test_attention_refusals(kw, code):
    rc = attention(**kw)
    if code == OK:
        assert rc == INVALID and message() == "ctx is NULL"
    else:
        assert rc == code and message() != "ctx is NULL", message()


def test_attention_needs_the_weight_it_adds_to():
    assert attention(c=cache(weight=None), flags=3) == INVALID and "weight" in message()


def test_attention_too_large_for_a_launch_or_its_rows():
    assert attention(ch=chunk(n_rows=1 << 27), heads=32) == UNSUP
    big = cache(n_seqs=1 << 20, kv_heads=4096)
    assert attention(c=big, heads=4096, q_stride=4096 * 128, out_stride=4096 * 128) == UNSUP


def test_attention_workspace():
    n = ctypes.c_size_t()
    c = cache()

    def size(ch, heads=32, flags=1, c=c):
        assert B.lib().msao_cache_attention_workspace(B._addr(c), B._addr(ch), heads, flags, ctypes.byref(n)) == OK, message()
        return n.value

    a, b = size(chunk()), size(chunk(), flags=3)
    assert a % 256 == 0 and b >= a + 10 * 32 * 4
    assert size(chunk(n_rows=0, max_new=0)) == 0
    one = cache(pages_per_seq=2, table_stride=2)  # 128 tokens: one part
    assert size(chunk(), c=one) == 0
    assert B.lib().msao_cache_attention_workspace(B._addr(c), B._addr(chunk()), 32, 1, None) == INVALID


def evict(c=None, to=None, budget=FAKE, first=4, recent=16, idx=FAKE, stride=20 * 64, ws=FAKE, ws_bytes=1 << 30):
    c = c or cache()
    return B.lib().msao_cache_evict(None, B._addr(c), B._addr(to) if to is not None else None, budget, first, recent, idx, stride,
                                    ws, ws_bytes, None)


OTHER = {"k": 2 * FAKE, "v": 2 * FAKE, "pages": 2 * FAKE, "length": 2 * FAKE, "weight": 2 * FAKE}


@pytest.mark.parametrize("kw,code", [
    ({}, OK), ({"to": OTHER}, OK), ({"to": dict(OTHER, weight=None)}, OK), ({"to": dict(OTHER, page_size=32)}, OK),
    ({"budget": None}, INVALID), ({"first": -1}, INVALID), ({"recent": -1}, INVALID), ({"idx": None}, INVALID),
    ({"stride": 20 * 64 - 1}, INVALID), ({"budget": FAKE + 1}, ALIGN), ({"idx": FAKE + 2}, ALIGN), ({"ws": None}, WS),
    ({"ws": FAKE + 4}, WS), ({"ws_bytes": 8}, WS), ({"to": dict(OTHER, dtype=B.F32)}, INVALID),
    ({"to": dict(OTHER, head_dim=64)}, INVALID), ({"to": dict(OTHER, kv_heads=4)}, INVALID), ({"to": dict(OTHER, n_seqs=3)}, INVALID),
    ({"to": dict(OTHER, pages=FAKE)}, INVALID), ({"to": dict(OTHER, length=FAKE)}, INVALID),
    ({"to": dict(OTHER, weight=FAKE)}, INVALID), ({"to": dict(OTHER, k=FAKE + 4)}, ALIGN)])
def test_evict_refusals(kw, code):
    if "to" in kw:
        kw = dict(kw, to=cache(**kw["to"]))
    rc = evict(**kw)
    if code == OK:
        assert rc == INVALID and message() == "ctx is NULL"
    else:
        assert rc == code and message() != "ctx is NULL", message()


@pytest.mark.parametrize("kw", [dict(n_seqs=0, pages=None, length=None, weight=None),
                                dict(pages_per_seq=0, table_stride=0, weight_stride=0, pages=None, weight=None)])
def test_evict_of_nothing_shares_no_array(kw):
    """Arrays of no element may be NULL in both caches."""
    to = dict(OTHER, **kw)
    assert evict(c=cache(**kw), to=cache(**to)) == INVALID and message() == "ctx is NULL"


def test_evict_needs_weight():
    assert evict(c=cache(weight=None)) == INVALID and "weight" in message()


def test_the_bindings_checks():
    k = torch.zeros(6, 2, 16, 64)
    pages, length = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    c = B.KvCache(k, k.clone(), pages, length, torch.zeros(3, 2, 32))
    assert (c.capacity, c.kv_heads, c.page_size, c.head_dim) == (32, 2, 16, 64)
    view = torch.zeros(6, 16, 2, 64).transpose(1, 2)
    assert list(B.KvCache(view, k, pages, length).struct.k_stride) == [16 * 2 * 64, 64, 128]
    for bad in (lambda: B.KvCache(k, k[:5], pages, length), lambda: B.KvCache(k.half(), k.half(), pages, length),
                lambda: B.KvCache(k, k, pages.long(), length), lambda: B.KvCache(k, k, pages[:2], length),
                lambda: B.KvCache(k, k, pages.t().contiguous().t(), length),
                lambda: B.KvCache(k, k, pages, length, torch.zeros(3, 2, 31)),
                lambda: B.KvCache(k, k, pages, length, torch.zeros(3, 1, 32)),
                lambda: B.KvCache(k.transpose(2, 3), k.transpose(2, 3), pages, length)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.MsaoError):  # pages of 12 tokens
        B.KvCache(k[:, :, :12], k[:, :, :12], pages, length)
    # host memory is no cache of a GPU
    start = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="not on a GPU"):
        B.msao_cache_attention(c, start, 1, torch.zeros(3, 2, 64))
    with pytest.raises(ValueError, match="not on a GPU"):
        B.msao_cache_append(c, start, 1, torch.zeros(3, 2, 64), torch.zeros(3, 2, 64))
    with pytest.raises(ValueError, match="not on a GPU"):
        B.msao_cache_evict(c, length)


def test_indexes_stay_in_bounds(tmp_path):
    exe = str(tmp_path / "cache_check")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-Wno-format-security",
                           "-Wno-format-extra-args", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           "-I", os.path.join(ROOT, "paper_2604_02945_amd", "csrc"),
                           os.path.join(ROOT, "tests", "c", "cache_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
