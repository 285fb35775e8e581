"""The entry points of a speculative round on the CPU: refusals before any device is touched,
workspace sizes, the binding's checks, and the indexing that the kernels share with the host
(tests/c/round_check.cpp)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import round_ref
from paper_2604_02945_amd import binding as B
from resize_ref import State
from test_cache_cpu import ALIGN, FAKE, INVALID, OK, ROOT, UNSUP, WS, cache, chunk, message


def refused(rc, code):
    if code == OK:  # every argument is right: only the context is missing
        assert rc == INVALID and message() == "ctx is NULL", (rc, message())
    else:
        assert rc == code and message() != "ctx is NULL", (rc, message())


def test_struct_layouts_match_the_header(tmp_path):
    names = {"msao_sampling": B.MsaoSampling, "msao_sample_out": B.MsaoSampleOut, "msao_verify_out": B.MsaoVerifyOut,
             "msao_page_pool": B.MsaoPagePool, "msao_resize": B.MsaoResize, "msao_prefix": B.MsaoPrefix}
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "msao.h"\nint main(void) {\n'
                   + "".join(f'printf("%zu ", sizeof({n}));\n' for n in names) + "return 0; }\n")
    exe = str(tmp_path / "s")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    assert [int(x) for x in subprocess.check_output([exe]).split()] == [ctypes.sizeof(t) for t in names.values()]


def test_indexes_stay_in_bounds(tmp_path):
    exe = str(tmp_path / "round_check")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2604_02945_amd", "csrc"),
                           os.path.join(ROOT, "tests", "c", "round_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


def sample(logits=FAKE, rows=5, vocab=1000, stride=1000, dtype=B.BF16, u=FAKE, out=True, ws=FAKE, ws_bytes=1 << 30, **kw):
    s = B.MsaoSampling(*[kw.get(k) for k in ("temperature", "top_k", "top_p", "min_p")])
    o = B.MsaoSampleOut(*[kw.get(k, FAKE) for k in ("token", "logprob", "kept")])
    return B.lib().msao_sample(None, logits, rows, vocab, stride, dtype, B._addr(s), u, B._addr(o) if out else None, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    ({}, OK), ({"rows": 0, "logits": None, "u": None}, OK), ({"vocab": 1}, OK), ({"vocab": 1 << 20, "stride": 1 << 20}, OK),
    ({"dtype": B.F32}, OK), ({"token": None, "kept": None}, OK), ({"dtype": 2}, INVALID), ({"rows": -1}, INVALID),
    ({"rows": 1 << 24}, UNSUP), ({"vocab": 0}, INVALID), ({"vocab": (1 << 20) + 1, "stride": 1 << 21}, UNSUP), ({"stride": 999}, INVALID),
    ({"stride": 1004}, ALIGN), ({"stride": 1 << 40}, INVALID), ({"logits": None}, INVALID), ({"logits": FAKE + 8}, ALIGN),
    ({"u": None}, INVALID), ({"u": FAKE + 2}, ALIGN), ({"out": False}, INVALID), ({"token": FAKE + 1}, ALIGN), ({"logprob": FAKE + 2}, ALIGN),
    ({"kept": FAKE + 3}, ALIGN), ({"temperature": FAKE + 1}, ALIGN), ({"top_k": FAKE + 2}, ALIGN), ({"min_p": FAKE + 3}, ALIGN)])
def test_sample_refusals(kw, code):
    refused(sample(**kw), code)


def test_sample_without_settings():
    o = B.MsaoSampleOut(FAKE, FAKE, FAKE)
    refused(B.lib().msao_sample(None, FAKE, 5, 1000, 1000, B.BF16, None, FAKE, B._addr(o), FAKE, 1 << 30, None), OK)


def verify(ch=None, seqs=4, tokens=FAKE, logits=FAKE, draft=None, vocab=1000, stride=1000, dstride=1000, dtype=B.BF16, ua=FAKE, u=FAKE,
           length=FAKE, out=True, ws=FAKE, ws_bytes=1 << 30, **kw):
    s = B.MsaoSampling(*[kw.get(k) for k in ("temperature", "top_k", "top_p", "min_p")])
    o = B.MsaoVerifyOut(*[kw.get(k, FAKE) for k in ("accepted", "next", "logprob", "length_out")])
    ch = chunk() if ch is None else ch
    return B.lib().msao_verify(None, B._addr(ch) if ch else None, seqs, tokens, logits, draft, vocab, stride, dstride, dtype,
                               B._addr(s), ua, u, length, B._addr(o) if out else None, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    ({}, OK), ({"draft": FAKE}, OK), ({"length": None, "length_out": None}, OK), ({"seqs": 0}, OK), ({"ch": False}, INVALID),
    ({"ch": chunk(n_rows=0), "tokens": None, "logits": None, "ua": None, "u": None}, OK),
    ({"ch": chunk(n_rows=-1)}, INVALID), ({"ch": chunk(max_new=-1)}, INVALID), ({"ch": chunk(start=None)}, INVALID),
    ({"ch": chunk(start=FAKE + 2)}, ALIGN), ({"ch": chunk(n_rows=1 << 30, max_new=1 << 24)}, UNSUP), ({"seqs": -1}, INVALID),
    ({"seqs": 1 << 23}, UNSUP), ({"vocab": 0}, INVALID), ({"vocab": 1 << 21, "stride": 1 << 21}, UNSUP), ({"dtype": 3}, INVALID),
    ({"stride": 992}, INVALID), ({"stride": 1001}, ALIGN), ({"draft": FAKE, "dstride": 992}, INVALID), ({"draft": FAKE + 4}, ALIGN),
    ({"tokens": None}, INVALID), ({"logits": None}, INVALID), ({"ua": None}, INVALID), ({"u": None}, INVALID), ({"length": None}, INVALID),
    ({"out": False}, INVALID), ({"tokens": FAKE + 1}, ALIGN), ({"ua": FAKE + 1}, ALIGN), ({"accepted": FAKE + 1}, ALIGN), ({"next": FAKE + 2}, ALIGN),
    ({"length_out": FAKE + 2}, ALIGN), ({"top_p": FAKE + 1}, ALIGN), ({"ws": None}, WS), ({"ws": FAKE + 16}, WS), ({"ws_bytes": 100}, WS)])
def test_verify_refusals(kw, code):
    refused(verify(**kw), code)


def resize(c=None, pool=True, free=FAKE, count=FAKE, want=FAKE, ws=FAKE, ws_bytes=1 << 40, given=True, **kw):
    r = B.MsaoResize()
    r.want = want
    for name, v in kw.items():
        setattr(r, name, v)
    p = B.MsaoPagePool(free, count)
    return B.lib().msao_cache_resize(None, B._addr(c or cache()), B._addr(p) if pool else None, B._addr(r) if given else None, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    ({}, OK), ({"held": FAKE, "columns": FAKE, "start": FAKE, "slots": FAKE, "positions": FAKE, "n_rows": 100, "granted": FAKE + 1}, OK),
    ({"ws": None, "ws_bytes": 0}, OK), ({"c": cache(n_pages=0, k=None, v=None), "free": None}, OK), ({"c": cache(head_dim=12)}, INVALID),
    ({"pool": False}, INVALID), ({"free": None}, INVALID), ({"count": None}, INVALID), ({"want": None}, INVALID), ({"given": False}, INVALID),
    ({"n_rows": -1}, INVALID), ({"want": FAKE + 1}, ALIGN), ({"held": FAKE + 2}, ALIGN), ({"columns": FAKE + 2}, ALIGN), ({"start": FAKE + 2}, ALIGN),
    ({"slots": FAKE + 4, "n_rows": 1}, ALIGN), ({"positions": FAKE + 2}, ALIGN), ({"free": FAKE + 1}, ALIGN), ({"count": FAKE + 1}, ALIGN),
    ({"slots": FAKE, "n_rows": 10000, "ws": None}, WS), ({"slots": FAKE, "n_rows": 10000, "ws": FAKE + 8}, WS),
    ({"slots": FAKE, "n_rows": 10000, "ws_bytes": 256}, WS), ({"c": cache(n_seqs=2000), "ws_bytes": 256}, WS),
    ({"c": cache(n_seqs=1 << 27), "ws_bytes": 1 << 60}, UNSUP)])
def test_resize_refusals(kw, code):
    refused(resize(**kw), code)


def shared(c=None, p=None, ch=None, q=FAKE, qs=32 * 128, heads=32, scale=0.1, flags=1, out=16 * FAKE, os_=32 * 128, lse=None, ws=FAKE,
           ws_bytes=1 << 40):
    p = B.MsaoPrefix(FAKE, FAKE, 2, 2, 512, 0) if p is None else p
    return B.lib().msao_cache_attention_shared(None, B._addr(c or cache()), B._addr(p) if p else None, B._addr(ch or chunk()), q, qs, heads,
                                               scale, flags, out, os_, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    ({}, OK), ({"flags": 3}, OK), ({"p": B.MsaoPrefix(None, None, 0, 0, 0, 0)}, OK), ({"p": B.MsaoPrefix(FAKE, FAKE, 2, 1 << 30, 1 << 30, 1 << 30)}, OK),
    ({"p": False}, INVALID), ({"p": B.MsaoPrefix(None, FAKE, 2, 2, 512, 0)}, INVALID), ({"p": B.MsaoPrefix(FAKE, None, 2, 2, 512, 0)}, INVALID),
    ({"p": B.MsaoPrefix(FAKE, FAKE, -1, 2, 512, 0)}, INVALID), ({"p": B.MsaoPrefix(FAKE, FAKE, 2, -2, 512, 0)}, INVALID),
    ({"p": B.MsaoPrefix(FAKE, FAKE, 2, 2, -5, 0)}, INVALID), ({"p": B.MsaoPrefix(FAKE, FAKE, 2, 2, 5, -1)}, INVALID),
    ({"p": B.MsaoPrefix(FAKE + 2, FAKE, 2, 2, 512, 0)}, ALIGN), ({"p": B.MsaoPrefix(FAKE, FAKE + 1, 2, 2, 512, 0)}, ALIGN),
    ({"p": B.MsaoPrefix(FAKE, FAKE, 1 << 22, 2, 512, 0)}, UNSUP), ({"flags": 4}, INVALID), ({"heads": 12}, INVALID), ({"c": cache(weight=None), "flags": 3}, INVALID),
    ({"scale": float("nan")}, INVALID), ({"q": None}, INVALID), ({"qs": 100}, INVALID), ({"lse": FAKE + 2}, ALIGN),
    ({"ws": None}, WS), ({"ws": FAKE + 4}, WS), ({"ws_bytes": 64}, WS), ({"c": cache(n_seqs=1 << 22)}, UNSUP)])
def test_shared_refusals(kw, code):
    refused(shared(**kw), code)


def test_workspaces():
    n, ch, L = ctypes.c_size_t(7), chunk(), B.lib()
    assert L.msao_sample_workspace(5, 1000, B.BF16, ctypes.byref(n)) == OK and n.value % 256 == 0
    assert L.msao_sample_workspace(5, 0, B.BF16, ctypes.byref(n)) == INVALID and L.msao_sample_workspace(5, 10, 0, None) == INVALID
    assert L.msao_verify_workspace(B._addr(ch), 4, 1000, B.BF16, ctypes.byref(n)) == OK and n.value >= 120 and n.value % 256 == 0
    assert L.msao_verify_workspace(None, 4, 1000, B.BF16, ctypes.byref(n)) == INVALID
    p = B.MsaoPrefix(FAKE, FAKE, 2, 2, 512, 0)
    assert L.msao_cache_attention_shared_workspace(B._addr(cache()), B._addr(p), B._addr(ch), 32, 1, ctypes.byref(n)) == OK
    assert n.value % 256 == 0 and n.value >= 2 * 10 * 32 * 128 * 4
    r = B.MsaoResize()
    assert L.msao_cache_resize_workspace(B._addr(cache()), B._addr(r), ctypes.byref(n)) == OK and n.value == 0
    assert L.msao_cache_resize_workspace(B._addr(cache(n_seqs=5000)), B._addr(r), ctypes.byref(n)) == OK and n.value >= 5000 * 24
    for f in (lambda: L.msao_cache_resize_workspace(B._addr(cache()), B._addr(r), None), lambda: L.msao_verify_workspace(B._addr(ch), 4, 9, 1, None),
              lambda: L.msao_cache_attention_shared_workspace(B._addr(cache()), B._addr(p), B._addr(ch), 32, 1, None)):
        assert f() == INVALID


@pytest.mark.parametrize("seqs,rows,new,tokens,max_seqs,own", [(256, 1536, 6, 1 << 19, 256, 0), (256, 1536, 6, 1 << 19, 2, 0), (256, 1536, 6, 0, 256, 0),
                                                               (64, 4096, 64, 1 << 20, 1, 4096), (2, 8192, 4096, 1 << 20, 2, 64)])
def test_workspaces_of_wide_tables_are_bounded(seqs, rows, new, tokens, max_seqs, own):
    """The parts of every row, whatever the table's width: at most 2^14 tiles of prefixes and as many of the rest, of 128 rows
    of 516 bytes, and as many tiles as there are more than that."""
    n, L = ctypes.c_size_t(), B.lib()
    c = cache(n_seqs=seqs, pages_per_seq=1 << 14, table_stride=1 << 14, weight_stride=1 << 20)
    p = B.MsaoPrefix(FAKE, FAKE, 4, max_seqs, tokens, own)
    ch = chunk(n_rows=rows, max_new=new)
    assert L.msao_cache_attention_shared_workspace(B._addr(c), B._addr(p), B._addr(ch), 32, 1, ctypes.byref(n)) == OK, message()
    tiles = 8 * -(-rows * 4 // 64)
    assert n.value <= 2 * (2 ** 14 + tiles + seqs * 8) * 128 * 520


def test_the_bindings_checks():
    k = torch.zeros(6, 2, 16, 64)
    pages, length = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    c = B.KvCache(k, k.clone(), pages, length)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    x = torch.zeros(4, 64)
    for match, bad in (("one entry", lambda: B.PagePool(i32(6), i32(2))), ("int32", lambda: B.PagePool(i32(6).long(), i32(1))),
                       ("not on a GPU", lambda: B.msao_cache_resize(c, B.PagePool(i32(6), i32(1)), i32(3))),
                       ("an entry more", lambda: B.SharedPrefix(i32(3), i32(3), 1, 1)), ("int32", lambda: B.SharedPrefix(x[0], i32(3), 1, 1)),
                       ("out of range", lambda: B.SharedPrefix(i32(2), i32(1), 1 << 40, 1)),
                       ("not on a GPU", lambda: B.msao_cache_attention_shared(c, B.SharedPrefix(i32(2), i32(1), 1, 1), i32(4), 1, torch.zeros(3, 2, 64))),
                       ("not on a GPU", lambda: B.msao_sample(x, x[:, 0])), ("2-D", lambda: B.msao_sample(x[0], x[:, 0])),
                       ("2-D", lambda: B.msao_sample(x.double(), x[:, 0])), ("vocab", lambda: B.msao_sample(x, x[:, 0], vocab=65)),
                       ("vocab", lambda: B.msao_sample(x, x[:, 0], vocab=0)), ("contiguous", lambda: B.msao_sample(x.t(), x[:, 0])),
                       ("not on a GPU", lambda: B.msao_verify(i32(2), 1, i32(4), x, x[:, 0], x[:, 0]))):
        with pytest.raises(ValueError, match=match):
            bad()
    s = B._settings
    for bad in (dict(temperature=i32(4)), dict(top_k=x[:, 0]), dict(top_p=torch.zeros(3)), dict(min_p=torch.zeros(8)[::2])):
        with pytest.raises(ValueError):
            s(4, -1, **{**dict(temperature=None, top_k=None, top_p=None, min_p=None), **bad})
    for bad in (dict(want=i32(4)), dict(want=i32(3), slots=i32(5)), dict(want=i32(3), slots=torch.zeros(5, dtype=torch.int64), positions=i32(4)),
                dict(want=i32(3), start=i32(3)), dict(want=i32(3), granted=i32(3)), dict(want=i32(6)[::2])):
        with pytest.raises(ValueError):
            B._resize_struct(c, **{**dict(held=None, columns=None, start=None, slots=None, positions=None, granted=None), **bad})
    with pytest.raises(ValueError, match="unknown output"):
        B._outputs(B.MsaoSampleOut(), {"tokens": i32(4)}, {"token": (4, torch.int32)}, None, -1, None)


# ---- the oracles of these operators, on cases whose answer can be seen ------------------

def test_the_oracle_of_distributions():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    for kw, want in (({}, [0.1, 0.4, 0.2, 0.3]), ({"top_k": 2}, [0, 4 / 7, 0, 3 / 7]), ({"top_p": 0.69}, [0, 4 / 7, 0, 3 / 7]),
                     ({"top_p": 0.71}, [0, 4 / 9, 2 / 9, 3 / 9]), ({"top_k": 3, "top_p": 0.77}, [0, 4 / 7, 0, 3 / 7]),
                     ({"min_p": 0.49}, [0, 4 / 9, 2 / 9, 3 / 9]), ({"temperature": 0}, [0, 1, 0, 0]),
                     ({"temperature": 0.5}, [1 / 30, 16 / 30, 4 / 30, 9 / 30])):
        assert np.allclose(round_ref.distribution(x, **kw)[2], want, atol=1e-14)
    p = np.array([0.25, 0.0, 0.5, 0.25])
    assert [round_ref.pick(p, u) for u in (0, 0.2, 0.25, 0.7, 0.75, 0.99, 1.0, 5, float("nan"), -1)] == [0, 0, 2, 2, 3, 3, 3, 3, 0, 0]
    assert round_ref.distribution([0.0, np.nan]) is None and round_ref.distribution([-np.inf] * 2) is None


def test_verified_tokens_are_distributed_as_drawn_ones():
    """Over a grid of numbers: the share of each token that follows a row is its probability, whatever the draft's."""
    x, y = np.log(np.array([[0.1, 0.2, 0.3, 0.4]] * 2)), np.log(np.array([[0.4, 0.3, 0.2, 0.1]] * 2))
    none = dict(temperature=None, top_k=None, top_p=None, min_p=None)
    n = 40
    grid = (np.arange(n) + 0.5) / n
    share = np.zeros(4)
    for draft, q in enumerate([0.4, 0.3, 0.2, 0.1]):
        for ua in grid:
            for u in grid:
                _, nxt, _, _ = round_ref.verify([0, 2], 2, [0, draft], x, y, [ua, 0], [u, 0], none, None)
                share[nxt[0]] += q / n / n
    assert np.allclose(share, [0.1, 0.2, 0.3, 0.4], atol=0.02)


def test_the_oracle_of_resizes():
    s = State([[3, -1, -1], [1, 4, -1]], [16, 20], [1, 2], [0, 2, 5], 16)
    assert s.resize([40, 10], [0, 0]) == ([0, 24, 24], [(5 * 16 + i, 16 + i) for i in range(16)] + [(2 * 16 + i, 32 + i) for i in range(8)], [1, 1])
    assert s.pages == [[3, 5, 2], [1, -1, -1]] and s.free == [0, 4] and s.length == [40, 10]
    assert s.resize([48, 48], [0, 0])[2] == [1, 1] and s.free == [] and s.pages == [[3, 5, 2], [1, 4, 0]]
