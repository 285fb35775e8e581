"""How many rows a draw or a verification may have, on the CPU: the launches that they take and the places of their
distributions (tests/c/round_launch_check.cpp, tests/c/round_places_check.cpp), and calls up to the stated limits."""
import ctypes
import gc
import os
import subprocess
import weakref

import pytest

from paper_2604_02945_amd import binding as B
from test_cache_cpu import FAKE, OK, ROOT, UNSUP, chunk
from test_round_cpu import refused, sample, verify


@pytest.mark.parametrize("name", ["round_launch_check", "round_places_check"])
def test_launches_and_places(tmp_path, name):
    exe = str(tmp_path / name)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2604_02945_amd", "csrc"),
                           os.path.join(ROOT, "tests", "c", name + ".cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


@pytest.mark.parametrize("vocab", [8, 1000, 5000, 1 << 20])
@pytest.mark.parametrize("rows", [(1 << 21) - 1, 1 << 21, (1 << 22) - 1, 1 << 22, (1 << 24) - 1, 1 << 24])
def test_rows_of_a_draw(rows, vocab):
    n, want = ctypes.c_size_t(), OK if rows < 1 << 24 else UNSUP
    assert B.lib().msao_sample_workspace(rows, vocab, B.BF16, ctypes.byref(n)) == want
    refused(sample(rows=rows, vocab=vocab, stride=vocab, ws_bytes=1 << 62), want)


@pytest.mark.parametrize("vocab", [8, 5000, 1 << 20])
@pytest.mark.parametrize("draft", [None, FAKE], ids=["certain", "drawn"])
@pytest.mark.parametrize("seqs,new,rows", [((1 << 21) - 1, 1, 1 << 21), (1 << 21, 1, 1 << 21), (1 << 20, 4, 1 << 22), (1 << 23, 1, 1 << 23),
                                           ((1 << 24) - 1, 1, 1 << 24), (1 << 23, 1, 10), (1 << 22, 3, 10), (1 << 24, 1, 10), (1 << 23, 2, 10)])
def test_rows_of_a_verification(seqs, new, rows, draft, vocab):
    """n_seqs * max_new below 2^24, however few rows there are."""
    n, ch, want = ctypes.c_size_t(), chunk(n_rows=rows, max_new=new), OK if seqs * new < 1 << 24 else UNSUP
    assert B.lib().msao_verify_workspace(B._addr(ch), seqs, vocab, B.BF16, ctypes.byref(n)) == want
    refused(verify(ch=ch, seqs=seqs, draft=draft, vocab=vocab, stride=vocab, dstride=vocab, ws_bytes=1 << 62), want)


def test_an_address_keeps_its_struct():
    """A call's temporary struct is there until the call has ended."""
    s = chunk()
    alive, a = weakref.ref(s), B._addr(s)
    del s
    gc.collect()
    assert alive() is not None and a.value == ctypes.addressof(alive())
