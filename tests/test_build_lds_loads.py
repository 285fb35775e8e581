"""Loads that go from memory to LDS, written as assembly: the hardware wants five wait states
between a vector instruction that writes a scalar register (a readfirstlane, a readlane) and a
memory instruction that reads it, and one between a write of M0 and such a load. The
compiler counts none of them for assembly text, so the text itself has to hold them:
whatever is placed before it then cannot be too near. Checked on the code object that the
library's flags give; no GPU needed."""
import os
import re
import subprocess

import pytest

from paper_2604_02945_amd import build as B

SOURCES = [s for s in B.SOURCES if re.search(r"buffer_load_\w+ .* lds", open(s).read())]


@pytest.fixture(scope="module", params=SOURCES, ids=os.path.basename)
def asm(request, tmp_path_factory):
    if not os.path.exists(B.HIPCC):
        pytest.skip("hipcc not installed")
    flags = [f for f in B.FLAGS if f not in ("-fPIC", "-shared")]
    out = tmp_path_factory.mktemp("asm") / "k.s"
    r = subprocess.run([B.HIPCC, *flags, "--cuda-device-only", "-S", "-o", str(out), request.param], capture_output=True,
                       text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    return out.read_text()


def loads_with_too_few_wait_states(asm):
    """(line, instructions before) of loads to LDS without `s_mov_b32 m0` and at least five wait states right before."""
    found, total = [], 0
    insts = [(i, l.strip()) for i, l in enumerate(asm.split("\n")) if l.strip() and not l.strip().startswith((";", ".", "/"))]
    for at, (line, inst) in enumerate(insts):
        if not re.match(r"buffer_load_\w+ .*\blds\b", inst):
            continue
        total += 1
        nop, move = insts[at - 1][1], insts[at - 2][1]
        m = re.match(r"s_nop (\d+)", nop)
        if not (m and int(m.group(1)) >= 4 and move.startswith("s_mov_b32 m0,")):
            found.append((line + 1, move, nop))
    return found, total


def test_wait_states_before_loads_to_lds(asm):
    found, total = loads_with_too_few_wait_states(asm)
    assert total > 0
    assert not found, (len(found), total, found[:3])


def other_uses_of_m0(asm):
    """Instructions that name M0 beside the writes before such loads, in functions that have them: the text
    that writes M0 does not tell the compiler."""
    found = []
    for f in re.finditer(r"^(_Z\S+):[^\n]*\n(.*?)^\.Lfunc_end", asm, re.M | re.S):
        insts = [l.strip() for l in f.group(2).split("\n") if l.strip() and not l.strip().startswith((";", "."))]
        insts = [l.split(";")[0] for l in insts]
        loads = [i for i, l in enumerate(insts) if re.match(r"buffer_load_\w+ .*\blds\b", l)]
        if loads:
            found += [l for i, l in enumerate(insts) if re.search(r"\bm0\b", l) and i + 2 not in loads]
    return found


def test_nothing_else_uses_m0(asm):
    assert other_uses_of_m0(asm) == []


def test_the_check_sees_one():
    text = "\ts_mov_b32 m0, s4\n\ts_nop %d\n\tbuffer_load_dwordx4 v1, s[8:11], 0 offen nt lds\n"
    assert loads_with_too_few_wait_states(text % 0) == ([(3, "s_mov_b32 m0, s4", "s_nop 0")], 1)
    assert loads_with_too_few_wait_states(text % 4) == ([], 1)
    body = "_Zk: ; @_Zk\n" + text % 4 + "%s\ts_endpgm\n.Lfunc_end0:\n"
    assert other_uses_of_m0(body % "") == [] and other_uses_of_m0(body % "\ts_mov_b32 m0, s1\n") == ["s_mov_b32 m0, s1"]
