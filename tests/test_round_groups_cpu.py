"""Which workgroups of attention with shared prefixes write which rows' parts, for any array of groups
(tests/c/round_groups_check.cpp), on the CPU."""
import os
import subprocess

from test_cache_cpu import ROOT


def test_no_two_groups_write_the_parts_of_one_row(tmp_path):
    exe = str(tmp_path / "round_groups_check")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2604_02945_amd", "csrc"),
                           os.path.join(ROOT, "tests", "c", "round_groups_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
