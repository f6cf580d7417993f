"""The host's side of an attention plan where memory runs out: a status, nothing leaked, and nothing given back that a copy still reads or writes."""
import os
import subprocess

import pytest

from paper_2309_06626_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no compiler")
def test_no_memory_is_given_back_under_a_copy(tmp_path):
    out = str(tmp_path / "plan")
    host = [build.HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O1", "-w", "-fPIC", "-x", "hip"]
    for source, to in ((os.path.join(HERE, "attention_plan_host.cpp"), "a.o"), (os.path.join(build.CSRC, "attention.hip"), "b.o")):
        subprocess.run([*host, "-c", source, "-o", str(tmp_path / to)], check=True)
    subprocess.run(["g++", str(tmp_path / "a.o"), str(tmp_path / "b.o"), "-Wl,--unresolved-symbols=ignore-in-object-files", "-o", out], check=True)
    run = subprocess.run([out], capture_output=True, text=True, timeout=60)
    lines = [line.split() for line in run.stdout.splitlines()]
    assert run.returncode == 0, run.stdout + run.stderr
    assert len(lines) > 8 and lines[-1][2] == "0"
    assert all(line[4] == "0" and line[6] == "0" for line in lines), run.stdout
