"""The prompt scan's roles against one another, on the CPU: the code of csrc/lq_scan.cuh compiled for the host (tests/host), its warps,
copies and products in random order.  What no run on a GPU shows: a wait that only the usual timing makes good."""
import os
import re
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_38166_b200", "csrc")
CUDA = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")


@pytest.fixture(scope="module")
def roles(tmp_path_factory):
    where = tmp_path_factory.mktemp("roles")
    for name in ("lq_rows.cuh", "lq_scan.cuh"):                                   # instructions in PTX become nothing, but for the loads of values
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        text, n = re.subn(r'asm volatile\("ldmatrix.*?"memory"\);', "read_values(at);", text, flags=re.S)
        assert n == (name == "lq_scan.cuh")
        (where / name).write_text(re.sub(r"\basm( volatile)?\(", "PTX(", text))
    exe = str(where / "scan_roles")
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-Wno-psabi", "-I", str(where), "-I", os.path.join(HERE, "host"), "-I", CSRC, "-I", CUDA,
                    os.path.join(HERE, "host", "scan_roles.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("seed", [0, 1000, 2000])
def test_any_order(roles, seed):
    out = subprocess.run([roles, str(seed), "1000"], capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stdout
