"""The prompt scan's CTAs leave behind everything that arrives in their shared memory: the model of test_scan_roles.py, in which an arrival of a product
behind the end of all of a CTA's warps is a fault."""
import os
import re
import subprocess

import pytest

from test_scan_roles import CSRC, CUDA, HERE


@pytest.fixture(scope="module")
def ends(tmp_path_factory):
    where = tmp_path_factory.mktemp("ends")
    for name in ("lq_rows.cuh", "lq_scan.cuh"):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        text, n = re.subn(r'asm volatile\("ldmatrix.*?"memory"\);', "read_values(at);", text, flags=re.S)
        assert n == (name == "lq_scan.cuh")
        (where / name).write_text(re.sub(r"\basm( volatile)?\(", "PTX(", text))
    with open(os.path.join(HERE, "host", "scan_roles.cpp")) as f:
        text = f.read()
    late = 'for (const Fiber &f : fibers) if (!f.done) { arrive(m.bar); return; } fail("a product arrives behind the CTA\'s end (barrier at %d)", (int)m.bar - (int)BASE);'
    text, n = re.subn(r"loose\.push_back\(\[=\] \{ arrive\(m\.bar\); \}\);", lambda _: "loose.push_back([=] { " + late + " });", text)
    assert n == 1
    (where / "scan_ends.cpp").write_text(text)
    exe = str(where / "scan_ends")
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-Wno-psabi", "-I", str(where), "-I", os.path.join(HERE, "host"), "-I", CSRC, "-I", CUDA,
                    str(where / "scan_ends.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("seed", [5000, 6000])
def test_nothing_arrives_behind_the_end(ends, seed):
    out = subprocess.run([ends, str(seed), "500"], capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stdout
