"""The product kernels' roles against one another, on the CPU: the code of csrc/lq_product.cuh compiled for the host (tests/host/product), its threads,
copies and products in random order, for all of its instances (seeds 18 apart have the same one).  What no run on a GPU shows: a wait that only the usual timing makes
good, an arrival behind a CTA's end."""
import os
import re
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_38166_b200", "csrc")
CUDA = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
# instructions in PTX become nothing, but for those that make or move values
CHANGES = {
    "lq_dependent.cuh": [],
    "lq_rows.cuh": [(r'asm\("cvt\.rn\.(bf16|f16)x2\.f32 %0, %1, %2;" : "=r"\(two\) : "f"\((.*?)\), "f"\((.*?)\)\);', r"two = two_\1(\3, \2);", 2)],
    "lq_product.cuh": [(r"PRODUCT_WAIT_LIMIT = 1 << 20;", "PRODUCT_WAIT_LIMIT = 3;", 1),
                       (r"extern __shared__ __align__\(1024\) uint8_t raw\[\];", "uint8_t *const raw = cta_memory();", 2),
                       (r'asm volatile\("st\.shared::cluster\.f32.*?"memory"\);', "store_cluster(addr, x);", 1)],
}


@pytest.fixture(scope="module")
def roles(tmp_path_factory):
    where = tmp_path_factory.mktemp("product")
    for name, changes in CHANGES.items():
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        for pattern, by, times in changes:
            text, n = re.subn(pattern, by, text, flags=re.S)
            assert n == times, (name, pattern)
        (where / name).write_text(re.sub(r"\basm( volatile)?\(", "PTX(", text).replace('"../../include/', '"'))
    exe = str(where / "product_roles")
    subprocess.run(["g++", "-std=c++17", "-O2", "-w", "-Wno-psabi", "-I", str(where), "-I", os.path.join(HERE, "host", "product"), "-I",
                    os.path.join(os.path.dirname(HERE), "include"), "-I", CUDA, os.path.join(HERE, "host", "product", "product_roles.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("seed", range(0, 144, 18))
def test_any_order(roles, seed):
    out = subprocess.run([roles, str(seed), "18"], capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stdout


@pytest.mark.parametrize("seed", range(0, 72, 18))
def test_a_copy_that_never_comes(roles, seed):
    out = subprocess.run([roles, str(seed), "18", "lose"], capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stdout
