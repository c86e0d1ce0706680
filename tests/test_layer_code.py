"""What the products' hand-counted waits take for granted of the code that the compiler makes around them (its own listing, no GPU).

The loops wait for loads by their number.  A register that the compiler put away in memory within a loop would be one more load or store
than counted, and an instruction of its own that needs m0 would take it from the load to LDS that it has been set for."""
import os
import re
import shutil
import subprocess

import pytest

from conftest import ROOT

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="needs hipcc")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Lines of every kernel of the two products by its mangled name."""
    from paper_2204_10562_amd import build
    folder, csrc = tmp_path_factory.mktemp("code"), os.path.join(ROOT, "paper_2204_10562_amd", "csrc")
    flags = [f for f in build.HIPCC_FLAGS] + ["-S", "--cuda-device-only", "-I", os.path.join(ROOT, "include"), "-I", csrc]
    names = ("pp_product_fp4", "pp_product_grad")
    jobs = [subprocess.Popen([HIPCC] + flags + [os.path.join(csrc, n + ".hip"), "-o", str(folder / (n + ".s"))], stderr=subprocess.DEVNULL) for n in names]
    found = {}
    for n, job in zip(names, jobs):
        assert job.wait(timeout=600) == 0
        lines = []
        for line in open(folder / (n + ".s")):
            start = re.match(r"(_Z\w*k_product\w+):", line)
            if start:
                lines = found.setdefault(start.group(1), [])
            elif line.startswith(".Lfunc_end"):
                lines = []
            lines.append(line.split(";")[0].strip())
    return found


def test_loops_hold_no_memory_but_what_is_counted(kernels):
    assert len(kernels) == 9 + 12 + 4           # forward: three tiles, three types; dx: four; dw: two, with db and without
    for name, lines in kernels.items():
        products = [i for i, l in enumerate(lines) if l.startswith("v_mfma")]
        assert products, name
        before = [l for l in lines[:products[-1]] if re.match(r"(scratch|flat)_", l)]
        assert not before, (name, before[:3])


def test_nothing_else_takes_m0(kernels):
    for name, lines in kernels.items():
        uses = [l for l in lines if re.search(r"\bm0\b", l)]
        assert uses and all(re.match(r"s_(add_u32|mov_b32) m0,", l) for l in uses), (name, uses[:5])
