"""What the kernels of a round on a drafted tree save to local memory, read off the compiler's own report: the streaming kernels nothing, the attention a
few bytes outside its loop over tiles, the verdict (128 registers, two CTAs to an SM) no more than it was measured with."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
# bytes stored, by what the kernel's name holds (Lb1E: rows that may begin off the boundaries of four entries)
MOST = {"adjust_": 0, "append_": 0, "tree_join_": 0, "tree_attention_kernel": 16, r"tree_verify_kernelILi\dELb0E": 140, r"tree_verify_kernelILi\dELb1E": 800}


def spills(tmp_path, name):
    csrc = os.path.join(ROOT, "paper_2507_12000_b200", "csrc")
    r = subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-Xptxas", "-v",
                        "-I", os.path.join(ROOT, "include"), "-I", csrc, "-c", "-o", str(tmp_path / (name + ".o")), os.path.join(csrc, name + ".cu")],
                       capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stderr[-2000:]
    return re.findall(r"Function properties for (\S+kernel\S+)\n\s*\d+ bytes stack frame, (\d+) bytes spill stores", r.stderr)


@pytest.mark.skipif(not shutil.which(NVCC), reason="needs nvcc")
def test_spills(tmp_path):
    with ThreadPoolExecutor(4) as pool:
        found = sum(pool.map(lambda n: spills(tmp_path, n), ("adjust_logits", "cache_append", "tree_attention", "tree_verify")), [])
    assert len(found) == 8 + 2 + 1 + 2 + 16 + 8
    for name, stored in found:
        most = [v for k, v in MOST.items() if re.search(k, name)]
        assert len(most) == 1 and int(stored) <= most[0], (name, stored)
