"""Every kernel of the head's loss and the block norm in the built library, none left out: none
spills, and a kernel that is renamed or new has to be listed here."""

import os
import re
import subprocess

import pytest

from paper_2606_18114_amd import ops
from test_head_kernels import READELF, code_objects

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2606_18114_amd", "csrc")
SOURCES = ("head_gemm.hip", "head_loss.hip", "block_norm.hip")
KERNELS = {"head_logits", "head_dh", "head_dw", "head_dw_sum", "head_dw_few", "few", "terms",
           "rows", "gather", "finish", "teach", "sparse", "dh_out", "block_norm",
           "block_norm_bwd"}


def test_list_is_the_sources():
    found = set()
    for name in SOURCES:
        with open(os.path.join(CSRC, name)) as f:
            found |= set(re.findall(r"__global__[^;{]*?\bvoid\s+(\w+)_kernel\(", f.read()))
    assert found == KERNELS


def test_no_kernel_spills(tmp_path):
    if not os.path.exists(READELF):
        pytest.skip("llvm-readelf is needed")
    if not os.path.exists(ops.lib_path()):
        from paper_2606_18114_amd import build
        build.build(verbose=False)
    with open(ops.lib_path(), "rb") as f:
        blob = f.read()
    path, scratch = tmp_path / "kernel.co", {}
    for code in code_objects(blob):
        if not any(k in code for k in (b"block_norm_kernel", b"head_dh_kernel", b"finish_kernel")):
            continue
        path.write_bytes(code)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True,
                               check=True).stdout
        for m in re.finditer(r"\.private_segment_fixed_size: (\d+).*?\.symbol:\s+(\S+)\.kd"
                             r".*?\.vgpr_spill_count: (\d+)", notes, re.S):
            # (mangled: the name with its length before it)
            hit = re.search(r"(\d+)(%s)_kernel" % "|".join(sorted(KERNELS, key=len, reverse=True)),
                            m.group(2))
            if hit and int(hit.group(1)[-2:]) == len(hit.group(2)) + len("_kernel"):
                scratch[m.group(2)] = int(m.group(1)), int(m.group(3))
    kinds = {re.search(r"\d(%s)_kernel" % "|".join(sorted(KERNELS, key=len, reverse=True)), n)
             .group(1) for n in scratch}
    assert kinds == KERNELS
    assert not {n: b for n, b in scratch.items() if b != (0, 0)}
