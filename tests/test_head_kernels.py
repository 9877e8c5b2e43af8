"""The compiler's report on the built kernels of the head's loss and the block norm:
accumulators and rows stay in registers."""

import os
import re
import struct
import subprocess

import pytest

from paper_2606_18114_amd import ops

READELF = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-readelf")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
KERNELS = re.compile(r"\d(head_(logits|dh|dw|dw_sum)|block_norm(_bwd)?|gather|list|finish|teach|"
                     r"terms|rows|sparse|dh_out)_kernel")


def code_objects(blob):
    at = blob.find(MAGIC)
    while at >= 0:
        pos = at + len(MAGIC)
        (n,) = struct.unpack_from("<Q", blob, pos)
        pos += 8
        for _ in range(n):
            off, size, length = struct.unpack_from("<QQQ", blob, pos)
            if b"gfx950" in blob[pos + 24:pos + 24 + length] and size:
                yield blob[at + off:at + off + size]
            pos += 24 + length
        at = blob.find(MAGIC, at + len(MAGIC))


def test_nothing_spills(tmp_path):
    if not os.path.exists(READELF):
        pytest.skip("llvm-readelf is needed")
    if not os.path.exists(ops.lib_path()):
        from paper_2606_18114_amd import build
        build.build(verbose=False)
    with open(ops.lib_path(), "rb") as f:
        blob = f.read()
    path = tmp_path / "kernel.co"
    bytes_of = {}
    for code in code_objects(blob):
        if not any(k in code for k in (b"block_norm_kernel", b"head_dh_kernel", b"finish_kernel")):
            continue
        path.write_bytes(code)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True,
                               check=True).stdout
        for m in re.finditer(r"\.private_segment_fixed_size: (\d+).*?\.symbol:\s+(\S+)\.kd", notes,
                             re.S):
            if KERNELS.search(m.group(2)):
                bytes_of[m.group(2)] = int(m.group(1))
    kinds = {KERNELS.search(n).group(1) for n in bytes_of}
    assert {"head_logits", "head_dh", "head_dw", "block_norm", "block_norm_bwd", "teach"} <= kinds
    assert not {n: b for n, b in bytes_of.items() if b}
