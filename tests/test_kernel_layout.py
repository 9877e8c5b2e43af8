"""What the kernels' LDS structures promise: fields that are read as vectors of
16 bytes lie at multiples of 16 in every element of an array."""

import os
import subprocess

import pytest

from paper_2606_18114_amd import build

SNIPPET = """
#include <cstddef>
#include "seq_scan_dev.hpp"
template <int Q> void check() {
  typedef tmk::Toks<Q> T;
  static_assert(alignof(T) % 16 == 0 && sizeof(T) % 16 == 0);
  static_assert(offsetof(T, hi) % 16 == 0 && offsetof(T, lo) % 16 == 0);
  static_assert(offsetof(T, dt) % 16 == 0 && offsetof(T, ec) % 16 == 0);
  static_assert(offsetof(T, eq) % 16 == 0);
}
template void check<tmk::kScQ>();
template void check<tmk::kScChunk>();
"""


def test_token_values_are_read_as_vectors(tmp_path):
    try:
        hipcc = build.hipcc()
    except RuntimeError as e:
        pytest.skip(str(e))
    src = tmp_path / "layout.hip"
    src.write_text(SNIPPET)
    proc = subprocess.run([hipcc, "-x", "hip", *build.COMMON_FLAGS, "-c", "-o",
                           str(tmp_path / "layout.o"), "-I",
                           os.path.abspath(build.CSRC), str(src)], capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr
