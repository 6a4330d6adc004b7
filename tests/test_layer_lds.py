"""The scan's LDS rows are declared at the alignment that its operand addresses rest on (exclusive ors within a row), not just
placed so by the compiler: read from the LLVM IR of this repository's source, before any pass."""
import os
import re
import subprocess

import pytest

from paper_2609_38166_amd import build

ROW = {"ILb1E": 256, "ILb0E": 512}            # bytes of a row of 128 channels: bf16, fp32


def test_lds_rows_are_aligned_to_a_row(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not found")
    out = str(tmp_path / "scan.ll")
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    subprocess.run([build.HIPCC, *flags, "-Xclang", "-disable-llvm-passes", "-I", os.path.join(build.ROOT, "include"),
                    "--offload-device-only", "-emit-llvm", "-S", os.path.join(build.PKG, "csrc", "lq_scan.hip"), "-o", out],
                   check=True, stderr=subprocess.DEVNULL)
    found = re.findall(r"^@\S*scan_prompt_kernel(ILb[01]E)\S*4rows = .*addrspace\(3\).*align (\d+)$", open(out).read(), re.M)
    assert len(found) == 6                    # two token types, three modes
    for kind, align in found:
        assert int(align) % ROW[kind] == 0, (kind, align)
