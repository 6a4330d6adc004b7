"""The projection operators' kernels keep to registers: no scratch memory and no spilled vector register in any of them, by what
the compiler reports of this repository's sources with the build's own options."""
import os
import re
import subprocess

import pytest

from paper_2609_38166_amd import build


@pytest.mark.parametrize("source", ["lq_matmul.hip", "lq_rows.hip"])
def test_kernels_use_no_scratch(source, tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not found")
    flags = [f for f in build.FLAGS if f != "-fPIC"] + build.SCHED.get(source, [])
    r = subprocess.run([build.HIPCC, *flags, "-I", os.path.join(build.ROOT, "include"), "--offload-device-only", "-c",
                        os.path.join(build.PKG, "csrc", source), "-o", str(tmp_path / "o"), "-Rpass-analysis=kernel-resource-usage"],
                       check=True, capture_output=True, text=True)
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    scratch = [int(x) for x in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)]
    spilled = [int(x) for x in re.findall(r"VGPRs Spill: (\d+)", r.stderr)]
    assert len(names) == len(scratch) == len(spilled) >= 20, r.stderr[-2000:]
    assert not [x for x in zip(names, scratch, spilled) if x[1] or x[2]]
