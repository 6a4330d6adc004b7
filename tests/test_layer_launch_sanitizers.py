"""UndefinedBehaviorSanitizer build of the layer operators' launchers with the C entry points before them (host code; the device
code is compiled beside it, without a sanitizer, and not run: no GPU is visible to the executable)."""
import os
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests.test_sanitizers import CLANG, ENV, HIPCC, ROOT, SAN, _run

CSRC = os.path.join(ROOT, "paper_2609_38166_amd", "csrc")


def test_layer_launchers_under_ubsan(tmp_path):
    if not (os.path.exists(HIPCC) and os.path.exists(CLANG)):
        pytest.skip("hipcc / clang++ not found")
    flags = ["-x", "hip", "--offload-arch=gfx950", "-std=c++17", "-O1", "-g",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    srcs = [os.path.join(CSRC, n) for n in ("lq_api.hip", "lq_layer_api.hip", "lq_conv.hip", "lq_norm.hip", "lq_scan.hip")]
    srcs.append(os.path.join(SAN, "layer_launch_check.cpp"))
    objs = [str(tmp_path / (os.path.basename(s) + ".o")) for s in srcs]
    with ThreadPoolExecutor(max_workers=4) as ex:
        list(ex.map(lambda p: _run([HIPCC, *flags, "-c", p[0], "-o", p[1]], str(tmp_path)), zip(srcs, objs)))
    exe = str(tmp_path / "layer_launch_check")
    _run([CLANG, "-fsanitize=undefined", *objs, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe], str(tmp_path))
    r = _run([exe], str(tmp_path), env=dict(ENV, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1"))
    assert "layer launch check ok" in r.stdout
