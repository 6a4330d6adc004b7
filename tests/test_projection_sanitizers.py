"""Sanitizer builds of the projection operators' host code: the entry points with stand-in launchers under AddressSanitizer and
UndefinedBehaviorSanitizer, and with their launchers under UndefinedBehaviorSanitizer (no GPU is visible to that executable;
the device code is compiled beside it, without a sanitizer).  A report aborts the executable."""
import os
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests.test_sanitizers import CLANG, ENV, HIPCC, ROOT, SAN, _run

CSRC = os.path.join(ROOT, "paper_2609_38166_amd", "csrc")
CHECK = os.path.join(SAN, "projection_check.cpp")


def build(tmp_path, srcs, flags, link):
    if not (os.path.exists(HIPCC) and os.path.exists(CLANG)):
        pytest.skip("hipcc / clang++ not found")
    flags = ["-x", "hip", "-std=c++17", "-O1", "-g", "-I", os.path.join(ROOT, "include"), "-I", CSRC, *flags]
    objs = [str(tmp_path / (os.path.basename(s) + ".o")) for s in srcs]
    with ThreadPoolExecutor(max_workers=4) as ex:
        list(ex.map(lambda p: _run([HIPCC, *flags, "-c", p[0], "-o", p[1]], str(tmp_path)), zip(srcs, objs)))
    exe = str(tmp_path / "projection_check")
    _run([CLANG, link, *objs, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe], str(tmp_path))
    return exe


def test_entry_points_under_asan_ubsan(tmp_path):
    srcs = [os.path.join(CSRC, "lq_api.hip"), os.path.join(CSRC, "lq_proj_api.hip"), CHECK]
    exe = build(tmp_path, srcs, ["--offload-host-only", "-DLAUNCHERS_STAND_IN", "-fno-omit-frame-pointer", "-Xarch_host", "-fsanitize=address",
                                 "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"],
                "-fsanitize=address,undefined")
    assert "projection check ok" in _run([exe], str(tmp_path), env=ENV).stdout


def test_launchers_under_ubsan(tmp_path):
    srcs = [os.path.join(CSRC, n) for n in ("lq_api.hip", "lq_proj_api.hip", "lq_rows.hip", "lq_matmul.hip")] + [CHECK]
    exe = build(tmp_path, srcs, ["--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                                 "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"], "-fsanitize=undefined")
    r = _run([exe], str(tmp_path), env=dict(ENV, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1"))
    assert "projection check ok" in r.stdout
