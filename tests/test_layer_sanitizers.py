"""AddressSanitizer / UndefinedBehaviorSanitizer build of the layer operators' host code: lq_api.hip and lq_layer_api.hip
(host pass only) with the launchers of tests/sanitize/layer_check.cpp.  A report aborts the executable."""
import os

import pytest

from tests.test_sanitizers import CLANG, ENV, HIPCC, ROOT, SAN, _run


def test_layer_host_code_under_asan_ubsan(tmp_path):
    if not (os.path.exists(HIPCC) and os.path.exists(CLANG)):
        pytest.skip("hipcc / clang++ not found")
    flags = ["-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
             "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
             "-Xarch_host", "-fno-sanitize-recover=all",
             "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2609_38166_amd", "csrc")]
    objs = []
    for src in (os.path.join(ROOT, "paper_2609_38166_amd", "csrc", "lq_api.hip"),
                os.path.join(ROOT, "paper_2609_38166_amd", "csrc", "lq_layer_api.hip"), os.path.join(SAN, "layer_check.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        _run([HIPCC, *flags, "-c", src, "-o", objs[-1]], str(tmp_path))
    exe = str(tmp_path / "layer_check")
    _run([CLANG, "-fsanitize=address,undefined", *objs, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe],
         str(tmp_path))
    r = _run([exe], str(tmp_path), env=ENV)
    assert "layer sanitizer check ok" in r.stdout
