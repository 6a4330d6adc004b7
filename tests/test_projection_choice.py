"""Which kernel a product goes to, by the library's own launch code with a stand-in for the HIP runtime (host only): the sizes of
tests/projection_sizes.py reach the kernels that they are listed for, at any depth, and no kernel is left out."""
import os
import re
import subprocess

import pytest

from paper_2609_38166_amd import build
from tests import projection_sizes as Z

CSRC = os.path.join(build.PKG, "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"


def kernel(name):
    """A kernel's place in the tables of sizes and its type of output."""
    kind, *args = re.fullmatch(r"_ZN2lq\S*?\d+product_(few_)?kernelILb([01])((?:ELi\d+)+)E+v\S*", name).groups()
    n = [int(x) for x in args[1].split("ELi")[1:]]
    size = tuple(n) if kind else (16 * n[0] * n[2], 16 * n[1] * n[3])
    return ("few" if kind else "tile", size), Z.F32 if args[0] == "1" else Z.BF


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    if not (os.path.exists(build.HIPCC) and os.path.exists(CLANG)):
        pytest.skip("hipcc / clang++ not found")
    path = tmp_path_factory.mktemp("choice")
    objs = []
    for src in (os.path.join(CSRC, "lq_matmul.hip"), os.path.join(build.ROOT, "tests", "host", "product_choice.cpp")):
        objs.append(str(path / (os.path.basename(src) + ".o")))
        subprocess.run([build.HIPCC, "-x", "hip", "-std=c++17", "-O1", "-I", os.path.join(build.ROOT, "include"), "-I", CSRC,
                        "--offload-host-only", "-c", src, "-o", objs[-1]], check=True)
    exe = str(path / "product_choice")
    # (the device code that is not there is never looked at)
    subprocess.run([CLANG, *objs, "-no-pie", "-Wl,--unresolved-symbols=ignore-all", "-o", exe], check=True)

    def run(sizes):
        """All kernels, and of each (tokens, k, n, type): its kernel, workgroups and tiles."""
        text = "".join(f"{t} {k} {n} {int(out == Z.BF)}\n" for t, k, n, out in sizes)
        lines = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        have = [kernel(x.split()[1]) for x in lines if x.startswith("have ")]
        got = [x.split() for x in lines if not x.startswith("have ")]
        assert len(got) == len(sizes)
        return have, [(kernel(a), int(b), int(c)) for a, b, c in got]
    return run


@pytest.mark.parametrize("k", [16, 112, 128, 1168, 4096])
def test_sizes_reach_their_kernels(choose, k):
    one, several = Z.one_each(), Z.several()
    have, got = choose([(t, k, n, out) for _, t, n, out in one + several])
    for (want, t, n, out), (name, groups, tiles) in zip(one, got):
        assert name == (want, out) and groups == tiles, (t, n, out, name)
    for (want, t, n, out), (name, groups, tiles) in zip(several, got[len(one):]):
        assert name == (want, out) and groups < tiles, (t, n, out, name, groups, tiles)
    assert len(have) == len(set(have)) and set(have) == {name for name, _, _ in got[:len(one)]}


def test_tiles_without_a_size_of_several_turns_have_none(choose):
    """64 tokens a tile, by either number of channels: never more tiles than workgroups."""
    sizes = [(t, 1024, n, out) for t in range(33, 20000, 61) for n in range(16, 20000, 1009) for out in (Z.BF, Z.F32)]
    for size, (name, groups, tiles) in zip(sizes, choose(sizes)[1]):
        assert groups == tiles or name[0][0] == "tile" and name[0][1] in Z.TURNS, (size, name, groups, tiles)
