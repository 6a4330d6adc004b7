"""Sizes of products (tokens, n) that reach every kernel of leapquant_matmul (test infrastructure), whole tiles and then ragged ones.  The
choice does not depend on k.  tests/test_projection_choice.py holds each to its kernel."""
import torch

BF, F32 = torch.bfloat16, torch.float32

# (pieces of 16 tokens, pieces of 16 channels) of a workgroup: few tokens, or few tiles
FEW = {(1, 1): [(16, 272), (1, 271)],
       (1, 2): [(16, 5120), (70, 1000)],
       (1, 4): [(16, 10240), (8, 12285)],
       (2, 2): [(64, 2560), (259, 1000)],
       (2, 4): [(64, 5120), (300, 1100)]}
# (tokens, channels) of a tile: at most one tile a workgroup
TILES = {(64, 64): [(320, 1664), (299, 1661)],
         (64, 128): [(2752, 384), (2745, 379)],
         (128, 128): [(640, 3328), (633, 3323)],
         (192, 128): [(960, 4224), (953, 4219)],
         (128, 256): [(1024, 5632), (1017, 5627)],
         (192, 256): [(2496, 3328), (2489, 3323)],
         (256, 256): [(2560, 4864), (2553, 4859)]}
# ... and several (tiles of 64 tokens never are that many: larger ones take less time)
TURNS = {(128, 128): {BF: (6656, 1152), F32: (6656, 1152)},
         (192, 128): {BF: (8256, 1408), F32: (8256, 1408)},
         (128, 256): {BF: (3200, 5120), F32: (4480, 2816)},
         (192, 256): {BF: (4381, 5380), F32: (6720, 2816)},
         (256, 256): {BF: (8192, 4096)}}

TYPES = {(256, 256): (BF,)}         # (no fp32 outputs)


def one_each():
    """(kernel, tokens, n, type of output) of every kernel at each of its sizes with one tile a workgroup."""
    return [((kind, kernel), t, n, out) for kind, sizes in (("few", FEW), ("tile", TILES)) for kernel, s in sizes.items()
            for t, n in s for out in (TYPES.get(kernel, (BF, F32)) if kind == "tile" else (BF, F32))]


def several():
    return [(("tile", kernel), *size, out) for kernel, s in TURNS.items() for out, size in s.items()]


def name(case):
    (kind, (a, b)), t, n, out = case
    return f"{kind}{a}x{b}-{t}x{n}-{str(out)[6:]}"
