"""The workspace of a prompt's scan (host only): one sized for the longest prompt serves all shorter ones."""
import ctypes as C

import pytest
import torch

from paper_2609_38166_amd import binding as B
from tests.test_layer_abi import GOOD, scan

TOKENS = sorted({*range(0, 1100, 7), 64, 192, 193, 256, 257, 512, 520, 1024, 2048, 2056, 4096, 8192, 8319, 8320, 16383, 32768, 33279,
                 33280, 65536, 1 << 20})


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,hv", [(1, 1), (1, 3), (2, 4), (1, 64), (1, 100), (1, 127), (1, 128), (1, 170), (1, 511), (15, 32),
                                      (16, 32), (100, 4), (300, 1)])
def test_the_need_without_max_len_holds_for_fewer_tokens_and_any_max_len(batch, hv, dtype):
    d = B.make_dims(batch, hv, 1, rule=B.LQ_RULE_ADD)
    most = 0
    for n in TOKENS:
        for longest in {1, n // 3, n - 1, n, n + 1, 1 << 30} - {0, -1}:
            most = max(most, B.leapquant_scan_workspace_bytes(d, n, dtype, longest))
        assert B.leapquant_scan_workspace_bytes(d, n, dtype) >= most, n
    # and it is no wild guess: some call comes near it
    assert B.leapquant_scan_workspace_bytes(d, TOKENS[-1], dtype) <= 1.25 * most


@pytest.mark.parametrize("tokens,needs", [(64, False), (256, False), (257, True), (1 << 16, True)])
def test_a_long_prompt_on_few_heads_needs_its_workspace(tokens, needs):
    """... and is refused without it, or with a short or misaligned one, before anything is enqueued."""
    L, d = B.lib(), B.make_dims(1, 4, 2, rule=B.LQ_RULE_ADD)
    for max_len in (0, tokens):
        s = scan(tokens=tokens, n_slots=1, max_len=max_len)
        n = C.c_size_t(0)
        assert L.leapquant_scan_workspace_bytes(C.byref(d), C.byref(s), C.byref(n)) == B.LQ_OK
        assert bool(n.value) == needs
        if not needs:
            continue
        s.workspace_bytes = n.value
        assert L.leapquant_scan_prompt(C.byref(d), C.byref(s), None) == B.LQ_EINVAL
        s.workspace = GOOD + 8
        assert L.leapquant_scan_prompt(C.byref(d), C.byref(s), None) == B.LQ_EALIGN
        s.workspace, s.workspace_bytes = GOOD, n.value - 1
        assert L.leapquant_scan_prompt(C.byref(d), C.byref(s), None) == B.LQ_EINVAL
