"""The workspace of a prompt's scan (host only): one sized for the longest prompt serves all shorter ones."""
import pytest
import torch

from paper_2609_38166_amd import binding as B

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
