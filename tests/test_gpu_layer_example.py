"""The example runs the layer operators together: prompts, their final states quantized, single tokens."""
import importlib.util
import os

import pytest
import torch

from paper_2609_38166_amd import binding as B
from tests import layer_reference as R

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "prompt_then_decode.py")


def example():
    spec = importlib.util.spec_from_file_location("prompt_then_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_runs_and_the_eight_bit_path_stays_near():
    # codes of 7 bits and a sign, tokens and records in FP16: the state is within 2^-8 of a channel's largest value
    assert example().main(["--requests", "5", "--heads", "6", "--key-heads", "3", "--tokens", "40"]) < 2.0 ** -6


def test_prompt_then_dense_tokens_equal_the_whole_sequences():
    """The layer's chain against the same chain in 64 bits, prompt and tokens as one sequence (rounded where the chain
    stores bf16: the convolution's and the norm's outputs of the prompt)."""
    E = example()
    p = E.layer(2, 1)
    lengths, extra = [9, 70], 5
    n = sum(lengths)
    g = torch.Generator().manual_seed(3)
    x = torch.randn(n + 2 * extra, p["channels"], generator=g).bfloat16()
    dt = (0.5 * torch.randn(n + 2 * extra, 2, generator=g)).bfloat16()
    o, conv_state, state = E.prompts(p, x[:n].cuda(), dt[:n].cuda(), lengths)
    dec = E.Decoder(p, conv_state, state, False)
    tokens = [dec.step(x[n + 2 * t:n + 2 * t + 2].cuda(), dt[n + 2 * t:n + 2 * t + 2].cuda()).clone().cpu() for t in range(extra)]
    at = 0
    for b, length in enumerate(lengths):
        rows = torch.cat([x[at:at + length], x[n + b::2]])
        steps = torch.cat([dt[at:at + length], dt[n + b::2]])
        c, _, _ = R.conv(rows, p["conv"], [(0, len(rows))], p["conv_bias"], True)
        c[:length] = c[:length].float().bfloat16().double()
        v, k, q = E.split(p, c)
        q, k = (R.qk_norm(y, "l2", 1e-6) for y in (q, k))
        q[:length], k[:length] = (y[:length].float().bfloat16().double() for y in (q, k))
        want, size, _, _ = R.scan(q, k, v, steps, p["A"], [(0, len(rows))], p["D"], p["dt_bias"])
        got = torch.cat([o[at:at + length].cpu().double(), torch.stack([t[b] for t in tokens]).double()])
        # bf16 inputs of the scan may differ by a rounding (2^-8 of the value) where the chain's value lies on a boundary:
        # rarely, so the distance of the outputs as a whole stays that of one rounding to bf16
        assert float((got - want).norm() / want.norm()) < 2.0 ** -8
        assert bool(((got - want).abs() <= 2.0 ** -6 * size).all())
        at += length
