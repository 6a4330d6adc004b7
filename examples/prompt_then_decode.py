"""One state space layer from its prompts to its single tokens, all in the library's kernels.

A batch of prompts of different lengths goes through the short convolution, the norm of queries and keys and the selective
scan; the final states are quantized, and decoding goes on token by token over the 8-bit state, beside the same tokens over
the dense fp32 state.  Weights and inputs are random: the example shows the calls, and how far the 8-bit path is from the
dense one.

    python examples/prompt_then_decode.py [--requests 8] [--heads 8] [--key-heads 4] [--tokens 64]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_38166_amd import binding as B  # noqa: E402

D = 128


def layer(heads, key_heads, device="cuda", seed=0):
    """The layer's parameters: a convolution over [values | keys | queries], step bias, decay rates, skip weights."""
    g = torch.Generator(device=device).manual_seed(seed)
    channels = (heads + 2 * key_heads) * D
    step = torch.exp(torch.empty(heads, device=device).uniform_(-6.9, -2.3, generator=g))       # 0.001 .. 0.1
    return {"heads": heads, "key_heads": key_heads, "channels": channels,
            "conv": torch.randn(channels, 4, device=device, generator=g) / 2,
            "conv_bias": torch.randn(channels, device=device, generator=g) / 10,
            "dt_bias": step + torch.log(-torch.expm1(-step)),
            "A": -torch.empty(heads, device=device).uniform_(1, 16, generator=g),
            "D": torch.ones(heads, device=device)}


def split(p, c):
    """Values, keys and queries of convolved rows, as views (rows stay channels apart)."""
    n, hv, hk = c.shape[0], p["heads"], p["key_heads"]
    v, k, q = c.split([hv * D, hk * D, hk * D], dim=1)
    return v.view(n, hv, D), k.view(n, hk, D), q.view(n, hk, D)


def prompts(p, x, dt, lengths):
    """Outputs of packed prompts [tokens, heads, 128], and the states that decoding starts from."""
    batch, tokens = len(lengths), sum(lengths)
    cu = torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32).cuda()
    dims = B.make_dims(batch, p["heads"], p["key_heads"], rule=B.LQ_RULE_ADD)
    conv_state = torch.empty((batch, 3, p["channels"]), dtype=x.dtype, device="cuda")
    state = torch.empty((batch, p["heads"], D, D), device="cuda")
    c = torch.empty_like(x)
    B.leapquant_conv_prompt(x, p["conv"], c, cu, bias=p["conv_bias"], state=conv_state)
    v, k, q = split(p, c)
    kn, qn = (torch.empty((tokens, p["key_heads"], D), dtype=x.dtype, device="cuda") for _ in range(2))
    B.leapquant_qk_norm(q, k, qn, kn)
    o = torch.empty((tokens, p["heads"], D), dtype=x.dtype, device="cuda")
    B.leapquant_scan_prompt(dims, qn, kn, v, dt, p["A"], o, cu, D=p["D"], dt_bias=p["dt_bias"], state=state, max_len=max(lengths))
    return o, conv_state, state


class Decoder:
    """Single tokens of a batch over the 8-bit state (quantized) or the dense one."""

    def __init__(self, p, conv_state, state, quantized, window=16):
        self.p, self.batch, self.quantized = p, state.shape[0], quantized
        self.dims = B.make_dims(self.batch, p["heads"], p["key_heads"], window=window, n_comp=4, rule=B.LQ_RULE_ADD)
        self.conv_state, self.state = conv_state.clone(), state.clone()
        if quantized:
            self.state = B.State.empty(self.dims)
            B.leapquant_quantize_state(self.dims, state, self.state)
        n, hv, hk = self.batch, p["heads"], p["key_heads"]
        new = lambda *shape: torch.empty(shape, device="cuda")                              # noqa: E731
        self.c, self.q, self.k, self.v = new(n, p["channels"]), new(n, hk, D), new(n, hk, D), new(n, hv, D)
        self.alpha, self.beta, self.o = new(n, hv), new(n, hv), new(n, hv, D)
        self.position = 0

    def step(self, x, dt):
        p = self.p
        B.leapquant_conv_step(x, p["conv"], self.c, self.conv_state, bias=p["conv_bias"])    # fp32 out, for the decode step
        v, k, q = split(p, self.c)
        B.leapquant_qk_norm(q, k, self.q, self.k)
        dt = dt.float()
        if not self.quantized:
            B.leapquant_scan_step(self.dims, self.state, self.q, self.k, v, dt, p["A"], self.o, D=p["D"], dt_bias=p["dt_bias"])
            return self.o
        self.v.copy_(v)                                                                      # the decode step reads dense rows
        B.leapquant_scan_gates(self.dims, dt, p["A"], self.alpha, self.beta, dt_bias=p["dt_bias"])
        B.leapquant_decode_step(self.dims, self.state, self.q, self.k, self.v, self.alpha, self.beta, self.o)
        self.position += 1
        if self.position % self.dims.window == 0:
            B.leapquant_window_commit(self.dims, self.state)
        return self.o.addcmul_(p["D"][:, None], self.v)


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--requests", type=int, default=8)
    a.add_argument("--heads", type=int, default=8)
    a.add_argument("--key-heads", type=int, default=4)
    a.add_argument("--tokens", type=int, default=64)
    a = a.parse_args(argv)
    torch.manual_seed(0)
    p = layer(a.heads, a.key_heads)
    lengths = [37 + 61 * i for i in range(a.requests)]
    x = torch.randn(sum(lengths), p["channels"], device="cuda").bfloat16()
    dt = (0.5 * torch.randn(sum(lengths), a.heads, device="cuda")).bfloat16()
    o, conv_state, state = prompts(p, x, dt, lengths)
    print(f"prompts: {a.requests} of {lengths[0]}..{lengths[-1]} tokens, output rms {o.float().square().mean().sqrt():.3f}")
    eight, dense = (Decoder(p, conv_state, state, q) for q in (True, False))
    off = size = 0.0
    for t in range(a.tokens):
        x = torch.randn(a.requests, p["channels"], device="cuda").bfloat16()
        dt = (0.5 * torch.randn(a.requests, a.heads, device="cuda")).bfloat16()
        got, want = eight.step(x, dt), dense.step(x, dt)
        off, size = off + float((got - want).square().sum()), size + float(want.square().sum())
    assert B.leapquant_check_error(eight.state) == 0
    rel = (off / size) ** 0.5
    print(f"decode: {a.tokens} tokens, 8-bit state against dense fp32: relative distance of the outputs {rel:.2e}")
    return rel


if __name__ == "__main__":
    main()
