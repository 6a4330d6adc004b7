"""The projection operators as they are used: together with the layer operators around them, in captured graphs, on several
streams, and over arrays past 32-bit offsets.  Each stage is compared with its definition in 64 bits on what the stage before
gave on the GPU; tolerances are those of tests/test_gpu_projection.py and tests/test_gpu_layer.py."""
import pytest
import torch

from paper_2609_38166_amd import binding as B
from tests import layer_reference as L
from tests import projection_reference as R
from tests.test_gpu_projection import BF, E4, F32, U, close, close_codes, encoded, rnd, scales

pytestmark = pytest.mark.gpu

HIDDEN, HV, HK, D = 512, 4, 2, 128
CONV = (HV + 2 * HK) * D
WIDE = CONV + HV * D + HV                                       # values, keys, queries | gate | dt


def weights(seed=0):
    """A layer's parameters, its two weights in E4M3."""
    p = {"norm": 1 + 0.1 * rnd(seed, HIDDEN).cuda(), "head_norm": 1 + 0.1 * rnd(seed + 1, D).cuda(),
         "conv": rnd(seed + 2, CONV, 4).cuda() / 2, "A": -torch.rand(HV, device="cuda") - 0.5, "dt_bias": rnd(seed + 3, HV).cuda() - 3}
    for name, n, k in (("in", WIDE, HIDDEN), ("out", HIDDEN, HV * D)):
        w = (rnd(seed + 4 + n, n, k) / k ** 0.5).bfloat16().cuda()
        p[name] = torch.empty((n, k), dtype=E4, device="cuda")
        p[name + "_scale"] = torch.empty((R.blocks(n), R.blocks(k)), device="cuda")
        B.leapquant_quantize_weight(w, p[name], p[name + "_scale"])
    return p


class Layer:
    """A layer over t rows, its buffers made once; `residual` [t, HIDDEN] fp32 is updated in place."""

    def __init__(self, p, t, batch, prompt):
        new = lambda *s, dtype=BF: torch.empty(s, dtype=dtype, device="cuda")                   # noqa: E731
        self.p, self.prompt, self.dims = p, prompt, B.make_dims(batch, HV, HK, rule=B.LQ_RULE_ADD)
        self.h8, self.hs = new(t, HIDDEN, dtype=E4), new(t, HIDDEN // 128, dtype=F32)
        self.wide = new(t, WIDE + 4)[:, :WIDE]                                                  # (rows start at multiples of 16 bytes)
        self.c, self.q, self.k = new(t, CONV), new(t, HK, D), new(t, HK, D)
        self.o = new(t, HV, D)
        self.g8, self.gs = new(t, HV, D, dtype=E4), new(t, HV, dtype=F32)
        self.y = new(t, HIDDEN)

    def run(self, x, residual, conv_state, state, cu=None, max_len=0):
        p, t = self.p, x.shape[0]
        B.leapquant_add_norm(x, self.h8, residual=residual, residual_out=residual, weight=p["norm"], scale=self.hs)
        B.leapquant_matmul(self.h8, self.hs, p["in"], p["in_scale"], self.wide)
        x, gate, dt = self.wide.split([CONV, HV * D, HV], dim=1)
        if self.prompt:
            B.leapquant_conv_prompt(x, p["conv"], self.c, cu, state=conv_state)
        else:
            B.leapquant_conv_step(x, p["conv"], self.c, conv_state)
        v, k, q = self.c.split([HV * D, HK * D, HK * D], dim=1)
        v = v.view(t, HV, D)
        B.leapquant_qk_norm(q.view(t, HK, D), k.view(t, HK, D), self.q, self.k)
        if self.prompt:
            B.leapquant_scan_prompt(self.dims, self.q, self.k, v, dt, p["A"], self.o, cu, dt_bias=p["dt_bias"], state=state, max_len=max_len)
        else:
            B.leapquant_scan_step(self.dims, state, self.q, self.k, v, dt, p["A"], self.o, dt_bias=p["dt_bias"])
        B.leapquant_gate_norm(self.o, gate.view(t, HV, D), self.g8, weight=p["head_norm"], scale=self.gs)
        B.leapquant_matmul(self.g8.view(t, -1), self.gs, p["out"], p["out_scale"], self.y)
        return self.y


def products(x8, xs, w8, ws, got):
    y, size = R.matmul(x8, xs, w8, ws)
    close(got, y, ((256 + R.blocks(x8.shape[1]) + 20) * U + 7 * 2.0 ** -13) * size)


@pytest.mark.parametrize("lens", [[1], [9, 70, 1, 0, 33]])
def test_a_layer_from_hidden_rows_to_hidden_rows(lens):
    p, t = weights(), sum(lens)
    cu = torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32)
    x, r = rnd(50, t, HIDDEN).bfloat16(), rnd(51, t, HIDDEN)
    residual = r.cuda()
    conv_state, state = torch.zeros(len(lens), 3, CONV, dtype=BF, device="cuda"), torch.zeros(len(lens), HV, D, D, device="cuda")
    f = Layer(p, t, len(lens), True)
    y = f.run(x.cuda(), residual, conv_state, state, cu.cuda(), max(lens))
    h, want = R.add_norm(x, r, p["norm"])
    close(residual, h, U * (x.double().abs() + r.double().abs()))
    close_codes(f.h8, f.hs, want, 80 * U * (want.abs() + 1e-3 * (x.double().abs() + r.double().abs())) + 80 * U, R.row_scales(want))
    products(f.h8, f.hs, p["in"], p["in_scale"], f.wide)
    xw, gate, dt = f.wide.cpu().split([CONV, HV * D, HV], dim=1)
    spans = L.lengths(cu, t)
    want, size, _ = L.conv(xw, p["conv"], spans, None, True)
    close(f.c, want, 1e-6 * (size + 1))
    v, k, q = f.c.cpu().split([HV * D, HK * D, HK * D], dim=1)
    for got, z in ((f.q, q), (f.k, k)):
        want = L.qk_norm(z.reshape(t, HK, D), "l2", 1e-6)
        close(got, want, 24 * U * want.abs().amax(-1, keepdim=True))
    want, size, new, nsize = L.scan(f.q, f.k, v.reshape(t, HV, D), dt, p["A"], spans, None, p["dt_bias"])
    count = min(max(lens), 512)
    close(f.o, want, (2 * count + 16) * U * size + 2.0 ** -16 * size)
    close(state, new, (2 * count + 16) * U * nsize + 2.0 ** -16 * nsize)
    want = R.gate_norm(f.o, gate.reshape(t, HV, D), p["head_norm"]).reshape(t, -1)
    close_codes(f.g8.view(t, -1), f.gs, want, 48 * U * want.abs(), R.row_scales(want))
    products(f.g8.view(t, -1), f.gs, p["out"], p["out_scale"], y)


def test_tokens_of_a_layer_in_a_captured_graph():
    """Two layers in one graph, replayed on new inputs with eager work of its own in between, against the same calls made
    eagerly."""
    batch, steps = 5, 4
    layers = [Layer(weights(10 * i), batch, batch, False) for i in range(2)]
    xs, r0 = rnd(60, steps, batch, HIDDEN).bfloat16().cuda(), rnd(61, batch, HIDDEN).cuda()

    def states():
        return [(torch.zeros(batch, 3, CONV, dtype=BF, device="cuda"), torch.zeros(batch, HV, D, D, device="cuda")) for _ in layers]

    def token(x, r, st):
        for f, s in zip(layers, st):
            x = f.run(x, r, *s)
        return x

    st, want = states(), []
    for i in range(steps):
        r = r0.clone()
        want.append((token(xs[i], r, st).clone(), r))
    final = [z.clone() for s in st for z in s]
    st, x, r = states(), xs[0].clone(), r0.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        token(x, r, st)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = token(x, r, st)
    for s in st:
        for z in s:
            z.zero_()
    for i in range(steps):
        x.copy_(xs[i])
        r.copy_(r0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i][0]) and torch.equal(r, want[i][1]), i
        other = torch.empty(300, 256, device="cuda")            # eager work between the replays
        B.leapquant_matmul(encoded(1, 300, 128).cuda(), scales(2, 300, 1).cuda(), encoded(3, 256, 128).cuda(), scales(4, 2, 1).cuda(), other)
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((z for s in st for z in s), final))


def test_calls_on_several_streams_and_on_a_given_one():
    sizes = [(300, 1040, 520), (1, 4096, 600), (77, 272, 1000), (2100, 512, 2048)]
    jobs = []
    for i, (t, k, n) in enumerate(sizes):
        a = (encoded(4 * i, t, k).cuda(), scales(4 * i + 1, t, R.blocks(k)).cuda(), encoded(4 * i + 2, n, k).cuda(),
             scales(4 * i + 3, R.blocks(n), R.blocks(k)).cuda())
        wide = -(-n // 8) * 8
        want = torch.empty(t, wide, device="cuda")[:, :n]
        B.leapquant_matmul(*a, want)
        jobs.append((a, want, [torch.empty(t, wide, device="cuda")[:, :n] for _ in range(2)]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for turn in range(3):
        for s, (a, want, out) in zip(streams, jobs):
            with torch.cuda.stream(s):
                B.leapquant_matmul(*a, out[0])
            B.leapquant_matmul(*a, out[1], stream=s)
    torch.cuda.synchronize()
    for a, want, out in jobs:
        assert torch.equal(out[0], want) and torch.equal(out[1], want)


def test_rows_past_32_bit_offsets():
    """Rows far apart, so that the last ones lie past 2^32 bytes (and 2^32 elements)."""
    apart = (1 << 32) + 64
    x = torch.zeros(apart + 256, dtype=BF, device="cuda").as_strided((2, 256), (apart, 1))
    x.copy_(rnd(1, 2, 256))
    out = torch.zeros(apart + 256, dtype=E4, device="cuda").as_strided((2, 256), (apart, 1))
    scale = torch.zeros(2, 2, device="cuda")
    B.leapquant_add_norm(x, out, scale=scale)
    _, y = R.add_norm(x.cpu())
    close_codes(out, scale, y, 80 * U * y.abs(), R.row_scales(y))
    gate = rnd(2, 2, 2, 128).cuda()
    got = torch.zeros(apart + 256, dtype=BF, device="cuda").as_strided((2, 2, 128), (apart, 128, 1))
    B.leapquant_gate_norm(x.as_strided((2, 2, 128), (apart, 128, 1)), gate, got)
    want = R.gate_norm(x.cpu().view(2, 2, 128), gate)
    close(got, want, 48 * U * want.abs())


@pytest.mark.parametrize("out_dtype", [BF, F32])
def test_products_past_32_bit_offsets(out_dtype):
    """Outputs, rows of x and rows of the weight past 2^32 bytes: the last rows against those of a small call."""
    t, n, k = 560000, 4160, 128
    x8, xs = encoded(1, 64, k).cuda(), scales(2, 64, 1).cuda()
    w8, ws = encoded(3, n, k).cuda(), scales(4, R.blocks(n), 1).cuda()
    far = 8192                                                  # rows of x 8 KiB apart: 4.6 GB
    x = torch.empty(t, far, dtype=torch.uint8, device="cuda").view(E4)[:, :k]
    x.view(torch.uint8).zero_()
    x.view(torch.uint8)[-64:] = x8.view(torch.uint8)
    x_scale = torch.ones(t, 1, device="cuda")
    x_scale[-64:] = xs
    out = torch.empty(t, n, dtype=out_dtype, device="cuda")
    B.leapquant_matmul(x, x_scale, w8, ws, out)
    y, size = R.matmul(x8, xs, w8, ws)
    close(out[-64:], y, (280 * U + (7 * 2.0 ** -13 if out_dtype == BF else 0)) * size)
    assert (out[0] == 0).all() and (out[t // 2] == 0).all()
    del out, x
    rows = 600
    wide = torch.empty(rows, (1 << 23), dtype=torch.uint8, device="cuda").view(E4)[:, :k]      # 5 GB between the first and the last
    wide.copy_(w8[:rows])
    for tokens in (3, 64):
        got = torch.empty(tokens, rows, dtype=out_dtype, device="cuda")
        B.leapquant_matmul(x8[:tokens], xs[:tokens], wide, ws[:R.blocks(rows)], got)
        close(got, y[:tokens, :rows], (280 * U + (7 * 2.0 ** -13 if out_dtype == BF else 0)) * size[:tokens, :rows])
