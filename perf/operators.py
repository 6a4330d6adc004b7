"""Performance cases of the layer operators around the decode step: what a serving program runs on a layer's tokens before
the recurrent state takes over, for whole prompts and for single tokens.

Operators
  conv_prompt   short causal convolution per channel over packed sequences, with its state (leapquant_conv_prompt)
  conv_step     the same for one token of every request (leapquant_conv_step)
  qk_norm       norm of queries and keys per head, with the position rotation (leapquant_qk_norm)
  scan_prompt   selective state space scan over packed sequences: outputs and final states (leapquant_scan_prompt)
  scan_step     the same for one token of every request, dense state (leapquant_scan_step)

Inputs are drawn on the GPU from the seed.  Activations are SiLU(N(0, 1)) or N(0, 1), queries and keys of the scan unit
vectors; steps softplus(dt + bias) start out log-uniform in [0.001, 0.1] and A uniform in [-16, -1], as such layers are
initialised; sequences of a packed batch differ in length, and a batch of four or more holds an empty one and one of a
single token.

`own` chooses the side: the framework's calls, or the plain form in elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

D = 128
CHUNK = 64
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def _conv(op, seqs, tokens, channels, width, dtype, out, silu=True, bias=True, carry=True, name=None):
    c = {"op": op, "seqs": seqs, "tokens": tokens, "channels": channels, "width": width, "dtype": dtype, "out": out,
         "silu": silu, "bias": bias, "carry": carry}
    return dict(c, name=name) if name else c


def _norm(tokens, heads_q, heads_k, d, norm, rot, interleaved, dtype, out, name=None):
    c = {"op": "qk_norm", "tokens": tokens, "heads_q": heads_q, "heads_k": heads_k, "d": d, "norm": norm, "rot": rot,
         "interleaved": interleaved, "dtype": dtype, "out": out}
    return dict(c, name=name) if name else c


def _scan(op, seqs, tokens, heads_v, heads_k, dtype, state="f32", skip=True, carry=True, name=None):
    c = {"op": op, "seqs": seqs, "tokens": tokens, "heads_v": heads_v, "heads_k": heads_k, "dtype": dtype,
         "state": state, "skip": skip, "carry": carry}
    return dict(c, name=name) if name else c


def listed():
    return [
        # prompts of 16 requests through the GQA GDN layer's convolution (32 value and 2 x 16 key heads of 128)
        _conv("conv_prompt", 16, 8192, 8192, 4, "bf16", "bf16", name="conv_prompt_gqa"),
        # a few short prompts of the tiny layer, fp32, odd width, no activation
        _conv("conv_prompt", 5, 131, 1536, 3, "f32", "f32", silu=False, bias=False, carry=False, name="conv_prompt_short"),
        # one token of 256 requests of the KDA layer (3 x 32 heads of 128), output in the decode step's fp32
        _conv("conv_step", 256, 256, 12288, 4, "bf16", "f32", name="conv_step_batch256"),
        # one token of the tiny layer's requests: latency
        _conv("conv_step", 4, 4, 1536, 4, "bf16", "bf16", name="conv_step_tiny"),
        # unit-norm queries and keys of a prompt of the GQA GDN layer
        _norm(8192, 16, 16, D, "l2", 0, False, "bf16", "bf16", name="qk_norm_prompt"),
        # one token of 64 requests: weighted norm, half of the channels rotated, output in fp32
        _norm(64, 32, 4, D, "rms", 64, False, "bf16", "f32", name="qk_norm_tokens"),
        # one long prompt of the long-trace layer (16 heads, 32768 tokens)
        _scan("scan_prompt", 1, 32768, 16, 16, "bf16", carry=False, name="scan_prompt_long"),
        # ragged prompts of 64 requests of the GQA GDN layer that continue from their states
        _scan("scan_prompt", 64, 16383, 32, 16, "bf16", name="scan_prompt_ragged"),
        # one prompt in fp32, all value heads on one key head
        _scan("scan_prompt", 1, 2048, 32, 1, "f32", carry=False, name="scan_prompt_fp32"),
        # a few short prompts of the tiny layer: latency
        _scan("scan_prompt", 4, 61, 4, 4, "bf16", carry=False, skip=False, name="scan_prompt_tiny"),
        # one token of 256 requests x 32 heads, fp32 state
        _scan("scan_step", 256, 256, 32, 32, "bf16", name="scan_step_batch256"),
        # one token of the tiny layer's requests, bf16 state: latency
        _scan("scan_step", 4, 4, 4, 4, "bf16", state="bf16", name="scan_step_tiny"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["conv_prompt", "conv_step", "qk_norm", "scan_prompt", "scan_prompt", "scan_step"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    heads_k = rng.choice([1, 2, 3, 4, 8, 16])
    heads_v = heads_k * rng.choice([1, 1, 2, 3] if heads_k < 16 else [1, 2])
    if op in ("conv_prompt", "conv_step"):
        channels = (heads_v + 2 * heads_k) * D
        seqs = _log_int(rng, 1, 256)
        tokens = seqs if op == "conv_step" else max(seqs, _log_int(rng, 16, (1 << 25) // channels))
        return _conv(op, seqs, tokens, channels, rng.choice([2, 3, 4, 4]), dtype, rng.choice([dtype, "f32"]),
                     silu=rng.random() < 0.7, bias=rng.random() < 0.5, carry=rng.random() < 0.5 or op == "conv_step")
    if op == "qk_norm":
        d = rng.choice([64, D, D, 256])
        return _norm(_log_int(rng, 1, (1 << 24) // (d * (heads_v + heads_k))), heads_v, heads_k, d,
                     rng.choice(["l2", "rms"]), rng.choice([0, d // 4, d // 2, d]), rng.random() < 0.5, dtype,
                     rng.choice([dtype, "f32"]))
    if op == "scan_prompt":
        seqs = _log_int(rng, 1, 64)
        most = (1 << 19) // (heads_v * (4 if dtype == "f32" else 1))
        return _scan(op, seqs, max(seqs, _log_int(rng, 16, most)), heads_v, heads_k, dtype, skip=rng.random() < 0.7,
                     carry=rng.random() < 0.5)
    batch = _log_int(rng, 1, 8192 // heads_v)
    return _scan(op, batch, batch, heads_v, heads_k, dtype, state=rng.choice(["f32", "bf16"]), skip=rng.random() < 0.7)


# ---------------------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _lengths(case, seed):
    """Lengths of a packed batch: a random split of the tokens; of four or more sequences one is empty, one a single token."""
    n, total = case["seqs"], case["tokens"]
    rng = random.Random(seed)
    if n >= 4 and total >= n:
        special = [0, 1]
    else:
        special = []
    rest, left = n - len(special), total - sum(special)
    w = [rng.uniform(0.25, 1.75) for _ in range(rest)]
    cut, acc = [0], 0.0
    for x in w:
        acc += x
        cut.append(int(round(left * acc / sum(w))))
    lens = [cut[i + 1] - cut[i] for i in range(rest)] + special
    rng.shuffle(lens)
    return lens


def _sequences(case, seed):
    lens = _lengths(case, seed)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return {"lens": lens, "cu": torch.tensor(cu, dtype=torch.int32, device="cuda")}


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _silu(x):
    return x / (1 + torch.exp(-x))


def prepare(case, seed):
    g = _generator(seed)
    dt = TYPES[case["dtype"]]
    op, n = case["op"], case["tokens"]
    if op in ("conv_prompt", "conv_step"):
        c, k = case["channels"], case["width"]
        s = {"x": _randn(g, n, c).to(dt), "weight": _randn(g, c, k) / math.sqrt(k),
             "bias": _randn(g, c) * 0.1 if case["bias"] else None,
             "state": _randn(g, case["seqs"], k - 1, c).to(dt),
             "out": torch.empty((n, c), dtype=TYPES[case["out"]], device="cuda")}
        if op == "conv_prompt":
            s.update(_sequences(case, seed))
    elif op == "qk_norm":
        d, hq, hk = case["d"], case["heads_q"], case["heads_k"]
        s = {"q": _silu(_randn(g, n, hq, d)).to(dt), "k": _silu(_randn(g, n, hk, d)).to(dt)}
        s["q_out"], s["k_out"] = (torch.empty(x.shape, dtype=TYPES[case["out"]], device="cuda") for x in (s["q"], s["k"]))
        rms = case["norm"] == "rms"
        s["q_weight"], s["k_weight"] = (1 + 0.1 * _randn(g, d) if rms else None for _ in range(2))
        s["cos"] = s["sin"] = s["positions"] = None
        if case["rot"]:
            freq = 10000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])
            angle = torch.arange(8192, device="cuda", dtype=torch.float64)[:, None] * freq
            s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
            s["positions"] = torch.randint(0, 8192, (n,), generator=g, device="cuda", dtype=torch.int32)
    else:
        hv, hk = case["heads_v"], case["heads_k"]
        step0 = torch.exp(torch.rand(hv, generator=g, device="cuda") * (math.log(0.1) - math.log(0.001)) + math.log(0.001))
        s = {"v": _silu(_randn(g, n, hv, D)).to(dt), "dt": (0.5 * _randn(g, n, hv)).to(dt)}
        for name in ("q", "k"):
            x = _randn(g, n, hk, D)
            s[name] = (x / x.norm(dim=-1, keepdim=True)).to(dt)
        s["dt_bias"] = step0 + torch.log(-torch.expm1(-step0))
        s["A"] = -(1 + 15 * torch.rand(hv, generator=g, device="cuda"))
        s["D"] = 1 + 0.1 * _randn(g, hv) if case["skip"] else None
        s["state"] = (0.1 * _randn(g, case["seqs"], hv, D, D)).to(TYPES[case["state"]])
        s["out"] = torch.empty((n, hv, D), dtype=dt, device="cuda")
        if op == "scan_prompt":
            s.update(_sequences(case, seed))
    s["case"] = case
    return s


# ------------------------------------------------------------------------------------------- the framework's operators

def _run_own(s):
    from paper_2609_38166_amd import binding as B
    case, op = s["case"], s["case"]["op"]
    if op == "conv_prompt":
        B.leapquant_conv_prompt(s["x"], s["weight"], s["out"], s["cu"], bias=s["bias"], silu=case["silu"],
                                state=s["state"], carry=case["carry"])
        return {"out": s["out"], "state": s["state"]}
    if op == "conv_step":
        B.leapquant_conv_step(s["x"], s["weight"], s["out"], s["state"], bias=s["bias"], silu=case["silu"])
        return {"out": s["out"], "state": s["state"]}
    if op == "qk_norm":
        B.leapquant_qk_norm(s["q"], s["k"], s["q_out"], s["k_out"],
                            norm=B.LQ_NORM_RMS if case["norm"] == "rms" else B.LQ_NORM_L2, eps=1e-6,
                            q_weight=s["q_weight"], k_weight=s["k_weight"], q_scale=D ** -0.5, cos=s["cos"], sin=s["sin"],
                            positions=s["positions"], interleaved=case["interleaved"])
        return {"q": s["q_out"], "k": s["k_out"]}
    dims = B.make_dims(case["seqs"], case["heads_v"], case["heads_k"], rule=B.LQ_RULE_ADD)
    if op == "scan_prompt":
        B.leapquant_scan_prompt(dims, s["q"], s["k"], s["v"], s["dt"], s["A"], s["out"], s["cu"], D=s["D"],
                                dt_bias=s["dt_bias"], state=s["state"], carry=case["carry"], max_len=max(s["lens"]))
    else:
        B.leapquant_scan_step(dims, s["state"], s["q"], s["k"], s["v"], s["dt"], s["A"], s["out"], D=s["D"],
                              dt_bias=s["dt_bias"])
    return {"out": s["out"], "state": s["state"]}


# --------------------------------------------------------------------------------------------------- the plain forms

def _sequence_of(cu, n):
    """Of every packed token its sequence and its place in it."""
    t = torch.arange(n, device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return seq, t - cu[seq]


def _plain_conv(s):
    case, x, w = s["case"], s["x"].float(), s["weight"]
    k, n, c = case["width"], case["tokens"], case["channels"]
    old = s["state"].float() if case["carry"] else torch.zeros_like(s["state"], dtype=torch.float32)
    if case["op"] == "conv_step":
        window = torch.cat([old, x[:, None]], 1)                                   # [B][K][C], oldest first
        new = window[:, 1:]
        y = (window * w.t()).sum(1)
    else:
        cu = s["cu"].long()
        seq, pos = _sequence_of(cu, n)
        i = torch.arange(k, device="cuda") - (k - 1)                               # offsets of the taps
        row = pos[:, None] + i                                                     # place in the sequence, < 0: the state
        both = torch.cat([x, old.reshape(-1, c)])
        at = torch.where(row >= 0, torch.arange(n, device="cuda")[:, None] + i, n + seq[:, None] * (k - 1) + row + k - 1)
        y = sum(both[at[:, j]] * w[:, j] for j in range(k))
        length = cu[1:] - cu[:-1]
        last = length[:, None] + torch.arange(k - 1, device="cuda") - (k - 1)
        b = torch.arange(case["seqs"], device="cuda")[:, None]
        at = torch.where(last >= 0, cu[:-1, None] + last, n + b * (k - 1) + last + k - 1)
        new = both[at]
    if s["bias"] is not None:
        y = y + s["bias"]
    if case["silu"]:
        y = _silu(y)
    s["state"].copy_(new)
    s["out"].copy_(y)
    return {"out": s["out"], "state": s["state"]}


def _plain_rotate(x, cos, sin, interleaved):
    r = 2 * cos.shape[-1]
    a, rest = x[..., :r], x[..., r:]
    a0, a1 = (a[..., 0::2], a[..., 1::2]) if interleaved else (a[..., :r // 2], a[..., r // 2:])
    cos, sin = cos[:, None], sin[:, None]
    b0, b1 = a0 * cos - a1 * sin, a1 * cos + a0 * sin
    both = torch.stack([b0, b1], -1).flatten(-2) if interleaved else torch.cat([b0, b1], -1)
    return torch.cat([both, rest], -1)


def _plain_norm(s):
    case = s["case"]
    for name in ("q", "k"):
        x = s[name].float()
        sq = (x * x).sum(-1, keepdim=True)
        x = x / torch.sqrt((sq / case["d"] if case["norm"] == "rms" else sq) + 1e-6)
        if s[name + "_weight"] is not None:
            x = x * s[name + "_weight"]
        if s["cos"] is not None:
            p = s["positions"].long()
            x = _plain_rotate(x, s["cos"][p], s["sin"][p], case["interleaved"])
        s[name + "_out"].copy_(x * D ** -0.5 if name == "q" else x)
    return {"q": s["q_out"], "k": s["k_out"]}


def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))


def _decays(x):
    """[..., n] steps' log decays -> [..., n, n]: from after step j to after step i, for i >= j, else 0."""
    n = x.shape[-1]
    low = torch.ones((n, n), dtype=torch.bool, device="cuda").tril(-1)
    total = torch.where(low, x[..., :, None].expand(*x.shape, n), torch.zeros((), device="cuda")).cumsum(-2)
    return torch.where(low | low.logical_not().tril(0), total.exp(), torch.zeros((), device="cuda"))


def _plain_scan_prompt(s):
    case = s["case"]
    b, n, hv, hk = case["seqs"], case["tokens"], case["heads_v"], case["heads_k"]
    c = -(-max(1, max(s["lens"])) // CHUNK)
    cu = s["cu"].long()
    pos = torch.arange(c * CHUNK, device="cuda")
    there = pos < (cu[1:] - cu[:-1])[:, None]                                      # [B][L]
    at = torch.where(there, cu[:-1, None] + pos, 0)

    def padded(x):                                                                 # [B][c][64][heads][...]
        x = x.float()[at] * there.view(b, -1, *[1] * (x.dim() - 1))
        return x.view(b, c, CHUNK, *x.shape[2:])

    def heads(x):                                                                  # [B][c][Hv][64][d]
        x = padded(x).transpose(2, 3)
        return x.repeat_interleave(hv // hk, dim=2) if x.shape[2] != hv else x

    step = _softplus(s["dt"].float() + s["dt_bias"])
    log_a = padded(step * s["A"]).transpose(2, 3)                                  # [B][c][Hv][64]
    step = padded(step).transpose(2, 3)
    q, k, v = heads(s["q"]), heads(s["k"]), heads(s["v"])
    within = _decays(log_a)
    y = (q @ k.transpose(-1, -2) * within * step[..., None, :]) @ v
    part = (k * (within[..., -1, :] * step)[..., None]).transpose(-1, -2) @ v      # [B][c][Hv][d_k][d_v]
    old = s["state"].float().transpose(-1, -2) if case["carry"] else torch.zeros_like(part[:, 0])
    parts = torch.cat([old[:, None], part], 1).transpose(1, 2).reshape(b, hv, c + 1, D * D)
    across = _decays(torch.nn.functional.pad(log_a.sum(-1).transpose(1, 2), (1, 0)))
    states = (across @ parts).view(b, hv, c + 1, D, D)
    y = y + (q * log_a.cumsum(-1).exp()[..., None]) @ states[:, :, :-1].transpose(1, 2)
    y = y.transpose(2, 3).reshape(b * c * CHUNK, hv, D)[there.view(-1)]
    if s["D"] is not None:
        y = y + s["D"][:, None] * s["v"].float()
    s["state"].copy_(states[:, :, -1].transpose(-1, -2))
    s["out"].copy_(y)
    return {"out": s["out"], "state": s["state"]}


def _plain_scan_step(s):
    case = s["case"]
    q, k = (s[x].float().repeat_interleave(case["heads_v"] // case["heads_k"], dim=1) for x in ("q", "k"))
    v = s["v"].float()
    step = _softplus(s["dt"].float() + s["dt_bias"])
    a = (step * s["A"]).exp()
    new = a[..., None, None] * s["state"].float() + v[..., :, None] * (step[..., None] * k)[..., None, :]
    s["state"].copy_(new)
    y = (s["state"].float() * q[..., None, :]).sum(-1)
    if s["D"] is not None:
        y = y + s["D"][:, None] * v
    s["out"].copy_(y)
    return {"out": s["out"], "state": s["state"]}


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    return {"conv_prompt": _plain_conv, "conv_step": _plain_conv, "qk_norm": _plain_norm,
            "scan_prompt": _plain_scan_prompt, "scan_step": _plain_scan_step}[op](s)


def work(case):
    n, es, op = case["tokens"], SIZE[case["dtype"]], case["op"]
    if op in ("conv_prompt", "conv_step"):
        c, k = case["channels"], case["width"]
        state = case["seqs"] * (k - 1) * c * es
        return {"bytes": n * c * (es + SIZE[case["out"]]) + state * (2 if case["carry"] else 1)
                + 4 * c * (k + (1 if case["bias"] else 0)), "flops": n * c * (2 * k + (4 if case["silu"] else 0))}
    if op == "qk_norm":
        e = n * (case["heads_q"] + case["heads_k"]) * case["d"]
        return {"bytes": e * (es + SIZE[case["out"]]) + n * 4 * case["rot"], "flops": 6 * e}
    hv, hk = case["heads_v"], case["heads_k"]
    token = n * (2 * hv * D + 2 * hk * D + hv) * es
    state = case["seqs"] * hv * D * D * SIZE[case["state"]]
    return {"bytes": token + state * (2 if case["carry"] else 1), "flops": n * hv * 4 * D * D}


# ------------------------------------------------------------------------------------- the same results in 64 bits

def _exact_conv(case, s):
    x, w, old = s["x"].double(), s["weight"].double(), s["state"].double()
    k, c = case["width"], case["channels"]
    if not case["carry"]:
        old = torch.zeros_like(old)
    lens = s["lens"] if case["op"] == "conv_prompt" else [1] * case["seqs"]
    out, new, at = [], [], 0
    for b, n in enumerate(lens):
        line = torch.cat([old[b], x[at:at + n]])
        at += n
        y = torch.zeros((n, c), dtype=torch.float64, device="cuda")
        if s["bias"] is not None:
            y += s["bias"].double()
        for j in range(k):
            y += line[j:j + n] * w[:, j]
        out.append(y * torch.sigmoid(y) if case["silu"] else y)
        new.append(line[n:])
    return {"out": torch.cat(out), "state": torch.stack(new)}


def _exact_norm(case, s):
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        size = x.square().mean(-1) if case["norm"] == "rms" else x.square().sum(-1)
        x = x * (size + 1e-6).rsqrt()[..., None]
        if s[name + "_weight"] is not None:
            x = x * s[name + "_weight"].double()
        if case["rot"]:
            r, p = case["rot"], s["positions"].long()
            turn = torch.complex(s["cos"][p].double(), s["sin"][p].double())[:, None]
            first, second = (range(0, r, 2), range(1, r, 2)) if case["interleaved"] else (range(r // 2), range(r // 2, r))
            z = torch.complex(x[..., list(first)], x[..., list(second)]) * turn
            x[..., list(first)], x[..., list(second)] = z.real, z.imag
        out[name] = x * D ** -0.5 if name == "q" else x
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("conv_prompt", "conv_step"):
        return _exact_conv(case, s)
    if case["op"] == "qk_norm":
        return _exact_norm(case, s)
    # the recurrence token by token, all sequences and heads side by side
    group = case["heads_v"] // case["heads_k"]
    q, k = (s[x].double().repeat_interleave(group, dim=1) for x in ("q", "k"))
    v = s["v"].double()
    raw = s["dt"].double() + s["dt_bias"].double()
    delta = torch.logaddexp(raw, torch.zeros_like(raw))
    alpha = torch.exp(delta * s["A"].double())
    k = k * delta[..., None]
    state = s["state"].double()
    if not case["carry"]:
        state = torch.zeros_like(state)
    lens = s["lens"] if case["op"] == "scan_prompt" else [1] * case["seqs"]
    start = [sum(lens[:i]) for i in range(len(lens))]
    out = torch.empty(v.shape, dtype=torch.float64, device="cuda")
    order = sorted(range(len(lens)), key=lambda i: -lens[i])                        # longest first
    state = state[order].contiguous()
    base = torch.tensor([start[i] for i in order], device="cuda")
    sizes = [lens[i] for i in order]
    m = len(sizes)
    for t in range(max(sizes)):
        while sizes[m - 1] <= t:
            m -= 1
        at = base[:m] + t
        live = state[:m]
        live *= alpha[at][..., None, None]
        live.addcmul_(v[at][..., :, None], k[at][..., None, :])
        if case["state"] == "bf16":
            # the step's output reads the state as it is stored
            out[at] = (live.float().bfloat16().double() * q[at][..., None, :]).sum(-1)
        else:
            out[at] = torch.matmul(live, q[at][..., None])[..., 0]
    if s["D"] is not None:
        out += s["D"].double()[:, None] * v
    new = torch.empty_like(state)
    new[order] = state
    return {"out": out, "state": new}
