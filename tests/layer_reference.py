"""The layer operators in 64 bits, token by token from their definitions, on the CPU (test infrastructure)."""
import torch


def lengths(cu, tokens):
    return [(int(cu[b]), int(cu[b + 1])) for b in range(len(cu) - 1)]


def conv(x, weight, spans, bias=None, silu=True, state=None):
    """Outputs [tokens][channels] (NaN where a token belongs to no sequence), the sum of the terms' magnitudes, and the
    new states; state [sequences][width-1][channels] or None (zeros)."""
    x, w = x.double().cpu(), weight.double().cpu()
    k, c = w.shape[1], x.shape[1]
    out = torch.full(x.shape, float("nan"), dtype=torch.float64)
    size = torch.zeros_like(out)
    new = torch.zeros((len(spans), k - 1, c), dtype=torch.float64)
    for b, (lo, hi) in enumerate(spans):
        old = torch.zeros((k - 1, c), dtype=torch.float64) if state is None else state[b].double().cpu()
        line = torch.cat([old, x[lo:hi]])
        for t in range(hi - lo):
            terms = line[t:t + k] * w.t()
            y = terms.sum(0)
            m = terms.abs().sum(0)
            if bias is not None:
                y, m = y + bias.double().cpu(), m + bias.double().cpu().abs()
            out[lo + t] = y / (1 + torch.exp(-y)) if silu else y
            size[lo + t] = m
        new[b] = line[hi - lo:]
    return out, size, new


def qk_norm(x, norm, eps, weight=None, scale=1.0, cos=None, sin=None, positions=None, interleaved=False):
    """One of q, k [tokens][heads][d]; norm "none", "l2" or "rms"."""
    x = x.double().cpu()
    if norm != "none":
        ss = (x * x).sum(-1, keepdim=True)
        x = x / torch.sqrt((ss / x.shape[-1] if norm == "rms" else ss) + eps)
        if weight is not None:
            x = x * weight.double().cpu()
    if cos is not None:
        out = x.clone()
        half = cos.shape[1]
        for t in range(x.shape[0]):
            p = int(positions[t])
            for j in range(half):
                i0, i1 = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
                if 0 <= p < cos.shape[0]:
                    c, s = float(cos[p, j]), float(sin[p, j])
                    out[t, :, i0] = x[t, :, i0] * c - x[t, :, i1] * s
                    out[t, :, i1] = x[t, :, i1] * c + x[t, :, i0] * s
                else:
                    out[t, :, i0] = out[t, :, i1] = float("nan")
        x = out
    return x * scale


def scan(q, k, v, dt, A, spans, D=None, dt_bias=None, softplus=True, state=None, state_bf16=False):
    """The recurrence: outputs (NaN where a token belongs to no sequence), final states S^T, and the same with every term's
    magnitude in place of the term (what rounding errors are measured against)."""
    q, k, v, dt, A = (x.double().cpu() for x in (q, k, v, dt, A))
    hv, group = v.shape[1], v.shape[1] // k.shape[1]
    q, k = q.repeat_interleave(group, 1), k.repeat_interleave(group, 1)
    raw = dt + (dt_bias.double().cpu() if dt_bias is not None else 0.0)
    delta = torch.clamp(raw, min=0) + torch.log1p(torch.exp(-raw.abs())) if softplus else raw
    alpha = torch.exp(delta * A)
    skip = D.double().cpu() if D is not None else torch.zeros(hv, dtype=torch.float64)
    o = torch.full(v.shape, float("nan"), dtype=torch.float64)
    osize = torch.zeros_like(o)
    new, size = [], []
    for b, (lo, hi) in enumerate(spans):
        S = torch.zeros((hv, v.shape[2], k.shape[2]), dtype=torch.float64) if state is None else state[b].double().cpu().clone()
        M = S.abs()
        new_b = S
        for t in range(lo, hi):
            kt = delta[t][:, None] * k[t]
            S = alpha[t][:, None, None] * S + v[t][:, :, None] * kt[:, None, :]
            M = alpha[t][:, None, None] * M + v[t].abs()[:, :, None] * kt.abs()[:, None, :]
            read = S.float().bfloat16().double() if state_bf16 else S
            o[t] = (read * q[t][:, None, :]).sum(-1) + skip[:, None] * v[t]
            osize[t] = (M * q[t].abs()[:, None, :]).sum(-1) + (skip[:, None] * v[t]).abs()
            new_b = S                                     # (a bf16 state: the value before its rounding)
            if state_bf16:
                S = read
        new.append(new_b)
        size.append(M)
    return o, osize, torch.stack(new), torch.stack(size)
