"""The projection operators in 64 bits from their definitions, on the CPU (test infrastructure).  Codes are not rounded here:
what a code is compared with is the value that it rounds."""
import torch

LEAST = 2.0 ** -100


def blocks(n):
    return -(-n // 128)


def add_norm(x, residual=None, weight=None, norm=True, eps=1e-6):
    """h and y, [tokens][channels]."""
    h = x.double().cpu()
    if residual is not None:
        h = h + residual.double().cpu()
    y = h
    if norm:
        y = h / torch.sqrt((h * h).sum(-1, keepdim=True) / h.shape[-1] + eps)
        if weight is not None:
            y = y * weight.double().cpu()
    return h, y


def gate_norm(x, gate, weight=None, act="silu", first=False, eps=1e-6):
    x, z = x.double().cpu(), gate.double().cpu()
    a = 1 / (1 + torch.exp(-z))
    if act == "silu":
        a = z * a
    if first:
        x = x * a
    y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + eps)
    if weight is not None:
        y = y * weight.double().cpu()
    return y if first else y * a


def row_scales(y):
    """[rows][channels] -> scales [rows][blocks]."""
    return torch.stack([part.abs().amax(1).clamp(min=LEAST) / 448 for part in y.split(128, 1)], 1)


def weight_scales(w):
    w = w.double().cpu()
    return torch.stack([torch.stack([b.abs().max().clamp(min=LEAST) / 448 for b in row.split(128, 1)]) for row in w.split(128, 0)])


def spread_rows(scale, channels):
    return scale.repeat_interleave(128, 1)[:, :channels]


def spread_weight(scale, n, k):
    return scale.repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]


def matmul(x, x_scale, w, w_scale, bias=None):
    """Products, and the sum of the terms' magnitudes (what rounding errors are measured against)."""
    (t, k), n = x.shape, w.shape[0]
    a = x.cpu().float().double() * spread_rows(x_scale.double().cpu(), k)
    b = w.cpu().float().double() * spread_weight(w_scale.double().cpu(), n, k)
    y, size = a @ b.t(), a.abs() @ b.abs().t()
    if bias is not None:
        y, size = y + bias.double().cpu(), size + bias.double().cpu().abs()
    return y, size
