"""Layer norm, embedding and the step for matrices from their definitions, in 64 bits: what the calls are compared with."""
import numpy as np
import torch

U = 2.0 ** -24                               # half a step of binary32 relative to the value
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}


def half_step(kind, x):
    """How far one rounding may take x."""
    return np.maximum(HALF[kind] * np.abs(x), LEAST[kind])


# ---- layer norm

def norm(x, w, b, eps):
    """-> out, mean, d, and what one unit of U may change out by: a row's sums are at most 64 additions deep, and the mean is off by at most that of the mean magnitude."""
    mean = x.mean(axis=1, keepdims=True)
    d = 1 / np.sqrt(((x - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    z = (x - mean) * d
    unit = np.abs(w) * (d * (np.abs(x).mean(axis=1, keepdims=True) + np.abs(x - mean)) + np.abs(z)) + np.abs(b)
    return z * w + b, mean[:, 0], d[:, 0], unit


def norm_backward(dy, x, mean, d, w):
    """From given means and d's: dx, dw, db, and what one unit of U may change each by."""
    z = (x - mean[:, None]) * d[:, None]
    h = dy * w
    one, two = h.mean(axis=1, keepdims=True), (h * z).mean(axis=1, keepdims=True)
    dx = d[:, None] * (h - one - z * two)
    unit = d[:, None] * (np.abs(h) + np.abs(h).mean(axis=1, keepdims=True) + np.abs(z) * np.abs(h * z).mean(axis=1, keepdims=True))
    return dx, (dy * z).sum(axis=0), dy.sum(axis=0), unit, np.abs(dy * z).sum(axis=0), np.abs(dy).sum(axis=0)


# ---- embedding

def embedding_backward(dy, tokens, rows, scale):
    """The gradient, the sums of magnitudes that go into it, and how many tokens each row has."""
    grad, size, count = np.zeros((rows, dy.shape[1])), np.zeros((rows, dy.shape[1])), np.zeros(rows, np.int64)
    for i, t in enumerate(tokens):
        if 0 <= t < rows:
            grad[t] += scale * dy[i]
            size[t] += abs(scale) * np.abs(dy[i])
            count[t] += 1
    return grad, size, count


# ---- the step for matrices

A, B, C = 3.4445, -4.7750, 2.0315
SCALE = 4096.0


def rounded(x, parts):
    """To one binary16 number, or to the sum of two, at the scale that the kernels keep."""
    if parts == 0:
        return x
    y = x * SCALE
    high = y.half().double()
    return (high if parts == 1 else high + (y - high).half().double()) / SCALE


def orthogonalised(u, iterations, parts, device="cpu"):
    """X after so many iterations; parts 0: nothing rounded, 1 and 2: operands rounded to one and two binary16 numbers, as the kernels round them."""
    turned = u.shape[0] > u.shape[1]
    x = torch.from_numpy(np.ascontiguousarray(u.T if turned else u)).double().to(device)
    x = rounded(x / max(float(x.square().sum().sqrt()), 1e-7), parts)
    for i in range(iterations):
        a = rounded(x @ x.t().contiguous(), parts)
        b = rounded(A * torch.eye(len(a), dtype=a.dtype, device=device) + B * a + C * (a @ a), parts)
        x = b @ x
        if i + 1 < iterations:
            x = rounded(x, parts)
    return (x.t() if turned else x).cpu().numpy()


def muon(p, g, m, lr, momentum, decay, iterations, nesterov, match_rms=False, parts=0):
    m = momentum * m + (1 - momentum) * g
    u = momentum * m + (1 - momentum) * g if nesterov else m
    rows, cols = p.shape
    factor = 0.2 * np.sqrt(max(rows, cols)) if match_rms else np.sqrt(max(1, rows / cols))
    return p * (1 - lr * decay) - lr * factor * orthogonalised(u, iterations, parts), m
