"""The optimiser's step and the 4-bit blocks from their definitions, in numpy and in 64 bits: what the layer calls are compared with."""
import math

import numpy as np

BLOCK = 32
E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])


def exponent_field(x):
    """Of binary32 magnitudes (or of one that a 64-bit value lies at, truncated)."""
    x = np.asarray(x, np.float64)
    f = x.astype(np.float32)
    f = np.where((f > x) & np.isfinite(x), np.nextafter(f, np.float32(0)), f).astype(np.float32)
    return (f.view(np.uint32) >> 23).astype(np.int64)


# ---- 4-bit blocks

def mx_quantize(x):
    """[rows, cols] binary32 -> codes [rows, blocks * 16], scale bytes [rows, blocks]."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    b = np.zeros((rows, blocks * BLOCK), np.float32)
    b[:, :cols] = x
    b = b.reshape(rows, blocks, BLOCK)
    a = np.abs(b)
    fine = np.isfinite(a).all(axis=2)
    e = exponent_field(np.where(np.isfinite(a), a, 0).max(axis=2))
    s = np.where(fine, np.maximum(e - 2, 0), 255)
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.where(fine[:, :, None], a, 0).astype(np.float64) / np.exp2(np.where(fine, s, 127) - 127.0)[:, :, None]
    # to the nearest of the eight values; in a tie the one with the even code
    d = np.abs(y[..., None] - E2M1)
    best = d.min(axis=-1, keepdims=True)
    tied = d == best
    even = tied & (np.arange(8) % 2 == 0)
    code = np.where(even.any(axis=-1), even.argmax(axis=-1), tied.argmax(axis=-1))
    code = np.where(y >= 6, 7, code) | (np.signbit(b) * 8)
    code = np.where(fine[:, :, None], code, 0).reshape(rows, blocks * 16, 2)
    return (code[:, :, 0] | (code[:, :, 1] << 4)).astype(np.uint8), s.astype(np.uint8)


def mx_values(codes, scales, cols):
    codes, scales = np.asarray(codes), np.asarray(scales)
    at = np.arange(cols)
    c = (codes[:, at // 2] >> (4 * (at % 2)).astype(np.uint8)) & 15
    v = np.where(c >= 8, -1.0, 1.0) * E2M1[c & 7]
    s = scales[:, at // BLOCK].astype(np.float64)
    return np.where(s == 255, np.nan, v * np.exp2(s - 127))


# ---- states in 8 bits

def e4m3_values():
    c = np.arange(128)
    e, f = c >> 3, c & 7
    v = np.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * np.exp2(e - 7.0))
    v[127] = np.nan
    return np.concatenate([v, -v])


def scale_bytes(x):
    """Of blocks [b, 32]."""
    a = np.abs(x)
    fine = np.isfinite(a).all(axis=1)
    e = exponent_field(np.where(np.isfinite(a), a, 0).max(axis=1))
    return np.where(fine & (e < 255), np.maximum(e - 7, 0), 255)


def mix(z):
    z = np.asarray(z, np.uint64)
    low = np.uint64(0xFFFFFFFF)
    z = z ^ (z >> np.uint64(15))
    z = (z * np.uint64(0x6A09E667)) & low
    z = z ^ (z >> np.uint64(13))
    z = (z * np.uint64(0xBB67AE85)) & low
    return z ^ (z >> np.uint64(16))


def random_words(seed, step, places):
    key = mix(np.uint64(seed & 0xFFFFFFFF))
    key = mix((key + np.uint64(seed >> 32)) & np.uint64(0xFFFFFFFF))
    key = mix((key + np.uint64(step & 0xFFFFFFFF)) & np.uint64(0xFFFFFFFF))
    z = mix((np.asarray(places, np.uint64) * np.uint64(0x9E3779B1) + key) & np.uint64(0xFFFFFFFF))
    return (z & np.uint64(0xFFFF)).astype(np.float64) / 65536, (z >> np.uint64(16)).astype(np.float64) / 65536


class State:
    """A state's parts as numpy arrays, cut out of its bytes."""

    def __init__(self, data, counts, bits):
        self.blocks = sum(-(-n // BLOCK) for n in counts)
        self.first = np.cumsum([0] + [-(-n // BLOCK) * BLOCK for n in counts])
        values, data = self.blocks * BLOCK, np.asarray(data, np.uint8)
        if bits == 32:
            self.m, self.v = (data[i * 4 * values:(i + 1) * 4 * values].view(np.float32).astype(np.float64) for i in range(2))
            return
        pad = -(-self.blocks // 16) * 16
        self.codes = [data[:values], data[values:2 * values]]
        self.scales = [data[2 * values:2 * values + self.blocks], data[2 * values + pad:2 * values + pad + self.blocks]]
        self.padding = [data[2 * values + self.blocks:2 * values + pad], data[2 * values + pad + self.blocks:2 * values + 2 * pad]]
        decoded = []
        for c, s in zip(self.codes, self.scales):
            size = np.where(s == 255, np.nan, np.exp2(s.astype(np.float64) - 127))
            decoded.append(e4m3_values()[c] * np.repeat(size, BLOCK))
        self.m, self.v = decoded[0], decoded[1] ** 2


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, decay):
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    with np.errstate(invalid="ignore", divide="ignore"):
        hat = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p - lr * decay * p - lr * hat, m, v


def grid_neighbours(x, scale):
    """The two neighbours of |x| / 2^(scale - 127) on e4m3's grid, and how far it is from the lower one to the upper one (0 .. 1)."""
    y = np.abs(x) / np.exp2(scale.astype(np.float64) - 127)
    with np.errstate(divide="ignore"):
        e = np.maximum(np.floor(np.log2(np.where(y > 0, y, 2.0 ** -40))), -6)
    q = np.exp2(e - 3)
    k = np.floor(y / q)
    return k * q, (k + 1) * q, y / q - k


def ulp(x, bits):
    """Spacing of binary floats with `bits` fraction bits at x."""
    x = np.abs(np.asarray(x, np.float64))
    return np.exp2(np.floor(np.log2(np.maximum(x, 2.0 ** -126))) - bits)


def half_ulp_of(name, x):
    bits, least = {"f32": (23, -149), "bf16": (7, -133), "f16": (10, -24)}[name]
    return 0.5 * np.maximum(ulp(x, bits), math.ldexp(1, least))
