"""4-bit blocks on the GPU against their definition in 64 bits: codes and scale bytes exactly, products within the error of binary32 sums."""
import numpy as np
import pytest
import torch

import layers_model as model
import paper_2502_18554_amd as zc
from paper_2502_18554_amd.binding import ZC_ERR_ARG, ZC_OK

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def room(rows, cols, more=0, fill=0xA5):
    """Codes and scale bytes for a matrix, with some more bytes to every row that the calls must leave alone."""
    return (torch.full((rows, zc.zc_mx_codes_stride(cols) + 16 * more), fill, dtype=torch.uint8, device=DEV),
            torch.full((rows, zc.zc_mx_scales_stride(cols) + 4 * more), fill, dtype=torch.uint8, device=DEV))


def matrix(rows, cols, seed, kind="f32", spread=3.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(spread * rng.standard_normal((rows, -(-cols // 7))).repeat(7, axis=1)[:, :cols])
    x[rng.random((rows, cols)) < 0.05] = 0
    if kind == "f16":
        x = np.clip(x, -60000, 60000)
    return torch.from_numpy(x.astype(np.float32)).to(TYPES[kind])


def quantize(x, along=True, down=True, more=0):
    rows, cols = x.shape
    held = room(rows, cols, more) if along else (None, None)
    held_t = room(cols, rows, more) if down else (None, None)
    assert zc.zc_mx_quantize(x, *held, *held_t) == ZC_OK
    return held, held_t


def check_held(held, x, cols):
    """Codes and scale bytes are the definition's; what lies behind a row's blocks is untouched."""
    codes, scales = (t.cpu().numpy() for t in held)
    blocks = -(-cols // 32)
    want_codes, want_scales = model.mx_quantize(x)
    assert np.array_equal(scales[:, :blocks], want_scales)
    assert np.array_equal(codes[:, :16 * blocks], want_codes)
    assert (codes[:, 16 * blocks:] == 0xA5).all() and (scales[:, blocks:] == 0xA5).all()


SHAPES = [(1, 1), (1, 31), (1, 32), (1, 33), (31, 1), (32, 32), (33, 65), (5, 1000), (1000, 5), (127, 129), (128, 128), (130, 260), (257, 511), (64, 4100), (2049, 96)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_blocks_are_the_definitions(shape, kind):
    x = matrix(*shape, seed=shape[0] * 7 + shape[1], kind=kind)
    held, held_t = quantize(x.to(DEV))
    ref = x.float().numpy()
    check_held(held, ref, shape[1])
    check_held(held_t, ref.T, shape[0])
    for along, down in ((True, False), (False, True)):                  # one of the two alone gives the same
        one, one_t = quantize(x.to(DEV), along, down)
        for a, b in zip(one + one_t, held + held_t):
            assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_that_lie_apart_and_start_anywhere(kind):
    base = matrix(70, 300, 5, kind).to(DEV)
    for x in (base[:, 1:200], base[3:, 7:40], base[::3, 5:], base[:1, 9:], base[:, 299:]):
        held, held_t = quantize(x, more=2)
        check_held(held, x.float().cpu().numpy(), x.shape[1])
        check_held(held_t, x.float().cpu().numpy().T, x.shape[0])


def test_rounding_of_every_code():
    """Ties, their neighbours, what lies above the largest code, signed zeros, tiny and subnormal and largest blocks."""
    grid = np.concatenate([model.E2M1, (model.E2M1[1:] + model.E2M1[:-1]) / 2, [6.5, 7, 7.99]]).astype(np.float32)
    grid = np.concatenate([grid, np.nextafter(grid, np.float32(0)), np.nextafter(grid, np.float32(8))])
    rows = []
    for exponent in (-149, -140, -128, -127, -126, -125, -124, -100, -20, -1, 0, 1, 20, 100, 124, 125):
        for sign in (1, -1):
            for at in range(0, grid.size, 28):
                part = np.zeros(32, np.float32)
                part[:grid[at:at + 28].size] = sign * np.ldexp(grid[at:at + 28], exponent)
                part[31] = np.ldexp(np.float32(4), exponent)
                part[30] = -0.0
                rows.append(part)
    x = np.stack(rows)
    assert np.isfinite(x).all()
    held, held_t = quantize(torch.from_numpy(x).to(DEV))
    check_held(held, x, 32)
    check_held(held_t, x.T, x.shape[0])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_a_value_that_is_not_finite_spoils_its_block_only(value, kind):
    x = matrix(40, 100, 3, kind)
    x[7, 40] = value
    x[39, 99] = value
    held, held_t = quantize(x.to(DEV))
    check_held(held, x.float().numpy(), 100)
    check_held(held_t, x.float().numpy().T, 40)
    back = torch.empty((40, 100), dtype=TYPES[kind], device=DEV)
    assert zc.zc_mx_dequantize(*held, back) == ZC_OK
    bad = torch.zeros((40, 100), dtype=torch.bool)
    bad[7, 32:64] = True
    bad[39, 96:] = True
    assert torch.equal(torch.isnan(back.cpu()), bad)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_dequantize(shape, kind):
    rows, cols = shape
    rng = np.random.default_rng(cols)
    codes, scales = room(rows, cols, 1)
    codes.copy_(torch.from_numpy(rng.integers(0, 256, codes.shape, dtype=np.uint8)))
    low, high = (118, 134) if kind == "f16" else (0, 253)
    scales.copy_(torch.from_numpy(rng.integers(low, high, scales.shape, dtype=np.uint8)))
    wide = torch.full((rows, cols + 3), 9.0, dtype=TYPES[kind], device=DEV)
    assert zc.zc_mx_dequantize(codes, scales, wide[:, 1:cols + 1]) == ZC_OK
    want = torch.from_numpy(model.mx_values(codes.cpu().numpy(), scales.cpu().numpy(), cols))
    assert torch.equal(wide[:, 1:cols + 1].cpu(), want.to(torch.float32).to(TYPES[kind]))
    assert (wide[:, 0] == 9).all() and (wide[:, cols + 1:] == 9).all()


def held_at_random(rows, cols, seed, low=120, high=134):
    rng = np.random.default_rng(seed)
    codes, scales = room(rows, cols, 0, 0)
    codes.copy_(torch.from_numpy(rng.integers(0, 256, codes.shape, dtype=np.uint8)))
    if cols % 32:
        at = torch.arange(codes.shape[1], device=DEV)
        codes &= (2 * at < cols).to(torch.uint8) * 15 | (2 * at + 1 < cols).to(torch.uint8) * 240
    scales.copy_(torch.from_numpy(rng.integers(low, high, scales.shape, dtype=np.uint8)))
    return codes, scales


def values(held, cols):
    return model.mx_values(held[0].cpu().numpy(), held[1].cpu().numpy(), cols)


def check_product(out, a, b, kind, bias=None, before=None):
    """Every sum of k products in binary32, in any order and cut off instead of rounded, is within (k + 2) 2^-23 of the sum of their magnitudes;
    the output's rounding comes on top."""
    want = a @ b.T
    size = np.abs(a) @ np.abs(b).T
    for more in (bias, before):
        if more is not None:
            want = want + more
            size = size + np.abs(more)
    tolerance = (a.shape[1] + 2) * 2.0 ** -23 * size
    tolerance = tolerance + model.half_ulp_of(kind, np.abs(want) + tolerance)
    out = out.double().cpu().numpy()
    if kind == "f16":                                        # (what is rounded to more than its largest value is infinite there)
        beyond = np.abs(want) + tolerance >= 65520
        assert (np.isinf(out) | (np.abs(want) - tolerance < 65520))[beyond].all() and (np.sign(out) == np.sign(want))[beyond].all()
        out, want = np.where(beyond & np.isinf(out), 0, out), np.where(beyond & np.isinf(out), 0, want)
    off = np.abs(out - want)
    assert (off <= tolerance).all(), (np.argwhere(off > tolerance)[:5], float((off - tolerance).max()))


PRODUCTS = [(1, 1, 1), (1, 5, 31), (1, 64, 32), (2, 16, 128), (3, 17, 129), (16, 16, 160), (17, 33, 1000), (1, 300, 4100), (8, 4096, 512), (33, 100, 2048),
            (64, 64, 64), (100, 257, 300), (128, 256, 256), (129, 255, 513), (256, 512, 1024), (300, 400, 96), (511, 130, 2085), (1000, 72, 40), (5, 7, 16500)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes", PRODUCTS, ids=str)
def test_product(sizes, kind):
    m, n, k = sizes
    a, b = held_at_random(m, k, 1), held_at_random(n, k, 2)
    ws = torch.full((zc.zc_mx_workspace_bytes(m, n, k) + 16,), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.full((m, n + 2), 7.0, dtype=TYPES[kind], device=DEV)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(4)).to(DEV) * 3
    va, vb = values(a, k), values(b, k)
    if kind == "f16":
        a[1].sub_(4)
        va = va / 16
    assert zc.zc_mx_product(*a, *b, k, out[:, :n], ws) == ZC_OK
    check_product(out[:, :n], va, vb, kind)
    assert (out[:, n:] == 7).all()
    before = out[:, :n].double().cpu().numpy()
    assert zc.zc_mx_product(*a, *b, k, out[:, :n], ws, d_bias=bias, add=True) == ZC_OK
    check_product(out[:, :n], va, vb, kind, bias.double().cpu().numpy(), before)
    assert (out[:, n:] == 7).all()
    again = torch.empty((m, n), dtype=TYPES[kind], device=DEV)
    ws.fill_(0)
    for _ in range(2):
        assert zc.zc_mx_product(*a, *b, k, again, ws, d_bias=bias) == ZC_OK
    first = again.clone()
    assert zc.zc_mx_product(*a, *b, k, again, ws, d_bias=bias) == ZC_OK and torch.equal(first, again)


@pytest.mark.parametrize("sizes", [(3, 20, 96), (200, 130, 700)], ids=str)
def test_product_of_operands_whose_rows_lie_apart(sizes):
    m, n, k = sizes
    a, b = held_at_random(m, k + 64, 1), held_at_random(n, k + 640, 2)
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    out = torch.empty((m, n), dtype=torch.float32, device=DEV)
    assert zc.zc_mx_product(*a, *b, k, out, ws) == ZC_OK
    va, vb = values(a, -(-k // 32) * 32), values(b, -(-k // 32) * 32)        # (whole blocks: what fills up the last one is the caller's)
    check_product(out, va, vb, "f32")


@pytest.mark.parametrize("m", [1, 20, 200])
def test_product_of_blocks_that_are_no_numbers(m):
    n, k = 150, 500
    a, b = held_at_random(m, k, 1), held_at_random(n, k, 2)
    b[1][3, 2] = 255
    b[1][149, 15] = 255
    a[1][m - 1, 7] = 255
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    out = torch.empty((m, n), dtype=torch.float32, device=DEV)
    assert zc.zc_mx_product(*a, *b, k, out, ws) == ZC_OK
    bad = torch.zeros((m, n), dtype=torch.bool)
    bad[:, [3, 149]] = True
    bad[m - 1] = True
    assert torch.equal(torch.isnan(out.cpu()), bad)


def test_what_lies_behind_the_last_block_is_not_read_into_the_sum():
    """Room behind a row's blocks that stands for no numbers, and operands at the very end of their memory."""
    for m, n, k in ((1, 40, 33), (5, 300, 161), (150, 300, 289)):
        a, b = held_at_random(m, k, 1), held_at_random(n, k, 2)
        blocks = -(-k // 32)
        a[1][:, blocks:] = 255
        b[1][:, blocks:] = 255
        ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
        out = torch.empty((m, n), dtype=torch.float32, device=DEV)
        assert zc.zc_mx_product(*a, *b, k, out, ws) == ZC_OK
        check_product(out, values(a, k), values(b, k), "f32")


@pytest.mark.parametrize("rows", [1, 4, 40])
def test_scales_from_end_to_end(rows):
    """Blocks of very large and very small values against each other: the products of the scales stay in binary32's range."""
    k, n = 128, 48
    a, b = held_at_random(rows, k, 1, 20, 30), held_at_random(n, k, 2, 225, 235)
    ws = torch.empty(zc.zc_mx_workspace_bytes(rows, n, k), dtype=torch.uint8, device=DEV)
    out = torch.empty((rows, n), dtype=torch.float32, device=DEV)
    assert zc.zc_mx_product(*a, *b, k, out, ws) == ZC_OK
    check_product(out, values(a, k), values(b, k), "f32")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes", PRODUCTS, ids=str)
def test_linear_is_the_product_of_its_quantised_input(sizes, kind):
    m, n, k = sizes
    x = matrix(m, k, 9, kind, spread=0.5).to(DEV)
    w = held_at_random(n, k, 2)
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    out = torch.empty((m, n), dtype=torch.float32, device=DEV)
    bias = torch.arange(n, dtype=torch.float32, device=DEV)
    assert zc.zc_mx_linear(x, *w, out, ws, d_bias=bias) == ZC_OK
    vx = model.mx_values(*model.mx_quantize(x.float().cpu().numpy()), k)
    check_product(out, vx, values(w, k), "f32", bias.double().cpu().numpy())
    before = out.double().cpu().numpy()
    assert zc.zc_mx_linear(x, *w, out, ws, add=True) == ZC_OK
    check_product(out, vx, values(w, k), "f32", None, before)


@pytest.mark.parametrize("m", [1, 3, 70])
def test_linear_on_rows_that_lie_apart_and_are_not_finite(m):
    k, n = 333, 90
    base = matrix(3 * m, k + 5, 9, "bf16", spread=0.5).to(DEV)
    x = base[::3, 3:k + 3]
    x[m - 1, 40] = float("inf")
    w = held_at_random(n, k, 2)
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    out = torch.empty((m, n), dtype=torch.float32, device=DEV)
    assert zc.zc_mx_linear(x, *w, out, ws) == ZC_OK
    assert torch.isnan(out[m - 1]).all()
    if m > 1:
        vx = model.mx_values(*model.mx_quantize(x[:m - 1].float().cpu().numpy()), k)
        check_product(out[:m - 1], vx, values(w, k), "f32")


@pytest.mark.parametrize("sizes", [(0, 5, 64), (5, 0, 64), (4, 6, 0)], ids=str)
def test_sizes_of_zero(sizes):
    m, n, k = sizes
    a, b = room(m, k, 1), room(n, k, 1)
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k) + 16, dtype=torch.uint8, device=DEV)
    out = torch.full((m, n), 3.0, device=DEV)
    bias = torch.arange(n, dtype=torch.float32, device=DEV)
    assert zc.zc_mx_product(*a, *b, k, out, ws, d_bias=bias, add=True) == ZC_OK
    assert torch.equal(out, (3.0 + bias).expand(m, n))
    assert zc.zc_mx_linear(torch.zeros((m, k), device=DEV), *b, out, ws, d_bias=bias) == ZC_OK
    assert torch.equal(out, bias.expand(m, n))
    assert zc.zc_mx_quantize(torch.zeros((m, k), device=DEV), *room(m, k, 1)) == ZC_OK
    assert zc.zc_mx_dequantize(*room(m, k, 1), torch.zeros((m, k), device=DEV)) == ZC_OK


def on_the_grid(rows, cols, rng):
    """Values that blocks hold exactly, along either axis."""
    return (rng.choice([-1.0, 1.0], (rows, cols)) * rng.choice(model.E2M1, (rows, cols))).astype(np.float32)


@pytest.mark.parametrize("sizes", [(5, 7, 9), (40, 33, 70), (130, 160, 290)], ids=str)
def test_gradients_of_a_layer(sizes):
    """dx = dy w and dw = dy^T x by the products of operands quantised along the other axis: against the formula, and against differences of
    the loss sum(dy * (x w^T)), with values that the blocks hold exactly."""
    m, n, k = sizes
    rng = np.random.default_rng(m)
    x, w, dy = on_the_grid(m, k, rng), on_the_grid(n, k, rng), on_the_grid(m, n, rng)
    x[m // 2, k // 2] = w[n // 2, k // 2] = 1.0                                 # where differences are taken: 0.5, 1 and 1.5 are codes
    dev = [torch.from_numpy(t).to(DEV) for t in (x, w, dy)]
    _, x_t = quantize(dev[0])
    _, w_t = quantize(dev[1])
    g, g_t = quantize(dev[2])
    ws = torch.empty(zc.zc_mx_workspace_bytes(max(m, n), max(n, k), max(m, n)), dtype=torch.uint8, device=DEV)
    dx, dw = torch.empty((m, k), device=DEV), torch.empty((n, k), device=DEV)
    assert zc.zc_mx_product(*g, *w_t, n, dx, ws) == ZC_OK
    assert zc.zc_mx_product(*g_t, *x_t, m, dw, ws) == ZC_OK
    check_product(dx, dy.astype(np.float64), w.T.astype(np.float64), "f32")
    check_product(dw, dy.T.astype(np.float64), x.T.astype(np.float64), "f32")

    def loss(x, w):
        out = torch.empty((m, n), device=DEV)
        held, _ = quantize(torch.from_numpy(w).to(DEV))
        assert zc.zc_mx_linear(torch.from_numpy(x).to(DEV), *held, out, ws_l) == ZC_OK
        return float((out.double().cpu().numpy() * dy).sum())

    ws_l = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    size = float((np.abs(dy) * (np.abs(x) @ np.abs(w).T)).sum()) * (k + 2) * 2.0 ** -23       # of the error of two losses
    for which, grad, i in ((0, dx, m // 2), (1, dw, n // 2)):
        up, down = [x.copy(), w.copy()], [x.copy(), w.copy()]
        up[which][i, k // 2] += 0.5
        down[which][i, k // 2] -= 0.5
        difference = loss(*up) - loss(*down)
        assert abs(difference - float(grad[i, k // 2])) <= 2 * size + 1e-5 * abs(difference)


def test_other_streams_and_graphs():
    m, n, k = 24, 512, 1024
    x, w = matrix(m, k, 1, "bf16", 0.5).to(DEV), held_at_random(n, k, 2)
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    out, want = torch.zeros((m, n), device=DEV), torch.zeros((m, n), device=DEV)
    assert zc.zc_mx_linear(x, *w, want, ws) == ZC_OK
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    assert zc.zc_mx_linear(x, *w, out, ws, stream=side) == ZC_OK
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert zc.zc_mx_linear(x, *w, out, ws) == ZC_OK
    for i in range(4):
        x.copy_(matrix(m, k, 10 + i, "bf16", 0.5))
        graph.replay()
        torch.cuda.synchronize()
        assert zc.zc_mx_linear(x, *w, want, ws) == ZC_OK
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_what_does_not_fit_together_is_refused():
    m, n, k = 8, 16, 64
    x, w, out = torch.zeros((m, k), device=DEV), room(n, k), torch.zeros((m, n), device=DEV)
    a = room(m, k)
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    refused = [
        lambda: zc.zc_mx_quantize(x, a[0][1:], a[1]), lambda: zc.zc_mx_quantize(x, a[0][:, :16], a[1]), lambda: zc.zc_mx_quantize(x, a[0], None),
        lambda: zc.zc_mx_quantize(x, None, None), lambda: zc.zc_mx_quantize(x.t(), *room(k, m)), lambda: zc.zc_mx_quantize(x.double(), *a),
        lambda: zc.zc_mx_quantize(x[0], *a), lambda: zc.zc_mx_quantize(x, *a, *a), lambda: zc.zc_mx_quantize(x, a[0].int(), a[1]),
        lambda: zc.zc_mx_dequantize(*a, torch.zeros((m, 96), device=DEV)), lambda: zc.zc_mx_dequantize(a[0], a[1][:, :1], x), lambda: zc.zc_mx_dequantize(*a, x.double()),
        lambda: zc.zc_mx_product(*a, *w, k + 64, out, ws), lambda: zc.zc_mx_product(*a, *w, k, out.t(), ws), lambda: zc.zc_mx_product(*a, *w, k, out[:4], ws),
        lambda: zc.zc_mx_product(*a, *w, k, out, ws, d_bias=out[0, :8]), lambda: zc.zc_mx_product(*a, *w, k, out, ws, d_bias=out[0].half()),
        lambda: zc.zc_mx_linear(x, *w, out, ws[:16]), lambda: zc.zc_mx_linear(x, *w, out, None), lambda: zc.zc_mx_linear(x[:4], *w, out, ws),
        lambda: zc.zc_mx_linear(x.int(), *w, out, ws), lambda: zc.zc_mx_linear(x, *w, out, ws[1:]),
        lambda: zc.zc_mx_product(a[0].view(-1)[8:8 + 7 * 32].view(7, 32), a[1][:7], *w, k, out[:7], ws),
    ]
    for i, call in enumerate(refused):
        assert call() == ZC_ERR_ARG, i
    torch.cuda.synchronize()
