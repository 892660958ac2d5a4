"""4-bit blocks on the GPU at sizes that fill it: every size of tile, workgroups that take several tiles, rows that lie far apart, offsets beyond 32 bits."""
import pytest
import torch

import paper_2502_18554_amd as zc
from paper_2502_18554_amd.binding import ZC_OK

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}           # of a value, at most
E2M1 = (0, .5, 1, 1.5, 2, 3, 4, 6)


def held_at_random(rows, cols, seed, more=0):
    """Blocks of values from 2^-6 to 1.5, and of zeros behind a row's last value."""
    gen = torch.Generator(DEV).manual_seed(seed)
    codes = torch.randint(0, 256, (rows, zc.zc_mx_codes_stride(cols) + 16 * more), dtype=torch.uint8, device=DEV, generator=gen)
    scales = torch.randint(122, 126, (rows, zc.zc_mx_scales_stride(cols) + 4 * more), dtype=torch.uint8, device=DEV, generator=gen)
    at = torch.arange(codes.shape[1], device=DEV)
    codes &= (2 * at < cols).to(torch.uint8) * 15 | (2 * at + 1 < cols).to(torch.uint8) * 240
    return codes, scales


def values(held, cols):
    """In binary64, from the definition."""
    codes, scales = held
    grid = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float64, device=DEV)
    at = torch.arange(cols, device=DEV)
    c = codes[:, at // 2] >> (4 * (at % 2)).to(torch.uint8) & 15
    return grid[c.int()] * torch.exp2(scales[:, at // 32].double() - 127)


def check(out, a, b, kind, bias=None, before=None):
    """As sums of k products in binary32 in any order, cut off instead of rounded: within (k + 2) 2^-23 of the sum of their magnitudes, and the output's rounding."""
    want, size = a @ b.T, a.abs() @ b.abs().T
    for more in (bias, before):
        if more is not None:
            want = want + more.double()
            size = size + more.double().abs()
    tolerance = (a.shape[1] + 2) * 2.0 ** -23 * size
    tolerance = tolerance + (want.abs() + tolerance) * HALF_ULP[kind] + 2.0 ** -25
    assert bool(((out.double() - want).abs() <= tolerance).all())


# tiles of 256 rows once and twice a workgroup, whole ones; of 128 once and twice; of 64 three times; k that ends inside a block, a step and a stage
FILLING = [(4200, 3800, 4165), (8150, 4090, 4165), (4096, 4096, 2048), (2000, 2000, 1000), (3000, 3500, 1001), (3000, 3500, 300), (2048, 2048, 512)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes", FILLING, ids=str)
def test_product(sizes, kind):
    m, n, k = sizes
    a, b = held_at_random(m, k, 1), held_at_random(n, k, 2)
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    wide = torch.full((m, n + 4), 7.0, dtype=TYPES[kind], device=DEV)
    out = wide[:, 1:n + 1] if m % 2 else wide[:, :n]
    bias = torch.randn(n, generator=torch.Generator(DEV).manual_seed(4), device=DEV)
    va, vb = values(a, k), values(b, k)
    assert zc.zc_mx_product(*a, *b, k, out, ws) == ZC_OK
    check(out, va, vb, kind)
    before = out.clone()
    assert zc.zc_mx_product(*a, *b, k, out, ws, d_bias=bias, add=True) == ZC_OK
    check(out, va, vb, kind, bias, before)
    assert bool((wide[:, n + 1:] == 7).all()) and bool((wide[:, 0] == 7).all() if out.storage_offset() else (wide[:, n] == 7).all())
    first, again = (torch.empty((m, n), dtype=TYPES[kind], device=DEV) for _ in range(2))
    for to in (first, again):
        assert zc.zc_mx_product(*a, *b, k, to, ws, d_bias=bias) == ZC_OK
    check(first, va, vb, kind, bias)
    assert torch.equal(first, again)


@pytest.mark.parametrize("m", [1, 20, 40, 200])
def test_operands_whose_rows_lie_far_apart(m):
    """Rows of b further apart than a buffer of a tile's rows can address; of the output, further than 32 bits."""
    n, k, apart = 150, 700, (1 << 23) + 64
    a, b = held_at_random(m, k, 1), held_at_random(n, k, 2)
    far = [torch.empty(n * apart, dtype=torch.uint8, device=DEV).view(n, apart)[:, :t.shape[1]] for t in b]
    for to, t in zip(far, b):
        to.copy_(t)
    out_apart = (1 << 32) // m
    out = torch.empty(m * out_apart, dtype=torch.bfloat16, device=DEV).view(m, out_apart)[:, :n]
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    for right in (b, far):
        out.fill_(5)
        assert zc.zc_mx_product(*a, *right, k, out, ws) == ZC_OK
        check(out, values(a, k), values(b, k), "bf16")
    out32 = torch.empty((n, m), dtype=torch.float32, device=DEV)
    assert zc.zc_mx_product(*far, *a, k, out32, ws) == ZC_OK
    check(out32, values(b, k), values(a, k), "f32")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_values_whose_rows_lie_far_apart(kind):
    rows, cols, n = 3, 1000, 70
    apart = (1 << 31) + 24 if kind == "bf16" else (1 << 30) + 24
    x = torch.empty((rows - 1) * apart + cols, dtype=TYPES[kind], device=DEV).as_strided((rows, cols), (apart, 1))
    x.copy_(torch.randn((rows, cols), generator=torch.Generator(DEV).manual_seed(1), device=DEV))
    near = x.contiguous()

    def room(r, c):
        return torch.zeros((r, zc.zc_mx_codes_stride(c)), dtype=torch.uint8, device=DEV), torch.zeros((r, zc.zc_mx_scales_stride(c)), dtype=torch.uint8, device=DEV)

    got, want = room(rows, cols) + room(cols, rows), room(rows, cols) + room(cols, rows)
    assert zc.zc_mx_quantize(x, *got) == ZC_OK and zc.zc_mx_quantize(near, *want) == ZC_OK
    for g, w in zip(got, want):
        assert torch.equal(g, w)
    w = held_at_random(n, cols, 2)
    ws = torch.empty(zc.zc_mx_workspace_bytes(rows, n, cols), dtype=torch.uint8, device=DEV)
    outs = [torch.empty((rows, n), device=DEV) for _ in range(2)]
    for to, values_of in zip(outs, (x, near)):
        assert zc.zc_mx_linear(values_of, *w, to, ws) == ZC_OK
        check(to, values(want[:2], cols), values(w, cols), "f32")
    assert zc.zc_mx_dequantize(*want[:2], x) == ZC_OK
    assert torch.equal(x.double(), values(want[:2], cols))


@pytest.mark.parametrize("m", [1, 2, 8, 9, 16, 17, 32, 33])
@pytest.mark.parametrize("n", [100, 8200, 16500])
def test_few_rows(m, n):
    """On either side of each border between the kernels for few rows: as values and as held."""
    k = 4096 if m % 2 else 2100
    x = torch.randn((m, k), generator=torch.Generator(DEV).manual_seed(m), device=DEV).to(torch.bfloat16)
    a = torch.zeros((m, zc.zc_mx_codes_stride(k)), dtype=torch.uint8, device=DEV), torch.zeros((m, zc.zc_mx_scales_stride(k)), dtype=torch.uint8, device=DEV)
    assert zc.zc_mx_quantize(x, *a) == ZC_OK
    b = held_at_random(n, k, 2)
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    out, other = torch.empty((m, n), device=DEV), torch.empty((m, n), device=DEV)
    assert zc.zc_mx_product(*a, *b, k, out, ws) == ZC_OK
    assert zc.zc_mx_linear(x, *b, other, ws) == ZC_OK
    va, vb = values(a, k), values(b, k)
    check(out, va, vb, "f32")
    check(other, va, vb, "f32")


def test_more_columns_than_a_launch_takes():
    k, n = 20, (1 << 28) + 77
    x = torch.randn((1, k), generator=torch.Generator(DEV).manual_seed(1), device=DEV)
    a = torch.zeros((1, 16), dtype=torch.uint8, device=DEV), torch.zeros((1, 4), dtype=torch.uint8, device=DEV)
    assert zc.zc_mx_quantize(x, *a) == ZC_OK
    b = held_at_random(n, k, 2)
    bias = torch.randn(n, generator=torch.Generator(DEV).manual_seed(4), device=DEV)
    ws = torch.empty(zc.zc_mx_workspace_bytes(1, n, k), dtype=torch.uint8, device=DEV)
    out = torch.empty((1, n), device=DEV)
    parts = [slice(0, 300), slice((1 << 28) - 150, (1 << 28) + 77), slice(123456789, 123457000)]
    for call in (lambda: zc.zc_mx_product(*a, *b, k, out, ws, d_bias=bias), lambda: zc.zc_mx_linear(x, *b, out, ws, d_bias=bias)):
        out.fill_(float("nan"))
        assert call() == ZC_OK
        assert not bool(torch.isnan(out).any())
        for part in parts:
            check(out[:, part], values(a, k), values([t[part] for t in b], k), "f32", bias[part])
