"""4-bit blocks of long thin matrices: more tiles than a grid counts, on each side of that border."""
import numpy as np
import pytest
import torch

import layers_model as model
import paper_2502_18554_amd as zc
from paper_2502_18554_amd.binding import ZC_ERR_ARG, ZC_OK

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
MOST = (1 << 24) - 1                 # workgroups of 256 threads that a grid counts


@pytest.fixture(autouse=True)
def room_for_others():
    yield
    torch.cuda.empty_cache()


def room(rows, cols):
    return (torch.full((rows, zc.zc_mx_codes_stride(cols)), 0xA5, dtype=torch.uint8, device=DEV),
            torch.full((rows, zc.zc_mx_scales_stride(cols)), 0xA5, dtype=torch.uint8, device=DEV))


def places(n, around):
    """Of n rows: the ends, those around some, and others at random."""
    rng = np.random.default_rng(n & 0xFFFF)
    near = [i + j for i in (0, n, *around) for j in range(-70, 70)]
    return torch.from_numpy(np.unique(np.concatenate([[i for i in near if 0 <= i < n], rng.integers(0, n, 2000)]))).to(DEV)


def check_rows(held, values, at):
    """Rows of blocks against the definition; values: a function of the rows' numbers."""
    codes, scales = model.mx_quantize(values(at).float().cpu().numpy())
    assert np.array_equal(held[0][at].cpu().numpy()[:, :codes.shape[1]], codes)
    assert np.array_equal(held[1][at].cpu().numpy()[:, :scales.shape[1]], scales)
    assert (held[1][:, scales.shape[1]:] == 0xA5).all()


@pytest.mark.parametrize("more", [0, 1, 67])
def test_blocks_down_the_columns_of_a_long_row(more):
    cols = MOST * 64 + more                                        # a tile has 64 columns of 32 bits
    x = torch.randn((1, cols), generator=torch.Generator(DEV).manual_seed(1), device=DEV)
    held_t = room(cols, 1)
    assert zc.zc_mx_quantize(x, None, None, *held_t) == ZC_OK
    check_rows(held_t, lambda at: x[0, at][:, None], places(cols, [MOST * 64]))


@pytest.mark.parametrize("more", [0, 1, 67])
def test_blocks_along_the_rows_of_a_long_column(more):
    rows = MOST * 32 + more                                        # a tile has 32 rows
    x = torch.randn((rows, 1), generator=torch.Generator(DEV).manual_seed(2), device=DEV, dtype=torch.bfloat16)
    held = room(rows, 1)
    assert zc.zc_mx_quantize(x, *held) == ZC_OK
    check_rows(held, lambda at: x[at], places(rows, [MOST * 32]))


def test_blocks_along_both_axes_of_a_long_column():
    rows, cols = MOST * 128 + 100, 1                               # a tile has 128 rows
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
    for i, part in enumerate(x.split(1 << 28)):
        part.copy_(torch.randn(part.shape, generator=torch.Generator(DEV).manual_seed(10 + i), device=DEV))
    held, held_t = room(rows, cols), room(cols, rows)
    assert zc.zc_mx_quantize(x, *held, *held_t) == ZC_OK
    border = MOST * 128
    check_rows(held, lambda at: x[at], places(rows, [border]))
    for first, last in ((0, 256), (border - 256, rows)):           # (from whole blocks on)
        codes, scales = model.mx_quantize(x[first:last].float().cpu().numpy().T)
        assert np.array_equal(held_t[0][:, first // 2:(first + 32 * scales.shape[1]) // 2].cpu().numpy(), codes)
        assert np.array_equal(held_t[1][:, first // 32:first // 32 + scales.shape[1]].cpu().numpy(), scales)


def test_a_layer_on_as_many_rows():
    m = MOST * 32 + 1001
    x = torch.randn((m, 1), generator=torch.Generator(DEV).manual_seed(4), device=DEV, dtype=torch.bfloat16)
    w = room(1, 1)
    assert zc.zc_mx_quantize(torch.full((1, 1), 3.0, device=DEV), *w) == ZC_OK
    out = torch.empty((m, 1), device=DEV)
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, 1, 1), dtype=torch.uint8, device=DEV)
    assert zc.zc_mx_linear(x, *w, out, ws) == ZC_OK
    at = places(m, [MOST * 32])
    want = 3 * model.mx_values(*model.mx_quantize(x[at].float().cpu().numpy()), 1)
    assert np.array_equal(out[at].double().cpu().numpy(), want)


def test_a_layer_with_too_many_results_launches_nothing():
    """More results than a product counts (their memory does not exist: the call is refused ahead of them)."""
    m, n, k = 4160, (1 << 31) - 1, 32
    x = torch.ones((m, k), device=DEV)
    ws = torch.full((zc.zc_mx_workspace_bytes(m, n, k),), 0xA5, dtype=torch.uint8, device=DEV)
    some = ws.data_ptr()
    assert zc.binding.lib().zc_mx_linear(x.data_ptr(), 0, k, some, 16, some, 4, m, n, k, None, some, 0, n, 0, ws.data_ptr(), ws.nbytes, None) == ZC_ERR_ARG
    torch.cuda.synchronize()
    assert (ws == 0xA5).all()
