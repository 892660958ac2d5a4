"""Layer norm of rows whose values are large: finite rows stay finite where binary32 holds their sums, by every way that a row goes (16 and 64 lanes, 256 and 512, several passes)."""
import numpy as np
import pytest
import torch

import paper_2502_18554_amd as zc
import training_model as model
from test_gpu_layer_norm import DEV, EPS, EPS32, check_forward, generator, matrix, values, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [100, 1500, 2049, 4096, 8192, 8193, 12000, 16384, 20000])
@pytest.mark.parametrize("kind,mean,scale", [("f32", 1e20, 1e16), ("f32", -1e20, 1e16), ("bf16", 2.5e19, 5e16)])
def test_a_mean_whose_square_passes_binary32(cols, kind, mean, scale):
    """2.5e19 squared is 6e38, behind the largest number; the sums of the row and of its squared deviations are not (20000 times 2.5e19 and, with bfloat16's steps of 1.4e17 there,
    20000 times (7.3e16)^2 = 1.1e38).  Values and means: fewer than 64 roundings relative to the mean magnitude M, as in test_gpu_layer_norm.py.

    d: a part of a row (a wave's) has squares around a mean of its own that is off by e1 <= 64 U M, and brings them to the row's mean, off by as much, so that with o the
    distance of the two exact means its sum of n_w squares is off by at most 2 n_w |o| e + n_w e^2, e = 2 x 64 U M.  Over the row, by Cauchy, sum n_w |o| <= n s (s^2 is the
    variance): relative to n s^2 that is 2 e / s + (e / s)^2, of d the half; and 64 roundings of its own."""
    x, _ = matrix(5, cols, kind, generator(cols), mean=mean, scale=scale)
    out, stats = torch.empty(5, cols, device=DEV), torch.empty(2, 5, device=DEV)
    assert zc.zc_layer_norm(x, None, None, out, stats, eps=EPS) == 0
    check_forward(x, None, None, out, None, "f32")
    _, want, d, _ = model.norm(values(x), np.ones(cols), np.zeros(cols), EPS32)
    size = np.abs(values(x)).mean(axis=1)
    e = 128 * model.U * size * d
    assert (np.abs(values(stats)[0] - want) <= 64 * model.U * size).all()
    assert (np.abs(values(stats)[1] - d) <= d * (64 * model.U + e + e * e / 2)).all()


@pytest.mark.parametrize("cols", [7, 100, 300, 777, 1500, 2050, 5001, 8200, 12000, 20001])
def test_gradients_of_constant_rows_of_large_values(cols):
    """The mean times d, 6e38, is behind binary32's range, (x - mean) d is 0: lanes behind the row's end have to stay out of its sums.  Statistics are given, so that the
    formula's gradients are those of the definition in 64 bits; tolerances as in test_gpu_layer_norm.py."""
    g = generator(cols)
    x, _ = matrix(5, cols, "f32", g)
    x[1], x[4] = 2e36, -2e36
    _, mean, d, _ = model.norm(values(x), np.ones(cols), np.zeros(cols), EPS32)
    mean[[1, 4]], d[[1, 4]] = float(np.float32(2e36)) * np.array([1, -1]), EPS32 ** -0.5
    stats = torch.tensor(np.stack([mean, d]), dtype=torch.float32, device=DEV)
    w = torch.rand(cols, generator=g, device=DEV).add_(0.5)
    dy, _ = matrix(5, cols, "f32", g)
    dx, dw, db = torch.empty_like(x), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    assert zc.zc_layer_norm_backward(dy, x, stats, w, dx, dw, db, workspace(5, cols)) == 0
    s = values(stats)
    wx, ww, wb, ux, uw, ub = model.norm_backward(values(dy), values(x), s[0], s[1], values(w))
    assert (np.abs(values(dx) - wx) <= 72 * model.U * ux + model.half_step("f32", wx) * (1 + 2 ** -6)).all()
    assert (np.abs(values(dw) - ww) <= 96 * model.U * uw).all()
    assert (np.abs(values(db) - wb) <= 96 * model.U * ub).all()
