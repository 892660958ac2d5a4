"""The step for matrices where test_gpu_muon.py leaves off: the bound that zc.h gives for two parts, thin matrices in two parts, gradients under the norm's floor.

In two parts p' is off by some 2^-18 of the step (zc.h): that is the tolerance in the 2-norm, with 2^-16, the largest that zc.h names, for sums of more than 4096 values.

By arithmetic: operands' roundings (two binary16 numbers: 2^-22) are far under that.  Sums are in binary32, made in steps of 16 values, each of which rounds the sum so far by half a step at most:
a random walk, sqrt(steps) 2^-24 / 3 of the sum for sums of squares (a rounding is 2^-24 / sqrt(3) at the root of the mean square, a growing sum at that 1 / sqrt(3) of its end).  Of the polynomial's
terms, up to 5 times what remains of them near 1.1, three more roundings.  A step of the iteration takes an error in a singular value s further by s p'(s) / p(s), at most 5 (at 1.2), so that few
singular values, which may all lie where that is large, come out worse than many: what it makes of a matrix of at most three rows is computed, not guessed (`walked`: the definition in 64 bits with
such roundings drawn at random), and three times the largest of eight draws is allowed."""
import numpy as np
import pytest
import torch

import paper_2502_18554_amd as zc
import training_model as model
from test_gpu_muon import DEV, TYPES, generator, gradient, off, parts_of, state_of, values, workspace

pytestmark = pytest.mark.gpu


def step(grads, wide, **how):
    """X of each, from no weights with a rate of one; and the momentum."""
    shapes = [tuple(g.shape) for g in grads]
    p, state = [torch.zeros(s, device=DEV) for s in shapes], state_of(shapes)
    assert zc.zc_muon(p, grads, state, workspace(shapes, wide), 1.0, momentum=0.0, nesterov=False, wide=wide, **how) == 0
    return p, parts_of(state, shapes)


def wanted(grad, iterations=5):
    r, c = grad.shape
    return -model.orthogonalised(values(grad), iterations, 0) * max(1, r / c) ** 0.5


def walked(u, seed):
    """X after five iterations with operands in two parts and random roundings of binary32 sums and terms."""
    g = torch.Generator()
    g.manual_seed(seed)
    turned = u.shape[0] > u.shape[1]
    x = torch.from_numpy(np.ascontiguousarray(u.T if turned else u))
    r, c = x.shape
    drawn = lambda *shape: torch.randn(*shape, generator=g, dtype=torch.float64)
    summed = lambda a, b, k: a @ b + model.U / 3 * max(k / 16, 1) ** 0.5 * a.norm(dim=1)[:, None] * b.norm(dim=0)[None] * drawn(a.shape[0], b.shape[1])
    x = model.rounded(x / x.norm(), 2)
    for i in range(5):
        a = model.rounded(summed(x, x.t().contiguous(), c), 2)
        b, d = model.B * a, model.C * summed(a, a, r)
        b = model.A * torch.eye(r, dtype=torch.float64) + b + d + model.U / 3 ** 0.5 * (b.abs() + d.abs() + model.A) * drawn(r, r)
        x = summed(model.rounded(b, 2), x, r)
        if i < 4:
            x = model.rounded(x, 2)
    return (x.t() if turned else x).numpy()


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (5, 3), (17, 17), (40, 30), (64, 64), (65, 130), (129, 257), (300, 100), (256, 512), (333, 1531), (513, 700), (96, 4000), (128, 9000), (9000, 65),
                                       (700, 20000)])
def test_two_parts_within_the_bound(rows, cols):
    """(With 128 rows or fewer a segment has two stages, fewer than the requests that run ahead.)"""
    g = generator(rows + 7 * cols)
    grad = gradient(rows, cols, g)
    (p,), _ = step([grad], True)
    room = 2.0 ** (-18 if max(rows, cols) <= 4096 else -16)
    assert off(values(p), wanted(grad)) <= room
    (_, q, r), _ = step([gradient(30, 50, g), grad, grad], True)
    assert off(values(q), wanted(grad)) <= room and torch.equal(q, r)


@pytest.mark.parametrize("rows,cols", [(1, 40000), (2, 70001), (50001, 3)])
def test_thin_matrices_in_two_parts(rows, cols):
    g = generator(rows + 7 * cols)
    grad = gradient(rows, cols, g)
    (p,), (m,) = step([grad], True)
    want = wanted(grad)
    room = 3 * max(off(walked(values(grad), seed), want / -max(1, rows / cols) ** 0.5) for seed in range(8))
    assert off(values(p), want) <= room
    assert torch.equal(m, grad)
    (_, q, r), _ = step([gradient(30, 50, g), grad, grad], True)
    assert off(values(q), want) <= room and torch.equal(q, r)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3e38])
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("wide", [False, True])
def test_gradients_that_are_not_finite(bad, nesterov, wide):
    """(3e38 times the scale of two is infinite.)  The matrix's weights become NaNs, the momentum only where the gradient is not finite; other matrices stay what they are without it."""
    g = generator(12)
    shapes = [(40, 50), (150, 20), (1, 1), (40, 50)]
    grads = [gradient(*s, g) for s in shapes]
    scale = torch.full((1,), 2.0, device=DEV)
    clean, p = ([torch.ones(s, device=DEV) for s in shapes] for _ in range(2))
    states = [state_of(shapes) for _ in range(2)]
    how = dict(nesterov=nesterov, wide=wide, d_grad_scale=scale)
    assert zc.zc_muon(clean, grads, states[0], workspace(shapes, wide), 0.1, **how) == 0
    grads[1][149, 3] = grads[2][0, 0] = bad
    assert zc.zc_muon(p, grads, states[1], workspace(shapes, wide), 0.1, **how) == 0
    assert torch.equal(p[0], clean[0]) and torch.equal(p[3], clean[3])
    assert bool(p[1].isnan().all()) and bool(p[2].isnan().all())
    for i, (got, want) in enumerate(zip(parts_of(states[1], shapes), parts_of(states[0], shapes))):
        touched = torch.zeros(shapes[i], dtype=torch.bool, device=DEV)
        if i in (1, 2):
            touched[-1, 3 if i == 1 else 0] = True
        assert not bool(got[touched].isfinite().any()) and torch.equal(got[~touched], want[~touched])


@pytest.mark.parametrize("wide", [False, True])
def test_gradients_under_the_floor(wide):
    """Norms under 1e-7, by which X is divided then.  6e-9: X is as any other.  6e-30: X, 6e-23 at 2^12, is less than half of binary16's smallest number, 3e-8, and so nothing."""
    g = generator(13)
    grad = torch.rand(50, 60, generator=g, device=DEV).sub_(0.5).mul_(4e-10)
    (p,), _ = step([grad], wide)
    exact = model.orthogonalised(values(grad), 5, 0)
    rounded = model.orthogonalised(values(grad), 5, 2 if wide else 1)
    assert 0.01 < np.abs(exact).max() < 1
    assert off(values(p), -exact) <= 1.5 * off(rounded, exact) + 2.0 ** -18
    (p,), _ = step([grad * 1e-21], wide)
    assert not bool(p.any())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_copies_that_are_the_matrices_themselves(kind, monkeypatch):
    """What .to() gives for the type that a tensor has already: the same call without them.  A copy that is another matrix is refused."""
    g = generator(14)
    shapes = [(70, 40), (64, 64), (5, 90)]
    grads = [gradient(*s, g) for s in shapes]
    start = [torch.randn(s, generator=g, device=DEV).to(TYPES[kind]) for s in shapes]

    def run(copies):
        p = [t.clone() for t in start]
        others = [torch.zeros_like(t) for t in p]
        state = state_of(shapes)
        assert zc.zc_muon(p, grads, state, workspace(shapes, False), 0.1, d_copies=copies(p, others)) == 0
        return (*p, state), others

    for _ in range(2):
        want, _ = run(lambda p, o: None)
        for copies in (lambda p, o: [t.to(TYPES[kind]) for t in p], lambda p, o: [p[0], o[1], p[2]]):
            got, others = run(copies)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(others[1], want[1]) and not bool(others[0].any())
        p = [t.clone() for t in start]
        assert zc.zc_muon([p[0], p[0].clone()], [grads[0]] * 2, state_of(shapes[:1] * 2), workspace(shapes[:1] * 2, False), 0.1, d_copies=[torch.zeros_like(p[0]), p[0]]) == zc.binding.ZC_ERR_ARG
        monkeypatch.setattr(zc.binding, "_native_layers", None)
