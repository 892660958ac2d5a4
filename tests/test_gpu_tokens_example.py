"""The example that runs embedding, layer norm, 4-bit layers, the collective's local work and both optimisers together: its gradients are those of the calls' definitions, and runs are alike bit by bit."""
import os
import sys

import numpy as np
import pytest
import torch

import training_model as model

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def values(t):
    return t.detach().double().cpu().numpy()


def test_gradients_between_the_layers():
    """From what stands between the calls: the norms' gradients, the residual's sum, and the table's."""
    import train_tokens as example
    m = example.Model(61, 40, 72, 3)
    g = torch.Generator(device=example.DEV).manual_seed(5)
    tokens = torch.randint(-1, 61, (150,), generator=g, device=example.DEV)
    targets = torch.randint(0, 61, (150,), generator=g, device=example.DEV)
    grads = [torch.full(s, 9.0, device=example.DEV) for s in m.shapes]
    loss, seen = example.gradients(m, tokens, targets, grads, scale=1.5)
    assert bool(torch.isfinite(loss)) and all(bool(torch.isfinite(t).all()) for t in grads)
    seen = {k: values(t) for k, t in seen.items()}
    u = model.U
    added = 0.0
    for x, dy, w, at, out in (("x1", "dy1", 3, 6, "dx1"), ("x0", "dy0", 1, 4, "dx")):
        w64 = values(m.others[w])
        _, mean, d, _ = model.norm(seen[x], w64, np.zeros(40), float(np.float32(1e-5)))
        dx, dw, db, ux, uw, ub = model.norm_backward(seen[dy], seen[x], mean, d, w64)
        # means and deviations of binary32 are off by what 64 roundings do to them, and so is z: on top of the 72 and 96 roundings of the gradients themselves
        far = 64 * u * (1 + d[:, None] * np.abs(seen[x]).mean(axis=1, keepdims=True))
        assert (np.abs(seen[out] - dx - added) <= (72 * u + 4 * far) * ux + 2 * u * np.abs(seen[out])).all()
        assert (np.abs(values(grads[at]) - dw) <= 96 * u * uw + (far * 2 * np.abs(seen[dy]) * (1 + np.abs(seen[x] - mean[:, None]) * d[:, None])).sum(axis=0)).all()
        assert (np.abs(values(grads[at + 1]) - db) <= 96 * u * ub).all()
        added = seen["dx1"]
    want, size, count = model.embedding_backward(seen["dx"], tokens.cpu().numpy(), 61, 1.5)
    assert (np.abs(values(grads[3]) - want) <= (count + 8)[:, None] * u * size).all()


def test_steps_are_alike():
    import train_tokens as example
    small = dict(ranks=2, rows=64, vocab=50, d=32, hidden=48, verbose=False)
    losses = example.train(steps=4, **small)
    assert all(l == l for l in losses)
    assert example.train(steps=4, **small) == losses
