"""Layer norm, embedding and the step for matrices at the largest sizes that zc.h names, as far as the GPU's memory holds them: indices that pass 31 and 32 bits."""
import numpy as np
import pytest
import torch

import paper_2502_18554_amd as zc
import training_model as model

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MOST = (1 << 31) - 1


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def test_norm_of_most_rows():
    """Rows of one value: out is the bias, the mean the value, dx nothing."""
    x = torch.empty(MOST, 1, dtype=torch.bfloat16, device=DEV).normal_(generator=generator(1))
    out, stats, b = torch.full_like(x, 9), torch.empty(2, MOST, device=DEV), torch.full((1,), 3.0, device=DEV)
    assert zc.zc_layer_norm(x, None, b, out, stats) == 0
    assert bool((out == 3).all()) and bool((stats[0] == x[:, 0]).all())
    dy = torch.zeros_like(x)
    places = torch.randint(0, MOST, (60,), generator=generator(2), device=DEV).unique()
    places[0], places[-1] = 0, MOST - 1
    dy[places] = 2
    db, ws = torch.zeros(1, device=DEV), torch.empty(zc.zc_layer_norm_workspace_bytes(MOST, 1), dtype=torch.uint8, device=DEV)
    assert zc.zc_layer_norm_backward(dy, x, stats, None, out, None, db, ws) == 0
    assert not bool(out.any()) and db.item() == 2 * len(places)


def test_most_tokens():
    tokens = torch.arange(MOST, dtype=torch.int32, device=DEV).remainder_(7).sub_(1)
    table = torch.arange(1.0, 7.0, device=DEV)[:, None].contiguous()
    out = torch.full((MOST, 1), 9, dtype=torch.bfloat16, device=DEV)
    assert zc.zc_embedding(table, tokens, out, scale=2.0) == 0
    assert bool((out[:, 0] == 2 * (tokens + 1)).all())             # (padding, -1, becomes 0)
    del out
    dy = torch.zeros(MOST, 1, dtype=torch.bfloat16, device=DEV)
    places = torch.randint(0, MOST, (90,), generator=generator(3), device=DEV).unique()
    places[0], places[-1] = 0, MOST - 1
    dy[places] = 1
    want = torch.bincount(tokens[places].long() + 1, minlength=7)[1:]
    grad, ws = torch.full((6, 1), 5.0, device=DEV), torch.full((zc.zc_embedding_workspace_bytes(MOST, 6, 1),), 0xFF, dtype=torch.uint8, device=DEV)
    assert zc.zc_embedding_backward(dy, tokens, grad, ws, scale=0.5) == 0
    assert torch.equal(grad[:, 0], want * 0.5)


def test_the_largest_table():
    rows = 1 << 29
    tokens = torch.randint(0, rows, (5000,), generator=generator(4), device=DEV)
    tokens[:4] = torch.tensor([rows - 1, rows, 0, rows - 1])
    dy = torch.randint(-8, 9, (5000, 2), generator=generator(5), device=DEV).bfloat16()      # (sums are exact)
    here = tokens < rows
    want = torch.zeros(rows, 2, dtype=torch.bfloat16, device=DEV).index_add_(0, tokens[here], dy[here])
    ws = torch.full((zc.zc_embedding_workspace_bytes(5000, rows, 2),), 0xFF, dtype=torch.uint8, device=DEV)
    grad = torch.full_like(want, 7)
    for add in (False, True):
        assert zc.zc_embedding_backward(dy, tokens, grad, ws, add=add) == 0
        assert torch.equal(grad, want * 2 if add else want)
    out = torch.empty(5000, 2, device=DEV)
    assert zc.zc_embedding(grad, tokens, out) == 0
    assert torch.equal(out[here], 2 * want[tokens[here]].float()) and not bool(out[1].any())


@pytest.mark.parametrize("rows,cols,wide", [(300, 1 << 20, True), (1 << 20, 500, False)])
def test_steps_of_the_largest_sides(rows, cols, wide):
    """Against 64 bits, within what zc.h gives: 2^-16 in two parts; without, some 2^-9, of which the factor of 1.5 that test_gpu_muon.py has makes 2^-8.4."""
    grad = torch.empty(rows, cols, device=DEV).normal_(generator=generator(6))
    p, shapes = torch.zeros(rows, cols, device=DEV), [(rows, cols)]
    state, ws = torch.zeros(zc.zc_muon_state_bytes(shapes) // 4, device=DEV), torch.full((zc.zc_muon_workspace_bytes(shapes, wide),), 0xFF, dtype=torch.uint8, device=DEV)
    assert zc.zc_muon([p], [grad], state, ws, 1.0, momentum=0.0, nesterov=False, wide=wide) == 0
    assert torch.equal(state[:rows * cols].view(rows, cols), grad)
    x = grad.double() if rows <= cols else grad.double().t().contiguous()
    x /= x.norm()
    for _ in range(5):
        a = x @ x.t().contiguous()
        x = (model.A * torch.eye(len(a), dtype=a.dtype, device=DEV) + model.B * a + model.C * (a @ a)) @ x
    got = -(p.double() if rows <= cols else p.double().t()) / max(1, rows / cols) ** 0.5
    assert float((got - x).norm() / x.norm()) <= (2.0 ** -16 if wide else 2.0 ** -8.4)
