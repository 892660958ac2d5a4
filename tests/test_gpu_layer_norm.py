"""Layer norm and its gradients against the definition in 64 bits.

Tolerances: a sum of a row is at most 32 values of a lane, 10 steps between lanes and waves, and 8 waves deep: under 64 roundings with those around it.  A sum down the columns is at most
rows / 512 + 16 + 32 + 16 deep, under 96 for the sizes here.  A result's own rounding comes on top."""
import numpy as np
import pytest
import torch

import paper_2502_18554_amd as zc
import training_model as model

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
EPS32 = float(np.float32(EPS))


def values(t):
    return t.detach().double().cpu().numpy()


def matrix(rows, cols, kind, g, pad=0, offset=0, scale=1.0, mean=0.0):
    """A matrix whose rows lie `pad` values further apart than they have to and begin `offset` values behind an aligned address; what lies between them is -7."""
    room = torch.full((rows * (cols + pad) + offset,), -7.0, dtype=TYPES[kind], device=DEV)
    m = room[offset:].view(rows, cols + pad)[:, :cols]
    m.copy_(mean + scale * torch.randn(rows, cols, generator=g, device=DEV))
    return m, room


def between(m, room):
    """What lies between the rows and before them."""
    keep = torch.ones_like(room, dtype=torch.bool)
    keep.as_strided(m.shape, m.stride(), m.storage_offset()).fill_(False)
    return room[keep]


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def workspace(rows, cols):
    return torch.full((max(zc.zc_layer_norm_workspace_bytes(rows, cols), 16),), 0xFF, dtype=torch.uint8, device=DEV)


def check_forward(x, w, b, out, stats, kind):
    w64 = values(w) if w is not None else np.ones(x.shape[1])
    b64 = values(b) if b is not None else np.zeros(x.shape[1])
    want, mean, d, unit = model.norm(values(x), w64, b64, EPS32)
    assert (np.abs(values(out) - want) <= 64 * model.U * unit + model.half_step(kind, want) * (1 + 2 ** -6)).all()
    if stats is not None:
        got = values(stats)
        assert (np.abs(got[0] - mean) <= 64 * model.U * np.abs(values(x)).mean(axis=1) + 1e-40).all()
        assert (np.abs(got[1] - d) <= 64 * model.U * d * (1 + d * np.abs(values(x)).mean(axis=1) * 64 * model.U)).all()


SIZES = [(1, 1), (3, 7), (2, 8), (5, 128), (17, 129), (64, 512), (33, 513), (9, 1024), (7, 1531), (4, 2048), (5, 2049), (3, 4096), (2, 5001), (3, 8192), (2, 8193), (2, 16384), (2, 16385), (3, 20001),
         (3000, 64), (700, 300), (2500, 1000), (1100, 2100)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("kinds", [("f32", "f32", "f32"), ("bf16", "bf16", "f32"), ("f32", "bf16", "bf16"), ("f16", "f32", "f16")])
def test_forward_and_backward(rows, cols, kinds):
    kx, ky, kw = kinds
    g = generator(rows * 31 + cols)
    x, _ = matrix(rows, cols, kx, g, mean=0.5)
    w, b = (1 + 0.3 * torch.randn(cols, generator=g, device=DEV)).to(TYPES[kw]), torch.randn(cols, generator=g, device=DEV).to(TYPES[kw])
    out, stats = torch.full((rows, cols), 9.0, dtype=TYPES[ky], device=DEV), torch.full((2, rows), 9.0, device=DEV)
    assert zc.zc_layer_norm(x, w, b, out, stats, eps=EPS) == 0
    check_forward(x, w, b, out, stats, ky)
    dy, _ = matrix(rows, cols, ky, g)
    dx, dw, db = torch.empty_like(x), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    assert zc.zc_layer_norm_backward(dy, x, stats, w, dx, dw, db, workspace(rows, cols)) == 0
    s = values(stats)
    wx, ww, wb, ux, uw, ub = model.norm_backward(values(dy), values(x), s[0], s[1], values(w))
    assert (np.abs(values(dx) - wx) <= 72 * model.U * ux + model.half_step(kx, wx) * (1 + 2 ** -6)).all()
    assert (np.abs(values(dw) - ww) <= 96 * model.U * uw).all()
    assert (np.abs(values(db) - wb) <= 96 * model.U * ub).all()


@pytest.mark.parametrize("rows,cols,pad,offset", [(5, 100, 3, 1), (9, 777, 1, 3), (6, 2048, 8, 0), (3, 3001, 5, 7), (4, 4096, 1, 1), (2, 9000, 2, 5), (2, 17000, 3, 1)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_that_lie_apart(rows, cols, pad, offset, kind):
    g = generator(7)
    x, _ = matrix(rows, cols, kind, g, pad, offset)
    out, out_room = matrix(rows, cols, kind, g, pad + 1, offset + 1)
    stats = torch.empty(2, rows, device=DEV)
    assert zc.zc_layer_norm(x, None, None, out, stats, eps=EPS) == 0
    check_forward(x, None, None, out, stats, kind)
    assert bool((between(out, out_room) == -7).all())
    dy, _ = matrix(rows, cols, kind, g, 2 * pad, offset)
    dx, dx_room = matrix(rows, cols, kind, g, pad, offset + 2)
    before = values(dx)
    db = torch.full((cols,), 2.0, device=DEV)
    assert zc.zc_layer_norm_backward(dy, x, stats, None, dx, None, db, workspace(rows, cols), add=True, add_weights=True) == 0
    s = values(stats)
    wx, _, wb, ux, _, ub = model.norm_backward(values(dy), values(x), s[0], s[1], np.ones(cols))
    want = wx + before
    assert (np.abs(values(dx) - want) <= 73 * model.U * (ux + np.abs(before)) + model.half_step(kind, want) * (1 + 2 ** -6)).all()
    assert bool((between(dx, dx_room) == -7).all())
    assert (np.abs(values(db) - 2 - wb) <= 97 * model.U * (ub + 2)).all()


@pytest.mark.parametrize("cols", [96, 1500, 4096, 12000, 17000])
def test_in_place(cols):
    g = generator(3)
    x, _ = matrix(700, cols, "bf16", g)
    w = torch.rand(cols, generator=g, device=DEV)
    out, stats = torch.empty_like(x), torch.empty(2, 700, device=DEV)
    assert zc.zc_layer_norm(x, w, None, out, stats) == 0
    y = x.clone()
    assert zc.zc_layer_norm(y, w, None, y) == 0
    assert torch.equal(y, out)
    dy, _ = matrix(700, cols, "bf16", g)
    dx, dw, ws = torch.empty_like(x), torch.empty(cols, device=DEV), workspace(700, cols)
    assert zc.zc_layer_norm_backward(dy, x, stats, w, dx, dw, None, ws) == 0
    over, again = dy.clone(), torch.empty(cols, device=DEV)
    assert zc.zc_layer_norm_backward(over, x, stats, w, over, again, None, ws) == 0
    assert torch.equal(over, dx) and torch.equal(again, dw)
    over = x.clone()
    assert zc.zc_layer_norm_backward(dy, over, stats, w, over, again, None, ws) == 0
    assert torch.equal(over, dx) and torch.equal(again, dw)


def test_far_rows():
    """Rows that lie more than 2^32 values apart in all."""
    rows, cols, apart = 70000, 40, 65000
    room = torch.empty(rows * apart, dtype=torch.bfloat16, device=DEV)
    x = room.view(rows, apart)[:, :cols]
    x.copy_(torch.randn(rows, cols, generator=generator(2), device=DEV))
    near, out, stats, near_stats = x.contiguous(), torch.empty(rows, cols, device=DEV), torch.empty(2, rows, device=DEV), torch.empty(2, rows, device=DEV)
    want = torch.empty_like(out)
    assert zc.zc_layer_norm(near, None, None, want, near_stats) == 0 and zc.zc_layer_norm(x, None, None, out, stats) == 0
    assert torch.equal(out, want) and torch.equal(stats, near_stats)
    ws, dw, again, near_dx = workspace(rows, cols), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV), torch.empty_like(near)
    assert zc.zc_layer_norm_backward(want, near, stats, None, near_dx, dw, None, ws) == 0
    assert zc.zc_layer_norm_backward(want, x, stats, None, x, again, None, ws) == 0
    assert torch.equal(x, near_dx) and torch.equal(dw, again)


def test_large_mean_and_constant_rows():
    g = generator(5)
    x, _ = matrix(6, 3000, "f32", g, mean=1000.0)
    x[2] = 3.25
    x[3] = 0
    x[4] *= 1e-20
    out, stats = torch.empty_like(x), torch.empty(2, 6, device=DEV)
    assert zc.zc_layer_norm(x, None, None, out, stats, eps=EPS) == 0
    check_forward(x, None, None, out, stats, "f32")
    assert bool((out[3] == 0).all())


@pytest.mark.parametrize("cols", [40, 1000, 4000, 20000])
def test_rows_that_are_not_finite_keep_to_themselves(cols):
    g = generator(6)
    x, _ = matrix(9, cols, "f32", g)
    clean, out = torch.empty_like(x), torch.empty_like(x)
    assert zc.zc_layer_norm(x, None, None, clean) == 0
    x[2, cols // 2] = float("nan")
    x[5, 0] = float("inf")
    x[6, cols - 1] = -float("inf")
    assert zc.zc_layer_norm(x, None, None, out) == 0
    bad = torch.tensor([2, 5, 6], device=DEV)
    good = torch.tensor([0, 1, 3, 4, 7, 8], device=DEV)
    assert bool(out[bad].isnan().all()) and torch.equal(out[good], clean[good])


def test_gradients_against_differences():
    """In 64 bits on the definition: the formula's gradients are the limits of differences, and the calls' are the formula's (above)."""
    g = generator(8)
    x, w, b, dy = (values(torch.randn(s, generator=g, device=DEV)) for s in ((3, 11), (11,), (11,), (3, 11)))
    loss = lambda x, w, b: (model.norm(x, w, b, EPS)[0] * dy).sum()
    _, mean, d, _ = model.norm(x, w, b, EPS)
    dx, dw, db, *_ = model.norm_backward(dy, x, mean, d, w)
    h = 1e-5
    for of, grad in ((0, dx), (1, dw), (2, db)):
        for at in np.ndindex(grad.shape):
            args = [x.copy(), w.copy(), b.copy()]
            args[of][at] += h
            up = loss(*args)
            args[of][at] -= 2 * h
            assert abs((up - loss(*args)) / (2 * h) - grad[at]) < 1e-6 * (1 + abs(grad[at]))


def test_no_rows():
    dw, db = torch.ones(50, device=DEV), torch.ones(50, dtype=torch.float32, device=DEV)
    x, stats, ws = torch.empty(0, 50, device=DEV), torch.empty(2, 0, device=DEV), torch.empty(16, dtype=torch.uint8, device=DEV)
    assert zc.zc_layer_norm(x, dw, db, x, stats) == 0
    assert zc.zc_layer_norm_backward(x, x, stats, None, x, dw, db, ws, add_weights=True) == 0
    assert bool((dw == 1).all())
    assert zc.zc_layer_norm_backward(x, x, stats, None, x, dw, db, ws) == 0
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_graph_streams_and_other_ways(monkeypatch):
    """A captured call replayed between others, a call on another stream, and the call by ctypes: the same bytes."""
    g = generator(9)
    x, _ = matrix(300, 1300, "bf16", g)
    dy, _ = matrix(300, 1300, "bf16", g)
    w = torch.rand(1300, generator=g, device=DEV)

    def make():
        return dict(out=torch.zeros_like(x), stats=torch.zeros(2, 300, device=DEV), dx=torch.zeros_like(x), dw=torch.zeros(1300, device=DEV), db=torch.zeros(1300, device=DEV), ws=workspace(300, 1300))

    def call(t, **how):
        assert zc.zc_layer_norm(x, w, None, t["out"], t["stats"], **how) == 0
        assert zc.zc_layer_norm_backward(dy, x, t["stats"], w, t["dx"], t["dw"], t["db"], t["ws"], **how) == 0

    def same(a, b):
        return all(torch.equal(a[k], b[k]) for k in ("out", "stats", "dx", "dw", "db"))

    eager, captured, other = make(), make(), make()
    call(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(captured)
    side = torch.cuda.Stream()
    for _ in range(3):
        for k in ("out", "stats", "dx", "dw", "db"):
            captured[k].zero_()
        graph.replay()
        call(make())
        torch.cuda.synchronize()
        assert same(captured, eager)
    torch.cuda.synchronize()
    call(other, stream=side)
    torch.cuda.synchronize()
    assert same(other, eager)
    monkeypatch.setattr(zc.binding, "_native_layers", None)
    by_ctypes = make()
    call(by_ctypes)
    assert same(by_ctypes, eager)
