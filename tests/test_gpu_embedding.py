"""Embedding and its gradient against the definitions.

The lookup is one product in binary32 and one rounding: compared bit for bit.  A gradient's sum is at most 64 places of a piece deep, then a quarter of the pieces, two more and the factor: with the sizes
here, under min(places, 256) + 8 roundings of binary32 on the sum of magnitudes, and the result's own."""
import numpy as np
import pytest
import torch

import paper_2502_18554_amd as zc
import training_model as model

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def values(t):
    return t.detach().double().cpu().numpy()


def workspace(n, rows, cols):
    return torch.full((zc.zc_embedding_workspace_bytes(n, rows, cols),), 0xFF, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("rows,cols,n", [(1, 1, 1), (5, 7, 3), (50, 8, 100), (300, 129, 77), (1000, 777, 333), (17, 2048, 40), (9, 5001, 30), (2000, 4096, 1), (70000, 16, 5000)])
@pytest.mark.parametrize("kinds", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("bits", [32, 64])
def test_lookup(rows, cols, n, kinds, bits):
    g = generator(rows + cols)
    table = torch.randn(rows, cols + 3, generator=g, device=DEV).to(TYPES[kinds[0]])[:, 1:cols + 1]            # (rows apart, and not where a load would like them)
    tokens = torch.randint(-2, rows + 2, (n,), generator=g, device=DEV).to(torch.int32 if bits == 32 else torch.int64)
    if bits == 64:
        tokens[0] = (1 << 40) + 1                                                                              # (far outside, and inside when cut to 32 bits)
    room = torch.full((n, cols + 2), -7.0, dtype=TYPES[kinds[1]], device=DEV)
    out = room[:, :cols]
    assert zc.zc_embedding(table, tokens, out, scale=0.3) == 0
    there = (tokens >= 0) & (tokens < rows)
    want = torch.where(there[:, None], table[torch.where(there, tokens, 0).long()].float() * 0.3, 0).to(out.dtype)
    assert torch.equal(out, want) and bool((room[:, cols:] == -7).all())


def test_far_rows():
    """Tables whose last rows lie more than 2^32 bytes behind their first ones, read and added to."""
    rows, cols = 300000, 8192
    table = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([rows - 1, 0, rows // 2, rows - 1, rows - 7, 262144, rows], device=DEV)
    g = generator(1)
    table[at[:-1]] = torch.randn(6, cols, generator=g, device=DEV).bfloat16()
    out = torch.empty(7, cols, dtype=torch.bfloat16, device=DEV)
    assert zc.zc_embedding(table, at, out) == 0
    assert torch.equal(out[:-1], table[at[:-1]]) and bool((out[-1] == 0).all())
    dy = torch.randint(-3, 4, (7, cols), generator=g, device=DEV).float()
    table[at[:-1]] = 1.0
    assert zc.zc_embedding_backward(dy, at, table, workspace(7, rows, cols), add=True) == 0
    want = 1 + dy[:-1]
    want[0] = want[3] = 1 + dy[0] + dy[3]
    assert torch.equal(table[at[:-1]].float(), want)
    table.zero_()
    assert zc.zc_embedding_backward(dy, at, table, workspace(7, rows, cols)) == 0
    assert torch.equal(table[at[:-1]].float(), want - 1) and int((table != 0).any(dim=1).sum()) == 5


def test_many_tokens():
    """More rows than workgroups, each of which takes several."""
    g = generator(9)
    for n, cols in ((40000, 24), (9001, 520), (5000, 4100)):
        table = torch.randn(977, cols, generator=g, device=DEV)
        tokens = torch.randint(-1, 977, (n,), generator=g, device=DEV, dtype=torch.int32)
        out = torch.full((n + 1, cols), -7.0, dtype=torch.float16, device=DEV)
        assert zc.zc_embedding(table, tokens, out[:n], scale=0.5) == 0
        assert torch.equal(out[:n], torch.where((tokens >= 0)[:, None], table[tokens.clamp(min=0).long()] * 0.5, 0).half()) and bool((out[n] == -7).all())


def check_gradient(dy, tokens, grad, before, scale, kind):
    want, size, count = model.embedding_backward(values(dy), tokens.cpu().numpy().reshape(-1), grad.shape[0], float(np.float32(scale)))
    if before is not None:
        want, size = want + before, size + np.abs(before)
    rough = (np.minimum(count, 256) + 8)[:, None] * model.U * size
    assert (np.abs(values(grad) - want) <= rough + model.half_step(kind, want) * (1 + 2 ** -6) * (size > 0)).all()
    if before is not None:
        assert np.array_equal(values(grad)[count == 0], before[count == 0])


CASES = [("one", 1, 1, 1), ("few", 5, 7, 3), ("even", 50, 8, 300), ("even", 300, 129, 1000), ("skewed", 1009, 777, 2117), ("skewed", 260, 2050, 500), ("same", 40, 300, 3000), ("same", 3, 8, 5000), ("outside", 70, 40, 200),
         ("stride", 300000, 4, 3000), ("runs", 30, 264, 2500), ("even", 2000000, 2, 3000)]


def tokens_of(how, rows, n, g):
    if how == "same":
        t = torch.full((n,), rows - 1, device=DEV)
        t[n // 3] = 0
    elif how == "outside":
        t = torch.where(torch.arange(n, device=DEV) % 2 == 0, -1, rows)
    elif how == "stride":                    # all of them dealt to the same workgroup, and different
        t = torch.arange(n, device=DEV) * 256 % rows
    elif how == "runs":                      # pieces that begin and end with a row's places
        t = (torch.arange(n, device=DEV) // 8) % rows
    elif how == "skewed":
        t = (torch.exp(torch.rand(n, generator=g, device=DEV) * np.log(rows + 1)) - 1).long()
        t[::7] = -1
    else:
        t = torch.randint(0, rows, (n,), generator=g, device=DEV)
    return t.long()


@pytest.mark.parametrize("how,rows,cols,n", CASES)
@pytest.mark.parametrize("kinds,add", [(("f32", "f32"), False), (("bf16", "f32"), True), (("f16", "bf16"), False), (("bf16", "f16"), True)])
def test_gradient(how, rows, cols, n, kinds, add):
    g = generator(n)
    tokens = tokens_of(how, rows, n, g)
    if add:
        tokens = tokens.int()
    dy = torch.randn(n, cols + 1, generator=g, device=DEV).to(TYPES[kinds[0]])[:, 1:]
    room = torch.randn(rows, cols + 1, generator=g, device=DEV).to(TYPES[kinds[1]])
    grad, guard = room[:, :cols], room[:, cols].clone()
    before = values(grad)
    ws = workspace(n, rows, cols)
    assert zc.zc_embedding_backward(dy, tokens, grad, ws, scale=0.7, add=add) == 0
    first = grad.clone()
    check_gradient(dy, tokens, grad, before if add else None, 0.7, kinds[1])
    assert torch.equal(room[:, cols], guard)
    grad.copy_(torch.from_numpy(before))
    assert zc.zc_embedding_backward(dy, tokens, grad, ws, scale=0.7, add=add) == 0
    assert torch.equal(grad, first)


def test_order_of_many_tokens():
    """Enough tokens and rows for every way through the order: each row's places are all there, by whole numbers that add exactly."""
    for rows, n in ((50021, 70001), (7, 70001), (600000, 30011)):
        g = generator(n)
        tokens = tokens_of("skewed", rows, n, g)
        dy = torch.randint(-8, 9, (n, 2), generator=g, device=DEV).float()
        dy[:, 1] = 1
        grad = torch.full((rows, 2), 5.0, device=DEV)
        assert zc.zc_embedding_backward(dy, tokens, grad, workspace(n, rows, 2)) == 0
        want = torch.zeros(rows + 1, 2, dtype=torch.float64, device=DEV)
        want.index_add_(0, torch.where(tokens >= 0, tokens, rows), dy.double())
        assert torch.equal(grad.double(), want[:rows])


def test_nothing_to_do():
    grad, ws = torch.ones(300, 5, device=DEV), workspace(0, 300, 5)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    assert zc.zc_embedding(grad, none, torch.empty(0, 5, device=DEV)) == 0
    assert zc.zc_embedding_backward(torch.empty(0, 5, device=DEV), none, grad, ws, add=True) == 0 and bool((grad == 1).all())
    assert zc.zc_embedding_backward(torch.empty(0, 5, device=DEV), none, grad, ws) == 0 and bool((grad == 0).all())
    out = torch.ones(4, 5, device=DEV)
    assert zc.zc_embedding(torch.empty(0, 5, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV), out) == 0 and bool((out == 0).all())
    assert zc.zc_embedding_backward(out, torch.zeros(4, dtype=torch.int64, device=DEV), torch.empty(0, 5, device=DEV), workspace(4, 0, 5)) == 0


def test_values_that_are_not_finite_keep_to_their_rows():
    g = generator(2)
    tokens = torch.randint(0, 20, (400,), generator=g, device=DEV)
    dy = torch.randn(400, 33, generator=g, device=DEV)
    clean, grad, ws = torch.empty(20, 33, device=DEV), torch.empty(20, 33, device=DEV), workspace(400, 20, 33)
    assert zc.zc_embedding_backward(dy, tokens, clean, ws) == 0
    at = int(tokens[17])
    dy[17, 3] = float("nan")
    assert zc.zc_embedding_backward(dy, tokens, grad, ws) == 0
    assert bool(grad[at, 3].isnan())
    grad[at, 3] = clean[at, 3]
    assert torch.equal(grad, clean)


def test_graph_streams_and_other_ways(monkeypatch):
    g = generator(4)
    tokens = tokens_of("skewed", 500, 1500, g)
    table, dy = torch.randn(500, 96, generator=g, device=DEV), torch.randn(1500, 96, generator=g, device=DEV).bfloat16()

    def make():
        return dict(out=torch.zeros(1500, 96, device=DEV), grad=torch.zeros(500, 96, device=DEV), ws=workspace(1500, 500, 96))

    def call(t, **how):
        assert zc.zc_embedding(table, tokens.view(3, 500), t["out"], scale=2.0, **how) == 0
        assert zc.zc_embedding_backward(dy, tokens.view(3, 500), t["grad"], t["ws"], scale=2.0, **how) == 0

    same = lambda a, b: torch.equal(a["out"], b["out"]) and torch.equal(a["grad"], b["grad"])
    eager, captured, other = make(), make(), make()
    call(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(captured)
    for i in range(3):
        tokens.copy_(tokens_of("skewed", 500, 1500, g))
        captured["out"].zero_(), captured["grad"].fill_(3)
        graph.replay()
        call(eager)
        torch.cuda.synchronize()
        assert same(captured, eager)
    call(other, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert same(other, eager)
    monkeypatch.setattr(zc.binding, "_native_layers", None)
    by_ctypes = make()
    call(by_ctypes)
    assert same(by_ctypes, eager)
