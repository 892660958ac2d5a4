"""CPU tests of the host side of layer norm, embedding and the step for matrices: sizes, refusals that need no GPU, the native calls' choice of way."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import paper_2502_18554_amd as zc
from paper_2502_18554_amd import binding as b

A, B, D, E = 0x10000, 0x20000, 0x30000, 0x40000          # addresses that are never used: every call here is refused first, or has nothing to do
OK, ARG = 0, 1
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    return b.lib()


def words(*values):
    return (C.c_uint64 * max(len(values), 1))(*values)


def caller(f, **defaults):
    def call(**o):
        assert set(o) <= set(defaults)
        return f(*{**defaults, **o}.values())
    return call


def test_sizes(L):
    for rows, cols in ((0, 5), (1, 1), (7, 128), (1000, 129), (5000, 4096), (3, 16384), (700, 16385)):
        assert zc.zc_layer_norm_workspace_bytes(rows, cols) <= 65536 + 16384 * (cols + 64)
        assert zc.zc_layer_norm_workspace_bytes(rows, cols) >= (8 * cols if rows else 0)
    assert zc.zc_layer_norm_workspace_bytes(1 << 31, 5) == 0 and zc.zc_layer_norm_workspace_bytes(5, (1 << 27) + 1) == 0
    for n, vocab, cols in ((0, 1, 1), (1, 5, 7), (8, 300, 4096), (65536, 200000, 8), (5117, 1009, 777), (1 << 31 - 1, 1 << 29, 1)):
        assert 8 * n + 4 * vocab <= zc.zc_embedding_workspace_bytes(n, vocab, cols)
    for n, vocab, cols in ((0, 1, 1), (1, 5, 7), (8, 300, 4096), (65536, 200000, 8), (5117, 1009, 777), (2047, 50, 2048), (2049, 50, 2048)):
        assert zc.zc_embedding_workspace_bytes(n, vocab, cols) <= (1 << 20) + 64 * n + 16 * vocab + (n // 8 + 2) * 8 * (cols + 64)
    assert zc.zc_embedding_workspace_bytes(5, (1 << 29) + 1, 5) == 0 and zc.zc_embedding_workspace_bytes(5, 5, (1 << 23) + 1) == 0
    assert zc.zc_muon_state_bytes([]) == 0 and zc.zc_muon_state_bytes([(3, 5), (0, 7), (32, 2)]) == 4 * (32 + 64) and zc.zc_muon_state_bytes([((1 << 20) + 1, 1)]) == 0
    one, two = zc.zc_muon_workspace_bytes([(100, 300)]), zc.zc_muon_workspace_bytes([(100, 300)], wide=True)
    assert 2 * (100 * 384 + 2 * 300 * 128 + 2 * 100 * 128) <= one < two <= 24 * (100 + 256) * (300 + 256)
    assert zc.zc_muon_workspace_bytes([(300, 100)]) == one and zc.zc_muon_workspace_bytes([(1 << 21, 5)]) == 0
    assert zc.zc_muon_workspace_bytes([(5, 5)] * 500) == zc.zc_muon_workspace_bytes([(5, 5)] * 64)            # (the next ones use the same place)


def test_refusals_of_the_norm(L):
    f = caller(L.zc_layer_norm, x=A, xt=1, rows=8, cols=64, xs=64, w=B, b=B, wt=0, eps=1e-5, out=D, ot=1, os=64, stats=E, stream=None)
    for bad in (dict(x=None), dict(x=A + 1), dict(xt=3), dict(xs=63), dict(w=B + 2), dict(b=B + 1), dict(wt=-1), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(eps=1e39), dict(out=None), dict(out=D + 1),
                dict(ot=7), dict(os=10), dict(stats=E + 2), dict(rows=1 << 31), dict(cols=(1 << 27) + 1, xs=1 << 28, os=1 << 28), dict(out=A, ot=2), dict(out=A, os=65)):
        assert f(**bad) == ARG, bad
    assert f(rows=0) == OK and f(cols=0, xs=0, os=0) == OK and f(rows=0, x=None, out=None) == OK
    g = caller(L.zc_layer_norm_backward, dy=A, dyt=1, dys=64, x=B, xt=0, xs=64, stats=E, w=D, wt=0, rows=8, cols=64, dx=D, dxt=0, dxs=64, dw=E, db=E + 4096, dwt=0, flags=3, ws=A, bytes=1 << 20, stream=None)
    for bad in (dict(dy=None), dict(dy=A + 1), dict(dyt=4), dict(dys=63), dict(x=None), dict(x=B + 2), dict(xt=9), dict(xs=0), dict(stats=None), dict(stats=E + 1), dict(w=D + 2), dict(wt=3),
                dict(rows=1 << 31), dict(dx=D + 2), dict(dxt=5), dict(dxs=63), dict(dw=E + 2), dict(db=E + 1), dict(db=E), dict(dwt=-1), dict(flags=4), dict(ws=None), dict(ws=A + 8), dict(bytes=8 * 64 - 1),
                dict(dx=A, dxt=0), dict(dx=A, dxt=1, dxs=65), dict(dx=B, dxs=80)):
        assert g(**bad) == ARG, bad
    assert g(cols=0, dys=0, xs=0, dxs=0) == OK and g(rows=0, dw=None, db=None) == OK


def test_refusals_of_the_embedding(L):
    f = caller(L.zc_embedding, table=A, tt=1, rows=100, cols=64, stride=64, tokens=B, bits=64, n=8, scale=1.0, out=D, ot=0, os=64, stream=None)
    for bad in (dict(table=None), dict(table=A + 1), dict(tt=3), dict(stride=63), dict(rows=(1 << 29) + 1), dict(cols=(1 << 23) + 1, stride=1 << 24, os=1 << 24), dict(tokens=None), dict(tokens=B + 4),
                dict(tokens=B + 2, bits=32), dict(bits=16), dict(n=1 << 31), dict(scale=NAN), dict(scale=INF), dict(scale=-1e39), dict(out=None), dict(out=D + 2), dict(ot=8), dict(os=63)):
        assert f(**bad) == ARG, bad
    assert f(n=0) == OK and f(cols=0, stride=0, os=0) == OK
    g = caller(L.zc_embedding_backward, dy=A, dyt=1, dys=64, tokens=B, bits=32, n=8, scale=1.0, grad=D, gt=0, rows=100, cols=64, stride=64, flags=1, ws=E, bytes=1 << 20, stream=None)
    for bad in (dict(dy=None), dict(dy=A + 1), dict(dyt=3), dict(dys=63), dict(tokens=None), dict(tokens=B + 2), dict(bits=8), dict(n=1 << 31), dict(scale=-INF), dict(scale=1e300), dict(grad=None), dict(grad=D + 2),
                dict(gt=3), dict(rows=(1 << 29) + 1), dict(stride=1), dict(flags=2), dict(ws=None), dict(ws=E + 4), dict(bytes=100)):
        assert g(**bad) == ARG, bad
    assert g(n=0) == OK and g(rows=0) == OK and g(cols=0, dys=0, stride=0) == OK


def test_refusals_of_the_step_for_matrices(L):
    f = caller(L.zc_muon, k=1, rows=words(16), cols=words(20), params=words(A), pt=0, grads=words(B), gt=1, copies=None, ct=0, state=D, bytes=4 * 320, lr=0.1, mu=0.9, wd=0.0, n=5, flags=1,
               scale=None, ws=0x100000, wsb=1 << 20, stream=None)
    for bad in (dict(k=-1), dict(rows=None), dict(cols=None), dict(params=None), dict(grads=None), dict(pt=3), dict(gt=-1), dict(copies=words(A), ct=4), dict(copies=words(A + 1), ct=1), dict(params=words(0)),
                dict(grads=words(0)), dict(params=words(A + 2)), dict(grads=words(B + 1)), dict(state=None), dict(state=D + 8), dict(bytes=4 * 320 - 1), dict(lr=-1.0), dict(lr=NAN), dict(lr=INF), dict(mu=1.0),
                dict(mu=-0.1), dict(mu=NAN), dict(wd=-1.0), dict(wd=INF), dict(n=0), dict(n=101), dict(flags=8), dict(scale=D + 2), dict(ws=None), dict(ws=0x100080), dict(wsb=4096), dict(rows=words((1 << 20) + 1))):
        assert f(**bad) == ARG, bad
    twice = dict(k=2, rows=words(16, 8), cols=words(20, 5), grads=words(B, B), bytes=8 * 320)
    for bad in (dict(params=words(A, A)), dict(params=words(A, D), copies=words(E, E)), dict(params=words(A, D), copies=words(D, 0)), dict(params=words(A, D), copies=words(0, A)),
                dict(params=words(A, D), copies=words(A, 0))):
        assert f(**twice, **bad) == ARG, bad
    assert f(k=0) == OK and f(rows=words(0), params=words(0), grads=words(0), state=None, bytes=0, ws=None, wsb=0) == OK


def test_tensors_that_are_not_on_the_gpu_are_refused_by_either_way(monkeypatch):
    x, v, t, ws = torch.zeros(4, 64), torch.zeros(64), torch.zeros(4, dtype=torch.int64), torch.zeros(1 << 16, dtype=torch.uint8)
    for _ in range(2):
        assert zc.zc_layer_norm(x, v, v, x) == ARG and zc.zc_layer_norm(x, None, None, x) == ARG
        assert zc.zc_layer_norm_backward(x, x, torch.zeros(2, 4), v, x, v, v, ws) == ARG
        assert zc.zc_embedding(x, t, x) == ARG
        assert zc.zc_embedding_backward(x, t, x, ws) == ARG
        assert zc.zc_muon([x], [x], ws, ws, 0.1) == ARG
        monkeypatch.setattr(b, "_native_layers", None)


def test_native_calls_leave_what_is_not_plain():
    b.lib()
    if b._native_layers is None:
        pytest.skip("the native calls are not built")
    calls = [C.cast(f, C.c_void_p).value for f in (b.lib().zc_layer_norm, b.lib().zc_layer_norm_backward, b.lib().zc_embedding, b.lib().zc_embedding_backward, b.lib().zc_muon)]
    assert b._native_layers.setup_training(*calls) is None
    with pytest.raises(ValueError):
        b._native_layers.setup_training(*calls[:4], 0)
    with pytest.raises(TypeError):
        b._native_layers.setup_training(*calls[:4])
    b._native_layers.setup_training(*calls)
    for name, count in (("layer_norm", 7), ("layer_norm_backward", 11), ("embedding", 5), ("embedding_backward", 7), ("muon", 12)):
        assert getattr(b._native_layers, name)(*[None] * count) is NotImplemented and getattr(b._native_layers, name)() is NotImplemented


def test_requests_end_with_the_last_tile(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "muon_ask_host")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", os.path.join(root, "tests", "host", "muon_ask_host.cpp"), "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout
