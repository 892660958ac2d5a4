"""The layer calls' way from tensors to the library: by native code and by ctypes alike, the same refusals and the same results."""
import pytest
import torch

import paper_2502_18554_amd as zc
from paper_2502_18554_amd import binding as b
from paper_2502_18554_amd.binding import ZC_ERR_ARG, ZC_OK

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(params=["native", "ctypes"])
def way(request, monkeypatch):
    b.lib()
    if request.param == "ctypes":
        monkeypatch.setattr(b, "_native_layers", None)
    elif b._native_layers is None:
        pytest.skip("the native calls are not built")
    return request.param


def room(rows, cols, fill=0):
    return (torch.full((rows, zc.zc_mx_codes_stride(cols)), fill, dtype=torch.uint8, device=DEV),
            torch.full((rows, zc.zc_mx_scales_stride(cols)), fill, dtype=torch.uint8, device=DEV))


def in_pieces(nbytes):
    """Tensors that say they have so many bytes: every second one of a buffer's, one byte, or one row, again and again, and a buffer across."""
    wide = torch.zeros(2 * nbytes, dtype=torch.uint8, device=DEV)
    return [wide[::2], wide[:1].expand(nbytes), wide[:16].expand(-(-nbytes // 16), 16), wide.view(2, nbytes).t()]


@pytest.mark.parametrize("bits", [32, 8])
def test_states_in_pieces_are_refused(way, bits):
    p, g = torch.ones(100, device=DEV), torch.ones(100, device=DEV)
    for state in in_pieces(zc.zc_adamw_state_bytes([100], bits)):
        assert state.nbytes >= zc.zc_adamw_state_bytes([100], bits) and not state.is_contiguous()
        assert zc.zc_adamw([p], [g], state, 1, 1e-3, state_bits=bits) == ZC_ERR_ARG
    torch.cuda.synchronize()
    assert (p == 1).all()


@pytest.mark.parametrize("m", [4, 40])
def test_workspaces_in_pieces_are_refused(way, m):
    n, k = 48, 200
    x, w, a = torch.ones(m, k, device=DEV), room(n, k, 0x22), room(m, k, 0x22)
    out = torch.full((m, n), 5.0, device=DEV)
    for ws in in_pieces(zc.zc_mx_workspace_bytes(m, n, k)):
        assert zc.zc_mx_linear(x, *w, out, ws) == ZC_ERR_ARG
        assert zc.zc_mx_product(*a, *w, k, out, ws) == ZC_ERR_ARG
    torch.cuda.synchronize()
    assert (out == 5).all()
    assert zc.zc_mx_linear(x, *w, out, torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)) == ZC_OK


def test_codes_and_scales_that_are_no_matrices_are_refused(way):
    m, n, k = 8, 16, 64
    x, a, w, out = torch.zeros(m, k, device=DEV), room(m, k), room(n, k), torch.zeros(m, n, device=DEV)
    ws = torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    for i in range(2):
        for change in (lambda t: t[0], lambda t: t[None], lambda t: t.view(-1), lambda t: t[0, 0]):
            flat, flat_w = list(a), list(w)
            flat[i], flat_w[i] = change(a[i]), change(w[i])
            assert zc.zc_mx_quantize(x, *flat) == ZC_ERR_ARG
            assert zc.zc_mx_quantize(x, None, None, *flat) == ZC_ERR_ARG
            assert zc.zc_mx_dequantize(*flat, x) == ZC_ERR_ARG
            assert zc.zc_mx_product(*flat, *w, k, out, ws) == ZC_ERR_ARG
            assert zc.zc_mx_product(*a, *flat_w, k, out, ws) == ZC_ERR_ARG
            assert zc.zc_mx_linear(x, *flat_w, out, ws) == ZC_ERR_ARG


def results(kind):
    """What every call makes of the same tensors: in pieces of wider ones, with and without what may be left out, on a stream of its own too."""
    m, n, k, dtype = 9, 33, 170, {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]
    gen = torch.Generator().manual_seed(5)
    random = lambda *shape: torch.randn(shape, generator=gen).to(dtype).to(DEV)
    side, out = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for stream in (None, side):
        x, w = random(m, k + 3)[:, 1:k + 1], random(n, k)
        a, a_t, b, alone, alone_t = room(m, k, 1), room(k, m, 2), room(n, k, 3), room(m, k, 4), room(k, m, 5)
        ws = torch.zeros(zc.zc_mx_workspace_bytes(m, n, k) + 16, dtype=torch.uint8, device=DEV)
        bias, back = torch.randn(n, generator=gen).to(DEV), torch.full((m, k + 5), 9.0, dtype=dtype, device=DEV)
        torch.cuda.synchronize()
        for status in (zc.zc_mx_quantize(x, *a, *a_t, stream=stream), zc.zc_mx_quantize(w, *b, stream=stream), zc.zc_mx_quantize(x, *alone, stream=stream),
                       zc.zc_mx_quantize(x, None, None, *alone_t, stream=stream), zc.zc_mx_dequantize(*a, back[:, 2:k + 2], stream=stream)):
            assert status == ZC_OK
        out += [*a, *a_t, *b, *alone, *alone_t, back]
        for rows in (m, 1):
            for more in (dict(), dict(d_bias=bias), dict(add=True), dict(d_bias=bias, add=True)):
                y, z = (torch.full((rows, n + 2), 0.5, dtype=dtype, device=DEV) for _ in range(2))
                torch.cuda.synchronize()
                assert zc.zc_mx_linear(x[:rows], *b, y[:, 1:n + 1], ws, stream=stream, **more) == ZC_OK
                assert zc.zc_mx_product(a[0][:rows], a[1][:rows], *b, k, z[:, :n], ws, stream=stream, **more) == ZC_OK
                out += [y, z]
        for bits in (32, 8):
            for copies, scale in ((None, None), ([torch.zeros(n * k, device=DEV), torch.zeros(m, device=DEV)], torch.full((1,), 0.5, device=DEV))):
                p, g = [random(n, k), random(m)], [random(n, k), random(m)]
                state = torch.zeros(zc.zc_adamw_state_bytes([n * k, m], bits), dtype=torch.uint8, device=DEV)
                torch.cuda.synchronize()
                for step in (1, 2):
                    assert zc.zc_adamw(p, g, state, step, 1e-2, 0.8, 0.95, 1e-6, 0.3, state_bits=bits, seed=11, d_copies=copies, d_grad_scale=scale, stream=stream) == ZC_OK
                out += [*p, state, *(copies or ())]
        torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_both_ways_are_alike(monkeypatch, kind):
    b.lib()
    if b._native_layers is None:
        pytest.skip("the native calls are not built")
    answers = []

    class Listening:
        def __getattr__(self, name):
            def listen(*args):
                answers.append(getattr(native, name)(*args))
                return answers[-1]
            return listen

    native = b._native_layers
    monkeypatch.setattr(b, "_native_layers", Listening())
    one = results(kind)
    assert answers and all(a == ZC_OK for a in answers)                  # (the native calls took all of them)
    monkeypatch.setattr(b, "_native_layers", None)
    other = results(kind)
    assert len(one) == len(other) and all(torch.equal(s, t) for s, t in zip(one, other))


@pytest.mark.parametrize("m", [4, 40])
def test_products_need_no_workspace(way, m):
    n, k = 48, 200
    a, w, one, other = room(m, k, 0x22), room(n, k, 0x31), torch.empty(m, n, device=DEV), torch.empty(m, n, device=DEV)
    assert zc.zc_mx_product(*a, *w, k, one, torch.empty(zc.zc_mx_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)) == ZC_OK
    assert zc.zc_mx_product(*a, *w, k, other, None) == ZC_OK
    assert torch.equal(one, other)
