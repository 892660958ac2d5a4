"""The optimiser's step where second moments are subnormal or zero in binary32, and where eps is: state bit by bit, weights against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2502_18554_amd as zc
from paper_2502_18554_amd.binding import ZC_OK

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F = np.float32
U = 2.0 ** -24
BETA1, BETA2, LR = 0.9, 0.999, 0.125


def moments(m, v, g):
    """The definition's own roundings, one operation of binary32 after the other."""
    return m * F(BETA1) + g * F(1 - BETA1), v * F(BETA2) + (g * F(1 - BETA2)) * g


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-40, 2.0 ** -126, 1e-30, 1e-20, 1e-8, 1.0, 2.0 ** 100, 1e38], ids=str)
def test_steps_of_small_gradients(bits, eps):
    """Gradients of 2^-20 to 2^-72, whose squares are normal, subnormal (from 2^-58 down) and zero (from 2^-71 down), in whole blocks of 32 of about one magnitude."""
    n = 53 * 32
    rng = np.random.default_rng(1)
    exponents = np.repeat(np.arange(-20, -73, -1), 32)
    if eps == 0:
        exponents = np.maximum(exponents, -68)                           # (no second moment that is zero: 0.001 x 2^-136 is two quanta of binary32 and more)
    state = torch.zeros(zc.zc_adamw_state_bytes([n], bits), dtype=torch.uint8, device=DEV)
    p = torch.zeros(n, device=DEV)
    m, v = np.zeros(n, F), np.zeros(n, F)
    for step in (1, 2, 3):
        g = (np.ldexp(rng.uniform(1, 2, n), exponents) * rng.choice([-1.0, 1.0], n)).astype(F)
        m, v = moments(m, v, g)
        p.zero_()                                                        # what is left is the step itself
        assert zc.zc_adamw([p], [torch.from_numpy(g).to(DEV)], state, step, LR, BETA1, BETA2, eps, 0.0, state_bits=bits) == ZC_OK
        # Roundings of half a unit: the constants root, eps and rate, product and sum of the denominator, the two products behind the reciprocal; of a whole
        # one: root and reciprocal.  Ten halves, and a bit for their products.
        d = np.sqrt(v.astype(np.float64)) / np.sqrt(1 - BETA2 ** step) + float(F(eps))
        want = -(LR / (1 - BETA1 ** step)) * m.astype(np.float64) / d
        got = p.double().cpu().numpy()
        beyond = np.abs(want) >= 2.0 ** 127
        assert (np.abs(got - want) <= 11 * U * np.abs(want) + 2.0 ** -148)[~beyond].all(), np.abs(got / want - 1)[~beyond].max()
        assert (np.sign(got) == np.sign(want))[np.abs(want) > 2.0 ** -147].all()
        if bits == 8:
            break                                                        # (the state is rounded further: from zeros only)
        held = state.view(torch.float32).cpu().numpy()
        assert np.array_equal(held[:n], m) and np.array_equal(held[n:], v)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [2.0 ** 60, 2.0 ** 95, 2.0 ** 96, 2.0 ** 100, 2.0 ** 126, 3e38], ids=str)
def test_steps_under_a_large_eps(bits, eps):
    """Denominators whose reciprocal is subnormal in binary32, under gradients that still make a step of it."""
    n = 21 * 32
    rng = np.random.default_rng(2)
    g = (np.ldexp(rng.uniform(1, 2, n), np.repeat(np.arange(40, 61), 32)) * rng.choice([-1.0, 1.0], n)).astype(F)
    state = torch.zeros(zc.zc_adamw_state_bytes([n], bits), dtype=torch.uint8, device=DEV)
    p = torch.zeros(n, device=DEV)
    m, v = moments(np.zeros(n, F), np.zeros(n, F), g)
    assert zc.zc_adamw([p], [torch.from_numpy(g).to(DEV)], state, 1, LR, BETA1, BETA2, eps, 0.0, state_bits=bits) == ZC_OK
    want = -(LR / (1 - BETA1)) * m.astype(np.float64) / (np.sqrt(v.astype(np.float64)) / np.sqrt(1 - BETA2) + float(F(eps)))
    assert (np.abs(p.double().cpu().numpy() - want) <= 11 * U * np.abs(want) + 2.0 ** -148).all()
