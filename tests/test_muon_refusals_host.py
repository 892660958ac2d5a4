"""CPU test: the step for matrices refuses factors that binary32, in which it works, does not hold.  Addresses are never used: what is not refused fails for want of a GPU."""
import pytest
import torch

from paper_2502_18554_amd import binding as b
from test_training_host import A, ARG, B, D, L, OK, caller, words          # noqa: F401

STEP = dict(k=1, rows=words(16), cols=words(20), params=words(A), pt=0, grads=words(B), gt=1, copies=None, ct=0, state=D, bytes=4 * 320, lr=0.1, mu=0.9, wd=0.0, n=5, flags=1,
            scale=None, ws=0x100000, wsb=1 << 20, stream=None)


@pytest.mark.parametrize("bad", [dict(lr=1e39), dict(lr=1e300), dict(lr=2e38, rows=words(20), cols=words(4)), dict(lr=2e38, flags=2, cols=words(100), bytes=4 * 1600), dict(wd=1e300), dict(wd=4e39),
                                 dict(lr=1e30, wd=1e10), dict(lr=1e300, wd=1e300), dict(mu=1 - 1e-9), dict(mu=1 - 2.0 ** -26)])
def test_factors_that_binary32_does_not_hold(L, bad):
    assert caller(L.zc_muon, **STEP)(**bad) == ARG


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are of nothing")
@pytest.mark.parametrize("good", [dict(), dict(lr=3e38), dict(lr=0.0, wd=1e300), dict(lr=1e-300, wd=1e300), dict(mu=1 - 2.0 ** -24), dict(mu=0.0)])
def test_factors_that_it_holds_are_not_refused(L, good):
    assert caller(L.zc_muon, **STEP)(**good) not in (OK, ARG)


def test_results_that_overlap(L):
    """Launches take many matrices together, so that of two results in one place one would be lost: also where they only reach into each other, or into the momentum."""
    f = caller(L.zc_muon, **STEP)
    two = dict(k=2, rows=words(16, 8), cols=words(20, 5), grads=words(B, B), bytes=4 * (320 + 64))
    size = 16 * 20 * 4                       # of the first matrix; of the second 160
    for bad in (dict(params=words(A, A + size - 4)), dict(params=words(A, A + 4)), dict(params=words(A + 156, A)), dict(params=words(A, D + 4)), dict(params=words(D - 4, A)), dict(params=words(D + 4 * 383, A)),
                dict(params=words(A, A + size), copies=words(0, A + size - 2), ct=1), dict(params=words(A, A + size), copies=words(A + size + 158, 0), ct=1),
                dict(params=words(A, A + size), copies=words(D, 0), ct=1)):
        assert f(**two, **bad) == ARG, bad
    many = 3000
    assert f(k=many, rows=words(*[4] * many), cols=words(*[4] * many), params=words(*[A + 64 * (i * 7 % many) for i in range(many - 1)], A + 40), grads=words(*[B] * many), state=1 << 30,
             bytes=128 * many) == ARG


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are of nothing")
def test_results_side_by_side_are_not_refused(L):
    f = caller(L.zc_muon, **STEP)
    size = 16 * 20 * 4
    two = dict(k=2, rows=words(16, 8), cols=words(20, 5), grads=words(B, B), bytes=4 * (320 + 64))
    for good in (dict(params=words(A, A + size)), dict(params=words(A + 160, A)), dict(params=words(D - size, D + 4 * 384)), dict(params=words(A, A + size), copies=words(A + size + 160, 0), ct=1),
                 dict(params=words(A, A + size), grads=words(A, A + size))):
        assert f(**{**two, **good}) not in (OK, ARG), good
    assert f(k=2, rows=words(16, 0), cols=words(20, 5), params=words(A, A), grads=words(B, B)) not in (OK, ARG)
