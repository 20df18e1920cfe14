"""How near bfloat16 results of the orthogonalised updates come: a model of their
binary16 factors on the CPU, the bound that follows from it, and the kernels
against that bound.

The products take factors of 11 bits with the diagonals of A and of a + b A + c A A
kept apart.  Their error is then 4.5e-4 to 8.2e-4 of the result's norm (the model,
Gaussian updates with sides of 128 to 2048), beside the result's own rounding of
1.66e-3; with the diagonals left in the factors it is 1.4e-3 to 1.9e-3.  The bound
lies between: the rounding of the exact result and 1.15e-3 of its norm, as two
errors that do not know each other."""
import numpy as np
import pytest
import torch

from tests import learn_util as U

FACTORS = 1.15e-3
MUON = (3.4445, -4.7750, 2.0315)


def _to_bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def _allowed(want):
    return np.hypot(np.linalg.norm(_to_bf16(want) - want), FACTORS * np.linalg.norm(want))


def _half(x):
    return x.astype(np.float16).astype(np.float64)


def _model(g, apart):
    """Five steps with factors in binary16, sums exact, X in two binary16;
    `apart`: the diagonals are kept out of the factors."""
    a, b, c = (float(np.float32(k)) for k in MUON)
    x = g / np.linalg.norm(g)
    for _ in range(5):
        hi = _half(4096 * x) / 4096
        both = hi + _half(4096 * (x - hi)) / 4096
        p = hi @ hi.T
        if apart:
            d = np.diag(p).copy()
            o = _half(4096 * (p - np.diag(d))) / 4096
            square = o @ o
            middle = b * o + c * (square + (d[:, None] + d[None, :]) * o)
            middle = _half(2048 * (middle - np.diag(np.diag(middle)))) / 2048
            x = (a + b * d + c * (d * d + np.diag(square)))[:, None] * both + middle @ hi
        else:
            p = _half(4096 * p) / 4096
            x = a * both + (_half(2048 * (b * p + c * (p @ p))) / 2048) @ hi
    return _to_bf16(x)


@pytest.mark.parametrize("m,n", [(128, 128), (128, 256), (129, 300), (256, 256), (300, 700)])
def test_the_bound_tells_the_diagonals(m, n):
    g = np.random.default_rng(m + n).standard_normal((m, n))
    want = U.newton_schulz(torch.from_numpy(g), 5, MUON, 0.0)
    assert np.linalg.norm(_model(g, True) - want) <= _allowed(want)
    assert np.linalg.norm(_model(g, False) - want) > _allowed(want)


@pytest.mark.gpu
@pytest.mark.parametrize("batch,m,n", [(1, 128, 128), (2, 128, 256), (1, 129, 300), (15, 256, 256), (1, 300, 700), (1, 700, 1100),
                                       (30, 500, 520), (1, 2048, 1024), (12, 1024, 1100)])
def test_bfloat16_results(batch, m, n):
    """Every kernel: one workgroup a matrix, tiles of 64, 128 and 256, narrow ones."""
    from paper_2204_02585_amd import learn
    g = torch.randn(batch, m, n, generator=torch.Generator().manual_seed(m + n)).cuda()
    got = learn.orthogonalise(g)
    for k in sorted({0, batch - 1}):
        want = U.newton_schulz(g[k], 5, MUON, 1e-7)
        off, allowed = np.linalg.norm(got[k].double().cpu().numpy() - want), _allowed(want)
        assert off <= allowed, (k, off / np.linalg.norm(want), allowed / np.linalg.norm(want))


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(128, 128), (256, 256), (700, 1100)])
def test_full_factors_then_bfloat16(m, n):
    """A binary32 result is within 6.8e-6 (20 roundings of 22 bits, twice their size,
    and the sums); rounded to bfloat16 an element is off by at most its rounding and
    twice that."""
    from paper_2204_02585_amd import learn
    g = torch.randn(m, n, generator=torch.Generator().manual_seed(m)).cuda()
    want = U.newton_schulz(g, 5, MUON, 1e-7)
    got = learn.orthogonalise(g, dtype=torch.float32).to(torch.bfloat16).double().cpu().numpy()
    assert np.linalg.norm(got - want) <= np.linalg.norm(_to_bf16(want) - want) + 2 * 6.8e-6 * np.linalg.norm(want)
