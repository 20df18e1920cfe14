"""Updates orthogonalised by Newton-Schulz products against 64 bits."""
import numpy as np
import pytest
import torch

from tests import learn_util as U

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.float16, torch.bfloat16]

# Most that a result may be off, as a 2-norm of it.  Factors of 11 bits are off
# by 2^-12 and those of 22 bits by 2^-23 at most, relative; a step rounds X
# twice (as a factor of A and of B X), A and B once each, over 5 steps; a
# rounding's effect on the result is taken as at most twice its own size (the
# slope of a step is 3.45 where singular values are small, and below 1 where
# they end).  Sums in binary32 add far less.  Then the result's rounding.
def _room(dtype, steps=5):
    factor = 2.0 ** -12 if dtype == torch.bfloat16 else 2.0 ** -23
    return 2 * 4 * steps * factor + U.UNIT[dtype] + 2e-6


@pytest.fixture(scope="module")
def learn():
    from paper_2204_02585_amd import learn
    return learn


def _gauss(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def _check(learn, g, dtype, steps=5, coefficients=None, eps=1e-7, out=None):
    coefficients = coefficients or learn.MUON
    got = learn.orthogonalise(g, steps=steps, coefficients=coefficients, eps=eps, dtype=dtype, out=out)
    assert got.shape == g.shape and got.dtype == dtype
    every = zip(g, got) if g.dim() == 3 else [(g, got)]
    for k, (x, y) in enumerate(every):
        want = U.newton_schulz(x, steps, coefficients, eps)
        off = np.linalg.norm(y.double().cpu().numpy() - want)
        assert off <= _room(dtype, steps) * np.linalg.norm(want), (k, off / np.linalg.norm(want))
    return got


@pytest.mark.parametrize("m,n", [(1, 1), (1, 9), (9, 1), (5, 3), (16, 16), (31, 33), (64, 64), (63, 129), (65, 64), (128, 128),
                                 (130, 127), (50, 256), (256, 42), (200, 77), (128, 257), (129, 300), (256, 256), (300, 700)])
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_sizes(learn, m, n, dtype):
    _check(learn, _gauss(m + n, m, n), dtype)


@pytest.mark.parametrize("m,n", [(700, 1100), (1025, 513), (1024, 2048)])
def test_large(learn, m, n):
    _check(learn, _gauss(m, m, n, dtype=torch.bfloat16), torch.bfloat16)
    _check(learn, _gauss(m, m, n), torch.float32)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_input_types_and_batches(learn, dtype):
    _check(learn, _gauss(1, 7, 40, 60, dtype=dtype), torch.bfloat16)
    _check(learn, _gauss(2, 3, 140, 60, dtype=dtype), torch.float32)


def test_low_rank(learn):
    """Singular values that one rounding of X to 11 bits would bury: at 1024 the
    noise's are 1/100 of the largest, and end as near 1 as those."""
    g = _gauss(1, 1024, 8) @ _gauss(2, 8, 1024) + 0.02 * _gauss(3, 1024, 1024)
    _check(learn, g, torch.bfloat16)
    _check(learn, g, torch.float32)


def test_layouts(learn):
    """Transposed, strided and broadcast updates, a view of a larger tensor, and
    the transposed update's result the transposed result."""
    g = _gauss(4, 90, 150)
    want = _check(learn, g, torch.bfloat16)
    assert torch.equal(learn.orthogonalise(g.t()), want.t())
    wide = _gauss(5, 4, 100, 200)
    _check(learn, wide[:, 3:80:2, 5:190:3], torch.bfloat16)
    _check(learn, wide.transpose(0, 2)[:30], torch.bfloat16)
    same = learn.orthogonalise(g.unsqueeze(0).expand(3, 90, 150))
    assert all(torch.equal(same[k], want) for k in range(3))
    big = torch.full((2, 100, 170), 7.0, device="cuda", dtype=torch.float32)
    out = big[:, 4:94, 11:161]
    assert _check(learn, torch.stack((g, -g)), torch.float32, out=out) is out
    keep = torch.ones_like(big, dtype=torch.bool)
    keep[:, 4:94, 11:161] = False
    assert bool((big[keep] == 7).all())
    turned = torch.empty((150, 90), device="cuda", dtype=torch.bfloat16).t()
    assert torch.equal(learn.orthogonalise(g, out=turned), want)


def test_in_place(learn):
    g = _gauss(6, 3, 70, 90, dtype=torch.bfloat16)
    want = learn.orthogonalise(g)
    learn.orthogonalise(g, out=g)
    assert torch.equal(g, want)


@pytest.mark.parametrize("shape", [(2, 40, 40), (2, 300, 200)])
def test_zero_nan_and_the_range_of_magnitudes(learn, shape):
    """A zero matrix stays zero, also for eps = 0; a NaN or an infinity spreads
    over its own matrix only; tiny and huge updates keep their directions."""
    for dtype in (torch.bfloat16, torch.float32):
        g = torch.zeros((5, *shape[1:]), device="cuda")
        g[1], g[2], g[3] = _gauss(1, *shape[1:]), _gauss(2, *shape[1:]), _gauss(3, *shape[1:])
        g[2, 5, 7], g[3, 39, 0] = float("nan"), float("-inf")
        g[4] = g[1]
        for eps in (0.0, 1e-7):
            got = learn.orthogonalise(g, eps=eps, dtype=dtype)
            assert bool((got[0] == 0).all())
            assert bool(torch.isnan(got[2]).all()) and bool(torch.isnan(got[3]).all())
            assert torch.equal(got[1], got[4]) and bool(torch.isfinite(got[1]).all())
        for size in (1e-30, 1e30):
            _check(learn, size * _gauss(4, *shape), dtype, eps=0.0)


@pytest.mark.parametrize("steps", [0, 1, 2, 9])
def test_steps_and_other_coefficients(learn, steps):
    """The cubic step ends at 1 for every singular value, so many steps give an
    orthogonal matrix."""
    g = _gauss(7, 60, 100)
    for dtype in (torch.bfloat16, torch.float32):
        _check(learn, g, dtype, steps=steps)
        _check(learn, g, dtype, steps=steps, coefficients=(1.5, -0.5, 0.0))
    x = learn.orthogonalise(g, steps=30, coefficients=(1.5, -0.5, 0.0), dtype=torch.float32).double()
    assert float((x @ x.t() - torch.eye(60, device="cuda")).abs().max()) < 1e-5


def test_the_same_bits_again(learn):
    g = _gauss(8, 2, 257, 300)
    for dtype in DTYPES:
        assert torch.equal(learn.orthogonalise(g, dtype=dtype), learn.orthogonalise(g, dtype=dtype))


def test_on_another_stream(learn):
    side = torch.cuda.Stream()
    g = _gauss(9, 500, 600)
    want = learn.orthogonalise(g)
    for _ in range(3):
        out = learn.orthogonalise(g * 1.0, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want)


def test_empty_batch(learn):
    assert learn.orthogonalise(torch.empty((0, 4, 5), device="cuda")).shape == (0, 4, 5)


def test_refusals(learn):
    from paper_2204_02585_amd import binding
    g = _gauss(1, 8, 8)
    for bad in (dict(coefficients=(4.0, 0.0, 0.0)), dict(coefficients=(3.0, -30.0, 30.0)),
                dict(coefficients=(float("nan"), 0.0, 0.0)), dict(steps=-1), dict(steps=65), dict(eps=-1.0),
                dict(eps=float("inf"))):
        with pytest.raises(binding.SqnError, match="invalid"):
            learn.orthogonalise(g, **bad)
    with pytest.raises(binding.SqnError, match="one place"):
        learn.orthogonalise(g, out=torch.empty((1, 8), device="cuda", dtype=torch.bfloat16).expand(8, 8))
    with pytest.raises(TypeError):
        learn.orthogonalise(g.double())
    with pytest.raises(TypeError):
        learn.orthogonalise(g, dtype=torch.float64)
    with pytest.raises(ValueError):
        learn.orthogonalise(g[0])
    with pytest.raises(ValueError):
        learn.orthogonalise(g.cpu())
    with pytest.raises(ValueError):
        learn.orthogonalise(g, out=torch.empty((8, 9), device="cuda"))
    with pytest.raises(ValueError):
        learn.orthogonalise(g, coefficients=(1.0, 2.0))
