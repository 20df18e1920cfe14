"""4-bit blocks: every code and scale, the values they stand for, and products
on them, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

from tests import learn_util as U

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def learn():
    from paper_2204_02585_amd import learn
    return learn


def _randn(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def _check_blocks(learn, x):
    q = learn.quantise(x)
    codes, scales, values = U.quantise(x)
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    bad = np.repeat(scales == 255, 16, axis=1)
    assert np.array_equal(q.codes.cpu().numpy()[~bad], codes[~bad])
    for dtype in DTYPES:
        want = torch.from_numpy(values).to(dtype)
        got = q.values(dtype).cpu()
        torch.testing.assert_close(got, want, rtol=0, atol=0, equal_nan=True)
    return q


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
def test_every_16_bit_number(learn, dtype):
    """Each number as the largest of its block and beside every larger power of
    two within the elements' range: ties, both zeros, subnormals, infinities
    and NaN."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
    _check_blocks(learn, every.view(-1, 1).cuda())
    beside = torch.zeros((65536, 64), dtype=dtype)
    for k in range(8):
        beside[:, 8 * k + k] = every
        top = torch.ldexp(torch.exp2(torch.floor(torch.log2(every.float().abs().clamp(min=1e-30)))), torch.tensor(k % 4))
        beside[:, 8 * k + 7 - (k == 7)] = top.to(dtype) if k < 7 else every
    _check_blocks(learn, beside.cuda())


def test_ties_and_limits(learn):
    x = torch.zeros((9, 32))
    x[0, :15] = torch.tensor([0.25, -0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.99, -0.0, -5.0, -7.5, 4.0])
    x[1] = 2.0 ** -149
    x[2] = 3.4e38
    x[3, 31] = 2.0 ** -126
    x[4, 3], x[4, 4] = 2.0 ** -125, 1e-40
    x[5, :2] = torch.tensor([float(np.nextafter(np.float32(4), np.float32(0))), 1.0])
    x[6, :3] = torch.tensor([2.0 ** 127, 2.0 ** 100, -2.0 ** 125])
    x[7, 0] = float("inf")
    x[8, 9] = float("nan")
    _check_blocks(learn, x.cuda())


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("cols", [1, 7, 8, 9, 31, 32, 33, 40, 63, 100, 256, 1000])
def test_blocks_of_ragged_rows(learn, dtype, cols):
    """Rows that end inside a block, strided and transposed inputs, no rows."""
    wide = _randn(cols, 37, cols + 11, dtype=dtype) * torch.exp(3 * _randn(1, 37, 1)).to(dtype)
    _check_blocks(learn, wide[:, :cols].contiguous())
    _check_blocks(learn, wide[:, 3:3 + cols])
    _check_blocks(learn, wide[:, :cols].contiguous().t())
    assert learn.quantise(wide[:0, :cols]).shape == (0, cols)
    assert learn.quantise(wide[:0, :cols]).values().shape == (0, cols)
    out = torch.full((37, cols + 5), 7.0, device="cuda", dtype=dtype)
    q = learn.quantise(wide[:, :cols])
    q.values(dtype, out=out[:, 2:2 + cols])
    assert torch.equal(out[:, 2:2 + cols], q.values(dtype))
    assert bool((out[:, :2] == 7).all()) and bool((out[:, 2 + cols:] == 7).all())


def _layer(x, w, bias, relu):
    """(x w^T + bias) from values in float64, and the sum of magnitudes."""
    y, size = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        b = bias.double().cpu().numpy()
        y, size = y + b, size + np.abs(b)
    return np.maximum(y, 0.0) if relu else y, size


def _check_product(learn, x, w, bias, relu, dtype):
    """K products of 4-bit numbers are exact; their sum in binary32, in any order,
    is within K + 1 units of the sum of magnitudes."""
    qw = learn.quantise(w)
    xv, wv = U.quantise(x)[2], U.quantise(w)[2]
    want, size = _layer(xv, wv, bias, relu)
    room = (x.shape[1] + 1) * 2.0 ** -24 * size + U.rounding(want, dtype) * (1 + 2.0 ** -10)
    for arg in (x, learn.quantise(x)):
        got = learn.product(arg, qw, bias=bias, relu=relu, dtype=dtype)
        assert got.shape == want.shape and got.dtype == dtype
        got64, rounded = got.double().cpu().numpy(), U.infinite(want, dtype)
        with np.errstate(invalid="ignore"):
            off = np.where(got64 == rounded, 0.0, np.abs(got64 - want))
        assert (off <= room).all(), (off - room).max()
        assert torch.equal(got, learn.product(arg, qw, bias=bias, relu=relu, dtype=dtype))


@pytest.mark.parametrize("points", [1, 2, 3, 15, 16, 17, 33, 64, 65, 200])
@pytest.mark.parametrize("units", [1, 15, 16, 17, 64, 100, 257])
def test_product_sizes(learn, points, units):
    for k, cols in enumerate([1, 31, 32, 33, 96, 128, 130, 256, 500, 1024]):
        x, w = _randn(k, points, cols, dtype=torch.float16), _randn(k + 50, units, cols)
        bias = _randn(k + 99, units) if k % 2 else None
        _check_product(learn, x, w, bias, k % 3 == 0, DTYPES[k % 3])


@pytest.mark.parametrize("points,units,cols", [(300, 513, 257), (129, 1025, 2080), (1000, 256, 256), (1, 4096, 4096),
                                               (5, 1000, 8192), (700, 700, 4096), (2048, 1300, 640)])
def test_larger_products(learn, points, units, cols):
    for k, dtype in enumerate(DTYPES):
        x = _randn(1, points, cols, dtype=dtype) * torch.exp(_randn(2, points, 1)).to(dtype)
        w = _randn(3, units, cols) * torch.exp(2 * _randn(4, 1, cols))
        _check_product(learn, x, w, _randn(5, units), k == 0, dtype)


@pytest.mark.parametrize("points,units,cols", [(1, 8192, 300), (16, 8215, 1000), (4, 16384, 513), (9, 16431, 70), (2, 17000, 32)])
def test_few_points_by_many_units(learn, points, units, cols):
    """Workgroups of 32 and 64 units, the last ones not full, and fewer waves than
    groups of units."""
    for k, dtype in enumerate(DTYPES):
        _check_product(learn, _randn(1, points, cols, dtype=dtype), _randn(3, units, cols), _randn(5, units), k == 1, dtype)


def test_product_scales_reach_far(learn):
    """Scales from the smallest to the largest that the sums can hold, in one
    product: the scale of every block is the one that is applied."""
    x, w = _randn(1, 40, 320), _randn(2, 48, 320)
    for b in range(10):
        x[:, 32 * b:32 * b + 32] *= 2.0 ** (12 * b - 60)
        w[:, 32 * b:32 * b + 32] *= 2.0 ** (60 - 12 * b)
    x[3] = 0.0
    w[5] = 0.0
    x[7] *= 2.0 ** -60
    _check_product(learn, x, w, None, False, torch.float32)


def test_product_keeps_nan_in_its_rows(learn):
    """A marked block makes its point's or unit's outputs NaN and no others, with
    the activation too."""
    x, w = _randn(1, 30, 200), _randn(2, 50, 200)
    clean = learn.product(x, learn.quantise(w), relu=True)
    x[4, 199], w[9, 3] = float("nan"), float("inf")
    for arg in (x, learn.quantise(x)):
        got = learn.product(arg, learn.quantise(w), relu=True)
        bad = torch.zeros((30, 50), dtype=torch.bool, device="cuda")
        bad[4], bad[:, 9] = True, True
        assert torch.equal(torch.isnan(got), bad)
        assert torch.equal(got[~bad], clean[~bad])


def test_product_layouts(learn):
    """Leading axes, strided and broadcast inputs, output rows apart, no points."""
    w = learn.quantise(_randn(1, 70, 90))
    x = _randn(2, 3, 5, 120)
    want = learn.product(x[..., :90].contiguous().view(15, 90), w)
    assert torch.equal(learn.product(x[..., :90], w), want.view(3, 5, 70))
    row = x[0, 0, :90]
    assert torch.equal(learn.product(row, w), want[0])
    assert torch.equal(learn.product(row.expand(20, 90), w), want[:1].expand(20, 70))
    big = torch.full((15, 100), 7.0, device="cuda")
    learn.product(x.view(15, 120)[:, :90], w, out=big[:, 13:83])
    assert torch.equal(big[:, 13:83], want) and bool((big[:, :13] == 7).all()) and bool((big[:, 83:] == 7).all())
    assert learn.product(x[:0, ..., :90], w).shape == (0, 5, 70)


def test_on_another_stream(learn):
    side = torch.cuda.Stream()
    x, w = _randn(1, 3000, 512, dtype=torch.float16), _randn(2, 512, 512)
    want = learn.product(x, learn.quantise(w))
    for _ in range(3):
        got = learn.product(x * 1.0, learn.quantise(w * 1.0, stream=side), stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)


def test_refusals(learn):
    x = _randn(1, 4, 40)
    q = learn.quantise(x)
    with pytest.raises(ValueError):
        learn.quantise(x[0])
    with pytest.raises(TypeError):
        learn.quantise(x.double())
    with pytest.raises(ValueError):
        learn.quantise(x.cpu())
    with pytest.raises(ValueError):
        learn.Quantised(q.codes, q.scales, 70)
    with pytest.raises(ValueError):
        learn.Quantised(q.codes, q.scales[:3], 40)
    with pytest.raises(ValueError):
        learn.Quantised(q.codes.to(torch.int8), q.scales, 40)
    with pytest.raises(ValueError):
        learn.Quantised(q.codes.cpu(), q.scales.cpu(), 40)
    with pytest.raises(TypeError):
        q.values(torch.float64)
    with pytest.raises(TypeError):
        learn.product(x, x)
    with pytest.raises(ValueError):
        learn.product(_randn(2, 4, 41), q)
    with pytest.raises(ValueError):
        learn.product(x, q, bias=torch.zeros(5, device="cuda"))
    with pytest.raises(ValueError):
        learn.product(x, q, bias=torch.zeros(4, device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError):
        learn.product(x, q, out=torch.empty((4, 5), device="cuda"))
    with pytest.raises(ValueError):
        learn.product(x.cpu(), q)
