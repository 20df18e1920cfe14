"""Rows of a table by index and the table's gradient against 64 bits: types,
index types, row lengths around the 16-byte runs, strides, indices outside
the table, and numbers of indices around the sort's steps."""
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


def _ids(seed, rows, shape, dtype=torch.int64, outside=0.1):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, rows, shape, generator=g)
    marks = torch.tensor([-1, rows, -(1 << 31), (1 << 31) - 1])[torch.randint(0, 4, shape, generator=g)]
    return torch.where(torch.rand(shape, generator=g) < outside, marks, ids).to(dtype).cuda()


def _plain_lookup(table, ids, scale):
    t, i = table.cpu(), ids.cpu().long()
    ok = (i >= 0) & (i < t.shape[0])
    rows = t[torch.where(ok, i, torch.zeros_like(i))].float() * np.float32(scale)
    return torch.where(ok.unsqueeze(-1), rows, torch.zeros_like(rows)).to(t.dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("cols", [1, 3, 4, 7, 8, 9, 24, 25, 129, 1030])
def test_lookup_is_exact(learn, dtype, cols):
    """One product in binary32 and one rounding: every bit is fixed."""
    for k, (shape, ids_dtype, scale) in enumerate([((1,), torch.int64, 1.0), ((0,), torch.int64, 1.0), ((), torch.int32, 2.0),
                                                   ((3, 67), torch.int32, 0.3), ((1291,), torch.int64, 45.25)]):
        table, ids = _randn(k, 77, cols, dtype=dtype), _ids(k, 77, shape, ids_dtype)
        got = learn.lookup(table, ids, scale=scale)
        assert got.shape == (*shape, cols) and got.dtype == dtype
        assert torch.equal(got.cpu(), _plain_lookup(table, ids, scale))


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_lookup_strides_and_special_values(learn, dtype):
    """Rows inside a wider table, at an odd element, a transposed table, a table
    of one row for all, output rows apart; infinities and NaN stay in their
    rows."""
    wide = _randn(1, 60, 50, dtype=dtype)
    wide[7, 11], wide[8, 12], wide[9, 13] = float("inf"), float("-inf"), float("nan")
    ids = _ids(2, 60, (500,))
    for table in (wide[:, 3:40], wide[::2, 1:10], wide.t(), wide[:1].expand(60, 50), wide[:, 5:6]):
        got = learn.lookup(table, ids, scale=0.5)
        torch.testing.assert_close(got.cpu(), _plain_lookup(table, ids, 0.5), rtol=0, atol=0, equal_nan=True)
    big = torch.full((500, 70), 7.0, dtype=dtype, device="cuda")
    out = big[:, 9:59]
    assert learn.lookup(wide, ids, out=out) is out
    torch.testing.assert_close(out.cpu(), _plain_lookup(wide, ids, 1.0), rtol=0, atol=0, equal_nan=True)
    assert bool((big[:, :9] == 7).all()) and bool((big[:, 59:] == 7).all())


def test_lookup_past_32_bit_offsets(learn):
    """A table of more than 2^32 bytes, and one of more than 2^31 elements."""
    rows, cols = (1 << 21) + 5, 1030
    table = torch.zeros((rows, cols), dtype=torch.float16, device="cuda")
    ids = torch.tensor([rows - 1, 0, 1 << 20, rows - 2], device="cuda")
    want = _randn(3, 4, cols, dtype=torch.float16)
    table[ids] = want
    assert torch.equal(learn.lookup(table, ids), want)


def _check_gradient(learn, grad, ids, rows, scale=1.0, dtype=torch.float32, old=None):
    """A sum of c terms in binary32, whatever their order, is within c units of
    the sum of magnitudes; the scale and the sum with the old value round
    once more each, then the result to its type."""
    kind = {} if old is None else dict(out=old.clone(), accumulate=True)
    got = learn.lookup_gradient(grad, ids, rows, scale=scale, dtype=dtype, **kind)
    assert got.shape == (rows, grad.shape[-1]) and got.dtype == dtype
    again = learn.lookup_gradient(grad, ids, rows, scale=scale, dtype=dtype,
                                  **({} if old is None else dict(out=old.clone(), accumulate=True)))
    assert torch.equal(got, again), "the order of the sums changed"
    want, size, count = U.gradient(grad, ids, rows, scale)
    if old is not None:
        want, size = want + old.double().cpu().numpy(), size + old.double().abs().cpu().numpy()
    room = (count + 2) * 2.0 ** -24 * size + U.rounding(want, dtype) * (1 + 2.0 ** -10)
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= room).all(), f"{(off - room).max()} past the bound"
    return got


@pytest.mark.parametrize("rows", [1, 2, 255, 256, 257, 65535, 70001])
@pytest.mark.parametrize("count", [1, 31, 32, 33, 64, 65, 4095, 4097, 20000])
def test_gradient_around_the_sort(learn, rows, count):
    """Keys of one to three digits (the mark of outside indices is `rows`
    itself), and counts around tiles and steps."""
    _check_gradient(learn, _randn(count, count, 8), _ids(rows, rows, (count,), torch.int32), rows, scale=0.25)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("out", DTYPES, ids=str)
@pytest.mark.parametrize("cols", [1, 3, 7, 8, 9, 25, 300, 1111])
def test_gradient_types_and_lengths(learn, dtype, out, cols):
    ids = _ids(cols, 90, (11, 53))
    _check_gradient(learn, _randn(5, 11, 53, cols, dtype=dtype), ids, 90, scale=3.0, dtype=out)
    old = _randn(6, 90, cols, dtype=out)
    got = _check_gradient(learn, _randn(5, 11, 53, cols, dtype=dtype), ids % 40, 90, dtype=out, old=old)
    assert torch.equal(got[40:], old[40:])       # rows without an index stay


@pytest.mark.parametrize("cols", [5, 24, 700])
def test_gradient_of_hot_rows(learn, cols):
    """Runs that cross many tiles, end on a tile's edge, or begin on one."""
    parts = [torch.full((n,), v) for v, n in ((3, 3000), (9, 32), (10, 32), (11, 33), (12, 31), (40, 64), (41, 1), (77, 95))]
    ids = torch.cat(parts)
    ids = ids[torch.randperm(len(ids), generator=torch.Generator().manual_seed(1))].cuda()
    _check_gradient(learn, _randn(7, len(ids), cols), ids, 100)
    _check_gradient(learn, _randn(8, 4100, cols, dtype=torch.bfloat16), torch.zeros(4100, dtype=torch.int64).cuda(), 1)


def test_gradient_of_many_indices(learn):
    """More than one step of keys in a workgroup's stretch (above 2^20 indices)."""
    ids = _ids(4, 50021, (1_300_003,), torch.int32)
    ids[::7] = 17
    _check_gradient(learn, _randn(9, 1_300_003, 4, dtype=torch.float16), ids, 50021)


@pytest.mark.parametrize("count", [300, 900, 3000, 8000, 20000, 60000])
@pytest.mark.parametrize("rows,first,some", [(300_000, 5000, 3000), (300_000, 299_000, 1000), (70_001, 1536, 512), (1 << 25, 1 << 24, 1 << 15),
                                             (1 << 24, 1 << 23, 1 << 15)])
def test_gradient_of_rows_close_together(learn, rows, first, some, count):
    """All indices in one bucket of the sort, in one or two passes, in LDS and past
    what it holds; marks of outside indices beside them."""
    ids = first + _ids(count, some, (count,), torch.int64, outside=0.0)
    ids[::9] = -1
    ids[1::9] = rows
    cols = 2 if rows > 1 << 20 else 12
    _check_gradient(learn, _randn(count, count, cols), ids, rows, scale=0.5)


def test_gradient_of_long_stretches(learn):
    """Stretches of 2^16 keys, all of one digit in the first ones: a count that
    16 bits do not hold."""
    count = 7 * 128 * 8192 + 5
    ids = _ids(4, 1500, (count,), torch.int32)
    ids[:200_000] = 3
    _check_gradient(learn, _randn(9, count, 2, dtype=torch.float16), ids, 1500)


def test_gradient_empty_and_outside(learn):
    """No indices, or none inside: zeros, or what was there."""
    for ids in (torch.zeros((0,), dtype=torch.int64), torch.full((100,), -1), torch.full((33,), 50)):
        grad = torch.full((len(ids), 13), float("nan"), device="cuda")
        got = learn.lookup_gradient(grad, ids.cuda(), 50)
        assert torch.equal(got, torch.zeros((50, 13), device="cuda"))
        old = _randn(1, 50, 13)
        assert torch.equal(learn.lookup_gradient(grad, ids.cuda(), 50, out=old.clone(), accumulate=True), old)


def test_gradient_layouts(learn):
    """A gradient spread by broadcasting (strides of zero), transposed, within a
    wider one; an output with rows apart, whose gaps stay."""
    ids = _ids(3, 30, (200,))
    wide = _randn(2, 200, 64)
    for grad in (wide[:, 5:20], wide[:1, :15].expand(200, 15), wide[:, :1].expand(200, 15),
                 torch.ones((), device="cuda").expand(200, 15), wide[:15, :].t()[:, :15].repeat(4, 1)[:200]):
        _check_gradient(learn, grad, ids, 30)
    for cols in (3, 15, 32):
        for dtype in (torch.float32, torch.bfloat16):
            big = torch.full((30, 40), 7.0, device="cuda", dtype=dtype)
            learn.lookup_gradient(wide[:, :cols], ids, 30, out=big[:, 5:5 + cols])
            assert torch.equal(big[:, 5:5 + cols], learn.lookup_gradient(wide[:, :cols], ids, 30, dtype=dtype))
            assert bool((big[:, :5] == 7).all()) and bool((big[:, 5 + cols:] == 7).all())


def test_gradient_keeps_special_values_in_their_rows(learn):
    ids = torch.arange(40, device="cuda") % 10
    grad = _randn(1, 40, 16)
    grad[3, 5], grad[14, 6], grad[24, 6], grad[5, 0] = float("nan"), float("inf"), float("-inf"), float("inf")
    got = learn.lookup_gradient(grad, ids, 10)
    bad = torch.zeros((10, 16), dtype=torch.bool)
    bad[3, 5] = bad[4, 6] = bad[5, 0] = True
    assert torch.equal(torch.isfinite(got).cpu(), ~bad)
    assert torch.isnan(got[3, 5]) and torch.isnan(got[4, 6]) and got[5, 0] == float("inf")


def test_autograd_against_differences(learn):
    """The loss is linear in the table, so its differences are the gradient up
    to their rounding: values of 2^-8 steps and a step of 1/4 make them exact."""
    g = torch.Generator().manual_seed(5)
    table = (torch.randint(-256, 256, (20, 9), generator=g) / 256.0).cuda()
    ids = _ids(6, 20, (4, 31))
    weight = (torch.randint(-256, 256, (4, 31, 9), generator=g) / 256.0).cuda()
    leaf = table.clone().requires_grad_()
    (learn.lookup(leaf, ids, scale=0.5) * weight).sum().backward()

    def loss(t):
        return float((learn.lookup(t, ids, scale=0.5).double() * weight.double()).sum())

    for v, c in ((0, 0), (7, 3), (19, 8), (11, 5)):
        up, down = table.clone(), table.clone()
        up[v, c] += 0.25
        down[v, c] -= 0.25
        assert (loss(up) - loss(down)) / 0.5 == float(leaf.grad[v, c])
    leaf.grad = None
    learn.lookup(leaf, ids).sum().backward()      # a gradient of strides zero
    count = torch.bincount(ids[(ids >= 0) & (ids < 20)], minlength=20).float()
    assert torch.equal(leaf.grad, count.unsqueeze(1).expand(20, 9))


def test_on_another_stream(learn):
    """The given stream waits for the current one's work, and the caller can
    order itself after it."""
    side = torch.cuda.Stream()
    table = _randn(1, 5000, 256)
    ids = _ids(2, 5000, (60000,), torch.int32)
    want = learn.lookup(table, ids, scale=2.0)
    grad = learn.lookup_gradient(want, ids, 5000)
    for _ in range(3):
        fresh = table * 1.0
        out = learn.lookup(fresh, ids, scale=2.0, stream=side)
        back = learn.lookup_gradient(out, ids, 5000, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want) and torch.equal(back, grad)


def test_refusals(learn):
    table, ids = _randn(1, 10, 6), torch.arange(4, device="cuda")
    grad = _randn(2, 4, 6)
    with pytest.raises(TypeError):
        learn.lookup(table.double(), ids)
    with pytest.raises(TypeError):
        learn.lookup(table, ids.float())
    with pytest.raises(ValueError):
        learn.lookup(table[0], ids)
    with pytest.raises(ValueError):
        learn.lookup(table, ids.cpu())
    with pytest.raises(ValueError):
        learn.lookup(table.cpu(), ids)
    with pytest.raises(ValueError):
        learn.lookup(table, ids, out=torch.empty((4, 7), device="cuda"))
    with pytest.raises(ValueError):
        learn.lookup(table, ids, out=torch.empty((6, 4), device="cuda").t())
    with pytest.raises(ValueError):
        learn.lookup_gradient(grad, ids[:3], 10)
    with pytest.raises(ValueError):
        learn.lookup_gradient(grad, ids, 10, accumulate=True)
    with pytest.raises(ValueError):
        learn.lookup_gradient(grad, ids, 10, out=torch.empty((9, 6), device="cuda"))
    from paper_2204_02585_amd import binding
    with pytest.raises(binding.SqnError, match="invalid"):
        learn.lookup_gradient(grad, ids, 0)
