"""The sorts behind the table's gradient against 64 bits: radix passes of 2 to
10 bits with counts around their steps, and buckets of rows with indices that
crowd: a row that takes most of them, rows close together, rows at a stride,
several such rows in one bucket."""
import math

import pytest
import torch

from tests.test_gpu_lookup import _check_gradient, _ids, _randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def learn():
    from paper_2204_02585_amd import learn
    return learn


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _crowd(seed, rows, count, share, hot):
    """Even indices, of which a share falls on the rows of `hot` instead; marks among them."""
    ids = torch.randint(0, rows, (count,), generator=_gen(seed))
    often = torch.tensor(hot)[torch.randint(0, len(hot), (count,), generator=_gen(seed + 1))]
    ids = torch.where(torch.rand(count, generator=_gen(seed + 2)) < share, often, ids)
    ids[::101], ids[1::101] = -1, rows
    return ids.cuda()


@pytest.mark.parametrize("rows", [1, 2, 3, 8, 700, 1023])
@pytest.mark.parametrize("count", [40961, 49151, 49152, 49153, 1048577])
def test_one_radix_pass(learn, rows, count):
    """One digit of 2 to 10 bits (the mark of outside indices is `rows`), counts
    around steps of 8192 keys and a second step of a stretch."""
    _check_gradient(learn, _randn(count, count, 4), _ids(rows, rows, (count,), torch.int32), rows, scale=0.5)


@pytest.mark.parametrize("rows", [1, 3, 8])
@pytest.mark.parametrize("count", [4096, 4097, 8191, 8192, 8193])
def test_few_rows(learn, rows, count):
    """Around the count from which few rows leave their buckets."""
    _check_gradient(learn, _randn(count, count, 9), _ids(rows, rows, (count,)), rows)


@pytest.mark.parametrize("rows", [(1 << 19) - 1, 600_000, (1 << 20) - 1, 1 << 20])
@pytest.mark.parametrize("hot", [0.0, 0.7])
def test_wide_digits(learn, rows, hot):
    """Two digits of 9 + 10 and 10 + 10 bits, three from 2^20 rows on, with rows
    that take most of the indices."""
    ids = _crowd(rows, rows, 130_003, hot, [5, rows - 1, rows // 2])
    _check_gradient(learn, _randn(3, 130_003, 2, dtype=torch.float16), ids, rows)


@pytest.mark.parametrize("rows,count", [(300, 20_000), (30_000, 5_000), (30_000, 20_000), (50_000, 81_000), (1 << 20, 20_000),
                                        (1 << 20, 122_000), (1 << 24, 60_000)])
@pytest.mark.parametrize("share", [0.3, 0.6, 0.9, 1.0])
def test_a_row_that_takes_most(learn, rows, count, share):
    """Its entries go ahead of its bucket's others, in their order."""
    cols = 2 if rows > 1 << 20 else 8
    _check_gradient(learn, _randn(count, count, cols), _crowd(count, rows, count, share, [rows // 3]), rows, scale=2.0)


@pytest.mark.parametrize("rows,count", [(5_000, 40_000), (50_000, 16_384), (50_000, 80_000), (1 << 20, 120_000)])
def test_rows_in_the_order_of_their_frequency(learn, rows, count):
    u = torch.rand(count, generator=_gen(count), dtype=torch.float64)
    ids = (torch.exp(u * math.log(rows + 1.0)) - 1.0).long().clamp_(0, rows - 1).cuda()
    _check_gradient(learn, _randn(1, count, 8), ids, rows)


@pytest.mark.parametrize("stride", [2, 64, 128, 512, 1024])
def test_rows_at_a_stride(learn, stride):
    """A column of texels, or every other row."""
    rows = 1 << 20
    ids = torch.randint(0, rows // stride, (50_000,), generator=_gen(stride)) * stride + 1
    _check_gradient(learn, _randn(2, 50_000, 4), ids.cuda(), rows)


@pytest.mark.parametrize("rows,high,count", [(40_000, 7, 30_000), (60_000, 7, 81_000), (1 << 20, 7, 60_000), (1 << 24, 9, 120_000)])
def test_several_crowded_rows_of_a_bucket(learn, rows, high, count):
    """More than LDS holds without the most frequent one: through global memory,
    in one and in two passes over the bits of the row in its bucket."""
    top = (rows - 1) >> high
    places = [0, 1, top // 3, top // 2, top - 1]
    hot = [r << high | (((77 - (r >> high)) ^ r) & ((1 << high) - 1)) for r in places]
    assert max(hot) < rows
    cols = 2 if rows > 1 << 20 else 8
    for share, some in ((0.95, hot), (0.95, hot[:2]), (1.0, hot)):
        _check_gradient(learn, _randn(count, count, cols), _crowd(count, rows, count, share, some), rows)
