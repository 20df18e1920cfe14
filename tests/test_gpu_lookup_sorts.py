"""The sorts behind the table's gradient against 64 bits: radix passes of 2 to
10 bits with counts around their steps."""
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
