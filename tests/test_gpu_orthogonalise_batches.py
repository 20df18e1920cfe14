"""Batches of updates whose tiles are chosen by how full they are: skinny ones,
sides just past a tile's, and ones that keep the larger tiles, against 64 bits."""
import pytest
import torch

from tests import learn_util as U
from tests.test_gpu_orthogonalise import _check, _gauss

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def learn():
    from paper_2204_02585_amd import learn
    return learn


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.float16], ids=str)
@pytest.mark.parametrize("batch,m,n", [(130, 5, 300), (70, 300, 1), (40, 130, 300), (64, 129, 129), (70, 200, 300), (51, 390, 257)])
def test_batches(learn, batch, m, n, dtype):
    """The whole batch against one matrix at a time, and some against 64 bits."""
    g = _gauss(batch + m, batch, m, n)
    some = [0, batch // 2, batch - 1]
    _check(learn, g[some], dtype)
    got = learn.orthogonalise(g, dtype=dtype)
    for k in some:
        want = U.newton_schulz(g[k], 5, learn.MUON, 1e-7)
        off = (got[k].double().cpu() - torch.from_numpy(want)).norm() / float((want * want).sum()) ** 0.5
        assert off <= 2 * 4 * 5 * (2.0 ** -12 if dtype == torch.bfloat16 else 2.0 ** -23) + U.UNIT[dtype] + 2e-6
    assert torch.equal(got, learn.orthogonalise(g, dtype=dtype))
