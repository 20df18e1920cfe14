"""Derivatives of the operators on learned tables and layers that take other
ways than a table's gradient: forward mode, forward over reverse, and refusals
where a derivative would be lost."""
import pytest
import torch
from torch.autograd import forward_ad

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def learn():
    from paper_2204_02585_amd import learn
    return learn


def _randn(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


IDS = torch.tensor([[3, 3, -1], [0, 9, 8]])


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("reverse_too", [False, True])
def test_lookup_in_forward_mode(learn, dtype, reverse_too):
    """The lookup is linear: its tangent is the tangent's lookup, every bit."""
    table, way, ids = _randn(1, 9, 5, dtype=dtype), _randn(2, 9, 5, dtype=dtype), IDS.cuda()
    with forward_ad.dual_level():
        leaf = table.clone().requires_grad_(reverse_too)
        got = forward_ad.unpack_dual(learn.lookup(forward_ad.make_dual(leaf, way), ids, scale=0.3))
        assert got.tangent is not None and got.tangent.dtype == dtype
        assert torch.equal(got.primal, learn.lookup(table, ids, scale=0.3))
        assert torch.equal(got.tangent, learn.lookup(way, ids, scale=0.3))
        plain = learn.lookup(table, ids)
        assert forward_ad.unpack_dual(plain).tangent is None


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16], ids=str)
def test_lookup_gradient_in_forward_mode(learn, out):
    grad, way, ids = _randn(1, 2, 3, 5), _randn(2, 2, 3, 5), IDS.cuda()
    with forward_ad.dual_level():
        got = forward_ad.unpack_dual(learn.lookup_gradient(forward_ad.make_dual(grad, way), ids, 9, scale=0.3, dtype=out))
        assert got.tangent is not None
        assert torch.equal(got.primal, learn.lookup_gradient(grad, ids, 9, scale=0.3, dtype=out))
        assert torch.equal(got.tangent, learn.lookup_gradient(way, ids, 9, scale=0.3, dtype=out))


def test_forward_over_reverse(learn):
    """The product of a Hessian and a direction: of sum (rows w)^3 it is, at a row
    of the table, the sum over its lookups of 6 w^3 row way."""
    ids = torch.tensor([2, 0, 2, 5, -1], device="cuda")
    table, way, w = _randn(1, 6, 4), _randn(2, 6, 4), _randn(3, 5, 4)
    with forward_ad.dual_level():
        leaf = table.clone().requires_grad_()
        loss = ((learn.lookup(forward_ad.make_dual(leaf, way), ids) * w) ** 3).sum()
        (grad,) = torch.autograd.grad(loss, leaf)
        got = forward_ad.unpack_dual(grad)
        assert got.tangent is not None
        primal, tangent = got.primal.double(), got.tangent.double()
    first, second = torch.zeros(6, 4, dtype=torch.float64), torch.zeros(6, 4, dtype=torch.float64)
    t, d, w64 = table.double().cpu(), way.double().cpu(), w.double().cpu()
    for k, v in enumerate(ids.tolist()):
        if v >= 0:
            first[v] += 3 * w64[k] ** 3 * t[v] ** 2
            second[v] += 6 * w64[k] ** 3 * t[v] * d[v]
    # at most ten roundings of binary32, of sums of two terms below 200 each
    torch.testing.assert_close(primal.cpu(), first, rtol=0, atol=10 * 400 * 2.0 ** -24)
    torch.testing.assert_close(tangent.cpu(), second, rtol=0, atol=10 * 400 * 2.0 ** -24)


def test_lost_tangents_are_refused(learn):
    """Where an operator has no forward-mode derivative it says so."""
    x, ids = _randn(1, 6, 40), torch.arange(6, device="cuda")
    w = learn.quantise(_randn(2, 7, 40))
    bias = _randn(3, 7)
    side = torch.cuda.Stream()
    with forward_ad.dual_level():
        dual, dual_bias = forward_ad.make_dual(x, torch.ones_like(x)), forward_ad.make_dual(bias, torch.ones_like(bias))
        for call in (lambda: learn.lookup(dual, ids, out=torch.empty_like(x)), lambda: learn.lookup(dual, ids, stream=side),
                     lambda: learn.lookup_gradient(dual, ids, 6, out=torch.empty_like(x)),
                     lambda: learn.lookup_gradient(dual, ids, 6, stream=side),
                     lambda: learn.orthogonalise(dual), lambda: learn.product(dual, w), lambda: learn.product(x, w, bias=dual_bias)):
            with pytest.raises(RuntimeError, match="forward-mode"):
                call()
        # tensors without a tangent are taken as outside of a level
        assert learn.product(x, w, bias=bias).shape == (6, 7)
        assert learn.orthogonalise(x).shape == (6, 40)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_backward_of_a_table_without_rows(learn, dtype):
    """Its lookup gives zeros for every index, and its gradient has no rows either."""
    table = torch.empty((0, 7), dtype=dtype, device="cuda", requires_grad=True)
    rows = learn.lookup(table, IDS.cuda())
    assert torch.equal(rows, torch.zeros((2, 3, 7), dtype=dtype, device="cuda"))
    rows.sum().backward()
    assert table.grad.shape == (0, 7) and table.grad.dtype == dtype
