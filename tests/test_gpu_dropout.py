"""Dropout against its plain form (tests/layer_util.py).  The mask is exact, and
so is a binary32 product with the binary32 share, which differs from the plain
form's by half a step; the sum with the residual is rounded once more, and the
result to its type."""
import numpy as np
import pytest
import torch

from tests import layer_util as U

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def draw(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def check(y, x, p, seed, residual=None):
    cols = x.shape[-1]
    v = U.double(x).reshape(-1, cols)
    want = U.share(*v.shape, p, seed) * v
    off = 4 * U.F32 * np.abs(want)
    if residual is not None:
        want = want + U.double(residual).reshape(-1, cols)
        off = off + 2 * U.F32 * np.abs(want)
    U.assert_within(y.reshape(-1, cols), want, off + U.half_step(np.abs(want) + off, x.dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (5, 8), (3, 9), (64, 64), (257, 33), (1000, 250), (2, 4099), (70000, 3)])
def test_values(dtype, rows, cols):
    from paper_2204_02585_amd import learn
    x, r = draw((rows, cols), dtype, 1), draw((rows, cols), dtype, 2)
    for p, seed in ((0.1, 3), (0.5, -1), (0.999, 1 << 63)):
        check(learn.dropout(x, p, seed=seed), x, p, seed)
        check(learn.dropout(x, p, seed=seed, residual=r), x, p, seed, r)


@pytest.mark.parametrize("dtype", TYPES)
def test_ends_of_p(dtype):
    """p = 0 leaves every value, a NaN too; p = 1 leaves none, an infinity neither;
    what is dropped is 0 whatever it was."""
    from paper_2204_02585_amd import learn
    x = draw((40, 24), dtype, 4)
    x[3], x[5] = float("nan"), float("inf")
    assert torch.equal(learn.dropout(x, 0.0, seed=1), x) or torch.equal(learn.dropout(x, 0.0, seed=1).view(torch.uint8), x.view(torch.uint8))
    assert torch.equal(learn.dropout(x, 1.0, seed=1), torch.zeros_like(x))
    y = learn.dropout(x, 0.5, seed=8)
    drop = torch.from_numpy(U.share(40, 24, 0.5, 8) == 0).cuda()
    assert (y[drop] == 0).all() and drop[3].any() and drop[5].any()
    assert y[3][~drop[3]].isnan().all() and (y[5][~drop[5]] == float("inf")).all()
    # a share below the words' resolution drops nothing
    assert torch.equal(learn.dropout(x[:3], 1e-12, seed=1), x[:3])


@pytest.mark.parametrize("dtype", TYPES)
def test_layouts(dtype):
    """Slices, broadcast rows, more dimensions, memory off its 16-byte boundaries,
    results in place; what lies around them stays as it was."""
    from paper_2204_02585_amd import learn
    big = draw((50, 91), dtype, 6)
    x = big[3:40, 5:66]
    check(learn.dropout(x, 0.3, seed=2), x, 0.3, 2)
    check(learn.dropout(big.t(), 0.3, seed=2), big.t(), 0.3, 2)
    row = big[:1].expand(30, 91)
    check(learn.dropout(row, 0.3, seed=2, residual=big[:30]), row, 0.3, 2, big[:30])
    cube = draw((4, 5, 6, 7), dtype, 7)
    check(learn.dropout(cube, 0.3, seed=2), cube, 0.3, 2)
    line = draw((1001,), dtype, 8)
    check(learn.dropout(line[1:], 0.3, seed=2), line[1:], 0.3, 2)
    out = torch.full((60, 70), 7.0, dtype=dtype, device="cuda")
    learn.dropout(x, 0.3, seed=2, out=out[2:39, 4:65])
    check(out[2:39, 4:65], x, 0.3, 2)
    out[2:39, 4:65] = 7.0
    assert (out == 7.0).all()
    for name in ("x", "residual"):
        a, b = x.clone(), x.flip(0).contiguous()
        want = learn.dropout(a, 0.3, seed=2, residual=b)
        assert torch.equal(learn.dropout(a, 0.3, seed=2, residual=b, out=a if name == "x" else b), want)


def test_empty():
    from paper_2204_02585_amd import learn
    for shape in ((0, 5), (5, 0), (2, 0, 3)):
        assert learn.dropout(torch.zeros(shape, device="cuda"), 0.5).shape == shape


def test_gradients():
    """The gradient has the forward call's mask, the residual's is the gradient
    itself; differences along a direction say the same, for the map is linear;
    twice differentiated too."""
    from paper_2204_02585_amd import learn
    x, r, g = (draw((37, 19), torch.float32, k).requires_grad_(k < 2) for k in (0, 1, 2))
    y = learn.dropout(x, 0.4, seed=11, residual=r)
    gx, gr = torch.autograd.grad(y, (x, r), g, retain_graph=True)
    check(gx, g, 0.4, 11)
    assert torch.equal(gr, g)
    along = draw((37, 19), torch.float32, 5)
    difference = (learn.dropout(x.detach() + along, 0.4, seed=11) - learn.dropout(x.detach(), 0.4, seed=11)).double()
    # each element's difference of two values below 8, times 1 / 0.6, has lost some steps of them
    assert torch.allclose((difference * g.double()).sum(), (gx.double() * along.double()).sum(), rtol=0, atol=37 * 19 * 8 * 16 * U.F32)
    gy = draw((37, 19), torch.float32, 6).requires_grad_()
    (first,) = torch.autograd.grad(y, x, gy, create_graph=True)
    (second,) = torch.autograd.grad(first, gy, along)
    check(second, along, 0.4, 11)


def test_forward_mode():
    from torch.autograd import forward_ad
    from paper_2204_02585_amd import learn
    x, t, r, u = (draw((9, 14), torch.float32, k) for k in range(4))
    with forward_ad.dual_level():
        y = learn.dropout(forward_ad.make_dual(x, t), 0.3, seed=5, residual=forward_ad.make_dual(r, u))
        value, tangent = forward_ad.unpack_dual(y)
        check(value, x, 0.3, 5, r)
        check(tangent, t, 0.3, 5, u)
        only = forward_ad.unpack_dual(learn.dropout(x, 0.3, seed=5, residual=forward_ad.make_dual(r, u))).tangent
        assert torch.equal(only, u)
        with pytest.raises(RuntimeError, match="forward-mode"):
            learn.dropout(forward_ad.make_dual(x, t), 0.3, out=torch.empty_like(x))


def test_step():
    """A step on the device is added to the seed; changed before the backward
    pass, it is refused."""
    from paper_2204_02585_amd import learn
    x = draw((30, 22), torch.float32, 1).requires_grad_()
    step = torch.tensor([41], device="cuda")
    y = learn.dropout(x, 0.5, seed=1, step=step)
    check(y, x, 0.5, 42)
    (g,) = torch.autograd.grad(y, x, torch.ones_like(y), retain_graph=True)
    check(g, torch.ones_like(x), 0.5, 42)
    step.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y, x, torch.ones_like(y))
    check(learn.dropout(x.detach(), 0.5, seed=1, step=step), x, 0.5, 43)
    check(learn.dropout(x.detach(), 0.5, seed=-1, step=torch.tensor([-7], device="cuda")), x, 0.5, -8)


def test_another_stream():
    from paper_2204_02585_amd import learn
    x = draw((300, 500), torch.float32, 1)
    side = torch.cuda.Stream()
    y = learn.dropout(x * 2, 0.5, seed=1, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check(y, x * 2, 0.5, 1)


def test_refusals():
    from paper_2204_02585_amd import learn
    x = torch.zeros((4, 6), device="cuda")
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(ValueError, match="p must"):
            learn.dropout(x, p)
    with pytest.raises(ValueError, match="CUDA"):
        learn.dropout(x.cpu(), 0.5)
    with pytest.raises(TypeError, match="float32, float16 or bfloat16"):
        learn.dropout(x.double(), 0.5)
    with pytest.raises(ValueError, match="residual"):
        learn.dropout(x, 0.5, residual=x[:1])
    with pytest.raises(ValueError, match="residual"):
        learn.dropout(x, 0.5, residual=x.half())
    with pytest.raises(ValueError, match="CUDA"):
        learn.dropout(x, 0.5, residual=x.cpu())
    with pytest.raises(ValueError, match="out must"):
        learn.dropout(x, 0.5, out=torch.empty((4, 5), device="cuda"))
    with pytest.raises(ValueError, match="step"):
        learn.dropout(x, 0.5, step=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="step"):
        learn.dropout(x, 0.5, step=torch.zeros(1, device="cuda"))
    with pytest.raises(ValueError, match="CUDA"):
        learn.dropout(x, 0.5, step=torch.zeros(1, dtype=torch.int64))
    with pytest.raises(ValueError, match="dimension"):
        learn.dropout(x[0, 0], 0.5)
