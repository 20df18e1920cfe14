"""A layer's gradients against the formulas in 64 bits (tests/layer_util.py),
against differences, and through autograd."""
import numpy as np
import pytest
import torch

from tests import layer_util as U
from tests.test_gpu_layer import ACTS, SIZES, TYPES, draw, inputs

pytestmark = pytest.mark.gpu


def check(got, grad, x, w, pre=None, activation=None, dropout=0.0, seed=0, what=""):
    flat = [t.reshape(-1, t.shape[-1]) if t is not None else None for t in (grad, x, w, pre)]
    want = U.gradients(*flat, activation, dropout, seed)
    for g, (v, off), name in zip(got, want, ("dx", "dw", "db")):
        if g is not None:
            if name == "db" and g.dtype != torch.float32:
                off = off + U.half_step(np.abs(v) + off, g.dtype)
            U.assert_within(g.reshape(v.shape), v, off, (name, what))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES + [(5000, 24, 40), (3001, 130, 66)])
def test_values(dtype, size):
    from paper_2204_02585_amd import learn
    x, w, _, grad = inputs(*size, dtype)
    check(learn.layer_gradient(grad, x, w), grad, x, w)
    pre = draw(grad.shape, dtype, torch.Generator().manual_seed(9))
    activation = ACTS[1 + sum(size) % 3]
    check(learn.layer_gradient(grad, x, w, pre, activation, 0.3, 5), grad, x, w, pre, activation, 0.3, 5, activation)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("activation", ACTS)
def test_parts(dtype, activation):
    """Each gradient alone and together, grad of binary32, both types of the bias's
    gradient, with and without a mask: what is not wanted is None."""
    from paper_2204_02585_amd import learn
    x, w, _, grad = inputs(60, 48, 33, dtype)
    pre = None if activation is None else draw(grad.shape, dtype, torch.Generator().manual_seed(9))
    for g in (grad, grad.float() * 1.001):
        for p in (0.0, 0.5, 1.0):
            for wanted in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 0, 0)):
                got = learn.layer_gradient(g, x, w, pre, activation, p, 4, for_x=wanted[0], for_w=wanted[1], for_bias=wanted[2],
                                           bias_dtype=dtype if wanted[0] else torch.float32)
                assert [t is not None for t in got] == [bool(k) for k in wanted]
                check(got, g, x, w, pre, activation, p, 4, (g.dtype, p, wanted))


@pytest.mark.parametrize("dtype", TYPES)
def test_many_tiles(dtype):
    """Tiles of 128 and 256 of both products, ragged at every end."""
    from paper_2204_02585_amd import learn
    for size in ((2100, 1700, 330), (3700, 3900, 200), (200, 3900, 3700)):
        x, w, _, grad = inputs(*size, dtype)
        dx, dw, _ = learn.layer_gradient(grad, x, w, for_bias=False)
        for got, a, b in ((dx, grad, w.t()), (dw, grad.t(), x.t())):
            a, b = a.double(), b.double()
            want = a @ b.t()
            off = 2 * U.F32 * (a.shape[1] + 8) * (a.abs() @ b.abs().t())
            bound = off + U.UNIT[dtype] * (want.abs() + off) + U.UNIT[dtype] * U.TINY[dtype]
            assert ((got.double() - want).abs() <= bound).all(), size


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("points,cols,units", [(16384, 256, 64), (20001, 250, 50), (16385, 50, 256), (16400, 100, 128), (16390, 33, 130), (17000, 1, 1),
                                               (131071, 64, 64), (131072, 64, 64), (131103, 128, 100), (131073, 40, 256), (140000, 8, 8)])
def test_many_points(dtype, points, cols, units):
    """Narrow layers of many points."""
    from paper_2204_02585_amd import learn
    x, w, _, grad = inputs(points, cols, units, dtype)
    dx, dw, db = learn.layer_gradient(grad, x, w)
    for got, a, b in ((dx, grad, w.t()), (dw, grad.t(), x.t())):
        a, b = a.double(), b.double()
        want = a @ b.t()
        off = 2 * U.F32 * (a.shape[1] + 8) * (a.abs() @ b.abs().t())
        assert ((got.double() - want).abs() <= off + U.UNIT[dtype] * (want.abs() + off) + U.UNIT[dtype] * U.TINY[dtype]).all()
    total = grad.double()
    assert ((db.double() - total.sum(0)).abs() <= 2 * U.F32 * (points + 8) * total.abs().sum(0)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("points,cols,units,activation,p", [
    (32768, 256, 256, "relu", 0.1), (40001, 250, 50, "gelu", 0.5), (32800, 136, 128, "silu", 0.0), (33000, 256, 64, None, 0.25),
    (32769, 129, 33, "gelu", 0.0), (50001, 256, 8, "relu", 0.9), (32768, 200, 200, "silu", 1.0), (40000, 256, 50, None, 0.0)])
def test_many_points_with_slopes(dtype, points, cols, units, activation, p):
    """Narrow layers of many points whose slopes are taken on the way; with the
    gradient's or the kept values' rows off the boundaries, each wanted alone."""
    from paper_2204_02585_amd import learn
    x, w, _, grad = inputs(points, cols, units, dtype)
    pre = draw((points, units), dtype, torch.Generator().manual_seed(4)) if activation else None
    share = torch.from_numpy(U.share(points, units, p, 77)).cuda()
    keep, s = (share > 0).double(), float(share.max()) or 1.0
    dz, off = keep * grad.double(), torch.zeros((), dtype=torch.float64, device="cuda")
    if activation:
        z = pre.double()
        t = torch.sigmoid(z)
        slope = {"relu": lambda: (z > 0).double(), "silu": lambda: t * (1 + z * (1 - t)),
                 "gelu": lambda: torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5}[activation]()
        off = keep * grad.double().abs() * 32 * U.F32 * (1 + z.abs()) * (activation != "relu")
        dz = dz * slope
    half, tiny = U.UNIT[dtype], U.TINY[dtype]
    rounded = off + half * (dz.abs() + off).clamp(min=tiny)
    want = []
    for a, b, o in ((dz, w.t(), rounded), (dz.t(), x.t(), rounded.t())):
        b = b.double()
        v, size = a @ b.t(), a.abs() @ b.abs().t()
        far = s * (2 * U.F32 * (a.shape[1] + 8) * size + o @ b.abs().t()) + 4 * U.F32 * s * v.abs()
        want.append((s * v, far + half * (s * v.abs() + far).clamp(min=tiny)))
    db = s * dz.sum(0)
    want.append((db, s * ((off + torch.zeros_like(dz)).sum(0) + 2 * U.F32 * (points + 8) * dz.abs().sum(0)) + 4 * U.F32 * db.abs()))

    def check_all(g, z, **wanted):
        for got, (v, bound), name in zip(learn.layer_gradient(g, x, w, z, activation, p, 77, **wanted), want, ("dx", "dw", "db")):
            if got is not None:
                bad = ~((got.double() - v).abs() <= bound)
                assert not bad.any(), (name, wanted, int(bad.sum()), bad.nonzero()[0].tolist())

    check_all(grad, pre)
    check_all(grad.float(), pre)
    check_all(grad, pre, for_w=False)
    check_all(grad, pre, for_bias=False)
    big = torch.full((points, units + 5), float("nan"), dtype=dtype, device="cuda")
    part = big[:, 3:3 + units]
    part.copy_(grad)
    check_all(part, pre)
    if activation:
        part.copy_(pre)
        check_all(grad, part)


@pytest.mark.parametrize("dtype", TYPES)
def test_layouts(dtype):
    """Slices off the 16-byte boundaries with NaN around them, broadcast and
    transposed gradients, more dimensions."""
    from paper_2204_02585_amd import learn
    gen = torch.Generator().manual_seed(5)
    for (points, cols, units), (row, col) in (((70, 90, 41), (1, 3)), ((70, 96, 40), (2, 8)), ((3, 130, 24), (1, 1)), ((150, 64, 128), (0, 16))):
        def inside(rows, columns):
            big = torch.full((rows + 3, columns + 24), float("nan"), dtype=dtype, device="cuda")
            part = big[row:row + rows, col:col + columns]
            part.copy_(draw((rows, columns), dtype, gen))
            return part
        x, w, grad, pre = inside(points, cols), inside(units, cols), inside(points, units), inside(points, units)
        check(learn.layer_gradient(grad, x, w), grad, x, w, what=(points, cols, units))
        check(learn.layer_gradient(grad, x, w, pre, "silu"), grad, x, w, pre, "silu", what=(points, cols, units))
    x, w, _, grad = inputs(30, 32, 24, dtype)
    one = grad[:1, :1].expand(30, 24)
    check(learn.layer_gradient(one, x, w), one, x, w)
    across = draw((24, 30), dtype, gen).t()
    check(learn.layer_gradient(across, x, w), across, x, w)
    cube, grads = draw((2, 3, 4, 32), dtype, gen), draw((2, 3, 4, 24), dtype, gen)
    got = learn.layer_gradient(grads, cube, w)
    assert got[0].shape == cube.shape
    check(got, grads, cube, w)
    check(learn.layer_gradient(grads[0, 0, 0], cube[0, 0, 0], w), grads[0, 0, :1], cube[0, 0, :1], w)


@pytest.mark.parametrize("dtype", TYPES)
def test_relu_at_zero(dtype):
    """act'(0) is 0, that of the smallest values is not; a NaN lets the gradient pass."""
    from paper_2204_02585_amd import learn
    tiny = torch.finfo(dtype).smallest_normal
    pre = torch.tensor([[0.0, -0.0, tiny, -tiny, float("inf"), -float("inf"), float("nan"), 1.0]], dtype=dtype, device="cuda")
    grad = torch.ones_like(pre)
    x, w = torch.ones((1, 8), dtype=dtype, device="cuda"), torch.ones((8, 8), dtype=dtype, device="cuda")
    _, dw, db = learn.layer_gradient(grad, x, w, pre, "relu")
    want = torch.tensor([0, 0, 1, 0, 1, 0, 1, 1.0], device="cuda")
    assert torch.equal(db, want) and torch.equal(dw[:, 0].float(), want)


def test_binary16_range():
    """dz is held before its share: gradients near binary16's largest value pass a
    mask that makes them ten times as large."""
    from paper_2204_02585_amd import learn
    x, w, _, grad = inputs(40, 32, 24, torch.float16)
    grad = torch.full_like(grad, 60000.0)
    w = w * 1e-3
    x = x * 1e-3
    check(learn.layer_gradient(grad, x, w, dropout=0.9, seed=3), grad, x, w, dropout=0.9, seed=3)


def test_no_points():
    from paper_2204_02585_amd import learn
    for dtype in TYPES:
        x, w, _, grad = inputs(0, 40, 24, dtype)
        dx, dw, db = learn.layer_gradient(grad, x, w, grad, "gelu")
        assert dx.shape == (0, 40) and dw.shape == (24, 40) and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("activation", ACTS)
def test_autograd(dtype, activation):
    """Through autograd: the same as layer_gradient from what the forward call kept,
    the bias's gradient of its type, the residual's the gradient itself."""
    from paper_2204_02585_amd import learn
    leaves = [t.requires_grad_() for t in inputs(70, 40, 56, dtype)]
    leaves[2] = leaves[2].detach().to(dtype).requires_grad_()
    x, w, bias, residual = leaves
    y = learn.layer(x, w, bias, activation, residual, dropout=0.2, seed=6)
    grad = draw(y.shape, dtype, torch.Generator().manual_seed(1))
    got = torch.autograd.grad(y, leaves, grad)
    assert [g.dtype for g in got] == [t.dtype for t in leaves] and torch.equal(got[3], grad)
    pre = torch.empty_like(residual) if activation else None
    plain = [t.detach() for t in leaves]
    again = learn.layer(plain[0], plain[1], plain[2], activation, plain[3], dropout=0.2, seed=6, pre=pre)
    assert torch.equal(again, y)
    want = learn.layer_gradient(grad, plain[0], plain[1], pre, activation, 0.2, 6, bias_dtype=dtype)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    check(want, grad, plain[0], plain[1], pre, activation, 0.2, 6)
    # some of the leaves only
    (only,) = torch.autograd.grad(learn.layer(x.detach(), w, plain[2], activation), w, grad)
    assert only.shape == w.shape
    (only,) = torch.autograd.grad(learn.layer(plain[0], plain[1], bias, activation), bias, grad)
    assert only.shape == bias.shape
    (only,) = torch.autograd.grad(learn.layer(plain[0], plain[1], None, activation, residual), residual, grad)
    assert torch.equal(only, grad)


@pytest.mark.parametrize("activation", ["gelu", "silu", None])
def test_differences(activation):
    """Central differences of the layer in binary32 along random directions.  With
    steps of h = 2^-6 a difference is off by h^2 / 6 of the third derivative along
    it, and by the two values' own bounds over 2 h."""
    from paper_2204_02585_amd import learn
    gen = torch.Generator().manual_seed(3)
    x, w, bias, residual = inputs(12, 20, 10, torch.float32)
    g = draw((12, 10), torch.float32, gen)
    pre = torch.empty_like(residual) if activation else None
    learn.layer(x, w, bias, activation, residual, pre=pre)
    grads = learn.layer_gradient(g, x, w, pre, activation)
    h = 2.0 ** -6
    for k, leaf in enumerate((x, w, bias)):
        d = draw(leaf.shape, torch.float32, gen, leaf.numel() ** -0.5)
        ends = []
        for sign in (1, -1):
            moved = [x, w, bias]
            moved[k] = leaf + sign * h * d
            _, off, *_ = U.layer(*moved, activation, residual, 0.0, 0, torch.float32)
            ends.append((U.double(learn.layer(*moved, activation, residual)), off))
        difference = (U.double(g) * (ends[0][0] - ends[1][0])).sum() / (2 * h)
        # z moves by v along a unit step; activations' third derivatives are below 2
        v = {0: lambda: U.double(d) @ U.double(w).T, 1: lambda: U.double(x) @ U.double(d).T, 2: lambda: U.double(d)[None, :]}[k]()
        off = (np.abs(U.double(g)) * (h * h / 3 * np.abs(v) ** 3 + (ends[0][1] + ends[1][1]) / (2 * h))).sum()
        # the gradient's own bound along d
        want = U.gradients(g, x, w, pre, activation, 0.0, 0)[k][1]
        off += (want.reshape(leaf.shape) * np.abs(U.double(d))).sum()
        # moving the leaf by h d rounds it: half a step of its elements, times the slopes
        off += (np.abs(U.double(grads[k])) * U.F32 * 2 * np.abs(U.double(leaf)) / h).sum()
        assert abs(difference - (U.double(grads[k]) * U.double(d)).sum()) <= off, (k, difference, off)


def test_saved_values_are_watched():
    """Weights changed in place before the backward pass are refused."""
    from paper_2204_02585_amd import learn
    x, w, bias, _ = inputs(20, 16, 8, torch.float32)
    w.requires_grad_()
    y = learn.layer(x.requires_grad_(), w, bias, "relu")
    with torch.no_grad():
        w.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_refusals():
    from paper_2204_02585_amd import learn
    x, w, bias, grad = inputs(4, 8, 6, torch.float32)
    for call, kind, word in ((lambda: learn.layer_gradient(grad[:3], x, w), ValueError, "grad must"),
                             (lambda: learn.layer_gradient(grad.half(), x, w), ValueError, "grad must"),
                             (lambda: learn.layer_gradient(grad.cpu(), x, w), ValueError, "grad must live"),
                             (lambda: learn.layer_gradient(grad, x, w, activation="relu"), ValueError, "pre goes"),
                             (lambda: learn.layer_gradient(grad, x, w, grad), ValueError, "pre goes"),
                             (lambda: learn.layer_gradient(grad, x, w, grad.half(), "relu"), ValueError, "pre must"),
                             (lambda: learn.layer_gradient(grad, x, w, bias_dtype=torch.float16), TypeError, "bias_dtype"),
                             (lambda: learn.layer_gradient(grad, x, w.half()), TypeError, "one dtype"),
                             (lambda: learn.layer_gradient(grad, x, w, dropout=-1), ValueError, "p must")):
        with pytest.raises(kind, match=word):
            call()
    y = learn.layer(x.requires_grad_(), w)
    (g,) = torch.autograd.grad(y, x, grad.requires_grad_(), create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()
