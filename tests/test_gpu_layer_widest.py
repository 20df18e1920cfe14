"""Layers whose tiles are the widest, and the epilogues of narrow layers of many
points, every value against 64 bits on the GPU."""
import numpy as np
import pytest
import torch

from tests import layer_util as U
from tests.test_gpu_layer import draw, inputs
from tests.test_gpu_layer_gradient_digits import check, want_of
from tests.test_layer_widest_cpu import GRADIENTS, SOME, WHOLE

pytestmark = pytest.mark.gpu


def layer_of(x, w, bias, activation, residual, p, seed, dtype):
    """(y, its bound, z, its bound) in 64 bits; as layer_util.layer has them."""
    x64, w64 = x.double(), w.double().t().contiguous()
    z, size = x64 @ w64, x64.abs() @ w64.abs()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    off_z = 2 * U.F32 * (x.shape[1] + 9) * size + 2 * U.F32 * z.abs()
    m = torch.from_numpy(U.share(*z.shape, p, seed)).cuda()
    y = {None: lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: 0.5 * z * torch.special.erfc(z * -0.5 ** 0.5),
         "silu": lambda: z * torch.sigmoid(z)}[activation]() * m
    off = m * (1.13 * off_z + 16 * U.F32 * z.abs())
    if residual is not None:
        y = y + residual.double()
    off = off + 8 * U.F32 * y.abs()

    def rounded(v, o, t):
        return o + U.UNIT[t] * (v.abs() + o).clamp(min=U.TINY[t])
    return y, rounded(y, off, dtype), z, rounded(z, off_z, x.dtype)


def check_layer(x, w, bias, activation, residual, p, seed, dtype=None, keep=True):
    from paper_2204_02585_amd import learn
    dtype = dtype or x.dtype
    pre = torch.empty((len(x), len(w)), dtype=x.dtype, device="cuda") if keep else None
    y = learn.layer(x, w, bias, activation, residual, dropout=p, seed=seed, dtype=dtype, pre=pre)
    assert y.dtype == dtype
    want, off, z, off_z = layer_of(x, w, bias, activation, residual, p, seed, dtype)
    for got, v, bound in ((y, want, off), (pre, z, off_z)):
        if got is not None:
            bad = ~((got.double() - v).abs() <= bound)
            assert not bad.any(), (activation, p, int(bad.sum()), bad.nonzero()[0].tolist())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("out", ["same", "float32"])
def test_widest_tiles(dtype, out):
    """Tiles of 256 with all of an epilogue and with some of it."""
    out = dtype if out == "same" else torch.float32
    x, w, bias, residual = inputs(*WHOLE, dtype, out)
    check_layer(x, w, bias, "gelu", residual, 0.1, 5, out)
    check_layer(x, w, bias, "gelu", None, 0.1, 6, out)
    x, w, bias, _ = inputs(*SOME, dtype, out)
    check_layer(x, w, bias, "silu", None, 0.3, 7, out, keep=False)
    check_layer(x, w, None, "gelu", None, 0.1, 8, out, keep=False)
    check_layer(x, w, None, None, None, 0.0, 0, out, keep=False)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("size", GRADIENTS)
@pytest.mark.parametrize("activation,p", [(None, 0.0), ("relu", 0.1), ("gelu", 0.1)])
def test_widest_gradients(dtype, size, activation, p):
    """Both products in tiles of 256: grad as it lies, with slopes, and in parts."""
    from paper_2204_02585_amd import learn
    x, w, _, grad = inputs(*size, dtype)
    pre = draw(grad.shape, dtype, torch.Generator().manual_seed(9)) if activation else None
    check(learn.layer_gradient(grad, x, w, pre, activation, p, 5), want_of(grad, x, w, pre, activation, p, 5), (activation, p))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("activation", ["gelu", "silu", "relu", None])
@pytest.mark.parametrize("points,cols,units", [(16384, 42, 250), (20001, 7, 50), (33000, 64, 200), (32768, 256, 256), (40000, 100, 130),
                                               (131103, 64, 64), (131072, 128, 100), (16385, 130, 33)])
def test_narrow_epilogues(dtype, activation, points, cols, units):
    """Kept elements of a masked layer of many points are its values times the share,
    onto the residual; the same kept z."""
    x, w, bias, residual = inputs(points, cols, units, dtype)
    check_layer(x, w, bias, activation, residual, 0.3, 11)
    check_layer(x, w, bias.to(dtype), activation, None, 0.5, 12, torch.float32)
