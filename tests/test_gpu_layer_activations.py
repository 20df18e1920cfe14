"""The activations and their slopes of binary32 results, relative to themselves, far
below zero too."""
import numpy as np
import pytest
import torch

from tests import layer_util as U
from tests.test_gpu_layer import inputs

pytestmark = pytest.mark.gpu


def points(dtype):
    z = torch.cat([torch.linspace(-12, 12, 60001), torch.linspace(-1.2, 1.2, 20001)]).to(dtype)
    return z[z != 0].cuda()[:, None]


def formulas(z):
    """{name: (act(z), slope, sum of the magnitudes that make the slope)} in 64 bits.
    erfc, unlike ndtr, is accurate relative to itself far below zero."""
    share, bell, s = 0.5 * torch.special.erfc(z * -0.5 ** 0.5), torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5, torch.sigmoid(z)
    return {"gelu": (z * share, share + z * bell, share + z.abs() * bell),
            "silu": (z * s, s + z * s * torch.sigmoid(-z), s + z.abs() * s)}


# half steps of binary32.  GELU: exp2's unit in the last place is two, its correction and the products with
# bell, t and z one each; the polynomial's nine fused steps one each of partial sums that are 2.2 q together
# (their magnitudes at t = 1), and t's own 1.5 change q by as much; so below 32.  SiLU: exp2 two, its
# correction, the sum, the quotient and the product one each, z's exponent one more.  A slope is sums of such.
STEPS = {"gelu": 32, "silu": 8}


@pytest.mark.parametrize("name", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_values(name, dtype):
    """One unit of one column and a weight of one: z is x.  A result of binary32 keeps
    its digits whatever the factors' type; few points, and many."""
    from paper_2204_02585_amd import learn
    z = points(dtype)
    want = formulas(z.double())[name][0]
    w = torch.ones((1, 1), dtype=dtype, device="cuda")
    for part in (slice(None), slice(0, 16), slice(100, 1000)):
        got = learn.layer(z[part], w, activation=name, dtype=torch.float32).double()
        off = (got - want[part]).abs() / want[part].abs()
        assert off.max() <= STEPS[name] * U.F32, (part, float(off.max() / U.F32), float(z[part][off.argmax()]))


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_slopes(name):
    from paper_2204_02585_amd import learn
    z = points(torch.float32)
    _, want, size = formulas(z.double())[name]
    one = torch.ones((1, 1), device="cuda")
    grad = torch.ones_like(z)
    for part in (slice(None), slice(0, 16), slice(100, 1000)):
        n = len(z[part])
        dx, _, db = learn.layer_gradient(grad[part], torch.ones_like(z[part]), one, z[part], name)
        off = (dx.double() - want[part]).abs() / size[part]
        assert off.max() <= (STEPS[name] + 4) * U.F32, (part, float(off.max() / U.F32), float(z[part][off.argmax()]))
        total = size[part].sum()
        assert abs(float(db) - float(want[part].sum())) <= (STEPS[name] + 4 + 2 * (n + 8)) * U.F32 * total


@pytest.mark.parametrize("name", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_ends(name, dtype):
    """Values at the range's ends and none: as the formula gives them."""
    from paper_2204_02585_amd import learn
    inf, nan = float("inf"), float("nan")
    z = torch.tensor([0.0, -0.0, inf, -inf, nan, 60000.0, -60000.0, 150.0, -150.0], dtype=dtype, device="cuda")[:, None]
    w = torch.ones((1, 1), dtype=dtype, device="cuda")
    y = learn.layer(z, w, activation=name, dtype=torch.float32)[:, 0]
    assert y[0] == 0 and y[1] == 0 and y[2] == inf and y[3].isnan() and y[4].isnan()
    assert y[5] == float(z[5]) and y[6] == 0 and y[7] == 150 and y[8] == 0
    dx = learn.layer_gradient(torch.ones_like(z), z, w, z, name)[0][:, 0]
    assert dx[0] == 0.5 and dx[1] == 0.5 and dx[4].isnan() and dx[5] == 1 and dx[6] == 0 and dx[7] == 1 and dx[8] == 0


@pytest.mark.parametrize("name", ["gelu", "silu"])
@pytest.mark.parametrize("size", [(16, 64, 40), (300, 200, 136), (2100, 128, 1700), (17000, 42, 250), (40000, 100, 250), (33000, 64, 200)])
def test_layers_in_binary32(name, size):
    """Every kernel's epilogue: y from the z that it kept."""
    from paper_2204_02585_amd import learn
    x, w, bias, _ = inputs(*size, torch.float32)
    pre = torch.empty((size[0], size[2]), device="cuda")
    y = learn.layer(x, w, 3 * bias, name, pre=pre)
    want = formulas(pre.double())[name][0]
    assert ((y.double() - want).abs() <= STEPS[name] * U.F32 * want.abs() + 2.0 ** -126).all()
