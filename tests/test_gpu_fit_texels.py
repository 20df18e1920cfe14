"""The example that uses the operators on learned tables and layers together:
the loss falls, and 4-bit layers decode what the exact ones do."""
import pytest

pytestmark = pytest.mark.gpu


def test_fit_texels():
    from examples import fit_texels
    r = fit_texels.fit(side=48, points=4096, steps=60)
    # the colours' own variance is above 0.03: an error of a tenth of the first loss needs a table that
    # learned; 4-bit layers add errors of some 2^-3 of a value's size, relative to colours of at most 1
    assert r["last_loss"] < 0.1 * r["first_loss"]
    assert r["exact"] < 0.1 * r["first_loss"]
    assert r["blocks"] < 0.5 * r["first_loss"]
    # the same blocks and products, in another order of sums: 32 terms of binary32, each below ten times
    # the largest sum, make 32 * 2^-24 * 10 = 2e-5 of it
    assert r["few_apart"] < 1e-4
    assert r["bytes_blocks"] * 7 < r["bytes_exact"]
