"""Choices of the operators on learned tables and layers that bound what a call
takes, on the CPU (tests/fake_hip.py)."""
from tests import fake_hip
from tests.test_learn_cpu import SETUP

NAMES = r"""
import re
def names(status):
    assert status == 0, B.last_error()
    return [re.search(r"\d+([a-z_]+)_kernel", l.split()[0]).group(1) for l in launches()]
fake.fake_reset()
"""


def test_many_indices_to_few_rows_take_the_radix_sort():
    """A bucket is one workgroup's: the few buckets of a few rows get no more
    indices than they sort at once."""
    got = fake_hip.run(SETUP + NAMES + r"""
print(json.dumps([[rows, n, names(gradient(n, rows, 8))] for rows, n in
                  ((1, 4096), (1, 4097), (8, 4096), (8, 4097), (8, 40000), (16, 8192), (16, 8193), (700, 40000))]))
""")
    for rows, n, kernels in got:
        want = "bucket" if (rows, n) in ((1, 4096), (8, 4096), (16, 8192), (700, 40000)) else "count"
        assert kernels[0] == want, (rows, n, kernels)


def test_scratch_of_skinny_updates():
    """Matrices of few rows are not filled up to the largest tiles: the scratch is
    within 1.6 times what tiles of 64 take, whatever the batch."""
    cases = [(batch, m, n, out) for out in (0, 2) for batch, m, n in
             ((1000, 16, 4096), (65535, 1, 129), (65535, 1, 257), (200, 40, 2000), (24, 70, 1500), (24, 130, 1300), (64, 129, 129),
              (64, 260, 260), (64, 300, 300), (16, 257, 900), (3, 1, 32768), (1000, 4096, 16), (500, 65, 258))]
    got = fake_hip.run(SETUP + """
print(json.dumps([lib.sqn_orthogonalise_workspace(b, m, n, o) for b, m, n, o in DATA]))
""", cases)
    for (batch, m, n, out), size in zip(cases, got):
        m, n = sorted((m, n))
        if m <= 128 and n <= (256 if out == 2 else 128):
            assert size == 0
            continue
        mp, np = -(-m // 64) * 64, -(-n // 64) * 64
        # X and its transposes (4 arrays of binary16; 6 and one of binary32 where factors are split), O and B, diagonals, norms
        one = (8 if out == 2 else 16) * mp * np + (4 if out == 2 else 8) * mp * mp + 8 * mp + 2048
        assert 0 < size <= 1.6 * batch * one, (batch, m, n, out, size, batch * one)


def test_large_updates_keep_large_tiles():
    got = fake_hip.run(SETUP + r"""
out = []
fake.fake_reset()
for b, m, n, o in DATA:
    assert orth(batch(b, m, n), batch(b, m, n, o), steps=1) == 0, B.last_error()
    out.append(launches()[2])
print(json.dumps(out))
""", [(1, 4096, 4096, 2), (1, 4096, 4096, 0), (64, 390, 390, 2), (24, 520, 520, 2), (64, 200, 300, 0), (24, 130, 1300, 2), (1000, 16, 4096, 2)])
    for name, side in zip(got, (256, 128, 256, 128, 128, 64, 64)):
        assert f"ILi{side}E" in name, (name, side)


def test_many_points_by_several_tiles_of_units():
    """The ends of the range of products, each within it: as many tiles of 64 x 64 as
    a product may have, and one more."""
    cases = [(1 << 26, 500, 100), (1 << 26, 512, 33), ((1 << 23) // 5 * 64, 300, 100), (1 << 29, 64, 40), (32768, 1 << 20, 40), (17, 1 << 20, 1),
             (185_000, 185_000, 64)]
    got = fake_hip.run(SETUP + """
out = []
fake.fake_reset()
for points, units, cols in DATA:
    out.append([layer(points, units, cols), len(launches()), product(points, units, cols), len(launches())])
print(json.dumps([out, layer((1 << 26) + 1, 512, 100), product((1 << 26) + 1, 512, 100), len(launches())]))
""", cases)
    assert all(-(-p // 64) * -(-u // 64) <= 1 << 23 for p, u, _ in cases)
    for case, (status, launched, status_blocks, launched_blocks) in zip(cases, got[0]):
        assert status == status_blocks == 0 and launched > 0 and launched_blocks > 0, case
    assert got[1] == got[2] == 4 and got[3] == 0
