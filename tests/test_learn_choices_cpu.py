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
