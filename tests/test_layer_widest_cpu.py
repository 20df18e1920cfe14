"""Sizes that take tiles of 256, as the choice of kernels has them now: the GPU
tests of those kernels (tests/test_gpu_layer_widest.py) reach them by these sizes."""
import re

from tests import fake_hip
from tests.test_layer_cpu import LAYERS

# points, cols, units, ragged at every end; with all of an epilogue, and with what leaves the residual out
WHOLE, SOME = (3989, 4090, 4075), (4308, 2520, 2886)
GRADIENTS = [(2081, 6995, 2292), (3989, 4090, 4075)]


def test_they_take_tiles_of_256():
    got = fake_hip.run(LAYERS + r"""
def names(status):
    assert status == 0, B.last_error()
    return [l.split()[0] for l in launches()]
fake.fake_reset()
whole, some, gradients = DATA
out = []
for t in (F16, BF16):
    for o in (t, F32):
        p, c, u = whole
        for r in (None, mat(p, u, o)):
            out.append([[p, c, u, t, o], 1, names(forward(p, u, c, t, out=mat(p, u, o), act=2, drop=mask(), pre=mat(p, u, t), residual=r))])
        p, c, u = some
        for act, drop in ((0, None), (2, mask()), (3, mask())):
            out.append([[p, c, u, t, o], 1, names(forward(p, u, c, t, out=mat(p, u, o), act=act, drop=drop))])
    for p, c, u in gradients:
        for act in (0, 1, 2):
            out.append([[p, c, u, t, act], 2, names(backward(p, u, c, t, act=act))])
print(json.dumps(out))
""", [WHOLE, SOME, GRADIENTS])
    assert len(got) == 32
    for case, count, names in got:
        tiles = [n for n in names if re.search(r"\d+(tile|pair)_kernel", n)]
        assert len(tiles) == count and all("ShapeILi256E" in n for n in tiles), (case, tiles)
