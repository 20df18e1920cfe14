"""Sizes that take tiles of 256, as the choice of kernels has them now: the GPU
tests of those kernels (tests/test_gpu_layer_widest.py) reach them by these sizes."""
import os
import re
import subprocess

import pytest

from paper_2204_02585_amd import build
from tests import fake_hip
from tests.test_build_guard import LLVM, device_code_objects
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


@pytest.mark.skipif(not os.path.exists(f"{LLVM}/llvm-readelf"), reason="ROCm llvm tools missing")
def test_binary32_has_none(tmp_path):
    """Tiles of 256 are built for factors of 16 bits only: hardly a size chose them in
    binary32, where four tiles of 128 take no longer than one."""
    names = set()
    for k, (_, blob) in enumerate(device_code_objects(build.LIB_PATH, str(tmp_path))):
        if b"tile_kernel" in blob:
            path = tmp_path / f"object{k}.o"
            path.write_bytes(blob)
            symbols = subprocess.run([f"{LLVM}/llvm-readelf", "--symbols", "--wide", str(path)], check=True, capture_output=True, text=True).stdout
            names.update(re.findall(r"\S*tile_kernelINS0_5ShapeILi256E\S*", symbols))
    assert any("ShapeILi256EEEDF16_" in n for n in names)
    assert not any("ShapeILi256EEEf" in n for n in names), sorted(names)
