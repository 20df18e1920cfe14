"""Layers and dropout refuse memory and streams of another device than the
current one, on the CPU (tests/fake_devices.c)."""
import json
import os
import subprocess
import sys

import pytest

from tests import fake_hip
from tests.test_layer_cpu import LAYERS

CALLS = r"""
N, C, U = 300, 100, 400
fake.fake_set_device.argtypes = [ctypes.c_int]

def call(name, on, stream=None):
    # `on[k]` is the device of the call's k-th piece of memory; the rest is on device 0
    def at(k, size=8 << 20):
        fake.fake_set_device(on.get(k, 0))
        p = alloc(size)
        fake.fake_set_device(0)
        return p
    m = lambda rows, cols, k: mat(rows, cols, F32, data=at(k))
    if name == "dropout":
        return lib.sqn_dropout(m(N, C, 0), mask(step=at(1)), m(N, C, 2), m(N, C, 3), stream)
    x, w = m(N, C, 0), m(U, C, 1)
    if name == "layer":
        e = epilogue(bias=at(2), act=1, drop=mask(step=at(3)), residual=m(N, U, 4), pre=m(N, U, 5))
        return lib.sqn_layer(x, w, e, m(N, U, 6), at(7), 8 << 20, stream)
    return lib.sqn_layer_gradient(m(N, U, 2), x, w, m(N, U, 3), 2, mask(step=at(4)), m(N, C, 5), m(U, C, 6), at(7), F32, at(8), 8 << 20, stream)
"""

PIECES = {"dropout": 4, "layer": 8, "gradient": 9}


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("fake") / "fake_devices.so")
    subprocess.run(["gcc", "-O1", "-Wall", "-shared", "-fPIC", "-o", lib, os.path.join(fake_hip.HERE, "fake_devices.c")], check=True)

    def go(code, data=None):
        script = f"ROOT, FAKE, DATA = {fake_hip.ROOT!r}, {lib!r}, {data!r}\n" + fake_hip.PRELUDE + LAYERS + CALLS + code
        p = subprocess.run([sys.executable, "-c", script], capture_output=True, text=True, timeout=100)
        assert p.returncode == 0, p.stderr[-3000:]
        return json.loads(p.stdout.splitlines()[-1])
    return go


@pytest.mark.parametrize("name", PIECES)
def test_memory_of_another_device_is_refused(run, name):
    refused, status, launched = run(r"""
name, pieces = DATA
out = []
fake.fake_reset()
for k in range(pieces):
    out.append([call(name, {k: 1}), B.last_error(), launches()])
print(json.dumps([out, call(name, {}), launches()]))
""", (name, PIECES[name]))
    for k, (s, detail, log) in enumerate(refused):
        # scratch that a call does not need is not looked at
        if name == "layer" and k == 7 and s == 0:
            continue
        assert s == 1 and "lives on device 1, current device is 0" in detail and not log, (k, s, detail, log)
    assert status == 0 and launched


@pytest.mark.parametrize("name", PIECES)
def test_streams_of_another_device_are_refused(run, name):
    (other, detail, none), own, null = run(r"""
fake.fake_reset()
out = []
for stream in (0x1001, 0x1000, None):
    out.append([call(DATA, {}, stream), B.last_error(), len(launches())])
print(json.dumps(out))
""", name)
    assert other == 1 and "stream belongs to device 1, current device is 0" in detail and none == 0
    assert own[0] == null[0] == 0 and own[2] > 0 and null[2] > 0
