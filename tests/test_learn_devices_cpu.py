"""The operators on learned tables and layers refuse memory and streams of
another device than the current one, on the CPU (tests/fake_devices.c): a
launch on the current device would not be ordered with the other's work."""
import json
import os
import subprocess
import sys

import pytest

from tests import fake_hip
from tests.test_learn_cpu import SETUP

CALLS = r"""
N = 300

def call(name, on, stream=None):
    # `on[k]` is the device of the call's k-th piece of memory; the rest is on device 0
    def at(k, size):
        fake.fake_set_device(on.get(k, 0))
        p = alloc(size)
        fake.fake_set_device(0)
        return p
    big = 4 << 20
    if name == "lookup":
        return lib.sqn_lookup(mat(90, 8, data=at(0, big)), at(1, big), I64, 1.0, mat(N, 8, data=at(2, big)), stream)
    if name == "gradient":
        size = lib.sqn_lookup_gradient_workspace(N, 90, 8)
        return lib.sqn_lookup_gradient(mat(N, 8, data=at(0, big)), at(1, big), I64, 1.0, 0, mat(90, 8, data=at(2, big)),
                                       at(3, size), size, stream)
    if name == "orthogonalise":
        size = lib.sqn_orthogonalise_workspace(2, 200, 300, BF16)
        return lib.sqn_orthogonalise(batch(2, 200, 300, data=at(0, big)), 5, MUON, 1e-7, batch(2, 200, 300, BF16, data=at(1, big)),
                                     at(2, size), size, stream)
    if name == "quantise":
        return lib.sqn_quantise(mat(N, 100, data=at(0, big)), quant(N, 100, at(1, big), at(2, big)), stream)
    if name == "values":
        return lib.sqn_quantised_values(quant(N, 100, at(0, big), at(1, big)), mat(N, 100, data=at(2, big)), stream)
    if name == "product":
        size = lib.sqn_quantised_product_workspace(N, 400, 100)
        return lib.sqn_quantised_product(quant(N, 100, at(0, big), at(1, big)), quant(400, 100, at(2, big), at(3, big)),
                                         at(4, big), 0, mat(N, 400, data=at(5, big)), at(6, size), size, stream)
    size = lib.sqn_quantised_layer_workspace(N, 400, 100)
    return lib.sqn_quantised_layer(mat(N, 100, data=at(0, big)), quant(400, 100, at(1, big), at(2, big)), at(3, big), 0,
                                   mat(N, 400, data=at(4, big)), at(5, size), size, stream)

fake.fake_set_device.argtypes = [ctypes.c_int]
"""

PIECES = {"lookup": 3, "gradient": 4, "orthogonalise": 3, "quantise": 3, "values": 3, "product": 7, "layer": 6}


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    """As fake_hip.run, with tests/fake_devices.c in the runtime's place."""
    lib = str(tmp_path_factory.mktemp("fake") / "fake_devices.so")
    subprocess.run(["gcc", "-O1", "-Wall", "-shared", "-fPIC", "-o", lib, os.path.join(fake_hip.HERE, "fake_devices.c")], check=True)

    def go(code, data=None):
        script = f"ROOT, FAKE, DATA = {fake_hip.ROOT!r}, {lib!r}, {data!r}\n" + fake_hip.PRELUDE + SETUP + CALLS + code
        p = subprocess.run([sys.executable, "-c", script], capture_output=True, text=True, timeout=100)
        assert p.returncode == 0, p.stderr[-3000:]
        return json.loads(p.stdout.splitlines()[-1])
    return go


@pytest.mark.parametrize("name", PIECES)
def test_memory_of_another_device_is_refused(run, name):
    got = run(r"""
name, pieces = DATA
out = []
fake.fake_reset()
for k in range(pieces):
    out.append([call(name, {k: 1}), B.last_error(), launches()])
print(json.dumps([out, call(name, {}), launches()]))
""", (name, PIECES[name]))
    refused, status, launched = got
    for k, (s, detail, log) in enumerate(refused):
        assert s == 1 and "lives on device 1, current device is 0" in detail and not log, (k, s, detail, log)
    assert status == 0 and launched


@pytest.mark.parametrize("name", PIECES)
def test_streams_of_another_device_are_refused(run, name):
    got = run(r"""
fake.fake_reset()
out = []
for stream in (0x1001, 0x1000, None):
    out.append([call(DATA, {}, stream), B.last_error(), len(launches())])
print(json.dumps(out))
""", name)
    (other, detail, none), own, null = got
    assert other == 1 and "stream belongs to device 1, current device is 0" in detail and none == 0
    assert own[0] == null[0] == 0 and own[2] > 0 and null[2] > 0


def test_another_current_device(run):
    """Everything on device 1, and device 1 current: accepted; the current device
    changed since the allocations: refused."""
    got = run(r"""
fake.fake_set_device(1)
a = [mat(90, 8), alloc(8 * N), mat(N, 8)]
fake.fake_reset()
here = [lib.sqn_lookup(a[0], a[1], I64, 1.0, a[2], 0x1001), len(launches())]
fake.fake_set_device(0)
there = [lib.sqn_lookup(a[0], a[1], I64, 1.0, a[2], None), B.last_error(), len(launches())]
print(json.dumps([here, there]))
""")
    (status, launched), (refused, detail, none) = got
    assert status == 0 and launched == 1
    assert refused == 1 and "lives on device 1, current device is 0" in detail and none == 0
