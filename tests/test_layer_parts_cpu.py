"""Gradients whose dz is held in two parts: which calls take them, and their
scratch, on the CPU (tests/fake_hip.py)."""
from tests import fake_hip
from tests.test_layer_cpu import LAYERS


def test_which_calls_take_parts():
    """GELU, SiLU and a binary32 gradient of 16-bit factors; binary16 factors are put
    into parts themselves, the narrow kernel makes the parts on its way."""
    got = fake_hip.run(LAYERS + r"""
import re
def names(status):
    assert status == 0, B.last_error()
    return [re.search(r"\d+([a-z_]+)_kernel", l.split()[0]).group(1) for l in launches()]
fake.fake_reset()
out = {}
for name, t in (("f16", F16), ("bf16", BF16)):
    for act in (0, 1, 2, 3):
        out["%s_%d" % (name, act)] = names(backward(8192, 8192, 4096, t, act=act))
    out[name + "_f32"] = names(backward(8192, 8192, 4096, t, grad=mat(8192, 8192)))
    out[name + "_narrow"] = names(backward(65536, 256, 256, t, act=2))
    out[name + "_bias"] = names(backward(65536, 256, 256, t, act=2, to_x=False, to_w=False))
out["f32"] = names(backward(8192, 8192, 4096, F32, act=2))
print(json.dumps(out))
""")
    apart = ["slope", "tile", "tile", "sums"]
    for name in ("f16_1", "bf16_1", "bf16_2", "bf16_3", "bf16_f32"):
        assert got[name] == apart, (name, got[name])
    assert "part" not in got["f32"]
    # nothing stands between grad and dz: it is read as it lies
    assert got["f16_0"] == got["bf16_0"] == ["slope", "tile", "tile", "sums"]
    for name in ("f16_2", "f16_3", "f16_f32"):
        assert got[name] == ["slope", "part", "part", "tile", "tile", "sums"], (name, got[name])
    assert got["bf16_narrow"] == ["narrow", "tile", "sums"]
    assert got["f16_narrow"][:3] == ["slope", "part", "part"] and "narrow" not in got["f16_narrow"]
    assert got["f16_bias"] == got["bf16_bias"] == ["slope", "sums"]


def test_scratch_is_bounded():
    """Two parts of dz and of binary16 factors, the sums of the bias and the parts of
    products: no more."""
    sizes = [(1, 1, 1), (16, 5, 4096), (65536, 256, 256), (50001, 50, 256), (8192, 8192, 4096), (131072, 128, 64), (4097, 4095, 4093)]
    cases = [(p, u, c, t, act, g) for p, u, c in sizes for t in (1, 2) for act, g in ((2, t), (0, 0), (3, 0))]
    got = fake_hip.run(LAYERS + r"""
def of(p, u, c, t, act, g):
    x, w, grad = B.Matrix(1 << 44, p, c, c, t, 0), B.Matrix(1 << 44, u, c, c, t, 0), B.Matrix(1 << 44, p, u, u, g, 0)
    return [lib.sqn_layer_gradient_workspace(grad, x, w, act, None, *wanted) for wanted in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1))]
print(json.dumps([of(*c) for c in DATA]))
""", cases)
    for (p, u, c, t, act, g), sizes in zip(cases, got):
        dz, sums, parts = 2 * (2 * p * (u + 7) + 256), 4 * 1024 * u + 256, 1 << 26
        x, w = ((2 * (2 * n * (c + 7) + 256)) for n in (p, u))
        for size, most in zip(sizes, (dz + x + w + sums + 2 * parts, dz + w + parts, dz + x + parts, sums)):
            assert size <= most, (p, u, c, t, act, g, size, most)
        # of the parts alone, at least what they take
        assert sizes[0] >= 2 * 2 * p * u
