"""Layers and dropout on the CPU: the plain forms' own pins, what the calls
refuse, and that every size they accept is a legal launch (tests/fake_hip.py)."""
import os

import numpy as np
import pytest

from tests import fake_hip, layer_util
from tests.test_learn_cpu import SETUP

LAYERS = SETUP + r"""
def mask(p=0.1, seed=5, step=None):
    return B.DropoutMask(p, seed, step)

def epilogue(bias=None, bias_dtype=F32, act=0, drop=None, residual=None, pre=None):
    e = B.Epilogue(bias, bias_dtype, act)
    e.kept = drop, residual, pre
    for name, value in (("dropout", drop), ("residual", residual), ("pre", pre)):
        if value is not None:
            setattr(e, name, ctypes.addressof(value))
    return e

def forward(points, units, cols, dtype=F32, out=None, short=0, shift=0, x=None, w=None, **more):
    x, w = x or mat(points, cols, dtype), w or mat(units, cols, dtype)
    size = lib.sqn_layer_workspace(x, w)
    return lib.sqn_layer(x, w, epilogue(**more), out or mat(points, units, dtype), alloc(size + 256) + shift, size - short, None)

def backward(points, units, cols, dtype=F32, act=0, drop=None, pre=None, grad=None, short=0, x=None, w=None, to_x=True, to_w=True,
             bias=True, bias_dtype=F32, out_x=None, out_w=None):
    x, w, grad = x or mat(points, cols, dtype), w or mat(units, cols, dtype), grad or mat(points, units, dtype)
    if act and pre is None:
        pre = mat(points, units, dtype)
    size = lib.sqn_layer_gradient_workspace(grad, x, w, act, drop, to_x, to_w, bool(bias))
    bias = alloc(max(4, 4 * units)) if bias is True else bias or None
    return lib.sqn_layer_gradient(grad, x, w, pre or None, act, drop, (out_x or mat(points, cols, dtype)) if to_x else None,
                                  (out_w or mat(units, cols, dtype)) if to_w else None, bias, bias_dtype, alloc(size + 256), size - short, None)

def drop(x, m=True, residual=None, out=None):
    return lib.sqn_dropout(x, mask() if m is True else m, residual, out or mat(x.rows, x.cols, x.dtype), None)
"""


def test_words_of_the_mask():
    """Seed 0 is its own mixed seed: the published outputs of SplitMix64."""
    path = os.path.join(os.path.dirname(__file__), "golden", "splitmix64_seed0.txt")
    want = [int(l.split()[0], 0) for l in open(path) if l.strip() and not l.startswith("#")]
    got = layer_util.words(0, len(want))
    assert len(want) >= 3 and [int(v) for v in got] == want


def test_share_of_the_mask():
    """Rows of odd length start with a word of their own; the share of zeros is
    within five standard deviations of p."""
    w = [int(v) for v in layer_util.words(9, 6)]
    p = 0.3
    bound = round(p * 2 ** 32)
    got = layer_util.share(2, 5, p, 9)
    for row in range(2):
        for col in range(5):
            bits = w[3 * row + col // 2] >> (32 * (col % 2)) & 0xFFFFFFFF
            assert got[row, col] == (0.0 if bits < bound else 1.0 / 0.7)
    for p in (0.01, 0.5, 0.9):
        zeros = (layer_util.share(1000, 301, p, 77) == 0).mean()
        assert abs(zeros - p) < 5 * (p * (1 - p) / 301000) ** 0.5


@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
def test_slopes_are_the_activations(name):
    """Central differences of step h: off by h^2 / 6 of a third derivative (below 2) and a rounding over h."""
    z = np.linspace(-6, 6, 97) + 0.01
    h = 1e-5
    difference = (layer_util.act(z + h, name) - layer_util.act(z - h, name)) / (2 * h)
    assert np.abs(difference - layer_util.slope(z, name)).max() < h * h + 6 * 2.0 ** -52 / h


def test_refusals():
    got = fake_hip.run(LAYERS + r"""
out = []
def bad(status, word, want=BAD):
    out.append([status, want, B.last_error(), word, launches()])
fake.fake_reset()
x = mat(20, 12)
nan = float("nan")
bad(drop(x, None), "mask is NULL")
for p in (-0.1, 1.0001, nan):
    bad(drop(x, mask(p)), "outside [0, 1]")
bad(drop(x, mask(step=alloc(16) + 4)), "8 bytes")
bad(drop(x, mask(step=777)), "step")
bad(drop(x, residual=mat(20, 11)), "residual must be")
bad(drop(x, residual=mat(20, 12, F16)), "residual must be")
bad(drop(x, out=mat(19, 12)), "out must be")
bad(drop(x, out=mat(20, 12, F16)), "out must be")
bad(drop(x, out=mat(20, 12, stride=0, data=x.data)), "stride")
bad(drop(mat(20, 12, 7)), "dtype")
bad(drop(mat(21, 12, data=x.data)), "x")
bad(lib.sqn_layer(None, x, None, x, None, 0, None), "x is NULL")
bad(lib.sqn_layer(x, None, None, x, None, 0, None), "w is NULL")
bad(lib.sqn_layer(x, mat(5, 12), None, None, None, 0, None), "out is NULL")
bad(forward(20, 30, 12, w=mat(30, 13)), "columns")
bad(forward(20, 30, 12, w=mat(30, 12, F16)), "one dtype")
bad(forward(20, 30, 12, w=mat(0, 12)), "rows")
bad(forward(20, 30, 12, w=mat((1 << 20) + 1, 12), out=mat(20, 30)), "rows")
bad(forward(20, 30, 12, out=mat(20, 31)), "out must be")
bad(forward(20, 30, 12, F16, out=mat(20, 30, BF16)), "x's dtype")
bad(forward(20, 30, 12, F32, out=mat(20, 30, BF16)), "x's dtype")
bad(forward(20, 30, 12, act=4), "activation")
bad(forward(20, 30, 12, act=-1), "activation")
bad(forward(20, 30, 12, bias=alloc(119)), "bias")
bad(forward(20, 30, 12, bias=alloc(124) + 1), "bias")
bad(forward(20, 30, 12, bias=alloc(120), bias_dtype=BF16), "bias")
bad(forward(20, 30, 12, drop=mask(2.0)), "outside [0, 1]")
bad(forward(20, 30, 12, F16, residual=mat(20, 30)), "residual must be")
bad(forward(20, 30, 12, F16, residual=mat(20, 29, F16)), "residual must be")
bad(forward(20, 30, 12, F16, pre=mat(20, 30)), "pre must be")
bad(forward(20, 30, 12, pre=mat(20, 30, stride=0, data=x.data)), "stride")
bad(forward(20, 30, 4001, short=1), "workspace of")
bad(forward(20, 30, 4001, shift=8), "256 bytes")
bad(forward(1 << 18, 1 << 18, 8), "tiles", NO)
bad(backward(20, 30, 12, grad=mat(20, 29)), "grad must be")
bad(backward(20, 30, 12, F16, grad=mat(20, 30, BF16)), "grad must be")
bad(backward(20, 30, 12, act=1, pre=mat(20, 29)), "pre must be")
bad(backward(20, 30, 12, BF16, act=1, pre=mat(20, 30)), "pre must be")
bad(backward(20, 30, 12, act=2, pre=False), "pre goes with")
bad(backward(20, 30, 12, act=0, pre=mat(20, 30)), "pre goes with")
bad(backward(20, 30, 12, act=9), "activation")
bad(backward(20, 30, 12, drop=mask(nan)), "outside [0, 1]")
bad(backward(20, 30, 12, out_x=mat(20, 13)), "grad_x must be")
bad(backward(20, 30, 12, F16, out_x=mat(20, 12)), "grad_x must be")
bad(backward(20, 30, 12, out_w=mat(30, 13)), "grad_w must be")
bad(backward(20, 30, 12, out_w=mat(30, 12, stride=11, data=x.data)), "stride")
bad(backward(20, 30, 12, bias=alloc(119)), "grad_bias")
bad(backward(20, 30, 12, bias_dtype=F16), "grad_bias")
bad(backward(20, 30, 12, w=mat(30, 11)), "columns")
bad(backward(20, 30, 12, act=1, short=1), "workspace of")
bad(backward(1 << 26, 8, 2048), "tiles", NO)
bad(lib.sqn_layer_gradient(None, x, mat(30, 12), None, 0, None, None, None, None, 0, None, 0, None), "grad is NULL")
print(json.dumps(out))
""")
    assert len(got) > 50
    for status, want, detail, word, log in got:
        assert status == want and word in detail and not log, (status, want, detail, word, log)


def test_workspace_of_what_is_refused():
    got = fake_hip.run(LAYERS + r"""
x, w = mat(20, 12), mat(30, 12)
print(json.dumps([lib.sqn_layer_workspace(None, w), lib.sqn_layer_workspace(x, None), lib.sqn_layer_workspace(x, mat(30, 13)),
                  lib.sqn_layer_workspace(mat(20, 12, 9), mat(30, 12, 9)), lib.sqn_layer_workspace(x, mat(0, 12)),
                  lib.sqn_layer_gradient_workspace(None, x, w, 0, None, 1, 1, 1),
                  lib.sqn_layer_gradient_workspace(mat(20, 30), x, mat(30, 13), 0, None, 1, 1, 1)]))
""")
    assert got == [0] * 7


def test_no_work():
    """No points: nothing to write forward, and gradients of zeros backward."""
    got = fake_hip.run(LAYERS + r"""
fake.fake_reset()
out = [drop(mat(0, 12)), forward(0, 30, 12), backward(20, 30, 12, to_x=False, to_w=False, bias=False)]
none = launches()
out.append(backward(0, 30, 12, act=1))
print(json.dumps([out, none, len(launches())]))
""")
    assert got[0] == [0] * 4 and got[1] == [] and got[2] > 0


SIZES = [(1, 1, 1), (1, 1 << 20, 1), (1 << 29, 1, 1), (1, 1, 1 << 20), (16, 5, 1 << 20), (17, 1 << 20, 7), (65536, 256, 256),
         (50001, 50, 256), (1 << 26, 500, 33), (181_000, 181_000, 64), (8192, 8192, 4096), (100, 2048, 2048), ((1 << 29) - 3, 64, 9),
         (4097, 4095, 4093)]


def test_every_accepted_size_is_a_legal_launch():
    got = fake_hip.run(LAYERS + r"""
out = []
def ok(name, status):
    log = launches()
    out.append([name, status, B.last_error() if status else "", len(log)])
fake.fake_reset()
M = (1 << 31) - 1
for rows, cols in ((1, 1), (M, 1), (M, 1 << 20), (3, 1 << 20)):
    for dtype in (F32, BF16):
        ok(["dropout", rows, cols, dtype], drop(mat(rows, cols, dtype), residual=mat(rows, cols, dtype)))
for points, units, cols in DATA:
    for dtype, o in ((F32, F32), (F16, F16), (BF16, F32)):
        ok(["layer", points, units, cols, dtype], forward(points, units, cols, dtype, out=mat(points, units, o), act=2, drop=mask()))
        if (points + 63) // 64 * ((cols + 63) // 64) <= 1 << 23 and (units + 63) // 64 * ((cols + 63) // 64) <= 1 << 23:
            for act in (0, 3):
                ok(["gradient", points, units, cols, dtype], backward(points, units, cols, dtype, act=act))
            ok(["gradient of f32", points, units, cols, dtype], backward(points, units, cols, dtype, grad=mat(points, units)))
print(json.dumps(out))
""", SIZES)
    assert len(got) > 80
    for name, status, detail, launched in got:
        assert status == 0 and launched > 0, (name, status, detail, launched)


def test_scratch_is_bounded():
    """Copies of factors off their boundaries, dz, and the parts of sums: never
    more than the factors themselves filled up to eight columns, and 64 MB of
    parts."""
    cases = [(p, u, c, t) for p, u, c in SIZES for t in (0, 2)]
    got = fake_hip.run(LAYERS + r"""
def of(p, u, c, t):
    x, w, g = B.Matrix(1 << 44, p, c, c, t, 0), B.Matrix(1 << 44, u, c, c, t, 0), B.Matrix(1 << 44, p, u, u, t, 0)
    return [lib.sqn_layer_workspace(x, w), lib.sqn_layer_gradient_workspace(g, x, w, 1, None, 1, 1, 1)]
print(json.dumps([of(*c) for c in DATA]))
""", cases)
    for (p, u, c, t), (forward, backward) in zip(cases, got):
        size = 4 if t == 0 else 2
        filled = size * (p + u) * (c + 7) + 512
        parts = 1 << 26
        assert forward <= filled + parts, (p, u, c, t, forward)
        assert backward <= filled + size * p * (u + 7) + 4 * 1024 * u + 512 + parts, (p, u, c, t, backward)


def test_choice_of_kernels():
    """Few points take one launch and no scratch, narrow layers of many points one;
    matrices off the 16-byte boundaries are copied first, save the few and the
    narrow; products of few tiles are split."""
    got = fake_hip.run(LAYERS + r"""
import re
def names(status):
    assert status == 0, B.last_error()
    return [re.search(r"\d+([a-z_]+)_kernel", l.split()[0]).group(1) for l in launches()]
fake.fake_reset()
out = {}
for p, c, u, t in ((1, 4096, 4096, BF16), (16, 33, 5, F32), (17, 4096, 4096, BF16), (17, 64, 64, F32), (2000, 1001, 600, F16), (16384, 42, 250, F32),
                   (16384, 256, 256, F16), (32768, 256, 256, F16), (32768, 256, 64, F16), (32768, 257, 256, F16), (32768, 43, 256, F16), (16383, 42, 250, F32)):
    out["f%d_%d_%d" % (p, c, u)] = names(forward(p, u, c, t))
spaces = [lib.sqn_layer_workspace(mat(p, c, t), mat(u, c, t)) for p, c, u, t in ((16, 4096, 4096, BF16), (32768, 256, 256, F16), (16384, 42, 250, F32))]
for p, c, u, t in ((100, 2048, 2048, BF16), (50000, 256, 50, F32), (65536, 256, 256, F16), (300, 64, 64, F16), (8192, 4096, 8192, BF16)):
    out["b%d_%d_%d" % (p, c, u)] = names(backward(p, u, c, t, act=1))
    out["n%d_%d_%d" % (p, c, u)] = names(backward(p, u, c, t, bias=False))
out["db"] = names(backward(3000, 64, 64, F32, to_x=False, to_w=False))
out["none"] = names(backward(0, 64, 64, F32))
print(json.dumps([out, spaces]))
""")
    out, spaces = got
    assert spaces == [0, 0, 0]
    assert out["f1_4096_4096"] == out["f16_33_5"] == ["few"]
    assert out["f17_4096_4096"] == ["tile", "parts"] and out["f17_64_64"] == ["tile"]
    assert out["f2000_1001_600"] == ["pack", "pack", "tile"]
    assert out["f16384_42_250"] == out["f32768_256_256"] == ["narrow"]
    assert out["f16384_256_256"] == out["f32768_256_64"] == ["tile"]
    assert out["f32768_257_256"] == ["pack", "pack", "tile"] and out["f32768_43_256"] == ["pack", "narrow"]
    assert out["f16383_42_250"] == ["pack", "pack", "tile"]
    # both products of few tiles in one launch, and what is left of all sums in one
    assert out["b300_64_64"][:2] == ["slope", "pair"] and out["n300_64_64"] == ["pair"]
    # the slopes of narrow layers on the way to the points' gradient
    assert out["b65536_256_256"] == ["narrow", "tile", "sums"] and out["n65536_256_256"] == ["narrow", "tile", "sums"]
    assert out["b50000_256_50"] == ["narrow", "tile", "sums"]
    # the sums of few points are the bias's gradient at once
    assert out["b100_2048_2048"] in (["slope", "pair"], ["slope", "pair", "sums"])
    assert out["b8192_4096_8192"] == ["slope", "tile", "tile", "sums"] and out["n8192_4096_8192"] == ["tile", "tile"]
    assert out["db"] == ["slope", "sums"] and out["none"] == ["sums"]
