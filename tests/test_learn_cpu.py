"""Host code of the operators on learned tables and layers, on the CPU
(tests/fake_hip.py): what they refuse, that every size they accept is a legal
launch, and which kernels they choose."""
from tests import fake_hip

SETUP = r"""
F32, F16, BF16, I32, I64 = B.SQN_F32, B.SQN_F16, B.SQN_BF16, B.SQN_I32, B.SQN_I64
ES = {F32: 4, F16: 2, BF16: 2}
BAD, NO = B.SQN_ERR_INVALID_ARG, B.SQN_ERR_UNSUPPORTED

def mat(rows, cols, dtype=F32, stride=None, data=None, reserved=0):
    stride = cols if stride is None else stride
    if data is None:
        data = alloc(max(1, ((rows - 1) * stride + cols) * ES.get(dtype, 4)))
    return B.Matrix(data, rows, cols, stride, dtype, reserved)

def batch(n, rows, cols, dtype=F32, strides=None, data=None):
    strides = strides or (rows * cols, cols, 1)
    if data is None:
        data = alloc(max(1, ((n - 1) * strides[0] + (rows - 1) * strides[1] + (cols - 1) * strides[2] + 1) * ES.get(dtype, 4)))
    return B.Batch(data, n, rows, cols, dtype, *strides)

def quant(rows, cols, codes=None, scales=None):
    blocks = (cols + 31) // 32
    return B.QuantisedMatrix(alloc(max(1, 16 * rows * blocks)) if codes is None else codes,
                             alloc(max(1, rows * blocks)) if scales is None else scales, rows, cols)

MUON = (ctypes.c_float * 3)(3.4445, -4.7750, 2.0315)

def lookup(table, n, ids=None, kind=I64, out=None, scale=1.0):
    ids = alloc(max(1, 8 * n)) if ids is None else ids
    return lib.sqn_lookup(table, ids, kind, scale, out or mat(n, table.cols, table.dtype), None)

def gradient(n, rows, cols, dtype=F32, out=F32, kind=I64, accumulate=0, short=0, shift=0, **more):
    size = lib.sqn_lookup_gradient_workspace(n, rows, cols)
    return lib.sqn_lookup_gradient(more.get("grad") or mat(n, cols, dtype), alloc(max(1, 8 * n)), kind, 1.0, accumulate,
                                   more.get("table") or mat(rows, cols, out), alloc(size + 256) + shift, size - short, None)

def orth(src, dst, steps=5, k=MUON, eps=1e-7, short=0):
    size = lib.sqn_orthogonalise_workspace(dst.batch, dst.rows, dst.cols, dst.dtype)
    return lib.sqn_orthogonalise(src, steps, k, eps, dst, alloc(max(1, size)), size - short, None)

def layer(points, units, cols, dtype=F32, out=None, bias=None, relu=0, short=0, w=None):
    size = lib.sqn_quantised_layer_workspace(points, units, cols)
    return lib.sqn_quantised_layer(mat(points, cols, dtype), w or quant(units, cols), bias, relu, out or mat(points, units),
                                   alloc(max(1, size)), size - short, None)

def product(points, units, cols, out=None):
    size = lib.sqn_quantised_product_workspace(points, units, cols)
    return lib.sqn_quantised_product(quant(points, cols), quant(units, cols), None, 0, out or mat(points, units),
                                     alloc(max(1, size)), size, None)
"""


def test_refusals():
    """Each call names what is wrong with an argument and launches nothing."""
    got = fake_hip.run(SETUP + r"""
out = []
def bad(status, word, want=BAD):
    out.append([status, want, B.last_error(), word, launches()])

t = mat(10, 6)
fake.fake_reset()
bad(lib.sqn_lookup(None, alloc(8), I64, 1.0, t, None), "table is NULL")
bad(lookup(mat(10, 6, dtype=3), 4), "dtype")
bad(lookup(mat(10, 6, reserved=1), 4), "reserved")
bad(lookup(mat(10, 0, data=alloc(8)), 4), "10 x 0")
bad(lookup(mat(-1, 6, data=alloc(8)), 4), "-1 x 6")
bad(lookup(mat(1 << 31, 6), 4), "outside")
bad(lookup(mat(10, 6, stride=-6, data=alloc(1000)), 4), "stride")
bad(lookup(mat(11, 6, data=t.data), 4, out=mat(4, 6)), "table")
bad(lookup(mat(10, 6, data=t.data + 2), 4), "aligned")
bad(lookup(t, 4, kind=2), "ids_type")
bad(lookup(t, 4, ids=12345), "ids")
bad(lookup(t, 4, ids=alloc(8 * 4)  + 4), "aligned")
bad(lookup(t, 400, ids=alloc(8)), "ids")
bad(lookup(t, 4, out=mat(4, 7)), "columns")
bad(lookup(t, 4, out=mat(4, 6, F16)), "dtype")
bad(lookup(t, 4, out=mat(4, 6, stride=5)), "stride")
bad(gradient(300, 10, 6, kind=7), "ids_type")
bad(gradient(300, 10, 6, accumulate=2), "accumulate")
bad(gradient(300, 10, 6, short=1), "workspace of")
bad(gradient(300, 10, 6, shift=8), "256 bytes")
bad(gradient(300, 10, 6, table=mat(10, 7)), "columns")
bad(gradient(300, 10, 6, table=mat(0, 6)), "a row")
bad(gradient(300, 10, 6, grad=mat((1 << 30) + 1, 6)), "2^30")
g = batch(2, 300, 200)
for steps in (-1, 65):
    bad(orth(g, batch(2, 300, 200, BF16), steps=steps), "steps")
for eps in (-1.0, float("nan"), float("inf")):
    bad(orth(g, batch(2, 300, 200, BF16), eps=eps), "eps")
for k in ((4.0, 0.0, 0.0), (2.0, -1.0, 9.0), (0.0, 30.0, -30.0), (float("inf"), 0.0, 0.0)):
    bad(orth(g, batch(2, 300, 200, BF16), k=(ctypes.c_float * 3)(*k)), "oefficients")
bad(orth(g, batch(2, 300, 200, 5, data=g.data)), "dtype")
bad(orth(g, batch(2, 200, 300, BF16)), "out is")
bad(orth(g, batch(2, 300, 200, BF16, strides=(60000, 0, 1))), "one place")
bad(orth(g, batch(2, 300, 200, BF16, strides=(60000, 199, 1))), "one place")
bad(orth(g, batch(2, 300, 200, BF16, strides=(100, 200, 1))), "one place")
bad(orth(g, batch(2, 300, 200, BF16), short=1), "workspace of")
bad(orth(batch(1, 32769, 2), batch(1, 32769, 2, BF16)), "32768")
bad(orth(batch(2, 300, 201, data=g.data), batch(2, 300, 201, BF16)), "updates")
q = quant(40, 100)
bad(lib.sqn_quantise(mat(40, 101), q, None), "x's rows")
bad(lib.sqn_quantise(mat(40, 100), quant(40, 100, codes=q.codes + 8), None), "16 bytes")
bad(lib.sqn_quantise(mat(40, 100), quant(40, 100, scales=alloc(159)), None), "out")
bad(lib.sqn_quantised_values(q, mat(40, 99), None), "x's rows")
bad(lib.sqn_quantised_values(None, mat(40, 99), None), "x is NULL")
bad(layer(100, 40, 1000, w=quant(40, 999)), "columns")
bad(layer(100, 40, 1000, out=mat(100, 41)), "the product")
bad(layer(100, 40, 1000, relu=2), "relu")
bad(layer(100, 40, 1000, bias=alloc(159)), "bias")
bad(layer(100, 40, 1000, bias=alloc(164) + 1), "bias")
bad(layer(100, 40, 1000, short=1), "workspace of")
bad(layer(100, 0, 1000, out=mat(100, 1)), "w")
bad(layer(1 << 18, 1 << 18, 64), "tiles", NO)
print(json.dumps(out))
""")
    for status, want, detail, word, log in got:
        assert status == want and word in detail and not log, (status, want, detail, word, log)


def test_no_work_is_no_launch():
    got = fake_hip.run(SETUP + r"""
out = [lookup(mat(10, 6), 0), gradient(0, 10, 6, accumulate=1), orth(batch(0, 4, 5), batch(0, 4, 5, BF16)),
       lib.sqn_quantise(mat(0, 6), quant(0, 6), None), lib.sqn_quantised_values(quant(0, 6), mat(0, 6), None),
       layer(0, 5, 100), product(0, 5, 100)]
print(json.dumps([out, launches()]))
""")
    assert got == [[0] * 7, []]


def test_every_accepted_size_is_a_legal_launch():
    """The ends of the ranges, and sizes around the changes of kernel: the
    stand-in for the runtime refuses a grid that the runtime would."""
    got = fake_hip.run(SETUP + r"""
out = []
def ok(name, status):
    log = launches()
    out.append([name, status, B.last_error() if status else "", len(log)])

M = (1 << 31) - 1
for rows, cols, n in ((1, 1, 1), (M, 1, 1 << 20), (10, 1 << 20, M), (M, 3, M), (0, 9, 5), (M, 1 << 20, 3)):
    for dtype in (F32, F16):
        ok(["lookup", rows, cols, n], lookup(mat(rows, cols, dtype), n))
for n, rows, cols in ((1, 1, 1), (256, M, 1), (257, M, 1), (257, 1, 1), (1 << 17, 1 << 24, 1), (122880, 1 << 24, 1), (122881, 1 << 24, 1), (256, 4_000_000, 1 << 16), (1 << 30, M, 1), (1 << 30, 7, 1 << 20),
                      (16384, 5, 9), (16385, 5, 9), (1025, 1 << 20, 40), (1, 300_000, 1 << 20)):
    for dtype, o in ((F32, F32), (BF16, F16)):
        ok(["gradient", n, rows, cols], gradient(n, rows, cols, dtype, o))
        ok(["accumulate", n, rows, cols], gradient(n, rows, cols, dtype, o, accumulate=1))
for b, m, n in ((65535, 1, 1), (65535, 128, 256), (65535, 129, 1), (1, 32768, 32768), (3, 1, 32768), (65535, 40, 257), (1, 128, 129),
                (2, 255, 255), (1, 1600, 1600), (1, 3600, 3600)):
    for o in (BF16, F32, F16):
        for steps in (0, 2):
            ok(["orth", b, m, n, o, steps], orth(batch(b, m, n), batch(b, m, n, o), steps=steps))
for rows, cols in ((M, 1), (M, 1 << 20), (1, 1 << 20)):
    ok(["quantise", rows, cols], lib.sqn_quantise(mat(rows, cols), quant(rows, cols), None))
    ok(["values", rows, cols], lib.sqn_quantised_values(quant(rows, cols), mat(rows, cols), None))
for points, units, cols in ((1, 1, 1), (16, 1 << 20, 64), (17, 1, 1), (17, 1 << 20, 520), ((1 << 29) - 64, 300, 100), (1 << 29, 1, 512),
                            ((1 << 29), 1, 7), (181_000, 181_000, 1 << 20), (16, 5, 1 << 20)):
    if (points + 63) // 64 * ((units + 63) // 64) > 1 << 23:
        continue
    ok(["layer", points, units, cols], layer(points, units, cols))
    ok(["product", points, units, cols], product(points, units, cols))
print(json.dumps(out))
""")
    assert len(got) > 80
    for name, status, detail, launched in got:
        assert status == 0 and launched > 0, (name, status, detail, launched)


def test_choice_of_kernels():
    """Few indices, points or rows take one launch and no scratch."""
    got = fake_hip.run(SETUP + r"""
import re
def names(status):
    assert status == 0, B.last_error()
    return [re.search(r"\d+([a-z_]+)_kernel", l.split()[0]).group(1) for l in launches()]
out = {}
fake.fake_reset()
out["g256"], out["g257"] = names(gradient(256, 90, 8)), names(gradient(257, 90, 8))
out["g81920"], out["g81921"] = names(gradient(81920, 5000, 8)), names(gradient(81921, 5000, 8))
out["rows24"], out["rows25"] = names(gradient(300, 1 << 24, 1)), names(gradient(300, (1 << 24) + 1, 1))
out["g1023"] = names(gradient(200000, 1023, 8))      # ten bits hold the mark of outside indices
out["g1024"] = names(gradient(200000, 1024, 8))
for m, n, o in ((128, 256, BF16), (256, 128, BF16), (129, 200, BF16), (128, 257, BF16), (128, 128, F32), (100, 129, F16)):
    out["o%d_%d_%d" % (m, n, o)] = names(orth(batch(2, m, n), batch(2, m, n, o), steps=2))
for b, m, n, o in ((1, 704, 1100, F32), (1, 705, 1100, F32), (1, 704, 1100, BF16), (7, 200, 200, BF16), (8, 200, 200, BF16)):
    assert orth(batch(b, m, n), batch(b, m, n, o), steps=1) == 0
    out["n%d_%d_%d" % (b, m, o)] = ["Narrow" in l for l in launches()[2:]]
for p, u, c in ((16, 300, 999), (17, 300, 999), (17, 256, 512), (17, 256, 513), (17, 257, 512), (17, 256, 7)):
    out["l%d_%d_%d" % (p, u, c)] = names(layer(p, u, c))
for p, c in ((4, 1 << 20), (5, 13107), (5, 13108), (16, 4096), (16, 4097)):
    out["f%d_%d" % (p, c)] = names(layer(p, 9, c))
out["p16"], out["p17"] = names(product(16, 9, 100)), names(product(17, 9, 100))
spaces = [lib.sqn_lookup_gradient_workspace(256, 90, 8), lib.sqn_orthogonalise_workspace(2, 128, 256, BF16),
          lib.sqn_quantised_layer_workspace(16, 300, 999), lib.sqn_quantised_layer_workspace(17, 256, 512)]
print(json.dumps([out, spaces]))
""")
    out, spaces = got
    assert spaces == [0, 0, 0, 0]
    tiles = ["norm", "start"] + ["gram", "square", "step"] * 2
    assert out["g256"] == ["direct"] and out["g257"] == ["bucket", "sum", "join"]
    assert out["g81920"] == out["rows24"] == ["bucket", "sum", "join"]
    assert out["g81921"] == ["count", "place"] * 2 + ["sum", "join"]
    assert out["rows25"] == ["count", "place"] * 3 + ["sum", "join"]
    assert out["g1023"] == ["count", "place", "sum", "join"]
    assert out["g1024"] == ["count", "place"] * 2 + ["sum", "join"]
    for name in ("o128_256_2", "o256_128_2", "o128_128_0"):
        assert out[name] == ["small"], (name, out[name])
    for name in ("o129_200_2", "o128_257_2", "o100_129_1"):
        assert out[name] == tiles, (name, out[name])
    for name in ("n1_704_0", "n1_704_2", "n7_200_2"):     # at most 256 narrow tiles, symmetric products only
        assert out[name] == [True, True, False], (name, out[name])
    for name in ("n1_705_0", "n8_200_2"):
        assert out[name] == [False] * 3, (name, out[name])
    for name in ("f4_1048576", "f5_13107", "f16_4096"):
        assert out[name] == ["few"], (name, out[name])
    for name in ("f5_13108", "f16_4097"):
        assert out[name] == ["quantise_packed", "product"], (name, out[name])
    assert out["l16_300_999"] == ["few"] and out["l17_300_999"] == ["quantise_packed", "product"]
    assert out["l17_256_512"] == ["layer"]
    for name in ("l17_256_513", "l17_257_512", "l17_256_7"):
        assert out[name] == ["quantise_packed", "product"], (name, out[name])
    assert out["p16"] == ["few"] and out["p17"] == ["pack", "product"]
