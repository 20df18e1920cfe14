"""Cases of a trained layer and of dropout (paper_2204_02585_amd.learn), what
each computes in plain torch operations, and the same in 64 bits.

Three kinds of call:

  layer     y = D(act(x w^T + b)) + residual, with D the dropout of the mask
            below (where p > 0); a training call keeps z = x w^T + b too
  gradient  from dy and the kept z: dx, dw and db of such a layer
  dropout   D(x), or D(x) + residual; with the same seed it is its own gradient

The mask is never stored.  Element (row, col) of `cols` columns is kept or
dropped by 32 bits of SplitMix64's word number row ceil(cols / 2) + col / 2 (the
low half for an even column) of the stream that starts at the mixed seed:
dropped below round(p 2^32), times 1 / (1 - p) otherwise.

In a program the layers are the networks whose outputs the caches hold, or a
model's linear layers, while they are trained or asked.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _layer(name, points, cols, units, dtype="bf16", act=None, bias=True, residual=False, p=0.0, keep=False):
    """keep: the call of a training step, which returns z too."""
    return dict(name=name, kind="layer", points=points, cols=cols, units=units, dtype=dtype, act=act or "none", bias=bias,
                residual=residual, p=p, keep=keep)


def _gradient(name, points, cols, units, dtype="bf16", act=None, p=0.0):
    return dict(name=name, kind="gradient", points=points, cols=cols, units=units, dtype=dtype, act=act or "none", p=p)


def _dropout(name, rows, cols, dtype="bf16", p=0.1, residual=False):
    return dict(name=name, kind="dropout", rows=rows, cols=cols, dtype=dtype, p=p, residual=residual)


def listed():
    return [
        # one token through a large layer and onto its residual: latency
        _layer("layer_step", 1, 4096, 4096, act="silu", residual=True),
        # a hidden layer of a position network on a 256 grid
        _layer("layer_points", 256 * 256, 256, 256, dtype="f16", act="relu"),
        # a network's first layer in binary32: encoded positions, an odd number of points
        _layer("layer_encoded", 50001, 42, 256, dtype="f32", act="relu", keep=True),
        # a training batch through a wide layer
        _layer("layer_wide", 8192, 4096, 8192, act="gelu", p=0.1, keep=True),
        # a layer of middling size in binary32, onto its residual
        _layer("layer_residual", 2048, 1024, 2048, dtype="f32", residual=True, p=0.1),
        # a hidden layer of a position network in training
        _gradient("gradient_points", 256 * 256, 256, 256, dtype="f16", act="relu", p=0.1),
        # the head of a position network, 2 + 6 D outputs of D = 8, an odd number of points, binary32
        _gradient("gradient_head", 50001, 256, 50, dtype="f32"),
        # a few requests' points through a square layer
        _gradient("gradient_few", 100, 2048, 2048, act="silu"),
        # the wide layer of a training batch
        _gradient("gradient_wide", 8192, 4096, 8192, act="gelu", p=0.1),
        # a few rows: latency
        _dropout("dropout_step", 32, 1024),
        # a training batch's activations onto their residual
        _dropout("dropout_residual", 16384, 8192, residual=True),
        # odd rows in binary32, half of them dropped
        _dropout("dropout_odd", 65537, 257, dtype="f32", p=0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["layer", "layer", "gradient", "gradient", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    p = rng.choice([0.0, 0.1, 0.5])
    if kind == "dropout":
        rows = _log(rng, 1, 65536)
        cols = min(_log(rng, 1, 16384), (1 << 27) // rows)
        return _dropout("", rows, cols, dtype, rng.choice([0.05, 0.1, 0.5]), rng.random() < 0.5)
    points, cols, units = _log(rng, 1, 65536), _log(rng, 16, 8192), _log(rng, 16, 8192)
    points = max(1, min(points, (1 << 36) // (cols * units)))
    if rng.random() < 0.6:
        # most layers have sizes that fill whole lines
        cols, units = -(-cols // 8) * 8, -(-units // 8) * 8
    act = rng.choice([None, "relu", "gelu", "silu"])
    if kind == "gradient":
        return _gradient("", points, cols, units, dtype, act, p)
    return _layer("", points, cols, units, dtype, act, rng.random() < 0.8, rng.random() < 0.5, p, rng.random() < 0.5)


# ---- inputs

def _randn(shape, gen, dtype="f32", spread=1.0):
    return (spread * torch.randn(shape, generator=gen, device="cuda")).to(DTYPES[dtype])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    # the mask's seed: a training step's own
    s = {"case": case, "seed": 1000003 * seed + 17}
    dtype = case["dtype"]
    if case["kind"] == "dropout":
        s["x"] = _randn((case["rows"], case["cols"]), gen, dtype)
        s["residual"] = _randn((case["rows"], case["cols"]), gen, dtype) if case["residual"] else None
        return s
    points, cols, units = case["points"], case["cols"], case["units"]
    s["x"] = _randn((points, cols), gen, dtype)
    s["w"] = _randn((units, cols), gen, dtype, math.sqrt(2.0 / cols))
    if case["kind"] == "layer":
        s["bias"] = _randn((units,), gen, "f32", 0.1) if case["bias"] else None
        s["residual"] = _randn((points, units), gen, dtype) if case["residual"] else None
        return s
    s["grad"] = _randn((points, units), gen, dtype, 1e-2)
    # what the forward call kept
    s["z"] = None if case["act"] == "none" else (s["x"].float() @ s["w"].float().t()).to(DTYPES[dtype])
    return s


# ---- the plain forms

GOLDEN, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _mix(z):
    """SplitMix64's output function on int64 tensors, whose products wrap."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(MIX1)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(MIX2)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _kept(rows, cols, p, seed):
    """Truth values [rows, cols]: what the mask keeps."""
    pairs = (cols + 1) // 2
    key = _mix(torch.tensor(_signed(seed), dtype=torch.int64, device="cuda"))
    n = torch.arange(1, rows * pairs + 1, dtype=torch.int64, device="cuda")
    word = _mix(n * _signed(GOLDEN) + key)
    bound = int(round(p * 4294967296.0))
    keep = torch.stack(((word & 0xFFFFFFFF) >= bound, ((word >> 32) & 0xFFFFFFFF) >= bound), dim=1)
    return keep.view(rows, 2 * pairs)[:, :cols]


def _drop(v, case, seed):
    p = case["p"]
    if p == 0.0:
        return v
    return torch.where(_kept(v.shape[0], v.shape[1], p, seed), v * (1.0 / (1.0 - p)), torch.zeros_like(v))


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _plain(s):
    case = s["case"]
    to = DTYPES[case["dtype"]]
    if case["kind"] == "dropout":
        y = _drop(s["x"].float(), case, s["seed"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(to)
    x, w = s["x"].float(), s["w"].float()
    if case["kind"] == "layer":
        z = x @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _drop(_act(z, case["act"]), case, s["seed"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return (y.to(to), z.to(to)) if case["keep"] else y.to(to)
    dz = _drop(s["grad"].float(), case, s["seed"])
    if s["z"] is not None:
        dz = dz * _slope(s["z"].float(), case["act"])
    return (dz @ w).to(to), (dz.t() @ x).to(to), dz.sum(dim=0)


def run(s):
    if not own:
        return _plain(s)
    from paper_2204_02585_amd import learn
    case = s["case"]
    if case["kind"] == "dropout":
        return learn.dropout(s["x"], case["p"], seed=s["seed"], residual=s["residual"])
    act = None if case["act"] == "none" else case["act"]
    if case["kind"] == "gradient":
        return learn.layer_gradient(s["grad"], s["x"], s["w"], pre=s["z"], activation=act, dropout=case["p"], seed=s["seed"])
    options = dict(bias=s["bias"], activation=act, residual=s["residual"], dropout=case["p"], seed=s["seed"])
    if not case["keep"]:
        return learn.layer(s["x"], s["w"], **options)
    z = torch.empty((case["points"], case["units"]), dtype=s["x"].dtype, device=s["x"].device)
    return learn.layer(s["x"], s["w"], pre=z, **options), z


def work(case):
    e = SIZE[case["dtype"]]
    if case["kind"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * e * (3 if case["residual"] else 2), "flops": n}
    m, k, n = case["points"], case["cols"], case["units"]
    if case["kind"] == "layer":
        outs = m * n * (1 + int(case["keep"]) + int(case["residual"]))
        return {"bytes": (m * k + n * k + outs) * e + 4 * n * int(case["bias"]), "flops": 2 * m * n * k}
    return {"bytes": (2 * (m * k + n * k) + m * n * (1 if case["act"] == "none" else 2)) * e + 4 * n, "flops": 4 * m * n * k}


# ---- 64 bits, from the definitions

def _exact_share(rows, cols, p, seed):
    """1 / (1 - p) where an element is kept and 0 where it is not, in binary64,
    a few rows at a time: the words as halves of 32 bits, whose products stay
    within 64."""
    low = (1 << 32) - 1

    def times(a, c):
        # (hi, lo) by a constant, modulo 2^64
        hi, lo = a
        c_hi, c_lo = c >> 32, c & low
        # lo c_lo in parts of 16 bits of the constant
        part0 = lo * (c_lo & 0xFFFF)
        part1 = lo * (c_lo >> 16)
        total = part0 + ((part1 & 0xFFFF) << 16)
        new_lo = total & low
        carry = (total >> 32) + (part1 >> 16)
        cross = sum(((v * (d & 0xFFFF)) & low) + ((((v * (d >> 16)) & 0xFFFF) << 16)) for v, d in ((lo, c_hi), (hi, c_lo)))
        return (carry + cross) & low, new_lo

    def plus(a, b):
        lo = a[1] + b[1]
        return (a[0] + b[0] + (lo >> 32)) & low, lo & low

    def shifted(a, k):
        # a ^ (a >> k) for k < 32
        hi, lo = a
        return hi ^ (hi >> k), lo ^ ((lo >> k) | ((hi << (32 - k)) & low))

    def mixed(a):
        return shifted(times(shifted(times(shifted(a, 30), MIX1), 27), MIX2), 31)

    pairs = -(-cols // 2)
    seed &= (1 << 64) - 1
    start = torch.tensor([seed >> 32, seed & low], dtype=torch.int64, device="cuda")
    key = mixed((start[0], start[1]))
    out = torch.empty((rows, cols), dtype=torch.float64, device="cuda")
    share, bound = 1.0 / (1.0 - p), int(math.floor(p * 2.0 ** 32 + 0.5))
    chunk = max(1, (1 << 24) // pairs)
    for at in range(0, rows, chunk):
        count = min(chunk, rows - at)
        number = torch.arange(at * pairs + 1, (at + count) * pairs + 1, dtype=torch.int64, device="cuda")
        hi, lo = mixed(plus(times((number >> 32, number & low), GOLDEN), key))
        both = torch.empty((count, 2 * pairs), dtype=torch.float64, device="cuda")
        both[:, 0::2] = (lo >= bound).view(count, pairs) * share
        both[:, 1::2] = (hi >= bound).view(count, pairs) * share
        out[at:at + count] = both[:, :cols]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    act = case["act"] if case["kind"] != "dropout" else "none"

    def normal(z):
        # the share of a normal distribution below z
        return torch.special.ndtr(z)

    def dropped(v):
        return v * _exact_share(v.shape[0], v.shape[1], case["p"], s["seed"]) if case["p"] else v

    if case["kind"] == "dropout":
        y = dropped(s["x"].double())
        return y if s["residual"] is None else y.add_(s["residual"])
    x, w = s["x"].double(), s["w"].double()
    if case["kind"] == "layer":
        z = torch.mm(x, w.t().contiguous())
        if s["bias"] is not None:
            z += s["bias"].double()
        y = {"none": lambda: z, "relu": lambda: torch.clamp(z, min=0.0), "gelu": lambda: z * normal(z),
             "silu": lambda: z * torch.sigmoid(z)}[act]()
        y = dropped(y)
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return (y, z) if case["keep"] else y
    dz = dropped(s["grad"].double())
    if s["z"] is not None:
        z = s["z"].double()
        if act == "relu":
            dz = torch.where(z > 0, dz, torch.zeros_like(dz))
        elif act == "gelu":
            dz = dz * (normal(z) + z * torch.exp(-z.square() / 2.0) / math.sqrt(2.0 * math.pi))
        else:
            up = torch.sigmoid(z)
            dz = dz * (up + z * up * torch.sigmoid(-z))
    return torch.mm(dz, w), torch.mm(dz.t().contiguous(), x), torch.sum(dz, dim=0)
