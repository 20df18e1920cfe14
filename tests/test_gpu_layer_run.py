"""Layers and dropout as a program uses them: a training step of a network on
looked-up rows, eager and captured in a HIP graph whose mask moves on with each
replay, on two streams at once, and the example."""
import numpy as np
import pytest
import torch

from tests import layer_util as U

pytestmark = pytest.mark.gpu


def network(dtype, gen, table=900, cols=42, units=72, heads=50):
    def draw(*shape, spread=1.0):
        return (spread * torch.randn(*shape, generator=gen)).to(dtype).cuda()
    return {"table": draw(table, cols), "w1": draw(units, cols, spread=cols ** -0.5), "b1": draw(units, spread=0.1),
            "w2": draw(units, units, spread=units ** -0.5), "w3": draw(heads, units, spread=units ** -0.5)}


def forward(learn, s, ids, step):
    rows = learn.lookup(s["table"], ids)
    h = learn.layer(rows, s["w1"], s["b1"], "relu", dropout=0.1, seed=1, step=step)
    h = learn.layer(h, s["w2"], None, "gelu", residual=h, dropout=0.2, seed=2, step=step)
    return learn.layer(learn.dropout(h, 0.3, seed=3, step=step), s["w3"], dtype=torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("points", [5, 300])
def test_training_step(dtype, points):
    """The gradients of a whole step against the same network in 64 bits with the
    same masks.  Layers' roundings pass on through the ones behind them, so the
    bound is one on the whole tensor: each of the six values a gradient goes
    through is off by half a step of its type at most, sums of them by as much of
    their sizes' norm, and the slopes of rows near a relu's border may flip in a
    share of about a step of all rows (a flip moves a gradient by its own size)."""
    from paper_2204_02585_amd import learn
    gen = torch.Generator().manual_seed(points)
    s = {k: v.requires_grad_() for k, v in network(dtype, gen).items()}
    ids = torch.randint(0, 900, (points,), generator=gen).cuda()
    step = torch.tensor([7], device="cuda")
    y = forward(learn, s, ids, step)
    g = torch.randn(y.shape, generator=gen).cuda()
    got = torch.autograd.grad(y, list(s.values()), g)

    def share(shape, p, seed):
        return torch.from_numpy(U.share(*shape, p, seed + 7))
    d = {k: v.detach().double().cpu().requires_grad_() for k, v in s.items()}
    h = torch.relu(d["table"][ids.cpu()] @ d["w1"].t() + d["b1"]) * share((points, 72), 0.1, 1)
    h = torch.nn.functional.gelu(h @ d["w2"].t()) * share((points, 72), 0.2, 2) + h
    want_y = (h * share((points, 72), 0.3, 3)) @ d["w3"].t()
    want = torch.autograd.grad(want_y, list(d.values()), g.double().cpu())
    half = U.UNIT[dtype]
    for name, a, b in zip(("y", *s), (y, *got), (want_y, *want)):
        a = a.detach().double().cpu()
        off = ((a - b).norm() / b.norm()).item()
        assert off < 6 * half + 3 * (2 * half) ** 0.5 * (dtype != torch.float32) + 1e-4 * (dtype == torch.float32), (name, off)


def test_training_step_in_a_graph():
    """Captured once, with autograd's backward pass inside, and replayed with other
    inputs and the step moved on: the same bits as eager steps, and another mask
    each time."""
    from paper_2204_02585_amd import learn
    gen = torch.Generator().manual_seed(5)
    s = network(torch.bfloat16, gen)
    ids = torch.randint(0, 900, (20000,), generator=gen).cuda()
    step = torch.tensor([0], device="cuda")
    g = torch.randn(20000, 50, generator=gen).cuda()

    def run(step):
        leaves = {k: v.detach().requires_grad_() for k, v in s.items()}
        y = forward(learn, leaves, ids, step)
        grads = torch.autograd.grad(y, list(leaves.values()), g)
        x, pre = s["table"], torch.empty(900, 72, dtype=torch.bfloat16, device="cuda")
        small = learn.layer(x[:7], s["w1"], s["b1"], "silu", pre=pre[:7])
        return [y.detach(), *grads, small, *learn.layer_gradient(small, x[:7], s["w1"], pre[:7], "silu"),
                *learn.layer_gradient(y.detach()[:, :48].bfloat16(), s["w2"][:1, :40].expand(20000, 40), s["w2"][:48, :40])]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(step)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(step)
        step.add_(1)
    seen = []
    for k in range(4):
        ids.copy_(torch.randint(0, 900, (20000,), generator=gen))
        for name, v in network(torch.bfloat16, gen).items():
            s[name].copy_(v)
        step.fill_(10 + k)
        want = run(torch.tensor([10 + k], device="cuda"))
        torch.cuda.synchronize()
        for t in got:
            t.zero_()
        graph.replay()
        for n, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (k, n)
        assert step.item() == 11 + k
        seen.append(got[0].clone())
    assert not any(torch.equal(seen[0], t) for t in seen[1:])


def test_two_streams_at_once():
    """Calls on two streams share nothing."""
    from paper_2204_02585_amd import learn
    gen = torch.Generator().manual_seed(6)
    x = [torch.randn(500, 2000, generator=gen).cuda() for _ in range(2)]
    w = [torch.randn(300, 2000, generator=gen).cuda() for _ in range(2)]
    want = [(learn.layer(x[k], w[k], dropout=0.5, seed=k), *learn.layer_gradient(x[k][:, :300], x[k], w[k])) for k in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for k, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[k].append((learn.layer(x[k], w[k], dropout=0.5, seed=k), *learn.layer_gradient(x[k][:, :300], x[k], w[k])))
    torch.cuda.synchronize()
    for k in range(2):
        for run in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(run, want[k]))


def test_far_rows():
    """Rows whose offsets pass 32 bits: the last of a tall matrix and of one with a
    wide stride."""
    from paper_2204_02585_amd import learn
    points = (1 << 31) // 1024 + 40                    # 4 GB of binary16, 2^31 elements and more
    x = torch.zeros(points, 1024, dtype=torch.float16, device="cuda")
    gen = torch.Generator().manual_seed(7)
    last = torch.randn(70, 1024, generator=gen).half().cuda()
    w = (torch.randn(16, 1024, generator=gen) / 32).half().cuda()
    x[-70:] = last
    y = learn.layer(x, w)
    z, off, *_ = U.layer(last, w, None, None, None, 0.0, 0, torch.float16)
    U.assert_within(y[-70:], z, off)
    assert not y[:-70].any()
    _, dw, _ = learn.layer_gradient(y, x, w, for_x=False)
    # the sum of y's last rows, in binary16 as they are: everything before is zero
    want = U.gradients(y[-70:], last, w, None, None, 0.0, 0)[1]
    bound = want[1] + 2 * U.F32 * points * (np.abs(U.double(y[-70:])).T @ np.abs(U.double(last)))
    U.assert_within(dw, want[0], bound)
    # the mask's words of rows past 2^32 elements, and in place
    drop = learn.dropout(x, 0.5, seed=9, out=x)
    tail = drop[-70:].float()
    pairs, first = 512, points - 70
    with np.errstate(over="ignore"):
        key = U.mix(np.array([9], dtype=np.uint64))
        n = np.arange(first * pairs + 1, points * pairs + 1, dtype=np.uint64)
        words = U.mix(n * np.uint64(0x9E3779B97F4A7C15) + key)
    bits = np.stack([words & np.uint64(0xFFFFFFFF), words >> np.uint64(32)], 1).reshape(70, 1024)
    keep = torch.from_numpy(bits >= np.uint64(1 << 31)).cuda()
    assert torch.equal(tail, torch.where(keep, last.float() * 2, torch.zeros_like(tail)))
    del x, y, drop
    # four rows, a gigabyte and more apart
    flat = torch.zeros(3 * (1 << 29) + 2048, dtype=torch.float16, device="cuda")
    far = flat.as_strided((4, 1024), (1 << 29, 1))
    far.copy_(last[:4])
    U.assert_within(learn.layer(far, w), *U.layer(last[:4], w, None, None, None, 0.0, 0, torch.float16)[:2])
    many = flat.as_strided((20, 1024), (1 << 26, 1))
    many.copy_(last[:20])
    U.assert_within(learn.layer(many, w), *U.layer(last[:20], w, None, None, None, 0.0, 0, torch.float16)[:2])
    dx, dw, _ = learn.layer_gradient(learn.layer(many, w), many, w)
    g = learn.layer(last[:20].contiguous(), w)
    (vx, ox), (vw, ow), _ = U.gradients(learn.layer(many, w), last[:20], w, None, None, 0.0, 0)
    U.assert_within(dx, vx, ox)
    U.assert_within(dw, vw, ow)


def test_example_with_layers():
    """The example's layers run as the library's, with a mask, and their gradients
    reach the table and every layer."""
    from examples import fit_texels
    r = fit_texels.fit(side=24, points=1024, steps=3, dropout=0.1)
    assert np.isfinite(r["last_loss"])
    gen = torch.Generator().manual_seed(1)
    layers = [torch.randn(u, c, generator=gen).cuda().requires_grad_() for u, c in ((32, 16), (32, 32), (3, 32))]
    rows = torch.randn(100, 16, generator=gen).cuda().requires_grad_()
    y = fit_texels.decode(rows, layers, dropout=0.25, seed=4)
    got = torch.autograd.grad(y, [rows, *layers], torch.ones_like(y))
    d = [t.detach().double().cpu().requires_grad_() for t in (rows, *layers)]
    h = torch.relu(torch.relu(d[0] @ d[1].t()) @ d[2].t()) * torch.from_numpy(U.share(100, 32, 0.25, 4))
    want = torch.autograd.grad((h @ d[3].t()).sum(), d)
    for a, b in zip(got, want):
        # sums of at most 132 binary32 terms through three layers, and flips at a relu's border in a share of 2^-20
        assert ((a.double().cpu() - b).norm() / b.norm()).item() < 1e-3
