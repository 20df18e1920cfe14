"""The operators on learned tables and layers captured in one HIP graph and
replayed with other inputs, eager calls and synchronisations between the
replays: the same bits as eager calls every time."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_operators_in_a_graph():
    from paper_2204_02585_amd import learn
    gen = torch.Generator().manual_seed(3)

    def draw():
        return {"table": torch.randn(900, 40, generator=gen).cuda(), "ids": torch.randint(-5, 905, (3000,), generator=gen).cuda(),
                "few": torch.randint(0, 900, (100,), generator=gen).cuda(), "many": torch.randint(0, 900, (50000,), generator=gen).cuda(),
                "rows": torch.randn(50000, 40, generator=gen).cuda(),
                "update": torch.randn(2, 100, 130, generator=gen).cuda(), "large": torch.randn(1, 300, 500, generator=gen).cuda(),
                "x": torch.randn(1000, 300, generator=gen).cuda(), "w": torch.randn(400, 300, generator=gen).cuda()}

    def run(s):
        q = learn.quantise(s["w"])
        rows = learn.lookup(s["table"], s["ids"], scale=0.5)
        return [rows, learn.lookup_gradient(rows, s["ids"], 900), learn.lookup_gradient(s["rows"][:100], s["few"], 900),
                learn.lookup_gradient(s["rows"], s["many"], 900, dtype=torch.bfloat16),
                learn.orthogonalise(s["update"]), learn.orthogonalise(s["large"]), learn.orthogonalise(s["large"], dtype=torch.float32),
                q.values(), learn.product(s["x"], q), learn.product(s["x"][:3], q, relu=True),
                learn.product(s["x"][:, :256].contiguous(), learn.quantise(s["w"][:200, :256].contiguous()))]

    state = draw()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(state)
    for _ in range(4):
        for name, value in draw().items():
            state[name].copy_(value)
        want = run(state)
        torch.cuda.synchronize()
        for g in got:
            g.zero_()
        graph.replay()
        for k, (g, w) in enumerate(zip(got, want)):
            assert torch.equal(g, w), k
