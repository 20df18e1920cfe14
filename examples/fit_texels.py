"""A plane of learned texels and a small decoder, trained and then held in 4 bits.

A coarse table of features, one row per texel of an n x n plane, is read by
index; three layers turn a row into a colour, the hidden ones' outputs thinned
by dropout if asked to.  Training moves the table by its lookup gradient and the
layers by orthogonalised momentum (Muon); then the layers are put into 4-bit
blocks and the plane is decoded from them, once for all texels and once for a
handful of them, as a cursor would ask.

    python -m examples.fit_texels [--side 256] [--steps 200] [--dropout 0.0]
"""
import argparse

import torch

from paper_2204_02585_amd import learn


def target(side: int, device) -> torch.Tensor:
    """Smooth colours with an edge, [side * side, 3] in [0, 1]."""
    axis = torch.linspace(-1.0, 1.0, side, device=device)
    v, u = torch.meshgrid(axis, axis, indexing="ij")
    inside = ((u * u + v * v) < 0.5).float()
    return torch.stack([0.5 + 0.5 * torch.sin(5 * u + 2 * v), 0.25 + 0.5 * inside, 0.5 + 0.4 * torch.cos(4 * v * u)], -1).reshape(-1, 3)


def decode(rows: torch.Tensor, layers, dropout: float = 0.0, seed: int = 0) -> torch.Tensor:
    """Colours of rows [n, features]; a mask of seed `seed` on the last hidden layer."""
    first, second, head = layers
    hidden = learn.layer(rows, first, activation="relu")
    hidden = learn.layer(hidden, second, activation="relu", dropout=dropout, seed=seed)
    return learn.layer(hidden, head)


def fit(side: int = 256, features: int = 32, units: int = 128, points: int = 16384, steps: int = 200,
        device="cuda", seed: int = 0, dropout: float = 0.0) -> dict:
    gen = torch.Generator(device="cpu").manual_seed(seed)

    def draw(*shape, spread):
        return (spread * torch.randn(*shape, generator=gen)).to(device)

    colours = target(side, device)
    table = draw(side * side, features, spread=0.1).requires_grad_()
    first = draw(units, features, spread=features ** -0.5).requires_grad_()
    second = draw(units, units, spread=units ** -0.5).requires_grad_()
    head = draw(3, units, spread=units ** -0.5).requires_grad_()
    layers = [first, second, head]
    momentum = [torch.zeros_like(w) for w in layers]

    losses = []
    for step in range(steps):
        ids = torch.randint(0, side * side, (points,), generator=gen).to(device)
        rows = learn.lookup(table, ids)
        loss = torch.mean((decode(rows, layers, dropout, seed=step) - colours[ids]) ** 2)
        loss.backward()
        rate = 0.02 * (1.0 - step / steps)
        with torch.no_grad():
            # a texel is in few of a step's points: its own step is normalised by
            # its gradient's size, rows that no point touched stay where they are
            g = table.grad
            table -= 4 * rate * g / g.norm(dim=1, keepdim=True).clamp_min(1e-12)
            for w, m in zip(layers, momentum):
                m.mul_(0.9).add_(w.grad)
                # a step of one size in every direction of the layer
                w -= rate * learn.orthogonalise(m, dtype=torch.float32)
            for p in (table, *layers):
                p.grad = None
        losses.append(loss.detach())

    with torch.no_grad():
        exact = decode(table, layers)
        q = [learn.quantise(w) for w in layers]

        def decode_blocks(rows):
            h = learn.product(rows, q[0], relu=True)
            return learn.product(learn.product(h, q[1], relu=True), q[2])

        blocks = decode_blocks(table)                                       # the whole plane
        few = torch.arange(0, side * side, max(1, side * side // 5), device=device)[:5]
        asked = learn.lookup(table, few)                                    # a handful of texels
        hidden = learn.product(table, q[0], relu=True)
        apart = (learn.product(asked, q[0], relu=True) - hidden[few]).abs().max() / hidden.abs().max()

    def error_of(x, of):
        return float(torch.mean((x - of) ** 2))

    stored = sum(t.codes.numel() + t.scales.numel() for t in q)
    return {"first_loss": float(losses[0]), "last_loss": float(losses[-1]),
            "exact": error_of(exact, colours), "blocks": error_of(blocks, colours),
            "few": error_of(decode_blocks(asked), colours[few]), "few_apart": float(apart),
            "bytes_exact": sum(4 * w.numel() for w in layers), "bytes_blocks": stored}


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--side", type=int, default=256)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--dropout", type=float, default=0.0)
    args = ap.parse_args()
    r = fit(side=args.side, steps=args.steps, dropout=args.dropout)
    print(f"loss {r['first_loss']:.5f} -> {r['last_loss']:.5f} over {args.steps} steps")
    print(f"plane decoded: squared error {r['exact']:.5f} exact, {r['blocks']:.5f} from 4-bit blocks "
          f"({r['bytes_exact']} -> {r['bytes_blocks']} bytes of layers)")
    print(f"five texels alone: squared error {r['few']:.5f}, their first layer within {r['few_apart']:.1e} of the plane's")


if __name__ == "__main__":
    main()
