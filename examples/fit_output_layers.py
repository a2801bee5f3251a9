"""Fits output layers to given embeddings: each node's PinSage embedding, through a
hidden layer with a weight per node type (pins, boards) and a shared output layer,
is brought to a target embedding (say, the space an earlier model's index was built
in, so that a retrained model can be served beside it).

Every product runs in the library: the forward pass of both layers (the residual
-target makes the output layer return y - target, the squared error's gradient),
their backward passes, and the optimiser step that orthogonalises each weight's
update. Run it from the repository's root:

    python examples/fit_output_layers.py --steps 60 --dtype bf16
"""

from __future__ import annotations

import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_1806_01973_amd as ps
import synth


def node_embeddings(workload: str):
    """All nodes' embeddings (pins, then boards) of a synthetic graph, fp32."""
    wl = synth.WORKLOADS[workload]
    data = synth.make_workload(wl)
    graph = ps.DeviceGraph(data["offsets"], data["col"], wl.num_pins, wl.num_boards)
    layers = [ps.DeviceLayer(L["Q"], L["q"], L["W"], L["w"]) for L in data["layers"]]
    job = ps.EmbedAll(graph, layers, wl.walks, wl.hops, wl.T, wl.seed)
    return job.run(torch.as_tensor(data["x"]).cuda()), wl.num_pins


def teacher(h: torch.Tensor, pins: int, d_out: int, gen: torch.Generator) -> torch.Tensor:
    """The targets: another map of the embeddings, different for pins and boards."""
    maps = [torch.randn(h.shape[1], d_out, generator=gen, device="cuda") / math.sqrt(h.shape[1])
            for _ in range(2)]
    z = torch.cat([torch.tanh(4 * h[:pins] @ maps[0]), torch.tanh(4 * h[pins:] @ maps[1])])
    return z / z.norm(dim=1, keepdim=True)


def fit(workload: str = "tiny", hidden: int = 128, d_out: int = 64, steps: int = 60,
        lr: float = 0.02, dtype: torch.dtype = torch.float32, seed: int = 0) -> list:
    """Returns the mean squared error (per row) before each step and after the last."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    h, pins = node_embeddings(workload)
    n, d_in = h.shape
    target = teacher(h, pins, d_out, gen)
    # Rows of unit norm have small entries; the layers see them at unit scale.
    x = (h * math.sqrt(d_in)).to(dtype)
    minus_target = (-target * math.sqrt(d_out)).to(dtype)
    offsets = torch.tensor([0, pins, n], dtype=torch.int64, device="cuda")

    def weight(*shape):
        return (torch.randn(shape, generator=gen, device="cuda") / math.sqrt(shape[-1])).to(dtype)

    W1, b1 = weight(2, hidden, d_in), torch.zeros(2, hidden, device="cuda")
    W2, b2 = weight(d_out, hidden), torch.zeros(d_out, device="cuda")
    m1, m2 = torch.zeros(W1.shape, device="cuda"), torch.zeros(W2.shape, device="cuda")
    rows = torch.tensor([[pins], [n - pins]], device="cuda")

    def forward():
        y1, u1 = ps.dense_forward(x, W1, b1, "gelu", offsets=offsets, want_preact=True)
        return y1, u1, ps.dense_forward(y1, W2, b2, residual=minus_target)

    losses = []
    for step in range(steps):
        y1, u1, error = forward()
        losses.append((error.float().square().sum(1).mean() / d_out).item())
        dy1, dW2, db2 = ps.dense_backward(error, y1, W2)
        _, dW1, db1 = ps.dense_backward(dy1, x, W1, u1, "gelu", offsets=offsets, need_dx=False)
        rate = lr * (1 - step / steps)
        # The update's direction is orthogonalised: its size does not depend on dy's scale.
        ps.muon_step(W1, dW1, m1, lr=rate, weight_decay=0.01)
        ps.muon_step(W2, dW2, m2, lr=rate, weight_decay=0.01)
        b1 -= rate * db1 / rows
        b2 -= rate * db2 / n
    losses.append((forward()[2].float().square().sum(1).mean() / d_out).item())
    return losses


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--workload", default="tiny", choices=sorted(synth.WORKLOADS))
    p.add_argument("--hidden", type=int, default=128)
    p.add_argument("--out", type=int, default=64)
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = p.parse_args()
    dtype = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    losses = fit(a.workload, a.hidden, a.out, a.steps, dtype=dtype)
    for k in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {k:4d}  mean squared error {losses[k]:.4f}", flush=True)
    print(f"after {a.steps} steps {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
