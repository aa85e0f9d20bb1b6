"""The workers' step as a program runs it: forward, backward into G, aggregation, update."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import layers_oracle as lo

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def test_every_workers_gradient_through_two_blocks():
    """G against the 64-bit formulas on the checkpoints that forward kept.  In fp32 a product of at most 200 terms is off by at
    most 200 u of their magnitudes; through four of them in a row, and the sums over a worker's rows, 2e-5 of the norm."""
    import worker_step as ws
    gen = torch.Generator(device="cuda").manual_seed(3)
    model = ws.Model(96, 200, 2, gen)
    sizes = [40, 0, 77, 1, 130]
    rows = sum(sizes)
    x = torch.randn(rows, 96, generator=gen, device="cuda")
    dx = torch.randn(rows, 96, generator=gen, device="cuda")
    _, kept = model.forward(x)
    G = torch.full((5, model.n + 7), -3.0, device="cuda")
    model.backward(dx, kept, sizes, G)
    assert bool((G[:, model.n:] == -3.0).all())
    d = _host(dx)
    for b, place, (rstd, normalised, active) in zip(reversed(model.blocks()), reversed(model.places), reversed(kept)):
        a = lo.unpack(active.codes.cpu().numpy(), active.exponents.cpu().numpy(), 200)
        xhat = lo.unpack(normalised.codes.cpu().numpy(), normalised.exponents.cpu().numpy(), 96)
        want = {}
        want["W2"], want["b2"] = lo.linear_grad(d, a, sizes)
        du = (d @ _host(b["W2"])) * (a > 0)
        want["W1"], want["b1"] = lo.linear_grad(du, xhat, sizes, _host(b["gamma"]), _host(b["beta"]))
        d, want["gamma"], want["beta"] = lo.layer_norm_backward(du @ _host(b["W1"]), xhat, _host(rstd), sizes, _host(b["gamma"]), d)
        for name, (at, count, _) in place.items():
            got = _host(G[:, at:at + count])
            for w in range(5):
                ref = want[name][w].reshape(-1)
                assert np.linalg.norm(got[w] - ref) <= 2e-5 * np.linalg.norm(ref), (name, w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_with_byzantine_workers(dtype):
    import worker_step as ws
    fa = ws.train(dtype=dtype)
    assert fa[-1] < 0.5 * fa[0]
    assert ws.train(dtype=dtype, aggregate="krum")[-1] < 0.5 * fa[0]
    mean = ws.train(dtype=dtype, aggregate="mean")[-1]
    assert not mean < 1.3 * fa[-1]            # (or NaN)
