"""The example that fits heads by element type, run as a program would run it (GPU)."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location(
        "fit_type_heads", os.path.join(ROOT, "examples", "fit_type_heads.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_heads_and_their_gradients(example):
    # against automatic differentiation in 64 bits
    x, energy, species = example.frames(1, torch.device("cuda", 0), reps=3)
    heads = example.Heads(x.shape[1], 24, 118, species)
    for b in heads.b:
        b.normal_()
    e, kept = heads.energies(x)
    de = e - energy
    dw, db = heads.gradients(de, kept)

    params = [p.double().cpu().requires_grad_() for p in heads.w + heads.b]
    ids, rows = species.long().cpu(), x.double().cpu()

    def layer(i, x):
        return (x[:, None, :] @ params[i][ids])[:, 0] + params[3 + i][ids]

    y1 = torch.nn.functional.silu(layer(0, rows))
    y2 = torch.nn.functional.silu(layer(1, y1)) + y1
    want = layer(2, y2)[:, 0]
    # float32 layers of depth below 1,000 keep 2^-14 of what they add up
    assert (e.cpu().double() - want).abs().max() < 2.0 ** -14 * (1 + want.abs().max())
    (want - energy.cpu().double()).square().sum().div(2).backward()
    for got, p in zip(dw + db, params):
        assert torch.linalg.vector_norm(got.cpu().double() - p.grad) < 2.0 ** -12 * torch.linalg.vector_norm(p.grad)


def test_fit_learns(example):
    x, energy, species = example.frames(2, torch.device("cuda", 0), reps=4)
    target = energy - energy.mean()
    _, errors = example.fit(x, target, species, 118, hidden=32, steps=100)
    assert errors[-1] < 0.25 * errors[0]
    assert errors[-1] < 0.5 * target.square().mean().sqrt().item()
