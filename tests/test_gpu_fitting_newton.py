"""Newton-Schulz iterations and Muon updates as exact as float32, on tiles of both sizes (GPU).

What the formula is off in float32 says how its steps make errors grow.  The kernels round
an operand to 2^-22 of itself where float32 rounds to 2^-24, so their results may be four
times as far from the formula in 64 bits, and then they round to the output's type once.
"""
import pytest
import torch

import paper_2608_19041_amd as dp

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
F64, U = torch.float64, 2.0 ** -24
ABC = (3.4445, -4.7750, 2.0315)


def newton(g, dtype, steps=5, eps=1e-7):
    a, b, c = ABC
    x = g.to(dtype)
    turned = x.shape[-2] > x.shape[-1]
    x = x.mT.contiguous() if turned else x
    x = x / (torch.linalg.matrix_norm(x.to(F64), keepdim=True).to(dtype) + eps)
    for _ in range(steps):
        p = x @ x.mT.contiguous()
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.mT if turned else x


def gradient(g, shape, dtype):
    # a gradient's spectrum falls off
    fall = torch.arange(1, shape[-1] + 1, device="cuda", dtype=torch.float32).pow(-0.5)
    return (torch.randn(*shape, generator=g, device="cuda") * fall * 1e-3).to(dtype)


SMALL = [(64, 1, 1), (64, 1, 9), (64, 9, 1), (64, 2, 8), (16, 16, 8), (16, 4, 344), (16, 64, 64), (16, 65, 63),
         (4, 16, 688), (4, 129, 127), (2, 256, 1376), (2, 541, 384), (2, 130, 700), (2, 33, 2000)]
LARGE = [(175, 541, 384), (236, 384, 384), (200, 380, 384), (260, 230, 500)]   # 128 x 128 tiles


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", SMALL + LARGE)
def test_orthogonalize(shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(shape[1] * 1000 + shape[2])
    m = gradient(g, shape, DT[dtype])
    (o,) = dp.orthogonalize([m])
    want = newton(m, F64)
    least = (want.to(DT[dtype]).to(F64) - want).norm()
    bound = 1.01 * least + 4 * (newton(m, torch.float32).to(F64) - want).norm() + 2 * U * want.norm()
    off = (o.to(F64) - want).norm()
    assert off <= bound, (off / want.norm()).item()


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shapes", [SMALL, LARGE[:1]], ids=["small", "large"])
def test_muon_step(shapes, dtype, nesterov):
    g = torch.Generator(device="cuda").manual_seed(len(shapes))
    ws = [(torch.randn(*s, generator=g, device="cuda") * s[1] ** -0.5).to(DT[dtype]) for s in shapes]
    ms = [gradient(g, s, torch.float32) for s in shapes]
    lr, beta, decay = 0.05, 0.9, 0.1
    for _ in range(2):
        gs = [gradient(g, s, DT[dtype]) for s in shapes]
        old_w, old_m = [w.to(F64) for w in ws], [m.to(F64) for m in ms]
        dp.muon_step(ws, gs, ms, lr=lr, momentum=beta, nesterov=nesterov, weight_decay=decay)
        for i, s in enumerate(shapes):
            grad = gs[i].to(F64)
            m = beta * old_m[i] + grad
            # beta comes as float32, the product and the sum round
            assert ((ms[i].to(F64) - m).abs() <= 3 * U * (beta * old_m[i].abs() + grad.abs())).all()
            u = grad + beta * m if nesterov else m
            scale = lr * max(1.0, s[2] / s[1]) ** 0.5
            o = newton(u, F64)
            want = (1 - lr * decay) * old_w[i] - scale * o
            least = (want.to(DT[dtype]).to(F64) - want).norm()
            # lr, the decay, the scale and the momentum's rounding: a few u of either term
            bound = (1.01 * least + 4 * scale * (newton(u, torch.float32).to(F64) - o).norm() +
                     4 * U * (old_w[i].norm() + scale * o.norm()))
            off = (ws[i].to(F64) - want).norm()
            assert off <= bound, (s, (off / want.norm()).item())
