"""The example that trains and answers in MX4: it learns, its clipped gradients are those of the formulas, and it answers with
what it was trained to."""
import importlib.util
import os

import pytest
import torch

import paper_1802_04434_amd as ss

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "mx4_training.py")
    spec = importlib.util.spec_from_file_location("mx4_training", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def values(x):
    """what MX4 makes of x, in 64 bits"""
    q = ss.new_mx4(*x.shape)
    ss.mx4_quantize(x, q)
    return ss.mx4_dequantize(q, torch.empty(x.shape, device=DEV)).double()


def test_it_learns_and_the_same_way_every_time(example):
    losses, layers, bias, teacher = example.train(steps=150)
    again, _, again_bias, _ = example.train(steps=150)
    assert losses == again and torch.equal(bias, again_bias)
    assert sum(losses[-10:]) < 0.25 * sum(losses[:10]), (losses[:10], losses[-10:])
    x = torch.randn(16, teacher.shape[1], device=DEV).bfloat16()
    want = x.float() @ teacher.t()
    before = float(want.norm())
    assert float((example.answer(layers, bias, x).float() - want).norm()) < 0.75 * before


def test_a_workers_vector_is_the_clipped_gradient(example):
    torch.manual_seed(1)
    rows, (k, h, n) = 130, (70, 96, 33)
    lengths = [h * k, h, n * h]
    x = torch.zeros(sum(lengths), device=DEV)
    w1, bias, w2 = x.split(lengths)
    for p in (w1, bias, w2):
        p.normal_(0, 0.1)
    layers = example.Layer(w1.view(h, k), rows), example.Layer(w2.view(n, h), rows)
    for layer in layers:
        layer.quantize()
    batch, target = torch.randn(rows, k, device=DEV).bfloat16(), torch.randn(rows, n, device=DEV)
    worker = example.Worker([x], lengths, x.numel())
    worker.gradients(layers, bias, batch, target, 0.01)
    # the same from the layers' inputs, in 64 bits; sums of at most 130 products in fp32 differ by 130 * 2^-23 of their magnitudes
    hidden = layers[0].y
    kept = (hidden > 0) * hidden
    dy = ((layers[1].y.float() - target) / rows).bfloat16()
    dh = layers[1].dx * (hidden > 0)
    left, right = [values(dh.t().contiguous()), values(dy.t().contiguous())], [values(batch.t().contiguous()), values(kept.t().contiguous())]
    want = [left[0] @ right[0].t(), dh.double().sum(0), left[1] @ right[1].t()]
    bound = [rows * 2.0 ** -23 * (left[0].abs() @ right[0].abs().t()), rows * 2.0 ** -23 * dh.double().abs().sum(0), rows * 2.0 ** -23 * (left[1].abs() @ right[1].abs().t())]
    norm = float(torch.cat([g.flatten() for g in want]).norm())
    slack = float(torch.cat([b.flatten() for b in bound]).norm())
    assert abs(float(worker.norm) - norm) <= slack + norm * 2.0 ** -23
    scale = min(1.0, 0.01 / (norm + 1e-6))
    for part, g, b in zip(worker.parts, want, bound):
        # the factor's own error: the norm's, and the roundings of a sum, a quotient and a product
        assert bool(((part.double() - scale * g.flatten()).abs() <= scale * (b.flatten() + g.flatten().abs() * (slack / norm + 2.0 ** -21)) + 2.0 ** -149).all())
