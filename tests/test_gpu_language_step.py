"""The example that trains a small language model: it runs, the loss's gradients in it are those of the formula, and the layer takes the orthogonalised step."""
import os
import sys

import pytest
import torch

import loss_plain as plain
from test_gpu_loss import check

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_gradients_and_the_layers_step():
    import language_step as example
    model, crew, batches = example.setup(vocab=131, width=96, rows=64, workers=2)
    for _ in range(3):
        layer, m, head = model.layer.clone(), model.m.clone(), model.head16.cpu()
        given = batches()
        loss = example.step(model, crew, given)
        assert torch.isfinite(loss)
        for worker, (_, target) in zip(crew, given):
            want = plain.softmax_loss(worker.h.cpu(), head, target.cpu(), worker.dloss.cpu())
            check({"loss": worker.loss, "lse": worker.lse, "dh": worker.dh, "dw": worker.dhead}, want, (target >= 0).cpu())
            there = (target >= 0).cpu()
            assert (worker.dh.cpu()[~there] == 0).all()
        g = crew[0].dlayer                                # the workers' sum
        b = torch.tensor(0.9, dtype=torch.float32, device=g.device)
        m = b * m + (1 - b) * g
        assert torch.equal(model.m, m)
        u = (b * m + (1 - b) * g).cpu()
        want = layer.cpu().double() - 2e-2 * plain.orthogonalized(u)
        allowed = 2e-2 * plain.orthogonal_bound(u) + 3 * plain.U32 * float(want.norm() + layer.norm())
        assert float((model.layer.cpu().double() - want).norm()) <= allowed


def test_it_runs():
    import language_step as example
    model, crew, batches = example.setup()
    for _ in range(5):
        loss = example.step(model, crew, batches())
    assert torch.isfinite(loss) and torch.isfinite(model.tables).all() and torch.isfinite(model.layer).all()
