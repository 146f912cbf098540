"""The example that trains a language model by sketched gradients: its gradients against automatic differentiation in 64 bits on
the CPU, and a short training, whose loss has to fall most of the way to the data's entropy."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
import train_language_model as example  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradients_match_automatic_differentiation():
    """in 32 bits, products of up to 300 terms by a library: 1e-5 of the largest gradient of a tensor"""
    chain = example.Chain(300, 4, DEV, 5)
    model = example.Model(300, 48, 128, 2, DEV, 6)
    token, target = chain.draw(128)
    loss = model.gradients(1, token, target)
    p = {name: t.detach().cpu().double().requires_grad_() for name, t in model.params.items()}
    token, target = token.cpu(), target.cpu()
    mixed = p["table"][token] @ p["mix"]
    hidden = torch.nn.functional.layer_norm(mixed, (48,), p["weight"], p["bias"])
    each = torch.nn.functional.cross_entropy(hidden @ p["head"].t(), target, reduction="none")
    each.mean().backward()
    torch.testing.assert_close(loss.cpu().double(), each.detach(), rtol=1e-5, atol=1e-5)
    for name, want in p.items():
        got = model.worker_views[1][name].cpu().double()
        assert (got - want.grad).abs().max() <= 1e-5 * want.grad.abs().max(), name
    assert not model.worker_grads[0].any()


def test_training_learns():
    losses, entropy, model, _ = example.train(steps=150)
    losses = losses.cpu()
    assert torch.isfinite(losses).all()
    assert losses[0] > 7.0 and losses[-10:].mean() < entropy + 0.4 * (losses[0] - entropy)
    assert all(torch.isfinite(t).all() for t in model.params.values())
