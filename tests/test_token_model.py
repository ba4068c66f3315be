"""The example model that runs the token operators and the circulant layers together: its gradients against autograd on the dense
weights in 64 bits, a training run that learns, and single tokens scored with 8-bit activations."""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("token_model", Path(__file__).resolve().parent.parent / "examples" / "token_model.py")
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def dense(w):
    p, q, k = w.shape
    i = torch.arange(k, device=w.device)
    return w[:, :, (i[:, None] - i[None, :]) % k].permute(0, 2, 1, 3).reshape(p * k, q * k)


def plain_losses(w, ids, targets, eps, padding):
    def norm(x, gain):
        return x * torch.rsqrt((x * x).mean(1, keepdim=True) + eps) * gain

    x = torch.where((ids != padding)[:, None], w["E"][ids] * math.sqrt(w["E"].shape[1]), 0.0)
    s = x + torch.relu(norm(x, w["g1"]) @ dense(w["W1"]).T) @ dense(w["W2"]).T
    z = norm(s, w["g2"]) @ dense(w["W3"]).T
    loss = torch.logsumexp(z, 1) - z.gather(1, targets.clamp(min=0)[:, None]).squeeze(1)
    return torch.where(targets >= 0, loss, 0.0)


def test_gradients(example):
    model = example.TokenModel(vocab=320, n=64, hidden=128, k=16, tokens=100)
    ids, targets = example.batch(model, 0)
    mean = model.gradients(ids, targets)
    w = {name: t.double().requires_grad_() for name, t in model.weights.items()}
    want = plain_losses(w, ids, targets, example.EPS, example.PADDING).sum() / (targets >= 0).sum()
    want.backward()
    want = want.detach()
    assert abs(float(mean) - float(want)) <= 1e-4 * float(want)
    for name, t in w.items():
        # the layers' split-operand products are exact to 1e-4 of the largest value, and three of them follow one another
        err = (model.grads[name].double() - t.grad).abs().max() / t.grad.abs().max()
        assert float(err) <= 3e-4, (name, float(err))
    model.close()


def test_training_and_scoring(example):
    model = example.TokenModel(vocab=256, n=128, hidden=256, k=16, tokens=512)
    losses = []
    for i in range(80):
        mean, norm = model.step(*example.batch(model, i), rate=4.0, max_norm=0.5)
        losses.append(float(mean))
        assert math.isfinite(losses[-1]) and math.isfinite(float(norm))
        clipped = math.sqrt(sum(float(g.double().square().sum()) for g in model.grads.values()))
        assert clipped <= 0.5 * (1 + 1e-5)
    assert losses[-1] < 0.5 * losses[0]
    ids, targets = example.batch(model, 1000)
    for n in (1, 7):
        got = model.score(ids[:n], targets[:n]).double()
        w = {name: t.double() for name, t in model.weights.items()}
        want = plain_losses(w, ids[:n], targets[:n], example.EPS, example.PADDING)
        assert float((got - want).abs().max()) <= 0.5          # 8-bit activations: 1/16 relative each, averaged over the widths
    model.close()
