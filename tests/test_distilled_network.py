"""The example network that runs the top selection, the distillation and the group norms together with circulant convolutions: its gradients against
autograd on dense weights in 64 bits, and a step that runs."""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("distilled_network", Path(__file__).resolve().parent.parent / "examples" / "distilled_network.py")
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def dense(w):
    """[..][p][q][k] defining vectors -> [..][p k][q k]."""
    *taps, p, q, k = w.shape
    i = torch.arange(k, device=w.device)
    return w[..., (i[:, None] - i[None, :]) % k].transpose(-3, -2).reshape(*taps, p * k, q * k)


def plain_loss(w, x, answers, groups, eps, tau, weights):
    def conv(v, name):
        return torch.nn.functional.conv2d(v.permute(0, 3, 1, 2), dense(w[name]).permute(2, 3, 0, 1), padding=1).permute(0, 2, 3, 1)

    def norm(v, gain, bias):
        n, h, ww, c = v.shape
        t = v.reshape(n, h * ww, groups, -1)
        t = (t - t.mean((1, 3), keepdim=True)) / torch.sqrt(t.var((1, 3), unbiased=False, keepdim=True) + eps)
        return t.reshape(v.shape) * gain + bias

    a = torch.relu(norm(conv(x, "C1"), w["g1"], w["b1"]))
    a = torch.nn.functional.silu(norm(conv(a, "C2"), w["g2"], w["b2"]))
    z = (a.flatten(1) @ dense(w["W"]).T + w["theta"]) / tau
    log_q = torch.log_softmax(z, 1)
    ids, p = answers.ids.long(), torch.exp(answers.values.double() / tau - answers.lse.double()[:, None])
    rest = 1 - p.sum(1)
    assert bool((rest > 0.01).all())
    outside = torch.ones_like(log_q, dtype=torch.bool).scatter_(1, ids, False)
    log_rest = torch.logsumexp(torch.where(outside, log_q, -math.inf), 1)
    loss = (p * (torch.log(p) - log_q.gather(1, ids))).sum(1) + rest * (torch.log(rest) - log_rest)
    weights = torch.ones_like(loss) if weights is None else weights.double()
    return tau ** 2 * (loss * weights).sum() / weights.sum()


@pytest.mark.parametrize("weighted", [False, True])
def test_gradients(example, weighted):
    net = example.DistilledNetwork(images=10, size=5, channels=32, groups=4, classes=112, k=16, count=9, temperature=1.5)
    x, logits = example.batch(net, 0)
    answers = example.top_answers(logits, 9, 1.5)
    want_ids = torch.argsort(logits.double(), dim=1, descending=True, stable=True)[:, :9]
    assert torch.equal(answers.ids.long(), want_ids) and torch.equal(answers.values, logits.gather(1, want_ids))
    weights = torch.rand(10, device="cuda") + 0.2 if weighted else None
    got = net.gradients(x, answers, weights)
    w = {name: t.double().requires_grad_() for name, t in net.weights.items()}
    want = plain_loss(w, x.double(), answers, net.groups, example.EPS, 1.5, weights)
    want.backward()
    want = want.detach()
    assert abs(float(got) - float(want)) <= 1e-4 * float(want)
    for name, t in w.items():
        # the layers' split-operand products are exact to 1e-4 of the largest value; three follow one another, and values beside a ReLU's 0 change sides
        err = (net.grads[name].double() - t.grad).norm() / t.grad.norm()
        assert float(err) <= 1e-3, (name, float(err))
    net.close()


def test_a_few_steps_run(example):
    net = example.DistilledNetwork(images=16, size=6, channels=32, groups=4, classes=96, k=16, count=8)
    for i in range(3):
        x, logits = example.batch(net, i)
        assert math.isfinite(float(net.step(x, example.top_answers(logits, 8, net.temperature), rate=0.05)))
    assert all(bool(torch.isfinite(t).all()) for t in net.weights.values())
    net.close()
