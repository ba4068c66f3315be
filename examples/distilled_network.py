"""A small image network whose convolution and output layers are block-circulant, trained against the stored answers of an uncompressed one.

    a1 = relu(gnorm(conv1(x)));  a2 = silu(gnorm(conv2(a1)));  z = W a2 (all pixels and channels) + theta
    loss = mean over the images of the divergence from the teacher's list of top logits, the classes outside it as one class more

The teacher is a dense linear network here; what the training keeps of it is ``Answers``: a short list of logits and classes an image, and
the log of the sum over all of them.  torch owns the memory, sums the output layer's bias gradient and subtracts the gradients; everything
else runs in the library.

    python examples/distilled_network.py [steps]
"""
from __future__ import annotations

import math
import sys
from pathlib import Path
from typing import NamedTuple

import torch

if __name__ == "__main__":
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

import paper_1708_08917_b200 as circ

EPS = 1e-5


class Answers(NamedTuple):
    values: torch.Tensor      # [images][count], descending
    ids: torch.Tensor         # int32, their classes
    lse: torch.Tensor         # [images], log sum exp(logits / temperature)


def top_answers(logits: torch.Tensor, count: int, temperature: float) -> Answers:
    """What is stored of a teacher's logits [images][classes]."""
    n, classes = logits.shape
    h = circ.circ_top_create(classes, count)
    circ.circ_top_set_dtypes(h, circ.CIRC_F32, circ.CIRC_I32)
    circ.circ_top_set_temperature(h, temperature)
    out = Answers(torch.empty(n, count, device="cuda"), torch.empty(n, count, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda"))
    circ.circ_top_forward(h, logits, classes, *out, n, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_top_destroy(h)
    return out


class DistilledNetwork:
    """float32 weights: the convolutions' defining vectors C1, C2 ([3][3][c / k][c_in / k][k]), the norms' gains and biases, and the output layer's
    defining vectors W with its bias theta."""

    def __init__(self, images: int = 64, size: int = 8, channels: int = 64, groups: int = 8, classes: int = 320, k: int = 16, count: int = 16,
                 temperature: float = 2.0, seed: int = 1):
        self.images, self.size, self.channels, self.classes, self.k, self.temperature = images, size, channels, classes, k, temperature
        self.features = size * size * channels
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def normal(*shape, std):
            return torch.randn(*shape, device="cuda", generator=g) * std

        c = channels // k
        ones, zeros = torch.ones(channels, device="cuda"), torch.zeros(channels, device="cuda")
        self.weights = {"C1": normal(3, 3, c, c, k, std=1 / math.sqrt(9 * channels)), "g1": ones.clone(), "b1": zeros.clone(),
                        "C2": normal(3, 3, c, c, k, std=1 / math.sqrt(9 * channels)), "g2": ones.clone(), "b2": zeros.clone(),
                        "W": normal(classes // k, self.features // k, k, std=1 / math.sqrt(self.features)), "theta": torch.zeros(classes, device="cuda")}
        self.grads = {name: torch.empty_like(w) for name, w in self.weights.items()}
        self.norm = [circ.circ_gnorm_create(channels, groups, EPS) for _ in range(2)]
        for h, act in zip(self.norm, (circ.CIRC_ACT_RELU, circ.CIRC_ACT_SILU)):
            circ.circ_gnorm_set_activation(h, act)
            circ.circ_gnorm_reserve(h, images, size, size)
        self.groups = groups
        self.distill = circ.circ_distill_create(classes, count)
        circ.circ_distill_set_dtypes(self.distill, circ.CIRC_F32, circ.CIRC_F32, circ.CIRC_I32)
        circ.circ_distill_set_temperature(self.distill, temperature)
        circ.circ_distill_set_rest(self.distill, 1)
        circ.circ_distill_reserve(self.distill, images)
        self.layers = {}
        self._load_layers()

    def _load_layers(self):
        """The layers hold transforms of their weights, so new weights mean new layers."""
        for h in self.layers.values():
            circ.circ_destroy(h)
        self.layers = {name: circ.circ_conv_create(self.channels, self.channels, 3, 1, self.k, self.weights[name]) for name in ("C1", "C2")}
        for h in self.layers.values():
            circ.circ_set_io_dtype(h, circ.CIRC_F32, circ.CIRC_F32)
        self.layers["W"] = circ.circ_fc_create(self.classes, self.features, self.k, self.weights["W"])
        circ.circ_set_bias(self.layers["W"], self.weights["theta"])

    def gradients(self, x: torch.Tensor, answers: Answers, weights: torch.Tensor | None = None) -> torch.Tensor:
        """The mean loss (a device tensor); the gradients are in ``grads``.  ``x`` [images][size][size][channels], ``weights``: of the images."""
        w, d, n, s, st = self.weights, self.grads, len(x), self.size, torch.cuda.current_stream()

        def stats():
            return torch.empty(n, self.groups, device="cuda"), torch.empty(n, self.groups, device="cuda")

        (m1, r1), (m2, r2) = stats(), stats()
        u1, a1, u2, a2 = (torch.empty_like(x) for _ in range(4))
        z, mean = torch.empty(n, self.classes, device="cuda"), torch.empty(1, device="cuda")
        circ.circ_conv_forward(self.layers["C1"], x, u1, n, s, s, st)
        circ.circ_gnorm_forward(self.norm[0], u1, w["g1"], w["b1"], a1, m1, r1, n, s, s, st)
        circ.circ_conv_forward(self.layers["C2"], a1, u2, n, s, s, st)
        circ.circ_gnorm_forward(self.norm[1], u2, w["g2"], w["b2"], a2, m2, r2, n, s, s, st)
        circ.circ_fc_forward(self.layers["W"], a2, z, n, st)
        # backwards; the gradient of the scores takes their place, those of the norms' inputs the place of those of their outputs
        circ.circ_distill_backward(self.distill, z, self.classes, *answers, weights, None, None, mean, z, self.classes, self.temperature ** 2, n, st)
        torch.sum(z, 0, out=d["theta"])
        da = torch.empty_like(x)
        circ.circ_fc_backward(self.layers["W"], a2, z, da, d["W"], n, st)
        circ.circ_gnorm_backward(self.norm[1], u2, w["g2"], w["b2"], m2, r2, da, da, d["g2"], d["b2"], n, s, s, st)
        circ.circ_conv_backward_weight(self.layers["C2"], a1, da, d["C2"], n, s, s, st)
        db = torch.empty_like(x)
        circ.circ_conv_backward_input(self.layers["C2"], da, db, n, s, s, st)
        circ.circ_gnorm_backward(self.norm[0], u1, w["g1"], w["b1"], m1, r1, db, db, d["g1"], d["b1"], n, s, s, st)
        circ.circ_conv_backward_weight(self.layers["C1"], x, db, d["C1"], n, s, s, st)
        return mean * self.temperature ** 2

    def step(self, x: torch.Tensor, answers: Answers, rate: float) -> torch.Tensor:
        loss = self.gradients(x, answers)
        for name, w in self.weights.items():
            w -= rate * self.grads[name]
        self._load_layers()
        return loss

    def close(self):
        torch.cuda.synchronize()
        for h in self.layers.values():
            circ.circ_destroy(h)
        for h in self.norm:
            circ.circ_gnorm_destroy(h)
        circ.circ_distill_destroy(self.distill)


def batch(net: DistilledNetwork, step: int) -> tuple[torch.Tensor, torch.Tensor]:
    """Random images and the logits of a fixed dense network for them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    teacher = torch.randn(net.channels, net.classes, device="cuda", generator=g) / 4
    g.manual_seed(1000 + step)
    x = torch.randn(net.images, net.size, net.size, net.channels, device="cuda", generator=g)
    x += 2 * torch.randn(net.images, 1, 1, net.channels, device="cuda", generator=g)
    return x, torch.relu(x).mean((1, 2)) @ teacher


def main(steps: int = 60) -> None:
    net = DistilledNetwork()
    for i in range(steps):
        x, logits = batch(net, i % 8)
        loss = net.step(x, top_answers(logits, 16, net.temperature), rate=0.05)
        if i % 10 == 0 or i == steps - 1:
            print(f"step {i:4d}  loss {float(loss):.4f}")
    net.close()


if __name__ == "__main__":
    main(*map(int, sys.argv[1:2]))
