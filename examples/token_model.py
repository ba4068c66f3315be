"""A small model that predicts tokens, its projections block-circulant: one training step through the library, from the ids to the
clipped gradients, and the scoring of one token with its activations handed on in 8 bits.

    x = E[ids] sqrt(n);  u = norm(x) g1;  v = relu(W1 u);  s = x + W2 v;  z = W3 (norm(s) g2);  loss = cross entropy(z, targets)

torch owns the memory, masks the ReLU's gradient and subtracts the clipped gradients; everything else runs in the library.

    python examples/token_model.py [steps]
"""
from __future__ import annotations

import math
import sys
from pathlib import Path

import torch

if __name__ == "__main__":
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

import paper_1708_08917_b200 as circ

EPS = 1e-5
PADDING = 0      # the id of positions without a token


class TokenModel:
    """float32 weights: the table E [vocab][n], the gains g1, g2 [n], and the defining vectors of W1, W2, W3 ([rows / k][columns / k][k])."""

    def __init__(self, vocab: int = 1024, n: int = 256, hidden: int = 512, k: int = 16, tokens: int = 512, seed: int = 1):
        self.vocab, self.n, self.hidden, self.k, self.tokens = vocab, n, hidden, k, tokens
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def circulant(rows, columns):
            return torch.randn(rows // k, columns // k, k, device="cuda", generator=g) / math.sqrt(columns)

        self.weights = {"E": torch.randn(vocab, n, device="cuda", generator=g) / math.sqrt(n), "g1": torch.ones(n, device="cuda"),
                        "g2": torch.ones(n, device="cuda"), "W1": circulant(hidden, n), "W2": circulant(n, hidden), "W3": circulant(vocab, n)}
        self.grads = {name: torch.empty_like(w) for name, w in self.weights.items()}
        self.embed = circ.circ_embed_create(vocab, n)
        circ.circ_embed_set_scale(self.embed, math.sqrt(n))
        circ.circ_embed_set_padding(self.embed, PADDING)
        circ.circ_embed_reserve(self.embed, tokens)
        self.norm = circ.circ_norm_create(n, EPS)
        circ.circ_norm_reserve(self.norm)
        self.norm8 = circ.circ_norm_create(n, EPS)
        circ.circ_norm_set_dtypes(self.norm8, circ.CIRC_F32, circ.CIRC_E4M3)
        self.loss = circ.circ_loss_create(vocab)
        circ.circ_loss_reserve(self.loss, tokens)
        self.clip = circ.circ_clip_create([w.numel() for w in self.grads.values()], circ.CIRC_F32, circ.CIRC_F32)
        circ.circ_clip_set_tensors(self.clip, list(self.grads.values()), None, torch.cuda.current_stream())
        self.layers = {}
        self._load_layers()

    def _load_layers(self):
        """The layers hold transforms of their weights, so new weights mean new layers."""
        for h in self.layers.values():
            circ.circ_destroy(h)
        sizes = {"W1": (self.hidden, self.n), "W2": (self.n, self.hidden), "W3": (self.vocab, self.n)}
        self.layers = {name: circ.circ_fc_create(m, n, self.k, self.weights[name]) for name, (m, n) in sizes.items()}
        circ.circ_set_activation(self.layers["W1"], 1)

    def gradients(self, ids: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """The mean loss (a device tensor); the gradients are in ``grads``.  ``ids``, ``targets``: int64 [tokens]."""
        w, d, t, st = self.weights, self.grads, len(ids), torch.cuda.current_stream()

        def rows(width):
            return torch.empty(t, width, device="cuda")

        x, u, s, h = (rows(self.n) for _ in range(4))
        r1, r2 = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
        v, f, z, mean = rows(self.hidden), rows(self.n), rows(self.vocab), torch.empty(1, device="cuda")
        circ.circ_embed_forward(self.embed, w["E"], ids, x, t, st)
        circ.circ_norm_forward(self.norm, x, None, w["g1"], None, u, None, r1, t, st)
        circ.circ_fc_forward(self.layers["W1"], u, v, t, st)
        circ.circ_fc_forward(self.layers["W2"], v, f, t, st)
        circ.circ_norm_forward(self.norm, x, f, w["g2"], s, h, None, r2, t, st)
        circ.circ_fc_forward(self.layers["W3"], h, z, t, st)
        # backwards; the gradient of the scores takes their place
        circ.circ_loss_backward(self.loss, z, self.vocab, targets, None, None, mean, z, self.vocab, 1.0, t, st)
        dh, ds, dv, du = rows(self.n), rows(self.n), rows(self.hidden), rows(self.n)
        circ.circ_fc_backward(self.layers["W3"], h, z, dh, d["W3"], t, st)
        circ.circ_norm_backward(self.norm, s, w["g2"], r2, dh, None, ds, d["g2"], t, st)
        circ.circ_fc_backward(self.layers["W2"], v, ds, dv, d["W2"], t, st)
        dv *= v > 0
        circ.circ_fc_backward(self.layers["W1"], u, dv, du, d["W1"], t, st)
        circ.circ_norm_backward(self.norm, x, w["g1"], r1, du, ds, ds, d["g1"], t, st)      # what flows past the layer is added on the way
        circ.circ_embed_backward(self.embed, ids, ds, d["E"], t, st)
        return mean

    def step(self, ids: torch.Tensor, targets: torch.Tensor, rate: float, max_norm: float) -> tuple[torch.Tensor, torch.Tensor]:
        """One update; (mean loss, norm of the gradients before they were clipped), device tensors."""
        mean, norm = self.gradients(ids, targets), torch.empty(1, device="cuda")
        circ.circ_clip_forward(self.clip, max_norm, norm, torch.cuda.current_stream())
        for name, w in self.weights.items():
            w -= rate * self.grads[name]
        self._load_layers()
        return mean, norm

    def score(self, ids: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """The loss of each position (one token or some), with the normed activations handed on in 8 bits."""
        w, t, st = self.weights, len(ids), torch.cuda.current_stream()

        def normed(x, residual, gain, total):
            q, scale, y = torch.empty(t, self.n, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(t, 1, device="cuda"), torch.empty_like(x)
            circ.circ_norm_forward(self.norm8, x, residual, gain, total, q, scale, None, t, st)
            circ.circ_norm_unpack(self.norm8, q, scale, y, circ.CIRC_F32, t, st)
            return y

        x, v, f = torch.empty(t, self.n, device="cuda"), torch.empty(t, self.hidden, device="cuda"), torch.empty(t, self.n, device="cuda")
        z, loss = torch.empty(t, self.vocab, device="cuda"), torch.empty(t, device="cuda")
        circ.circ_embed_forward(self.embed, w["E"], ids, x, t, st)
        circ.circ_fc_forward(self.layers["W1"], normed(x, None, w["g1"], None), v, t, st)
        circ.circ_fc_forward(self.layers["W2"], v, f, t, st)
        circ.circ_fc_forward(self.layers["W3"], normed(x, f, w["g2"], None), z, t, st)
        circ.circ_loss_forward(self.loss, z, self.vocab, targets, loss, None, None, t, st)
        return loss

    def close(self):
        torch.cuda.synchronize()
        for h in self.layers.values():
            circ.circ_destroy(h)
        circ.circ_embed_destroy(self.embed)
        circ.circ_norm_destroy(self.norm)
        circ.circ_norm_destroy(self.norm8)
        circ.circ_loss_destroy(self.loss)
        circ.circ_clip_destroy(self.clip)


def batch(model: TokenModel, step: int):
    """Random tokens, some positions without one; the token behind is a fixed function of the one before."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 + step)
    ids = torch.randint(1, model.vocab, (model.tokens,), device="cuda", generator=g)
    targets = (5 * ids + 3) % model.vocab
    gap = torch.rand(model.tokens, device="cuda", generator=g) < 0.1
    return ids.masked_fill(gap, PADDING), targets.masked_fill(gap, -100)


def main(steps: int = 200) -> None:
    model = TokenModel()
    for i in range(steps):
        mean, norm = model.step(*batch(model, i), rate=4.0, max_norm=0.5)
        if i % 20 == 0 or i == steps - 1:
            print(f"step {i:4d}  loss {float(mean):.4f}  gradient norm {float(norm):.3f}")
    ids, targets = batch(model, steps)
    print(f"loss of one token: {float(model.score(ids[:1], targets[:1])[0]):.4f}")
    model.close()


if __name__ == "__main__":
    main(*map(int, sys.argv[1:2]))
