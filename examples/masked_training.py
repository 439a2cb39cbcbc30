"""A small network trained with masked convolutions, every step of it through the library.

    python examples/masked_training.py [--steps N] [--keep8]

Per step: conv1 (masked) -> group norm + SiLU -> conv2 (masked) -> group norm + SiLU -> a linear layer over many
classes with softmax cross entropy; backwards through the same layers with the masked weight gradient on the stored
encodings and dgrad; the convolutions' weights move along the orthogonalised gradient, everything else along the
gradient.  The images are synthetic: one random prototype per class under noise of twice its size, so that the loss falls
over the whole run (6.5 to 0.24 in 30 steps).  With --keep8 the norms' inputs are kept from the forward to the backward pass
in 8 bits instead of 32.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2207_00083_b200 import binding as dk  # noqa: E402
from paper_2207_00083_b200 import synth  # noqa: E402

K, G = 4, 8                    # private inputs per virtual batch, virtual batches
SIZE, CLASSES, GROUPS = 12, 500, 8
CHANNELS = (8, 32, 48)
SIGMA = 100.0                  # of the masking noise
EPS, QUINTIC = 1e-5, (3.4445, -4.7750, 2.0315)


class Network:
    def __init__(self, seed: int = 0, keep8: bool = False):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape):
            return torch.randn(shape, generator=g, device="cuda")

        self.ctx, self.n, self.keep8 = dk.Context(0), K * G, keep8
        self.rng, self.gen = np.random.default_rng(seed), g
        self.convs = [dk.dk_problem(dk.DK_CONV2D, dk.DK_NHWC, CHANNELS[i], CHANNELS[i + 1], SIZE, SIZE, 3, 3, 1, 1, K, G,
                                    dk.DK_PREC_DEFAULT, 1e-4) for i in range(2)]
        self.W = [normal(CHANNELS[i + 1], 3, 3, CHANNELS[i]) * (2 / (9 * CHANNELS[i])) ** 0.5 for i in range(2)]
        self.norms = [dk.dk_norm(self.n, SIZE, SIZE, CHANNELS[i + 1], GROUPS, dk.DK_ACT_SILU, dk.DK_F32, EPS)
                      for i in range(2)]
        self.gamma = [torch.ones(CHANNELS[i + 1], device="cuda") for i in range(2)]
        self.beta = [torch.zeros(CHANNELS[i + 1], device="cuda") for i in range(2)]
        self.d = SIZE * SIZE * CHANNELS[2]
        self.head = dk.dk_xent(self.n, self.d, CLASSES, dk.DK_F32)
        self.V = normal(CLASSES, self.d) * self.d ** -0.5
        self.updates = [dk.dk_ortho(1, w.shape[0], w[0].numel(), dk.DK_F32, 5, *QUINTIC, 1e-7) for w in self.W]
        for q in (*self.convs, *self.norms, self.head, *self.updates):
            self.ctx.ensure_workspace(q)

    def gradients(self, x, target):
        """Mean loss, gradients of every parameter, and the integrity verdicts of the masked products."""
        ctx, empty = self.ctx, lambda c: torch.empty((self.n, SIZE, SIZE, c), device="cuda")
        a, kept, verdicts = x, [], []
        for p, W, q, gamma, beta in zip(self.convs, self.W, self.norms, self.gamma, self.beta):
            C = synth.draw_coefficients(self.rng, K, G)
            r = torch.randn((G, SIZE, SIZE, p.cin), generator=self.gen, device="cuda") * SIGMA
            z, encoded = empty(p.cout), torch.empty((G * (K + 2), SIZE, SIZE, p.cin), device="cuda")
            v = dk.new_verdict()
            dk.dk_masked_linear(ctx, p, W, a, r, C, None, z, encoded, v)
            y, stats = empty(p.cout), torch.empty((self.n, GROUPS, 2), device="cuda")
            if self.keep8:
                k8 = dk.dk_ckpt8(self.n * SIZE * SIZE, p.cout, dk.DK_F32)
                held = torch.empty(dk.dk_ckpt8_bytes(k8), dtype=torch.uint8, device="cuda")
                dk.dk_group_norm_fwd_ckpt8(ctx, q, z, gamma, beta, y, stats, held)
                z = held
            else:
                dk.dk_group_norm_fwd(ctx, q, z, gamma, beta, y, stats)
            kept.append((C, encoded, z, stats))
            verdicts.append(v)
            a = y
        loss, lse = torch.empty(self.n, device="cuda"), torch.empty(self.n, device="cuda")
        dh, dV = torch.empty_like(a), torch.empty_like(self.V)
        dk.dk_linear_xent_fwd(ctx, self.head, a, self.V, target, loss, lse)
        dk.dk_linear_xent_bwd(ctx, self.head, a, self.V, target, lse, None, 1.0 / self.n, dh, dV)
        grads = {"V": dV}
        for i in (1, 0):
            C, encoded, z, stats = kept[i]
            p, dz = self.convs[i], empty(self.convs[i].cout)
            grads[f"gamma{i}"], grads[f"beta{i}"] = torch.empty_like(self.gamma[i]), torch.empty_like(self.beta[i])
            back = dk.dk_group_norm_bwd_ckpt8 if self.keep8 else dk.dk_group_norm_bwd
            back(ctx, self.norms[i], dh, z, self.gamma[i], self.beta[i], stats, dz, grads[f"gamma{i}"], grads[f"beta{i}"])
            grads[f"W{i}"] = torch.empty_like(self.W[i])
            dk.dk_linear_bwd_wgrad(ctx, p, dz, encoded, K + 2, C, synth.draw_gamma(self.rng, K, G), 1.0, grads[f"W{i}"])
            if i:
                dh = torch.empty((self.n, SIZE, SIZE, p.cin), device="cuda")
                dk.dk_linear_bwd_dgrad(ctx, p, self.W[i], dz, dh)
        return loss.mean(), grads, [dk.read_verdict(v) for v in verdicts]

    def step(self, x, target, lr: float = 0.02):
        loss, grads, verdicts = self.gradients(x, target)
        for i in range(2):
            q = self.updates[i]
            scale = -lr * max(1.0, q.m / q.n) ** 0.5
            dk.dk_orthogonalize(self.ctx, q, grads[f"W{i}"], scale, 1.0, self.W[i])
            self.gamma[i] -= lr * grads[f"gamma{i}"]
            self.beta[i] -= lr * grads[f"beta{i}"]
        self.V -= 0.5 * lr * grads["V"]
        assert all(v["ok"] == 1 for v in verdicts)
        return float(loss)


def images(n: int, seed: int = 1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    prototypes = torch.randn((CLASSES, SIZE, SIZE, CHANNELS[0]), generator=g, device="cuda")
    while True:
        target = torch.randint(0, 16, (n,), generator=g, device="cuda")      # a few of the classes come up
        yield prototypes[target] + 2.0 * torch.randn((n, SIZE, SIZE, CHANNELS[0]), generator=g, device="cuda"), target


def main(steps: int = 30, keep8: bool = False):
    net = Network(keep8=keep8)
    losses = []
    for i, (x, target) in zip(range(steps), images(net.n)):
        losses.append(net.step(x, target))
        print(f"step {i}: loss {losses[-1]:.4f}", flush=True)
    assert dk.dk_device_status(net.ctx) == 0
    net.ctx.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--keep8", action="store_true")
    args = ap.parse_args()
    main(args.steps, args.keep8)
