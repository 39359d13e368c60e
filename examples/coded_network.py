"""A small image network trained by coded gradient descent: the layers and the aggregation as a user runs them together.

    frozen 8-bit layer -> group norm + SiLU + dropout (gamma, beta trained) -> linear head (w trained)

Every image is `positions` rows of `inner` numbers.  The frozen layer turns each row into `channels` channels
(cr_quantize_rows, cr_int8_product); the normalised, dropped features of an image are what the head sees.  The data set
is cut into partitions.  A step computes every partition's partial gradient of the head (cr_partial_gradients_loss, into
the slots of all workers that hold it) and of the normalisation (cr_group_norm_backward, a row per partition), and decodes
both from the workers that did not straggle (cr_aggregate).

    python examples/coded_network.py [--steps 20]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1902_01981_b200 import binding as B  # noqa: E402
from paper_1902_01981_b200 import inputs  # noqa: E402

EPS, DROP = 1e-5, 0.1


class CodedNetwork:
    """(n, L)-tree of workers, `P` partitions of `rows` images of `positions` x `inner` numbers."""

    def __init__(self, n=4, L=2, s=1, P=24, rows=16, positions=16, inner=48, channels=64, groups=8, seed=0):
        self.P, self.rows, self.positions, self.channels, self.groups = P, rows, positions, channels, groups
        self.samples, self.d = P * rows, positions * channels
        device = torch.cuda.current_device()
        # one plan per gradient vector; the same code, so the same slots and straggler masks
        self.head_plan = B.cr_plan_create(n, L, s, P, self.d, device=device)
        self.norm_plan = B.cr_plan_create(n, L, s, P, 2 * channels, device=device)
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
        self.images = rand(self.samples * positions, inner)
        frozen = rand(channels, inner) / inner ** 0.5
        # the frozen layer is laid out once: codes in rows of a multiple of 16 bytes, a scale per channel
        self.w_codes = torch.zeros((channels, (inner + 15) // 16 * 16), dtype=torch.int8, device="cuda")[:, :inner]
        self.w_scale = torch.empty(channels, device="cuda")
        B.cr_quantize_rows(self.head_plan, frozen, self.w_codes, self.w_scale)
        self.w, self.gamma, self.beta = torch.zeros(self.d, device="cuda"), torch.ones(channels, device="cuda"), torch.zeros(channels, device="cuda")
        self.h = torch.empty((self.samples, positions, channels), device="cuda")
        self.codes = torch.empty((self.samples * positions, (inner + 15) // 16 * 16), dtype=torch.int8, device="cuda")[:, :inner]
        self.code_scale = torch.empty(self.samples * positions, device="cuda")
        self.features, self.dh_out = torch.empty_like(self.h), torch.empty_like(self.h)
        self.mean, self.rstd = torch.empty((self.samples, groups), device="cuda"), torch.empty((self.samples, groups), device="cuda")
        self.norm_rows = torch.empty((P, 2 * channels), device="cuda")
        N, m = B.cr_plan_num_nodes(self.head_plan), B.cr_plan_load(self.head_plan)
        self.slot_part = torch.from_numpy(B.slot_partitions(self.head_plan).astype(np.int64).reshape(-1)).cuda()
        self.head_slots = torch.empty((N, m, self.d), device="cuda")
        self.norm_slots = torch.empty((N, m, 2 * channels), device="cuda")
        scratch = max(16, B.cr_partial_gradients_workspace_bytes(self.head_plan, rows),
                      B.cr_group_norm_workspace_bytes(self.head_plan, self.h, groups),
                      B.cr_group_norm_backward_workspace_bytes(self.head_plan, self.h, groups))
        self.workspace = torch.empty(scratch, dtype=torch.uint8, device="cuda")
        self.head_grad, self.norm_grad = torch.empty((1, self.d), device="cuda"), torch.empty((1, 2 * channels), device="cuda")
        # labels of a network of the same kind with a head of its own
        self.forward(0, drop=0.0)
        teacher = rand(self.d) / self.d ** 0.5
        self.labels = (self.features.view(self.samples, self.d) @ teacher).contiguous()

    def close(self):
        B.cr_plan_destroy(self.head_plan)
        B.cr_plan_destroy(self.norm_plan)

    def forward(self, step, drop=DROP, first=0, count=None):
        """Features of `count` images from number `first` on; the dropout of an image depends on its number and the
        step, not on what is processed beside it."""
        count = self.samples if count is None else count
        rows = slice(first * self.positions, (first + count) * self.positions)
        part = slice(first, first + count)
        B.cr_quantize_rows(self.head_plan, self.images[rows], self.codes[rows], self.code_scale[rows])
        B.cr_int8_product(self.head_plan, self.codes[rows], self.code_scale[rows], self.w_codes, self.w_scale,
                          self.h[part].view(-1, self.channels))
        B.cr_group_norm(self.head_plan, self.h[part], self.gamma, self.beta, self.groups, self.features[part],
                        self.mean[part], self.rstd[part], eps=EPS, act=B.CR_ACT_SILU, p=drop, seed=step,
                        offset=first * self.d, workspace=self.workspace)
        return self.features[part]

    def step(self, step, masks, rate):
        """One step of gradient descent under the straggler pattern `masks`; returns the loss before it."""
        self.forward(step)
        flat = self.features.view(self.samples, self.d)
        residual = flat @ self.w - self.labels
        # the head: partial gradients straight into the slots of the workers
        B.cr_partial_gradients_loss(self.head_plan, B.CR_LOSS_SQUARED, self.features, self.labels, self.rows, self.w,
                                    self.head_slots, self.workspace)
        # the normalisation: a row [dgamma, dbeta] per partition, then the same gather that fills the slots
        torch.mul(residual[:, None], self.w, out=self.dh_out.view(self.samples, self.d))
        B.cr_group_norm_backward(self.head_plan, self.dh_out, self.h, self.gamma, self.beta, self.mean, self.rstd, self.groups, None,
                                 self.norm_rows[:, :self.channels], self.norm_rows[:, self.channels:], act=B.CR_ACT_SILU, p=DROP,
                                 seed=step, workspace=self.workspace)
        torch.index_select(self.norm_rows, 0, self.slot_part, out=self.norm_slots.view(-1, 2 * self.channels))
        B.cr_aggregate(self.head_plan, self.head_slots, masks, self.head_grad)
        B.cr_aggregate(self.norm_plan, self.norm_slots, masks, self.norm_grad)
        self.w -= rate / self.samples * self.head_grad[0]
        self.gamma -= rate / self.samples * self.norm_grad[0, :self.channels]
        self.beta -= rate / self.samples * self.norm_grad[0, self.channels:]
        return 0.5 * float(residual.square().mean())


def train(steps=20, rate=0.02, seed=0, **shape):
    """Losses of `steps` steps, every one with a random straggler in every sibling group."""
    net = CodedNetwork(seed=seed, **shape)
    try:
        masks = inputs.straggler_masks(shape.get("n", 4), shape.get("L", 2), shape.get("s", 1), steps, seed=seed + 1, exactly_s=True)
        return [net.step(t, masks[t], rate) for t in range(steps)]
    finally:
        net.close()


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=20)
    losses = train(ap.parse_args().steps)
    print("loss", " ".join(f"{v:.4f}" for v in losses))
