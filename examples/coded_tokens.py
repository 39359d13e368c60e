"""A small token model trained by coded gradient descent against a teacher: the token layers and the aggregation together.

    table (trained) -> token + previous token -> root-mean-square norm (gamma trained) -> frozen head -> distillation

Every partition holds `rows` tokens, each with the token before it.  A row's state is the sum of both tokens' rows of the
table, normalised; a frozen head gives logits over the vocabulary, and the teacher, a model of the same kind, gives its best
alternatives (cr_token_log_probs), which cr_distill trains on.  A step computes every partition's partial gradient of the
table (cr_embedding_backward) and of gamma (cr_rms_norm_backward), puts them into the slots of the workers that hold it and
decodes both from those that did not straggle (cr_aggregate).  The model answers in 8 bits: cr_rms_norm_codes,
cr_int8_product, cr_token_log_probs.

    python examples/coded_tokens.py [--steps 20]
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

EPS, TOP, TEMPERATURE = 1e-5, 8, 2.0


class CodedTokens:
    """(n, L)-tree of workers, `P` partitions of `rows` tokens over a vocabulary, states of `width` numbers."""

    def __init__(self, n=4, L=2, s=1, P=24, rows=64, vocab=500, width=48, seed=0):
        self.P, self.rows, self.vocab, self.width, self.count = P, rows, vocab, width, P * rows
        self.scale = width ** 0.5
        device = torch.cuda.current_device()
        # one plan per gradient vector; the same code, so the same slots and straggler masks
        self.table_plan = B.cr_plan_create(n, L, s, P, vocab * width, device=device)
        self.norm_plan = B.cr_plan_create(n, L, s, P, width, device=device)
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
        new = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
        # tokens of each partition, then the tokens before them: one list per partition, as the table's gradient takes it
        self.ids = (vocab ** torch.rand((P, 2, rows), generator=g, device="cuda")).long().clamp_(max=vocab) - 1
        self.ids[:, 1, 0] = -1                               # the first token has none before it
        self.head = rand(vocab, width) / width ** 0.5
        self.codes = torch.zeros((vocab, (width + 15) // 16 * 16), dtype=torch.int8, device="cuda")[:, :width]
        self.codes_scale = new(vocab)
        B.cr_quantize_rows(self.table_plan, self.head, self.codes, self.codes_scale)
        self.both, self.h, self.y = new(P, 2, rows, width), new(P, rows, width), new(P, rows, width)
        self.rstd, self.logits = new(self.count), new(self.count, vocab)
        self.loss, self.dlogits, self.dy = new(self.count), new(self.count, vocab), new(P, rows, width)
        self.dboth, self.dtable, self.dgamma = new(P, 2, rows, width), new(P, vocab, width), new(P, width)
        N, m = B.cr_plan_num_nodes(self.table_plan), B.cr_plan_load(self.table_plan)
        self.slot_part = torch.from_numpy(B.slot_partitions(self.table_plan).astype(np.int64).reshape(-1)).cuda()
        self.table_slots, self.norm_slots = new(N, m, vocab * width), new(N, m, width)
        self.table_grad, self.norm_grad = new(1, vocab * width), new(1, width)
        scratch = max(16, B.cr_embedding_backward_workspace_bytes(self.table_plan, self.ids, self.dtable),
                      B.cr_rms_norm_backward_workspace_bytes(self.table_plan, self.h, P))
        self.workspace = torch.empty(scratch, dtype=torch.uint8, device="cuda")
        # the teacher: tables of its own, whose best alternatives are kept
        self.table, self.gamma = rand(vocab, width) / width, 1 + 0.2 * rand(width)
        self.forward()
        self.teacher, self.teacher_ids = new(self.count, TOP), torch.empty((self.count, TOP), dtype=torch.int64, device="cuda")
        B.cr_token_log_probs(self.table_plan, self.logits, None, top_logp=self.teacher, top_ids=self.teacher_ids)
        self.table, self.gamma = rand(vocab, width) / width, torch.ones(width, device="cuda")

    def close(self):
        B.cr_plan_destroy(self.table_plan)
        B.cr_plan_destroy(self.norm_plan)

    def forward(self, part=slice(None)):
        """Logits of the partitions `part`; a partition's numbers do not depend on what is processed beside it."""
        both, h, y = self.both[part], self.h[part], self.y[part]
        rows = slice(*(k * self.rows for k in part.indices(self.P)[:2]))
        B.cr_embedding(self.table_plan, self.ids[part], self.table, both, scale=self.scale)
        for p in range(both.shape[0]):                        # a partition's tokens and those before them lie one behind the other
            B.cr_rms_norm(self.table_plan, both[p, 0], self.gamma, y[p], residual=both[p, 1], h=h[p],
                          rstd=self.rstd[rows][p * self.rows:(p + 1) * self.rows], eps=EPS)
        torch.mm(y.view(-1, self.width), self.head.t(), out=self.logits[rows])
        return self.logits[rows]

    def step(self, masks, rate):
        """One step of gradient descent under the straggler pattern `masks`; returns the loss before it."""
        self.forward()
        B.cr_distill(self.table_plan, self.logits, self.teacher_ids, self.teacher, self.loss, self.dlogits, temperature=TEMPERATURE)
        torch.mm(self.dlogits, self.head, out=self.dy.view(-1, self.width))
        # both summands of the state have the same gradient
        dx = self.dy
        B.cr_rms_norm_backward(self.table_plan, self.dy, self.h, self.gamma, self.rstd, dx, self.dgamma, workspace=self.workspace)
        self.dboth.copy_(dx[:, None])
        B.cr_embedding_backward(self.table_plan, self.ids, self.dboth, self.dtable, scale=self.scale, workspace=self.workspace)
        torch.index_select(self.dtable.view(self.P, -1), 0, self.slot_part, out=self.table_slots.view(-1, self.vocab * self.width))
        torch.index_select(self.dgamma, 0, self.slot_part, out=self.norm_slots.view(-1, self.width))
        B.cr_aggregate(self.table_plan, self.table_slots, masks, self.table_grad)
        B.cr_aggregate(self.norm_plan, self.norm_slots, masks, self.norm_grad)
        self.table -= rate / self.count * self.table_grad.view(self.vocab, self.width)
        self.gamma -= rate / self.count * self.norm_grad[0]
        return float(self.loss.mean())

    def answer(self, part, top=3):
        """The model's answers for a partition in 8 bits: (entropy, best alternatives, their log probabilities) a row."""
        B.cr_embedding(self.table_plan, self.ids[part], self.table, self.both[part], scale=self.scale)
        x, r = self.both[part]
        q = torch.empty((self.rows, self.codes.stride(0)), dtype=torch.int8, device="cuda")[:, :self.width]
        scale, logits = torch.empty(self.rows, device="cuda"), torch.empty((self.rows, self.vocab), device="cuda")
        B.cr_rms_norm_codes(self.table_plan, x, self.gamma, q, scale, residual=r, eps=EPS)
        B.cr_int8_product(self.table_plan, q, scale, self.codes, self.codes_scale, logits)
        entropy, logp = torch.empty(self.rows, device="cuda"), torch.empty((self.rows, top), device="cuda")
        ids = torch.empty((self.rows, top), dtype=torch.int64, device="cuda")
        B.cr_token_log_probs(self.table_plan, logits, None, entropy=entropy, top_logp=logp, top_ids=ids)
        return entropy, ids, logp, logits


def train(steps=20, rate=2.0, seed=0, **shape):
    """Losses of `steps` steps, every one with a random straggler in every sibling group."""
    model = CodedTokens(seed=seed, **shape)
    try:
        masks = inputs.straggler_masks(shape.get("n", 4), shape.get("L", 2), shape.get("s", 1), steps, seed=seed + 1, exactly_s=True)
        return [model.step(masks[t], rate) for t in range(steps)]
    finally:
        model.close()


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=20)
    losses = train(ap.parse_args().steps)
    print("loss", " ".join(f"{v:.4f}" for v in losses))
