"""The token layers, the 8-bit product and the coded aggregation together: examples/coded_tokens.py."""
import numpy as np
import pytest

from oracle import cr_layers as L
from oracle import cr_tokens as O
from paper_1902_01981_b200 import binding as B
from paper_1902_01981_b200 import build as cr_build
from paper_1902_01981_b200 import inputs

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def built():
    cr_build.build()
    assert torch.cuda.is_available()


def f64(t):
    return t.detach().double().cpu().numpy()


def whole_loss(net, table, gamma, teacher_ids, teacher, temperature):
    """The sum of the losses over all tokens in 64 bits, with the arrays that lead to it."""
    ids = net.ids.cpu().numpy()
    both = O.embedding(ids, table, net.scale)
    y, h, rstd = O.rms_norm(both[:, 0], both[:, 1], gamma, 1e-5)
    x = y.reshape(-1, net.width) @ f64(net.head).T
    loss, d = O.distill(x, teacher_ids, teacher, None, temperature)
    return loss.sum(), ids, h, rstd, d


def test_a_step_under_stragglers_is_the_gradient_of_the_whole_data_set():
    from examples.coded_tokens import TEMPERATURE, CodedTokens
    net = CodedTokens(rows=37, vocab=211, width=40, seed=3)
    try:
        table, gamma = f64(net.table), f64(net.gamma)
        masks = inputs.straggler_masks(4, 2, 1, 1, seed=9, exactly_s=True)[0]
        net.step(masks, rate=0.0)
        tid, t = net.teacher_ids.cpu().numpy(), f64(net.teacher)
        loss, ids, h, rstd, d = whole_loss(net, table, gamma, tid, t, TEMPERATURE)
        dy = (d @ f64(net.head)).reshape(net.P, net.rows, net.width)
        dx, dgamma, _ = O.rms_norm_backward(dy, h, gamma, rstd)
        dtable, _ = O.embedding_backward(ids.reshape(1, -1), np.stack([dx, dx], 1).reshape(1, -1, net.width), net.vocab, net.scale)
        rel = lambda a, b: np.linalg.norm(a - b) / np.linalg.norm(b)  # noqa: E731
        # fp32 throughout (the products of torch.mm in TF32 or better would show at 1e-3), amplified by the code's conditioning
        assert rel(f64(net.loss.sum()), loss) <= 1e-5
        assert rel(f64(net.table_grad).reshape(net.vocab, net.width), dtable[0]) <= 2e-5
        assert rel(f64(net.norm_grad[0]), dgamma[0]) <= 2e-5
        # and that of differences: along the gradient itself the loss rises by its squared norm
        step = 1e-4
        up = whole_loss(net, table + step * dtable[0] / np.linalg.norm(dtable[0]), gamma, tid, t, TEMPERATURE)[0]
        down = whole_loss(net, table - step * dtable[0] / np.linalg.norm(dtable[0]), gamma, tid, t, TEMPERATURE)[0]
        assert abs((up - down) / (2 * step) / np.linalg.norm(dtable[0]) - 1) <= 1e-4
    finally:
        net.close()


def test_a_worker_gets_the_bits_of_its_partition():
    """Each holder of a partition computes the same numbers, whatever it processes beside it."""
    from examples.coded_tokens import CodedTokens
    net = CodedTokens(rows=50, vocab=300, width=24, seed=5)
    try:
        net.step(inputs.straggler_masks(4, 2, 1, 1, seed=2, exactly_s=True)[0], rate=0.0)
        y, rstd, dgamma, dtable = net.y.clone(), net.rstd.clone(), net.dgamma.clone(), net.dtable.clone()
        net.y.zero_()
        for p in (7, 0, 23):
            one = slice(p, p + 1)
            net.forward(one)
            assert torch.equal(net.y[p], y[p]) and torch.equal(net.rstd, rstd)
            need = B.cr_embedding_backward_workspace_bytes(net.table_plan, net.ids[one], net.dtable[one])
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            net.dtable[one].fill_(float("nan"))
            B.cr_embedding_backward(net.table_plan, net.ids[one], net.dboth[one], net.dtable[one], scale=net.scale, workspace=ws)
            assert torch.equal(net.dtable, dtable) and torch.equal(net.dgamma, dgamma)
    finally:
        net.close()


def test_a_worker_gets_the_bits_of_its_norm_gradient():
    """The gradient of gamma, and that of the state, of one partition alone."""
    from examples.coded_tokens import CodedTokens
    net = CodedTokens(rows=50, vocab=300, width=24, seed=5)
    try:
        net.step(inputs.straggler_masks(4, 2, 1, 1, seed=2, exactly_s=True)[0], rate=0.0)
        dx, dgamma = net.dy.clone(), net.dgamma.clone()
        torch.mm(net.dlogits, net.head, out=net.dy.view(-1, net.width))         # the step has written dx over it
        dy = net.dy.clone()
        assert not torch.equal(dy, dx)
        for p in (7, 0, 23):
            one, rows = slice(p, p + 1), slice(p * net.rows, (p + 1) * net.rows)
            net.dgamma[one] = float("nan")
            ws = torch.empty(B.cr_rms_norm_backward_workspace_bytes(net.norm_plan, net.h[one]), dtype=torch.uint8, device="cuda")
            B.cr_rms_norm_backward(net.norm_plan, dy[one], net.h[one], net.gamma, net.rstd[rows], net.dy[one], net.dgamma[one], workspace=ws)
            assert torch.equal(net.dgamma, dgamma) and torch.equal(net.dy[one], dx[one])
    finally:
        net.close()


def test_answers_in_eight_bits():
    from examples.coded_tokens import CodedTokens
    net = CodedTokens(rows=40, vocab=333, width=64, seed=6)
    try:
        entropy, ids, logp, logits = net.answer(4)
        _, _, _, want_e, want_ids, want_lp = O.token_log_probs(f64(logits), np.zeros(40, dtype=int), 1.0, 3)
        assert np.array_equal(ids.cpu().numpy(), want_ids)
        assert np.allclose(f64(logp), want_lp, atol=1e-5) and np.allclose(f64(entropy), want_e, atol=1e-4)
        # the logits against the model without codes: every code is half a step of 1/127 of its row's largest value off
        both = O.embedding(net.ids[4].cpu().numpy(), f64(net.table), net.scale)
        y, _, _ = O.rms_norm(both[0], both[1], f64(net.gamma), 1e-5)
        w = f64(net.head)
        step_y, step_w = np.abs(y).max(1) / 254, np.abs(w).max(1) / 254
        bound = np.outer(step_y, np.abs(w).sum(1)) + np.outer(np.abs(y).sum(1), step_w) + net.width * np.outer(step_y, step_w)
        assert np.all(np.abs(f64(logits) - y @ w.T) <= 1.001 * bound + 1e-5)
        codes, scale = L.quantize_rows(net.head.cpu().numpy())
        assert np.array_equal(net.codes.cpu().numpy(), codes) and np.array_equal(net.codes_scale.cpu().numpy(), scale)
    finally:
        net.close()


def test_training_runs():
    from examples.coded_tokens import train
    losses = train(steps=4, rows=20, vocab=97, width=16)
    assert len(losses) == 4 and np.isfinite(losses).all()
