"""The layers, the partial gradients and the coded aggregation together: examples/coded_network.py."""
import numpy as np
import pytest

from oracle import cr_layers as O
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


def test_a_step_under_stragglers_is_the_gradient_of_the_whole_data_set():
    from examples.coded_network import DROP, EPS, CodedNetwork
    net = CodedNetwork(rows=6, positions=9, inner=50, channels=40, groups=5, seed=3)
    try:
        # a head that is not zero, so that the normalisation has a gradient
        net.w.copy_(torch.randn(net.d, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda") / net.d ** 0.5)
        w, gamma, beta = f64(net.w), f64(net.gamma), f64(net.beta)
        masks = inputs.straggler_masks(4, 2, 1, 1, seed=9, exactly_s=True)[0]
        step = 17
        net.step(step, masks, rate=0.0)
        n, s, c = net.h.shape
        # the frozen layer: codes exact, features within the rounding of four fp32 operations
        codes, scale = O.quantize_rows(net.images.cpu().numpy())
        wc = net.w_codes.cpu().numpy().astype(np.int64)
        h, _ = O.int8_product(codes, wc, scale, net.w_scale.cpu().numpy())
        assert np.max(np.abs(f64(net.h).reshape(n * s, c) - h)) <= 1e-6 * np.max(np.abs(h))
        # from the very h that the kernels had: features, residuals, gradients of the sum over all images
        x = f64(net.h)
        factors = O.dropout_factors((n, s, c), DROP, step, 0)
        y, _, _, _ = O.group_norm(x, gamma, beta, net.groups, EPS, "silu", factors)
        flat = y.reshape(n, s * c)
        residual = flat @ w - f64(net.labels)
        want_w = flat.T @ residual
        dy = (residual[:, None] * w[None, :]).reshape(n, s, c)
        _, dg, db, _, _, _ = O.group_norm_backward(dy, x, gamma, beta, net.groups, EPS, "silu", factors)
        want = np.concatenate([dg[0], db[0]])
        rel = lambda a, b: np.linalg.norm(a - b) / np.linalg.norm(b)  # noqa: E731
        # fp32 throughout, amplified by the code's conditioning (at most 100 of 6e-8 a step, mostly cancelling)
        assert rel(f64(net.head_grad[0]), want_w) <= 1e-5
        assert rel(f64(net.norm_grad[0]), want) <= 1e-5
    finally:
        net.close()


def test_a_worker_gets_the_bits_of_its_partition():
    """Each holder of a partition computes the same features, whatever it processes beside it."""
    from examples.coded_network import CodedNetwork
    net = CodedNetwork(rows=5, positions=12, seed=5)
    try:
        whole = net.forward(8).clone()
        net.features.zero_()
        for p in (7, 0, 23):
            alone = net.forward(8, first=p * net.rows, count=net.rows)
            assert torch.equal(alone, whole[p * net.rows:(p + 1) * net.rows])
    finally:
        net.close()


def test_training_lowers_the_loss():
    from examples.coded_network import train
    losses = train(steps=12)
    assert np.isfinite(losses).all() and losses[-1] < 0.7 * losses[0]
