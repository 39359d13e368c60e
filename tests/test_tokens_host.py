"""What the token layers refuse, and what they ask for, without a device."""
import pytest

from paper_1902_01981_b200 import binding as B

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def plan():
    p = B.cr_plan_create(4, 2, 1, 24, 1024)
    yield p
    B.cr_plan_destroy(p)


def test_tensors_of_the_host_are_refused(plan):
    x, ids = torch.zeros(4, 16), torch.zeros(4, dtype=torch.int64)
    v, many = torch.zeros(4), torch.zeros((4, 3), dtype=torch.int64)
    calls = [lambda: B.cr_embedding(plan, ids, x, x), lambda: B.cr_embedding_backward(plan, ids, x, x),
             lambda: B.cr_rms_norm(plan, x, None, x), lambda: B.cr_rms_norm_codes(plan, x, None, x.to(torch.int8), v),
             lambda: B.cr_rms_norm_backward(plan, x, x, None, v, x), lambda: B.cr_token_log_probs(plan, x, ids, v),
             lambda: B.cr_token_log_probs_backward(plan, x, ids, torch.zeros(4, 2), v, v, v, x),
             lambda: B.cr_distill(plan, x, many, torch.zeros(4, 3), v)]
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_shapes_are_refused_before_anything_else(plan):
    x, ids = torch.zeros(4, 16), torch.zeros(4, dtype=torch.int64)
    calls = [lambda: B.cr_embedding(plan, ids, x[0], x), lambda: B.cr_embedding_backward(plan, ids, x, torch.zeros(2, 3, 16)),
             lambda: B.cr_embedding_backward(plan, ids, x, x, padding=1 << 64), lambda: B.cr_rms_norm(plan, torch.tensor(1.0), None, x),
             lambda: B.cr_rms_norm(plan, x[:, :0], None, x), lambda: B.cr_token_log_probs(plan, x[0], ids),
             lambda: B.cr_token_log_probs(plan, x[:, :0], ids), lambda: B.cr_distill(plan, x, ids, x)]
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_workspaces(plan):
    """Grow with what they hold, and are 0 where nothing is needed or nothing can be asked for."""
    ids, table = torch.zeros((3, 100), dtype=torch.int64), torch.zeros(3, 50, 8)
    need = B.cr_embedding_backward_workspace_bytes(plan, ids, table)
    assert need >= 3 * 100 * 16 and need % 16 == 0
    lib = B.lib()
    ask = lambda *a: lib.cr_embedding_backward_workspace_bytes(plan, *a)  # noqa: E731
    assert ask(100, 3, 50, 8) == need
    assert ask(0, 3, 50, 8) == 0 and ask(100, 0, 50, 8) == 0 and ask(100, 3, 0, 8) == 0 and ask(100, 3, 50, 0) == 0
    assert ask(-1, 3, 50, 8) == 0 and ask((1 << 30) + 1, 1, 50, 8) == 0 and ask(100, 3, 1 << 31, 8) == 0
    assert ask(1 << 30, 1, 50, 8) > 16 << 30
    x = torch.zeros(12, 64)
    assert B.cr_rms_norm_backward_workspace_bytes(plan, x, 3) >= 12 * 4
    ask = lambda *a: lib.cr_rms_norm_backward_workspace_bytes(plan, *a)  # noqa: E731
    assert ask(12, 64, 5) == 0 and ask(12, 64, 0) == 0 and ask(12, 0, 3) == 0 and ask(0, 64, 3) == 0
    assert ask(16384, 4096, 8) == 16384 * 4 + 8 * 256 * 4096 * 4


def test_workspaces_of_tables_up_to_the_device(plan):
    """Asked for as long as such tables could lie on a device, and not beyond."""
    ask = lambda *a: B.lib().cr_embedding_backward_workspace_bytes(plan, *a)  # noqa: E731
    for parts, vocab in ((1 << 24, 2080), (1 << 24, 32), (24, 2 ** 31 - 1)):
        assert parts * vocab * 4 > 1 << 30 and ask(1, parts, vocab, 1) > 0
    for parts, vocab in ((1 << 24, 4096), (800, 2 ** 31 - 1)):
        assert parts * vocab * 4 > 200e9 and ask(1, parts, vocab, 1) == 0


def test_a_host_only_plan_does_no_device_work(plan):
    assert B.lib().cr_rms_norm(plan, 16, 8, None, 0, None, None, 0, 16, 8, None, 1, 8, B.CR_ELEM_F32, 1e-5, None) == B.CR_ERR_CUDA
    assert B.lib().cr_embedding(plan, 16, 8, 16, 8, 16, 8, 1, 1, 8, B.CR_ELEM_F32, 1.0, None) == B.CR_ERR_CUDA
    assert B.lib().cr_distill(plan, 16, 8, 16, 8, 16, 1, None, 16, None, 0, 1, 8, B.CR_ELEM_F32, 1.0, None) == B.CR_ERR_CUDA
