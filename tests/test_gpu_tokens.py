"""Embedding, root-mean-square norm, log probabilities of tokens and distillation against 64-bit arithmetic."""
import numpy as np
import pytest

from oracle import cr_layers as L
from oracle import cr_tokens as O
from paper_1902_01981_b200 import binding as B
from paper_1902_01981_b200 import build as cr_build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# a stored value is off by half a step of its type at most: relative, and f16's smallest step besides
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}
STEP = 2.0 ** -24        # an fp32 operation


@pytest.fixture(scope="module", autouse=True)
def built():
    cr_build.build()
    assert torch.cuda.is_available()


@pytest.fixture(scope="module")
def plan():
    p = B.cr_plan_create(4, 2, 1, 24, 1024, device=0)
    yield p
    torch.cuda.synchronize()
    assert B.cr_plan_device_status(p) == B.CR_OK
    B.cr_plan_destroy(p)


def f64(t):
    return t.detach().double().cpu().numpy()


def place(values, dtype, pad=0, shift=0):
    """`values` on the device as rows that are `pad` elements longer, `shift` elements behind an aligned address; what lies
    between and behind the rows is NaN."""
    shape = tuple(np.shape(values))
    width = shape[-1] + pad
    store = torch.full((int(np.prod(shape[:-1])) * width + shift + 8,), float("nan"), dtype=TYPES[dtype], device="cuda")
    strides, step = [1], width
    for n in reversed(shape[1:-1]):
        strides.insert(0, step)
        step *= n
    strides.insert(0, step)
    view = torch.as_strided(store, shape, strides if len(shape) > 1 else [1], shift)
    view.copy_(torch.from_numpy(np.asarray(values, dtype=np.float32)))
    view.store = store
    return view


def outside_untouched(view):
    """Whether everything of place()'s memory that is no element of the view is still NaN."""
    store = view.store.clone()
    torch.as_strided(store, view.shape, view.stride(), view.storage_offset()).fill_(float("nan"))
    return bool(torch.isnan(store).all())


def check(got, want, dtype, arith):
    """`arith`: the bound of the fp32 arithmetic in front of the one rounding, a number or an array."""
    got, want = f64(got), np.asarray(want, dtype=np.float64)
    assert got.shape == want.shape
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True)
    tol = np.where(odd, 0, HALF[dtype] * np.abs(np.where(odd, 0, want)) * 1.01 + TINY[dtype] + arith)
    off = np.abs(np.where(odd, 0, got) - np.where(odd, 0, want))
    bad = ~(off <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size}; worst {off.max():.3e}, allowed there {np.broadcast_to(tol, off.shape)[off == off.max()][0]:.3e}"


def dev32(v):
    return None if v is None else torch.from_numpy(np.asarray(v, dtype=np.float32)).cuda()


def dev_ids(v, kind):
    return torch.from_numpy(np.asarray(v).astype({"i32": np.int32, "i64": np.int64}[kind])).cuda()


def scratch(nbytes):
    """Workspace of exactly that size, in front of bytes that must stay."""
    return torch.full((nbytes + 64,), 0x5A, dtype=torch.uint8, device="cuda")


def whole(ws, nbytes):
    return bool((ws[nbytes:] == 0x5A).all())


# ------------------------------------------------------------------------------------------------ embedding

# tokens, vocab, width, pad, shift
LOOKUPS = [(1, 1, 1, 0, 0), (7, 5, 8, 0, 0), (39, 5004, 60, 0, 0), (39, 5004, 60, 4, 1), (130, 257, 5, 0, 0), (3, 11, 4096, 0, 0),
           (2, 3, 20001, 0, 0), (1000, 33, 96, 8, 0), (5, 100, 2056, 0, 3), (70000, 9, 16, 0, 0)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", LOOKUPS)
def test_lookup(plan, shape, dtype):
    tokens, vocab, width, pad, shift = shape
    rng = np.random.default_rng(tokens + width)
    table = place(rng.standard_normal((vocab, width)), dtype, pad, shift)
    ids = rng.integers(0, vocab, tokens)
    ids[::5] = [-1, vocab, vocab + 3, -(2 ** 31)][tokens % 4]     # names nothing
    if tokens > 1:
        ids[-1] = vocab - 1
    kind = ["i32", "i64"][tokens % 2]
    y = place(np.zeros((tokens, width)), dtype, pad, shift)
    scale = [1.0, 0.3, width ** 0.5][width % 3]
    B.cr_embedding(plan, dev_ids(ids, kind), table, y, scale=scale)
    want = O.embedding(ids, f64(table), scale)
    check(y, want, dtype, 3 * STEP * np.abs(want))      # the factor's rounding and the product's
    assert outside_untouched(y)


def test_lookup_of_nothing(plan):
    table = torch.randn(4, 16, device="cuda")
    B.cr_embedding(plan, torch.empty(0, dtype=torch.int64, device="cuda"), table, torch.empty((0, 16), device="cuda"))
    y = torch.full((3, 16), 7.0, device="cuda")
    B.cr_embedding(plan, torch.zeros(3, dtype=torch.int64, device="cuda"), torch.empty((0, 16), device="cuda"), y)
    assert not y.any()            # an empty table has no row 0
    ids = torch.tensor([[2 ** 40, 1], [-(2 ** 40), 2 ** 32 + 1]], device="cuda")
    y = torch.full((2, 2, 16), 7.0, device="cuda")
    B.cr_embedding(plan, ids, table, y)
    assert torch.equal(y[0, 1], table[1]) and not y[0, 0].any() and not y[1].any()


# partitions, tokens, vocab, width, pad, shift
TABLES = [
    (1, 1, 1, 1, 0, 0),
    (1, 0, 5, 8, 0, 0),            # no tokens: zeros
    (1, 33, 2, 8, 0, 0),           # one more than a tile
    (3, 39, 257, 60, 4, 0),
    (3, 39, 257, 60, 4, 1),        # off every boundary
    (2, 1000, 1, 16, 0, 0),        # all tokens the same: a sum over all tiles
    (2, 1025, 3, 36, 0, 0),        # more than one CTA sorts
    (1, 5000, 70000, 8, 0, 0),     # three digits
    (4, 300, 255, 130, 0, 0),
    (2, 4097, 256, 264, 0, 0),
    (1, 20000, 300, 20, 0, 2),
    (5, 64, 1000, 1032, 0, 0),
    (2, 64, 1, 8, 0, 0),           # the longest sum that is not cut
    (2, 65, 1, 8, 0, 0),           # the shortest that is
    (1, 2100, 40, 516, 0, 0),      # sums of about 64 tokens
    (24, 39, 5004, 12, 0, 0),
    (1, 140000, 40, 8, 0, 0),      # longer tiles
]


def grads(plan, ids, dy, vocab, scale=1.0, padding=-1, ld_pad=0):
    parts, width = ids.shape[0], dy.shape[-1]
    store = torch.full((parts, vocab + (1 if ld_pad else 0), width + ld_pad), float("nan"), device="cuda")
    d = store[:, :vocab, :width]
    need = B.cr_embedding_backward_workspace_bytes(plan, ids, d)
    ws = scratch(need)
    B.cr_embedding_backward(plan, ids, dy, d, scale=scale, padding=padding, workspace=ws[:need] if need else None)
    assert whole(ws, need)
    if ld_pad:
        assert torch.isnan(store[:, :, width:]).all() and torch.isnan(store[:, vocab:]).all()
    return d


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", TABLES)
def test_table_gradient(plan, shape, dtype):
    parts, tokens, vocab, width, pad, shift = shape
    rng = np.random.default_rng(tokens + vocab)
    # a few numbers often, most seldom, some that name nothing
    ids = np.minimum((vocab ** rng.random((parts, tokens))).astype(np.int64) - 1, vocab - 1)
    ids = np.where(rng.random(ids.shape) < 0.1, [-1, vocab, -(2 ** 31)][vocab % 3], ids)
    dy = place(rng.standard_normal((parts, tokens, width)), dtype, pad, shift) if tokens else torch.empty((parts, 0, width), dtype=TYPES[dtype], device="cuda")
    padding = [-1, 0][vocab % 2]
    scale = width ** 0.5
    kind = ["i32", "i64"][tokens % 2]
    want, size = O.embedding_backward(ids, f64(dy), vocab, scale, padding)
    d = grads(plan, dev_ids(ids, kind), dy, vocab, scale, padding, ld_pad=[0, 4, 3][width % 3])
    # a chain of at most `tile` additions, then of the pieces: 4 to 256 threads share them, so at most a quarter of the tiles and
    # 256 sums more, or all tiles one by one; rounding of the factor and the product.  Each addition's error is 2^-24 of a
    # partial sum, which the sum of the terms' sizes bounds
    tile = 32
    while tokens // tile > 4096:
        tile *= 2
    tiles = (tokens + tile - 1) // tile
    chain = min(tokens, tile + 63) + min(tiles, tiles / 4 + 256) + 4      # a tile may begin up to 63 tokens early
    check(d, want, "f32", chain * STEP * size)
    again = grads(plan, dev_ids(ids, kind), dy, vocab, scale, padding, ld_pad=[0, 4, 3][width % 3])
    assert torch.equal(d, again)


@pytest.mark.parametrize("tokens", [5, 64, 1500, 5000])
def test_table_gradient_of_padding(plan, tokens):
    """Partitions without a named token beside one that has a single one; an infinite gradient stays in its row."""
    ids = torch.full((3, tokens), -1, dtype=torch.int64, device="cuda")
    ids[1, tokens // 2] = 6
    ids[2, :] = 3                                     # the padding's own number
    dy = torch.randn(3, tokens, 40, device="cuda")
    dy[1, tokens // 2, 7] = float("inf")
    dy[0, 0, 0] = float("nan")                        # of a token that names nothing
    d = grads(plan, ids, dy, 50, scale=2.0, padding=3)
    want = torch.zeros((3, 50, 40), device="cuda")
    want[1, 6] = 2 * dy[1, tokens // 2]
    assert torch.equal(d, want)


def test_table_gradient_of_a_partition_has_the_bits_of_the_batch(plan):
    rng = np.random.default_rng(5)
    ids = dev_ids(np.minimum((500 ** rng.random((6, 3000))).astype(np.int64) - 1, 499), "i64")
    dy = place(rng.standard_normal((6, 3000, 72)), "bf16")
    d = grads(plan, ids, dy, 500)
    for p in (0, 3, 5):
        assert torch.equal(d[p], grads(plan, ids[p:p + 1].contiguous(), dy[p:p + 1], 500)[0])
    one = torch.full((500, 72), float("nan"), device="cuda")
    need = B.cr_embedding_backward_workspace_bytes(plan, ids[2], one)
    B.cr_embedding_backward(plan, ids[2], dy[2], one, workspace=scratch(need))
    assert torch.equal(one, d[2])


# ------------------------------------------------------------------------------------------------ root-mean-square norm

# rows, cols, pad, shift
NORMS = [(1, 1, 0, 0), (3, 8, 0, 0), (5, 60, 4, 0), (5, 60, 4, 1), (1, 4096, 0, 0), (39, 5004, 0, 0), (7, 1001, 0, 0), (300, 128, 0, 0),
         (2, 16384, 0, 0), (3, 20000, 0, 0), (2, 40000, 0, 0), (2, 17001, 0, 0), (3, 33001, 7, 0), (1000, 33, 0, 0), (64, 2056, 8, 0), (2, 70000, 0, 0)]


def norm_inputs(shape, dtype, seed, residual):
    rows, cols, pad, shift = shape
    rng = np.random.default_rng(seed)
    spread = np.exp(rng.standard_normal((rows, 1)))
    x = place(rng.standard_normal((rows, cols)), dtype, pad, shift)
    r = place(2 * spread * rng.standard_normal((rows, cols)), dtype, pad, shift) if residual else None
    return x, r, dev32(1 + 0.2 * rng.standard_normal(cols)) if seed % 3 else None


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", NORMS)
def test_norm_forward_and_backward(plan, shape, dtype):
    rows, cols, pad, shift = shape
    seed = rows + cols
    x, r, gamma = norm_inputs(shape, dtype, seed, seed % 2 == 0)
    y, h = place(np.zeros((rows, cols)), dtype, pad, shift), place(np.zeros((rows, cols)), dtype, pad, shift)
    rstd = torch.full((rows,), float("nan"), device="cuda")
    eps = 1e-5
    B.cr_rms_norm(plan, x, gamma, y, residual=r, h=h, rstd=rstd, eps=eps)
    g64 = None if gamma is None else f64(gamma)
    want_y, want_h, want_r = O.rms_norm(f64(x), None if r is None else f64(r), g64, eps)
    # a sum of squares: positive terms, so its relative error is that of the chain a thread adds up (at most 128 vectors of up
    # to 8 elements; five levels of two reductions); the root halves it
    chain = min(cols, 1100) + 16
    check(h, want_h, dtype, STEP * np.abs(want_h))
    check(rstd, want_r, "f32", (chain / 2 + 4) * STEP * want_r)
    check(y, want_y, dtype, (chain / 2 + 8) * STEP * np.abs(want_y))
    assert outside_untouched(y) and outside_untouched(h)
    # backward, from what the forward pass has left
    rng = np.random.default_rng(seed + 1)
    parts = next(k for k in (7, 5, 3, 2, 1) if rows % k == 0)
    dy = place(rng.standard_normal((rows, cols)), dtype, pad, shift)
    dh = place(rng.standard_normal((rows, cols)), dtype, pad, shift) if rows % 2 else None
    dx = place(np.zeros((rows, cols)), dtype, pad, shift)
    wide = torch.full((parts, cols + 5), float("nan"), device="cuda")
    need = B.cr_rms_norm_backward_workspace_bytes(plan, h, parts)
    ws = scratch(need)
    B.cr_rms_norm_backward(plan, dy, h, gamma, rstd, dx, wide[:, 1:cols + 1], dh=dh, workspace=ws[:need])
    assert whole(ws, need) and outside_untouched(dx) and torch.isnan(wide[:, 0]).all() and torch.isnan(wide[:, cols + 1:]).all()
    want_dx, want_dg, size_dg = O.rms_norm_backward(f64(dy), f64(h), g64, f64(rstd), None if dh is None else f64(dh), parts)
    # the mean of g xhat: its terms' sizes times the chain; xhat times that; a few operations on terms of their own size
    xhat = f64(h) * f64(rstd)[:, None]
    g = f64(dy) * (1.0 if g64 is None else g64)
    mean_size = (np.abs(g * xhat)).mean(1, keepdims=True)
    terms = f64(rstd)[:, None] * (np.abs(g) + np.abs(xhat) * mean_size) + (0 if dh is None else np.abs(f64(dh)))
    check(dx, want_dx, dtype, 8 * STEP * terms + f64(rstd)[:, None] * np.abs(xhat) * mean_size * chain * STEP)
    # at most 64 rows a chunk, 32 chunks a warp, eight warps; three roundings a term
    check(wide[:, 1:cols + 1], want_dg, "f32", (64 + 32 + 8 + 4) * STEP * size_dg)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", NORMS)
def test_norm_codes(plan, shape, dtype):
    rows, cols, pad, shift = shape
    x, r, gamma = norm_inputs(shape, dtype, rows + cols + 1, cols % 2 == 0)
    wide = torch.full((rows, (cols + 15) // 16 * 16 + 16), 99, dtype=torch.int8, device="cuda")
    q = wide[:, :cols]
    scale, rstd = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    h = place(np.zeros((rows, cols)), dtype, pad, shift)
    B.cr_rms_norm_codes(plan, x, gamma, q, scale, residual=r, h=h, rstd=rstd)
    want_y, want_h, want_r = O.rms_norm(f64(x), None if r is None else f64(r), None if gamma is None else f64(gamma), 1e-5)
    top = np.abs(want_y).max(1)
    chain = min(cols, 1100) / 2 + 24
    check(h, want_h, dtype, STEP * np.abs(want_h))
    check(scale, top / 127, "f32", chain * STEP * top / 127)
    # the code of a value is off by half a step and by what the fp32 y is off
    exact = want_y * (127 / np.where(top > 0, top, 1))[:, None]
    assert np.all(np.abs(f64(q) - exact) <= 0.5 + 4 * chain * STEP * 127)
    assert np.all(np.abs(f64(q)).max(1) == 127)
    assert (wide[:, cols:] == 99).all() and outside_untouched(h)


def test_norm_in_place(plan):
    for cols, dtype in ((4096, "bf16"), (1001, "f32"), (40000, "f16"), (40001, "bf16")):
        x, r, gamma = norm_inputs((6, cols, 0, 0), dtype, 7, True)
        y, h = torch.empty_like(x), torch.empty_like(x)
        B.cr_rms_norm(plan, x, gamma, y, residual=r, h=h)
        a, b = x.clone(), r.clone()
        B.cr_rms_norm(plan, a, gamma, a, residual=b, h=b)
        assert torch.equal(a, y) and torch.equal(b, h)
        dy, rstd = torch.randn_like(x), torch.rand(6, device="cuda")
        ws = scratch(B.cr_rms_norm_backward_workspace_bytes(plan, h, 2))
        dx, dg = torch.empty_like(x), torch.empty((2, cols), device="cuda")
        B.cr_rms_norm_backward(plan, dy, h, gamma, rstd, dx, dg, dh=x, workspace=ws)
        for which in range(3):
            t = [dy.clone(), h.clone(), x.clone()]
            dg2 = torch.empty_like(dg)
            B.cr_rms_norm_backward(plan, t[0], t[1], gamma, rstd, t[which], dg2, dh=t[2], workspace=ws)
            assert torch.equal(t[which], dx) and torch.equal(dg, dg2)


def test_norm_of_odd_rows(plan):
    """Zeros, infinities and NaN stay in their rows."""
    x = torch.randn(6, 512, device="cuda")
    x[1], x[2, 5], x[3, 7], x[4] = 0, float("inf"), float("nan"), 1e-30
    y, q, s = torch.empty_like(x), torch.empty((6, 512), dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    B.cr_rms_norm(plan, x, None, y)
    B.cr_rms_norm_codes(plan, x, None, q, s)
    assert torch.isfinite(y[[0, 1, 4, 5]]).all() and not y[1].any()
    assert not y[2, :5].any() and torch.isnan(y[2, 5])           # inf * 0
    assert torch.isnan(y[3]).all()
    assert s[1] == 0 and not q[1].any() and torch.isnan(s[2]) and torch.isnan(s[3]) and not q[2:4].any()
    assert s[4] > 0 and (q[4] == 127).all()


def test_norm_backward_parts(plan):
    """dx alone, dgamma alone, no rows."""
    x, _, gamma = norm_inputs((12, 264, 0, 0), "bf16", 4, False)
    dy, rstd = torch.randn_like(x), torch.rand(12, device="cuda")
    ws = scratch(B.cr_rms_norm_backward_workspace_bytes(plan, x, 3))
    dx, dg, dx2, dg2 = torch.empty_like(x), torch.empty((3, 264), device="cuda"), torch.empty_like(x), torch.empty((3, 264), device="cuda")
    B.cr_rms_norm_backward(plan, dy, x, gamma, rstd, dx, dg, workspace=ws)
    B.cr_rms_norm_backward(plan, dy, x, gamma, rstd, dx2, workspace=ws)
    B.cr_rms_norm_backward(plan, dy, x, gamma, rstd, None, dg2, workspace=ws)
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2)
    # a partition alone: the bits of the batch
    B.cr_rms_norm_backward(plan, dy[4:8], x[4:8], gamma, rstd[4:8], dx2[4:8], dg2[1:2], workspace=ws)
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2)
    none = torch.empty((0, 264), dtype=torch.bfloat16, device="cuda")
    B.cr_rms_norm_backward(plan, none, none, gamma, torch.empty(0, device="cuda"), none, dg)
    assert not dg.any()
    B.cr_rms_norm(plan, none, gamma, none)


# rows, cols, partitions: more chunks of 64 rows than 256, in one kernel and in two
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", [(40000, 8, 1), (34000, 7, 2), (16500, 8200, 1)])
def test_norm_gradient_of_long_partitions(plan, shape, dtype):
    rows, cols, parts = shape
    rng = np.random.default_rng(rows)
    if cols > 100:
        gen = torch.Generator(device="cuda").manual_seed(rows)
        h, dy = (torch.randn(rows, cols, generator=gen, device="cuda").to(TYPES[dtype]) for _ in range(2))
    else:
        h, dy = place(rng.standard_normal((rows, cols)), dtype), place(rng.standard_normal((rows, cols)), dtype)
    rstd = dev32(1 + 0.1 * rng.random(rows))
    dg, dx = torch.full((parts, cols), float("nan"), device="cuda"), torch.empty_like(h)
    need = B.cr_rms_norm_backward_workspace_bytes(plan, h, parts)
    ws = scratch(need)
    B.cr_rms_norm_backward(plan, dy, h, None, rstd, dx, dg, workspace=ws[:need])
    assert whole(ws, need)
    terms = dy.double() * h.double() * rstd.double()[:, None]
    want, size = f64(terms.view(parts, -1, cols).sum(1)), f64(terms.abs().view(parts, -1, cols).sum(1))
    # a chain of 64 rows, then every eighth chunk one after the other, then eight sums; three roundings a term
    chunks = -(-(rows // parts) // 64)
    check(dg, want, "f32", (64 + -(-chunks // 8) + 8 + 4) * STEP * size)


# ------------------------------------------------------------------------------------------------ log probabilities

# rows, vocab, pad, shift
VOCABS = [(1, 1, 0, 0), (2, 3, 0, 0), (3, 8, 0, 0), (5, 33, 0, 0), (4, 257, 0, 0), (39, 5004, 4, 0), (39, 5004, 4, 1), (7, 1000, 0, 0), (2, 32000, 0, 0),
          (3, 50257, 0, 0), (300, 200, 0, 0), (1, 128000, 0, 0), (2, 262145, 0, 0), (1, 300000, 0, 0), (700, 1024, 8, 0), (3, 2048, 0, 0), (3, 2056, 0, 0),
          (2, 1100001, 0, 0), (1, 2200000, 0, 0)]        # more chunks than slots


def logits_of(shape, dtype, seed, masked=0.2):
    rows, vocab, pad, shift = shape
    rng = np.random.default_rng(seed)
    x = 3 * rng.standard_normal((rows, vocab))
    x[:, rng.integers(0, vocab)] += 6
    off = rng.random((rows, vocab)) < masked
    off[:, rng.integers(0, vocab)] = False
    x[off] = -np.inf
    return place(x, dtype, pad, shift), rng


def log_arith(x64, temperature):
    """What log p may be off by: the difference to the largest logit, its product with the rounded factor, the logarithm of a
    sum of positive terms (a chain of at most 128 vectors of 8, a few levels of joining, ex2 to 2^-22)."""
    finite = np.where(np.isfinite(x64), x64, 0)
    span = np.abs(finite - finite.max(-1, keepdims=True)).max(-1) / temperature
    return (6 * span + min(x64.shape[-1], 1100) + 40) * STEP


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", VOCABS)
def test_log_probs_forward_and_backward(plan, shape, dtype):
    rows, vocab, pad, shift = shape
    temperature = [1.0, 0.7, 2.0][vocab % 3]
    x, rng = logits_of(shape, dtype, vocab, [0.0, 0.2][rows % 2])
    x64 = f64(x)
    ids = rng.integers(0, vocab, rows)
    ids = np.where(np.isfinite(x64[np.arange(rows), ids]), ids, x64.argmax(1))
    if rows > 2:
        ids[1] = [-1, vocab, -(2 ** 31)][rows % 3]
    kind = ["i32", "i64"][rows % 2]
    top = min(vocab, [1, 5, 20, 32][vocab % 4])
    dids = dev_ids(ids, kind)
    logp, entropy = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    stats, top_logp = torch.full((rows, 2), float("nan"), device="cuda"), torch.full((rows, top), float("nan"), device="cuda")
    top_ids = torch.full((rows, top), -7, dtype=dids.dtype, device="cuda")
    B.cr_token_log_probs(plan, x, dids, logp, stats, entropy, top_logp, top_ids, temperature=temperature)
    want_logp, m, log_sum, want_h, order, want_top = O.token_log_probs(x64, ids, temperature, top)
    arith = log_arith(x64, temperature)
    assert np.array_equal(top_ids.cpu().numpy(), order)
    check(logp, want_logp, "f32", arith)
    check(top_logp, want_top, "f32", arith[:, None])
    assert np.array_equal(f64(stats)[:, 0], m)
    check(stats[:, 1], log_sum, "f32", arith)
    # the entropy: log_sum, and a mean of u whose terms are as large as the span
    span = np.abs(np.where(np.isfinite(x64), x64 - m[:, None], 0)).max(1) / temperature
    check(entropy, want_h, "f32", arith * (1 + span))
    # the same without the alternatives, and each output alone
    alone = torch.full((rows,), float("nan"), device="cuda")
    B.cr_token_log_probs(plan, x, dids, alone, temperature=temperature)
    assert torch.equal(alone, logp)
    B.cr_token_log_probs(plan, x, None, entropy=alone, temperature=temperature)
    assert torch.equal(alone, entropy)
    # backward
    dlogp, dent = rng.standard_normal(rows), 0.3 * rng.standard_normal(rows)
    if rows > 3:
        dlogp[3] = dent[3] = 0
    a, b = dev32(dlogp), dev32(dent)
    p = np.exp(O.log_p(x64, temperature)[0])
    for da, db in ((a, b), (a, None), (None, b)):
        d = place(np.zeros((rows, vocab)), dtype, pad, shift)
        B.cr_token_log_probs_backward(plan, x, dids, stats, entropy, da, db, d, temperature=temperature)
        want = O.token_log_probs_backward(x64, ids, None if da is None else f64(da), None if db is None else f64(db), temperature)
        size = np.abs(0 if da is None else f64(da)) + np.abs(0 if db is None else f64(db)) * (2 * span + 4 + np.abs(want_h))
        # p is off by what log p is off (and ex2); each term by a few roundings; 1 - p where p is near one
        check(d, want, dtype, (size[:, None] * (p * (4 * arith[:, None] + 12 * STEP) + 2 * STEP * (np.arange(vocab) == ids[:, None])) / temperature))
        assert outside_untouched(d)
        other = place(np.zeros((rows, vocab)), dtype, pad + 1, shift + 3)       # rows that lie elsewhere relative to 16 bytes
        B.cr_token_log_probs_backward(plan, x, dids, stats, entropy, da, db, other, temperature=temperature)
        assert torch.equal(other, d) and outside_untouched(other)
        if da is a and db is b:
            y = x.clone() if x.is_contiguous() else x
            if y is not x:
                B.cr_token_log_probs_backward(plan, y, dids, stats, entropy, a, b, y, temperature=temperature)
                assert torch.equal(y, d)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_log_probs_rows_do_not_see_each_other(plan, dtype):
    for vocab in (1000, 5004, 50257):
        x, rng = logits_of((400, vocab, 0, 0), dtype, 3)
        x = x.contiguous()
        ids = dev_ids(np.zeros(400), "i64")
        out = [torch.empty(400, device="cuda"), torch.empty((400, 2), device="cuda"), torch.empty(400, device="cuda")]
        B.cr_token_log_probs(plan, x, ids, *out)
        for first, count in ((0, 1), (8, 3), (200, 39)):
            part = [torch.empty(count, device="cuda"), torch.empty((count, 2), device="cuda"), torch.empty(count, device="cuda")]
            rows = slice(first, first + count)
            B.cr_token_log_probs(plan, x[rows], ids[rows], *part)
            assert all(torch.equal(a, b[rows]) for a, b in zip(part, out))


@pytest.mark.parametrize("vocab,dtype,count", [(9001, "bf16", 700), (9008, "bf16", 700), (70000, "bf16", 700), (20000, "bf16", 1000), (32000, "f16", 900),
                                               (40008, "bf16", 450), (131080, "bf16", 120), (9004, "f32", 900), (20000, "f32", 450)])
def test_a_few_rows_have_the_bits_of_many(plan, vocab, dtype, count):
    """However many warps and CTAs share a row: scores, alternatives, loss and gradients."""
    x, rng = logits_of((count, vocab, 0, 0), dtype, 8)
    x = x.contiguous()
    ids, tid, t = dev_ids(rng.integers(0, vocab, count), "i64"), dev_ids(rng.integers(0, vocab, (count, 20)), "i64"), dev32(rng.standard_normal((count, 20)))

    def run(rows):
        n = rows.stop - rows.start
        out = [torch.empty(n, device="cuda"), torch.empty((n, 2), device="cuda"), torch.empty(n, device="cuda"),
               torch.empty((n, 20), device="cuda"), torch.empty((n, 20), dtype=torch.int64, device="cuda"), torch.empty(n, device="cuda"),
               torch.empty_like(x[rows])]
        B.cr_token_log_probs(plan, x[rows], ids[rows], *out[:5])
        B.cr_distill(plan, x[rows], tid[rows], t[rows], *out[5:])
        return out

    whole = run(slice(0, count))
    for rows in (slice(0, 1), slice(16, 55), slice(count // 3, count // 3 + 48), slice(count - 1, count)):
        assert all(torch.equal(a.nan_to_num(), b[rows].nan_to_num()) for a, b in zip(run(rows), whole))


def test_log_probs_of_odd_rows(plan):
    inf, nan = float("inf"), float("nan")
    for dtype in TYPES:
        low = torch.finfo(TYPES[dtype]).min
        for vocab in (40, 33, 4096, 70001):
            x = torch.zeros((8, vocab), dtype=TYPES[dtype], device="cuda")
            x[0] = -inf                                # nothing left
            x[1] = low                                 # all at the lowest value: uniform
            x[2], x[2, vocab - 1] = -inf, 1.0          # one left
            x[3, 7] = inf
            x[4, 9] = nan
            x[5, 1:] = low                             # masked by the lowest value
            x[6] = 0.0
            x[6, ::2] = -0.0                           # -0 = 0: ties by index
            x[7] = torch.arange(vocab, device="cuda").to(TYPES[dtype]) * 0.01
            ids = torch.tensor([3, 3, vocab - 1, 3, 3, 0, 5, vocab - 1], device="cuda")
            logp, stats, ent = torch.empty(8, device="cuda"), torch.empty((8, 2), device="cuda"), torch.empty(8, device="cuda")
            tl, ti = torch.empty((8, 32), device="cuda"), torch.empty((8, 32), dtype=torch.int64, device="cuda")
            B.cr_token_log_probs(plan, x, ids, logp, stats, ent, tl, ti)
            logn = np.log(vocab)
            lp, e = f64(logp), f64(ent)
            assert lp[0] == -inf and e[0] == 0 and (f64(tl)[0] == -inf).all() and ti[0].tolist() == list(range(32))
            assert abs(lp[1] + logn) < 1e-5 and abs(e[1] - logn) < 1e-4 and ti[1].tolist() == list(range(32))
            assert lp[2] == 0 and e[2] == 0 and ti[2].tolist() == [vocab - 1] + list(range(31))
            assert lp[3] == -inf and np.isnan(e[3]) and ti[3, 0] == 7
            assert np.isnan(lp[4]) and np.isnan(e[4]) and ti[4, 0] == 9 and torch.isnan(tl[4]).all()
            assert lp[5] == 0 and e[5] == 0 and ti[5].tolist() == list(range(32))
            assert abs(lp[6] + logn) < 1e-5 and ti[6].tolist() == list(range(32))
            order = np.argsort(-f64(x)[7], kind="stable")[:32]
            assert ti[7].tolist() == order.tolist()
            one, d = torch.ones(8, device="cuda"), torch.full_like(x, 5.0)
            B.cr_token_log_probs_backward(plan, x, ids, stats, ent, one, one, d)
            g = f64(d)
            assert not g[0].any() and not g[2].any()
            hot = np.zeros(vocab)
            hot[3] = 1
            assert np.allclose(g[1], hot - 1 / vocab, rtol=0.01, atol=1e-4)
            assert np.isfinite(g[5]).all() and np.isnan(g[4]).all()
            B.cr_token_log_probs_backward(plan, x, ids, stats, ent, 0 * one, 0 * one, d)
            assert not d.any()                         # nothing from above: zero whatever the logits hold


@pytest.mark.parametrize("dtype", list(TYPES))
def test_numbers_of_tokens_at_the_lowest_value(plan, dtype):
    """Tokens masked by the type's lowest value, not by -infinity, have a log probability that fp32 can hold."""
    for vocab in (40, 1000, 50257):
        rng = np.random.default_rng(vocab)
        lowest = torch.finfo(TYPES[dtype]).min
        values = rng.standard_normal((6, vocab))
        values[:, 5:] = lowest                        # fewer tokens than alternatives are left
        x = place(values, dtype)
        x[2] = lowest
        x64, ids = f64(x), np.array([0, 7, 7, vocab - 1, 4, 5])
        for temperature in (1.0, 2.0):
            logp, ent = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
            tl, ti = torch.empty((6, 8), device="cuda"), torch.empty((6, 8), dtype=torch.int64, device="cuda")
            B.cr_token_log_probs(plan, x, dev_ids(ids, "i64"), logp, None, ent, tl, ti, temperature=temperature)
            want, _, _, want_e, order, want_top = O.token_log_probs(x64, ids, temperature, 8)
            assert np.isfinite(want).all() and np.isfinite(want_top).all() and np.array_equal(ti.cpu().numpy(), order)
            # the difference, its product with the rounded reciprocal and the last subtraction on terms of their own size, the
            # logarithm of a sum as in log_arith
            near = 4 * STEP * np.log(vocab) + (min(vocab, 1100) + 40) * STEP
            check(logp, want, "f32", 6 * STEP * np.abs(want) + near)
            check(tl, want_top, "f32", 6 * STEP * np.abs(want_top) + near)
            check(ent, want_e, "f32", (6 * 8 + min(vocab, 1100) + 40) * STEP * (1 + 8 + np.log(vocab)))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_distillation_of_tokens_at_the_lowest_value(plan, dtype):
    """The teacher wants a token that the student masks by the type's lowest value: a large loss that fp32 can hold."""
    lowest = torch.finfo(TYPES[dtype]).min
    x = torch.randn(4, 1000, device="cuda").to(TYPES[dtype])
    x[1, 2], x[2, :] = lowest, lowest
    x[3, 8:] = lowest
    ids, t = np.tile(np.arange(8), (4, 1)), np.zeros((4, 8), dtype=np.float32)
    for temperature in (0.5, 1.0, 2.0):
        loss, d = torch.empty(4, device="cuda"), torch.empty_like(x)
        want, want_d = O.distill(f64(x), ids, t, None, temperature)
        # eight shares of 1/8; the factor T^2 (1/8) |log p| of the lowest value is below the largest fp32 number
        assert np.isfinite(want.astype(np.float32)).all()
        B.cr_distill(plan, x, dev_ids(ids, "i64"), dev32(t), loss, d, temperature=temperature)
        check(loss, want, "f32", temperature ** 2 * 1100 * STEP + 16 * STEP * np.abs(want))
        check(d, want_d, dtype, temperature * 1200 * STEP * np.abs(want_d).max())


# ------------------------------------------------------------------------------------------------ distillation

DISTILS = [(1, 1, 0, 0, 1), (3, 8, 0, 0, 3), (39, 5004, 4, 0, 16), (39, 5004, 4, 1, 16), (4, 257, 0, 0, 64), (2, 32000, 0, 0, 64), (3, 50257, 0, 0, 20),
           (1, 128000, 0, 0, 8), (2, 262145, 0, 0, 5), (300, 200, 0, 0, 200), (700, 1024, 8, 0, 1024), (1, 300000, 0, 0, 300), (5, 2048, 0, 0, 33),
           (900, 17000, 0, 0, 128), (460, 33000, 8, 0, 40), (120, 131080, 0, 0, 12), (2, 1100001, 0, 0, 9), (1, 2200000, 0, 0, 40)]      # many rows; more chunks than slots


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", DISTILS)
def test_distillation(plan, shape, dtype):
    rows, vocab, pad, shift, top = shape
    temperature = [1.0, 0.7, 2.0][vocab % 3]
    x, rng = logits_of((rows, vocab, pad, shift), dtype, vocab + 1, 0.0)
    x64 = f64(x)
    ids = rng.integers(0, vocab, (rows, top))      # some named twice
    ids = np.where(rng.random(ids.shape) < 0.1, [-1, vocab][top % 2], ids)
    teacher = 3 * rng.standard_normal((rows, top)).astype(np.float32)
    teacher[rng.random(ids.shape) < 0.05] = -np.inf
    weight = rng.standard_normal(rows).astype(np.float32)
    if rows > 2:
        ids[2], weight[1] = -1, 0
    kind = ["i32", "i64"][rows % 2]
    want, want_d = O.distill(x64, ids, teacher, weight, temperature)
    loss, d = torch.full((rows,), float("nan"), device="cuda"), place(np.zeros((rows, vocab)), dtype, pad, shift)
    args = (dev_ids(ids, kind), dev32(teacher))
    B.cr_distill(plan, x, *args, loss, d, dev32(weight), temperature)
    # both logarithms are off as log p is, the teacher's over its own span
    finite = np.where(np.isfinite(teacher), teacher, 0)
    steps = (6 * np.abs(finite - finite.max(1, keepdims=True)).max(1) / temperature + top + 40) * STEP
    arith = log_arith(x64, temperature) + steps
    # p below is the teacher's share, which multiplies the terms: their sizes are at most the sum of the spans and log_sum
    lp, _, _ = O.log_p(x64, temperature)
    sizes = np.abs(lp).max(1) + np.abs(finite).max(1) * 2 / temperature + np.log(top)
    check(loss, want, "f32", temperature ** 2 * (2 * arith + (top / 256 + 20) * STEP * sizes + 4 * steps * sizes))
    p = np.exp(lp)
    share = np.abs(want_d / np.where(weight == 0, 1, weight * temperature)[:, None] - p) * (weight != 0)[:, None]
    check(d, want_d, dtype, np.abs(weight)[:, None] * temperature * (p * (4 * arith[:, None] + 12 * STEP) + share * (4 * steps[:, None] + (top + 8) * STEP)))
    assert outside_untouched(d)
    alone = torch.full((rows,), float("nan"), device="cuda")
    B.cr_distill(plan, x, *args, alone, temperature=temperature)
    assert torch.equal(alone, loss)
    d2 = torch.full_like(x, 3.0) if x.is_contiguous() else None
    if d2 is not None:
        B.cr_distill(plan, x, *args, None, d2, dev32(weight), temperature)
        assert torch.equal(d2, d)
        y = x.clone()
        B.cr_distill(plan, y, *args, alone, y, dev32(weight), temperature)
        assert torch.equal(y, d) and torch.equal(alone, loss)


def test_distillation_of_odd_rows(plan):
    inf, nan = float("inf"), float("nan")
    x = torch.randn(6, 1000, device="cuda")
    ids = torch.arange(8, device="cuda").repeat(6, 1)
    t = torch.zeros((6, 8), device="cuda")
    t[0] = -inf                       # a teacher that wants nothing
    x[0, 3] = nan
    x[1, 2] = -inf                    # the teacher wants what is masked
    x[2, 900] = -inf                  # masked elsewhere
    x[3, 2], t[3, 2] = -inf, -inf     # masked for both
    w = torch.ones(6, device="cuda")
    w[4], x[4, 7] = 0, nan
    loss, d = torch.empty(6, device="cuda"), torch.empty_like(x)
    B.cr_distill(plan, x, ids, t, loss, d, w)
    lo, g = f64(loss), f64(d)
    assert lo[0] == 0 and not g[0].any()
    assert lo[1] == inf and np.isfinite(g[1]).all() and abs(g[1, 2] + 1 / 8) < 1e-6
    assert np.isfinite(lo[2]) and g[2, 900] == 0 and np.isfinite(lo[3]) and g[3, 2] == 0
    assert np.isnan(lo[4]) and not g[4].any() and abs(g[5].sum()) < 1e-5
    x[5] = -inf                       # a student without a distribution
    B.cr_distill(plan, x, ids, t, loss, d, w)
    assert f64(loss)[5] == inf and np.allclose(f64(d)[5, :8], -1 / 8) and not d[5, 8:].any()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("temperature", [0.7, 1.0, 2.0])
def test_distillation_from_teachers_far_from_zero(plan, temperature, dtype):
    """A constant per row drops out of the teacher's logits: offsets, rows of the type's lowest and of nearly its largest value."""
    rng = np.random.default_rng(21)
    lowest, top, vocab = np.finfo(np.float32).min, 16, 1000
    t = (3 * rng.standard_normal((9, top))).astype(np.float32)
    for r, offset in enumerate((0, 30, 1e3, 1e4, 1e5, -1e5)):
        t[r] += np.float32(offset)
    t[6] = lowest
    t[7, 4:], t[7, :4] = lowest, 3e38
    t[8, 1:], t[8, 0] = lowest, 0.5                   # masked by the lowest value: all that counts is the first
    rows = len(t)
    x, _ = logits_of((rows, vocab, 0, 0), dtype, 5, 0.0)
    x64, weight = f64(x), (1 + 0.1 * rng.standard_normal(rows)).astype(np.float32)
    ids = np.stack([rng.permutation(vocab)[:top] for _ in range(rows)])
    want, want_d = O.distill(x64, ids, t, weight, temperature)
    loss, d = torch.full((rows,), float("nan"), device="cuda"), place(np.zeros((rows, vocab)), dtype)
    B.cr_distill(plan, x, dev_ids(ids, "i64"), dev32(t), loss, d, dev32(weight), temperature)
    # differences to the largest are exact up to half a step of their own, so that the bounds of test_distillation hold with the
    # span of those that have a share, wherever the row lies
    near = t.astype(np.float64) - t.max(1, keepdims=True)
    span = np.abs(np.where(near < -200, 0, near)).max(1) / temperature
    steps = (6 * span + top + 40) * STEP
    arith = log_arith(x64, temperature) + steps
    lp, _, _ = O.log_p(x64, temperature)
    sizes = np.abs(lp).max(1) + span + np.log(top)
    check(loss, want, "f32", temperature ** 2 * (2 * arith + (top / 256 + 20) * STEP * sizes + 4 * steps * sizes))
    p = np.exp(lp)
    share = np.abs(want_d / (weight * temperature)[:, None] - p)
    check(d, want_d, dtype, np.abs(weight)[:, None] * temperature * (p * (4 * arith[:, None] + 12 * STEP) + share * (4 * steps[:, None] + (top + 8) * STEP)))


def test_distillation_by_differences(plan):
    """The gradient is that of the loss."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 50))
    ids, t = rng.integers(0, 50, (3, 6)), rng.standard_normal((3, 6))
    d = torch.empty((3, 50), device="cuda")
    B.cr_distill(plan, dev32(x), dev_ids(ids, "i64"), dev32(t), None, d, temperature=1.5)
    for r, v in ((0, 3), (1, int(ids[1, 0])), (2, int(ids[2, 5]))):
        up, down = x.copy(), x.copy()
        up[r, v] += 1e-4
        down[r, v] -= 1e-4
        slope = (O.distill(up, ids, t, None, 1.5)[0].sum() - O.distill(down, ids, t, None, 1.5)[0].sum()) / 2e-4
        assert abs(slope - f64(d)[r, v]) < 1e-5


# ------------------------------------------------------------------------------------------------ together

def test_norm_codes_feed_the_integer_product(plan):
    """Norm, 8-bit product and scores as an evaluation runs them; each stage against 64 bits of what it was given."""
    rng = np.random.default_rng(11)
    rows, cols, vocab = 39, 256, 1000
    x, r = place(rng.standard_normal((rows, cols)), "bf16"), place(rng.standard_normal((rows, cols)), "bf16")
    gamma = dev32(1 + 0.2 * rng.standard_normal(cols))
    head = dev32(rng.standard_normal((vocab, cols)) / 4)
    w, ws = torch.empty((vocab, cols), dtype=torch.int8, device="cuda"), torch.empty(vocab, device="cuda")
    B.cr_quantize_rows(plan, head, w, ws)
    q, s, h = torch.empty((rows, cols), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    B.cr_rms_norm_codes(plan, x, gamma, q, s, residual=r, h=h)
    logits = torch.empty((rows, vocab), device="cuda")
    B.cr_int8_product(plan, q, s, w, ws, logits)
    want, _ = L.int8_product(q.cpu().numpy(), w.cpu().numpy(), f64(s), f64(ws))
    assert np.max(np.abs(f64(logits) - want)) <= 1e-6 * np.max(np.abs(want))
    ids = dev_ids(rng.integers(0, vocab, rows), "i32")
    logp, ent = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    tl, ti = torch.empty((rows, 5), device="cuda"), torch.empty((rows, 5), dtype=torch.int32, device="cuda")
    B.cr_token_log_probs(plan, logits, ids, logp, None, ent, tl, ti)
    lp, _, _, e, order, _ = O.token_log_probs(f64(logits), ids.cpu().numpy(), 1.0, 5)
    assert np.allclose(f64(logp), lp, atol=1e-5) and np.allclose(f64(ent), e, atol=1e-4) and np.array_equal(ti.cpu().numpy(), order)
    # the whole row against the norm before its codes: a code is half a step of 1/127 of the row's largest value off
    y, _, _ = O.rms_norm(f64(x), f64(r), f64(gamma), 1e-5)
    assert np.max(np.abs(f64(q) * f64(s)[:, None] - y)) <= 0.5001 * np.max(np.abs(y)) / 127


def test_capture_and_other_streams(plan):
    """Every call inside one graph, replayed on changed inputs; workspaces of its own."""
    rng = np.random.default_rng(2)
    parts, tokens, vocab, width = 3, 500, 700, 64
    ids = dev_ids(rng.integers(0, vocab, (parts, tokens)), "i64")
    table, gamma = dev32(rng.standard_normal((vocab, width))), dev32(1 + 0.1 * rng.standard_normal(width))
    y, h, n = (torch.empty((parts, tokens, width), device="cuda") for _ in range(3))
    rstd, dn, dx = torch.empty(parts * tokens, device="cuda"), torch.empty_like(y), torch.empty_like(y)
    logits, dl = torch.empty((parts * tokens, vocab), device="cuda"), torch.empty((parts * tokens, vocab), device="cuda")
    tid, t = dev_ids(rng.integers(0, vocab, (parts * tokens, 4)), "i64"), dev32(rng.standard_normal((parts * tokens, 4)))
    loss, dg, dt = torch.empty(parts * tokens, device="cuda"), torch.empty((parts, width), device="cuda"), torch.empty((parts, vocab, width), device="cuda")
    w1 = scratch(B.cr_embedding_backward_workspace_bytes(plan, ids, dt))
    w2 = scratch(B.cr_rms_norm_backward_workspace_bytes(plan, y, parts))
    lp, st, en = torch.empty(parts * tokens, device="cuda"), torch.empty((parts * tokens, 2), device="cuda"), torch.empty(parts * tokens, device="cuda")
    flat = ids.view(-1)

    def step():
        B.cr_embedding(plan, ids, table, y, scale=2.0)
        B.cr_rms_norm(plan, y, gamma, n, h=h, rstd=rstd)
        torch.mm(n.view(-1, width), table.t(), out=logits)
        B.cr_token_log_probs(plan, logits, flat, lp, st, en)
        B.cr_distill(plan, logits, tid, t, loss, dl)
        torch.mm(dl, table, out=dn.view(-1, width))
        B.cr_rms_norm_backward(plan, dn, h, gamma, rstd, dx, dg, workspace=w2)
        B.cr_embedding_backward(plan, ids, dx, dt, scale=2.0, workspace=w1)

    outs = (y, n, lp, st, en, loss, dl, dx, dg, dt)
    step()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    ids.copy_(dev_ids(rng.integers(0, vocab, (parts, tokens)), "i64"))
    table.add_(0.1)
    step()
    want = [o.clone() for o in outs]
    for o in outs:
        o.fill_(float("nan"))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_a_stream_of_its_own(plan):
    """Every call in another stream's order: its inputs come late there, its outputs and workspaces are its own."""
    rng = np.random.default_rng(4)
    parts, tokens, vocab, width = 3, 900, 700, 64
    rows = parts * tokens
    ids = dev_ids(rng.integers(0, vocab, (parts, tokens)), "i64")
    table, gamma = dev32(rng.standard_normal((vocab, width))), dev32(1 + 0.1 * rng.standard_normal(width))
    tid, t = dev_ids(rng.integers(0, vocab, (rows, 4)), "i64"), dev32(rng.standard_normal((rows, 4)))
    da, db = dev32(rng.standard_normal(rows)), dev32(rng.standard_normal(rows))
    logits, dh = dev32(2 * rng.standard_normal((rows, vocab))), dev32(rng.standard_normal((parts, tokens, width)))
    nan = lambda *shape: torch.full(shape, float("nan"), device="cuda")  # noqa: E731

    def outputs():
        o = dict(y=nan(parts, tokens, width), h=nan(parts, tokens, width), n=nan(parts, tokens, width), rstd=nan(rows), scale=nan(rows),
                 q=torch.full((parts, tokens, width), 7, dtype=torch.int8, device="cuda"), lp=nan(rows), st=nan(rows, 2), en=nan(rows), tl=nan(rows, 6),
                 ti=torch.full((rows, 6), -7, device="cuda"), ds=nan(rows, vocab), loss=nan(rows), dl=nan(rows, vocab), dx=nan(parts, tokens, width),
                 dg=nan(parts, width), dt=nan(parts, vocab, width))
        w1 = scratch(B.cr_embedding_backward_workspace_bytes(plan, ids, o["dt"]))
        w2 = scratch(B.cr_rms_norm_backward_workspace_bytes(plan, o["y"], parts))
        return o, w1, w2

    def step(o, w1, w2):
        B.cr_embedding(plan, ids, table, o["y"], scale=2.0)
        B.cr_rms_norm(plan, o["y"], gamma, o["n"], residual=dh, h=o["h"], rstd=o["rstd"])
        B.cr_rms_norm_codes(plan, o["y"], gamma, o["q"], o["scale"])
        B.cr_token_log_probs(plan, logits, ids.view(-1), o["lp"], o["st"], o["en"], o["tl"], o["ti"])
        B.cr_token_log_probs_backward(plan, logits, ids.view(-1), o["st"], o["en"], da, db, o["ds"])
        B.cr_distill(plan, logits, tid, t, o["loss"], o["dl"])
        B.cr_rms_norm_backward(plan, dh, o["h"], gamma, o["rstd"], o["dx"], o["dg"], workspace=w2)
        B.cr_embedding_backward(plan, ids, o["dx"], o["dt"], scale=2.0, workspace=w1)

    # once without a second stream, on the old inputs
    before = outputs()
    step(*before)
    there = outputs()
    late = [x.clone() for x in (table, logits, dh, t)]
    late = [x.mul_(0.5).add_(0.25) for x in late]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)                 # about ten milliseconds, in which a call in the wrong stream reads the old inputs
        for x, new in zip((table, logits, dh, t), late):
            x.copy_(new)
        step(*there)
    torch.cuda.synchronize()
    here = outputs()
    step(*here)
    for name, want in here[0].items():
        assert torch.equal(there[0][name], want), name
        if name != "ti":                              # the order of the logits is that of half of them and a quarter
            assert not torch.equal(before[0][name], want), name


FIRST_CALLS = """
import sys
import torch
from paper_1902_01981_b200 import binding as B
plan = B.cr_plan_create(4, 2, 1, 24, 1024, device=0)
failed = []

def call(what, f):
    try:
        f()
    except B.CodedReduceError as e:
        failed.append((what, str(e)))

new = lambda *shape, dtype=torch.float32: torch.ones(shape, dtype=dtype, device="cuda")
for dtype in (torch.float32, torch.bfloat16, torch.float16):
    for cols in range(32, 8193, 32):
        x, rstd, dx = new(2, cols, dtype=dtype), new(2), new(2, cols, dtype=dtype)
        ws = new(64, dtype=torch.uint8)
        call(("norm gradient", dtype, cols), lambda: B.cr_rms_norm_backward(plan, x, x, None, rstd, dx, workspace=ws))
    for top in range(64, 1025, 64):
        for vocab in (2048, 65536, 524288):
            x, ids, t, loss = new(1, vocab, dtype=dtype), torch.arange(top, device="cuda").view(1, -1), new(1, top), new(1)
            call(("distillation", dtype, vocab, top), lambda: B.cr_distill(plan, x, ids, t, loss))
    for chunks in range(128, 257, 16):
        x, ids, t = new(75, chunks * 1024, dtype=dtype), new(75, 1, dtype=torch.int64), new(75, 1)
        call(("scores", dtype, chunks), lambda: B.cr_token_log_probs(plan, x, None, top_logp=t, top_ids=ids))
for kind in (torch.int32, torch.int64):
    for tokens in range(64, 2049, 64):
        ids, dy, dt = new(tokens, dtype=kind), new(tokens, 4), new(3, 4)
        ws = new(B.cr_embedding_backward_workspace_bytes(plan, ids, dt), dtype=torch.uint8)
        call(("table gradient", kind, tokens), lambda: B.cr_embedding_backward(plan, ids, dy, dt, workspace=ws))
torch.cuda.synchronize()
print(failed[:4], len(failed))
sys.exit(len(failed) > 0)
"""


def test_first_calls_of_a_process():
    """Sizes in ascending order in a process of its own: no call may live on shared memory that a larger one has asked for."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]


def test_threads_with_plans_of_their_own():
    """Calls of one kind from several host threads, a plan each, whose kernels need different amounts of shared memory, all above
    what a kernel has without asking: no call may take from another what it has asked for."""
    import sys
    import threading
    lib, f32 = B.lib(), B.CR_ELEM_F32
    count, keep = 8, []
    plans = [B.cr_plan_create(4, 2, 1, 24, 1024, device=0) for _ in range(count)]

    def new(shape, value, dtype=torch.float32):
        keep.append(torch.full(shape, value, dtype=dtype, device="cuda"))
        return keep[-1].data_ptr()

    # the C calls with their arguments ready, so that the threads spend their time inside them
    def sorts(p, tokens, stream):
        need = lib.cr_embedding_backward_workspace_bytes(p, tokens, 1, 3, 4)
        args = (new((tokens,), 0, torch.int64), 8, new((tokens, 4), 1.0), 4, new((3, 4), 7.0), 4, 12, tokens, 1, 3, 4, f32, 1.0, -1,
                new((need,), 0, torch.uint8), need, stream)
        return lambda: lib.cr_embedding_backward(p, *args)

    def norms(p, cols, stream):
        x, dx = new((2, cols), 1.0), new((2, cols), 7.0)
        args = (x, cols, x, cols, None, new((2,), 1.0), None, 0, dx, cols, None, cols, 1, 2, cols, f32, new((64,), 0, torch.uint8), 64, stream)
        return lambda: lib.cr_rms_norm_backward(p, *args)

    def distils(p, vocab, stream):
        args = (new((1, vocab), 0.0), vocab, new((1, 1024), 0, torch.int64), 8, new((1, 1024), 0.0), 1024, None, new((1,), 7.0), None, 0, 1, vocab,
                f32, 1.0, stream)
        return lambda: lib.cr_distill(p, *args)

    def scores(p, vocab, stream):
        args = (new((75, vocab), 0.0), vocab, None, 8, 75, vocab, f32, 1.0, None, None, None, 1, new((75, 1), 7.0), new((75, 1), 0, torch.int64), stream)
        return lambda: lib.cr_token_log_probs(p, *args)

    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        for make, sizes, times in ((sorts, (1100, 2048), 6000), (norms, (4864, 8192), 6000), (norms, (2560, 4096), 6000), (distils, (4096, 262144), 6000),
                                   (scores, (245760, 327680), 250)):
            streams = [torch.cuda.Stream() for _ in range(count)]
            calls = [make(plans[i], sizes[i % 2], streams[i].cuda_stream) for i in range(count)]
            torch.cuda.synchronize()
            failed, begin = [0] * count, threading.Barrier(count)

            def work(i):
                begin.wait()
                for _ in range(times):
                    failed[i] += calls[i]() != B.CR_OK

            threads = [threading.Thread(target=work, args=(i,)) for i in range(count)]
            for t in threads:
                t.start()
            for t in threads:
                t.join()
            torch.cuda.synchronize()
            assert not any(failed), (make.__name__, sizes, failed)
            keep.clear()
    finally:
        sys.setswitchinterval(interval)
        torch.cuda.synchronize()
        for p in plans:
            B.cr_plan_destroy(p)


# ------------------------------------------------------------------------------------------------ refusals

def test_refusals(plan):
    """What the library or the binding turns away, before anything is launched."""
    x = torch.randn(4, 64, device="cuda")
    ids, many = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros((4, 40), dtype=torch.int64, device="cuda")
    v, t40 = torch.zeros(4, device="cuda"), torch.zeros((4, 40), device="cuda")
    st = torch.zeros((4, 2), device="cuda")
    dt = torch.zeros((8, 64), device="cuda")
    n = B.cr_plan_launch_count(plan)

    def refused(status, call):
        with pytest.raises(B.CodedReduceError) as e:
            call()
        assert e.value.status == status

    def wrong(call):
        with pytest.raises(ValueError):
            call()

    bad = B.CR_ERR_INVALID_ARG
    refused(bad, lambda: B.cr_embedding(plan, ids, x, x, scale=float("nan")))
    refused(bad, lambda: B.cr_embedding(plan, ids, x, x, scale=1e39))
    wrong(lambda: B.cr_embedding(plan, ids.float(), x, x))
    wrong(lambda: B.cr_embedding(plan, ids, x.half(), x))
    wrong(lambda: B.cr_embedding(plan, ids[:3], x, x))
    wrong(lambda: B.cr_embedding(plan, ids, x, x.t().contiguous().t()))
    wrong(lambda: B.cr_embedding(plan, ids, x, x[:1].expand(4, 64)))
    wrong(lambda: B.cr_embedding(plan, ids.cpu(), x, x))
    wrong(lambda: B.cr_embedding(plan, ids, x.double(), x.double()))
    need = B.cr_embedding_backward_workspace_bytes(plan, ids, dt)
    refused(B.CR_ERR_OOM, lambda: B.cr_embedding_backward(plan, ids, x, dt))
    refused(B.CR_ERR_OOM, lambda: B.cr_embedding_backward(plan, ids, x, dt, workspace=scratch(need)[:need - 1]))
    refused(bad, lambda: B.cr_embedding_backward(plan, ids, x, dt, workspace=scratch(need + 8)[8:]))
    wrong(lambda: B.cr_embedding_backward(plan, ids, x, dt.half(), workspace=scratch(need)))
    wrong(lambda: B.cr_embedding_backward(plan, ids, x, dt[:1].expand(8, 64), workspace=scratch(need)))
    wrong(lambda: B.cr_embedding_backward(plan, ids, x, dt.view(2, 4, 64), workspace=scratch(need)))
    refused(bad, lambda: B.cr_rms_norm(plan, x, None, x, eps=-1.0))
    refused(bad, lambda: B.cr_rms_norm(plan, x, None, x, eps=float("nan")))
    refused(bad, lambda: B.cr_rms_norm(plan, x, None, x, h=x))          # two outputs in one place
    wrong(lambda: B.cr_rms_norm(plan, x, v, x))
    wrong(lambda: B.cr_rms_norm(plan, x, None, x.half()))
    wrong(lambda: B.cr_rms_norm(plan, x, None, x, residual=x[:3]))
    wrong(lambda: B.cr_rms_norm(plan, x[:, :0], None, x[:, :0]))
    wrong(lambda: B.cr_rms_norm_codes(plan, x, None, x, v))
    refused(bad, lambda: B.cr_rms_norm_codes(plan, x, None, torch.zeros((4, 64), dtype=torch.int8, device="cuda"), None))
    need = B.cr_rms_norm_backward_workspace_bytes(plan, x)
    refused(B.CR_ERR_OOM, lambda: B.cr_rms_norm_backward(plan, x, x, None, v, x))
    refused(bad, lambda: B.cr_rms_norm_backward(plan, x, x, None, None, x, workspace=scratch(need)))
    refused(bad, lambda: B.cr_rms_norm_backward(plan, x, x, None, v, x, torch.zeros((3, 64), device="cuda"), workspace=scratch(need)))
    wrong(lambda: B.cr_rms_norm_backward(plan, x, x, None, v, x, v, workspace=scratch(need)))
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-20):
        refused(bad, lambda: B.cr_token_log_probs(plan, x, ids, v, temperature=t))
        refused(bad, lambda: B.cr_token_log_probs_backward(plan, x, ids, st, v, v, v, x, temperature=t))
        refused(bad, lambda: B.cr_distill(plan, x, many, t40, v, temperature=t))
    refused(bad, lambda: B.cr_token_log_probs(plan, x, ids, v, top_logp=t40, top_ids=many))               # more than 32
    refused(bad, lambda: B.cr_token_log_probs(plan, x[:, :4], ids, v, top_logp=t40[:, :5].contiguous(), top_ids=many[:, :5].contiguous()))
    refused(bad, lambda: B.cr_token_log_probs(plan, x, ids, v, stats=torch.zeros(9, device="cuda")[1:].view(4, 2)))
    wrong(lambda: B.cr_token_log_probs(plan, x, None, v))
    wrong(lambda: B.cr_token_log_probs(plan, x, ids, v[:3]))
    wrong(lambda: B.cr_token_log_probs(plan, x, ids, v, top_logp=t40[:, :4].contiguous()))
    wrong(lambda: B.cr_token_log_probs(plan, x, ids, v, top_logp=t40[:, :4].contiguous(), top_ids=many[:, :4].int().contiguous()))
    wrong(lambda: B.cr_token_log_probs(plan, x[0], ids, v))
    wrong(lambda: B.cr_token_log_probs_backward(plan, x, ids, st, None, None, v, x))
    wrong(lambda: B.cr_token_log_probs_backward(plan, x, None, st, v, v, v, x))
    wrong(lambda: B.cr_token_log_probs_backward(plan, x, ids, None, v, v, v, x))
    wrong(lambda: B.cr_distill(plan, x, many, v, v))
    wrong(lambda: B.cr_distill(plan, x, many, t40, v, x.half()))
    wrong(lambda: B.cr_distill(plan, x, many.t().contiguous().t(), t40, v))
    refused(bad, lambda: B.cr_distill(plan, x, many[:, :0].contiguous(), t40[:, :0].contiguous(), v))
    big, bigt = torch.zeros((4, 1025), dtype=torch.int64, device="cuda"), torch.zeros((4, 1025), device="cuda")
    refused(bad, lambda: B.cr_distill(plan, x, big, bigt, v))
    store = torch.zeros(4 * 64 * 4 + 4, dtype=torch.uint8, device="cuda")
    off = store[2:2 + 4 * 64 * 2].view(torch.bfloat16)         # on its elements
    B.cr_rms_norm(plan, off.view(4, 64), None, off.view(4, 64))
    assert B.cr_plan_launch_count(plan) == n + 1
    host = B.cr_plan_create(4, 2, 1, 24, 1024)
    refused(B.CR_ERR_CUDA, lambda: B.cr_rms_norm(host, x, None, x))
    B.cr_plan_destroy(host)


def test_tables_beyond_the_grid_are_refused(plan):
    """More rows of tables than blocks that could zero them (more than the device holds): an argument that is refused, not a launch
    that fails."""
    n = B.cr_plan_launch_count(plan)
    for parts, vocab in ((1 << 24, 4096), (800, 2 ** 31 - 1)):
        assert B.lib().cr_embedding_backward(plan, None, 8, None, 1, 16, 1, vocab, 0, parts, vocab, 1, B.CR_ELEM_F32, 1.0, -1, None, 0, None) == B.CR_ERR_INVALID_ARG
    assert B.cr_plan_launch_count(plan) == n


# ------------------------------------------------------------------------------------------------ long strides

def test_offsets_beyond_32_bits(plan):
    """Rows whose last element lies beyond 2^31 elements."""
    ld = (1 << 30) + 8
    store = torch.empty(2 * ld + 4096, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(store, (3, 4096), (ld, 1))
    x.copy_(torch.randn(3, 4096, device="cuda"))
    near = x.contiguous()
    y, y2, rstd = torch.empty_like(near), torch.empty_like(near), torch.empty(3, device="cuda")
    B.cr_rms_norm(plan, x, None, y, rstd=rstd)
    B.cr_rms_norm(plan, near, None, y2)
    assert torch.equal(y, y2)
    ids = torch.tensor([2, 0, 1, 2], device="cuda")
    z = torch.empty((4, 4096), dtype=torch.bfloat16, device="cuda")
    B.cr_embedding(plan, ids, x, z)
    assert torch.equal(z, near[ids])
    lp, lp2 = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    B.cr_token_log_probs(plan, x, ids[:3], lp)
    B.cr_token_log_probs(plan, near, ids[:3], lp2)
    assert torch.equal(lp, lp2)
    tid, t = torch.tensor([[1, 4095]] * 3, device="cuda"), torch.zeros((3, 2), device="cuda")
    d = torch.empty_like(near)
    B.cr_distill(plan, near, tid, t, lp2, d)
    B.cr_distill(plan, x, tid, t, lp, x)
    assert torch.equal(lp, lp2) and torch.equal(x, d)
    x.copy_(near)
    ws = scratch(B.cr_rms_norm_backward_workspace_bytes(plan, x))
    dx, dg, dg2 = torch.empty_like(near), torch.empty((1, 4096), device="cuda"), torch.empty((1, 4096), device="cuda")
    B.cr_rms_norm_backward(plan, y, near, None, rstd, dx, dg, workspace=ws)
    B.cr_rms_norm_backward(plan, y, x, None, rstd, x, dg2, workspace=ws)
    assert torch.equal(x, dx) and torch.equal(dg, dg2)
    dt, dt2 = torch.empty((5, 4096), device="cuda"), torch.empty((5, 4096), device="cuda")
    ws = scratch(B.cr_embedding_backward_workspace_bytes(plan, ids[:3], dt))
    B.cr_embedding_backward(plan, ids[:3], x, dt, workspace=ws)
    B.cr_embedding_backward(plan, ids[:3], dx, dt2, workspace=ws)
    assert torch.equal(dt, dt2)


# ------------------------------------------------------------------------------------------------ the largest sizes

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("tokens", [70, 3000])
def test_gradient_of_the_longest_table(plan, tokens):
    """Numbers of 31 bits: four digits, in one CTA's sort and in the cluster's."""
    rng = np.random.default_rng(tokens)
    ids = rng.integers(0, MOST, tokens)
    ids[::7], ids[1::7], ids[2::11], ids[3::13] = MOST - 1, 0, MOST, -1
    ids[4::17] = 1 << 24
    dy = torch.randn(tokens, 1, device="cuda")
    table = torch.full((MOST, 1), float("nan"), device="cuda")
    need = B.cr_embedding_backward_workspace_bytes(plan, dev_ids(ids, "i64"), table)
    B.cr_embedding_backward(plan, dev_ids(ids, "i64"), dy, table, workspace=scratch(need)[:need])
    named = (ids >= 0) & (ids < MOST)
    where, back = np.unique(ids[named], return_inverse=True)
    want, size = np.zeros(len(where)), np.zeros(len(where))
    np.add.at(want, back, f64(dy)[named, 0])
    np.add.at(size, back, np.abs(f64(dy)[named, 0]))
    check(table[torch.from_numpy(where).cuda(), 0], want, "f32", (95 + tokens / 32 + 4) * STEP * size)
    assert int(torch.count_nonzero(table)) == np.count_nonzero(want)
    if tokens == 70:
        y = torch.empty((tokens, 1), device="cuda")
        B.cr_embedding(plan, dev_ids(ids, "i64"), table, y)
        check(y[:, 0], np.where(named, f64(table[torch.from_numpy(np.where(named, ids, 0)).cuda(), 0]), 0), "f32", 0)


def test_many_partitions(plan):
    parts = 70000
    ids = torch.arange(parts, device="cuda").view(parts, 1) % 5 - 1
    dy = torch.randn(parts, 1, 4, device="cuda")
    d = torch.full((parts, 3, 4), float("nan"), device="cuda")
    need = B.cr_embedding_backward_workspace_bytes(plan, ids, d)
    B.cr_embedding_backward(plan, ids, dy, d, workspace=scratch(need)[:need])
    want = torch.zeros_like(d)
    named = ((ids >= 0) & (ids < 3))[:, 0]
    want[named, ids[named, 0]] = dy[named, 0]
    assert torch.equal(d, want)
    x, g, rstd = torch.randn(parts, 16, device="cuda"), torch.randn(parts, 16, device="cuda"), torch.rand(parts, device="cuda")
    dx, dg = torch.empty_like(x), torch.full((parts, 16), float("nan"), device="cuda")
    ws = scratch(B.cr_rms_norm_backward_workspace_bytes(plan, x, parts))
    B.cr_rms_norm_backward(plan, g, x, None, rstd, dx, dg, workspace=ws)
    want_dx, want_dg, size = O.rms_norm_backward(f64(g), f64(x), None, f64(rstd), None, parts)
    check(dg, want_dg, "f32", 3 * STEP * size)


@pytest.mark.parametrize("vocab", [MOST, MOST - 7])
def test_the_longest_rows_of_logits(plan, vocab):
    """One row of 2^31 logits, off and on the 16-byte boundaries: a few that stand out, all others alike."""
    x = torch.full((1, vocab), -1.0, dtype=torch.bfloat16, device="cuda")
    where = [5, vocab - 1, vocab - 2000, 1 << 30, vocab // 3]
    x[0, where] = torch.tensor([20.0, 19.0, 18.0, 17.0, 16.0], dtype=torch.bfloat16, device="cuda")
    x64 = np.array([20.0, 19.0, 18.0, 17.0, 16.0])
    total = np.exp(x64 - 20).sum() + (vocab - 5) * np.exp(-21.0)
    log_sum = np.log(total)
    # a chain of one addition for each of a lane's 64 elements, 2048 chunks of a slot with two roundings each, the levels of joining
    arith = (64 + 2 * 2048 + 60 + 6 * 21) * STEP
    ids = torch.tensor([vocab - 1], device="cuda")
    logp, stats, ent = torch.empty(1, device="cuda"), torch.empty((1, 2), device="cuda"), torch.empty(1, device="cuda")
    tl, ti = torch.empty((1, 8), device="cuda"), torch.empty((1, 8), dtype=torch.int64, device="cuda")
    B.cr_token_log_probs(plan, x, ids, logp, stats, ent, tl, ti)
    assert ti[0].tolist() == where + [0, 1, 2]
    check(tl[0], np.concatenate([x64, [-1, -1, -1]]) - 20 - log_sum, "f32", arith)
    check(logp, [-1 - log_sum], "f32", arith)
    p = np.exp(x64 - 20) / total
    rest = (vocab - 5) * np.exp(-21.0) / total
    check(ent, [-(p * np.log(p)).sum() + rest * (21 + log_sum)], "f32", arith * 23)
    t = torch.tensor([[1.0, 2.0, 0.5]], device="cuda")
    tid = torch.tensor([[vocab - 1, 7, 5]], device="cuda")
    loss, d = torch.empty(1, device="cuda"), torch.empty_like(x)
    B.cr_distill(plan, x, tid, t, loss, d)
    share = np.exp([1.0, 2.0, 0.5]) / np.exp([1.0, 2.0, 0.5]).sum()
    lp = np.array([-1.0, -21.0, 0.0]) - log_sum
    check(loss, [(share * (np.log(share) - lp)).sum()], "f32", 2 * arith)
    at = lambda g: f64(g[0, [vocab - 1, 7, 5, vocab - 2000, 6, vocab - 2]])  # noqa: E731
    q = np.exp(np.array([19.0, -1, 20, 18, -1, -1]) - 20) / total
    got = at(d)
    assert np.all(np.abs(got - (q - np.concatenate([share, [0, 0, 0]]))) <= 2.0 ** -8 * 1.01 * np.abs(got) + arith * np.maximum(q, 1e-9) + 8 * STEP)
    assert abs(float(d[0, 8:1 << 20].double().sum()) / ((1 << 20) - 8) / q[4] - 1) <= 2.0 ** -8 + arith
    one = torch.ones(1, device="cuda")
    B.cr_token_log_probs_backward(plan, x, ids, stats, ent, one, None, x)
    hot = np.array([1.0, 0, 0, 0, 0, 0])
    got = at(x)
    assert np.all(np.abs(got - (hot - q)) <= 2.0 ** -8 * 1.01 * np.abs(got) + arith * np.maximum(q, 1e-9) + 8 * STEP)


@pytest.mark.parametrize("cols", [MOST, MOST - 7])
def test_norm_of_the_longest_rows(plan, cols):
    x = torch.full((1, cols), 0.5, dtype=torch.bfloat16, device="cuda")
    x[0, [3, cols - 1]] = torch.tensor([1000.0, -2000.0], dtype=torch.bfloat16, device="cuda")
    mean = ((cols - 2) * 0.25 + 1e6 + 4e6) / cols
    rstd = torch.empty(1, device="cuda")
    B.cr_rms_norm(plan, x, None, x, rstd=rstd, eps=0.0)
    # 16 warps go over 2^22 pieces of 512 (2^20 of 1024) elements: a chain of a quarter of a million additions, then of each piece's own
    pieces = -(-cols // 512) / 16
    check(rstd, [mean ** -0.5], "f32", (pieces + 600) / 2 * STEP * mean ** -0.5)
    got = f64(x[0, [3, cols - 1, 0, cols - 2, cols // 2]])
    want = np.array([1000.0, -2000.0, 0.5, 0.5, 0.5]) * mean ** -0.5
    assert np.all(np.abs(got - want) <= (2.0 ** -8 * 1.01 + (pieces + 600) / 2 * STEP) * np.abs(want))
