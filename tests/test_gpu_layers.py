"""Group norm with activation and dropout, dropout, 8-bit codes and products against 64-bit arithmetic."""
import numpy as np
import pytest

from oracle import cr_layers as O
from paper_1902_01981_b200 import binding as B
from paper_1902_01981_b200 import build as cr_build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# Rounding of a stored value: half a unit of the last place of bf16 (8 bits) and f16 (11 bits; also its smallest step),
# a whole one of f32 (24 bits).
ROUND = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -24}
# fp32 arithmetic before that: a value is a dozen operations of 2^-24 each on numbers of the size of the largest
# output, and the statistics are sums of chains of at most a few hundred additions whose errors mostly cancel
ARITH = 2e-5


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
    """`values` on the device as rows that are `pad` elements longer, `shift` elements behind an aligned address."""
    shape = values.shape
    store = torch.full((int(np.prod(shape[:-1])) * (shape[-1] + pad) + shift + 8,), float("nan"), dtype=TYPES[dtype], device="cuda")
    strides, step = [1], shape[-1] + pad
    for n in reversed(shape[1:-1]):
        strides.insert(0, step)
        step *= n
    strides.insert(0, step)
    view = torch.as_strided(store, shape, strides if len(shape) > 1 else [1], shift)
    view.copy_(torch.from_numpy(np.asarray(values, dtype=np.float32)))
    return view


def check(got, want, dtype, extra=0.0):
    got, want = f64(got), np.asarray(want)
    size = np.max(np.abs(want)) if want.size else 0.0
    tol = ROUND[dtype] * np.abs(want) + TINY[dtype] + ARITH * size + extra
    bad = np.abs(got - want) > tol
    assert not bad.any(), f"{bad.sum()} of {bad.size}, worst {np.max(np.abs(got - want)):.3e} at size {size:.3e}"


# ------------------------------------------------------------------------------------------------ group norm

# samples, positions, channels, groups, pad, shift
SHAPES = [
    (1, 1, 1, 1, 0, 0),            # a group of one value
    (2, 1, 16, 16, 0, 0),          # the same in vectors
    (3, 1, 24, 3, 0, 0),           # one position
    (3, 5, 7, 7, 0, 0),            # a group per channel, odd
    (3, 5, 12, 3, 4, 1),           # rows inside wider rows, misaligned
    (1, 64, 128, 32, 0, 0),        # four channels a group
    (5, 221, 60, 5, 4, 0),         # twelve channels a group
    (4, 33, 96, 8, 8, 0),
    (2, 17, 4096, 4, 0, 0),        # more channels than a block has vectors
    (1, 5000, 16, 2, 0, 0),        # many positions
    (2, 1024, 64, 8, 0, 8),
    (1, 20000, 40, 1, 0, 0),       # one group over everything
    (70, 9, 32, 8, 0, 0),
    (1, 70001, 32, 4, 0, 0),       # a sample of several megabytes
    (3, 130, 88, 11, 0, 0),        # the last slab is narrower than the others
    (2, 200, 80, 5, 0, 0),         # sixteen channels a group, a slab of 48 and one of 32 (or 16s)
    (2000, 4, 32, 8, 0, 0),        # more samples than CTAs: each walks over several
    (300, 260, 64, 8, 0, 0),       # the same in clusters
    (2, 50, 5000, 1, 0, 0),        # a group wider than a tile
    (2, 50, 2310, 2, 0, 0),
]


def norm_data(shape, seed, offset_mean=0.5):
    n, s, c = shape
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, s, c)) * np.exp(0.3 * rng.standard_normal(c)) + offset_mean * rng.standard_normal(c)
    return x, 1 + 0.2 * rng.standard_normal(c), 0.3 * rng.standard_normal(c), rng.standard_normal((n, s, c))


def dev32(v):
    return None if v is None else torch.from_numpy(np.asarray(v, dtype=np.float32)).cuda()


def scratch(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def forward(plan, x, gamma, beta, groups, dtype, pad=0, shift=0, **kw):
    y = place(np.zeros(x.shape), dtype, pad, shift)
    mean = torch.full((x.shape[0], groups), float("nan"), device="cuda")
    rstd = torch.full((x.shape[0], groups), float("nan"), device="cuda")
    ws = scratch(B.cr_group_norm_workspace_bytes(plan, x, groups))
    B.cr_group_norm(plan, x, gamma, beta, groups, y, mean, rstd, workspace=ws, **kw)
    return y, mean, rstd


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES)
def test_group_norm_forward_and_backward(plan, shape, dtype):
    n, s, c, groups, pad, shift = shape
    act = ["none", "relu", "silu"][(n + s + groups) % 3]
    p = [0.0, 0.3][(s + groups) % 2]
    seed, offset = 1234567890123 + c, [0, 3, (1 << 33) + 2][(n + c) % 3]
    xv, gv, bv, dyv = norm_data((n, s, c), seed % 1000)
    x, dy = place(xv, dtype, pad, shift), place(dyv, dtype, pad, shift)
    gamma, beta = dev32(gv), dev32(bv)
    if n == 3:
        gamma = beta = None
    g64, b64 = (None, None) if gamma is None else (f64(gamma), f64(beta))
    factors = O.dropout_factors((n, s, c), p, seed, offset) if p else None
    kw = dict(act=B.CR_ACT[act], p=p, seed=seed, offset=offset)
    y, mean, rstd = forward(plan, x, gamma, beta, groups, dtype, pad, shift, eps=1e-5, **kw)
    want, mean64, rstd64, z = O.group_norm(f64(x), g64, b64, groups, 1e-5, act, factors)
    check(mean, mean64, "f32", extra=1e-6 * np.max(np.abs(xv)))
    # rstd: a group of one value has rstd = eps^-1/2 exactly; elsewhere the relative error of the variance halves
    check(rstd, rstd64, "f32")
    # z of a nearly constant group is rstd times a difference of nearly equal numbers, whose rounding rstd magnifies
    spread = np.max(rstd64) * np.max(np.abs(xv)) * 2.0 ** -23
    check(y, want, dtype, extra=4 * spread)
    # backward, a partition per sample, rows of parameter gradients inside wider rows
    parts = n
    wide = torch.full((parts, 2 * c + 3), float("nan"), device="cuda")
    dgamma, dbeta = wide[:, 1:c + 1], wide[:, c + 2:2 * c + 2]
    dx = place(np.zeros(xv.shape), dtype, pad, shift)
    ws = scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, groups))
    B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, groups, dx, dgamma, dbeta, workspace=ws, **kw)
    dx64, dg64, db64, z, ag, ab = O.group_norm_backward(f64(dy), f64(x), g64, b64, groups, 1e-5, act, factors, parts)
    # where z is within its own error of the kink of relu, either slope is right
    edge = (np.abs(z) < 4 * spread + 1e-5) if act == "relu" else np.zeros(z.shape, bool)
    top = np.max(np.abs(f64(dy))) * (1.0 if factors is None else np.max(factors))
    near = edge.reshape(parts, -1, c).sum(1) * top
    assert np.all(np.abs(f64(dbeta) - db64) <= 1e-5 * ab + near + 1e-30)
    assert np.all(np.abs(f64(dgamma) - dg64) <= 1e-5 * ag + near * np.max(np.abs(z) + 1) + 4 * spread * ab + 1e-30)
    assert torch.isnan(wide[:, 0]).all() and torch.isnan(wide[:, c + 1]).all() and torch.isnan(wide[:, 2 * c + 2]).all()
    assert edge.mean() < 0.01 or z.size < 100
    gsize = 1.0 if g64 is None else np.max(np.abs(g64))
    extra = np.max(rstd64) * gsize * top * (np.max(near) / top / max(1, s) * 4 + 8 * spread + 1e-6)
    check(torch.where(torch.from_numpy(edge).cuda(), torch.zeros_like(dx), dx), np.where(edge, 0, dx64), dtype, extra=extra)


def test_a_group_of_one_value_has_no_gradient(plan):
    xv, gv, bv, dyv = norm_data((4, 1, 8), 3)
    x, dy = place(xv, "f32"), place(dyv, "f32")
    gamma, beta = dev32(gv), dev32(bv)
    y, mean, rstd = forward(plan, x, gamma, beta, 8, "f32")
    assert torch.equal(y, beta.expand(4, 1, 8))
    dx = torch.full_like(x, float("nan"))
    B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, 8, dx,
                             workspace=scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, 8)))
    assert torch.equal(dx, torch.zeros_like(dx))


@pytest.mark.parametrize("shape", [(2, 50, 32, 4), (1, 3000, 64, 8), (2, 7, 30, 5)])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_group_norm_gradient_against_differences(plan, shape, act):
    """<dL/dx, v> against (L(x + h v) - L(x - h v)) / 2h for L = <y, u>, and the same for gamma and beta, with the
    kernel's own forward pass in fp32.  With h = 2^-6 the third-order term is about h^2 / 6 = 4e-5 of the value; the
    rounding of y (2^-24 of values of a few units, over count^1/2 random terms, divided by h) adds 1e-5 count^1/2."""
    n, s, c, groups = shape
    xv, gv, bv, uv = norm_data((n, s, c), 77)
    rng = np.random.default_rng(78)
    p, seed, offset = 0.25, 99, 5
    kw = dict(act=B.CR_ACT[act], p=p, seed=seed, offset=offset)
    gamma, beta = dev32(gv), dev32(bv)
    x, u = place(xv, "f32"), place(uv, "f32")
    _, mean, rstd = forward(plan, x, gamma, beta, groups, "f32", **kw)
    dx, dg, db = torch.empty_like(x), torch.empty((1, c), device="cuda"), torch.empty((1, c), device="cuda")
    B.cr_group_norm_backward(plan, u, x, gamma, beta, mean, rstd, groups, dx, dg, db,
                             workspace=scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, groups)), **kw)
    h = 2.0 ** -6

    def loss(x, gamma, beta):
        return float(np.sum(f64(forward(plan, x, gamma, beta, groups, "f32", **kw)[0]) * f64(u)))

    for which, grad in (("x", dx), ("gamma", dg[0]), ("beta", db[0])):
        v = torch.from_numpy(rng.standard_normal(tuple(grad.shape)).astype(np.float32)).cuda()
        args = {"x": x, "gamma": gamma, "beta": beta}
        ends = [loss(**{**args, which: args[which] + sign * h * v}) for sign in (1, -1)]
        slope = (ends[0] - ends[1]) / (2 * h)
        want = float(np.sum(f64(grad) * f64(v)))
        size = float(np.linalg.norm(f64(grad))) * float(np.linalg.norm(f64(v))) / np.sqrt(v.numel())
        assert abs(slope - want) <= 1e-3 * (abs(want) + size) + 1e-5 * np.sqrt(x.numel())


@pytest.mark.parametrize("shape,dtype", [((12, 40, 64, 8), "bf16"), ((12, 40, 64, 8), "f32"), ((8, 700, 30, 5), "f32"),
                                         ((8, 700, 30, 5), "f16"), ((4, 9000, 48, 1), "bf16"), ((200, 1030, 64, 8), "f16")])
def test_partitions_add_up_and_do_not_see_each_other(plan, shape, dtype):
    """Per-partition gradients are what a worker that holds the partition alone computes, bit for bit: the same
    samples, the index of its first element as offset.  Items of one CTA, of clusters, and of the streaming form."""
    n, s, c, groups = shape
    parts = 4
    xv, gv, bv, dyv = norm_data((n, s, c), 5)
    x, dy = place(xv, dtype), place(dyv, dtype)
    gamma, beta = dev32(gv), dev32(bv)
    kw = dict(act=B.CR_ACT_SILU, p=0.2, seed=11)
    y, mean, rstd = forward(plan, x, gamma, beta, groups, dtype, offset=7, **kw)
    dx, dg, db = torch.empty_like(x), torch.empty((parts, c), device="cuda"), torch.empty((parts, c), device="cuda")
    ws = scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, groups))
    B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, groups, dx, dg, db, workspace=ws, offset=7, **kw)
    per = n // parts
    for q in range(parts):
        mine = slice(q * per, (q + 1) * per)
        offset = 7 + q * per * s * c
        y1, mean1, rstd1 = forward(plan, x[mine], gamma, beta, groups, dtype, offset=offset, **kw)
        assert torch.equal(y1, y[mine]) and torch.equal(mean1, mean[mine]) and torch.equal(rstd1, rstd[mine])
        dx1, dg1, db1 = torch.empty_like(x[mine]), torch.empty((1, c), device="cuda"), torch.empty((1, c), device="cuda")
        B.cr_group_norm_backward(plan, dy[mine], x[mine], gamma, beta, mean1, rstd1, groups, dx1, dg1, db1, workspace=ws,
                                 offset=offset, **kw)
        assert torch.equal(dx1, dx[mine]) and torch.equal(dg1[0], dg[q]) and torch.equal(db1[0], db[q])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", [(6, 40, 64, 8), (3, 700, 64, 8), (2, 9000, 48, 4), (2, 50, 4096, 1), (4, 60, 24, 8)])
def test_bits_depend_on_the_layout_only_by_its_alignment(plan, shape, dtype):
    """Packed rows and rows inside wider ones, both in 16-byte vectors: the same bits.  So for two layouts that are off them.
    From one to the other the sums are taken in another order."""
    n, s, c, groups = shape
    xv, gv, bv, dyv = norm_data((n, s, c), 61)
    gamma, beta = dev32(gv), dev32(bv)
    kw = dict(act=B.CR_ACT_SILU, p=0.2, seed=5, offset=3)

    def step(*layouts):                              # (pad, shift) of x, y, dy, dx
        (x, dy), (y, dx) = ((place(a, dtype, *layouts[k]), place(b, dtype, *layouts[k + 2])) for k, a, b in ((0, xv, dyv), (1, 0 * xv, 0 * xv)))
        mean, rstd = torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda")
        dg, db = torch.empty((n, c), device="cuda"), torch.empty((n, c), device="cuda")
        B.cr_group_norm(plan, x, gamma, beta, groups, y, mean, rstd, workspace=scratch(B.cr_group_norm_workspace_bytes(plan, x, groups, y)), **kw)
        B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, groups, dx, dg, db,
                                 workspace=scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, groups, dy, dx)), **kw)
        return [t.contiguous() for t in (y, mean, rstd, dx, dg, db)]

    packed, wider, moved = (0, 0), (16, 0), (0, 16)
    on = step(packed, packed, packed, packed)
    for layouts in ((wider,) * 4, (packed, wider, moved, packed), (moved, packed, wider, wider)):
        assert all(torch.equal(a, b) for a, b in zip(on, step(*layouts)))
    odd, off = (1, 0), (0, 1)
    others = step(odd, odd, odd, odd)
    for layouts in ((off,) * 4, (packed, off, packed, odd), (off, packed, wider, off)):
        assert all(torch.equal(a, b) for a, b in zip(others, step(*layouts)))


def test_a_nan_stays_in_its_group_and_statistics_survive_a_large_mean(plan):
    n, s, c, groups = 3, 100, 32, 4
    xv, gv, bv, _ = norm_data((n, s, c), 6)
    x = place(xv, "f32")
    x[1, 7, 9] = float("nan")
    y, mean, rstd = forward(plan, x, dev32(gv), dev32(bv), groups, "f32")
    dead = torch.zeros((n, s, c), dtype=torch.bool, device="cuda")
    dead[1, :, 8:16] = True
    assert torch.isnan(y[dead]).all() and torch.isfinite(y[~dead]).all()
    # mean 4096, spread 1: x holds the spread to 2^-12 / 2, sums of squares of x itself would lose it
    rng = np.random.default_rng(8)
    x = place(4096 + rng.standard_normal((2, 3000, 32)), "f32")
    y, mean, rstd = forward(plan, x, None, None, 4, "f32")
    want, mean64, rstd64, _ = O.group_norm(f64(x), None, None, 4, 1e-5)
    # the mean is known to half a unit of 4096 (2^-12); that is the error of x - mean, one part in 4096
    assert np.max(np.abs(f64(mean) - mean64)) <= 2.0 ** -11
    assert np.max(np.abs(f64(rstd) / rstd64 - 1)) <= 1e-5
    assert np.max(np.abs(f64(y) - want)) <= 2.0 ** -10


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", [(3, 300, 32, 4), (2, 40, 30, 3), (1, 1100, 64, 8)])
def test_statistics_whatever_comes_first(plan, shape, dtype):
    """The first values of every group are a hundred standard deviations off, and so is the mean of one sample: one-pass
    sums around either would lose four of seven digits of the variance."""
    n, s, c, groups = shape
    xv, gv, bv, dyv = norm_data((n, s, c), 21)
    xv[:, 0, :] += 100.0
    xv[0] += 50.0
    x, gamma, beta = place(xv, dtype), dev32(gv), dev32(bv)
    y, mean, rstd = forward(plan, x, gamma, beta, groups, dtype, act=B.CR_ACT_SILU)
    want, mean64, rstd64, _ = O.group_norm(f64(x), f64(gamma), f64(beta), groups, 1e-5, "silu")
    # sums of values up to 150, each rounded to 2^-24 of the running sum
    assert np.max(np.abs(f64(mean) - mean64)) <= 150 * 2e-6
    assert np.max(np.abs(f64(rstd) / rstd64 - 1)) <= 2e-5
    check(y, want, dtype, extra=np.max(rstd64) * 150 * 2e-6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_values_with_a_small_spread(plan, dtype):
    """1e18 with a spread of 2 %: the squares of 8192 values leave the range of a float, those around the mean do not.
    The second sample starts with a row of zeros, so that no value of its first row is near the mean."""
    n, s, c, groups = 2, 256, 64, 2
    xv = 1e18 * (1 + 0.02 * np.random.default_rng(31).standard_normal((n, s, c)))
    xv[1, 0] = 0.0
    x = place(xv, dtype)
    y, mean, rstd = forward(plan, x, None, None, groups, dtype)
    want, mean64, rstd64, _ = O.group_norm(f64(x), None, None, groups, 1e-5)
    # as below: sums of values up to 1.1e18, each rounded to 2^-24 of the running sum
    assert np.max(np.abs(f64(mean) - mean64)) <= 1.1e18 * 2e-6
    assert np.max(np.abs(f64(rstd) / rstd64 - 1)) <= 2e-5
    check(y, want, dtype, extra=np.max(rstd64) * 1.1e18 * 2e-6)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape,shift", [((3, 100, 32, 4), 0), ((3, 100, 32, 4), 1), ((3, 700, 64, 4), 0), ((2, 9000, 32, 4), 0),
                                         ((3, 40, 24, 8), 0)])
def test_nan_and_infinities_reach_the_statistics(plan, shape, shift, dtype):
    """A group that holds one has no finite mean, rstd, output or gradient; the others are as without it."""
    n, s, c, groups = shape
    xv, gv, bv, dyv = norm_data((n, s, c), 6)
    inf = float("inf")
    dead = np.zeros((n, groups), bool)
    for i, j, k, v in ((0, 0, 0, float("nan")), (0, s - 1, c - 1, inf), (1, s // 2, c // groups, -inf), (1, 0, c - 1, inf), (1, 1, c - 1, -inf)):
        xv[i, j, k] = v
        dead[i, k * groups // c] = True
    x, dy, gamma, beta = place(xv, dtype, 0, shift), place(dyv, dtype, 0, shift), dev32(gv), dev32(bv)
    y, mean, rstd = forward(plan, x, gamma, beta, groups, dtype, shift=shift, act=B.CR_ACT_SILU)
    assert np.array_equal(np.isnan(f64(rstd)), dead) and np.array_equal(~np.isfinite(f64(mean)), dead)
    gone = np.repeat(dead, c // groups, axis=1)
    every = np.broadcast_to(gone[:, None, :], (n, s, c))
    assert np.isnan(f64(y)[every]).all()
    finite = np.where(np.isfinite(f64(x)), f64(x), 0.0)
    want, mean64, rstd64, _ = O.group_norm(finite, f64(gamma), f64(beta), groups, 1e-5, "silu")
    check(torch.from_numpy(np.where(every, 0, f64(y))), np.where(every, 0, want), dtype)
    check(torch.from_numpy(np.where(dead, 0, f64(rstd))), np.where(dead, 0, rstd64), "f32")
    dx, dg, db = place(np.zeros(xv.shape), dtype, 0, shift), torch.empty((n, c), device="cuda"), torch.empty((n, c), device="cuda")
    B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, groups, dx, dg, db, act=B.CR_ACT_SILU,
                             workspace=scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, groups)))
    assert np.isnan(f64(dx)[every]).all() and np.isnan(f64(dg)[gone]).all() and np.isnan(f64(db)[gone]).all()
    dx64, dg64, db64, _, ag, ab = O.group_norm_backward(f64(dy), finite, f64(gamma), f64(beta), groups, 1e-5, "silu", None, n)
    check(torch.from_numpy(np.where(every, 0, f64(dx))), np.where(every, 0, dx64), dtype)
    assert np.all(np.abs(f64(dg) - dg64)[~gone] <= 1e-5 * ag[~gone]) and np.all(np.abs(f64(db) - db64)[~gone] <= 1e-5 * ab[~gone])


@pytest.mark.parametrize("far", [100.0, 300.0, 1000.0])
@pytest.mark.parametrize("shape", [(1, 16384, 1, 1), (1, 65536, 4, 1), (1, 70001, 3, 1), (2, 3000, 30, 3)])
def test_streaming_statistics_whatever_comes_first(plan, shape, far):
    """The first row far off, in front of hundreds to thousands of rows that are summed around it."""
    n, s, c, groups = shape
    xv = np.random.default_rng(22).standard_normal((n, s, c))
    xv[:, 0, :] += far
    x = place(xv, "f32")
    y, mean, rstd = forward(plan, x, None, None, groups, "f32")
    want, mean64, rstd64, _ = O.group_norm(f64(x), None, None, groups, 1e-5)
    # sums of values up to far + 5, each rounded to 2^-24 of the running sum
    assert np.max(np.abs(f64(mean) - mean64)) <= (far + 5) * 2e-6
    assert np.max(np.abs(f64(rstd) / rstd64 - 1)) <= 2e-5
    check(y, want, "f32", extra=np.max(rstd64) * (far + 5) * 2e-6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_values_with_a_small_spread_in_odd_rows(plan, dtype):
    """As test_large_values_with_a_small_spread, in the streaming form: a first row of zeros before values of 1e18."""
    n, s, c, groups = 2, 256, 64, 2
    xv = 1e18 * (1 + 0.02 * np.random.default_rng(31).standard_normal((n, s, c)))
    xv[1, 0] = 0.0
    x = place(xv, dtype, 0, 1)
    y, mean, rstd = forward(plan, x, None, None, groups, dtype, shift=1)
    want, mean64, rstd64, _ = O.group_norm(f64(x), None, None, groups, 1e-5)
    assert np.max(np.abs(f64(mean) - mean64)) <= 1.1e18 * 2e-6
    assert np.max(np.abs(f64(rstd) / rstd64 - 1)) <= 2e-5
    check(y, want, dtype, extra=np.max(rstd64) * 1.1e18 * 2e-6)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape,shift", [((4, 50, 64, 8), 0), ((4, 50, 64, 8), 1), ((2, 9000, 32, 4), 0), ((4, 50, 30, 5), 0)])
def test_gradients_from_above_where_relu_is_off_do_not_count(plan, shape, shift, dtype):
    """Infinities and NaN there give the very gradients that zeros give."""
    n, s, c, groups = shape
    xv, gv, bv, dyv = norm_data((n, s, c), 41)
    x, gamma, beta = place(xv, dtype, 0, shift), dev32(gv), dev32(bv)
    _, mean, rstd = forward(plan, x, gamma, beta, groups, dtype, shift=shift, act=B.CR_ACT_RELU)
    z = O.group_norm(f64(x), f64(gamma), f64(beta), groups, 1e-5)[3]
    off = np.argwhere(z < -0.5)
    off = off[:: max(1, len(off) // 7)]
    out = []
    for values in ([0.0], [float("inf"), float("-inf"), float("nan")]):
        for k, at in enumerate(off):
            dyv[tuple(at)] = values[k % len(values)]
        dy, dx = place(dyv, dtype, 0, shift), place(np.zeros(xv.shape), dtype, 0, shift)
        dg, db = torch.empty((n, c), device="cuda"), torch.empty((n, c), device="cuda")
        B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, groups, dx, dg, db, act=B.CR_ACT_RELU,
                                 workspace=scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, groups)))
        out.append((dx, dg, db))
    for zeros, others in zip(*out):
        assert torch.isfinite(others).all() and torch.equal(zeros, others)


def test_group_norm_in_place_on_another_stream_and_without_statistics(plan):
    xv, gv, bv, dyv = norm_data((6, 300, 64), 9)
    gamma, beta = dev32(gv), dev32(bv)
    x = place(xv, "f16")
    y, mean, rstd = forward(plan, x, gamma, beta, 8, "f16", act=B.CR_ACT_RELU)
    ws = scratch(B.cr_group_norm_workspace_bytes(plan, x, 8))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x2 = x.clone()
        B.cr_group_norm(plan, x2, gamma, beta, 8, x2, act=B.CR_ACT_RELU, workspace=ws)
    side.synchronize()
    assert torch.equal(x2, y)
    dy = place(dyv, "f16")
    ws = scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, 8))
    dx, dg, db = torch.empty_like(x), torch.empty((2, 64), device="cuda"), torch.empty((2, 64), device="cuda")
    B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, 8, dx, dg, db, act=B.CR_ACT_RELU, workspace=ws)
    only = torch.empty((2, 64), device="cuda")
    B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, 8, None, None, only, act=B.CR_ACT_RELU, workspace=ws)
    assert torch.equal(only, db)
    B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, 8, dy, act=B.CR_ACT_RELU, workspace=ws)
    assert torch.equal(dy, dx)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", [(3, 700, 64, 8), (1500, 512, 64, 8), (700, 512, 32, 32), (40, 9, 32, 8), (2, 9000, 32, 4), (5, 300, 30, 5)])
def test_group_norm_in_place_in_every_form(plan, shape, dtype):
    """y = x gives the bits of y elsewhere: items of one CTA, of clusters (one and several a cluster), and of the streaming form."""
    n, s, c, groups = shape
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn((n, s, c), generator=g, device="cuda").add_(3.0).to(TYPES[dtype])
    y, mean, rstd = forward(plan, x, None, None, groups, dtype, act=B.CR_ACT_SILU)
    ws = scratch(B.cr_group_norm_workspace_bytes(plan, x, groups))
    for _ in range(5):
        x2, mean2, rstd2 = x.clone(), torch.empty_like(mean), torch.empty_like(rstd)
        B.cr_group_norm(plan, x2, None, None, groups, x2, mean2, rstd2, act=B.CR_ACT_SILU, workspace=ws)
        assert torch.equal(x2, y) and torch.equal(mean2, mean) and torch.equal(rstd2, rstd)


@pytest.mark.parametrize("which", ["y", "dy", "dx"])
def test_workspace_of_tensors_that_are_less_aligned_than_x(plan, which):
    n, s, c, groups = 4, 300, 64, 8
    xv, gv, bv, dyv = norm_data((n, s, c), 51)
    gamma, beta = dev32(gv), dev32(bv)
    off = {which: 1}
    x, y = place(xv, "f32"), place(np.zeros(xv.shape), "f32", 0, off.get("y", 0))
    dy, dx = place(dyv, "f32", 0, off.get("dy", 0)), place(np.zeros(xv.shape), "f32", off.get("dx", 0), 0)
    mean, rstd = torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda")
    B.cr_group_norm(plan, x, gamma, beta, groups, y, mean, rstd,
                    workspace=scratch(B.cr_group_norm_workspace_bytes(plan, x, groups, y)))
    want = O.group_norm(f64(x), f64(gamma), f64(beta), groups, 1e-5)
    check(y, want[0], "f32")
    need = B.cr_group_norm_backward_workspace_bytes(plan, x, groups, dy, dx)
    B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, groups, dx, workspace=scratch(need))
    check(dx, O.group_norm_backward(f64(dy), f64(x), f64(gamma), f64(beta), groups, 1e-5)[0], "f32")
    # what the call itself asks for: one byte less is refused
    stats = (mean, rstd)
    ends = {"y": lambda ws: B.cr_group_norm(plan, x, gamma, beta, groups, y, *stats, workspace=ws)}
    ends["dy"] = ends["dx"] = lambda ws: B.cr_group_norm_backward(plan, dy, x, gamma, beta, *stats, groups, dx, workspace=ws)
    if which == "y":
        need = B.cr_group_norm_workspace_bytes(plan, x, groups, y)
        assert need > B.cr_group_norm_workspace_bytes(plan, x, groups, None) == 0
    with pytest.raises(B.CodedReduceError) as e:
        ends[which](scratch(need)[:need - 1])
    assert e.value.status == B.CR_ERR_OOM


def test_group_norm_of_no_samples(plan):
    x = torch.empty((0, 5, 8), device="cuda")
    B.cr_group_norm(plan, x, None, None, 2, torch.empty_like(x), torch.empty((0, 2), device="cuda"), torch.empty((0, 2), device="cuda"))
    dg = torch.full((3, 8), float("nan"), device="cuda")
    db = torch.full((3, 8), float("nan"), device="cuda")
    B.cr_group_norm_backward(plan, x, x, None, None, torch.empty((0, 2), device="cuda"), torch.empty((0, 2), device="cuda"), 2,
                             torch.empty_like(x), dg, db)
    assert not dg.any() and not db.any()


def test_group_norm_step_in_a_graph(plan):
    xv, gv, bv, dyv = norm_data((8, 256, 64), 12)
    x, dy, gamma, beta = place(xv, "bf16"), place(dyv, "bf16"), dev32(gv), dev32(bv)
    y, mean, rstd = torch.empty_like(x), torch.empty((8, 8), device="cuda"), torch.empty((8, 8), device="cuda")
    dx, dg, db = torch.empty_like(x), torch.empty((4, 64), device="cuda"), torch.empty((4, 64), device="cuda")
    ws1 = scratch(B.cr_group_norm_workspace_bytes(plan, x, 8))
    ws2 = scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, 8))
    kw = dict(act=B.CR_ACT_SILU, p=0.1, seed=4)

    def step():
        B.cr_group_norm(plan, x, gamma, beta, 8, y, mean, rstd, workspace=ws1, **kw)
        B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, 8, dx, dg, db, workspace=ws2, **kw)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (y, mean, rstd, dx, dg, db)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (y, mean, rstd, dx, dg, db):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (y, mean, rstd, dx, dg, db)))
    del graph


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 700, 64, 8), (600, 1024, 64, 8), (40, 1100, 48, 8)])
def test_group_norm_under_the_shortest_wait_limit(shape, dtype):
    """Items in clusters, whose CTAs wait for each other.  A limit of a microsecond may or may not run out: where it does the
    status says so; either way the call ends, writes nothing beside its outputs, and the next call is right."""
    n, s, c, groups = shape
    plan = B.cr_plan_create(4, 2, 1, 24, 1024, device=0)
    try:
        g = torch.Generator(device="cuda").manual_seed(n)
        rand = lambda: torch.randn((n, s, c), generator=g, device="cuda").to(TYPES[dtype])  # noqa: E731
        x, dy = rand(), rand()

        def step():
            wide = torch.full((2, n * s + 2, c), 7.0, dtype=TYPES[dtype], device="cuda")
            y, dx = wide[0, 1:-1].view(n, s, c), wide[1, 1:-1].view(n, s, c)
            mean, rstd = torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda")
            dg, db = torch.empty((n, c), device="cuda"), torch.empty((n, c), device="cuda")
            B.cr_group_norm(plan, x, None, None, groups, y, mean, rstd, act=B.CR_ACT_SILU)
            forward_status = B.cr_plan_device_status(plan)
            B.cr_group_norm_backward(plan, dy, x, None, None, mean, rstd, groups, dx, dg, db, act=B.CR_ACT_SILU,
                                     workspace=scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, groups)))
            status = B.cr_plan_device_status(plan)
            assert {status, forward_status} <= {B.CR_OK, B.CR_ERR_TIMEOUT}
            assert (wide[:, 0] == 7).all() and (wide[:, -1] == 7).all()
            return status, [t.clone() for t in (y, mean, rstd, dx, dg, db)]

        status, want = step()
        assert status == B.CR_OK
        for _ in range(10):
            B.cr_plan_set_wait_limit(plan, 1000)
            status, got = step()
            assert status == B.CR_ERR_TIMEOUT or all(torch.equal(a, b) for a, b in zip(got, want))
            B.cr_plan_clear_status(plan)
            B.cr_plan_set_wait_limit(plan, 2_000_000_000)
            status, got = step()
            assert status == B.CR_OK and all(torch.equal(a, b) for a, b in zip(got, want))
    finally:
        B.cr_plan_destroy(plan)


# ------------------------------------------------------------------------------------------------ dropout

@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (1, 7, 0, 0), (3, 8, 0, 0), (39, 5004, 0, 0), (5, 100, 12, 0),
                                                 (17, 33, 3, 1), (4, 64, 0, 2), (300, 96, 32, 0), (1, 100003, 0, 0)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(plan, rows, cols, pad, shift, dtype, residual):
    rng = np.random.default_rng(rows * cols)
    p, seed = [0.5, 0.1, 0.9][(rows + cols) % 3], (1 << 63) + 12345
    x = place(rng.standard_normal((rows, cols)), dtype, pad, shift)
    r = place(rng.standard_normal((rows, cols)), dtype, 0, shift) if residual else None
    for offset in (0, 1, 2, 3, (1 << 40) + 7):
        y = place(np.zeros((rows, cols)), dtype, pad, 0)
        B.cr_dropout(plan, x, y, p, seed, offset=offset, residual=r)
        want = f64(x) * O.dropout_factors((rows, cols), p, seed, offset)
        if residual:
            want = want + f64(r)
        else:
            assert np.array_equal(f64(y) == 0, want == 0)     # the mask itself
        assert np.all(np.abs(f64(y) - want) <= ROUND[dtype] * np.abs(want) + TINY[dtype] + 3e-7 * np.max(np.abs(f64(x))) * 10)


def test_dropout_of_parts_is_the_part_of_the_dropout(plan):
    x = torch.randn(1000, 37, device="cuda")
    y = torch.empty_like(x)
    B.cr_dropout(plan, x, y, 0.3, 42)
    for a, b in ((0, 1), (1, 400), (400, 1000)):
        part = torch.empty_like(x[a:b])
        B.cr_dropout(plan, x[a:b], part, 0.3, 42, offset=a * 37)
        assert torch.equal(part, y[a:b])
    keep = float((y != 0).float().mean())
    assert abs(keep - 0.7) <= 5 * (0.7 * 0.3 / 37000) ** 0.5      # five standard deviations
    other = torch.empty_like(x)
    B.cr_dropout(plan, x, other, 0.3, 43)
    both = float(((y != 0) & (other != 0)).float().mean())         # independent masks keep 0.49 of the elements in common
    assert abs(both - 0.49) <= 5 * (0.49 * 0.51 / 37000) ** 0.5


def test_dropout_ends_of_p_and_dropped_infinities(plan):
    for dtype in TYPES.values():
        x = torch.randn(50, 64, device="cuda").to(dtype)
        y = torch.empty_like(x)
        B.cr_dropout(plan, x, y, 0.0, 1)
        assert torch.equal(x, y)
        bad = torch.full_like(x, float("nan"))
        bad[::2] = float("inf")
        B.cr_dropout(plan, bad, y, 1.0, 1)
        assert not y.any()
        B.cr_dropout(plan, bad, y, 1.0, 1, residual=x)
        assert torch.equal(x, y)
        B.cr_dropout(plan, bad, y, 0.5, 1)
        gone = torch.from_numpy(O.dropout_factors((50, 64), 0.5, 1, 0) == 0).cuda()
        assert not y[gone].any() and not torch.isfinite(y[~gone]).any()
        z = x.clone()
        B.cr_dropout(plan, x, y, 0.25, 9, residual=x)
        B.cr_dropout(plan, z, z, 0.25, 9, residual=z)              # in place
        assert torch.equal(y, z)
    B.cr_dropout(plan, torch.empty((0, 5), device="cuda"), torch.empty((0, 5), device="cuda"), 0.5, 1)


def test_dropout_of_a_tensor_without_dimensions(plan):
    for offset in range(12):
        x = torch.tensor(3.0, device="cuda")
        y = torch.empty_like(x)
        B.cr_dropout(plan, x, y, 0.5, 7, offset=offset)
        assert float(y) == 3.0 * float(O.dropout_factors((1,), 0.5, 7, offset)[0])


# ------------------------------------------------------------------------------------------------ 8-bit products

def strided_codes(codes, ld, shift=0):
    rows, cols = codes.shape
    store = torch.full((rows * ld + shift + 16,), 77, dtype=torch.int8, device="cuda")
    view = torch.as_strided(store, (rows, cols), (ld, 1), shift)
    view.copy_(torch.from_numpy(codes.astype(np.int8)))
    return view


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 0), (5, 64, 0), (2, 4096, 0), (39, 5004, 12), (4, 9000, 0), (1, 40000, 8), (6, 333, 3)])
def test_quantize_rows(plan, rows, cols, pad, dtype):
    rng = np.random.default_rng(cols)
    values = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))
    if rows > 2:
        values[1] = 0.0
    x = place(values, dtype, pad)
    for ld in ((cols + 15) // 16 * 16, cols):
        q = strided_codes(np.full((rows, cols), 55), ld)
        scale = torch.full((rows,), float("nan"), device="cuda")
        B.cr_quantize_rows(plan, x, q, scale)
        codes, want = O.quantize_rows(f64(x))
        assert np.array_equal(q.cpu().numpy().astype(np.int64), codes)
        assert np.array_equal(scale.cpu().numpy(), want)


def test_quantize_rows_at_the_ends_of_the_range(plan):
    x = torch.zeros(9, 256, device="cuda")
    x[0] = torch.linspace(-1, 1, 256, device="cuda") * 3.4028234e38
    x[1, 3] = float("inf")
    x[2, 200] = float("nan")
    x[3] = torch.linspace(-1, 1, 256, device="cuda") * 2.0 ** -120
    x[4] = torch.linspace(-1, 1, 256, device="cuda") * 2.0 ** -121
    x[5, 0] = 1e-45
    x[6] = 5.0
    x[7] = (torch.arange(256, device="cuda") - 127.5).clamp(-127, 127)     # ties: half a code everywhere
    q = torch.full((9, 256), 55, dtype=torch.int8, device="cuda")
    scale = torch.empty(9, device="cuda")
    B.cr_quantize_rows(plan, x, q, scale)
    codes, want = O.quantize_rows(x.cpu().numpy())
    assert np.array_equal(q.cpu().numpy().astype(np.int64), codes)
    assert np.array_equal(scale.cpu().numpy(), want, equal_nan=True)


PRODUCTS = [(1, 1, 1), (1, 16, 16), (1, 4096, 512), (2, 64, 130), (3, 77, 7), (15, 128, 128), (16, 129, 129), (17, 640, 1),
            (33, 160, 300), (39, 5004, 1001), (64, 256, 256), (65, 272, 257), (100, 1000, 96), (129, 512, 384), (200, 2048, 130),
            (257, 96, 64), (300, 1040, 520), (1000, 48, 1000), (2048, 384, 256)]


@pytest.mark.parametrize("elem", list(TYPES))
@pytest.mark.parametrize("tokens,inner,outer", PRODUCTS)
def test_int8_product(plan, tokens, inner, outer, elem):
    rng = np.random.default_rng(tokens + inner + outer)
    xc = rng.integers(-127, 128, (tokens, inner))
    wc = rng.integers(-128, 128, (outer, inner))
    xs, ws = np.exp(rng.standard_normal(tokens)).astype(np.float32) / 50, np.exp(rng.standard_normal(outer)).astype(np.float32) / 900
    bias = rng.standard_normal(outer).astype(np.float32) if tokens % 2 else None
    want, sums = O.int8_product(xc, wc, xs, ws, bias)
    up = (inner + 15) // 16 * 16
    # rows on 16-byte boundaries, wider rows, and rows that start anywhere; outputs inside wider rows
    for ldx, ldw, shift, pad in ((up, up, 0, 0), (up + 16, up + 32, 16, 3), (inner, inner + 1, 1, 1)):
        x, w = strided_codes(xc, ldx, shift), strided_codes(wc, ldw, shift)
        y = place(np.zeros((tokens, outer)), elem, pad)
        B.cr_int8_product(plan, x, dev32(xs), w, dev32(ws), y, bias=dev32(bias))
        got = f64(y)
        # the sum is exact; its conversion, the product of the scales, the product and the sum with the bias round once each
        size = np.abs(sums * xs[:, None].astype(np.float64) * ws[None, :].astype(np.float64)) + (0 if bias is None else np.abs(bias))
        assert np.all(np.abs(got - want) <= 4 * 2.0 ** -24 * size + ROUND[elem] * 1.01 * np.abs(want) + TINY[elem])


def kernels_of(call):
    """Names of the kernels that `call` launches, from a graph that captures it."""
    from cuda.bindings import driver
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw = driver.CUgraph(graph.raw_cuda_graph())
    _, _, count = driver.cuGraphGetNodes(raw, 0)
    _, nodes, _ = driver.cuGraphGetNodes(raw, count)
    names = []
    for node in nodes[:count]:
        err, params = driver.cuGraphKernelNodeGetParams(node)
        assert err == driver.CUresult.CUDA_SUCCESS
        err, name = driver.cuFuncGetName(params.func)
        assert err == driver.CUresult.CUDA_SUCCESS
        names.append(name.decode())
    return names


@pytest.mark.parametrize("tokens,inner,outer", [(1, 5004, 1001), (1, 77, 130), (1, 77, 1), (5, 77, 1), (300, 1000, 1)])
def test_one_row_of_codes_takes_the_tensor_cores(plan, tokens, inner, outer):
    """torch calls a view of one row contiguous and its stride is lost; it does not count."""
    rng = np.random.default_rng(tokens + inner)
    up = (inner + 15) // 16 * 16
    values = rng.standard_normal((tokens, inner))
    xf = place(values, "bf16", (inner + 7) // 8 * 8 - inner)
    q, scale = strided_codes(np.full((tokens, inner), 55), up), torch.empty(tokens, device="cuda")
    names = kernels_of(lambda: B.cr_quantize_rows(plan, xf, q, scale))
    assert len(names) == 1 and "cr_quantize_rows_kernel" in names[0] and "Li8E" in names[0]
    codes, want_scale = O.quantize_rows(f64(xf))
    assert np.array_equal(q.cpu().numpy().astype(np.int64), codes) and np.array_equal(scale.cpu().numpy(), want_scale)
    wc = rng.integers(-128, 128, (outer, inner))
    w, ws = strided_codes(wc, up), np.exp(rng.standard_normal(outer)).astype(np.float32) / 900
    y, ws_dev = torch.empty((tokens, outer), device="cuda"), dev32(ws)
    names = kernels_of(lambda: B.cr_int8_product(plan, q, scale, w, ws_dev, y))
    assert len(names) == 1 and "cr_int8_product_kernel" in names[0]
    want, sums = O.int8_product(codes, wc, want_scale, ws)
    assert np.all(np.abs(f64(y) - want) <= 4 * 2.0 ** -24 * np.abs(want) + 2.0 ** -23 * np.abs(want))


def test_int8_product_longest_sum_and_nan_scales(plan):
    inner = 131071
    x = torch.full((2, 131072), -128, dtype=torch.int8, device="cuda")[:, :inner]
    w = torch.full((130, 131072), -128, dtype=torch.int8, device="cuda")[:, :inner]
    w[5] = 127
    one = torch.ones(130, device="cuda")
    y = torch.empty((2, 130), device="cuda")
    B.cr_int8_product(plan, x, torch.tensor([1.0, float("nan")], device="cuda"), w, one, y)
    want = torch.full((130,), float(128 * 128 * inner), device="cuda")
    want[5] = float(-128 * 127 * inner)
    assert torch.equal(y[0], want) and torch.isnan(y[1]).all()


def test_int8_product_of_nothing_and_repeats_itself(plan):
    w = torch.zeros((16, 64), dtype=torch.int8, device="cuda")
    B.cr_int8_product(plan, torch.empty((0, 64), dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"), w,
                      torch.ones(16, device="cuda"), torch.empty((0, 16), device="cuda"))
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(-127, 128, (300, 4096), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-127, 128, (1024, 4096), generator=g, device="cuda", dtype=torch.int8)
    xs, ws = torch.rand(300, device="cuda"), torch.rand(1024, device="cuda")
    full = torch.empty((300, 1024), device="cuda")
    B.cr_int8_product(plan, x, xs, w, ws, full)
    # a token's result does not depend on the tokens beside it (other tiles, other splits of k)
    for a, b in ((0, 1), (1, 18), (18, 100), (100, 300)):
        part = torch.empty((b - a, 1024), device="cuda")
        B.cr_int8_product(plan, x[a:b], xs[a:b], w, ws, part)
        assert torch.equal(part, full[a:b])


@pytest.mark.parametrize("tokens,inner,outer", [(1, 131056, 300), (40, 131056, 300), (200, 8192, 16384), (2048, 131056, 512), (4096, 8192, 4096)])
def test_products_under_the_shortest_wait_limit(tokens, inner, outer):
    """A limit of a microsecond may or may not run out.  Where it does the status says so; either way the call ends, writes
    nothing beside its output, and the next call with an ordinary limit is right."""
    plan = B.cr_plan_create(4, 2, 1, 24, 1024, device=0)
    try:
        g = torch.Generator(device="cuda").manual_seed(tokens)
        x = torch.randint(-127, 128, (tokens, inner), generator=g, device="cuda", dtype=torch.int8)
        w = torch.randint(-127, 128, (outer, inner), generator=g, device="cuda", dtype=torch.int8)
        xs, ws = torch.rand(tokens, generator=g, device="cuda"), torch.rand(outer, generator=g, device="cuda")
        want = torch.empty((tokens, outer), device="cuda")
        B.cr_int8_product(plan, x, xs, w, ws, want)
        for _ in range(20):
            B.cr_plan_set_wait_limit(plan, 1000)
            wide = torch.full((tokens + 2, outer + 8), 7.0, device="cuda")
            y = wide[1:-1, 4:-4]
            B.cr_int8_product(plan, x, xs, w, ws, y)
            status = B.cr_plan_device_status(plan)
            assert status in (B.CR_OK, B.CR_ERR_TIMEOUT)
            assert status == B.CR_ERR_TIMEOUT or torch.equal(y, want)
            y.zero_()
            assert (wide[0] == 7).all() and (wide[-1] == 7).all() and (wide[:, :4] == 7).all() and (wide[:, -4:] == 7).all()
            B.cr_plan_clear_status(plan)
            B.cr_plan_set_wait_limit(plan, 2_000_000_000)
            B.cr_int8_product(plan, x, xs, w, ws, y)
            assert B.cr_plan_device_status(plan) == B.CR_OK and torch.equal(y, want)
    finally:
        B.cr_plan_destroy(plan)


# ------------------------------------------------------------------------------------------------ beyond 32 bits

def test_dropout_of_more_than_2_to_31_elements(plan):
    for count in ((1 << 31) + 4096, (1 << 31) + 4097):      # in vectors, and element by element
        x = torch.empty(count, dtype=torch.float16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
        y = torch.empty_like(x)
        B.cr_dropout(plan, x, y, 0.25, 77, offset=3)
        for a in (0, (1 << 31) - 500, count - 1000):
            factors = O.dropout_factors((1000,), 0.25, 77, 3 + a)
            got, want = f64(y[a:a + 1000]), f64(x[a:a + 1000]) * factors
            assert np.array_equal(got == 0, want == 0) and np.all(np.abs(got - want) <= ROUND["f16"] * np.abs(want) + TINY["f16"])
        del x, y


def test_group_norm_of_more_than_2_to_31_elements(plan):
    n, s, c, groups = 520, 4096, 1024, 32
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty((n, s, c), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    dy = torch.empty_like(x).normal_(generator=g)
    gamma, beta = torch.rand(c, generator=g, device="cuda") + 0.5, torch.rand(c, generator=g, device="cuda")
    kw = dict(act=B.CR_ACT_SILU, p=0.25, seed=5)
    y, mean, rstd = torch.empty_like(x), torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda")
    B.cr_group_norm(plan, x, gamma, beta, groups, y, mean, rstd, workspace=scratch(B.cr_group_norm_workspace_bytes(plan, x, groups)), **kw)
    dx, dg, db = torch.empty_like(x), torch.empty((n, c), device="cuda"), torch.empty((n, c), device="cuda")
    B.cr_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, groups, dx, dg, db,
                             workspace=scratch(B.cr_group_norm_backward_workspace_bytes(plan, x, groups)), **kw)
    k = n - 1                                               # the last sample lies beyond 2^31 elements
    factors = O.dropout_factors((1, s, c), 0.25, 5, k * s * c)
    want, mean64, _, _ = O.group_norm(f64(x[k:]), f64(gamma), f64(beta), groups, 1e-5, "silu", factors)
    check(y[k:], want, "bf16")
    assert np.max(np.abs(f64(mean[k:]) - mean64)) <= 1e-6
    dx64, dg64, db64, _, ag, ab = O.group_norm_backward(f64(dy[k:]), f64(x[k:]), f64(gamma), f64(beta), groups, 1e-5, "silu", factors)
    check(dx[k:], dx64, "bf16")
    assert np.all(np.abs(f64(dg[k:]) - dg64) <= 1e-5 * ag) and np.all(np.abs(f64(db[k:]) - db64) <= 1e-5 * ab)


def test_int8_product_of_weights_beyond_2_to_31_bytes(plan):
    outer, inner = 600000, 4096
    g = torch.Generator(device="cuda").manual_seed(3)
    w = torch.randint(-127, 128, (outer, inner), generator=g, device="cuda", dtype=torch.int8)
    for tokens in (2, 300):
        x = torch.randint(-127, 128, (tokens, inner), generator=g, device="cuda", dtype=torch.int8)
        y = torch.empty((tokens, outer), device="cuda")
        B.cr_int8_product(plan, x, torch.ones(tokens, device="cuda"), w, torch.ones(outer, device="cuda"), y)
        for a in (0, outer - 200):
            want, _ = O.int8_product(x.cpu().numpy(), w[a:a + 200].cpu().numpy(), np.ones(tokens), np.ones(200))
            assert np.max(np.abs(f64(y[:, a:a + 200]) - want) / (1 + np.abs(want))) <= 2.0 ** -23


# ------------------------------------------------------------------------------------------------ refusals

def test_refusals_launch_nothing(plan):
    x = torch.zeros(4, 10, 8, device="cuda")
    y, stats = torch.empty_like(x), torch.empty((4, 2), device="cuda")
    params = torch.empty((4, 8), device="cuda")
    ws = scratch(1 << 20)
    q, codes = torch.zeros((4, 64), dtype=torch.int8, device="cuda"), torch.zeros((4, 8), dtype=torch.int8, device="cuda")
    one, out = torch.ones(4, device="cuda"), torch.empty((4, 4), device="cuda")
    lib, before = B.lib(), B.cr_plan_launch_count(plan)
    bad = B.CR_ERR_INVALID_ARG
    p = lambda t: t.data_ptr()  # noqa: E731
    stream = torch.cuda.current_stream().cuda_stream

    def desc(**kw):
        v = dict(samples=4, positions=10, channels=8, groups=2, elem=0, act=0, eps=1e-5, p=0.0, seed=0, offset=0)
        v.update(kw)
        return B.cr_group_norm_t(**v)

    for kw in (dict(samples=-1), dict(positions=0), dict(channels=0), dict(groups=0), dict(groups=3), dict(elem=3), dict(elem=-1), dict(act=3),
               dict(eps=-1.0), dict(eps=float("nan")), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(offset=-1)):
        assert lib.cr_group_norm(plan, desc(**kw), p(x), 8, 0, 0, p(y), 8, 0, 0, p(ws), 1 << 20, stream) == bad, kw
        assert lib.cr_group_norm_workspace_bytes(plan, desc(**kw), 1) == 0
        assert lib.cr_group_norm_backward(plan, desc(**kw), p(x), 8, p(x), 8, 0, 0, p(stats), p(stats), p(y), 8, 0, 0, 8, 1, p(ws),
                                          1 << 20, stream) == bad, kw
    d = desc()
    assert lib.cr_group_norm(plan, d, 0, 8, 0, 0, p(y), 8, 0, 0, p(ws), 1 << 20, stream) == bad           # no x
    assert lib.cr_group_norm(plan, d, p(x), 7, 0, 0, p(y), 8, 0, 0, p(ws), 1 << 20, stream) == bad        # rows overlap
    assert lib.cr_group_norm(plan, d, p(x) + 2, 8, 0, 0, p(y), 8, 0, 0, p(ws), 1 << 20, stream) == bad    # off its element
    assert lib.cr_group_norm(plan, d, p(x), 8, 0, 0, p(y), 8, p(stats), 0, p(ws), 1 << 20, stream) == bad  # mean without rstd
    assert lib.cr_group_norm(0, d, p(x), 8, 0, 0, p(y), 8, 0, 0, p(ws), 1 << 20, stream) == bad
    back = lambda parts, ldp, nbytes, rstd=stats: lib.cr_group_norm_backward(  # noqa: E731
        plan, d, p(x), 8, p(x), 8, 0, 0, p(stats), 0 if rstd is None else p(rstd), p(y), 8, p(params), 0, ldp, parts, p(ws), nbytes, stream)
    assert back(3, 8, 1 << 20) == bad and back(0, 8, 1 << 20) == bad and back(4, 7, 1 << 20) == bad and back(4, 8, 1 << 20, None) == bad
    need = lib.cr_group_norm_backward_workspace_bytes(plan, d, 1)
    assert need and back(4, 8, need - 1) == B.CR_ERR_OOM
    need = lib.cr_group_norm_workspace_bytes(plan, d, 0)     # rows off their vectors: the streaming form
    assert need and lib.cr_group_norm(plan, d, p(x) + 4, 8, 0, 0, p(y), 8, 0, 0, p(ws), need - 1, stream) == B.CR_ERR_OOM
    assert lib.cr_group_norm(plan, d, p(x) + 4, 8, 0, 0, p(y), 8, 0, 0, p(ws) + 4, need, stream) == bad
    drop = lambda ld=8, rows=40, elem=0, pr=0.5, off=0: lib.cr_dropout(plan, p(x), ld, 0, 0, p(y), 8, rows, 8, elem, pr, 1, off, stream)  # noqa: E731
    assert [drop(ld=7), drop(rows=-1), drop(elem=9), drop(pr=2.0), drop(pr=float("nan")), drop(off=-4)] == [bad] * 6
    quant = lambda rows=4, cols=8, ldq=8, elem=0: lib.cr_quantize_rows(plan, p(x), 8, rows, cols, elem, p(codes), ldq, p(one), stream)  # noqa: E731
    assert [quant(rows=-1), quant(cols=0), quant(ldq=7), quant(elem=5)] == [bad] * 4
    prod = lambda k=64, ld=64, elem=0, m=4, sc=one: lib.cr_int8_product(  # noqa: E731
        plan, p(q), ld, p(sc) if sc is not None else 0, p(q), 64, p(one), 0, p(out), 4, m, 4, k, elem, stream)
    assert [prod(k=0), prod(k=131072), prod(ld=63), prod(elem=3), prod(m=-1), prod(sc=None), prod(m=(1 << 31) - 300)] == [bad] * 7
    host = B.cr_plan_create(4, 2, 1, 24, 1024, device=-1)
    assert lib.cr_dropout(host, p(x), 8, 0, 0, p(y), 8, 40, 8, 0, 0.5, 1, 0, stream) == B.CR_ERR_CUDA
    B.cr_plan_destroy(host)
    assert B.cr_plan_launch_count(plan) == before
    # the binding's own checks
    for call in (lambda: B.cr_dropout(plan, x, y[:2], 0.5, 1), lambda: B.cr_dropout(plan, x, y.half(), 0.5, 1),
                 lambda: B.cr_dropout(plan, x.double(), y, 0.5, 1), lambda: B.cr_dropout(plan, x.cpu(), y, 0.5, 1),
                 lambda: B.cr_dropout(plan, x.transpose(0, 1), y.transpose(0, 1), 0.5, 1),
                 lambda: B.cr_dropout(plan, x[..., ::2], y[..., ::2], 0.5, 1),
                 lambda: B.cr_dropout(plan, x[0, 0].expand(40, 8), y.view(40, 8), 0.5, 1),          # one row, forty times
                 lambda: B.cr_dropout(plan, x[:1].expand(4, 10, 8), y, 0.5, 1),
                 lambda: B.cr_group_norm_backward(plan, one[0].expand(4, 10, 8), x, None, None, stats, stats, 2, y, workspace=ws),
                 lambda: B.cr_group_norm(plan, x, one, None, 2, y, workspace=ws),
                 lambda: B.cr_group_norm(plan, x[0], None, None, 2, y[0], workspace=ws),
                 lambda: B.cr_int8_product(plan, x[0], one, q, one, out), lambda: B.cr_int8_product(plan, q[:, :32], one, q, one, out),
                 lambda: B.cr_quantize_rows(plan, x[0], q[:, :8], one)):
        with pytest.raises(ValueError):
            call()
    assert B.cr_plan_launch_count(plan) == before


def test_fp32_operands_off_their_elements_are_refused(plan):
    x = torch.zeros(4, 10, 8, device="cuda")
    y, stats, params = torch.empty_like(x), torch.zeros((4, 2), device="cuda"), torch.zeros((5, 8), device="cuda")
    codes, one, out, ws = torch.zeros((4, 64), dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda"), torch.empty((4, 4), device="cuda"), scratch(1 << 20)
    lib, before, bad = B.lib(), B.cr_plan_launch_count(plan), B.CR_ERR_INVALID_ARG
    p = lambda t: t.data_ptr()  # noqa: E731
    stream = torch.cuda.current_stream().cuda_stream
    desc = B.cr_group_norm_t(4, 10, 8, 2, B.CR_ELEM_F32, 0, 1e-5, 0.0, 0, 0)
    for off in (1, 2, 3):
        for k in range(4):      # gamma, beta, mean, rstd
            a = [p(one) if k < 2 else 0, p(one) if k < 2 else 0, p(stats), p(stats)]
            a[k] += off
            assert lib.cr_group_norm(plan, desc, p(x), 8, a[0], a[1], p(y), 8, a[2], a[3], p(ws), 1 << 20, stream) == bad
        for k in range(6):      # gamma, beta, mean, rstd, dgamma, dbeta
            a = [p(one), p(one), p(stats), p(stats), p(params), p(params)]
            a[k] += off
            assert lib.cr_group_norm_backward(plan, desc, p(x), 8, p(x), 8, a[0], a[1], a[2], a[3], p(y), 8, a[4], a[5], 8, 4, p(ws),
                                              1 << 20, stream) == bad
        assert lib.cr_quantize_rows(plan, p(x), 8, 4, 8, B.CR_ELEM_F32, p(codes), 16, p(one) + off, stream) == bad
        for k in range(3):      # x_scale, w_scale, bias
            a = [p(one), p(one), p(one)]
            a[k] += off
            assert lib.cr_int8_product(plan, p(codes), 64, a[0], p(codes), 64, a[1], a[2], p(out), 4, 4, 4, 64, B.CR_ELEM_F32, stream) == bad
    assert B.cr_plan_launch_count(plan) == before


def test_numbers_that_a_field_would_cut_are_refused(plan):
    x = torch.zeros(4, 10, 8, device="cuda")
    y, stats, ws = torch.empty_like(x), torch.zeros((4, 2), device="cuda"), scratch(1 << 20)
    wide = x[0, 0, :1].expand(1, 1, (1 << 32) + 8)
    before = B.cr_plan_launch_count(plan)
    for kw in (dict(groups=(1 << 32) + 2), dict(act=1 << 32), dict(offset=1 << 64), dict(offset=(1 << 63) + 1), dict(seed=1 << 64)):
        args = dict(dict(groups=2, workspace=ws), **kw)
        with pytest.raises(ValueError):
            B.cr_group_norm(plan, x, None, None, y=y, **args)
        with pytest.raises(ValueError):
            B.cr_group_norm_backward(plan, x, x, None, None, stats, stats, dx=y, **args)
        if "seed" in kw or "offset" in kw:
            with pytest.raises(ValueError):
                B.cr_dropout(plan, x, y, 0.5, kw.get("seed", 1), offset=kw.get("offset", 0))
    for query in (B.cr_group_norm_workspace_bytes, B.cr_group_norm_backward_workspace_bytes):
        for t, groups in ((x, (1 << 32) + 2), (wide, 2), (x[0], 2), (x[None], 2)):
            with pytest.raises(ValueError):
                query(plan, t, groups)
    assert B.cr_plan_launch_count(plan) == before
    B.cr_dropout(plan, x, y, 0.5, -1)
    B.cr_dropout(plan, x, x, 0.5, (1 << 64) - 1)
    assert torch.equal(x, y)
