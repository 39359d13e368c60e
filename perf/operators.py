"""Measured cases of the layer operators: group norm with activation and dropout, dropout, 8-bit integer product.

Each case runs either in plain form (elementary torch operations in 32 bits) or, where `own` is true, through
the package's binding.  Sizes are those of the repository's workloads (partitions of 39 x 5004 and 2048 x 4096,
48 and 168 partitions, 32 x 32 images) and generic ones around them.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # one sample of a late, small feature map: nothing but latency
        dict(name="norm_one_sample", op="norm", dtype="bf16", samples=1, positions=64, channels=128, groups=32, act="silu",
             p=0.0, pad=0),
        # a partition of 39 samples with odd feature maps: 221 positions, 12 channels a group, rows inside wider rows
        dict(name="norm_odd_partition", op="norm", dtype="f32", samples=39, positions=221, channels=60, groups=5, act="relu",
             p=0.0, pad=4),
        # training forward of a 32 x 32 feature map for a whole step's batch, dropout behind the activation
        dict(name="norm_train_batch", op="norm", dtype="bf16", samples=256, positions=1024, channels=256, groups=32, act="silu",
             p=0.1, pad=0),
        # two full-size images: a group is larger than what a few SMs can hold
        dict(name="norm_images", op="norm", dtype="f16", samples=2, positions=65536, channels=64, groups=8, act="silu",
             p=0.0, pad=0),
        # gradients of 48 partitions of one sample each at the end of a network
        dict(name="norm_grad_small", op="norm_grad", dtype="f32", samples=48, positions=49, channels=96, groups=8, act="silu",
             p=0.0, pad=0, partitions=48),
        # gradients of a training batch cut into 48 partitions, dropout in front
        dict(name="norm_grad_train", op="norm_grad", dtype="bf16", samples=192, positions=1024, channels=256, groups=32,
             act="silu", p=0.1, pad=0, partitions=48),
        # the features of one partition of the logistic workload
        dict(name="dropout_partition", op="dropout", dtype="f32", rows=39, cols=5004, p=0.5, residual=False, pad=0),
        # a residual branch of a large batch
        dict(name="dropout_residual", op="dropout", dtype="bf16", rows=16384, cols=4096, p=0.1, residual=True, pad=0),
        # one token through a square layer: the weights are what is read
        dict(name="int8_one_token", op="int8", dtype="bf16", out="bf16", tokens=1, inner=4096, outer=4096, bias=True),
        # a partition of 39 samples of 5004 features into an odd number of channels
        dict(name="int8_odd_partition", op="int8", dtype="f32", out="f32", tokens=39, inner=5004, outer=1001, bias=True),
        # a partition of 2048 samples of 4096 features
        dict(name="int8_partition", op="int8", dtype="bf16", out="bf16", tokens=2048, inner=4096, outer=4096, bias=False),
        # several partitions at once
        dict(name="int8_batch", op="int8", dtype="bf16", out="bf16", tokens=16384, inner=4096, outer=8192, bias=True),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "dropout", "int8"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op == "int8":
        tokens, inner = _log_int(rng, 1, 16384), _log_int(rng, 64, 8192)
        outer = _log_int(rng, 64, min(16384, max(64, 2 ** 38 // (tokens * inner))))
        return dict(op=op, dtype=dtype, out=rng.choice(["f32", "bf16", "f16"]), tokens=tokens, inner=inner, outer=outer,
                    bias=rng.random() < 0.5)
    p = rng.choice([0.0, 0.1, 0.25, 0.5])
    if op == "dropout":
        cols = _log_int(rng, 1, 16384)
        rows = _log_int(rng, 1, max(1, 2 ** 25 // cols))
        return dict(op=op, dtype=dtype, rows=rows, cols=cols, p=p or 0.1, residual=rng.random() < 0.5,
                    pad=rng.choice([0, 0, 0, 8, 3]))
    groups = rng.choice([1, 2, 4, 8, 16, 32, 5])
    channels = groups * _log_int(rng, 1, 64)
    positions = _log_int(rng, 16, min(65536, 2 ** 24 // channels))   # feature maps from 4 x 4 on
    samples = _log_int(rng, 1, max(1, min(512, 2 ** 25 // (channels * positions))))
    case = dict(op=op, dtype=dtype, samples=samples, positions=positions, channels=channels, groups=groups,
                act=rng.choice(["none", "relu", "silu"]), p=p, pad=rng.choice([0, 0, 0, 8, 3]))
    if op == "norm_grad":
        case["partitions"] = rng.choice([k for k in range(1, samples + 1) if samples % k == 0])
    return case


def work(case):
    op, size = case["op"], SIZE[case["dtype"]]
    if op == "int8":
        m, k, n = case["tokens"], case["inner"], case["outer"]
        return {"bytes": m * k * size + n * k + 4 * n * (2 if case["bias"] else 1) + m * n * SIZE[case["out"]],
                "flops": 2 * m * n * k}
    if op == "dropout":
        count = case["rows"] * case["cols"]
        return {"bytes": count * size * (3 if case["residual"] else 2), "flops": count * (2 if case["residual"] else 1)}
    count = case["samples"] * case["positions"] * case["channels"]
    stats = 8 * case["samples"] * case["groups"] + 8 * case["channels"]
    if op == "norm":
        return {"bytes": 2 * count * size + stats, "flops": 10 * count}
    return {"bytes": 3 * count * size + stats + 8 * case["partitions"] * case["channels"], "flops": 20 * count}


# ------------------------------------------------------------------------------------------------ inputs

def _rows_of(shape, pad, dtype, values):
    """`values` (32 bits) rounded to `dtype`, as a view into rows that are `pad` elements longer."""
    if not pad:
        return values.to(dtype)
    wide = torch.zeros(*shape[:-1], shape[-1] + pad, dtype=dtype, device=values.device)
    wide[..., :shape[-1]] = values
    return wide[..., :shape[-1]]


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    dtype = DTYPES[case["dtype"]]
    s = {"case": case, "seed": (seed * 7919 + 17) % (1 << 62)}
    if case["op"] == "dropout":
        shape = (case["rows"], case["cols"])
        s["offset"] = (seed % 5) * case["rows"] * case["cols"]   # one of the first five such blocks of a data set
        s["x"] = _rows_of(shape, case["pad"], dtype, rand(*shape))
        s["residual"] = _rows_of(shape, 0, dtype, rand(*shape)) if case["residual"] else None
        return s
    if case["op"] == "int8":
        m, k, n = case["tokens"], case["inner"], case["outer"]
        s["x"] = (rand(m, k) * torch.exp(0.5 * rand(m, 1))).to(dtype)
        w = rand(n, k) * (torch.exp(0.3 * rand(n, 1)) / math.sqrt(k))
        s["w_scale"] = w.abs().amax(1) / 127.0
        s["w"] = torch.zeros(n, (k + 15) // 16 * 16, dtype=torch.int8, device="cuda")   # rows on 16-byte boundaries
        s["w"][:, :k] = torch.round(w / s["w_scale"][:, None]).clamp(-127, 127).to(torch.int8)
        s["w"] = s["w"][:, :k]
        s["bias"] = 0.1 * rand(n) if case["bias"] else None
        return s
    shape = (case["samples"], case["positions"], case["channels"])
    s["offset"] = (seed % 5) * shape[0] * shape[1] * shape[2]
    values = rand(*shape).mul_(torch.exp(0.3 * rand(shape[2]))).add_(0.5 * rand(shape[2]))   # channels with their own mean and spread
    s["x"] = _rows_of(shape, case["pad"], dtype, values)
    s["gamma"], s["beta"] = 1 + 0.2 * rand(shape[2]), 0.2 * rand(shape[2])
    if case["op"] == "norm_grad":
        s["dy"] = rand(*shape).to(dtype)
        s["mean"], s["rstd"] = _statistics(s["x"].float(), case["groups"])
    return s


_kept = {}


def _plan():
    """The plan that a program on this device keeps."""
    if "plan" not in _kept:
        from paper_1902_01981_b200 import binding as B
        _kept["binding"] = B
        _kept["plan"] = B.cr_plan_create(4, 2, 1, 48, 4096, device=torch.cuda.current_device())
    return _kept["binding"], _kept["plan"]


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        s["binding"], s["plan"] = _plan()
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


def _own_norm(s):
    B, c, x = s["binding"], s["case"], s["x"]
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    mean = torch.empty((c["samples"], c["groups"]), device=x.device)
    rstd = torch.empty((c["samples"], c["groups"]), device=x.device)
    need = B.cr_group_norm_workspace_bytes(s["plan"], x, c["groups"])
    ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    B.cr_group_norm(s["plan"], x, s["gamma"], s["beta"], c["groups"], y, mean, rstd, eps=EPS, act=B.CR_ACT[c["act"]],
                    p=c["p"], seed=s["seed"], offset=s["offset"], workspace=ws)
    return {"y": y, "mean": mean, "rstd": rstd}


def _own_norm_grad(s):
    B, c, x = s["binding"], s["case"], s["x"]
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dgamma = torch.empty((c["partitions"], c["channels"]), device=x.device)
    dbeta = torch.empty((c["partitions"], c["channels"]), device=x.device)
    need = B.cr_group_norm_backward_workspace_bytes(s["plan"], x, c["groups"])
    ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    B.cr_group_norm_backward(s["plan"], s["dy"], x, s["gamma"], s["beta"], s["mean"], s["rstd"], c["groups"], dx, dgamma,
                             dbeta, act=B.CR_ACT[c["act"]], p=c["p"], seed=s["seed"], offset=s["offset"], workspace=ws)
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _own_dropout(s):
    B, c, x = s["binding"], s["case"], s["x"]
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    B.cr_dropout(s["plan"], x, y, c["p"], s["seed"], offset=s["offset"], residual=s["residual"])
    return y


def _own_int8(s):
    B, c, x = s["binding"], s["case"], s["x"]
    q = torch.empty((c["tokens"], (c["inner"] + 15) // 16 * 16), dtype=torch.int8, device=x.device)[:, :c["inner"]]
    scale = torch.empty(c["tokens"], device=x.device)
    y = torch.empty((c["tokens"], c["outer"]), dtype=DTYPES[c["out"]], device=x.device)
    B.cr_quantize_rows(s["plan"], x, q, scale)
    B.cr_int8_product(s["plan"], q, scale, s["w"], s["w_scale"], y, bias=s["bias"])
    return y


_own = {"norm": _own_norm, "norm_grad": _own_norm_grad, "dropout": _own_dropout, "int8": _own_int8}


def _srl(z, k):
    return (z >> k) & ((1 << (64 - k)) - 1)


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


_C1, _C2, _GAMMA = _signed(0xBF58476D1CE4E5B9), _signed(0x94D049BB133111EB), _signed(0x9E3779B97F4A7C15)


def _mix(z):
    z = (z ^ _srl(z, 30)) * _C1
    z = (z ^ _srl(z, 27)) * _C2
    return z ^ _srl(z, 31)


def _threshold(p):
    return int(round(p * 65536))


def _kept_elements(count, p, seed, offset):
    """Truth values of `count` elements from index `offset` on, and the scale of the kept ones."""
    first, last = offset // 4, (offset + count + 3) // 4
    key = _mix(torch.tensor(_signed(seed), device="cuda"))
    words = _mix(key + (torch.arange(first, last, device="cuda") + 1) * _GAMMA)
    lanes = (words[:, None] >> torch.tensor([0, 16, 32, 48], device="cuda")) & 0xFFFF
    t = _threshold(p)
    return (lanes.view(-1)[offset - 4 * first:][:count] >= t), 65536.0 / (65536 - t)


def _dropped(v, p, seed, offset):
    if p == 0.0:
        return v
    keep, scale = _kept_elements(v.numel(), p, seed, offset)
    return torch.where(keep.view(v.shape), v * scale, 0.0)


def _statistics(x, groups):
    v = x.reshape(x.shape[0], x.shape[1], groups, -1)
    mean = v.mean((1, 3))
    var = (v - mean[:, None, :, None]).square().mean((1, 3))
    return mean, 1.0 / torch.sqrt(var + EPS)


def _normalised(x, mean, rstd, groups):
    v = x.view(x.shape[0], x.shape[1], groups, -1)
    return ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).view(x.shape)


def _plain_norm(s):
    c, x = s["case"], s["x"].float().contiguous()
    mean, rstd = _statistics(x, c["groups"])
    z = _normalised(x, mean, rstd, c["groups"]) * s["gamma"] + s["beta"]
    if c["act"] == "relu":
        z = torch.where(z > 0, z, 0.0)
    elif c["act"] == "silu":
        z = z / (1 + torch.exp(-z))
    return {"y": _dropped(z, c["p"], s["seed"], s["offset"]).to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _plain_norm_grad(s):
    c, x = s["case"], s["x"].float().contiguous()
    xhat = _normalised(x, s["mean"], s["rstd"], c["groups"])
    dz = _dropped(s["dy"].float(), c["p"], s["seed"], s["offset"])
    z = xhat * s["gamma"] + s["beta"]
    if c["act"] == "relu":
        dz = torch.where(z > 0, dz, 0.0)
    elif c["act"] == "silu":
        sig = 1 / (1 + torch.exp(-z))
        dz = dz * sig * (1 + z * (1 - sig))
    parts = (c["partitions"], -1, c["channels"])
    out = {"dgamma": (dz * xhat).reshape(parts).sum(1), "dbeta": dz.reshape(parts).sum(1)}
    split = (c["samples"], c["positions"], c["groups"], -1)
    dxhat, xhat = (dz * s["gamma"]).view(split), xhat.view(split)
    dx = dxhat - dxhat.mean((1, 3), keepdim=True) - xhat * (dxhat * xhat).mean((1, 3), keepdim=True)
    out["dx"] = (dx * s["rstd"][:, None, :, None]).view(x.shape).to(s["x"].dtype)
    return out


def _plain_dropout(s):
    c = s["case"]
    y = _dropped(s["x"].float(), c["p"], s["seed"], s["offset"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _plain_int8(s):
    x, w = s["x"].float(), s["w"].float()
    largest = x.abs().amax(1, keepdim=True)
    full = torch.full_like(largest, 127.0)
    alive = largest >= 2.0 ** -120
    q = torch.where(alive, torch.round(x * (full / largest)), 0.0)
    scale = torch.where(alive, largest / full, 0.0)
    y = (q @ w.t()) * (scale * s["w_scale"])
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(DTYPES[s["case"]["out"]])


_plain = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "dropout": _plain_dropout, "int8": _plain_int8}


# ------------------------------------------------------------------------------------------------ 64 bits

def _mask_64(count, p, seed, offset):
    """Multipliers (0 or the scale) of `count` elements, by unsigned 64-bit arithmetic on the host."""
    if p == 0.0:
        return None
    u = np.uint64

    def finish(z):
        z ^= z >> u(30)
        z *= u(0xBF58476D1CE4E5B9)
        z ^= z >> u(27)
        z *= u(0x94D049BB133111EB)
        z ^= z >> u(31)
        return z

    start = finish(np.array([seed], dtype=u))
    words = np.arange(offset // 4 + 1, (offset + count + 3) // 4 + 1, dtype=u)
    words *= u(0x9E3779B97F4A7C15)
    words += start
    halves = finish(words).view(np.uint16)     # little end first: bits 0..15 belong to the first of four elements
    t = int(round(p * 65536))
    keep = halves[offset % 4: offset % 4 + count] >= t
    return torch.from_numpy(keep).cuda().double() * (65536.0 / (65536 - t))


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "dropout":
        y = s["x"].double() * _mask_64(s["x"].numel(), case["p"], s["seed"], s["offset"]).view(s["x"].shape)
        return y if s["residual"] is None else y + s["residual"].double()
    if case["op"] == "int8":
        x = s["x"].double()
        top = torch.linalg.vector_norm(x, ord=math.inf, dim=1)
        codes = torch.round(torch.einsum("mk,m->mk", x, 127.0 / top))
        y = torch.einsum("mk,nk->mn", codes, s["w"].double()) * torch.outer(top / 127.0, s["w_scale"].double())
        return y + s["bias"].double() if case["bias"] else y
    # the definition of the forward pass; the gradient is left to automatic differentiation
    grad = case["op"] == "norm_grad"
    x = s["x"].double().contiguous().requires_grad_(grad)
    spread = (case["partitions"], case["samples"] // case["partitions"], case["channels"]) if grad else None
    gamma, beta = s["gamma"].double(), s["beta"].double()
    if grad:   # a copy of the parameters for each partition
        gamma, beta = (v.expand(case["partitions"], -1).clone().requires_grad_(True) for v in (gamma, beta))
        by_sample = [v[:, None, :].expand(spread).reshape(case["samples"], 1, -1) for v in (gamma, beta)]
    else:
        by_sample = [gamma, beta]
    per = x.unflatten(2, (case["groups"], -1)).transpose(1, 2).flatten(2)
    var, mean = torch.var_mean(per, dim=2, correction=0)
    rstd = (var + EPS).rsqrt()
    widen = lambda v: v.repeat_interleave(case["channels"] // case["groups"], 1)[:, None, :]  # noqa: E731
    z = (x - widen(mean)) * widen(rstd) * by_sample[0] + by_sample[1]
    y = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu}[case["act"]](z)
    mask = _mask_64(y.numel(), case["p"], s["seed"], s["offset"])
    if mask is not None:
        y = y * mask.view(y.shape)
    if not grad:
        return {"y": y, "mean": mean, "rstd": rstd}
    dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), s["dy"].double())
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
