"""Measured cases of the token layers: embedding, root-mean-square norm, log probabilities of tokens, distillation.

Each case runs either in plain form (elementary torch operations in 32 bits) or, where `own` is true, through the
package's binding.  Sizes are those of the repository's workloads (partitions of 39 rows, 5004 features, 2048 x 4096,
24 and 48 partitions) and generic ones around them.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
IDS = {"i32": torch.int32, "i64": torch.int64}
ID_SIZE = {"i32": 4, "i64": 8}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # the categorical features of one partition of 39 rows: nothing but latency
        dict(name="embed_partition", op="embed", dtype="f32", ids="i64", tokens=39, vocab=5004, width=60, pad=0),
        # the tokens of a whole training step
        dict(name="embed_batch", op="embed", dtype="bf16", ids="i64", tokens=65536, vocab=32000, width=2048, pad=0),
        # gradients of 24 small partitions over the 256 byte values and one more
        dict(name="embed_grad_small", op="embed_grad", dtype="f32", ids="i32", partitions=24, tokens=39, vocab=257, width=60,
             pad=4),
        # gradients of a training step cut into four partitions; frequent tokens take thousands of rows each
        dict(name="embed_grad_train", op="embed_grad", dtype="bf16", ids="i64", partitions=4, tokens=16384, vocab=32000,
             width=1024, pad=0),
        # one new token between two layers
        dict(name="norm_token", op="norm", dtype="bf16", rows=1, cols=4096, residual=True, pad=0),
        # a training batch in front of an 8-bit layer: the sum goes on as residual stream, the norm into codes
        dict(name="norm_codes_batch", op="norm_codes", dtype="bf16", rows=16384, cols=4096, residual=True, pad=0),
        # gradients of a step's batch in eight partitions, with the residual stream's own gradient
        dict(name="norm_grad_train", op="norm_grad", dtype="bf16", partitions=8, rows=2048, cols=4096, stream=True, pad=0),
        # one sampled token over a large vocabulary, with the alternatives that an answer shows
        dict(name="probs_token", op="probs", dtype="bf16", ids="i64", rows=1, vocab=128000, top=8, masked=0.0, temperature=1.0),
        # scoring a batch of answers
        dict(name="probs_batch", op="probs", dtype="bf16", ids="i64", rows=4096, vocab=32000, top=20, masked=0.02,
             temperature=0.8),
        # gradient through scored tokens and their entropy; an odd vocabulary, rows off every boundary
        dict(name="probs_grad_odd", op="probs_grad", dtype="f32", ids="i64", rows=1024, vocab=50257, masked=0.0, temperature=1.0),
        # one partition against the 16 best alternatives of a teacher
        dict(name="distill_partition", op="distill", dtype="f32", ids="i32", rows=39, vocab=5004, top=16, temperature=1.0,
             grad=True),
        # a training step's logits against the 64 best alternatives of a teacher, loss and gradient
        dict(name="distill_train", op="distill", dtype="bf16", ids="i64", rows=8192, vocab=32000, top=64, temperature=2.0,
             grad=True),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(max(low, high))))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "norm", "norm_codes", "norm_grad", "probs", "probs_grad", "distill"])
    case = dict(op=op, dtype=rng.choice(["f32", "bf16", "f16"]))
    if op in ("embed", "embed_grad"):
        case["ids"], case["pad"] = rng.choice(["i32", "i64"]), rng.choice([0, 0, 0, 8, 3])
        case["width"] = _log_int(rng, 8, 4096)
        if op == "embed":
            case["tokens"] = _log_int(rng, 1, min(65536, 2 ** 26 // case["width"]))
            case["vocab"] = _log_int(rng, 16, min(131072, 2 ** 27 // case["width"]))
            return case
        parts = case["partitions"] = rng.choice([1, 2, 3, 4, 8, 24, 48])
        case["tokens"] = _log_int(rng, 1, min(16384, 2 ** 25 // (case["width"] * parts)))
        case["vocab"] = _log_int(rng, 16, min(131072, 2 ** 26 // (case["width"] * parts)))
        return case
    if op in ("norm", "norm_codes", "norm_grad"):
        case["cols"], case["pad"] = _log_int(rng, 8, 16384), rng.choice([0, 0, 0, 8, 3])
        if op == "norm_grad":
            parts = case["partitions"] = rng.choice([1, 2, 3, 4, 8, 24, 48])
            case["rows"] = _log_int(rng, 1, max(1, min(8192, 2 ** 25 // (case["cols"] * parts))))
            case["stream"] = rng.random() < 0.5
            return case
        case["rows"] = _log_int(rng, 1, min(16384, 2 ** 25 // case["cols"]))
        case["residual"] = rng.random() < 0.7
        return case
    case["ids"] = rng.choice(["i32", "i64"])
    case["vocab"] = _log_int(rng, 64, 262144)
    case["rows"] = _log_int(rng, 1, min(4096, 2 ** 26 // case["vocab"]))
    case["temperature"] = rng.choice([0.7, 1.0, 1.0, 2.0])
    if op == "distill":
        case["top"], case["grad"] = rng.choice([1, 8, 20, 50]), rng.random() < 0.8
        return case
    case["masked"] = rng.choice([0.0, 0.0, 0.02, 0.3])
    if op == "probs":
        case["top"] = rng.choice([0, 1, 5, 20, 32])
    return case


def work(case):
    op, size = case["op"], SIZE[case["dtype"]]
    if op == "embed":
        rows = min(case["tokens"], case["vocab"])   # a row that several tokens name is read once
        return {"bytes": case["tokens"] * (ID_SIZE[case["ids"]] + case["width"] * size) + rows * case["width"] * size,
                "flops": case["tokens"] * case["width"]}
    if op == "embed_grad":
        tokens = case["partitions"] * case["tokens"]
        return {"bytes": tokens * (ID_SIZE[case["ids"]] + case["width"] * size) + 4 * case["partitions"] * case["vocab"] * case["width"],
                "flops": 2 * tokens * case["width"]}
    if op in ("norm", "norm_codes"):
        count = case["rows"] * case["cols"]
        return {"bytes": count * (size * (3 if case["residual"] else 1) + (2 if op == "norm_codes" else size)) + 4 * case["cols"] + 4 * case["rows"],
                "flops": count * (8 if op == "norm_codes" else 5)}
    if op == "norm_grad":
        count = case["partitions"] * case["rows"] * case["cols"]
        return {"bytes": count * size * (4 if case["stream"] else 3) + 4 * case["partitions"] * (case["rows"] + case["cols"]) + 4 * case["cols"],
                "flops": 9 * count}
    count, ids = case["rows"] * case["vocab"], ID_SIZE[case["ids"]]
    if op == "probs":
        return {"bytes": count * size + case["rows"] * (ids + 16 + case["top"] * (4 + ids)), "flops": 6 * count}
    if op == "probs_grad":
        return {"bytes": 2 * count * size + case["rows"] * (ids + 20), "flops": 8 * count}
    return {"bytes": count * size * (2 if case["grad"] else 1) + case["rows"] * (8 + case["top"] * (4 + ids)),
            "flops": count * (8 if case["grad"] else 4)}


# ------------------------------------------------------------------------------------------------ inputs

def _rows_of(values, pad, dtype):
    """`values` (32 bits) rounded to `dtype`, as a view into rows that are `pad` elements longer."""
    if not pad:
        return values.to(dtype)
    wide = torch.zeros(*values.shape[:-1], values.shape[-1] + pad, dtype=dtype, device=values.device)
    wide[..., :values.shape[-1]] = values
    return wide[..., :values.shape[-1]]


def _tokens(g, shape, vocab, dtype, padding):
    """Token numbers whose frequencies fall as 1 / rank, the ranks strewn over the vocabulary; a share of -1 (padding)."""
    u = torch.rand(shape, generator=g, device="cuda", dtype=torch.float64)
    rank = torch.exp(u * math.log(vocab)).long().clamp_(max=vocab) - 1
    step = next(k for k in range(int(vocab * 0.618) + 1, 2 * vocab + 2) if math.gcd(k, vocab) == 1)
    ids = (rank * step + 7) % vocab
    if padding:
        ids = torch.where(torch.rand(shape, generator=g, device="cuda") < padding, -1, ids)
    return ids.to(dtype)


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    op, dtype = case["op"], DTYPES[case["dtype"]]
    s = {"case": case}
    if op == "embed":
        s["table"] = _rows_of(rand(case["vocab"], case["width"]), case["pad"], dtype)
        s["ids"] = _tokens(g, (case["tokens"],), case["vocab"], IDS[case["ids"]], 0.02 if case["tokens"] > 1 else 0.0)
        s["scale"] = math.sqrt(case["width"])
        return s
    if op == "embed_grad":
        shape = (case["partitions"], case["tokens"])
        s["ids"] = _tokens(g, shape, case["vocab"], IDS[case["ids"]], 0.02 if case["tokens"] > 1 else 0.0)
        s["dy"] = _rows_of(rand(*shape, case["width"]), case["pad"], dtype)
        s["scale"] = math.sqrt(case["width"])
        return s
    if op in ("norm", "norm_codes", "norm_grad"):
        shape = (case["partitions"], case["rows"], case["cols"]) if op == "norm_grad" else (case["rows"], case["cols"])
        spread = torch.exp(0.5 * rand(*shape[:-1], 1))      # rows of a residual stream differ in size
        s["gamma"] = 1 + 0.2 * rand(case["cols"])
        if op != "norm_grad":
            s["x"] = _rows_of(rand(*shape), case["pad"], dtype)
            s["residual"] = _rows_of(rand(*shape) * (2 * spread), 0, dtype) if case["residual"] else None
            return s
        s["h"] = _rows_of(rand(*shape) * (2 * spread), case["pad"], dtype)
        s["dy"] = _rows_of(rand(*shape), 0, dtype)
        s["dh"] = _rows_of(rand(*shape), 0, dtype) if case["stream"] else None
        s["rstd"] = (s["h"].double().square().mean(-1) + EPS).rsqrt().float()
        return s
    shape = (case["rows"], case["vocab"])
    # logits of a model that has learned something: a few tokens of each row stand out
    logits = rand(*shape).mul_(2.0)
    if op == "distill":
        top = min(case["top"], case["vocab"])
        s["teacher_ids"] = torch.topk(torch.rand(shape, generator=g, device="cuda"), top, dim=1).indices.to(IDS[case["ids"]])
        s["teacher"] = 6 + 2 * rand(case["rows"], top)
        logits.scatter_add_(1, s["teacher_ids"].long(), s["teacher"] * 0.8 + rand(case["rows"], top))
        left_out = torch.rand(case["rows"], generator=g, device="cuda") < (0.05 if case["rows"] > 1 else 0.0)
        s["teacher_ids"][left_out] = -1                      # rows that are padding have no teacher
        s["weight"] = torch.where(left_out, 0.0, 1 + 0.1 * rand(case["rows"]))
        s["logits"] = logits.to(dtype)
        return s
    s["ids"] = _tokens(g, (case["rows"],), case["vocab"], IDS[case["ids"]], 0.0)
    logits.scatter_add_(1, s["ids"].long()[:, None], 4 + 3 * rand(case["rows"], 1))
    if case["masked"]:
        off = torch.rand(shape, generator=g, device="cuda") < case["masked"]      # tokens that a grammar forbids
        off.scatter_(1, s["ids"].long()[:, None], False)
        off[:, :40] = False
        logits.masked_fill_(off, -math.inf)
    s["logits"] = logits.to(dtype)
    if op == "probs_grad":
        s["dlogp"], s["dentropy"] = rand(case["rows"]), 0.1 * rand(case["rows"])
        # what the forward pass has left: each row's largest logit, the logarithm of the sum relative to it, the entropy
        largest = s["logits"].double().amax(1)
        z = (s["logits"].double() - largest[:, None]) / case["temperature"]
        log_sum = torch.logsumexp(z, 1)
        p = torch.exp(z - log_sum[:, None])
        s["stats"] = torch.stack([largest, log_sum], 1).float()
        s["entropy"] = (log_sum - (p * torch.where(p > 0, z, 0.0)).sum(1)).float()
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


def _scratch(need):
    return torch.empty(need, dtype=torch.uint8, device="cuda") if need else None


def _own_embed(s):
    B, c = s["binding"], s["case"]
    y = torch.empty((c["tokens"], c["width"]), dtype=s["table"].dtype, device="cuda")
    B.cr_embedding(s["plan"], s["ids"], s["table"], y, scale=s["scale"])
    return y


def _own_embed_grad(s):
    B, c = s["binding"], s["case"]
    dtable = torch.empty((c["partitions"], c["vocab"], c["width"]), device="cuda")
    ws = _scratch(B.cr_embedding_backward_workspace_bytes(s["plan"], s["ids"], dtable))
    B.cr_embedding_backward(s["plan"], s["ids"], s["dy"], dtable, scale=s["scale"], workspace=ws)
    return dtable


def _own_norm(s):
    B, x = s["binding"], s["x"]
    y, rstd = torch.empty(x.shape, dtype=x.dtype, device="cuda"), torch.empty(x.shape[0], device="cuda")
    h = None if s["residual"] is None else torch.empty(x.shape, dtype=x.dtype, device="cuda")
    B.cr_rms_norm(s["plan"], x, s["gamma"], y, residual=s["residual"], h=h, rstd=rstd, eps=EPS)
    return {"y": y, "rstd": rstd} if h is None else {"y": y, "rstd": rstd, "h": h}


def _own_norm_codes(s):
    B, x = s["binding"], s["x"]
    q = torch.empty((x.shape[0], (x.shape[1] + 15) // 16 * 16), dtype=torch.int8, device="cuda")[:, :x.shape[1]]
    scale = torch.empty(x.shape[0], device="cuda")
    h = None if s["residual"] is None else torch.empty(x.shape, dtype=x.dtype, device="cuda")
    B.cr_rms_norm_codes(s["plan"], x, s["gamma"], q, scale, residual=s["residual"], h=h, eps=EPS)
    values = torch.empty(x.shape, dtype=torch.bfloat16, device="cuda")
    torch.mul(q, scale[:, None], out=values)      # what the codes stand for
    return {"values": values} if h is None else {"values": values, "h": h}


def _own_norm_grad(s):
    B, c, h = s["binding"], s["case"], s["h"]
    dx = torch.empty(h.shape, dtype=h.dtype, device="cuda")
    dgamma = torch.empty((c["partitions"], c["cols"]), device="cuda")
    ws = _scratch(B.cr_rms_norm_backward_workspace_bytes(s["plan"], h, c["partitions"]))
    B.cr_rms_norm_backward(s["plan"], s["dy"], h, s["gamma"], s["rstd"], dx, dgamma, dh=s["dh"], workspace=ws)
    return {"dx": dx, "dgamma": dgamma}


def _own_probs(s):
    B, c, x = s["binding"], s["case"], s["logits"]
    logp, entropy = torch.empty(c["rows"], device="cuda"), torch.empty(c["rows"], device="cuda")
    stats = torch.empty((c["rows"], 2), device="cuda")
    out = {"logp": logp, "stats": stats, "entropy": entropy}
    if c["top"]:
        out["top_logp"] = torch.empty((c["rows"], c["top"]), device="cuda")
        out["top_ids"] = torch.empty((c["rows"], c["top"]), dtype=s["ids"].dtype, device="cuda")
    B.cr_token_log_probs(s["plan"], x, s["ids"], logp, stats=stats, entropy=entropy, top_logp=out.get("top_logp"),
                         top_ids=out.get("top_ids"), temperature=c["temperature"])
    return out


def _own_probs_grad(s):
    B, x = s["binding"], s["logits"]
    dlogits = torch.empty_like(x)
    B.cr_token_log_probs_backward(s["plan"], x, s["ids"], s["stats"], s["entropy"], s["dlogp"], s["dentropy"],
                                  dlogits, temperature=s["case"]["temperature"])
    return dlogits


def _own_distill(s):
    B, c, x = s["binding"], s["case"], s["logits"]
    loss = torch.empty(c["rows"], device="cuda")
    dlogits = torch.empty_like(x) if c["grad"] else None
    B.cr_distill(s["plan"], x, s["teacher_ids"], s["teacher"], loss, dlogits=dlogits, weight=s["weight"],
                 temperature=c["temperature"])
    return {"loss": loss, "dlogits": dlogits} if c["grad"] else {"loss": loss}


_own = {"embed": _own_embed, "embed_grad": _own_embed_grad, "norm": _own_norm, "norm_codes": _own_norm_codes,
        "norm_grad": _own_norm_grad, "probs": _own_probs, "probs_grad": _own_probs_grad, "distill": _own_distill}


def _plain_embed(s):
    ids = s["ids"].long()
    y = s["table"][ids.clamp(min=0)].float() * s["scale"]
    return torch.where((ids >= 0)[:, None], y, 0.0).to(s["table"].dtype)


def _plain_embed_grad(s):
    c = s["case"]
    ids = s["ids"].long()
    rows = torch.where(ids >= 0, ids, c["vocab"]) + torch.arange(c["partitions"], device="cuda")[:, None] * (c["vocab"] + 1)
    d = torch.zeros((c["partitions"] * (c["vocab"] + 1), c["width"]), device="cuda")     # the last row takes the padding
    d.index_add_(0, rows.view(-1), s["dy"].reshape(-1, c["width"]).float() * s["scale"])
    return d.view(c["partitions"], c["vocab"] + 1, c["width"])[:, :c["vocab"]]


def _plain_sum_and_norm(s):
    h = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
    rstd = 1.0 / torch.sqrt(h.square().mean(1) + EPS)
    return h, rstd, h * rstd[:, None] * s["gamma"]


def _plain_norm(s):
    h, rstd, z = _plain_sum_and_norm(s)
    out = {"y": z.to(s["x"].dtype), "rstd": rstd}
    if s["residual"] is not None:
        out["h"] = h.to(s["x"].dtype)
    return out


def _plain_norm_codes(s):
    h, _, z = _plain_sum_and_norm(s)
    largest = z.abs().amax(1, keepdim=True)
    codes = torch.round(z * (127.0 / largest))
    out = {"values": (codes * (largest / 127.0)).to(torch.bfloat16)}
    if s["residual"] is not None:
        out["h"] = h.to(s["x"].dtype)
    return out


def _plain_norm_grad(s):
    dy, xhat = s["dy"].float(), s["h"].float() * s["rstd"][..., None]
    g = dy * s["gamma"]
    dx = (g - xhat * (g * xhat).mean(-1, keepdim=True)) * s["rstd"][..., None]
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["h"].dtype), "dgamma": (dy * xhat).sum(1)}


def _plain_probs(s):
    c = s["case"]
    x = s["logits"].float()
    largest = x.amax(1, keepdim=True)
    z = (x - largest) * (1.0 / c["temperature"])
    e = torch.exp(z)
    total = e.sum(1)
    log_sum = torch.log(total)
    mean = (e * torch.where(e > 0, z, 0.0)).sum(1) / total
    out = {"logp": z.gather(1, s["ids"].long()[:, None])[:, 0] - log_sum, "entropy": log_sum - mean,
           "stats": torch.stack([largest[:, 0], log_sum], 1)}
    if c["top"]:
        bits = (x + 0.0).view(torch.int32).long()
        order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))     # whole numbers in the values' order
        order = (order << 32) + (0x7FFFFFFF - torch.arange(c["vocab"], device="cuda"))    # equal values: the lowest index first
        best = torch.topk(order, c["top"], dim=1).indices
        out["top_logp"] = z.gather(1, best) - log_sum[:, None]
        out["top_ids"] = best.to(s["ids"].dtype)
    return out


def _plain_probs_grad(s):
    inverse = 1.0 / s["case"]["temperature"]
    log_p = (s["logits"].float() - s["stats"][:, :1]) * inverse - s["stats"][:, 1:]
    p = torch.exp(log_p)
    a, b = s["dlogp"][:, None], s["dentropy"][:, None]
    d = -p * (a + b * (torch.where(p > 0, log_p, 0.0) + s["entropy"][:, None]))
    d.scatter_add_(1, s["ids"].long()[:, None], a)
    return (d * inverse).to(s["logits"].dtype)


def _plain_distill(s):
    t = s["case"]["temperature"]
    z = s["logits"].float() * (1.0 / t)
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    ids = s["teacher_ids"].long()
    there = ids >= 0
    ids = ids.clamp(min=0)
    u = torch.where(there, s["teacher"] * (1.0 / t), -math.inf)
    best = u.amax(1, keepdim=True)
    best = torch.where(best > -math.inf, best, 0.0)
    pe = torch.exp(u - best)
    mass = pe.sum(1, keepdim=True)
    some = mass > 0
    mass = torch.where(some, mass, 1.0)
    p = pe / mass
    terms = p * ((torch.where(there, u, 0.0) - best - torch.log(mass)) - (z.gather(1, ids) - lse))
    out = {"loss": t * t * terms.sum(1)}
    if s["case"]["grad"]:
        d = torch.where(some, e / total, 0.0)
        d.scatter_add_(1, ids, -p)
        out["dlogits"] = (d * (t * s["weight"])[:, None]).to(s["logits"].dtype)
    return out


_plain = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_codes": _plain_norm_codes,
          "norm_grad": _plain_norm_grad, "probs": _plain_probs, "probs_grad": _plain_probs_grad, "distill": _plain_distill}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    return _exact[case["op"]](case, s)


def _exact_embed(case, s):
    wide = torch.cat([s["table"].double(), torch.zeros(1, case["width"], dtype=torch.float64, device="cuda")])    # -1 names the last row
    return torch.nn.functional.embedding(s["ids"].long() % (case["vocab"] + 1), wide) * s["scale"]


def _exact_embed_grad(case, s):
    # the gradient of a lookup, left to automatic differentiation, a partition at a time
    grads = []
    for k in range(case["partitions"]):
        table = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda", requires_grad=True)
        named = s["ids"][k] != -1
        y = torch.nn.functional.embedding(s["ids"][k][named].long(), table) * s["scale"]
        grads.append(torch.autograd.grad(y, table, s["dy"][k][named].double())[0])
    return torch.stack(grads)


def _exact_sum_and_norm(case, s):
    h = s["x"].double() if s["residual"] is None else torch.add(s["x"].double(), s["residual"].double())
    rstd = torch.rsqrt(torch.einsum("rc,rc->r", h, h) / case["cols"] + EPS)
    return h, rstd, torch.einsum("rc,r,c->rc", h, rstd, s["gamma"].double())


def _exact_norm(case, s):
    h, rstd, z = _exact_sum_and_norm(case, s)
    return {"y": z, "rstd": rstd} if s["residual"] is None else {"y": z, "rstd": rstd, "h": h}


def _exact_norm_codes(case, s):
    h, _, z = _exact_sum_and_norm(case, s)
    step = torch.linalg.vector_norm(z, ord=math.inf, dim=1, keepdim=True) / 127
    values = torch.round(z / step) * step
    return {"values": values} if s["residual"] is None else {"values": values, "h": h}


def _exact_norm_grad(case, s):
    # rstd is an input, but its dependence on the row is the operator's: differentiate h / sqrt(mean h^2 + eps)
    h = s["h"].double().requires_grad_(True)
    gamma = s["gamma"].double().expand(case["partitions"], -1).clone().requires_grad_(True)
    y = torch.nn.functional.rms_norm(h, (case["cols"],), eps=EPS) * gamma[:, None, :]
    dx, dgamma = torch.autograd.grad(y, (h, gamma), s["dy"].double())
    return {"dx": dx if s["dh"] is None else dx + s["dh"].double(), "dgamma": dgamma}


def _exact_probs(case, s):
    z = s["logits"].double() / case["temperature"]
    log_p = torch.log_softmax(z, 1)
    largest, where = s["logits"].double().max(1)
    out = {"logp": log_p.gather(1, s["ids"].long()[:, None]).squeeze(1),
           "stats": torch.stack([largest, -log_p.gather(1, where[:, None]).squeeze(1)], 1), "entropy": torch.special.entr(torch.softmax(z, 1)).sum(1)}
    if case["top"]:
        values, ids = torch.sort(s["logits"].double(), dim=1, descending=True, stable=True)
        out["top_ids"] = ids[:, :case["top"]].to(s["ids"].dtype)
        out["top_logp"] = log_p.gather(1, ids[:, :case["top"]])
    return out


def _exact_probs_grad(case, s):
    x = s["logits"].double().requires_grad_(True)
    log_p = torch.log_softmax(x / case["temperature"], 1)
    entropy = -(log_p.exp() * torch.where(log_p > -math.inf, log_p, 0.0)).sum(1)
    logp = log_p.gather(1, s["ids"].long()[:, None]).squeeze(1)
    return torch.autograd.grad((logp, entropy), x, (s["dlogp"].double(), s["dentropy"].double()))[0]


def _exact_distill(case, s):
    t = case["temperature"]
    x = s["logits"].double().requires_grad_(case["grad"])
    with torch.no_grad():
        there = s["teacher_ids"] >= 0
        kept = there.any(1)
        log_p = torch.log_softmax(torch.where(there | ~kept[:, None], s["teacher"].double(), -math.inf) / t, 1)
        p = torch.where(there, log_p.exp(), 0.0)
    log_q = torch.log_softmax(x / t, 1).gather(1, s["teacher_ids"].long().clamp(min=0))
    loss = t * t * (torch.special.xlogy(p, p) - p * log_q).sum(1)
    if not case["grad"]:
        return {"loss": loss}
    return {"loss": loss.detach(), "dlogits": torch.autograd.grad(loss, x, s["weight"].double())[0]}


_exact = {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "norm": _exact_norm, "norm_codes": _exact_norm_codes,
          "norm_grad": _exact_norm_grad, "probs": _exact_probs, "probs_grad": _exact_probs_grad, "distill": _exact_distill}
