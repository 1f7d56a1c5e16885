"""The operators at both ends of a network over a vocabulary and the norm between its layers, as measurable cases.

Three operators: the embedding lookup with scaling and its gradient by sorted tokens, layer norm forward and backward with the sums of its weight's
gradient, and the softmax cross-entropy of a last layer's product without its logits in memory, with its gradients.  `op` says which call a case makes; the
other fields are shapes, types and options.

With `own` false, run() computes an operator from elementary torch operations in float32, rounded once at the end; with `own` true it
calls the framework's operators.  exact() computes the same from the definitions in float64.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
IGNORE = -100


def _embedding(name, op, rows, vocab, width, dtype, **kw):
    case = {"name": name, "op": op, "rows": rows, "vocab": vocab, "width": width, "dtype": dtype, "tokens": "i64", "scale": 1.0, "ignored": 0.0, "pad": 0}
    case.update(kw)
    return case


def _norm(name, op, rows, width, dtype, **kw):
    case = {"name": name, "op": op, "rows": rows, "width": width, "dtype": dtype, "pad": 0}
    case.update({"keep": False} if op == "layer_norm_forward" else {"residual": False})
    case.update(kw)
    return case


def _loss(name, rows, k, classes, dtype, **kw):
    case = {"name": name, "op": "linear_cross_entropy", "rows": rows, "in": k, "classes": classes, "dtype": dtype, "grads": True, "bias": True, "smoothing": 0.0,
            "ignored": 0.0, "masked": 0.0, "pad": 0}
    case.update(kw)
    return case


def listed():
    return [
        # One token on its way into a network that answers: a launch.
        _embedding("embed_one_token", "embedding_forward", 1, 50001, 4096, "bf16"),
        # The tokens of a large training batch, scaled by the root of the width.
        _embedding("embed_batch", "embedding_forward", 32768, 50001, 2048, "bf16", scale=math.sqrt(2048.0), ignored=0.05),
        # The gradient of a small table, float32, odd sizes, rows of a wider table, 32-bit tokens.
        _embedding("embed_grad_small_f32", "embedding_backward", 257, 1001, 301, "f32", tokens="i32", pad=3),
        # The gradient of the large batch: tokens as text has them, a few very often and most of the table never.
        _embedding("embed_grad_batch", "embedding_backward", 32768, 50001, 2048, "bf16", scale=math.sqrt(2048.0), ignored=0.05),
        # One row between two layers of a network that answers: a launch.
        _norm("norm_one_row", "layer_norm_forward", 1, 4096, "bf16"),
        # The same network on a large training batch, statistics kept.
        _norm("norm_batch", "layer_norm_forward", 16384, 4096, "bf16", keep=True),
        # The odd width of 617-301-150-26 (24 workers of 100 rows) backwards, float32, rows of a wider table.
        _norm("norm_grad_617_f32", "layer_norm_backward", 2400, 617, "f32", pad=3),
        # The large batch backwards, with the gradient that comes around the layer added on the way out.
        _norm("norm_grad_batch", "layer_norm_backward", 16384, 4096, "bf16", residual=True),
        # How likely an answer of 64 tokens is: the loss alone, a read of the weights.
        _loss("loss_of_64_rows", 64, 1024, 50001, "bf16", grads=False),
        # A small vocabulary trained in float32 on ten workers' 12 rows.
        _loss("loss_120_rows_f32", 120, 500, 1001, "f32", smoothing=0.1, ignored=0.1),
        # A training batch over a vocabulary of odd size: smoothed labels, padding positions, classes ruled out by their bias.
        _loss("loss_50001_classes", 4096, 1024, 50001, "bf16", smoothing=0.1, ignored=0.15, masked=0.02),
        # A wide network on a large batch and a large vocabulary: three products of 4.4e12 operations each.
        _loss("loss_65536_classes", 8192, 4096, 65536, "bf16", bias=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges: one row to many, narrow tables to wide ones, a few classes to a large vocabulary."""
    op = rng.choice(["embedding_forward", "embedding_backward", "layer_norm_forward", "layer_norm_backward", "linear_cross_entropy", "linear_cross_entropy"])
    dtype, pad = rng.choice(["bf16", "bf16", "f32"]), rng.choice([0, 0, 0, 8, 3])
    if op.startswith("embedding"):
        rows, vocab, width = _log(rng, 1, 131072), _log(rng, 2, 131072), _log(rng, 8, 8192)
        if rng.random() < 0.5:          # widths as networks have them, mostly
            width = max(8, width // 16 * 16)
        while rows * width > 1.3e8 or vocab * width > 1.3e8:
            rows, vocab, width = max(1, rows * 2 // 3), max(2, vocab * 3 // 4), max(8, width * 4 // 5)
        case = _embedding("", op, rows, vocab, width, dtype, tokens=rng.choice(["i64", "i64", "i32"]), scale=rng.choice([1.0, math.sqrt(width)]),
                          ignored=rng.choice([0.0, 0.0, 0.05, 0.5]), pad=pad)
    elif op.startswith("layer_norm"):
        rows, width = _log(rng, 1, 65536), _log(rng, 8, 16384)
        if rng.random() < 0.5:
            width = max(8, width // 16 * 16)
        while rows * width > 1.3e8:
            rows = max(1, rows * 2 // 3)
        case = _norm("", op, rows, width, dtype, pad=pad)
        key = "keep" if op == "layer_norm_forward" else "residual"
        case[key] = rng.random() < 0.5
    else:
        rows, k, classes = _log(rng, 1, 8192), _log(rng, 16, 4096), _log(rng, 2, 131072)
        if rng.random() < 0.5:
            k, classes = max(16, k // 16 * 16), max(16, classes // 16 * 16)
        most = 1.3e13 if dtype == "bf16" else 4e11
        while 6.0 * rows * k * classes > most or rows * classes > 5.3e8:
            rows, k, classes = max(1, rows * 2 // 3), max(16, k * 3 // 4), max(2, classes * 3 // 4)
        case = _loss("", rows, k, classes, dtype, grads=rng.random() < 0.75, bias=rng.random() < 0.7, smoothing=rng.choice([0.0, 0.0, 0.1]),
                     ignored=rng.choice([0.0, 0.1, 0.5]), pad=pad)
        if case["bias"]:
            case["masked"] = rng.choice([0.0, 0.0, 0.05, 0.5])
    del case["name"]
    return case


# ---- inputs ----

def _table(gen, rows, cols, pad, dtype, scale=1.0):
    """Normal values; with `pad`, rows of a wider table."""
    t = scale * torch.randn(rows, cols + pad, generator=gen, device=gen.device)
    return t.to(dtype)[:, :cols]


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device=gen.device)


def _frequent_first(gen, rows, vocab):
    """Tokens as text has them: the n-th most frequent about n times rarer than the first, in an order that is not the table's."""
    at = torch.clamp(torch.exp(_uniform(gen, rows).double() * math.log(vocab + 1.0)).long() - 1, 0, vocab - 1)
    return torch.randperm(vocab, generator=gen, device=gen.device)[at]


def _prepare_embedding(case, gen):
    dt, rows, vocab, width = TYPES[case["dtype"]], case["rows"], case["vocab"], case["width"]
    tokens = _frequent_first(gen, rows, vocab)
    tokens = tokens.masked_fill(_uniform(gen, rows) < case["ignored"], IGNORE).to(TYPES[case["tokens"]])
    state = {"tokens": tokens, "scale": case["scale"], "vocab": vocab}
    if case["op"] == "embedding_forward":
        state["w"] = _table(gen, vocab, width, case["pad"], dt, 1.0 / math.sqrt(width))
    else:
        state["dy"] = _table(gen, rows, width, case["pad"], dt, 1.0 / rows)
    return state


def _prepare_norm(case, gen):
    dt, rows, width, dev = TYPES[case["dtype"]], case["rows"], case["width"], gen.device
    x = torch.randn(rows, width + case["pad"], generator=gen, device=dev) * (0.5 + 2.0 * _uniform(gen, rows, 1))     # rows and columns differ in scale and place
    x = (x + 0.5 * torch.randn(width + case["pad"], generator=gen, device=dev) + 0.3).to(dt)[:, :width]
    state = {"x": x, "weight": (1.0 + 0.2 * torch.randn(width, generator=gen, device=dev)).to(dt), "eps": 1e-5}
    if case["op"] == "layer_norm_forward":
        state["bias"], state["keep"] = (0.1 * torch.randn(width, generator=gen, device=dev)).to(dt), case["keep"]
    else:
        state["mean"] = x.double().mean(1).float()
        state["rstd"] = (1.0 / torch.sqrt((x.double() - x.double().mean(1, keepdim=True)).square().mean(1) + state["eps"])).float()
        state["dy"] = _table(gen, rows, width, case["pad"], dt, 1.0 / rows)
        state["residual"] = _table(gen, rows, width, case["pad"], dt, 1.0 / rows) if case["residual"] else None
    return state


def _prepare_loss(case, gen):
    dt, rows, k, classes, dev = TYPES[case["dtype"]], case["rows"], case["in"], case["classes"], gen.device
    w = ((2 * _uniform(gen, k, classes + case["pad"]) - 1) * math.sqrt(3.0 / k)).to(dt)[:, :classes]
    out = _uniform(gen, classes) < case["masked"]
    out[0] = False
    left = torch.nonzero(~out)[:, 0]
    labels = left[torch.randint(left.numel(), (rows,), generator=gen, device=dev)]
    x = torch.randn(rows, k, generator=gen, device=dev) + 4.0 * _uniform(gen, rows, 1) * w[:, labels].float().t()       # a network that has learned something
    wide = torch.zeros(rows, k + case["pad"], dtype=dt, device=dev)
    wide[:, :k] = x
    bias = None
    if case["bias"]:
        bias = (0.1 * torch.randn(classes, generator=gen, device=dev)).masked_fill(out, -math.inf).to(dt)
    return {"x": wide[:, :k], "w": w, "bias": bias, "labels": labels.masked_fill(_uniform(gen, rows) < case["ignored"], IGNORE),
            "smoothing": case["smoothing"], "grads": case["grads"]}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    state = _prepare_embedding(case, gen) if op.startswith("embedding") else _prepare_norm(case, gen) if op.startswith("layer_norm") else _prepare_loss(case, gen)
    state["op"] = op
    return state


# ---- plain forms ----

def _embedding_forward_plain(s):
    known = s["tokens"] != IGNORE
    rows = s["w"][torch.where(known, s["tokens"], 0).long()].float() * s["scale"]
    return (torch.where(known[:, None], rows, 0.0).to(s["w"].dtype),)


def _embedding_backward_plain(s):
    known, dy = s["tokens"] != IGNORE, s["dy"]
    dw = torch.zeros(s["vocab"], dy.shape[1], device=dy.device)
    dw.index_add_(0, torch.where(known, s["tokens"], 0).long(), torch.where(known[:, None], dy.float(), 0.0))
    return ((dw * s["scale"]).to(dy.dtype),)


def _norm_forward_plain(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + s["eps"])
    y = (x - mean) * rstd * s["weight"].float() + s["bias"].float()
    return (y.to(s["x"].dtype),) + ((mean[:, 0], rstd[:, 0]) if s["keep"] else ())


def _norm_backward_plain(s):
    dy, dt = s["dy"].float(), s["x"].dtype
    normed = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"].float()
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - normed * (g * normed).mean(1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return dx.to(dt), (dy * normed).sum(0).to(dt), dy.sum(0).to(dt)


def _loss_plain(s):
    """Classes whose logit is -inf are ruled out; smoothing goes to the classes that are left."""
    x, w, labels, eps = s["x"].float(), s["w"].float(), s["labels"], s["smoothing"]
    dt = s["x"].dtype
    z = x @ w
    if s["bias"] is not None:
        z = z + s["bias"].float()
    valid = labels != IGNORE
    count = torch.clamp(valid.sum(), min=1).float()
    at = torch.where(valid, labels, 0)[:, None]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    left = z > -math.inf
    n_left = left.sum(1).float()
    rows = (top + torch.log(total))[:, 0] - (1.0 - eps) * z.gather(1, at)[:, 0]
    if eps:
        rows = rows - eps * torch.where(left, z, 0.0).sum(1) / n_left
    rows = torch.where(valid, rows, 0.0)
    out = (rows.sum() / count, rows)
    if not s["grads"]:
        return out
    grad = e / total
    if eps:
        grad = grad - torch.where(left, eps / n_left[:, None], 0.0)
    grad.scatter_add_(1, at, torch.full_like(at, -(1.0 - eps), dtype=torch.float32))
    grad = torch.where(valid[:, None], grad / count, 0.0)
    out += ((grad @ w.t()).to(dt), (x.t() @ grad).to(dt))
    return out + ((grad.sum(0).to(dt),) if s["bias"] is not None else ())


def run(state):
    op = state["op"]
    if not own:
        return {"embedding_forward": _embedding_forward_plain, "embedding_backward": _embedding_backward_plain, "layer_norm_forward": _norm_forward_plain,
                "layer_norm_backward": _norm_backward_plain, "linear_cross_entropy": _loss_plain}[op](state)
    from paper_2012_15469_amd import ops
    if op == "embedding_forward":
        out = (ops.embedding_forward(state["tokens"], state["w"], scale=state["scale"], ignore_index=IGNORE),)
    elif op == "embedding_backward":
        out = (ops.embedding_backward(state["dy"], state["tokens"], state["vocab"], scale=state["scale"], ignore_index=IGNORE),)
    elif op == "layer_norm_forward":
        out = ops.layer_norm_forward(state["x"], state["weight"], state["bias"], eps=state["eps"], keep_stats=state["keep"])
    elif op == "layer_norm_backward":
        out = ops.layer_norm_backward(state["dy"], state["x"], state["mean"], state["rstd"], state["weight"], residual=state["residual"])
    else:
        grads = state["grads"]
        out = ops.linear_cross_entropy(state["x"], state["w"], state["labels"], state["bias"], smoothing=state["smoothing"], ignore_index=IGNORE,
                                       need_dx=grads, need_dw=grads, need_db=grads and state["bias"] is not None)
    return tuple(t for t in out if t is not None)


# ---- work ----

def work(case):
    """Each input read once, each output written once.  (A lookup reads a row of the table per token at most, and no more than the table.)"""
    width = 2 if case["dtype"] == "bf16" else 4
    rows = float(case["rows"])
    if case["op"].startswith("embedding"):
        cols, token = case["width"], 4 if case["tokens"] == "i32" else 8
        other = min(rows, case["vocab"]) if case["op"] == "embedding_forward" else case["vocab"]
        return {"bytes": token * rows + width * cols * (rows + other), "flops": rows * cols}
    if case["op"] == "layer_norm_forward":
        return {"bytes": width * (2 * rows + 2) * case["width"] + (8 * rows if case["keep"] else 0), "flops": 8.0 * rows * case["width"]}
    if case["op"] == "layer_norm_backward":
        return {"bytes": width * ((3 + case["residual"]) * rows + 3) * case["width"] + 8 * rows, "flops": 14.0 * rows * case["width"]}
    k, classes = case["in"], float(case["classes"])
    tables = rows * k + k * classes + (classes if case["bias"] else 0)
    return {"bytes": width * tables * (2 if case["grads"] else 1) + 12 * rows, "flops": (6.0 if case["grads"] else 2.0) * rows * k * classes}


# ---- from the definitions, in 64 bits ----

def _exact_embedding(case, s):
    used = torch.nonzero(s["tokens"] != IGNORE)[:, 0]
    tokens = s["tokens"].long()[used]
    if case["op"] == "embedding_forward":
        y = torch.zeros(case["rows"], case["width"], dtype=torch.float64, device=used.device)
        y[used] = s["w"].double()[tokens] * case["scale"]
        return (y,)
    dw = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device=used.device)
    for part in used.split(16384):
        dw.index_put_((s["tokens"].long()[part],), case["scale"] * s["dy"][part].double(), accumulate=True)
    return (dw,)


def _exact_norm(case, s):
    if case["op"] == "layer_norm_forward":
        y, means, rstds = [], [], []
        for x in s["x"].split(4096):
            var, mean = torch.var_mean(x.double(), 1, correction=0, keepdim=True)
            rstd = torch.rsqrt(var + s["eps"])
            y.append(torch.addcmul(s["bias"].double(), (x.double() - mean) * rstd, s["weight"].double()))
            means.append(mean[:, 0])
            rstds.append(rstd[:, 0])
        return (torch.cat(y),) + ((torch.cat(means), torch.cat(rstds)) if case["keep"] else ())
    dxs, dw, db = [], 0.0, 0.0
    for at in torch.arange(case["rows"], device=s["x"].device).split(4096):
        x, dy, rstd = s["x"][at].double(), s["dy"][at].double(), s["rstd"][at, None].double()
        u = (x - s["mean"][at, None].double()) * rstd
        dw, db = dw + torch.einsum("ij,ij->j", dy, u), db + dy.sum(0)
        g = dy * s["weight"].double()
        along, mean = (g * u).sum(1, keepdim=True) / case["width"], g.sum(1, keepdim=True) / case["width"]
        dx = (g - mean - u * along) * rstd
        dxs.append(dx + s["residual"][at].double() if case["residual"] else dx)
    return torch.cat(dxs), dw, db


def _exact_loss(case, s):
    labels, eps, w = s["labels"], s["smoothing"], s["w"].double()
    count = max(1, int((labels != IGNORE).sum()))
    losses, dxs, dw, db = [], [], 0.0, 0.0
    for x, y in zip(s["x"].split(512), labels.split(512)):          # (a few rows at a time: 64 bits of a large vocabulary)
        x = x.double()
        z = torch.mm(x, w)
        if case["bias"]:
            z += s["bias"].double()
        logp = z - torch.logsumexp(z, 1, keepdim=True)
        target = torch.zeros_like(z).scatter_(1, y.clamp(min=0)[:, None], 1.0 - eps)
        if eps:
            left = (~torch.isinf(z)).double()
            target += eps * left / left.sum(1, keepdim=True)
        used = (y != IGNORE).double()
        losses.append(-torch.where(target > 0, target * logp, 0.0).sum(1) * used)
        if case["grads"]:
            g = (torch.exp(logp) - target) * used[:, None] / count
            dxs.append(torch.mm(g, w.t()))
            dw, db = dw + torch.mm(x.t(), g), db + g.sum(0)
    losses = torch.cat(losses)
    out = (losses.sum() / count, losses)
    if not case["grads"]:
        return out
    return out + (torch.cat(dxs), dw) + ((db,) if case["bias"] else ())


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"].startswith("embedding"):
        return _exact_embedding(case, state)
    return _exact_norm(case, state) if case["op"].startswith("layer_norm") else _exact_loss(case, state)
