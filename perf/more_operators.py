"""Performance cases of the operators at the two ends of a language model: the
embedding lookup and its gradient, the layer norm, the softmax cross entropy over
a vocabulary from the last hidden states, and the distillation from a teacher's
top logits, each with its gradients.

A pass is one call, or a forward and a backward call, as a program makes it, on
tensors that it has in hand. The plain forms are elementary torch operations in
32 bits that keep every logit.
"""
import math

import torch

own = False

EPS = 1e-5
IGNORE = -100
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _norm(name, rows, width, prec, residual, form):
    return dict(name=name, op="norm", rows=rows, width=width, prec=prec, residual=residual, form=form)


def _embed(name, tokens, vocab, width, prec, form, padding=False):
    return dict(name=name, op="embed", tokens=tokens, vocab=vocab, width=width, prec=prec, form=form, padding=padding)


def _loss(name, rows, width, vocab, prec, form, ignored=0.0):
    return dict(name=name, op="loss", rows=rows, width=width, vocab=vocab, prec=prec, form=form, ignored=ignored)


def _distill(name, rows, width, vocab, top, prec, form, temperature=1.0, ignored=0.0):
    return dict(name=name, op="distill", rows=rows, width=width, vocab=vocab, top=top, prec=prec, form=form, temperature=temperature,
                ignored=ignored)


def listed():
    return [
        # one token of a small model being decoded: latency only
        _norm("layer_norm_token_bf16", 1, 1024, "bf16", True, "plain"),
        # fp32 training at sizes that fill no vector, tile or wave
        _norm("layer_norm_train_f32_odd", 2053, 771, "f32", False, "train"),
        # a training batch of 32 sequences of 1024 tokens, with the residual's gradient
        _norm("layer_norm_train_bf16", 32768, 2048, "bf16", True, "train"),
        # the next token of 64 sequences: latency
        _embed("embed_token_bf16", 64, 32768, 1024, "bf16", "plain"),
        # a small fp32 model's padded batch: odd sizes, tokens that repeat a lot
        _embed("embed_train_f32_odd", 5003, 10007, 333, "f32", "train", padding=True),
        # a training batch into a large table
        _embed("embed_train_bf16", 32768, 131072, 2048, "bf16", "train"),
        # scoring the next token of 32 sequences: the head's weights have to be read
        _loss("loss_score_bf16", 32, 1024, 32768, "bf16", "plain"),
        # a small fp32 model, prompts left out of the loss: odd sizes everywhere
        _loss("loss_train_f32_odd", 777, 500, 10007, "f32", "train", ignored=0.4),
        # a small model's training batch
        _loss("loss_train_bf16", 2048, 1024, 32768, "bf16", "train"),
        # a large vocabulary's: the logits alone would be 4 GB in 32 bits
        _loss("loss_train_bf16_large", 8192, 2048, 131072, "bf16", "train"),
        # a small fp32 student, a few of the teacher's logits, some rows left out
        _distill("distill_train_f32_odd", 401, 260, 5003, 10, "f32", "train", temperature=2.0, ignored=0.2),
        # a training batch of a bf16 student
        _distill("distill_train_bf16", 4096, 2048, 65536, 32, "bf16", "train", temperature=2.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    w = _log(rng, lo, hi)
    return max(lo, w // 8 * 8) if rng.random() < 0.6 else w


def draw(rng):
    op = rng.choice(("norm", "embed", "loss", "distill"))
    prec = rng.choice(("f32", "bf16"))
    form = rng.choice(("plain", "train"))
    if op == "norm":
        while True:
            rows, width = _log(rng, 1, 40000), _width(rng, 8, 16384)
            if rows * width <= 32768 * 2048:
                return dict(op=op, rows=rows, width=width, prec=prec, residual=rng.random() < 0.5, form=form)
    if op == "embed":
        while True:
            tokens, vocab, width = _log(rng, 1, 65536), _log(rng, 50, 200000), _width(rng, 8, 8192)
            if tokens * width <= 32768 * 2048 and vocab * width <= 131072 * 2048 // (1 if prec == "bf16" else 2):
                return dict(op=op, tokens=tokens, vocab=vocab, width=width, prec=prec, form=form, padding=rng.random() < 0.3)
    most = 8192 * 2048 * 131072 // (1 if prec == "bf16" else 16)
    while True:
        rows, width, vocab = _log(rng, 1, 8192), _width(rng, 32, 4096), _log(rng, 100, 131072)
        if rows * width * vocab <= most:
            break
    ignored = rng.choice((0.0, 0.0, 0.3, 0.7))
    if op == "loss":
        return dict(op=op, rows=rows, width=width, vocab=vocab, prec=prec, form=form, ignored=ignored)
    return dict(op=op, rows=rows, width=width, vocab=vocab, top=min(_log(rng, 1, 64), vocab), prec=prec, form=form,
                temperature=rng.choice((1.0, 2.0, 4.0)), ignored=ignored)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 11)
    return g


def _normal(g, shape, dtype=torch.float32, mean=0.0, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)


def _uniform(g, shape):
    return torch.rand(shape, generator=g, device="cuda")


def _tokens(g, n, vocab):
    """Tokens as text has them: the frequency of the k-th is about 1 / k."""
    return (torch.exp(_uniform(g, (n,)).double() * math.log(vocab + 1.0)) - 1).long().clamp_(0, vocab - 1)


def _left_out(case):
    return int(case["rows"] * case["ignored"])


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case=case)
    t = TYPES[case["prec"]]
    if case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        st["x"] = _normal(g, (rows, width), t, mean=0.5)
        st["r"] = _normal(g, (rows, width), t, std=3.0) if case["residual"] else None
        st["w"], st["b"] = _normal(g, (width,), mean=1.0, std=0.2), _normal(g, (width,), std=0.2)
        if case["form"] == "train":
            st["dy"] = _normal(g, (rows, width), t)
            st["ds"] = _normal(g, (rows, width), t) if case["residual"] else None
        return st
    if case["op"] == "embed":
        n, vocab, width = case["tokens"], case["vocab"], case["width"]
        st["w"] = _normal(g, (vocab, width), t, std=0.02)
        st["tokens"] = _tokens(g, n, vocab)
        st["scale"] = math.sqrt(width)
        st["padding"] = None
        if case["padding"]:
            st["padding"] = vocab - 1
            st["tokens"][_uniform(g, (n,)) < 0.2] = vocab - 1
        if case["form"] == "train":
            st["dy"] = _normal(g, (n, width), t, std=1e-2)
        return st
    rows, width, vocab = case["rows"], case["width"], case["vocab"]
    st["w"] = _normal(g, (vocab, width), t, std=2.0 / math.sqrt(width))
    out = torch.randperm(rows, generator=g, device="cuda")[:_left_out(case)]
    if case["op"] == "loss":
        first = st["targets"] = _tokens(g, rows, vocab)
        # hidden states that know their target more or less
        x = _normal(g, (rows, width)) + 2.5 * _uniform(g, (rows, 1)) * st["w"][first].float()
        st["targets"][out] = IGNORE
    else:
        k = case["top"]
        start, step = _tokens(g, rows, vocab), (_uniform(g, (rows,)) * max(1, vocab // k)).long().clamp_(1, max(1, vocab // k))
        ids = (start[:, None] + step[:, None] * torch.arange(k, device="cuda")) % vocab
        x = _normal(g, (rows, width)) + 2.5 * _uniform(g, (rows, 1)) * st["w"][ids[:, 0]].float()
        st["logits"] = _normal(g, (rows, k), std=3.0).sort(1, descending=True).values.to(t)
        if k > 2:  # a few rows with fewer entries
            short = _uniform(g, (rows, 1)) < 0.1
            ids = torch.where(short & (torch.arange(k, device="cuda") >= (k + 1) // 2), -1, ids)
        ids[out] = -1
        st["ids"], st["T"] = ids.int(), case["temperature"]
    st["x"] = x.to(t)
    if case["form"] == "train":  # a mean's share, and the rows' own weights
        st["dloss"] = (0.5 + _uniform(g, (rows,))) / max(1, rows - _left_out(case))
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(st):
    return {"norm": _run_norm, "embed": _run_embed, "loss": _run_loss, "distill": _run_distill}[st["case"]["op"]](st)


def _run_norm(st):
    train = st["case"]["form"] == "train"
    if own:
        from paper_2408_01331_amd import operators as ops
        y, s, stats = ops.layer_norm(st["x"], st["w"], st["b"], residual=st["r"], eps=EPS, keep=train)
        if not train:
            return dict(y=y, s=s)
        dx, dw, db = ops.layer_norm_backward(st["dy"], s, st["w"], stats, ds=st["ds"])
        return dict(y=y, s=s, dx=dx, dw=dw, db=db)
    x, w, b, t = st["x"], st["w"], st["b"], st["x"].dtype
    s = x if st["r"] is None else (x.float() + st["r"].float()).to(t)
    c = s.float()
    c = c - c.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    xhat = c * rstd
    y = (xhat * w + b).to(t)
    if not train:
        return dict(y=y, s=s)
    dy = st["dy"].float()
    dyw = dy * w
    dx = rstd * (dyw - dyw.mean(1, keepdim=True) - xhat * (dyw * xhat).mean(1, keepdim=True))
    if st["ds"] is not None:
        dx = dx + st["ds"].float()
    return dict(y=y, s=s, dx=dx.to(t), dw=(dy * xhat).sum(0), db=dy.sum(0))


def _run_embed(st):
    case, tokens, w, scale, padding = st["case"], st["tokens"], st["w"], st["scale"], st["padding"]
    if own:
        from paper_2408_01331_amd import operators as ops
        y = ops.embedding(tokens, w, scale=scale)
        if case["form"] == "plain":
            return dict(y=y)
        return dict(y=y, dw=ops.embedding_backward(st["dy"], tokens, case["vocab"], scale=scale, padding=padding))
    y = (w[tokens].float() * scale).to(w.dtype)
    if case["form"] == "plain":
        return dict(y=y)
    dy = st["dy"].float()
    if padding is not None:
        dy = torch.where((tokens == padding)[:, None], 0.0, dy)
    # (in 64 bits: the frequent tokens' sums are long, and their order changes from pass to pass)
    dw = torch.zeros(w.shape, dtype=torch.float64, device=w.device).index_add_(0, tokens, dy.double())
    return dict(y=y, dw=(dw * scale).to(w.dtype))


def _run_loss(st):
    case, x, w, targets = st["case"], st["x"], st["w"], st["targets"]
    train = case["form"] == "train"
    if own:
        from paper_2408_01331_amd import operators as ops
        loss, lse = ops.vocab_loss(x, w, targets, ignore=IGNORE)
        if not train:
            return dict(loss=loss, lse=lse)
        dx, dw = ops.vocab_loss_backward(x, w, targets, lse, st["dloss"], ignore=IGNORE)
        return dict(loss=loss, lse=lse, dx=dx, dw=dw)
    t, x, w = x.dtype, x.float(), w.float()
    live = targets != IGNORE
    at = torch.where(live, targets, 0)[:, None]
    z = x @ w.t()
    top = z.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    loss = torch.where(live, (lse - z.gather(1, at))[:, 0], 0.0)
    shown = torch.where(live, lse[:, 0], 0.0)
    if not train:
        return dict(loss=loss, lse=shown)
    each = torch.where(live, st["dloss"], 0.0)[:, None]
    g = torch.exp(z - lse)
    g.scatter_add_(1, at, torch.full_like(lse, -1.0))
    g = g * each
    return dict(loss=loss, lse=shown, dx=(g @ w).to(t), dw=(g.t() @ x).to(t))


def _run_distill(st):
    case, x, w, ids, logits, T = st["case"], st["x"], st["w"], st["ids"], st["logits"], st["T"]
    train = case["form"] == "train"
    if own:
        from paper_2408_01331_amd import operators as ops
        loss, lse, picked = ops.distill_loss(x, w, ids, logits, temperature=T)
        if not train:
            return dict(loss=loss, lse=lse)
        dx, dw = ops.distill_loss_backward(x, w, ids, logits, lse, picked, st["dloss"], temperature=T)
        return dict(loss=loss, lse=lse, dx=dx, dw=dw)
    t, x, w = x.dtype, x.float(), w.float()
    there = ids >= 0
    live = there.any(1)
    at = torch.where(there, ids, 0).long()
    u = torch.where(there, logits.float() / T, -math.inf)
    u = u - torch.where(live, u.amax(1), 0.0)[:, None]
    e = torch.exp(u)
    total = torch.where(live, e.sum(1), 1.0)[:, None]
    p, logp = e / total, torch.where(there, u, 0.0) - torch.log(total)
    z = (x @ w.t()) / T
    top = z.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    loss = torch.where(live, T * T * (p * (logp - z.gather(1, at) + lse)).sum(1), 0.0)
    shown = torch.where(live, lse[:, 0], 0.0)
    if not train:
        return dict(loss=loss, lse=shown)
    g = torch.exp(z - lse)
    g.scatter_add_(1, at, -p)
    g = g * torch.where(live, T * st["dloss"], 0.0)[:, None]
    return dict(loss=loss, lse=shown, dx=(g @ w).to(t), dw=(g.t() @ x).to(t))


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    b, train = SIZE[case["prec"]], case["form"] == "train"
    if case["op"] == "norm":
        n, rows, width, r = case["rows"] * case["width"], case["rows"], case["width"], case["residual"]
        size, flops = n * b * (4 if r else 2) + 8 * width, 8 * n   # x (and the residual in, their sum out), y; weight and bias
        if train:  # dy, the sum (again), its gradient, dx; the weight and the two gradients
            size += n * b * (4 if r else 3) + 12 * width
            flops += 13 * n
        return {"bytes": size, "flops": flops}
    if case["op"] == "embed":
        n, width, vocab = case["tokens"], case["width"], case["vocab"]
        size, flops = 2 * n * width * b + 8 * n, n * width
        if train:
            size += (n + vocab) * width * b + 8 * n
            flops += n * width + vocab * width
        return {"bytes": size, "flops": flops}
    rows, width, vocab = case["rows"] - _left_out(case), case["width"], case["vocab"]
    size, flops = (rows + vocab) * width * b + 16 * rows, 2 * rows * width * vocab + 4 * rows * vocab
    if case["op"] == "distill":
        size += rows * case["top"] * (4 + b)
    if train:  # the hidden states and the weights again, and the gradients of both
        size += (rows + case["rows"] + 2 * vocab) * width * b + 8 * rows
        flops += 4 * rows * width * vocab + 4 * rows * vocab
    return {"bytes": size, "flops": flops}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    return {"norm": _exact_norm, "embed": _exact_embed, "loss": _exact_loss, "distill": _exact_distill}[case["op"]](st)


def _exact_norm(st):
    x, w, b = st["x"].double(), st["w"].double(), st["b"].double()
    s = x if st["r"] is None else (x + st["r"].double()).to(st["x"].dtype).double()  # the norm is that of the stored sum
    var, mean = torch.var_mean(s, dim=1, correction=0, keepdim=True)
    sd = (var + EPS).pow(0.5)
    y = (s - mean) / sd * w + b
    if st["case"]["form"] != "train":
        return dict(y=y, s=s)
    dy, n = st["dy"].double(), s.shape[1]
    a = dy * w
    # dx = J^T a, with J = (I - 1 1^T / n - h h^T / n) / sd
    h = (s - mean) / sd
    dx = (a - a.sum(1, keepdim=True) / n - h * (h * a).sum(1, keepdim=True) / n) / sd
    if st["ds"] is not None:
        dx += st["ds"].double()
    return dict(y=y, s=s, dx=dx, dw=torch.einsum("ij,ij->j", dy, h), db=dy.sum(0))


def _exact_embed(st):
    case, tokens, w = st["case"], st["tokens"], st["w"].double()
    y = torch.index_select(w, 0, tokens) * st["scale"]
    if case["form"] != "train":
        return dict(y=y)
    keep = torch.ones_like(tokens, dtype=torch.bool) if st["padding"] is None else tokens != st["padding"]
    order = torch.sort(tokens[keep], stable=True)
    dy = st["dy"][keep].double()[order.indices]
    ids, counts = torch.unique_consecutive(order.values, return_counts=True)
    ends = torch.cumsum(counts, 0)
    sums = torch.cat([torch.zeros_like(dy[:1]), torch.cumsum(dy, 0)])
    dw = torch.zeros_like(w)
    dw[ids] = (sums[ends] - sums[ends - counts]) * st["scale"]
    return dict(y=y, dw=dw)


def _exact_head(st, live, share, at, T, scale):
    """(lse of x w^T / T, the picked values at `at`, and for training the gradients) of a loss whose gradient at the logits is
    scale (softmax - sum of share at `at`), rows in pieces."""
    x, w, train = st["x"].double(), st["w"].double(), st["case"]["form"] == "train"
    lses, picks, dxs = [], [], []
    dw = torch.zeros_like(w) if train else None
    for a in range(0, x.shape[0], 2048):
        rows = slice(a, a + 2048)
        z = torch.mm(x[rows], w.t()) / T
        lse = torch.logsumexp(z, 1)
        lses.append(lse), picks.append(torch.take_along_dim(z, at[rows], 1))
        if train:
            z = torch.softmax(z, 1)
            z.scatter_add_(1, at[rows], -share[rows])
            z *= torch.where(live[rows], scale[rows], 0.0)[:, None]
            dxs.append(torch.mm(z, w))
            dw += torch.mm(z.t(), x[rows])
    return torch.cat(lses), torch.cat(picks), dict(dx=torch.cat(dxs), dw=dw) if train else {}


def _exact_loss(st):
    targets = st["targets"]
    live = targets >= 0
    at = targets.clamp(min=0)[:, None]
    scale = st["dloss"].double() if "dloss" in st else None
    lse, pick, grads = _exact_head(st, live, torch.ones(at.shape, dtype=torch.float64, device="cuda"), at, 1.0, scale)
    return dict(loss=(lse - pick[:, 0]).masked_fill(~live, 0.0), lse=lse.masked_fill(~live, 0.0), **grads)


def _exact_distill(st):
    ids, T = st["ids"].long(), st["T"]
    there = ids >= 0
    live = there.any(1)
    at = ids.clamp(min=0)
    # a row without entries gets one, whose share is masked with the row
    u = (st["logits"].double() / T).masked_fill(~there & live[:, None], -math.inf)
    logp = torch.log_softmax(u, 1)
    p = logp.exp()
    scale = T * st["dloss"].double() if "dloss" in st else None
    lse, pick, grads = _exact_head(st, live, p, at, T, scale)
    terms = torch.where(p > 0, p * (logp.masked_fill(p == 0, 0.0) - (pick - lse[:, None])), 0.0)
    return dict(loss=(T * T * terms.sum(1)).masked_fill(~live, 0.0), lse=lse.masked_fill(~live, 0.0), **grads)
