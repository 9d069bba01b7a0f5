"""Performance cases of the operators on device tensors: the RMS norm with a
residual's addition, the gated linear recurrence, and the AdamW step over many
tensors, each with its gradients or its updated state.

A pass is one call as a program makes it, on tensors that it has in hand. The
plain forms are elementary torch operations in 32 bits (64 where a value next
to a rounding border would otherwise fall to the other side).
"""
import math

import torch

own = False

EPS = 1e-6
BETAS, ADAM_EPS, LR, DECAY = (0.9, 0.999), 1e-8, 1e-4, 0.01
QBLOCK = 256        # values that share a scale in the 8-bit optimizer states
E4M3_MAX = 448.0
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _norm(name, rows, width, prec, residual, form):
    return dict(name=name, op="norm", rows=rows, width=width, prec=prec, residual=residual, form=form)


def _scan(name, batch, tokens, width, prec, form, ragged=False, start=False):
    return dict(name=name, op="scan", batch=batch, tokens=tokens, width=width, prec=prec, form=form, ragged=ragged, start=start)


def _adamw(name, kind, total, bits, grad, copies):
    return dict(name=name, op="adamw", kind=kind, total=total, bits=bits, grad=grad, copies=copies)


def listed():
    return [
        # one token of a small model being decoded: latency only
        _norm("norm_token_bf16", 1, 1024, "bf16", True, "plain"),
        # a prompt's rows on their way into 8-bit products: codes, scales and the residual stream
        _norm("norm_e4m3_prompt", 8192, 4096, "bf16", True, "e4m3"),
        # fp32 training at sizes that fill no vector, tile or wave
        _norm("norm_train_f32_odd", 1037, 999, "f32", False, "train"),
        # a training batch of 32 sequences of 1024 tokens, with the residual's gradient
        _norm("norm_train_bf16", 32768, 2048, "bf16", True, "train"),
        # single tokens of 64 sequences, each from its state: latency
        _scan("scan_token_bf16", 64, 1, 1024, "bf16", "plain", start=True),
        # a padded fp32 batch: odd sizes, some sequences empty or of one token
        _scan("scan_train_f32_ragged", 12, 777, 515, "f32", "train", ragged=True, start=True),
        # the usual training batch
        _scan("scan_train_bf16", 16, 2048, 1024, "bf16", "train"),
        # one very long sequence: few channels in all, so the long axis has to be split
        _scan("scan_train_bf16_long", 1, 65536, 512, "bf16", "train"),
        # the tensors of a few small MLPs (this repository's eight-MLP hybrid in size): 35, most of them short
        _adamw("adamw32_small", "mlp", 2_000_000, 32, "f32", False),
        # a large model's tensors, states in 32 bits, bf16 gradients and working copies
        _adamw("adamw32_large", "wide", 200_000_000, 32, "bf16", True),
        # a small model with 8-bit states
        _adamw("adamw8_small", "mlp", 6_000_000, 8, "f32", True),
        # a large one
        _adamw("adamw8_large", "wide", 200_000_000, 8, "bf16", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "scan", "adamw"))
    if op == "norm":
        while True:
            rows, width = _log(rng, 1, 40000), _log(rng, 8, 16384)
            if rng.random() < 0.6:
                width = max(8, width // 8 * 8)
            if rows * width <= 32768 * 2048:
                return dict(op=op, rows=rows, width=width, prec=rng.choice(("f32", "bf16")), residual=rng.random() < 0.5,
                            form=rng.choice(("plain", "e4m3", "train")))
    if op == "scan":
        while True:
            batch, tokens, width = _log(rng, 1, 128), _log(rng, 1, 65536), _log(rng, 8, 4096)
            if rng.random() < 0.6:
                width = max(8, width // 8 * 8)
            if batch * tokens * width <= 16 * 2048 * 1024:
                return dict(op=op, batch=batch, tokens=tokens, width=width, prec=rng.choice(("f32", "bf16")),
                            form=rng.choice(("plain", "train")), ragged=rng.random() < 0.3, start=rng.random() < 0.5)
    return dict(op=op, kind=rng.choice(("mlp", "wide")), total=_log(rng, 50_000, 150_000_000), bits=rng.choice((32, 8)),
                grad=rng.choice(("f32", "bf16")), copies=rng.random() < 0.5)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 7)
    return g


def _normal(g, shape, dtype=torch.float32, mean=0.0, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)


def sizes(case):
    """Sizes of the tensors of an optimizer case, from its kind and total alone."""
    total, out = case["total"], []
    if case["kind"] == "mlp":   # Linear layers as of small MLPs: weight, bias, weight, bias, ...
        widths, k = (784, 512, 256, 333, 128, 97, 10), 0
        while total > 0:
            a, b = widths[k % 7], widths[(k + 1) % 7]
            for n in (a * b, b):
                out.append(min(n, total))
                total -= out[-1]
                if total <= 0:
                    break
            k += 1
        return out
    # blocks of a wide model: four square matrices, two long ones and their vectors
    d = max(64, int(math.sqrt(total / 48)) // 8 * 8)
    block = [d * d] * 4 + [4 * d * d, 4 * d * d, 4 * d, d, d, d + 1]
    k = 0
    while total > 0:
        out.append(min(block[k % len(block)], total))
        total -= out[-1]
        k += 1
    return out


def _starts(ns):
    """First element of each tensor in one buffer, each at a multiple of QBLOCK, and the buffer's length."""
    at, out = 0, []
    for n in ns:
        out.append(at)
        at += -(-n // QBLOCK) * QBLOCK
    return out, at


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case=case)
    if case["op"] == "norm":
        rows, width, t = case["rows"], case["width"], TYPES[case["prec"]]
        st["x"] = _normal(g, (rows, width), t)
        st["r"] = _normal(g, (rows, width), t, std=3.0) if case["residual"] else None
        st["w"] = _normal(g, (width,), mean=1.0, std=0.2)
        if case["form"] == "train":
            st["dy"] = _normal(g, (rows, width), t)
            st["ds"] = _normal(g, (rows, width), t) if case["residual"] else None
    elif case["op"] == "scan":
        b, n, d, t = case["batch"], case["tokens"], case["width"], TYPES[case["prec"]]
        # the two halves of one projection's output: gates that keep a while, and values
        z = torch.empty((b, n, 2 * d), dtype=t, device="cuda")
        z[..., :d] = _normal(g, (b, n, d), t, mean=2.0, std=2.0)
        z[..., d:] = _normal(g, (b, n, d), t)
        st["gate"], st["value"] = z[..., :d], z[..., d:]
        st["h0"] = _normal(g, (b, d)) if case["start"] else None
        st["lens"] = None
        if case["ragged"]:
            lens = torch.randint(0, n + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
            lens[0] = n
            if b > 2:
                lens[1], lens[2] = 0, min(1, n)
            st["lens"] = lens
        if case["form"] == "train":
            st["dh"] = _normal(g, (b, n, d), t)
            st["dlast"] = _normal(g, (b, d))
    else:
        ns = sizes(case)
        starts, total = _starts(ns)
        live = torch.zeros(total, dtype=torch.bool, device="cuda")
        for a, n in zip(starts, ns):
            live[a:a + n] = True
        st["p"] = _normal(g, (total,), std=0.05) * live
        st["g"] = (_normal(g, (total,), std=1e-3) * live).to(TYPES[case["grad"]])
        m, u = _normal(g, (total,), std=3e-4) * live, _normal(g, (total,), std=2e-4).abs() * live + 5e-4 * live
        st["copy"] = st["p"].to(torch.bfloat16) if case["copies"] else None
        st["step"] = 100
        if case["bits"] == 32:
            st["m"], st["v"] = m, u * u
        else:
            for name, x in (("m", m), ("v", u)):
                blocks = x.view(-1, QBLOCK)
                e = _exponent(blocks.abs().amax(1, keepdim=True))
                st[name] = torch.ldexp(blocks, -e).to(torch.float8_e4m3fn).view(-1)
                st[name + "_scale"] = _e8m0(e).view(-1)
        if own:
            st["own"] = _own_adamw(st, starts, ns)
    return st


def _own_adamw(st, starts, ns):
    from paper_2408_01331_amd import operators as ops

    def parts(x, per=1):
        return None if x is None else [x[a // per:(a + n + per - 1) // per] for a, n in zip(starts, ns)]

    return ops.AdamW(parts(st["p"]), parts(st["g"]), parts(st["m"]), parts(st["v"]), copies=parts(st["copy"]),
                     m_scales=parts(st.get("m_scale"), QBLOCK), v_scales=parts(st.get("v_scale"), QBLOCK))


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(st):
    return {"norm": _run_norm, "scan": _run_scan, "adamw": _run_adamw}[st["case"]["op"]](st)


def _run_norm(st):
    form = st["case"]["form"]
    if own:
        from paper_2408_01331_amd import operators as ops
        if form == "e4m3":
            q, scale, s = ops.rms_norm_e4m3(st["x"], st["w"], residual=st["r"], eps=EPS)
            return dict(q=q, scale=scale, s=s)
        y, s, rstd = ops.rms_norm(st["x"], st["w"], residual=st["r"], eps=EPS, keep=form == "train")
        if form == "plain":
            return dict(y=y, s=s)
        dx, dw = ops.rms_norm_backward(st["dy"], s, st["w"], rstd, ds=st["ds"])
        return dict(y=y, s=s, dx=dx, dw=dw)
    x, w, t = st["x"], st["w"], st["x"].dtype
    s = x if st["r"] is None else (x.float() + st["r"].float()).to(t)
    s32 = s.float()
    rstd = 1.0 / torch.sqrt((s32 * s32).mean(1, keepdim=True) + EPS)
    xhat = s32 * rstd
    y = xhat * w
    if form == "e4m3":
        scale = y.abs().amax(1).clamp_min(1e-30) / E4M3_MAX
        return dict(q=(y / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale=scale, s=s)
    if form == "plain":
        return dict(y=y.to(t), s=s)
    dy = st["dy"].float()
    dyw = dy * w
    dx = rstd * (dyw - xhat * (dyw * xhat).mean(1, keepdim=True))
    if st["ds"] is not None:
        dx = dx + st["ds"].float()
    return dict(y=y.to(t), s=s, dx=dx.to(t), dw=(dy * xhat).sum(0))


def _prefix(a, b):
    """Along axis 1, the composition of the maps h -> a h + b up to each place, by doubling."""
    n, k = a.shape[1], 1
    while k < n:
        b = torch.cat([b[:, :k], a[:, k:] * b[:, :-k] + b[:, k:]], 1)
        a = torch.cat([a[:, :k], a[:, k:] * a[:, :-k]], 1)
        k *= 2
    return a, b


def _run_scan(st):
    case, gate, value, lens, h0 = st["case"], st["gate"], st["value"], st["lens"], st["h0"]
    n, d, train = case["tokens"], case["width"], case["form"] == "train"
    if own:
        from paper_2408_01331_amd import operators as ops
        h, last, states = ops.gated_scan(gate, value, h0=h0, lens=lens, keep=train)
        if not train:
            return dict(h=h, last=last)
        dz = torch.empty((case["batch"], n, 2 * d), dtype=gate.dtype, device=gate.device)
        dh0 = ops.gated_scan_backward(gate, value, states, st["dh"], dlast=st["dlast"], lens=lens,
                                      out=(dz[..., :d], dz[..., d:]))
        if lens is None and gate.dtype == torch.float32:
            st["dh"][:, -1] += st["dlast"]  # as the pass below leaves this buffer, so that the next pass has its inputs
        return dict(h=h, last=last, dz=dz, dh0=dh0)
    t = gate.dtype
    g, v = gate.float(), value.float()
    a, keep = torch.sigmoid(g), torch.sigmoid(-g)
    first = torch.zeros_like(v[:, 0]) if h0 is None else h0
    there = None
    if lens is not None:
        there = (torch.arange(n, device=g.device) < lens[:, None])[..., None]
        a, keep = torch.where(there, a, 1.0), torch.where(there, keep, 0.0)
    A, Bv = _prefix(a, keep * v)
    h = A * first[:, None] + Bv
    last = h[:, -1].clone()
    shown = h if there is None else torch.where(there, h, 0.0)
    if not train:
        return dict(h=shown.to(t), last=last)
    del A, Bv
    dh = st["dh"].float()
    if there is not None:
        dh = torch.where(there, dh, 0.0)
    dh[:, -1] += st["dlast"]
    # e_t = dh_t + a_{t+1} e_{t+1}: the same composition from the other end
    back = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1).flip(1)
    e = _prefix(back, dh.flip(1))[1].flip(1)
    before = torch.cat([first[:, None], h[:, :-1]], 1)
    dv = keep * e
    dg = a * dv * (before - v)
    if there is not None:
        dg = torch.where(there, dg, 0.0)
    return dict(h=shown.to(t), last=last, dz=torch.cat([dg, dv], 2).to(t), dh0=a[:, 0] * e[:, 0])


# --- 8-bit states: e4m3 codes, and a power of two for every QBLOCK of them
def _exponent(amax):
    """The least e with amax <= 448 * 2^e (amax as 32-bit values), at least -127."""
    frac, e = torch.frexp(amax)         # amax = frac * 2^e, frac in [1/2, 1)
    e = e - 9 + (frac > 0.875).int()    # 448 = 7/8 * 2^9
    return torch.where(amax > 0, e, -127).clamp(-127, 127)


def _e8m0(e):
    return (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _from_e8m0(s):
    return s.view(torch.uint8).int() - 127


def _random(n, key, device):
    """32 bits for every element from its number and the step's key (whole-number arithmetic mod 2^32)."""
    low = 0xFFFFFFFF
    x = (torch.arange(n, device=device, dtype=torch.int64) * 0x9E3779B9 + key) & low
    x ^= x >> 16
    x = (x * 0x6A09E667) & low
    x ^= x >> 15
    x = (x * 0xBB67AE85) & low
    return x ^ (x >> 16)


def _round_e4m3(x, r):
    """|x| <= 448 onto e4m3, up or down by the 16-bit number r: 1/2^16 steps of the way to the next code."""
    mag = x.abs()
    # steps of the code's last place: 2^(exponent - 3), at least 2^-9
    e = (torch.frexp(mag)[1] - 1).clamp_min(-6) - 3
    q = torch.floor(torch.ldexp(mag.double(), -e) + r.double() / 65536.0)
    return torch.where(x < 0, -1.0, 1.0) * torch.ldexp(q, e).float()


def _key(step):
    return (0x5EED + step * 0x01000193) & 0xFFFFFFFF


def _run_adamw(st):
    case, step = st["case"], st["step"]
    st["step"] += 1
    names = [k for k in ("p", "copy", "m", "v", "m_scale", "v_scale") if st.get(k) is not None]
    if own:
        st["own"].step(LR, step, betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY, key=_key(step))
        return {k: st[k] for k in names}
    p, g = st["p"], st["g"].float()
    b1, b2 = BETAS
    f32 = lambda x: torch.tensor(x, dtype=torch.float32).item()  # noqa: E731
    c1, c2, size = f32(1 - b1), f32(1 - b2), f32(LR / (1 - b1 ** step))
    scale = f32(1 / math.sqrt(1 - b2 ** step))
    eight = case["bits"] == 8
    if eight:
        em, ev = _from_e8m0(st["m_scale"])[:, None], _from_e8m0(st["v_scale"])[:, None]
        m = torch.ldexp(st["m"].float().view(-1, QBLOCK), em).view(-1)
        u = torch.ldexp(st["v"].float().view(-1, QBLOCK), ev).view(-1)
        v = u * u
    else:
        m, v = st["m"], st["v"]
    # one rounding each, as a fused multiply-add has: the 8-bit codes lie next to borders
    m = (m.double() * f32(b1) + (g * c1).double()).float()
    v = (v.double() * f32(b2) + (g * c2 * g).double()).float()
    root = torch.sqrt(v)
    p.copy_(p * f32(1 - LR * DECAY) - size * (m / (root * scale + f32(ADAM_EPS))))
    if st["copy"] is not None:
        st["copy"].copy_(p)
    if not eight:
        st["m"].copy_(m)
        st["v"].copy_(v)
        return {k: st[k] for k in names}
    r = _random(m.numel(), _key(step), m.device).view(-1, QBLOCK)
    for name, x, bits in (("m", m, r & 0xFFFF), ("v", root, r >> 16)):
        x = x.view(-1, QBLOCK)
        e = _exponent(x.abs().amax(1, keepdim=True))
        q = _round_e4m3(torch.ldexp(x, -e), bits)
        if name == "v":  # a second moment that is not zero never becomes zero
            q = torch.where((x > 0) & (q == 0), 2.0 ** -9, q)
        st[name].copy_(q.view(-1).to(torch.float8_e4m3fn))
        st[name + "_scale"].copy_(_e8m0(e).view(-1))
    return {k: st[k] for k in names}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["op"] == "norm":
        n, b, rows, width = case["rows"] * case["width"], SIZE[case["prec"]], case["rows"], case["width"]
        r = case["residual"]
        size = n * b * (3 if r else 1) + 4 * width          # x (and the residual in, their sum out), the weight
        size += n + 4 * rows if case["form"] == "e4m3" else n * b
        flops = 5 * n
        if case["form"] == "train":  # dy, the sum (again), its gradient, dx; the weight and its gradient
            size += n * b * (4 if r else 3) + 8 * width
            flops += 9 * n
        return {"bytes": size, "flops": flops}
    if case["op"] == "scan":
        n, b, chan = case["batch"] * case["tokens"] * case["width"], SIZE[case["prec"]], case["batch"] * case["width"]
        size, flops = 3 * n * b + 4 * chan * (2 if case["start"] else 1), 8 * n
        if case["form"] == "train":
            size += 5 * n * b + 8 * chan
            flops += 20 * n
        return {"bytes": size, "flops": flops}
    n = sum(sizes(case))
    per = 8 + SIZE[case["grad"]] + (16 if case["bits"] == 32 else 4 + 4 / QBLOCK) + (2 if case["copies"] else 0)
    return {"bytes": n * per, "flops": 16 * n}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    return {"norm": _exact_norm, "scan": _exact_scan, "adamw": _exact_adamw}[case["op"]](st)


def _exact_norm(st):
    x, w, form = st["x"].double(), st["w"].double(), st["case"]["form"]
    s = x if st["r"] is None else (x + st["r"].double()).to(st["x"].dtype).double()  # the norm is that of the stored sum
    width = s.shape[1]
    denom = (s.pow(2).sum(1) / width + EPS).pow(0.5)[:, None]
    y = s / denom * w
    if form == "e4m3":
        scale = y.abs().max(1).values.clamp(min=1e-30) / E4M3_MAX
        return dict(q=y / scale[:, None], scale=scale, s=s)
    if form == "plain":
        return dict(y=y, s=s)
    dy = st["dy"].double()
    inner = (dy * w * s).sum(1, keepdim=True) / width
    dx = dy * w / denom - s * inner / denom.pow(3)
    if st["ds"] is not None:
        dx += st["ds"].double()
    return dict(y=y, s=s, dx=dx, dw=(dy * s / denom).sum(0))


def _exact_scan(st):
    case = st["case"]
    b, n, d = case["batch"], case["tokens"], case["width"]
    lens = [n] * b if st["lens"] is None else st["lens"].tolist()
    ends = torch.tensor(lens, device="cuda")
    g, v = st["gate"].double(), st["value"].double()
    a = 1 / (1 + torch.exp(-g))
    keep = 1 / (1 + torch.exp(g))
    first = torch.zeros((b, d), dtype=torch.float64, device="cuda") if st["h0"] is None else st["h0"].double()
    h = torch.zeros((b, n, d), dtype=torch.float64, device="cuda")
    now = first.clone()
    for t in range(n):
        new = a[:, t] * now + keep[:, t] * v[:, t]
        if st["lens"] is not None:
            on = (ends > t)[:, None]
            h[:, t] = torch.where(on, new, 0.0)
            now = torch.where(on, new, now)
        else:
            h[:, t] = now = new
    if case["form"] != "train":
        return dict(h=h, last=now)
    dz = torch.zeros((b, n, 2 * d), dtype=torch.float64, device="cuda")
    dh = st["dh"].double()
    carry = st["dlast"].double()
    for t in reversed(range(n)):
        e = carry + dh[:, t]
        prev = h[:, t - 1] if t else first
        dv = keep[:, t] * e
        dg = a[:, t] * dv * (prev - v[:, t])
        new = a[:, t] * e
        if st["lens"] is not None:
            on = (ends > t)[:, None]
            dv, dg, new = torch.where(on, dv, 0.0), torch.where(on, dg, 0.0), torch.where(on, new, carry)
        dz[:, t, :d], dz[:, t, d:], carry = dg, dv, new
    return dict(h=h, last=now, dz=dz, dh0=carry)


def _exact_adamw(st):
    case, step = st["case"], st["step"]
    b1, b2 = BETAS
    g = st["g"].double()
    if case["bits"] == 8:
        wide = lambda k: (st[k].double().view(-1, QBLOCK) * torch.pow(2.0, _from_e8m0(st[k + "_scale"]).double())[:, None]).view(-1)  # noqa: E731
        m, v = wide("m"), wide("v") ** 2
    else:
        m, v = st["m"].double(), st["v"].double()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    mhat, vhat = m / (1 - b1 ** step), v / (1 - b2 ** step)
    p = st["p"].double()
    p = p - LR * DECAY * p - LR * mhat / (vhat.sqrt() + ADAM_EPS)
    out = dict(p=p, copy=p if case["copies"] else None, m=m, v=v)
    if case["bits"] == 8:
        # which of two neighbouring codes a value gets is the random number's choice, so no value in 64 bits is the code's
        out.update(m=None, v=None, m_scale=None, v_scale=None)
    return out
