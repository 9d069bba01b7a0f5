"""The operators on device tensors in 64 bits on the CPU, by their definitions,
with bounds on what 32-bit arithmetic may be off.

Bounds. u = 2^-24 is half a step of fp32 relative to the value; a stored type
adds half of its own step (bf16 2^-8). Sums are bounded by (number of additions
on the longest path) u times the sum of magnitudes.
"""
import torch

U32 = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2


def d(x):
    return x.detach().double().cpu()


def close(got, want, bound, what):
    """|got - want| <= bound everywhere, NaN and infinities alike."""
    got, want, bound = d(got), d(want), d(bound)
    assert got.shape == want.shape, what
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities differ"
    off = (got - want).abs()[fine] - bound.expand_as(want)[fine]
    if off.numel():
        worst = off.max().item()
        assert worst <= 0, f"{what}: {worst:.3g} beyond the bound; at {torch.nonzero((got - want).abs() > bound.expand_as(want))[:3].tolist()}"


# ---------------------------------------------------------------------------
# RMS norm
# ---------------------------------------------------------------------------
# 1/rms: a thread adds up to 16 squares, 6 steps join a wave and up to 16 waves
# follow: 38 u of the sum, of which the root halves; with the division, the sum
# with eps, the root and the reciprocal: under 32 u relative. The value itself:
# two products more.
NORM_U = 36 * U32


def norm_fwd(x, r, w, eps):
    s = d(x) if r is None else d((d(x) + d(r)).to(x.dtype))
    q = 1 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    return s, q, s * q * d(w)


def norm_bwd(dy, s, w, eps, ds):
    s, dy, w = d(s), d(dy), d(w)
    q = 1 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    xh = s * q
    c = (dy * w * xh).mean(-1, keepdim=True)
    mag = (dy * w * xh).abs().mean(-1, keepdim=True)
    dx = q * (dy * w - xh * c)
    # q carries 32 u, c its own 60 u of its terms' magnitudes; a product or sum each 1 u
    bound = U32 * (70 * q * (dy * w).abs() + 140 * q * xh.abs() * mag)
    if ds is not None:
        dx = dx + d(ds)
        bound = bound + 2 * U32 * d(ds).abs()
    rows = dy.reshape(-1, dy.shape[-1])
    xr = xh.reshape(rows.shape)
    dw = (rows * xr).sum(0)
    dw_bound = (rows * xr).abs().sum(0) * U32 * (rows.shape[0] + 40)
    return dx, bound, dw, dw_bound


# ---------------------------------------------------------------------------
# Gated linear recurrence
# ---------------------------------------------------------------------------
# a and 1 - a: the exponential's argument is off by |g| log2(e) u (up to 12 u at
# |g| = 8; fp32 adds the rounding error back), and four roundings follow; the
# step's own product and sum, and those of joining the waves' maps: within 32 u a
# step. The error of the state follows the recurrence itself.
SCAN_U = 32 * U32
# Below 2^-126 fp32 has no full precision: a or 1 - a of a gate beyond +-87 is off by up to that much whatever its
# own size (sigmoid(-200) is 1.4e-87 and 0 in fp32), and what it multiplies is off by that times the other factors.
TINY = 2.0 ** -126


def scan_fwd(gate, value, h0, lens):
    """(h, its bound, last, its bound)"""
    g, v = d(gate), d(value)
    b, n, w = g.shape
    now = torch.zeros(b, w, dtype=torch.float64) if h0 is None else d(h0)
    err, mag = torch.zeros_like(now), now.abs()
    a, k = torch.sigmoid(g), torch.sigmoid(-g)
    h, eh = torch.zeros_like(g), torch.zeros_like(g)
    ends = None if lens is None else lens.cpu().clamp(0, n)
    for t in range(n):
        new = a[:, t] * now + k[:, t] * v[:, t]
        nm = a[:, t] * mag + k[:, t] * v[:, t].abs()
        ne = a[:, t] * err + SCAN_U * nm + TINY * (mag + v[:, t].abs())
        if ends is None:
            now, mag, err = new, nm, ne
            h[:, t], eh[:, t] = now, err
        else:
            on = (ends > t)[:, None]
            now, mag, err = torch.where(on, new, now), torch.where(on, nm, mag), torch.where(on, ne, err)
            h[:, t], eh[:, t] = torch.where(on, now, 0.0), torch.where(on, err, 0.0)
    return h, eh, now, err


def scan_bwd(gate, value, h0, lens, dh, dlast):
    """((dgate, bound), (dvalue, bound), (dh0, bound))"""
    g, v = d(gate), d(value)
    b, n, w = g.shape
    a, k = torch.sigmoid(g), torch.sigmoid(-g)
    ends = torch.full((b,), n) if lens is None else lens.cpu().clamp(0, n)
    now = torch.zeros(b, w, dtype=torch.float64) if h0 is None else d(h0)
    mag, err = now.abs(), torch.zeros_like(now)
    prev, pmag, perr = [], [], []
    for t in range(n):
        on = (ends > t)[:, None]
        prev.append(now), pmag.append(mag), perr.append(err)
        nm = a[:, t] * mag + k[:, t] * v[:, t].abs()
        now = torch.where(on, a[:, t] * now + k[:, t] * v[:, t], now)
        err = torch.where(on, a[:, t] * err + SCAN_U * nm + TINY * (mag + v[:, t].abs()), err)
        mag = torch.where(on, nm, mag)
    c = torch.zeros(b, w, dtype=torch.float64) if dlast is None else d(dlast)
    cm, ce = c.abs(), torch.zeros_like(c)
    out = [torch.zeros_like(g) for _ in range(4)]
    dd = d(dh)
    for t in reversed(range(n)):
        on = (ends > t)[:, None]
        dt = torch.where(on, dd[:, t], 0.0)
        e, em, ee = c + dt, cm + dt.abs(), ce + U32 * (cm + dt.abs())
        x, xm = prev[t] - v[:, t], pmag[t] + v[:, t].abs()
        out[0][:, t] = torch.where(on, a[:, t] * k[:, t] * e * x, 0.0)
        out[1][:, t] = torch.where(on, a[:, t] * k[:, t] * (ee * xm + em * perr[t] + SCAN_U * em * xm) + TINY * em * xm, 0.0)
        out[2][:, t] = torch.where(on, k[:, t] * e, 0.0)
        out[3][:, t] = torch.where(on, k[:, t] * (ee + SCAN_U * em) + TINY * em, 0.0)
        c = torch.where(on, a[:, t] * e, c)
        cm, ce = torch.where(on, a[:, t] * em, cm), torch.where(on, a[:, t] * (ee + SCAN_U * em) + TINY * em, ce)
    return (out[0], out[1]), (out[2], out[3]), (c, ce)


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
def adamw(p, g, m, v, lr, betas, eps, decay, t):
    """New (p, m, v) and the magnitude of p's update, in 64 bits."""
    b1, b2 = betas
    p, g, m, v = d(p), d(g), d(m), d(v)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    up = lr / (1 - b1 ** t) * m / (v.sqrt() / (1 - b2 ** t) ** 0.5 + eps)
    return p * (1 - lr * decay) - up, m, v, up.abs()


def widen(codes, scales, block=256):
    """8-bit values as what they stand for."""
    c = codes.cpu().float().double()
    e = scales.cpu().view(torch.uint8).double() - 127
    return c * torch.repeat_interleave(torch.pow(2.0, e), block)[:c.numel()]
