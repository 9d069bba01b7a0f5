"""The operators at the ends of a language model (layer norm, embedding, vocabulary
loss, distillation) in 64 bits on the CPU, by their definitions, with bounds on
what 32-bit arithmetic may be off. u = 2^-24 is half a step of fp32 relative to
the value."""
import torch

from _operator_refs import TINY, U32, close, d, half_step  # noqa: F401


# ---------------------------------------------------------------------------
# Layer norm
# ---------------------------------------------------------------------------
# A sum over a row: a thread adds up to 16 values, 6 steps join a wave and up to 16
# waves follow: 38 u of the magnitudes' sum; the mean's division one more, rounded up.
ROW_U = 40 * U32


class LayerNorm:
    """Everything of a row's norm, with the bounds of what follows from it."""

    def __init__(self, x, r, w, b, eps):
        self.s = d(x) if r is None else d((d(x) + d(r)).to(x.dtype))
        s, self.w = self.s, d(w)
        self.mean = s.mean(-1, keepdim=True)
        self.c = s - self.mean
        var = (self.c * self.c).mean(-1, keepdim=True) + eps
        self.q = var.rsqrt()
        self.h = self.c * self.q
        self.y = self.h * self.w + (0 if b is None else d(b))
        # the mean; then the squares of values that are off by the mean's error and a rounding, 42 u of their sum; the root
        # halves, and with the sum with eps, the root and the reciprocal 4 u and more follow
        self.e_mean = ROW_U * s.abs().mean(-1, keepdim=True)
        self.e_q = self.c.abs().mean(-1, keepdim=True) * self.e_mean / var + self.e_mean ** 2 / var + 30 * U32
        self.e_h = self.q * (self.e_mean + 2 * U32 * self.c.abs()) + self.h.abs() * self.e_q
        self.e_y = self.w.abs() * self.e_h + 2 * U32 * ((self.h * self.w).abs() + self.y.abs())

    def backward(self, dy, ds):
        dy = d(dy)
        a, h, q = dy * self.w, self.h, self.q
        c0, c1 = a.mean(-1, keepdim=True), (a * h).mean(-1, keepdim=True)
        dx = q * (a - c0 - h * c1)
        e0 = ROW_U * a.abs().mean(-1, keepdim=True)
        e1 = (ROW_U + 4 * U32) * (a * h).abs().mean(-1, keepdim=True) + (a.abs() * self.e_h).mean(-1, keepdim=True)
        mag = a.abs() + c0.abs() + (h * c1).abs()
        e = q * ((self.e_q + 8 * U32) * mag + e0 + h.abs() * e1 + self.e_h * c1.abs())
        if ds is not None:
            dx, e = dx + d(ds), e + 2 * U32 * d(ds).abs()
        rows, hr, er = (t.reshape(-1, t.shape[-1]) for t in (dy, h, self.e_h))
        n = U32 * (rows.shape[0] + 40)
        return (dx, e, (rows * hr).sum(0), ((rows * hr).abs() * n + rows.abs() * er).sum(0), rows.sum(0), rows.abs().sum(0) * n)


# ---------------------------------------------------------------------------
# Embedding
# ---------------------------------------------------------------------------
def embedding(tokens, weight, scale):
    """y, by definition: zeros for tokens outside the table."""
    t, w = tokens.cpu().long(), d(weight)
    there = (t >= 0) & (t < w.shape[0])
    return torch.where(there[..., None], w[t.clamp(0, w.shape[0] - 1)] * scale, 0.0)


def embedding_backward(dy, tokens, vocab, scale, padding, onto):
    """(dweight, its bound): sums of up to `count` terms in fp32, the scale's product, and the addition onto what is there.
    (The call holds the scale in fp32, which is off by up to u of it: one u more of the magnitudes.)"""
    t, g = tokens.cpu().long().flatten(), d(dy).reshape(-1, dy.shape[-1])
    keep = (t >= 0) & (t < vocab)
    if padding is not None:
        keep &= t != padding
    t, g = t[keep], g[keep]
    dw = torch.zeros(vocab, g.shape[1], dtype=torch.float64).index_add_(0, t, g) * scale
    mag = torch.zeros_like(dw).index_add_(0, t, g.abs()) * abs(scale)
    bound = mag * U32 * (torch.bincount(t, minlength=vocab).double()[:, None] + 3)
    if onto is not None:
        dw = dw + d(onto)
        bound = bound + U32 * (d(onto).abs() + mag) * (mag > 0)
    return dw, bound


# ---------------------------------------------------------------------------
# Losses over a vocabulary
# ---------------------------------------------------------------------------
def near(got, want, tol, what):
    """|got - want| <= tol |want| in the 2-norm over the whole tensor."""
    got, want = d(got), d(want)
    assert got.shape == want.shape, what
    off, size = (got - want).norm().item(), want.norm().item()
    assert off <= tol * size + 1e-300, f"{what}: {off / max(size, 1e-300):.3g} of its norm off, {tol:.3g} allowed"


class Head:
    """z = x w^T / T of the live rows and a loss whose gradient there is coef (softmax(z) - share).

    The errors, element by element. A product's sum of n terms (fp32 operands: six bf16 products for each, 6 n) rounds n
    times; the partial sums stay within |z| + 4 A, A the root of the terms' squares' sum, and n independent roundings of up to u
    add up to less than 6 u sqrt(n) of that. (The terms that the six products leave out are below 4.1 u of |x w|, which
    sqrt(n) >= 1 covers.) Softmax: an exponential of z - lse is off by (|z - lse| + 4) 2 u of itself, beside what z and lse are
    off; a sum over the vocabulary rounds at most 300 times on any path. g rounds to bf16 (half a step, 2^-8) with bf16 operands
    and to three terms (u) with fp32.

    Over a whole tensor (norm): g's rounding and the result's, in bf16, are independent from element to element, at most
    2^-8 / sqrt(3) of each, 2^-8 sqrt(2 / 3) together; allowed is 1.25 2^-8, as terms that cancel leave a norm smaller than
    that of the terms. fp32: independent roundings of partial sums that grow like a random walk, 0.41 u sqrt(n) of a product of
    n terms: half of u sqrt(n) is allowed for the gradient's product. g is off by what z - lse is off, in absolute terms: the
    problems here have |z| up to 12, 0.41 * 12 < 5 times u sqrt(n) of the logits' product, and 24 u for the exponential of
    such a z."""

    def __init__(self, x, w, share, live, T=1.0):
        self.t, self.live, self.T = x.dtype, live, T
        lead = live.shape
        self.lead = lead
        x = torch.where(live.reshape(-1, 1), d(x).reshape(-1, x.shape[-1]), 0.0)
        w = d(w)
        self.x, self.w, self.share = x, w, share
        self.n = (6 if self.t == torch.float32 else 1)
        z = x @ w.t()
        a = ((x * x) @ (w * w).t()).sqrt()
        self.z = z / T
        self.e_z = 6 * U32 * (self.n * x.shape[1] + 4) ** 0.5 * (z.abs() + 4 * a) / T + 2 * U32 * self.z.abs()
        self.lse = torch.logsumexp(self.z, 1)
        self.q = torch.exp(self.z - self.lse[:, None])
        self.e_lse = (self.q * self.e_z).sum(1) + 300 * U32 + 2 * U32 * self.lse.abs()

    def masked(self, t):
        return torch.where(self.live.reshape(-1), t, 0.0).reshape(self.lead)

    def gradients(self, coef, onto=None):
        """((dx, bound), (dw, bound)), without the results' own rounding."""
        coef = torch.where(self.live.reshape(-1), coef, 0.0)[:, None]
        # (below 2^-126 a probability, and its product with coef, is 0 or has fewer digits in 32 bits: off by up to 2^-126,
        # whatever its own size, exp(-500) in 64 bits being 7e-218)
        e_q = self.q * (self.e_z + self.e_lse[:, None] + 2 * U32 * ((self.z - self.lse[:, None]).abs() + 4)) + TINY
        g = coef * (self.q - self.share)
        half = U32 if self.t == torch.float32 else half_step(self.t)
        e_g = coef.abs() * (e_q + 2 * U32 * (self.q + self.share)) + 2 * half * g.abs() + TINY * (coef != 0)
        out = []
        for left, e_left, right in ((g, e_g, self.w), (g.t(), e_g.t(), self.x)):
            want = left @ right
            n = self.n * right.shape[0] + 4
            walk = 6 * U32 * n ** 0.5 * (want.abs() + 4 * ((left * left) @ (right * right)).sqrt())
            out.append((want, e_left @ right.abs() + walk))
        (dx, e_dx), (dw, e_dw) = out
        if onto is not None:
            dw, e_dw = dw + d(onto), e_dw + 2 * U32 * d(onto).abs()
        return (dx.reshape(*self.lead, -1), e_dx.reshape(*self.lead, -1)), (dw, e_dw)

    def norm_tol(self, rows):
        if self.t != torch.float32:
            return 1.25 * half_step(self.t)
        return U32 * (5 * (6 * self.x.shape[1]) ** 0.5 + 0.5 * (6 * rows) ** 0.5 + 24)


def cross_entropy(x, w, targets, ignore=-100):
    """(Head, loss, its bound, lse, its bound)"""
    t = targets.cpu().long().reshape(-1)
    live = (t >= 0) & (t < w.shape[0]) & (t != ignore)
    at = torch.where(live, t, 0)[:, None]
    share = torch.zeros(t.numel(), w.shape[0], dtype=torch.float64).scatter_(1, at, 1.0)
    h = Head(x, w, share, live.reshape(targets.shape))
    loss = h.lse - h.z.gather(1, at)[:, 0]
    bound = h.e_lse + h.e_z.gather(1, at)[:, 0] + 2 * U32 * loss.abs()
    return h, h.masked(loss), bound.reshape(h.lead), h.masked(h.lse), h.e_lse.reshape(h.lead)


def distillation(x, w, ids, logits, T):
    """(Head, loss, its bound, lse, its bound, picked, its bound)"""
    top = ids.shape[-1]
    i, u = ids.cpu().long().reshape(-1, top), d(logits).reshape(-1, top)
    there = (i >= 0) & (i < w.shape[0]) & (u != -float("inf"))
    live = there.any(1)
    u = torch.where(there, u / T, -float("inf"))
    u = torch.where(live[:, None], u, 0.0)
    p = torch.where(there, torch.softmax(u, 1), 0.0)
    logp = torch.where(there, torch.log_softmax(u, 1), 0.0)
    at = torch.where(there, i, 0)
    share = torch.zeros(i.shape[0], w.shape[0], dtype=torch.float64).scatter_add_(1, at, p)
    h = Head(x, w, share, live.reshape(ids.shape[:-1]), T)
    z, e_z = h.z.gather(1, at), h.e_z.gather(1, at)
    terms = torch.where(p > 0, p * (logp - z + h.lse[:, None]), 0.0)
    # p: the exponent and the sum of up to 128 terms; log p likewise; then the sum of the terms
    size = torch.where(p > 0, p * (logp.abs() + z.abs() + h.lse.abs()[:, None]), 0.0)
    slope = torch.where(p > 0, u.abs() + 1, 0.0)
    bound = T * T * ((p * (e_z + h.e_lse[:, None])).sum(1) + 40 * U32 * size.sum(1) + (4 * U32 * p * slope).sum(1) + 40 * U32)
    return (h, h.masked(T * T * terms.sum(1)), bound.reshape(h.lead), h.masked(h.lse), h.e_lse.reshape(h.lead),
            torch.where(there, z, 0.0).reshape(ids.shape), e_z.reshape(ids.shape))
