"""The operators at the ends of a language model (layer norm, embedding, vocabulary
loss, distillation) in 64 bits on the CPU, by their definitions, with bounds on
what 32-bit arithmetic may be off. u = 2^-24 is half a step of fp32 relative to
the value."""
import torch

from _operator_refs import U32, close, d, half_step  # noqa: F401


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
