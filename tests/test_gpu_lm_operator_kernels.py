"""GPU tests of the operators at the ends of a language model at sizes that take
each of their kernels (_lm_operator_sizes.py; which size takes which is held on the
CPU), against the definitions in 64 bits. The definitions run on the GPU here: the
sizes are large."""
import pytest

torch = pytest.importorskip("torch")

import _lm_operator_refs as R  # noqa: E402
import _lm_operator_sizes as S  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = (F32, BF16)


@pytest.fixture(scope="module")
def ops():
    from paper_2408_01331_amd import operators
    return operators


@pytest.fixture(autouse=True)
def _on_the_gpu(monkeypatch):
    monkeypatch.setattr(R, "d", lambda x: x.detach().double())


def rand(seed, shape, dtype=F32, mean=0.0, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)


def ints(seed, shape, high):
    return torch.randint(0, high, shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def within(got, want, bound, what):
    """|got - want| <= bound everywhere; all are finite."""
    assert got.shape == want.shape, what
    off = (got.double() - want).abs() - bound
    assert (off <= 0).all(), f"{what}: {off.max().item():.3g} beyond the bound, {(off > 0).sum().item()} values; first {torch.nonzero(~(off <= 0))[:3].tolist()}"


def stored(want, bound, dtype):
    return bound + (R.half_step(dtype) * (want.abs() + bound) if dtype != F32 else 0)


# ---------------------------------------------------------------------------
# Layer norm
# ---------------------------------------------------------------------------
def check_layer(ops, rows, width, dtype, residual, seed=0):
    x, w, b = rand(seed, (rows, width), dtype, mean=0.5), rand(seed + 1, (width,), mean=1.0, std=0.3), rand(seed + 2, (width,), std=0.5)
    r = rand(seed + 3, (rows, width), dtype, std=3.0) if residual else None
    dy, ds = rand(seed + 4, (rows, width), dtype), rand(seed + 5, (rows, width), dtype) if residual else None
    y, s, stats = ops.layer_norm(x, w, b, residual=r, keep=True)
    want = R.LayerNorm(x, r, w, b, 1e-5)
    assert torch.equal(s.double(), want.s)
    within(stats[..., 0], want.mean[..., 0], want.e_mean[..., 0], "mean")
    within(stats[..., 1], want.q[..., 0], (want.q * want.e_q)[..., 0], "rstd")
    within(y, want.y, stored(want.y, want.e_y, dtype), "y")
    dx, dw, db = ops.layer_norm_backward(dy, s, w, stats, ds=ds)
    wdx, edx, wdw, edw, wdb, edb = want.backward(dy, ds)
    within(dx, wdx, stored(wdx, edx, dtype), "dx")
    within(dw, wdw, edw, "dw")
    within(db, wdb, edb, "db")


@pytest.mark.parametrize("residual", [False, True], ids=["plain", "residual"])
@pytest.mark.parametrize("t,rows,width", [c[:3] for c in S.LAYER_TWO_ROWS])
def test_layer_norm_of_two_rows_a_thread(ops, t, rows, width, residual):
    check_layer(ops, rows, width, TYPES[t], residual)


@pytest.mark.parametrize("residual", [False, True], ids=["plain", "residual"])
@pytest.mark.parametrize("t,rows,width", S.LAYER_SHARES)
def test_layer_norm_of_several_rows_a_workgroup(ops, t, rows, width, residual):
    check_layer(ops, rows, width, TYPES[t], residual, seed=20)


@pytest.mark.parametrize("t,rows,width", [(1, 40001, 1000), (0, 33001, 700)])
def test_layer_norm_past_the_caches(ops, t, rows, width):
    """Above 256 MiB a call's reads pass the caches."""
    check_layer(ops, rows, width, TYPES[t], True, seed=40)


# ---------------------------------------------------------------------------
# Embedding
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["even", "text"])
@pytest.mark.parametrize("n,vocab,width", [c[:3] for c in S.EMBED_SORTS])
def test_embedding_sorts(ops, n, vocab, width, kind):
    """fp32 sums of each token's rows: the additions of a row are as many as its tokens, and are off by u of their magnitudes
    each; tokens outside the table and a padding token among them."""
    u = torch.rand(n, generator=torch.Generator().manual_seed(n + vocab), dtype=torch.float64)
    t = (u * (vocab + 1)).long() - 1 if kind == "even" else (torch.exp(u * torch.log(torch.tensor(vocab + 1.0))) - 1).long()
    t[0], t[n // 2], t[n - 1], t[n - 2], padding = vocab - 1, 0, vocab, vocab - 1, 1
    t = t.cuda()
    dy = rand(vocab, (n, width))
    got = ops.embedding_backward(dy, t, vocab, scale=0.5, padding=padding)
    keep = (t >= 0) & (t < vocab) & (t != padding)
    at, g = t[keep], dy.double()[keep]
    want = torch.zeros(vocab, width, dtype=torch.float64, device="cuda").index_add_(0, at, g) * 0.5
    size = torch.zeros_like(want).index_add_(0, at, g.abs()) * 0.5
    count = torch.bincount(at, minlength=vocab).double()[:, None]
    within(got, want, size * count * R.U32, "dw")
    onto = rand(1, (vocab, width))
    within(ops.embedding_backward(dy, t.int(), vocab, scale=0.5, padding=padding, out=onto.clone()), want + onto.double(),
           (size * (count + 1) + onto.double().abs()) * R.U32, "out")


# ---------------------------------------------------------------------------
# Losses over a vocabulary
# ---------------------------------------------------------------------------
def gradients(h, coef, onto=None, e_share=0.0):
    """((dx, bound), (dw, bound)) of a Head, without the results' own rounding. As Head.gradients, but for g's rounding: the
    terms of a sum of products with g are off by up to half a step of g each, independently and to either side, and a sum of
    independent errors of up to e_k exceeds 8 sqrt(sum of e_k^2) with a probability of 2 exp(-32), 1e-6 for all elements here
    together (Hoeffding's bound). A block of k that is lost or taken twice is 8 sqrt(rows) terms of it, far outside in bf16."""
    coef = torch.where(h.live.reshape(-1), coef, 0.0)[:, None]
    e_q = h.q * (h.e_z + h.e_lse[:, None] + 2 * R.U32 * ((h.z - h.lse[:, None]).abs() + 4)) + R.TINY
    g = coef * (h.q - h.share)
    e_g = coef.abs() * (e_q + e_share + 2 * R.U32 * (h.q + h.share)) + R.TINY * (coef != 0)
    half = R.U32 if h.t == F32 else R.half_step(h.t)
    out = []
    for left, e_left, right in ((g, e_g, h.w), (g.t(), e_g.t(), h.x)):
        want, n = left @ right, h.n * right.shape[0] + 4
        squares = right * right
        rounding = 8 * half * (((left.abs() + e_left) ** 2) @ squares).sqrt()
        walk = 6 * R.U32 * n ** 0.5 * (want.abs() + 4 * ((left * left) @ squares).sqrt())
        out.append([want, e_left @ right.abs() + rounding + walk])
    if onto is not None:
        out[1] = [out[1][0] + onto.double(), out[1][1] + 2 * R.U32 * onto.double().abs()]
    return out


def check_gradients(h, got, coef, dtype, onto=None, e_share=0.0):
    for g, (want, bound), name, n in zip(got, gradients(h, coef, onto, e_share), ("dx", "dw"), (h.w.shape[0], h.x.shape[0])):
        within(g, want, stored(want, bound, dtype), name)
        if onto is None or name == "dx":
            off, size = (g.double() - want).norm().item(), want.norm().item()
            assert off <= h.norm_tol(n) * size, f"{name}: {off / size:.3g} of its norm off, {h.norm_tol(n):.3g} allowed"


def weights(vocab, width, more, off, dtype):
    """Rows inside a wider buffer, beginning `off` elements late; what lies between is NaN."""
    w = rand(1, (vocab, width), dtype, std=2.0 / width ** 0.5)
    if not more:
        return w
    flat = torch.full((off + vocab * (width + more),), float("nan"), dtype=dtype, device="cuda")
    view = flat[off:].view(vocab, width + more)[:, :width]
    view.copy_(w)
    return view


def hidden(rows, w, first, dtype):
    return (rand(3, (rows, w.shape[1])) + 2.0 * torch.rand(rows, 1, device="cuda") * w[first].float()).to(dtype)


@pytest.mark.parametrize("t,rows,width,vocab,more,off", [c[:6] for c in S.HEADS])
def test_cross_entropy(ops, t, rows, width, vocab, more, off):
    dtype = TYPES[t]
    w, targets = weights(vocab, width, more, off, dtype), ints(2, (rows,), vocab)
    x, dloss = hidden(rows, w, targets, dtype), rand(4, (rows,), std=1.0 / rows)
    targets[:2], targets[-2:] = torch.tensor([0, vocab - 1], device="cuda"), torch.tensor([vocab - 1, 0], device="cuda")
    targets[3::10] = -100
    live = targets >= 0
    loss, lse = ops.vocab_loss(x, w, targets)
    at = targets.clamp(min=0)[:, None]
    h = R.Head(x, w, torch.zeros(rows, vocab, dtype=torch.float64, device="cuda").scatter_(1, at, 1.0), live)
    within(lse, h.masked(h.lse), h.e_lse, "lse")
    want = h.lse - h.z.gather(1, at)[:, 0]
    within(loss, h.masked(want), h.e_lse + h.e_z.gather(1, at)[:, 0] + 2 * R.U32 * want.abs(), "loss")
    check_gradients(h, ops.vocab_loss_backward(x, w, targets, lse, dloss), dloss.double(), dtype)
    onto = rand(5, (vocab, width + 3), dtype, std=1e-3)
    before = onto.clone()
    got = ops.vocab_loss_backward(x, w, targets, lse, dloss, out=onto[:, 1:width + 1])
    check_gradients(h, got, dloss.double(), dtype, onto=before[:, 1:width + 1])
    assert torch.equal(onto[:, 0], before[:, 0]) and torch.equal(onto[:, width + 1:], before[:, width + 1:])


@pytest.mark.parametrize("t,rows,width,vocab,more,off", [c[:6] for c in S.HEADS if c[1:4] in (
    (4877, 800, 5107), (6599, 728, 613), (8190, 1032, 33001), (5061, 624, 1154), (1793, 136, 46041))])
def test_distillation(ops, t, rows, width, vocab, more, off):
    dtype, top, T = TYPES[t], 21, 2.0
    w = weights(vocab, width, more, off, dtype)
    ids = (ints(2, (rows, 1), vocab) + torch.arange(top, device="cuda") * (vocab // top)) % vocab
    x, dloss = hidden(rows, w, ids[:, 0], dtype), rand(4, (rows,), std=1.0 / rows)
    logits = rand(6, (rows, top), std=3.0)
    ids[5::10] = -1
    live = ids[:, 0] >= 0
    loss, lse, picked = ops.distill_loss(x, w, ids, logits, temperature=T)
    at, u = ids.clamp(min=0), logits.double() / T
    p, logp = torch.softmax(u, 1), torch.log_softmax(u, 1)
    p = torch.where(live[:, None], p, 0.0)
    share = torch.zeros(rows, vocab, dtype=torch.float64, device="cuda").scatter_add_(1, at, p)
    # the teacher's p: the exponent t rounds by 2 u |t|, with |t| <= -log p; exponential, sum and quotient by less than 16 u
    e_p = p * (16 - 2 * logp) * R.U32
    e_share = torch.zeros_like(share).scatter_add_(1, at, e_p)
    h = R.Head(x, w, share, live, T)
    z, e_z = h.z.gather(1, at), h.e_z.gather(1, at)
    within(lse, h.masked(h.lse), h.e_lse, "lse")
    within(picked, torch.where(live[:, None], z, 0.0), e_z, "picked")
    terms = logp - z + h.lse[:, None]
    # a term's error: p's of it, log p's (2 u |t| and 16 u), z's and lse's; 40 u more of the magnitudes for the sums
    e_terms = e_p * terms.abs() + p * (e_z + h.e_lse[:, None] + (16 - 2 * logp) * R.U32) + 40 * R.U32 * p * (z.abs() + h.lse.abs()[:, None] - logp)
    within(loss, h.masked(T * T * (p * terms).sum(1)), T * T * e_terms.sum(1), "loss")
    check_gradients(h, ops.distill_loss_backward(x, w, ids, logits, lse, picked, dloss, temperature=T), T * dloss.double(), dtype, e_share=e_share)
