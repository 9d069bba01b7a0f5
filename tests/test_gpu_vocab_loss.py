"""GPU tests of the losses over a vocabulary on device tensors (cross entropy and
distillation from hidden states) against their definitions in 64 bits (bounds:
_lm_operator_refs.py)."""
import pytest

torch = pytest.importorskip("torch")

import _lm_operator_refs as R  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DTYPES = [F32, BF16]


@pytest.fixture(scope="module")
def ops():
    from paper_2408_01331_amd import operators
    return operators


def rand(seed, shape, dtype=F32, mean=0.0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).cuda()


def ints(seed, shape, high, dtype=torch.int64):
    return torch.randint(0, high, shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def stored(want, bound, dtype):
    return bound + (R.half_step(dtype) * (want.abs() + bound) if dtype != F32 else 0)


def problem(rows, width, vocab, dtype, seed=0, left_out=0.0, index=torch.int64):
    w = rand(seed, (vocab, width), dtype, std=2.0 / width ** 0.5)
    targets = ints(seed + 1, (rows,), vocab, index)
    x = (rand(seed + 2, (rows, width)) + 2.0 * torch.rand(rows, 1, device="cuda") * w[targets.long()].float()).to(dtype)
    if left_out:
        targets[torch.randperm(rows, generator=torch.Generator().manual_seed(seed))[:int(rows * left_out)].cuda()] = -100
    return x, w, targets


def check_grads(h, got, coef, dtype, onto=None, norms=True):
    (wdx, edx), (wdw, edw) = h.gradients(coef, onto)
    R.close(got[0], wdx, stored(wdx, edx, dtype), "dx")
    R.close(got[1], wdw, stored(wdw, edw, dtype), "dw")
    if norms and h.x.shape[0] >= 64:  # (few elements are no average)
        R.near(got[0], wdx, h.norm_tol(h.w.shape[0]), "dx")
        if onto is None:
            R.near(got[1], wdw, h.norm_tol(h.x.shape[0]), "dw")


def check_loss(ops, x, w, targets, dloss, ignore=-100, onto=None, norms=True):
    dtype = x.dtype
    loss, lse = ops.vocab_loss(x, w, targets, ignore=ignore)
    h, wl, el, ws, es = R.cross_entropy(x, w, targets, ignore)
    R.close(loss, wl, el, "loss")
    R.close(lse, ws, es, "lse")
    assert (loss >= 0).all()
    got = ops.vocab_loss_backward(x, w, targets, lse, dloss, ignore=ignore, out=None if onto is None else onto.clone())
    check_grads(h, got, R.d(dloss).reshape(-1).expand(h.live.numel()), dtype, onto, norms)
    return loss, lse, got


SIZES = [(1, 1, 1), (1, 8, 5), (3, 33, 100), (64, 64, 256), (65, 96, 257), (130, 520, 1000), (300, 40, 5000), (257, 1000, 300),
         (20, 2056, 700), (513, 264, 4097), (1100, 72, 520)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,width,vocab", SIZES)
@pytest.mark.parametrize("left_out", [0.0, 0.6])
def test_vocab_loss(ops, dtype, rows, width, vocab, left_out):
    x, w, targets = problem(rows, width, vocab, dtype, left_out=left_out, index=torch.int32 if rows % 2 else torch.int64)
    check_loss(ops, x, w, targets, rand(9, (rows,), std=1.0 / rows))


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,width,vocab", [(5, 33, 70), (130, 264, 1000)])
def test_onto(ops, dtype, rows, width, vocab):
    """dweight is added onto what is there, in rows that are apart, and what lies between keeps its bits."""
    x, w, targets = problem(rows, width, vocab, dtype, left_out=0.2)
    for off in (0, 1):
        wide = rand(5, (vocab, width + 9), dtype)
        before = wide.clone()
        onto = wide[:, off:off + width]
        loss, lse = ops.vocab_loss(x, w, targets)
        dloss = rand(6, (rows,))
        dx, dw = ops.vocab_loss_backward(x, w, targets, lse, dloss, out=onto)
        assert dw.data_ptr() == onto.data_ptr()
        h = R.cross_entropy(x, w, targets)[0]
        check_grads(h, (dx, dw), R.d(dloss), dtype, before[:, off:off + width])
        wide[:, off:off + width] = before[:, off:off + width]
        assert torch.equal(wide, before)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_strides_shapes_and_alignment(ops, dtype):
    """Operands inside wider buffers at every alignment give what dense ones give; axes of any number and order; one dloss for all."""
    x, w, targets = problem(24, 40, 300, dtype)
    dloss = rand(3, (24,))
    loss, lse = ops.vocab_loss(x, w, targets)
    dx, dw = ops.vocab_loss_backward(x, w, targets, lse, dloss)
    for off, more in ((0, 8), (1, 8), (3, 7), (8, 16)):
        bx, bw = rand(7, (24, 40 + more + off), dtype), rand(8, (300, 40 + more + off), dtype)
        bx[:, off:off + 40], bw[:, off:off + 40] = x, w
        x2, w2 = bx[:, off:off + 40], bw[:, off:off + 40]
        l2, s2 = ops.vocab_loss(x2, w2, targets)
        assert torch.equal(l2, loss) and torch.equal(s2, lse)
        for a, b in zip(ops.vocab_loss_backward(x2, w2, targets, lse, dloss), (dx, dw)):
            assert torch.equal(a, b)
    x3, t3 = x.view(4, 6, 40).transpose(0, 1), targets.view(4, 6).t()
    l3, s3 = ops.vocab_loss(x3, w, t3)
    assert l3.shape == (6, 4)
    check_loss(ops, x3, w, t3, rand(4, (6, 4)))
    check_loss(ops, x, w, targets, torch.tensor(0.25, device="cuda"))
    check_loss(ops, x[5], w, targets[5], torch.tensor(0.25, device="cuda"))
    check_loss(ops, x, w, targets, torch.tensor([0.25], device="cuda").expand(24))
    check_loss(ops, x, w, targets, rand(5, (48,))[::2])
    check_loss(ops, x3, w, t3, rand(6, (4, 6)).t())


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_rows_left_out(ops, dtype):
    """Rows without a target are not used, whatever they hold, and change nothing for the others; all rows may be left out."""
    x, w, targets = problem(200, 72, 500, dtype)
    targets[::3] = torch.tensor([-100, -1, 500, 2 ** 40], device="cuda")[torch.arange(67, device="cuda") % 4]
    targets[1::9] = 7
    dloss = rand(1, (200,))
    out = (targets < 0) | (targets >= 500) | (targets == 7)
    x2, d2 = x.clone(), dloss.clone()
    x2[out], d2[out] = float("nan"), float("inf")
    x2[0] = float("inf")
    loss, lse, (dx, dw) = check_loss(ops, x, w, targets, dloss, ignore=7)
    l2, s2 = ops.vocab_loss(x2, w, targets, ignore=7)
    assert torch.equal(l2, loss) and torch.equal(s2, lse) and (loss[out] == 0).all() and (lse[out] == 0).all()
    s2[out] = float("nan")
    g2 = ops.vocab_loss_backward(x2, w, targets, s2, d2, ignore=7)
    assert torch.equal(g2[0], dx) and torch.equal(g2[1], dw) and (dx[out] == 0).all()
    keep = ~out
    l3, _ = ops.vocab_loss(x[keep], w, targets[keep], ignore=7)
    assert torch.equal(l3, loss[keep])
    nothing = torch.full((200,), -100, device="cuda")
    l4, s4 = ops.vocab_loss(x2, w, nothing)
    assert (l4 == 0).all() and (s4 == 0).all()
    dx4, dw4 = ops.vocab_loss_backward(x2, w, nothing, s4, d2)
    assert (dx4 == 0).all() and (dw4 == 0).all()
    onto = rand(4, (500, 72), dtype)
    assert torch.equal(ops.vocab_loss_backward(x2, w, nothing, s4, d2, out=onto.clone())[1], onto)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_no_rows(ops, dtype):
    x, w, t = torch.empty(0, 40, dtype=dtype, device="cuda"), rand(1, (30, 40), dtype), torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = ops.vocab_loss(x, w, t)
    assert loss.shape == lse.shape == (0,)
    dx, dw = ops.vocab_loss_backward(x, w, t, lse, loss)
    assert dx.shape == x.shape and (dw == 0).all()
    onto = rand(2, (30, 40), dtype)
    assert torch.equal(ops.vocab_loss_backward(x, w, t, lse, loss, out=onto.clone())[1], onto)


def test_values_that_are_not_finite(ops):
    """An infinity or a NaN in a live row concerns that row's loss alone; a logit of -inf is a token of no probability."""
    x, w, targets = problem(70, 64, 300, BF16)
    clean = ops.vocab_loss(x, w, targets)[0]
    x2 = x.clone()
    x2[3, 5], x2[9, 1] = float("nan"), float("inf")
    loss = ops.vocab_loss(x2, w, targets)[0]
    keep = torch.ones(70, dtype=torch.bool, device="cuda")
    keep[[3, 9]] = False
    assert torch.equal(loss[keep], clean[keep]) and torch.isnan(loss[3]) and not torch.isfinite(loss[9])
    x3, w3 = x.abs() + 0.5, w.clone()
    w3[17] = -float("inf")
    t3 = torch.where(targets == 17, 18, targets)
    loss, lse = ops.vocab_loss(x3, w3, t3)
    without = torch.cat([w[:17], w[18:]])
    h, wl, el, ws, es = R.cross_entropy(x3, without, t3 - (t3 > 17).long())
    R.close(loss, wl, el, "loss")
    R.close(lse, ws, es, "lse")


def test_large_logits(ops):
    """Logits in the thousands: nothing overflows, and a sure row's loss is exactly small."""
    x, w, targets = problem(66, 64, 300, F32)
    check_loss(ops, x * 1000, w, targets, rand(1, (66,)), norms=False)
    check_loss(ops, x * -3000, w, targets, rand(1, (66,)), norms=False)


def test_three_terms(ops):
    """fp32 operands, all three terms of each: where the vocabulary is one token, lse is its logit; where rows and weights
    have one value each, a gradient is one product."""
    x, w = rand(1, (300, 1)), rand(2, (1, 1))
    t = torch.zeros(300, dtype=torch.int64, device="cuda")
    want = R.d(x) * R.d(w)
    # products that are left out: 4.1 u; six roundings: 11 u |z|. The sum is kept as s 2^M with a whole M next to z log2(e), so
    # s is in [1/2, 1]: its exponent rounds by u and the exponential by 2 u, log(s) (below 0.7) carries that and u of its own;
    # M ln 2, of |z| + 0.7, and the last sum round by u each: below 8 u + 3 u |z| in all.
    R.close(ops.vocab_loss(x, w, t)[1], want[:, 0], (want[:, 0].abs() * 14 + 8) * R.U32, "lse")
    for k in range(20):
        x, w = rand(k, (1, 3)), torch.diag(rand(k + 50, (3,)))[:, :3].contiguous()
        t = torch.tensor([k % 3], device="cuda")
        loss, lse = ops.vocab_loss(x, w, t)
        dx, dw = ops.vocab_loss_backward(x, w, t, lse, torch.tensor(0.7, device="cuda"))
        z = R.d(x) * R.d(w).diagonal()
        g = torch.softmax(z, 1)
        e_q = g * (24 * z.abs().max() + 24) * 2 * R.U32  # z and lse to 11 u and less of |z| <= 4, the exponential, the product
        g[0, k % 3] -= 1
        g, e = g * torch.tensor(0.7).double(), e_q + 12 * R.U32 * g.abs()
        R.close(dx, g * R.d(w).diagonal(), e * R.d(w).diagonal().abs(), "dx")
        R.close(dw, g.t() @ R.d(x), e.t() @ R.d(x).abs(), "dw")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_pieces_of_the_vocabulary(ops, dtype):
    """Enough rows for several pieces: the same gradients as those of the rows in parts that need one piece each."""
    rows, width, vocab = 8500, 40, 33000 if dtype == BF16 else 12000
    x, w, targets = problem(rows, width, vocab, dtype, left_out=0.1)
    dloss = rand(4, (rows,), std=1.0 / rows)
    loss, lse = ops.vocab_loss(x, w, targets)
    dx, dw = ops.vocab_loss_backward(x, w, targets, lse, dloss)
    total = torch.zeros(vocab, width, dtype=torch.float64, device="cuda")
    for a in range(0, rows, 1700):
        s = slice(a, a + 1700)
        l2, s2 = ops.vocab_loss(x[s], w, targets[s])
        # a row's tiles and sums are the same in any batch; a gradient's sum over the vocabulary may be cut otherwise
        assert torch.equal(l2, loss[s]) and torch.equal(s2, lse[s])
        X, W = x[s].double(), w.double()
        z = X @ W.t()
        g = torch.softmax(z, 1)
        live = targets[s] >= 0
        g[torch.arange(1700, device="cuda"), targets[s].clamp(min=0)] -= 1
        g *= torch.where(live, dloss[s].double(), 0.0)[:, None]
        h = R.Head.__new__(R.Head)
        h.t, h.x = dtype, X
        R.near(dx[s], g @ W, h.norm_tol(vocab), "dx")
        total += g.t() @ X
    h.x = x
    R.near(dw, total, h.norm_tol(rows), "dw")


def test_terms_laid_out(ops):
    """fp32 weights whose terms are laid out first, in several pieces, from rows that are apart: the losses' bits are those of
    calls on few rows, which split the weights on their way; targets in both pieces and at their borders."""
    rows, width, vocab, piece = 2100, 4100, 24000, (512 << 20) // (4160 * 6) // 256 * 256
    x, w, targets = problem(rows, width, vocab, F32, left_out=0.1)
    w = torch.cat([w, torch.full((vocab, 3), float("nan"), device="cuda")], 1)[:, :width]
    targets[:4] = torch.tensor([piece - 1, piece, vocab - 1, 0], device="cuda")
    dloss = rand(4, (rows,), std=1.0 / rows)
    # (the terms' piece is in the workspace of the one, and not of the other)
    assert ops._head_workspace(0, rows, width, vocab, 0) > piece * 4160 * 6 > ops._head_workspace(0, 64, width, vocab, 0)
    assert piece < vocab < 2 * piece
    loss, lse = ops.vocab_loss(x, w, targets)
    dx, dw = ops.vocab_loss_backward(x, w, targets, lse, dloss)
    for s in (slice(0, 64), slice(rows - 64, rows)):
        l2, s2 = ops.vocab_loss(x[s], w, targets[s])
        assert torch.equal(l2, loss[s]) and torch.equal(s2, lse[s])
    X, W = x.double(), w.double()
    z = X @ W.t()
    live = targets >= 0
    want = torch.where(live, torch.logsumexp(z, 1) - z.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0)
    h = R.Head.__new__(R.Head)
    h.t, h.x = F32, X
    R.near(loss, want, h.norm_tol(1), "loss")
    g = torch.softmax(z, 1)
    g[torch.arange(rows, device="cuda"), targets.clamp(min=0)] -= 1
    g *= torch.where(live, dloss.double(), 0.0)[:, None]
    R.near(dx, g @ W, h.norm_tol(vocab), "dx")
    R.near(dw, g.t() @ X, h.norm_tol(rows), "dw")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_a_row_alone_and_in_batches(ops, dtype):
    """A row's loss has the same bits in calls of one row and of thousands, from weights at any alignment."""
    rows, width, vocab = 3000, 520, 5000
    x, w, targets = problem(rows, width, vocab, dtype, left_out=0.1)
    targets[:1] = 77
    loss, lse = ops.vocab_loss(x, w, targets)
    apart = torch.cat([w, w[:, :3]], 1)[:, :width]
    for weights in (w, apart):
        for n in (1, 64, 130, 700, 3000):
            l2, s2 = ops.vocab_loss(x[:n], weights, targets[:n])
            assert torch.equal(l2, loss[:n]) and torch.equal(s2, lse[:n])


def test_few_tiles_of_a_long_width(ops):
    """fp32 in few workgroups, from terms laid out (tiles of their own); the losses' bits are those of a larger call."""
    rows, width, vocab = 1300, 3001, 700
    x, w, targets = problem(rows, width, vocab, F32, left_out=0.2)
    loss, lse = ops.vocab_loss(x, w, targets)
    for s in (slice(0, 40), slice(1000, 1130)):
        n = s.stop - s.start
        for backward in (0, 1):
            assert ops._head_workspace(0, n, width, vocab, backward) > 768 * 3008 * 6
        a = check_loss(ops, x[s], w, targets[s], rand(5, (n,), std=1.0 / n))
        assert torch.equal(a[0], loss[s]) and torch.equal(a[1], lse[s])


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_far_weights(ops, dtype):
    """Rows of the weights and of their gradient beyond 2^31 elements, at the largest stride that is taken."""
    vocab, width, ld = 1100, 72, 1 << 21
    x, dense, targets = problem(40, width, vocab, dtype)
    w = torch.empty((vocab - 1) * ld + width, dtype=dtype, device="cuda").as_strided((vocab, width), (ld, 1))
    w.copy_(dense)
    dloss = rand(3, (40,))
    loss, lse = ops.vocab_loss(x, dense, targets)
    dx, dw = ops.vocab_loss_backward(x, dense, targets, lse, dloss, out=dense.clone())
    got = ops.vocab_loss(x, w, targets)
    assert torch.equal(got[0], loss) and torch.equal(got[1], lse)
    # (the gradient in place of a copy of the weights that is as far apart)
    out = torch.empty((vocab - 1) * ld + width, dtype=dtype, device="cuda").as_strided((vocab, width), (ld, 1))
    out.copy_(dense)
    dx2, back = ops.vocab_loss_backward(x, w, targets, lse, dloss, out=out)
    assert back is out and torch.equal(dx2, dx) and torch.equal(out, dw)
    wider = torch.empty((vocab - 1) * (ld + 8) + width, dtype=dtype, device="cuda").as_strided((vocab, width), (ld + 8, 1))
    with pytest.raises(ops.UnError, match="stride of the weight"):
        ops.vocab_loss(x, wider, targets)


def test_against_differences(ops):
    """The gradients against central differences of the definition in 64 bits, in random directions."""
    x, w, targets = problem(40, 24, 90, F32, left_out=0.2)
    dloss = rand(5, (40,))
    _, lse = ops.vocab_loss(x, w, targets)
    grads = ops.vocab_loss_backward(x, w, targets, lse, dloss)
    ids, logits = ints(1, (40, 5), 90), rand(2, (40, 5), std=2.0)
    _, lse2, picked = ops.distill_loss(x, w, ids, logits, temperature=3.0)
    grads2 = ops.distill_loss_backward(x, w, ids, logits, lse2, picked, dloss, temperature=3.0)
    h = 1e-6

    def ce(x, w):
        return (R.cross_entropy(x, w, targets)[1] * R.d(dloss)).sum()

    def kd(x, w):
        return (R.distillation(x, w, ids, logits, 3.0)[1] * R.d(dloss)).sum()

    for f, gs in ((ce, grads), (kd, grads2)):
        base = [R.d(x), R.d(w)]
        for i, g in enumerate(gs):
            v = torch.randn(base[i].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64)
            at = [f(*[b + (k * h * v if j == i else 0) for j, b in enumerate(base)]) for k in (1, -1)]
            want = (at[0] - at[1]) / (2 * h)
            # fp32 gradients: 2e-5 of the terms' magnitudes; the differences themselves are off by h^2 and 1e-16 / h of f
            assert abs((R.d(g) * v).sum() - want) <= 2e-5 * (R.d(g) * v).abs().sum() + 1e-7


# ---------------------------------------------------------------------------
# Distillation
# ---------------------------------------------------------------------------
def check_distill(ops, x, w, ids, logits, T, dloss, onto=None):
    loss, lse, picked = ops.distill_loss(x, w, ids, logits, temperature=T)
    h, wl, el, ws, es, wp, ep = R.distillation(x, w, ids, logits, T)
    R.close(loss, wl, el, "loss")
    R.close(lse, ws, es, "lse")
    R.close(picked, wp, ep, "picked")
    got = ops.distill_loss_backward(x, w, ids, logits, lse, picked, dloss, temperature=T, out=None if onto is None else onto.clone())
    check_grads(h, got, T * R.d(dloss).reshape(-1).expand(h.live.numel()), x.dtype, onto)
    return loss, lse, picked, got


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,width,vocab,top,T", [
    (1, 1, 1, 1, 1.0), (3, 33, 100, 5, 2.0), (64, 64, 256, 1, 1.0), (130, 520, 1000, 20, 4.0), (257, 100, 300, 64, 0.7),
    (70, 2056, 700, 128, 2.0), (513, 264, 4097, 65, 1.0)])
def test_distill_loss(ops, dtype, rows, width, vocab, top, T):
    x, w, _ = problem(rows, width, vocab, dtype)
    ids = torch.stack([torch.randperm(vocab, generator=torch.Generator().manual_seed(k))[:top] for k in range(rows)]).cuda()
    ids = ids.to(torch.int32 if rows % 2 else torch.int64)
    logits = rand(3, (rows, ids.shape[1]), BF16 if top % 2 else F32, std=3.0)
    if rows > 5:
        ids[2, ids.shape[1] // 2:] = -1
        ids[4] = -1
        logits[5, 0] = -float("inf")
    check_distill(ops, x, w, ids, logits, T, rand(9, (rows,), std=1.0 / rows))


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_distill_entries(ops, dtype):
    """Ids that stand twice, outside the vocabulary, masked logits, rows that nothing is left of; values there are not used."""
    x, w, _ = problem(30, 72, 400, dtype)
    ids, logits = ints(1, (30, 6), 400), rand(2, (30, 6), std=2.0)
    ids[0] = 5
    ids[1, :3], ids[2, 4], ids[3, 2] = 7, 400, -9
    logits[4, 1:] = -float("inf")
    logits[5] = -float("inf")
    ids[6] = -1
    dloss = rand(3, (30,))
    loss, lse, picked, (dx, dw) = check_distill(ops, x, w, ids, logits, 2.0, dloss, onto=rand(8, (400, 72), dtype))
    assert (loss[[5, 6]] == 0).all() and (dx[[5, 6]] == 0).all() and (picked[[5, 6]] == 0).all()
    l2 = logits.clone()
    l2[2, 4], l2[3, 2], l2[6] = float("nan"), float("inf"), float("nan")
    x2 = x.clone()
    x2[[5, 6]] = float("nan")
    again = ops.distill_loss(x2, w, ids, l2, temperature=2.0)
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse) and torch.equal(again[2], picked)
    # a single entry is a target, at any temperature a cross entropy of z / T
    t = ints(5, (30,), 400)
    one, _, _ = ops.distill_loss(x, w, t[:, None], torch.zeros(30, 1, device="cuda"))
    ce, e = R.cross_entropy(x, w, t)[1:3]
    R.close(one, ce, e + 1e-5, "loss of one entry")


@pytest.mark.parametrize("logits_type", DTYPES, ids=["f32", "bf16"])
def test_distill_lowest_logits(ops, logits_type):
    """Entries masked with the type's lowest value, at a temperature below 1: none of their probability is left; a row of
    nothing else is one of equal logits."""
    low = torch.finfo(logits_type).min
    x, w, _ = problem(12, 72, 200, F32)
    ids, logits = ints(1, (12, 70), 200), rand(2, (12, 70), logits_type, std=2.0)
    same = logits.clone()
    logits[:4], same[:4] = low, 0.0
    logits[4:8, ::3], same[4:8, ::3] = low, -float("inf")
    logits[8, 1:], same[8, 1:] = low, -float("inf")
    dloss = rand(3, (12,))
    got, want = [], []
    for u, out in ((logits, got), (same, want)):
        loss, lse, picked = ops.distill_loss(x, w, ids, u, temperature=0.5)
        out += [loss, lse, *ops.distill_loss_backward(x, w, ids, u, lse, picked, dloss, temperature=0.5)]
    assert all(t.isfinite().all() for t in got)
    # (an entry without probability is a term of 0 where it counts; its g is the softmax either way, from z by its own
    # products or by the others': off by the logits' product, twice norm_tol's share of it as T is 1/2, and the exponential)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for g, v in zip(got[2:], want[2:]):
        R.near(g, v.double(), R.U32 * (2 * 5 * (6 * 72) ** 0.5 + 24), "gradient")


def test_distill_learned(ops):
    """A student that has the teacher's probabilities: the loss is near 0 and the gradient at the entries cancels to what is
    left over, exactly."""
    w, x = torch.eye(16, device="cuda"), rand(1, (50, 16), std=2.0)
    ids = torch.arange(16, device="cuda").expand(50, 16).contiguous()
    loss, lse, picked = ops.distill_loss(x, w, ids, x, temperature=1.0)
    assert loss.abs().max() <= 200 * R.U32
    dx, _ = ops.distill_loss_backward(x, w, ids, x, lse, picked, torch.ones(50, device="cuda"))
    assert dx.abs().max() <= 200 * R.U32


def test_distill_pieces(ops):
    """Entries in several pieces of the vocabulary."""
    rows, width, vocab, top = 8500, 40, 33000, 4
    x, w, _ = problem(rows, width, vocab, BF16)
    ids, logits, dloss = ints(1, (rows, top), vocab), rand(2, (rows, top), std=2.0), rand(4, (rows,), std=1.0 / rows)
    loss, lse, picked = ops.distill_loss(x, w, ids, logits)
    dx, dw = ops.distill_loss_backward(x, w, ids, logits, lse, picked, dloss)
    total = torch.zeros(vocab, width, dtype=torch.float64, device="cuda")
    h = R.Head.__new__(R.Head)
    h.t = BF16
    for a in range(0, rows, 1700):
        s = slice(a, a + 1700)
        g = torch.softmax(x[s].double() @ w.double().t(), 1).scatter_add_(1, ids[s], -torch.softmax(logits[s].double(), 1))
        g *= dloss[s].double()[:, None]
        h.x = x[s]
        R.near(dx[s], g @ w.double(), h.norm_tol(vocab), "dx")
        total += g.t() @ x[s].double()
    R.near(dw, total, h.norm_tol(rows), "dw")
