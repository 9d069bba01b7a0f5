"""GPU tests of the embedding lookup and its gradient on device tensors against
their definitions in 64 bits (bounds: _lm_operator_refs.py)."""
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


def rand(seed, shape, dtype=F32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).cuda()


def tokens_of(seed, n, vocab, kind, index=torch.int64):
    """even: every token alike; text: the k-th as 1 / k; one: a single token; outside: some outside the table."""
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(n, generator=g, dtype=torch.float64)
    t = (u * vocab).long() if kind != "text" else (torch.exp(u * torch.log(torch.tensor(vocab + 1.0))) - 1).long()
    t = t.clamp(0, vocab - 1)
    if kind == "one":
        t[:] = vocab // 2
    if kind == "outside":
        t[::3] = torch.tensor([-1, vocab, -2 ** 31, 2 ** 31 - 1])[torch.arange((n + 2) // 3) % 4]
    return t.to(index).cuda()


def check(ops, dtype, tokens, vocab, width, scale=1.0, padding=None, onto=None, seed=0):
    w, dy = rand(seed, (vocab, width), dtype), rand(seed + 1, (*tokens.shape, width), dtype)
    y = ops.embedding(tokens, w, scale=scale)
    want = R.embedding(tokens, w, scale)
    # the call holds the scale in fp32: |fl(s) - s| <= u |s|, so s w is off by u of itself before its own rounding, and
    # (1 + u)(1 + u) - 1 <= 2.0001 u; a stored type's step comes on top
    step = 2.0001 * R.U32 + (R.half_step(dtype) if dtype != F32 else 0)
    R.close(y, want, want.abs() * step, "y")
    dw = ops.embedding_backward(dy, tokens, vocab, scale=scale, padding=padding, out=None if onto is None else onto.clone())
    want, bound = R.embedding_backward(dy, tokens, vocab, scale, padding, onto)
    R.close(dw, want, bound + (R.half_step(dtype) * (want.abs() + bound) if dtype != F32 else 0), "dw")
    return dy, dw


SIZES = [(1, 1, 1), (1, 50, 7), (5, 3, 8), (64, 1000, 100), (33, 70, 520), (1000, 600, 36), (8192, 300, 12), (8193, 70000, 9),
         (5003, 10007, 33), (20000, 5000, 40), (0, 40, 16), (70, 300000, 5), (9000, 5000000, 1)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,width", SIZES)
@pytest.mark.parametrize("kind", ["even", "text", "one", "outside"])
def test_embedding(ops, dtype, n, vocab, width, kind):
    index = torch.int32 if kind in ("text", "outside") and n % 2 else torch.int64
    check(ops, dtype, tokens_of(1, n, vocab, kind, index), vocab, width, scale=1.0 if kind == "even" else 3.3)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n,kind", [(40, "text"), (300, "even"), (9000, "text"), (9000, "one")])
def test_onto(ops, dtype, n, kind):
    """Added onto what is there, in rows that are apart; rows that no token names, and what lies between, keep their bits."""
    vocab, width = 500, 77
    wide = rand(5, (vocab, 90), dtype)
    wide[3] = float("nan")
    onto = wide[:, 6:83]
    t = tokens_of(2, n, vocab, kind)
    t[t == 3] = 4
    dy = rand(1, (n, width), dtype)
    before = wide.clone()
    got = ops.embedding_backward(dy, t, vocab, scale=0.5, padding=7, out=onto)
    assert got.data_ptr() == onto.data_ptr()
    keep = torch.ones_like(wide, dtype=torch.bool)
    named = torch.unique(t)
    named = named[named != 7]
    keep[named, 6:83] = False
    same = (wide == before) | (wide != wide) & (before != before)
    assert same[keep].all()
    rows = named.cpu()
    want, bound = R.embedding_backward(dy, t, vocab, 0.5, 7, before[:, 6:83])
    want, bound = want[rows], bound[rows]
    R.close(onto[named], want, bound + (R.half_step(dtype) * (want.abs() + bound) if dtype != F32 else 0), "out")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_padding_and_values_in_masked_places(ops, dtype):
    """Rows of dy at padding or at tokens outside the table are not used, whatever they hold."""
    t = tokens_of(3, 700, 40, "outside")
    t[5::7] = 11
    dy = rand(4, (700, 65), dtype)
    clean = ops.embedding_backward(dy, t, 40, padding=11)
    out = (t < 0) | (t >= 40) | (t == 11)
    dy2 = dy.clone()
    dy2[out] = float("nan")
    dy2[torch.nonzero(out)[0, 0]] = float("inf")
    got = ops.embedding_backward(dy2, t, 40, padding=11)
    assert torch.equal(got, clean) and (got[11] == 0).all()
    everything = torch.full((30,), 11, device="cuda")
    assert (ops.embedding_backward(rand(1, (30, 9), dtype), everything, 40, padding=11) == 0).all()
    dy2[torch.nonzero(~out)[0, 0], 3] = float("nan")
    got = ops.embedding_backward(dy2, t, 40, padding=11)
    hit = t[torch.nonzero(~out)[0, 0]]
    assert torch.isnan(got[hit, 3]) and torch.isnan(got).sum() == 1


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_strides_and_shapes(ops, dtype):
    """A table and a gradient inside wider buffers at every alignment of the element; tokens of any shape and order."""
    for off in (0, 1, 3):
        w = rand(off, (30, 150), dtype)[:, off:off + 101]
        dy = rand(off + 9, (2, 17, 150), dtype)[..., off:off + 101]
        t = tokens_of(off, 34, 30, "even").view(17, 2).t()
        y = ops.embedding(t, w, scale=2.0)
        assert y.shape == (2, 17, 101) and torch.equal(y, (w[t].float() * 2).to(dtype))
        assert torch.equal(ops.embedding_backward(dy, t, 30), ops.embedding_backward(dy.contiguous(), t.contiguous(), 30))
    assert ops.embedding(torch.tensor(3, device="cuda"), w).shape == (101,)


def test_order_and_repeats(ops):
    """The same call gives the same bits, and the sum of a token's rows does not depend on the other tokens' values."""
    t = tokens_of(1, 30000, 2000, "text")
    dy = rand(2, (30000, 64))
    first = ops.embedding_backward(dy, t, 2000)
    for _ in range(3):
        assert torch.equal(ops.embedding_backward(dy, t, 2000), first)
    assert torch.equal(ops.embedding_backward(dy, t.int(), 2000), first)
    perm = torch.randperm(2000, generator=torch.Generator().manual_seed(1)).cuda()
    assert not torch.equal(t, perm[t])


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [700, 30000])
def test_other_tokens_rows(ops, dtype, n):
    """With the same tokens a row of the table has the same bits, whatever the other tokens' rows of dy hold; with others its
    terms are the same and may be grouped otherwise."""
    t = tokens_of(1, n, 2000, "text")
    dy = rand(2, (n, 64), dtype)
    first = ops.embedding_backward(dy, t, 2000)
    for watched in (t < 3, t % 2 == 1, t == t[n // 2]):
        other = torch.where(watched[:, None], dy, rand(3, (n, 64), dtype) * 100)
        other[torch.nonzero(~watched)[0, 0]] = float("nan")
        rows = torch.unique(t[watched])
        assert torch.equal(ops.embedding_backward(other, t, 2000)[rows], first[rows])
    moved = torch.where(t == 0, 1999, t)  # every run lies elsewhere
    want, bound = R.embedding_backward(dy, moved, 2000, 1.0, None, None)
    R.close(ops.embedding_backward(dy, moved, 2000), want, bound + (R.half_step(dtype) * (want.abs() + bound) if dtype != F32 else 0), "dw")


def test_far_rows(ops):
    """Rows beyond 2^31 elements of a table."""
    vocab, width = 600_000, 4096
    w = torch.empty(vocab, width, dtype=BF16, device="cuda")
    t = torch.tensor([0, vocab - 1, 550_000, 3], device="cuda")
    w[t] = rand(1, (4, width), BF16)
    assert torch.equal(ops.embedding(t, w), w[t])
    del w
    dy = rand(2, (4, width), BF16)
    dw = ops.embedding_backward(dy, t, vocab)
    assert torch.equal(dw[t], dy)
    dw[t] = 0
    assert not dw.any()


def test_far_tokens(ops):
    """Rows beyond 2^31 elements of the output and of its gradient."""
    n, vocab, width = 600_000, 700, 4096
    w, t = rand(1, (vocab, width), BF16), tokens_of(3, n, vocab, "even")
    y = ops.embedding(t, w)
    for a in range(0, n, 100_000):
        assert torch.equal(y[a:a + 100_000], w[t[a:a + 100_000]])
    y.zero_()
    far = torch.tensor([0, 524_288, 524_289, n - 1], device="cuda")
    t[far] = torch.tensor([5, 6, 7, 6], device="cuda")
    y[far] = rand(2, (4, width), BF16)
    dw = ops.embedding_backward(y, t, vocab)
    assert torch.equal(dw[5], y[far[0]]) and torch.equal(dw[7], y[far[2]])
    assert torch.equal(dw[6], (y[far[1]].float() + y[far[3]].float()).to(BF16))
    dw[5:8] = 0
    assert not dw.any()


def test_against_autograd(ops):
    """Lookup and gradient against torch's autograd of the definition in 64 bits."""
    w, t, dy = rand(1, (50, 33)), tokens_of(1, 200, 50, "text").view(4, 50), rand(3, (4, 50, 33))
    W = R.d(w).requires_grad_()
    out = W[t.cpu()] * 1.7
    want, = torch.autograd.grad(out, W, R.d(dy))
    R.close(ops.embedding(t, w, scale=1.7), out.detach(), out.detach().abs() * 2 * R.U32, "y")
    _, bound = R.embedding_backward(dy, t, 50, 1.7, None, None)
    R.close(ops.embedding_backward(dy, t, 50, scale=1.7), want, bound, "dw")
