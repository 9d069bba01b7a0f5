"""GPU tests of the operators at a language model's ends together: tokens through a
table, a norm and a loss over the same table, and back; streams, captures, versions."""
import pytest

torch = pytest.importorskip("torch")

import _lm_operator_refs as R  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    from paper_2408_01331_amd import operators
    return operators


def rand(seed, shape, dtype=F32, mean=0.0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).cuda()


def ints(seed, shape, high):
    return torch.randint(0, high, shape, generator=torch.Generator().manual_seed(seed)).cuda()


SCALE = 3.0


def step(ops, table, w, b, tokens, targets, ids, logits):
    """A step of a model with one table at both ends: losses of the next token and of a teacher, and all gradients."""
    n = tokens.numel()
    x = ops.embedding(tokens, table, scale=SCALE)
    y, s, stats = ops.layer_norm(x, w, b, keep=True)
    loss, lse = ops.vocab_loss(y, table, targets)
    kd, lse2, picked = ops.distill_loss(y, table, ids, logits, temperature=2.0)
    each = torch.full((), 1.0 / n, device="cuda")
    dy, dtable = ops.vocab_loss_backward(y, table, targets, lse, each)
    dy2, dtable = ops.distill_loss_backward(y, table, ids, logits, lse2, picked, each, temperature=2.0, out=dtable)
    dx, dw, db = ops.layer_norm_backward(dy + dy2, s, w, stats)
    dtable = ops.embedding_backward(dx, tokens, table.shape[0], scale=SCALE, padding=0, out=dtable)
    return loss, kd, dtable, dw, db


def args(seed, dtype=F32, shape=(3, 70), vocab=500, width=72):
    tokens, targets, ids = ints(seed, shape, vocab), ints(seed + 1, shape, vocab), ints(seed + 2, (*shape, 6), vocab)
    targets[0, :5], ids[1, :4], tokens[1, 3] = -100, -1, 0
    return (rand(seed + 3, (vocab, width), dtype, std=0.2), rand(seed + 4, (width,), mean=1.0, std=0.1), rand(seed + 5, (width,), std=0.1),
            tokens, targets, ids, rand(seed + 6, (*shape, 6), std=2.0))


def test_a_step(ops):
    """The losses and gradients against those of torch's autograd for the definitions in 64 bits."""
    a = args(1)
    got = step(ops, *a)
    table, w, b = (R.d(t).requires_grad_() for t in a[:3])
    tokens, targets, ids, logits = a[3].cpu(), a[4].cpu(), a[5].cpu(), R.d(a[6])
    # (padding: the token 0 has no gradient through the lookup)
    x = torch.where((tokens == 0)[..., None], table.detach()[tokens], table[tokens]) * SCALE
    y = torch.nn.functional.layer_norm(x, (72,), w, b, 1e-5)
    z = y @ table.t()
    loss = torch.nn.functional.cross_entropy(z.flatten(0, 1), targets.flatten(), reduction="none", ignore_index=-100).view(targets.shape)
    p = torch.softmax(logits / 2, -1)
    q = torch.log_softmax(z / 2, -1).gather(-1, ids.clamp(min=0))
    kd = torch.where(ids[..., 0] >= 0, 4 * (p * (p.log() - q)).sum(-1), 0.0)
    grads = torch.autograd.grad((loss.sum() + kd.sum()) / tokens.numel(), (table, w, b))
    # fp32 throughout; sums of up to 500 terms, products of six for each: 3000 terms, u sqrt(3000) of |z| <= 12 in g (660 u), as
    # much again in each of the two products and the norm that follow
    for g, want in zip(got, (loss, kd, *grads)):
        assert (R.d(g) - want.detach()).norm() <= 2000 * R.U32 * want.detach().norm()


def test_repeats(ops):
    """The same step twice gives the same bits, with other work in between, and its inputs stay as they are."""
    for dtype in (F32, BF16):
        a = args(7, dtype)
        before = [t.clone() for t in a]
        first = step(ops, *a)
        step(ops, *args(30, dtype, (2, 300), 4000, 200))
        for x, y in zip(step(ops, *a), first):
            assert torch.equal(x, y)
        for x, y in zip(a, before):
            assert torch.equal(x, y)


def test_another_stream(ops):
    """Work on a side stream follows that stream's order: the inputs are written there, after a long run of other work."""
    a = args(5)
    want = step(ops, *a)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        m = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):
            m = m @ m * 1e-2
        late = [t * 1 for t in a]
        got = step(ops, *late)
    s.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)


def test_two_streams_at_once(ops):
    """Two streams do not disturb one another."""
    cases = [args(40 + k, BF16, (4, 200), 3000, 136) for k in range(2)]
    want = [step(ops, *c) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(5):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(step(ops, *cases[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for g in got[k]:
            for x, y in zip(g, want[k]):
                assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,shape,vocab,width", [(F32, (3, 70), 500, 72), (BF16, (2, 150), 9000, 264), (BF16, (3, 800), 700, 80)])
def test_captured(ops, dtype, shape, vocab, width):
    """Captured once, replayed on new inputs with eager steps in between; other numbers of live rows among them."""
    sets = [args(50 * k, dtype, shape, vocab, width) for k in range(3)]
    sets[1][4][:] = -100
    sets[2][5][:, ::2] = -1
    want = [step(ops, *s) for s in sets]
    held = [t.clone() for t in sets[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(ops, *held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(ops, *held)
    for k in (0, 1, 2, 1, 0):
        for t, new in zip(held, sets[k]):
            t.copy_(new)
        graph.replay()
        eager = step(ops, *held)
        torch.cuda.synchronize()
        for a, b, c in zip(out, want[k], eager):
            assert torch.equal(a, b) and torch.equal(c, b)


def test_what_autograd_is_told(ops):
    """Tensors that require gradients are refused where autograd records; what a call adds onto gets a new version."""
    table, w, b, tokens, targets, ids, logits = args(3)
    x, dl = rand(1, (3, 70, 72)), torch.ones((), device="cuda")
    leaf, wleaf = table.clone().requires_grad_(), w.clone().requires_grad_()
    loss, lse = ops.vocab_loss(x, table, targets)
    _, lse2, picked = ops.distill_loss(x, table, ids, logits)
    for call in (lambda: ops.embedding(tokens, leaf), lambda: ops.layer_norm(x, wleaf), lambda: ops.vocab_loss(x, leaf, targets),
                 lambda: ops.vocab_loss_backward(x, leaf, targets, lse, dl), lambda: ops.distill_loss(x, leaf, ids, logits),
                 lambda: ops.distill_loss_backward(x, leaf, ids, logits, lse2, picked, dl),
                 lambda: ops.embedding_backward(x.requires_grad_(), tokens, 500)):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with torch.no_grad():
            call()
    x = x.detach()
    onto = table.clone()
    for call in (lambda: ops.embedding_backward(x, tokens, 500, out=onto), lambda: ops.vocab_loss_backward(x, table, targets, lse, dl, out=onto),
                 lambda: ops.distill_loss_backward(x, table, ids, logits, lse2, picked, dl, out=onto)):
        v = onto._version
        call()
        assert onto._version > v


def test_refusals(ops):
    """Arguments that do not fit are named, before anything runs."""
    table, w, b, tokens, targets, ids, logits = args(3)
    x, dl = rand(1, (3, 70, 72)), torch.ones((), device="cuda")
    loss, lse = ops.vocab_loss(x, table, targets)
    bad = [(lambda: ops.vocab_loss(x, table[:, :71], targets), "weight must have shape"), (lambda: ops.vocab_loss(x, table.to(BF16), targets), "weight must be"),
           (lambda: ops.vocab_loss(x, table, targets[:, :4]), "targets must have shape"), (lambda: ops.vocab_loss(x, table, targets.float()), "targets must be int"),
           (lambda: ops.vocab_loss(x, table, targets.cpu()), "targets must be on"), (lambda: ops.vocab_loss(x, table[0], targets), "weight must have shape"),
           (lambda: ops.vocab_loss_backward(x, table, targets, lse[0], dl), "lse must have shape"),
           (lambda: ops.vocab_loss_backward(x, table, targets, lse, dl.double()), "dloss must be"),
           (lambda: ops.vocab_loss_backward(x, table, targets, lse, 1.0), "dloss must be a tensor"),
           (lambda: ops.vocab_loss_backward(x, table, targets, lse, dl, out=table[:5]), "out must have shape"),
           (lambda: ops.distill_loss(x, table, ids[0], logits), "ids must be a tensor of shape"),
           (lambda: ops.distill_loss(x, table, ids, logits[..., :3]), "logits must have shape"),
           (lambda: ops.distill_loss(x, table, ids, logits.double()), "logits must be a float32 or bfloat16"),
           (lambda: ops.embedding(tokens, table.cpu()), "GPU"), (lambda: ops.embedding(tokens.cpu(), table), "tokens must be on"),
           (lambda: ops.embedding_backward(x, tokens, 500, out=table.to(BF16)), "out must be"),
           (lambda: ops.layer_norm(x, w, b[:5]), "bias must have shape")]
    for call, text in bad:
        with pytest.raises(ValueError, match=text):
            call()
    for call, text in ((lambda: ops.distill_loss(x, table, ids, logits, temperature=0.0), "temperature"),
                       (lambda: ops.distill_loss(x, table, ids, logits, temperature=float("nan")), "temperature"),
                       (lambda: ops.distill_loss(x, table, ids[..., :0], logits[..., :0]), "top >= 1"),
                       (lambda: ops.distill_loss(x, table, ids.repeat(1, 1, 30), logits.repeat(1, 1, 30)), "128"),
                       (lambda: ops.embedding(tokens, table, scale=float("inf")), "scale")):
        with pytest.raises(ops.UnError, match=text):
            call()
