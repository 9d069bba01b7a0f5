"""Results of the operators at the ends of a language model that are added onto a
tensor of the caller's: memory that an input still holds is refused, rows that lie
between an input's are taken. (The checks on the CPU, the calls on the GPU.)"""
import random

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ops():
    from paper_2408_01331_amd import operators
    return operators


def test_pieces_of_memory(ops):
    """Whether two sets of rows share a byte, against the bytes themselves."""
    rng = random.Random(1)
    met = 0
    for _ in range(20000):
        na, nb, wa, wb = (rng.randint(0, 5) for _ in range(4))
        la, lb = wa + rng.randint(0, 6) + (wa == 0), rng.randint(0, 11)
        if rng.random() < 0.4:
            lb = la
        a, b = (100, na, la, wa), (100 + rng.randint(-40, 40), nb, lb, wb)
        sa, sb = ({p + i * ld + j for i in range(n) for j in range(w)} for p, n, ld, w in (a, b))
        assert ops._meet(a, b) == bool(sa & sb), (a, b)
        met += bool(sa & sb)
    assert 2000 < met < 18000


def test_rows_of_a_tensor(ops):
    halves = torch.zeros(7, 16, dtype=torch.bfloat16)
    at = halves.data_ptr()
    for size, scale in ((2, 1), (4, 2)):  # (of fp32 the same rows are half as many values)
        out = halves[:, :8] if size == 2 else halves.view(torch.float32)[:, :4]
        ops._apart(out, 16 // scale, size, ("tokens", at + 300, 1, 0, 9), ("weight", at + 16, 7, 32, 16), ("lse", at, 1, 0, 0), ("x", at, 0, 32, 16))
        for b in ((at + 14, 7, 32, 16), (at + 16, 7, 32, 17), (at + 6 * 32 + 15, 1, 0, 4), (at - 3, 1, 0, 4)):
            with pytest.raises(ValueError, match="out overlaps weight"):
                ops._apart(out, 16 // scale, size, ("x", at + 16, 7, 32, 16), ("weight", *b))


def test_refused(ops, monkeypatch):
    """Every input of every call that adds onto a tensor, before anything reaches a device."""
    monkeypatch.setattr(ops, "_check_type", lambda x, name: (0, -1))  # (a CPU tensor's device has the number -1)
    rows, vocab, width, top = 6, 40, 10, 3
    out = torch.zeros(vocab, width)
    some = lambda n, dtype=torch.float32: out.view(-1)[18:18 + n].view(dtype)  # noqa: E731
    x, w = torch.zeros(rows, width), torch.zeros(vocab, width)
    t, lse, dl = torch.zeros(rows, dtype=torch.int32), torch.zeros(rows), torch.zeros(rows)
    ids, lo, picked = torch.zeros(rows, top, dtype=torch.int32), torch.zeros(rows, top), torch.zeros(rows, top)
    ce = dict(x=x, weight=w, targets=t, lse=lse, dloss=dl)
    kd = dict(x=x, weight=w, ids=ids, logits=lo, lse=lse, picked=picked, dloss=dl)
    for call, args in ((ops.vocab_loss_backward, ce), (ops.distill_loss_backward, kd)):
        for name in args:
            bad = out if name == "weight" else some(args[name].numel(), args[name].dtype).view(args[name].shape)
            with pytest.raises(ValueError, match=f"out overlaps {name}"):
                call(**{**args, name: bad}, out=out)
        with pytest.raises(ValueError, match="out overlaps dloss"):
            call(**{**args, "dloss": out[3, 4]}, out=out)
        with pytest.raises(ValueError, match="out overlaps dloss"):
            call(**{**args, "dloss": out[:rows, 4]}, out=out)
    tokens = torch.zeros(rows, dtype=torch.int64)
    with pytest.raises(ValueError, match="out overlaps dy"):
        ops.embedding_backward(out[10:10 + rows], tokens, vocab, out=out)
    with pytest.raises(ValueError, match="out overlaps tokens"):
        ops.embedding_backward(x, some(2 * rows, torch.int64), vocab, out=out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_rows_between_an_inputs(ops, dtype):
    """A table and its gradient as the halves of one buffer's rows, and hidden states between the gradient's rows."""
    g = torch.Generator().manual_seed(1)
    rand = lambda *shape: torch.randn(shape, generator=g).to(dtype).cuda()  # noqa: E731
    vocab, width, rows = 300, 40, 30
    both = rand(vocab, 2 * width)
    w, out = both[:, :width], both[:, width:]
    x, dl = rand(rows, width), torch.full((), 0.5, device="cuda")
    t = torch.randint(0, vocab, (rows,), generator=g).cuda()
    want_w = w.clone()
    loss, lse = ops.vocab_loss(x, want_w, t)
    dx, dw = ops.vocab_loss_backward(x, want_w, t, lse, dl, out=out.clone())
    got = ops.vocab_loss_backward(x, w, t, lse, dl, out=out)
    assert torch.equal(got[0], dx) and torch.equal(out, dw) and torch.equal(w, want_w)
    wide = rand(vocab, 2 * width + 3)  # the rows of dy between those of the table's gradient
    dy, onto = wide[:rows, width + 3:], wide[:, :width]
    want = ops.embedding_backward(dy.contiguous(), t, vocab, out=onto.clone())
    assert torch.equal(ops.embedding_backward(dy, t, vocab, out=onto), want) and torch.equal(onto, want)
    with pytest.raises(ValueError, match="out overlaps weight"):
        ops.vocab_loss_backward(x, w, t, lse, dl, out=w)
