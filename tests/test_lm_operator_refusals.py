"""CPU tests of the checks of the operators at the ends of a language model: every
refusal happens on the host, before anything reaches a device."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2408_01331_amd import unifiednn as U  # noqa: E402

P = 0x1000  # an address that is never used: every call here is refused


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(U.LIB_PATH):
        from paper_2408_01331_amd.build import build
        build()
    U.lib()


def refused(fn, struct, base, change, want, text):
    args = getattr(U, struct)(**{**base, **change})
    s = getattr(U.lib(), fn)(ctypes.byref(args), None)
    msg = U.lib().un_last_error(None).decode()
    assert s == want, msg
    assert text in msg and "un_" in msg


# ---------------------------------------------------------------------------
# Layer norm
# ---------------------------------------------------------------------------
NORM = dict(type=0, width=64, rows=4, eps=1e-6, x=P, ldx=64, weight=P, y=P, ldy=64)
NORMG = dict(type=1, width=64, rows=4, dy=P, lddy=64, s=P, lds=64, weight=P, stats=P, dx=P, lddx=64, dweight=P, workspace=P,
             workspace_bytes=1 << 20)


@pytest.mark.parametrize("change,want,text", [
    (dict(type=2), 1, "type"), (dict(width=0), 1, "width"), (dict(rows=-1), 1, "rows"),
    (dict(width=16385, ldx=20000, ldy=20000), 7, "16384"), (dict(eps=-1.0), 1, "eps"), (dict(eps=float("nan")), 1, "eps"),
    (dict(x=None), 1, "NULL"), (dict(weight=None), 1, "NULL"), (dict(y=None), 1, "NULL"), (dict(ldx=63), 1, "stride"),
    (dict(ldy=63), 1, "stride"), (dict(residual=P, ldr=1), 1, "stride"), (dict(sum=P, lds=0), 1, "stride"), (dict(rows=1 << 40), 7, "rows"),
])
def test_layer_norm_refused(change, want, text):
    refused("un_layer_norm", "un_layer_norm_args", NORM, change, want, text)


@pytest.mark.parametrize("change,want,text", [
    (dict(type=-1), 1, "type"), (dict(rows=-1), 1, "rows"), (dict(width=16385), 7, "16384"), (dict(workspace_bytes=0), 6, "workspace"),
    (dict(workspace=None), 6, "workspace"), (dict(stats=None), 1, "NULL"), (dict(dweight=None), 1, "NULL"), (dict(s=None), 1, "NULL"),
    (dict(ds=P, ldds=3), 1, "stride"), (dict(lddx=3), 1, "stride"),
])
def test_layer_norm_backward_refused(change, want, text):
    refused("un_layer_norm_backward", "un_layer_norm_grad_args", NORMG, change, want, text)


def test_null_arguments():
    for fn in ("un_layer_norm", "un_layer_norm_backward"):
        assert getattr(U.lib(), fn)(None, None) == U.UN_ERR_INVALID
        assert fn in U.lib().un_last_error(None).decode()


def test_no_rows():
    assert U.lib().un_layer_norm(ctypes.byref(U.un_layer_norm_args(**{**NORM, "rows": 0, "x": None})), None) == U.UN_OK


def test_layer_norm_python():
    from paper_2408_01331_amd import operators as ops
    x, w = torch.zeros(4, 8), torch.zeros(8)
    with pytest.raises(ValueError, match="GPU"):
        ops.layer_norm(x, w)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        ops.layer_norm(x.half(), w)
    with pytest.raises(ValueError, match="s must be a tensor"):
        ops.layer_norm_backward(x, None, w, w)


# ---------------------------------------------------------------------------
# Embedding
# ---------------------------------------------------------------------------
EMBED = dict(type=0, width=64, vocab=10, index_bits=64, tokens=4, ids=P, weight=P, ldw=64, scale=1.0, y=P, ldy=64)
EMBEDG = dict(type=1, width=64, vocab=10, index_bits=32, tokens=4, ids=P, dy=P, lddy=64, scale=1.0, padding=-1, dweight=P, lddw=64,
              workspace=P, workspace_bytes=1 << 20)
SIZES = [(dict(type=3), 1, "type"), (dict(width=0), 1, "width"), (dict(vocab=0), 1, "vocab"), (dict(tokens=-1), 1, "tokens"),
         (dict(index_bits=16), 1, "index_bits"), (dict(vocab=(1 << 31) - 1), 7, "vocabulary"), (dict(tokens=(1 << 30) + 1), 7, "2^30"),
         (dict(width=(1 << 24) + 1), 7, "2^24"), (dict(width=4096, tokens=1 << 30), 7, "too many"), (dict(scale=float("inf")), 1, "scale"),
         (dict(ids=None), 1, "NULL")]


@pytest.mark.parametrize("change,want,text", SIZES + [
    (dict(weight=None), 1, "NULL"), (dict(y=None), 1, "NULL"), (dict(ldw=63), 1, "stride"), (dict(ldy=63), 1, "stride")])
def test_embedding_refused(change, want, text):
    refused("un_embedding", "un_embedding_args", EMBED, change, want, text)


@pytest.mark.parametrize("change,want,text", SIZES + [
    (dict(dy=None), 1, "NULL"), (dict(dweight=None), 1, "NULL"), (dict(lddw=63), 1, "stride"), (dict(lddy=63), 1, "stride"),
    (dict(workspace=None), 6, "workspace"), (dict(workspace_bytes=10), 6, "workspace"), (dict(workspace=P + 4), 1, "aligned")])
def test_embedding_backward_refused(change, want, text):
    refused("un_embedding_backward", "un_embedding_grad_args", EMBEDG, change, want, text)


def test_embedding_without_tokens():
    L = U.lib()
    assert L.un_embedding(ctypes.byref(U.un_embedding_args(**{**EMBED, "tokens": 0, "y": None})), None) == U.UN_OK
    assert L.un_embedding_backward(ctypes.byref(U.un_embedding_grad_args(**{**EMBEDG, "tokens": 0, "accumulate": 1})), None) == U.UN_OK
    for fn in ("un_embedding", "un_embedding_backward"):
        assert getattr(L, fn)(None, None) == U.UN_ERR_INVALID


def test_embedding_workspace():
    b = ctypes.c_size_t(5)
    assert U.lib().un_embedding_workspace(0, 10, 64, ctypes.byref(b)) == U.UN_OK and b.value == 0
    assert U.lib().un_embedding_workspace(100, 10, 64, ctypes.byref(b)) == U.UN_OK and b.value >= 100 * 16
    assert U.lib().un_embedding_workspace(100, 10, 0, ctypes.byref(b)) == U.UN_ERR_INVALID
    assert U.lib().un_embedding_workspace(100, 10, 64, None) == U.UN_ERR_INVALID


@pytest.mark.parametrize("tokens,vocab,width", [((1 << 26) - 18, 10, 256), ((1 << 25) - 9, 10, 257), (1, (1 << 26) - 9, 1),
                                               ((1 << 18) - 1, 262391, 65280)])
def test_embedding_at_the_limit(tokens, vocab, width):
    """tokens * ceil(width / 256) + vocab = 2^26 - 8 is the most that a launch holds."""
    assert tokens * -(-width // 256) + vocab == (1 << 26) - 8
    b = ctypes.c_size_t()
    assert U.lib().un_embedding_workspace(tokens, vocab, width, ctypes.byref(b)) == U.UN_OK and b.value > 0
    for fn, struct, base in (("un_embedding", "un_embedding_args", EMBED), ("un_embedding_backward", "un_embedding_grad_args", EMBEDG)):
        size = dict(tokens=tokens, vocab=vocab, width=width)
        refused(fn, struct, base, {**size, "ids": None}, 1, "NULL")
        refused(fn, struct, base, {**size, "vocab": vocab + 1}, U.UN_ERR_UNSUPPORTED, "too many")


def test_embedding_python(monkeypatch):
    from paper_2408_01331_amd import operators as ops
    w, t = torch.zeros(5, 8), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        ops.embedding(t, w)
    monkeypatch.setattr(ops, "_check_type", lambda x, name: (0, -1))  # (a CPU tensor's device has the number -1)
    with pytest.raises(ValueError, match=r"weight must have shape \[vocab, width\]"):
        ops.embedding(t, w[0])
    with pytest.raises(ValueError, match="rows must not overlap"):
        ops.embedding(t, torch.zeros(8).expand(5, 8))
    with pytest.raises(ValueError, match="last axis"):
        ops.embedding(t, w.t())
    with pytest.raises(ValueError, match="tokens must be int32 or int64"):
        ops.embedding(t.float(), w)
    with pytest.raises(ValueError, match="tokens must be a tensor"):
        ops.embedding([1], w)
    with pytest.raises(ValueError, match="requires a gradient"):
        ops.embedding(t, w.clone().requires_grad_())
    with pytest.raises(ValueError, match="dy must have shape"):
        ops.embedding_backward(torch.zeros(4, 8), t, 5)
    with pytest.raises(ValueError, match="vocab must be"):
        ops.embedding_backward(torch.zeros(3, 8), t, 0)
    with pytest.raises(ValueError, match="out must have shape"):
        ops.embedding_backward(torch.zeros(3, 8), t, 5, out=torch.zeros(4, 8))
    with pytest.raises(ValueError, match="out's rows must not overlap"):
        ops.embedding_backward(torch.zeros(3, 8), t, 5, out=torch.zeros(8).expand(5, 8))


# ---------------------------------------------------------------------------
# Losses over a vocabulary
# ---------------------------------------------------------------------------
HEAD = dict(type=0, width=64, vocab=10, index_bits=64, rows=4, x=P, ldx=64, weight=P, ldw=64, lse=P, workspace=P, workspace_bytes=1 << 30)
GRADS = dict(dloss=P, dloss_stride=1, dx=P, lddx=64, dweight=P, lddw=64)
TEACHER = dict(top=3, logits_type=1, ids=P, logits=P, temperature=1.0, picked=P)
CALLS = {"un_vocab_loss": ("un_vocab_loss_args", {**HEAD, "targets": P, "loss": P}),
         "un_vocab_loss_backward": ("un_vocab_loss_grad_args", {**HEAD, **GRADS, "targets": P}),
         "un_distill_loss": ("un_distill_loss_args", {**HEAD, **TEACHER, "loss": P}),
         "un_distill_loss_backward": ("un_distill_loss_grad_args", {**HEAD, **GRADS, **TEACHER})}


@pytest.mark.parametrize("fn", CALLS)
@pytest.mark.parametrize("change,want,text", [
    (dict(type=2), 1, "type"), (dict(rows=-1), 1, "rows"), (dict(width=0), 1, "width"), (dict(vocab=0), 1, "vocab"),
    (dict(width=65537, ldx=70000, ldw=70000, lddx=70000, lddw=70000), 7, "65536"), (dict(rows=(1 << 24) + 1), 7, "2^24"),
    (dict(vocab=(1 << 30) + 1), 7, "2^30"), (dict(rows=1 << 24, vocab=1 << 24), 7, "too many"), (dict(index_bits=8), 1, "index_bits"),
    (dict(x=None), 1, "NULL"), (dict(weight=None), 1, "NULL"), (dict(lse=None), 1, "NULL"), (dict(ldx=63), 1, "stride"),
    (dict(ldw=63), 1, "stride"), (dict(ldw=(1 << 21) + 1), 7, "2^21"), (dict(workspace=None), 6, "workspace"),
    (dict(workspace_bytes=100), 6, "workspace"), (dict(workspace=P + 8), 1, "aligned")])
def test_head_refused(fn, change, want, text):
    struct, base = CALLS[fn]
    known = {k for k, _ in getattr(U, struct)._fields_}
    refused(fn, struct, base, {k: v for k, v in change.items() if k in known}, want, text)


@pytest.mark.parametrize("fn,change,want,text", [
    ("un_vocab_loss", dict(targets=None), 1, "NULL"), ("un_vocab_loss", dict(loss=None), 1, "NULL"),
    ("un_vocab_loss_backward", dict(targets=None), 1, "NULL"), ("un_distill_loss", dict(loss=None), 1, "NULL"),
    *[(fn, change, 1, text) for fn in ("un_vocab_loss_backward", "un_distill_loss_backward") for change, text in (
        (dict(dloss=None), "NULL"), (dict(dx=None), "NULL"), (dict(dweight=None), "NULL"), (dict(lddx=63), "stride"), (dict(lddw=63), "stride"),
        (dict(dloss_stride=-1), "stride"))],
    *[(fn, change, want, text) for fn in ("un_distill_loss", "un_distill_loss_backward") for change, want, text in (
        (dict(top=0), 1, "top"), (dict(top=129), 7, "128"), (dict(logits_type=3), 1, "logits"), (dict(temperature=0.0), 1, "temperature"),
        (dict(temperature=-1.0), 1, "temperature"), (dict(temperature=float("inf")), 1, "temperature"), (dict(ids=None), 1, "NULL"),
        (dict(logits=None), 1, "NULL"), (dict(picked=None), 1, "NULL"))]])
def test_head_refused_more(fn, change, want, text):
    struct, base = CALLS[fn]
    refused(fn, struct, base, change, want, text)


@pytest.mark.parametrize("fn", ["un_distill_loss", "un_distill_loss_backward"])
def test_temperatures_whose_square_is_lost(fn):
    """T^2 is 0 or infinite in 32 bits: the loss would be 0, infinite or NaN whatever the student has learned."""
    struct, base = CALLS[fn]
    for T in (1e-25, 2.0 ** -61, 2.0 ** 61, 1e20, 3e38, 1e-40):
        refused(fn, struct, base, dict(temperature=T), U.UN_ERR_UNSUPPORTED, "temperature")
    for T in (2.0 ** -60, 2.0 ** 60):  # the ends are taken: the next check's refusal
        refused(fn, struct, base, dict(temperature=T, ids=None), 1, "NULL")


def test_head_without_rows_or_arguments():
    L = U.lib()
    for fn, (struct, base) in CALLS.items():
        assert getattr(L, fn)(None, None) == U.UN_ERR_INVALID and fn in L.un_last_error(None).decode()
        if "backward" not in fn:
            a = getattr(U, struct)(**{**base, "rows": 0, "x": None, "workspace": None})
            assert getattr(L, fn)(ctypes.byref(a), None) == U.UN_OK


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("rows,width,vocab", [(0, 8, 8), (1, 1, 1), (777, 500, 10007), (8192, 2048, 131072), (1 << 18, 4096, 200000), (7, 65536, 1 << 20)])
def test_head_workspace(kind, backward, rows, width, vocab):
    """Grows with the problem and stays far below the logits of a large one; a call with other strides needs no more."""
    b = ctypes.c_size_t()
    assert U.lib().un_vocab_workspace(kind, rows, width, vocab, backward, ctypes.byref(b)) == U.UN_OK
    assert b.value > 0 or rows == 0
    if rows * vocab > 1 << 29:
        assert b.value < rows * vocab * 4
    assert U.lib().un_vocab_workspace(kind, rows, 0, vocab, backward, ctypes.byref(b)) == U.UN_ERR_INVALID
    assert U.lib().un_vocab_workspace(kind, rows, width, vocab, backward, None) == U.UN_ERR_INVALID
