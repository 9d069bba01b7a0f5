"""CPU tests of the operators' checks of sizes, of overlapping tensors and of messages."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2408_01331_amd import unifiednn as U  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not os.path.exists(U.LIB_PATH):
        from paper_2408_01331_amd.build import build
        build()
    U.lib()


# ---------------------------------------------------------------------------
# Sizes of the recurrence's states and workspace
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("batch,tokens,width,text", [
    (1, (1 << 30) + 1, 8, "tokens"), (1, (1 << 31) - 1, 8, "tokens"), (1, (1 << 31) - 60, 1, "tokens"),
    (1, 100, 1 << 24, "width"), (1, 100, (1 << 31) - 1, "width"), (1, (1 << 31) - 1, (1 << 31) - 1, "tokens"),
    ((1 << 31) - 1, 16, 64, "too many"), (1, 1 << 30, 100, "too many"), ((1 << 31) - 1, 1 << 30, (1 << 24) - 1, "too many"),
])
def test_scan_sizes_refused(batch, tokens, width, text):
    """Sizes that no call takes have no workspace either, up to the largest that the arguments can name."""
    n, b = ctypes.c_size_t(7), ctypes.c_size_t(7)
    assert U.lib().un_gated_scan_sizes(batch, tokens, width, ctypes.byref(n), ctypes.byref(b)) == U.UN_ERR_UNSUPPORTED
    assert text in U.lib().un_last_error(None).decode() and (n.value, b.value) == (7, 7)


@pytest.mark.parametrize("batch,tokens,width", [(1, 1 << 30, 1), (1, 1 << 30, 64), (3, 5, (1 << 24) - 1), (1 << 25, 16, 64)])
def test_scan_sizes_at_the_limits(batch, tokens, width):
    """A state every 64 tokens; the workspace, where there is one, holds a word per segment, sequence and channel at least."""
    n, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert U.lib().un_gated_scan_sizes(batch, tokens, width, ctypes.byref(n), ctypes.byref(b)) == U.UN_OK
    assert n.value == batch * -(-tokens // 64) * width
    assert (b.value >= 8 * (tokens // 256) * batch * width) if tokens > 1 << 20 else b.value == 0


# ---------------------------------------------------------------------------
# Tensors that overlap
# ---------------------------------------------------------------------------
def test_disjoint():
    """What is written shares no memory with anything; what is only read may share it with what is only read."""
    from paper_2408_01331_amd.operators import _disjoint
    x = torch.zeros(100)
    cut = lambda a, b: x[a:b]  # noqa: E731
    assert _disjoint([], []) and _disjoint([cut(0, 10), cut(10, 20)], [cut(20, 30), cut(20, 30), cut(25, 40)])
    assert _disjoint([cut(5, 5), cut(0, 10)], [cut(3, 3)])  # empty ones share nothing
    assert _disjoint([cut(40, 50)], [cut(0, 40), cut(10, 20), cut(50, 100)])
    for written, read in (([cut(0, 10), cut(9, 20)], []), ([cut(0, 10), cut(0, 10)], []), ([cut(0, 10)], [cut(0, 10)]),
                          ([cut(0, 10)], [cut(9, 12)]), ([cut(9, 12)], [cut(0, 10)]), ([cut(5, 6)], [cut(0, 100), cut(1, 2)]),
                          ([cut(0, 100), cut(200, 200)], [cut(99, 100)]), ([cut(0, 60), cut(80, 90)], [cut(70, 75), cut(20, 30)]),
                          ([cut(50, 60).view(torch.uint8), cut(10, 20)], [cut(59, 61)])):
        assert not _disjoint(written, read)


# ---------------------------------------------------------------------------
# Autograd
# ---------------------------------------------------------------------------
def test_tensors_that_require_gradients():
    """Refused where autograd records, taken where it does not."""
    from paper_2408_01331_amd.operators import _unrecorded
    x, leaf = torch.zeros(3), torch.zeros(3, requires_grad=True)
    _unrecorded(x, None, leaf.detach())
    for args in ((leaf,), (x, None, leaf), (x, leaf * 2)):
        with pytest.raises(ValueError, match="requires a gradient.*no_grad"):
            _unrecorded(*args)
        with torch.no_grad():
            _unrecorded(*args)
        with torch.inference_mode():
            _unrecorded(*args)


# ---------------------------------------------------------------------------
# Messages
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("shape", [(), (1,), (4, 1), (4, 3)])
def test_messages_of_dense_arguments(shape):
    """What does not fit is named, of tensors without axes too; contiguity only where nothing else is wrong."""
    from paper_2408_01331_amd.operators import _flat
    fits = torch.zeros(shape)
    _flat(fits, "rstd", shape, torch.float32, -1)  # (a CPU tensor's device has the number -1)
    for bad, text in ((fits[None], "shape"), (fits.double(), "float32"), (1.0, "a tensor"), (None, "a tensor")):
        with pytest.raises(ValueError, match=f"rstd must .*{text}"):
            _flat(bad, "rstd", shape, torch.float32, -1)
    with pytest.raises(ValueError, match="rstd must be on cuda:0"):
        _flat(fits, "rstd", shape, torch.float32, 0)
    if len(shape) == 2:
        with pytest.raises(ValueError, match="contiguous"):
            _flat(torch.zeros(8, shape[1])[::2], "rstd", shape, torch.float32, -1)


def test_step_of_a_closed_plan():
    from paper_2408_01331_amd.operators import AdamW
    opt = AdamW.__new__(AdamW)
    opt._plan = None
    opt.close()
    with pytest.raises(ValueError, match="closed"):
        opt.step(0.1, 1)


def test_adamw_without_gradients(monkeypatch):
    """A parameter's grad before any backward pass is None: refused by name."""
    from paper_2408_01331_amd import operators as ops
    monkeypatch.setattr(ops, "_check_type", lambda x, name: (0, 0))  # (a CPU tensor would be refused first)
    w = torch.zeros(3)
    with pytest.raises(ValueError, match=r"grads\[0\] must be a tensor"):
        ops.AdamW([w], [None], [w.clone()], [w.clone()])
