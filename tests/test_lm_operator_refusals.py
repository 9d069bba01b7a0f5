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
