"""CPU tests of the operators' checks: every refusal happens on the host, before
anything reaches a device, with the documented status and a message of the call."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2408_01331_amd import unifiednn as U  # noqa: E402

P = 0x1000  # an address that is never used: every call here is refused


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import os
    if not os.path.exists(U.LIB_PATH):
        from paper_2408_01331_amd.build import build
        build()
    U.lib()


def status(fn, args):
    s = getattr(U.lib(), fn)(ctypes.byref(args) if args is not None else None, None)
    return s, U.lib().un_last_error(None).decode()


NORM = dict(type=0, width=64, rows=4, eps=1e-6, x=P, ldx=64, weight=P, y=P, ldy=64)
NORMG = dict(type=1, width=64, rows=4, dy=P, lddy=64, s=P, lds=64, weight=P, rstd=P, dx=P, lddx=64, dweight=P, workspace=P,
             workspace_bytes=1 << 20)
SCAN = dict(type=0, batch=2, tokens=5, width=64, gate=P, value=P, ld_in=64, seq_in=320, h=P, ld_h=64, seq_h=320, last=P)
SCANG = dict(type=0, batch=2, tokens=5, width=64, gate=P, value=P, ld_in=64, seq_in=320, states=P, dh=P, ld_dh=64, seq_dh=320,
             dgate=P, dvalue=P, ld_out=64, seq_out=320)


@pytest.mark.parametrize("fn,base,change,want,text", [
    ("un_rms_norm", NORM, dict(type=2), 1, "type"),
    ("un_rms_norm", NORM, dict(width=0), 1, "width"),
    ("un_rms_norm", NORM, dict(rows=-1), 1, "rows"),
    ("un_rms_norm", NORM, dict(width=16385, ldx=20000, ldy=20000), 7, "16384"),
    ("un_rms_norm", NORM, dict(eps=-1.0), 1, "eps"),
    ("un_rms_norm", NORM, dict(eps=float("nan")), 1, "eps"),
    ("un_rms_norm", NORM, dict(x=None), 1, "NULL"),
    ("un_rms_norm", NORM, dict(weight=None), 1, "NULL"),
    ("un_rms_norm", NORM, dict(y=None), 1, "NULL"),
    ("un_rms_norm", NORM, dict(ldx=63), 1, "stride"),
    ("un_rms_norm", NORM, dict(residual=P, ldr=1), 1, "stride"),
    ("un_rms_norm", NORM, dict(sum=P, lds=0), 1, "stride"),
    ("un_rms_norm", NORM, dict(rows=1 << 40), 7, "rows"),
    ("un_rms_norm_backward", NORMG, dict(type=-1), 1, "type"),
    ("un_rms_norm_backward", NORMG, dict(workspace_bytes=0), 6, "workspace"),
    ("un_rms_norm_backward", NORMG, dict(workspace=None), 6, "workspace"),
    ("un_rms_norm_backward", NORMG, dict(rstd=None), 1, "NULL"),
    ("un_rms_norm_backward", NORMG, dict(dweight=None), 1, "NULL"),
    ("un_rms_norm_backward", NORMG, dict(ds=P, ldds=3), 1, "stride"),
    ("un_gated_scan", SCAN, dict(type=5), 1, "type"),
    ("un_gated_scan", SCAN, dict(tokens=-1), 1, "negative"),
    ("un_gated_scan", SCAN, dict(gate=None), 1, "NULL"),
    ("un_gated_scan", SCAN, dict(h=None), 1, "NULL"),
    ("un_gated_scan", SCAN, dict(ld_in=10), 1, "stride"),
    ("un_gated_scan", SCAN, dict(ld_h=10), 1, "stride"),
    ("un_gated_scan", SCAN, dict(seq_h=0), 1, "stride"),
    ("un_gated_scan", SCAN, dict(batch=1, tokens=100000), 6, "workspace"),
    ("un_gated_scan", SCAN, dict(batch=1, tokens=1000, workspace=P + 4, workspace_bytes=1 << 20), 1, "aligned"),
    ("un_gated_scan", SCAN, dict(width=1 << 24, ld_in=1 << 24, ld_h=1 << 24, seq_h=1 << 28), 7, "2^24"),
    ("un_gated_scan", SCAN, dict(ld_in=1 << 24), 7, "2^24"),
    ("un_gated_scan", SCAN, dict(tokens=(1 << 30) + 1), 7, "tokens"),
    ("un_gated_scan", SCAN, dict(batch=1 << 30, tokens=17, width=4096, ld_in=4096, ld_h=4096, seq_h=1 << 20), 7, "too many"),
    ("un_gated_scan_backward", SCANG, dict(states=None), 1, "NULL"),
    ("un_gated_scan_backward", SCANG, dict(dvalue=None), 1, "NULL"),
    ("un_gated_scan_backward", SCANG, dict(ld_out=63), 1, "stride"),
    ("un_gated_scan_backward", SCANG, dict(seq_out=0), 1, "stride"),
    ("un_gated_scan_backward", SCANG, dict(batch=1, tokens=100000), 6, "workspace"),
    ("un_gated_scan_backward", SCANG, dict(batch=1, tokens=1000, workspace=P + 4, workspace_bytes=1 << 20), 1, "aligned"),
    ("un_gated_scan_backward", SCANG, dict(ld_dh=1 << 24), 7, "2^24"),
])
def test_refused(fn, base, change, want, text):
    args = getattr(U, {"un_rms_norm": "un_rms_norm_args", "un_rms_norm_backward": "un_rms_norm_grad_args",
                       "un_gated_scan": "un_gated_scan_args", "un_gated_scan_backward": "un_gated_scan_grad_args"}[fn])(
        **{**base, **change})
    s, msg = status(fn, args)
    assert s == want, msg
    assert text in msg and "un_" in msg


@pytest.mark.parametrize("fn", ["un_rms_norm", "un_rms_norm_backward", "un_gated_scan", "un_gated_scan_backward"])
def test_null_arguments(fn):
    s, msg = status(fn, None)
    assert s == U.UN_ERR_INVALID and fn in msg


def test_empty_calls_need_no_device():
    """No rows, no sequences or no channels: nothing to do, whatever the pointers."""
    L = U.lib()
    assert L.un_rms_norm(ctypes.byref(U.un_rms_norm_args(**{**NORM, "rows": 0, "x": None})), None) == U.UN_OK
    for k in ("batch", "width"):
        assert L.un_gated_scan(ctypes.byref(U.un_gated_scan_args(**{**SCAN, k: 0})), None) == U.UN_OK
        assert L.un_gated_scan_backward(ctypes.byref(U.un_gated_scan_grad_args(**{**SCANG, k: 0})), None) == U.UN_OK


def test_sizes():
    L = U.lib()
    n, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert L.un_gated_scan_sizes(3, 129, 10, ctypes.byref(n), ctypes.byref(b)) == U.UN_OK
    assert n.value == 3 * 3 * 10 and b.value == 0  # a state every 64 steps
    assert L.un_gated_scan_sizes(1, 65536, 512, ctypes.byref(n), ctypes.byref(b)) == U.UN_OK
    assert n.value == 1024 * 512 and b.value > 0 and b.value % 8 == 0
    assert L.un_gated_scan_sizes(1, -1, 4, ctypes.byref(n), ctypes.byref(b)) == U.UN_ERR_INVALID
    assert L.un_rms_norm_workspace(0, 5, 100, ctypes.byref(b)) == U.UN_OK and b.value % 400 == 0 and b.value >= 400
    assert L.un_rms_norm_workspace(0, 5, 100, None) == U.UN_ERR_INVALID


TENSOR = dict(weight=P, grad=P, m=P, v=P, elements=10)


@pytest.mark.parametrize("change,n,grad,bits,want,text", [
    ({}, 0, 0, 32, 1, "no tensors"),
    ({}, 1, 2, 32, 1, "gradient type"),
    ({}, 1, 0, 16, 1, "state_bits"),
    (dict(elements=-1), 1, 0, 32, 1, "negative"),
    (dict(v=None), 1, 0, 32, 1, "NULL"),
    ({}, 1, 0, 8, 1, "m_scale"),
    (dict(m_scale=P, v_scale=P), 1, 0, 32, 1, "no scales"),
    (dict(elements=(1 << 42) + 1), 1, 0, 32, 7, "large"),
    (dict(elements=1 << 41), 1, 0, 32, 7, "too many"),
])
def test_adamw_create_refused(change, n, grad, bits, want, text):
    arr = (U.un_adamw_tensor * 1)(U.un_adamw_tensor(**{**TENSOR, **change}))
    out = ctypes.c_void_p(7)
    s = U.lib().un_adamw_create(arr, n, grad, bits, ctypes.byref(out))
    msg = U.lib().un_last_error(None).decode()
    assert s == want and text in msg and not out.value, msg


def test_adamw_null_calls():
    L = U.lib()
    assert L.un_adamw_create(None, 1, 0, 32, None) == U.UN_ERR_INVALID
    h = U.un_adamw_hyper(0.1, 0.9, 0.99, 1e-8, 0.0, 1, 0)
    assert L.un_adamw_step(None, ctypes.byref(h), None) == U.UN_ERR_INVALID
    L.un_adamw_destroy(None)


def test_python_checks():
    """The Python layer names the argument that does not fit (host tensors are refused too)."""
    from paper_2408_01331_amd import operators as ops
    x, w = torch.zeros(4, 8), torch.zeros(8)
    with pytest.raises(ValueError, match="GPU"):
        ops.rms_norm(x, w)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        ops.rms_norm(x.half(), w)
    with pytest.raises(ValueError, match="tensor"):
        ops.rms_norm([1.0], w)
    with pytest.raises(ValueError, match=r"\[batch, tokens, width\]"):
        ops.gated_scan(x, x)
    with pytest.raises(ValueError, match="no tensors"):
        ops.AdamW([], [], [], [])
    with pytest.raises(ValueError, match="grads must hold 2"):
        ops.AdamW([w, w], [w], [w, w], [w, w])


def test_8_bit_states_come_and_go(tmp_path):
    """An 8-bit state and its table are given back when the optimizer changes, and when their clearing fails."""
    import _host_hip as H
    res = H.run("""
spec = {"layers": [("linear", 16), ("relu",), ("linear", 3)], "num_classes": 3}
h = U.Hybrid([spec, spec], 4, (8,), "bf16")
h.set_optimizer(0, "adam")
n = sum(int(np.prod(s)) for s in ((16, 8), (16,), (3, 16), (3,)))
U.un_set_opt_state(h.ctx, 0, np.arange(2 * n, dtype=np.float32), 5)
held = stub.stub_device()
U.un_set_optimizer(h.ctx, 0, "adamw8")
result = [stub.stub_device() - held]
state, step = U.un_get_opt_state(h.ctx, 0)
result.append([float(np.abs(state).max()), int(step)])
U.un_set_opt_state(h.ctx, 0, np.arange(2 * n, dtype=np.float32), 5)
U.un_set_optimizer(h.ctx, 0, "adamw8")
result.append([float(np.abs(U.un_get_opt_state(h.ctx, 0)[0]).max()), stub.stub_device() - held])
U.un_set_optimizer(h.ctx, 1, "adamw8")
U.un_set_optimizer(h.ctx, 0, "sgd")
U.un_set_optimizer(h.ctx, 1, "adam")
result.append(stub.stub_device() - held)
stub.stub_fail_memset(0)
try:
    U.un_set_optimizer(h.ctx, 0, "adamw8")
except U.UnError as e:
    result.append([e.status == U.UN_ERR_DEVICE, stub.stub_device() - held])
stub.stub_fail_memset(-1)
h.close()
result.append(stub.stub_device())
""", tmp_path)
    assert res == [2, [0.0, 0], [0.0, 2], 0, [True, 0], 0]
