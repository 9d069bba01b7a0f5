"""Operators on device tensors: RMS norm, gated linear recurrence and AdamW
over many tensors, forward, backward and single-token forms (the C calls
un_rms_norm, un_gated_scan, un_adamw_step and their kin of include/unifiednn.h,
which a context's step runs for its own layers and optimizers too).

Argument checks and marshalling only; the work runs in the library's HIP
kernels, on torch's current stream of the tensors' device. A call allocates its
outputs and workspace from torch's allocator and does not wait for the device.
"""
from __future__ import annotations

import ctypes

import torch

from . import unifiednn as _un
from .unifiednn import UnError  # noqa: F401  (raised by every call here)

_TYPES = {torch.float32: 0, torch.bfloat16: 1}


def _require(ok, what):
    if not ok:
        raise ValueError(what)


def _check_type(x, name):
    _require(isinstance(x, torch.Tensor), f"{name} must be a tensor")
    _require(x.dtype in _TYPES, f"{name} must be float32 or bfloat16, not {x.dtype}")
    return _TYPES[x.dtype]


def _like(x, name, shape, dtype, device):
    """x is a tensor of this shape and type on this device, its last axis dense."""
    _require(isinstance(x, torch.Tensor), f"{name} must be a tensor")
    _require(x.device == device and device.type == "cuda", f"{name} must be on {device if device.type == 'cuda' else 'a GPU'}, not {x.device}")
    _require(x.dtype == dtype, f"{name} must be {dtype}, not {x.dtype}")
    _require(tuple(x.shape) == tuple(shape), f"{name} must have shape {tuple(shape)}, not {tuple(x.shape)}")
    _require(x.shape[-1] <= 1 or x.stride(-1) == 1, f"{name}'s last axis must be dense")
    return x


def _flat(x, name, shape, dtype, device):
    _like(x, name, shape, dtype, device)
    _require(x.is_contiguous(), f"{name} must be contiguous")
    return x


def _ptr(x):
    return None if x is None else x.data_ptr()


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


# ---------------------------------------------------------------------------
# RMS norm
# ---------------------------------------------------------------------------
def _rows(x):
    """x as rows: (rows, row stride, x to pass on). A tensor whose leading axes do not have one stride is copied."""
    width = x.shape[-1]
    if x.dim() == 2:
        return x.shape[0], x.stride(0) if x.shape[0] > 1 else width, x
    try:
        v = x.view(-1, width) if x.dim() > 1 else x.unsqueeze(0)
    except RuntimeError:
        v = x.reshape(-1, width)
    return v.shape[0], v.stride(0) if v.shape[0] > 1 else width, v


def _norm(x, weight, residual, eps, keep, e4m3):
    t = _check_type(x, "x")
    _require(x.dim() >= 1 and x.shape[-1] >= 1, "x needs a last axis of at least one value")
    dev, shape = x.device, x.shape
    _like(x, "x", shape, x.dtype, dev)
    _flat(weight, "weight", (shape[-1],), torch.float32, dev)
    if residual is not None:
        _like(residual, "residual", shape, x.dtype, dev)
    rows, ldx, xv = _rows(x)
    _, ldr, rv = _rows(residual) if residual is not None else (0, 0, None)
    y = torch.empty(shape, dtype=torch.float8_e4m3fn if e4m3 else x.dtype, device=dev)
    s = torch.empty(shape, dtype=x.dtype, device=dev) if residual is not None else x
    rstd = torch.empty(shape[:-1], dtype=torch.float32, device=dev) if keep else None
    scale = torch.empty(shape[:-1], dtype=torch.float32, device=dev) if e4m3 else None
    a = _un.un_rms_norm_args(t, shape[-1], rows, float(eps), _ptr(xv), ldx, _ptr(rv), ldr, _ptr(weight),
                             _ptr(s) if residual is not None else None, shape[-1], _ptr(y), shape[-1], _ptr(rstd), _ptr(scale))
    _un._check(_un.lib().un_rms_norm(ctypes.byref(a), _stream(dev)))
    return y, s, rstd, scale


def rms_norm(x, weight, residual=None, eps=1e-6, keep=False):
    """(y, s, rstd): s = x + residual in x's type (x itself without a residual),
    y = s / sqrt(mean(s^2) + eps) * weight over the last axis. x: [..., width]
    float32 or bfloat16; weight: float32 [width]. rstd (float32, None unless
    `keep`) and s are what rms_norm_backward needs."""
    return _norm(x, weight, residual, eps, keep, False)[:3]


def rms_norm_e4m3(x, weight, residual=None, eps=1e-6):
    """(codes, scale, s): as rms_norm, with the output as float8_e4m3fn codes and
    a float32 scale per row: y = codes * scale[..., None]."""
    y, s, _, scale = _norm(x, weight, residual, eps, False, True)
    return y, scale, s


def rms_norm_backward(dy, s, weight, rstd, ds=None):
    """(dx, dweight) of rms_norm from the gradient dy at y, and ds at s (None: s
    is used by nothing else). dx is the gradient at x and at the residual."""
    t = _check_type(s, "s")
    dev, shape = s.device, s.shape
    width = shape[-1]
    _like(s, "s", shape, s.dtype, dev)
    _like(dy, "dy", shape, s.dtype, dev)
    if ds is not None:
        _like(ds, "ds", shape, s.dtype, dev)
    _flat(weight, "weight", (width,), torch.float32, dev)
    _flat(rstd, "rstd", shape[:-1], torch.float32, dev) if s.dim() > 1 else _require(rstd.numel() == 1, "rstd must have one value")
    rows, lds, sv = _rows(s)
    _, lddy, dyv = _rows(dy)
    _, ldds, dsv = _rows(ds) if ds is not None else (0, 0, None)
    dx = torch.empty(shape, dtype=s.dtype, device=dev)
    dw = torch.empty(width, dtype=torch.float32, device=dev)
    need = ctypes.c_size_t()
    _un._check(_un.lib().un_rms_norm_workspace(t, rows, width, ctypes.byref(need)))
    ws = torch.empty(need.value, dtype=torch.uint8, device=dev)
    a = _un.un_rms_norm_grad_args(t, width, rows, _ptr(dyv), lddy, _ptr(sv), lds, _ptr(weight), _ptr(rstd), _ptr(dsv), ldds,
                                  _ptr(dx), width, _ptr(dw), _ptr(ws), need.value)
    _un._check(_un.lib().un_rms_norm_backward(ctypes.byref(a), _stream(dev)))
    return dx, dw


# ---------------------------------------------------------------------------
# Gated linear recurrence
# ---------------------------------------------------------------------------
def _strides(x):
    """(token, sequence) strides of [batch, tokens, width]."""
    return x.stride(1) if x.shape[1] > 1 else x.shape[2], x.stride(0)


def _scan_sizes(batch, tokens, width):
    n, ws = ctypes.c_size_t(), ctypes.c_size_t()
    _un._check(_un.lib().un_gated_scan_sizes(batch, tokens, width, ctypes.byref(n), ctypes.byref(ws)))
    return n.value, ws.value


def _scan_inputs(gate, value, lens):
    t = _check_type(gate, "gate")
    _require(gate.dim() == 3, "gate must be [batch, tokens, width]")
    dev, shape = gate.device, gate.shape
    _like(gate, "gate", shape, gate.dtype, dev)
    _like(value, "value", shape, gate.dtype, dev)
    _require(gate.numel() == 0 or _strides(gate) == _strides(value), "gate and value must have the same strides")
    if lens is not None:
        _flat(lens, "lens", shape[:1], torch.int32, dev)
    return t, dev, shape


def gated_scan(gate, value, h0=None, lens=None, keep=False, last=None):
    """(h, last, states): h_t = a_t h_{t-1} + (1 - a_t) value_t with
    a = sigmoid(gate), per sequence and channel. gate, value: [batch, tokens,
    width] float32 or bfloat16, of any equal strides with a dense last axis (the
    halves of one projection). h0: float32 [batch, width], None for zeros. lens:
    int32 [batch], steps used of each sequence (rows of h behind are zeros).
    last (the state after the last step, float32) may be given, h0 itself among
    others, to be written in place. states (None unless `keep`) is what
    gated_scan_backward needs."""
    t, dev, (b, n, d) = _scan_inputs(gate, value, lens)
    if h0 is not None:
        _flat(h0, "h0", (b, d), torch.float32, dev)
    if last is None:
        last = torch.empty((b, d), dtype=torch.float32, device=dev)
    else:
        _flat(last, "last", (b, d), torch.float32, dev)
    h = torch.empty((b, n, d), dtype=gate.dtype, device=dev)
    n_states, n_ws = _scan_sizes(b, n, d)
    states = torch.empty(n_states, dtype=torch.float32, device=dev) if keep else None
    ws = torch.empty(n_ws, dtype=torch.uint8, device=dev) if n_ws else None
    ld, seq = _strides(gate)
    a = _un.un_gated_scan_args(t, b, n, d, _ptr(gate), _ptr(value), ld, seq, _ptr(lens), _ptr(h0), _ptr(h), d, n * d, _ptr(last),
                               _ptr(states), _ptr(ws), n_ws)
    _un._check(_un.lib().un_gated_scan(ctypes.byref(a), _stream(dev)))
    return h, last, states


def gated_scan_backward(gate, value, states, dh, dlast=None, lens=None, out=None):
    """dh0, with the gradients at gate and value written to out = (dgate, dvalue)
    (two tensors of gate's shape and equal strides, the halves of one buffer, say);
    without `out`, (dgate, dvalue, dh0). gate, value, lens: as given to gated_scan;
    states: what it returned; dh: the gradient at h; dlast: at the last state."""
    t, dev, (b, n, d) = _scan_inputs(gate, value, lens)
    n_states, n_ws = _scan_sizes(b, n, d)
    _flat(states, "states", (n_states,), torch.float32, dev)
    _like(dh, "dh", (b, n, d), gate.dtype, dev)
    if dlast is not None:
        _flat(dlast, "dlast", (b, d), torch.float32, dev)
    given = out is not None
    dg, dv = out if given else torch.empty((2, b, n, d), dtype=gate.dtype, device=dev).unbind(0)
    _like(dg, "dgate", (b, n, d), gate.dtype, dev)
    _like(dv, "dvalue", (b, n, d), gate.dtype, dev)
    _require(dg.numel() == 0 or _strides(dg) == _strides(dv), "dgate and dvalue must have the same strides")
    dh0 = torch.empty((b, d), dtype=torch.float32, device=dev)
    ws = torch.empty(n_ws, dtype=torch.uint8, device=dev) if n_ws else None
    (ld, seq), (ldd, seqd), (ldo, seqo) = _strides(gate), _strides(dh), _strides(dg)
    a = _un.un_gated_scan_grad_args(t, b, n, d, _ptr(gate), _ptr(value), ld, seq, _ptr(lens), _ptr(states), _ptr(dh), ldd, seqd,
                                    _ptr(dlast), _ptr(dg), _ptr(dv), ldo, seqo, _ptr(dh0), _ptr(ws), n_ws)
    _un._check(_un.lib().un_gated_scan_backward(ctypes.byref(a), _stream(dev)))
    return dh0 if given else (dg, dv, dh0)


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
QBLOCK = 256  # elements that share a scale in the 8-bit states


class AdamW:
    """AdamW over many tensors in one launch, in place on tensors that the
    caller holds.

    params: float32; grads: all float32 or all bfloat16; copies: None, or
    bfloat16 tensors that receive the new values. States: float32 m and v, or in
    8 bits float8_e4m3fn m and v (v holds sqrt(v)) with m_scales and v_scales,
    float8_e8m0fnu, one per QBLOCK consecutive elements of a tensor
    (`AdamW.state8` makes fresh ones). Every tensor is contiguous; the plan holds
    references to all of them. Gradients are read where they were when the plan
    was made: write the next step's into the same tensors."""

    def __init__(self, params, grads, m, v, copies=None, m_scales=None, v_scales=None):
        self._plan = None
        n = len(params)
        _require(n >= 1, "no tensors")
        eight = m_scales is not None or v_scales is not None
        lists = dict(grads=grads, m=m, v=v)
        if copies is not None:
            lists["copies"] = copies
        if eight:
            _require(m_scales is not None and v_scales is not None, "8-bit states need both m_scales and v_scales")
            lists.update(m_scales=m_scales, v_scales=v_scales)
        for k, x in lists.items():
            _require(len(x) == n, f"{k} must hold {n} tensors, not {len(x)}")
        dev = params[0].device
        gt = grads[0].dtype
        _require(gt in _TYPES, f"gradients must be float32 or bfloat16, not {gt}")
        st = torch.float8_e4m3fn if eight else torch.float32
        arr = (_un.un_adamw_tensor * n)()
        for i, p in enumerate(params):
            shape, k = p.shape, p.numel()
            _flat(p.view(-1) if p.dim() == 0 else p, f"params[{i}]", shape or (1,), torch.float32, dev)
            for name, x, dt in (("grads", grads, gt), ("m", m, st), ("v", v, st), ("copies", copies, torch.bfloat16)):
                if x is not None:
                    y = x[i]
                    _require(isinstance(y, torch.Tensor) and y.device == dev and y.dtype == dt and y.numel() == k and y.is_contiguous(),
                             f"{name}[{i}] must be a contiguous {dt} tensor of {k} elements on {dev}")
            if eight:
                for name, x in (("m_scales", m_scales), ("v_scales", v_scales)):
                    _require(x[i].device == dev and x[i].dtype == torch.float8_e8m0fnu and x[i].numel() == -(-k // QBLOCK) and x[i].is_contiguous(),
                             f"{name}[{i}] must be a contiguous float8_e8m0fnu tensor of {-(-k // QBLOCK)} elements on {dev}")
            arr[i] = _un.un_adamw_tensor(_ptr(p), _ptr(grads[i]), _ptr(copies[i]) if copies is not None else None, _ptr(m[i]), _ptr(v[i]),
                                         _ptr(m_scales[i]) if eight else None, _ptr(v_scales[i]) if eight else None, k)
        self._held = [params, lists]
        self.device = dev
        plan = ctypes.c_void_p()
        with torch.cuda.device(dev):
            _un._check(_un.lib().un_adamw_create(arr, n, _TYPES[gt], 8 if eight else 32, ctypes.byref(plan)))
        self._plan = plan

    @staticmethod
    def state8(params):
        """Fresh 8-bit states: (m, v, m_scales, v_scales) for AdamW."""
        codes = lambda: [torch.zeros(p.numel(), dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn) for p in params]  # noqa: E731
        scales = lambda: [torch.zeros(-(-p.numel() // QBLOCK), dtype=torch.uint8, device=p.device).view(torch.float8_e8m0fnu) for p in params]  # noqa: E731
        return codes(), codes(), scales(), scales()

    def step(self, lr, step, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, key=0):
        """Step number `step` (from 1). key: with 8-bit states, another whole number each step."""
        h = _un.un_adamw_hyper(float(lr), float(betas[0]), float(betas[1]), float(eps), float(weight_decay), int(step), int(key) & 0xFFFFFFFF)
        _un._check(_un.lib().un_adamw_step(self._plan, ctypes.byref(h), _stream(self.device)))

    def close(self):
        if self._plan:
            _un.lib().un_adamw_destroy(self._plan)
            self._plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
