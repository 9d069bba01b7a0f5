"""Operators on device tensors: RMS norm, gated linear recurrence and AdamW
over many tensors, forward, backward and single-token forms (the C calls
un_rms_norm, un_gated_scan, un_adamw_step and their kin of include/unifiednn.h,
which a context's step runs for its own layers and optimizers too).

Argument checks and marshalling only; the work runs in the library's HIP
kernels, on torch's current stream of the tensors' device. A call allocates its
outputs and workspace from torch's allocator and does not wait for the device.
Nothing is recorded for autograd: the backward passes are calls of their own, and
a call on tensors that require gradients is refused where autograd records (call
it under torch.no_grad(), or in a torch.autograd.Function). Tensors that a call
writes in place get a new version, as by torch's own operations.
"""
from __future__ import annotations

import ctypes
import functools

import torch
from torch._C import _cuda_getDevice as _current_device
from torch._C import _cuda_getCurrentRawStream as _current_stream  # torch.cuda.current_stream(i).cuda_stream without its 1 us

from . import unifiednn as _un
from .unifiednn import UnError  # noqa: F401  (raised by every call here)

_F32, _BF16, _I32 = torch.float32, torch.bfloat16, torch.int32
_TYPES = {_F32: 0, _BF16: 1}
_byref, _empty_like = ctypes.byref, torch.empty_like
_written = torch.autograd.graph.increment_version


def _require(ok, what):
    if not ok:
        raise ValueError(what)


def _check_type(x, name):
    """The type's number and the device's index of an operator's first tensor."""
    _require(isinstance(x, torch.Tensor), f"{name} must be a tensor")
    t = _TYPES.get(x.dtype)
    _require(t is not None, f"{name} must be float32 or bfloat16, not {x.dtype}")
    dev = x.get_device()
    _require(dev >= 0, f"{name} must be on a GPU, not {x.device}")
    return t, dev


def _dense(x, name):
    _require(x.stride(-1) == 1 or x.shape[-1] <= 1, f"{name}'s last axis must be dense")


def _like(x, name, shape, dtype, dev):
    """x is a tensor of this shape and type on GPU `dev`, its last axis dense. (One test for what fits; a call's latency counts.)"""
    if not (isinstance(x, torch.Tensor) and x.dtype is dtype and x.get_device() == dev and x.shape == shape
            and (x.stride(-1) == 1 or x.shape[-1] <= 1)):
        _require(isinstance(x, torch.Tensor), f"{name} must be a tensor")
        _require(x.get_device() == dev, f"{name} must be on cuda:{dev}, not {x.device}")
        _require(x.dtype is dtype, f"{name} must be {dtype}, not {x.dtype}")
        _require(x.shape == shape, f"{name} must have shape {tuple(shape)}, not {tuple(x.shape)}")
        _dense(x, name)


def _flat(x, name, shape, dtype, dev):
    if not (isinstance(x, torch.Tensor) and x.dtype is dtype and x.get_device() == dev and x.shape == shape and x.is_contiguous()):
        _like(x, name, torch.Size(shape), dtype, dev)
        _require(False, f"{name} must be contiguous")


def _unrecorded(*tensors):
    """No graph is cut: none of the tensors (None: not given) requires a gradient while autograd records."""
    for x in tensors:
        if x is not None and x.requires_grad and torch.is_grad_enabled():
            raise ValueError("a tensor requires a gradient, and this call records nothing for autograd: call it under torch.no_grad() "
                             "or in a torch.autograd.Function, with the backward call of its own")


def _ptr(x):
    return None if x is None else x.data_ptr()


def _call(fn, args, dev, plan=None):
    """fn on torch's current stream of GPU `dev`. (The default stream has no device of its own: it is the current one's.)"""
    if _current_device() != dev:
        with torch.cuda.device(dev):
            return _call(fn, args, dev, plan)
    stream = _current_stream(dev)
    status = fn(_byref(args), stream) if plan is None else fn(plan, _byref(args), stream)
    if status:
        _un._check(status)


_fns = None


def _lib():
    global _fns
    if _fns is None:
        _fns = _un.lib()
    return _fns


# ---------------------------------------------------------------------------
# RMS norm
# ---------------------------------------------------------------------------
def _rows(x, name):
    """x as rows: (rows, row stride, x to pass on). A tensor whose leading axes do not have one stride is copied."""
    shape = x.shape
    _require(len(shape) >= 1 and shape[-1] >= 1, f"{name} needs a last axis of at least one value")
    width = shape[-1]
    if x.is_contiguous():
        return x.numel() // width, width, x
    _dense(x, name)
    if len(shape) == 2:
        rows = shape[0]
        return rows, x.stride(0) if rows > 1 else width, x
    try:
        v = x.view(-1, width)
    except RuntimeError:
        v = x.reshape(-1, width)
    return v.shape[0], v.stride(0) if v.shape[0] > 1 else width, v


def _operand(x, name, shape, dtype, dev):
    """(address, row stride, x to pass on) of another tensor of the same shape and type."""
    if isinstance(x, torch.Tensor) and x.dtype is dtype and x.get_device() == dev and x.shape == shape and x.is_contiguous():
        return x.data_ptr(), shape[-1], x
    _like(x, name, shape, dtype, dev)
    _, ld, v = _rows(x, name)
    return v.data_ptr(), ld, v


def _fresh(x, dtype):
    """A new dense tensor of x's shape."""
    return _empty_like(x, dtype=dtype) if x.is_contiguous() else x.new_empty(x.shape, dtype=dtype)


@functools.lru_cache(maxsize=1024)
def _norm_workspace(t, rows, width):
    need = ctypes.c_size_t()
    status = _lib().un_rms_norm_workspace(t, rows, width, _byref(need))
    if status:
        _un._check(status)
    return need.value


def _norm(x, weight, residual, eps, keep, e4m3):
    t, dev = _check_type(x, "x")
    rows, ldx, xv = _rows(x, "x")
    shape, dtype = x.shape, x.dtype
    width = shape[-1]
    _flat(weight, "weight", (width,), _F32, dev)
    y = _fresh(x, torch.float8_e4m3fn if e4m3 else dtype)
    rp, ldr, rv, sp, s = None, 0, None, None, x
    if residual is not None:
        rp, ldr, rv = _operand(residual, "residual", shape, dtype, dev)
    _unrecorded(x, weight, residual)
    if residual is not None:
        s = _fresh(x, dtype)
        sp = s.data_ptr()
    rstd = weight.new_empty(shape[:-1]) if keep else None
    scale = weight.new_empty(shape[:-1]) if e4m3 else None
    _call(_lib().un_rms_norm, _un.un_rms_norm_args(t, width, rows, float(eps), xv.data_ptr(), ldx, rp, ldr, weight.data_ptr(), sp, width,
                                                   y.data_ptr(), width, _ptr(rstd), _ptr(scale)), dev)
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
    t, dev = _check_type(s, "s")
    rows, lds, sv = _rows(s, "s")
    shape, dtype = s.shape, s.dtype
    width = shape[-1]
    dyp, lddy, dyv = _operand(dy, "dy", shape, dtype, dev)
    _flat(weight, "weight", (width,), _F32, dev)
    _flat(rstd, "rstd", shape[:-1], _F32, dev)
    dsp, ldds, dsv = (None, 0, None) if ds is None else _operand(ds, "ds", shape, dtype, dev)
    _unrecorded(dy, s, weight, rstd, ds)
    dx, dw = _fresh(s, dtype), _empty_like(weight)
    need = _norm_workspace(t, rows, width)
    ws = weight.new_empty(need // 4)
    _call(_lib().un_rms_norm_backward, _un.un_rms_norm_grad_args(t, width, rows, dyp, lddy, sv.data_ptr(), lds, weight.data_ptr(),
                                                                 rstd.data_ptr(), dsp, ldds, dx.data_ptr(), width, dw.data_ptr(),
                                                                 ws.data_ptr(), need), dev)
    return dx, dw


# ---------------------------------------------------------------------------
# Gated linear recurrence
# ---------------------------------------------------------------------------
def _strides(x, shape):
    """(token, sequence) strides of [batch, tokens, width]."""
    st = x.stride()
    return st[1] if shape[1] > 1 else shape[2], st[0] if shape[0] > 1 else 0


@functools.lru_cache(maxsize=1024)
def _scan_sizes(batch, tokens, width):
    n, ws = ctypes.c_size_t(), ctypes.c_size_t()
    status = _lib().un_gated_scan_sizes(batch, tokens, width, _byref(n), _byref(ws))
    if status:
        _un._check(status)
    return n.value, ws.value


def _scan_inputs(gate, value, lens):
    _require(isinstance(gate, torch.Tensor) and gate.dim() == 3, "gate must be a tensor [batch, tokens, width]")
    t, dev = _check_type(gate, "gate")
    shape, stride = gate.shape, gate.stride()
    if not (isinstance(value, torch.Tensor) and value.dtype is gate.dtype and value.get_device() == dev and value.shape == shape
            and value.stride() == stride and stride[2] == 1):
        _dense(gate, "gate")
        _like(value, "value", shape, gate.dtype, dev)
        _require(_strides(gate, shape) == _strides(value, shape) or gate.numel() == 0, "gate and value must have the same strides")
    st = _strides(gate, shape)
    if lens is not None:
        _flat(lens, "lens", shape[:1], _I32, dev)
    return t, dev, shape, st


def gated_scan(gate, value, h0=None, lens=None, keep=False, last=None):
    """(h, last, states): h_t = a_t h_{t-1} + (1 - a_t) value_t with
    a = sigmoid(gate), per sequence and channel. gate, value: [batch, tokens,
    width] float32 or bfloat16, of any equal strides with a dense last axis (the
    halves of one projection). h0: float32 [batch, width], None for zeros. lens:
    int32 [batch], steps used of each sequence (rows of h behind are zeros). The
    last bits of a sequence may depend on the batch's size (un_gated_scan).
    last (the state after the last step, float32) may be given, h0 itself among
    others, to be written in place. states (None unless `keep`) is what
    gated_scan_backward needs."""
    t, dev, shape, (ld, seq) = _scan_inputs(gate, value, lens)
    b, n, d = shape
    if h0 is not None:
        _flat(h0, "h0", (b, d), _F32, dev)
    if last is not None:
        _flat(last, "last", (b, d), _F32, dev)
    _unrecorded(gate, value, h0, last)
    if last is None:
        last = gate.new_empty((b, d), dtype=_F32) if h0 is None else _empty_like(h0)
    else:
        _written(last)
    h = gate.new_empty(shape)
    states = ws = None
    n_ws = 0
    if n > 16 or keep:  # (a short call keeps no states and needs no workspace)
        n_states, n_ws = _scan_sizes(b, n, d)
        states = gate.new_empty(n_states, dtype=_F32) if keep else None
        ws = gate.new_empty(n_ws, dtype=torch.uint8) if n_ws else None
    _call(_lib().un_gated_scan, _un.un_gated_scan_args(t, b, n, d, gate.data_ptr(), value.data_ptr(), ld, seq, _ptr(lens), _ptr(h0),
                                                       h.data_ptr(), d, n * d, last.data_ptr(), _ptr(states), _ptr(ws), n_ws), dev)
    return h, last, states


def gated_scan_backward(gate, value, states, dh, dlast=None, lens=None, out=None):
    """dh0, with the gradients at gate and value written to out = (dgate, dvalue)
    (two tensors of gate's shape and equal strides that overlap no input, the
    halves of one buffer, say); without `out`, (dgate, dvalue, dh0). gate, value,
    lens: as given to gated_scan; states: what it returned; dh: the gradient at h;
    dlast: at the last state."""
    t, dev, shape, (ld, seq) = _scan_inputs(gate, value, lens)
    b, n, d = shape
    dtype = gate.dtype
    n_states, n_ws = _scan_sizes(b, n, d)
    _flat(states, "states", (n_states,), _F32, dev)
    _like(dh, "dh", shape, dtype, dev)
    if dlast is not None:
        _flat(dlast, "dlast", (b, d), _F32, dev)
    given = out is not None
    dg, dv = out if given else gate.new_empty((2, b, n, d)).unbind(0)
    _like(dg, "dgate", shape, dtype, dev)
    _like(dv, "dvalue", shape, dtype, dev)
    (ldo, seqo), (ldd, seqd) = _strides(dg, shape), _strides(dh, shape)
    _require((ldo, seqo) == _strides(dv, shape) or dg.numel() == 0, "dgate and dvalue must have the same strides")
    _unrecorded(gate, value, states, dh, dlast, dg, dv)
    if given:
        _written((dg, dv))
    dh0 = gate.new_empty((b, d), dtype=_F32)
    ws = gate.new_empty(n_ws, dtype=torch.uint8) if n_ws else None
    _call(_lib().un_gated_scan_backward, _un.un_gated_scan_grad_args(t, b, n, d, gate.data_ptr(), value.data_ptr(), ld, seq, _ptr(lens),
                                                                     states.data_ptr(), dh.data_ptr(), ldd, seqd, _ptr(dlast),
                                                                     dg.data_ptr(), dv.data_ptr(), ldo, seqo, dh0.data_ptr(), _ptr(ws),
                                                                     n_ws), dev)
    return dh0 if given else (dg, dv, dh0)


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
QBLOCK = 256  # elements that share a scale in the 8-bit states


def _disjoint(written, read):
    """No (contiguous) tensor of `written` shares memory with another one of either list."""
    spans = sorted((y.data_ptr(), y.data_ptr() + y.numel() * y.element_size(), w) for x, w in ((written, True), (read, False))
                   for y in x if y.numel())
    end = end_written = 0
    for lo, hi, w in spans:
        if lo < (end if w else end_written):
            return False
        end = max(end, hi)
        if w:
            end_written = max(end_written, hi)
    return True


class AdamW:
    """AdamW over many tensors in one launch, in place on tensors that the
    caller holds.

    params: float32; grads: all float32 or all bfloat16; copies: None, or
    bfloat16 tensors that receive the new values. States: float32 m and v, or in
    8 bits float8_e4m3fn m and v (v holds sqrt(v)) with m_scales and v_scales,
    float8_e8m0fnu, one per QBLOCK consecutive elements of a tensor
    (`AdamW.state8` makes fresh ones). Every tensor is contiguous, and none that is
    written may overlap another, a gradient among them; the plan holds references
    to all of them.
    Gradients are read where they were when the plan was made: write the next
    step's into the same tensors."""

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
        _, dev = _check_type(params[0], "params[0]")
        device = params[0].device
        _require(isinstance(grads[0], torch.Tensor), "grads[0] must be a tensor")
        gt = grads[0].dtype
        _require(gt in _TYPES, f"gradients must be float32 or bfloat16, not {gt}")
        st = torch.float8_e4m3fn if eight else torch.float32
        arr = (_un.un_adamw_tensor * n)()
        lists = dict(params=params, **lists)
        types = dict(params=_F32, grads=gt, m=st, v=st, copies=_BF16, m_scales=torch.float8_e8m0fnu, v_scales=torch.float8_e8m0fnu)
        order = [(lists[k], types[k], k, k.endswith("scales")) if k in lists else None
                 for k in ("params", "grads", "copies", "m", "v", "m_scales", "v_scales")]
        for i, p in enumerate(params):
            _require(isinstance(p, torch.Tensor), f"params[{i}] must be a tensor")
            k = p.numel()
            at = []
            for entry in order:
                if entry is None:
                    at.append(None)
                    continue
                x, dt, name, scales = entry
                y, size = x[i], -(-k // QBLOCK) if scales else k
                if not (isinstance(y, torch.Tensor) and y.get_device() == dev and y.dtype is dt and y.numel() == size and y.is_contiguous()):
                    _require(False, f"{name}[{i}] must be a contiguous {dt} tensor of {size} elements on {device}")
                at.append(y.data_ptr())
            arr[i] = _un.un_adamw_tensor(*at, k)
        flat = lambda *lists: [y for x in lists for y in x or ()]  # noqa: E731
        _require(_disjoint(flat(params, m, v, copies, m_scales, v_scales), grads), "a tensor that is written overlaps another one")
        self._held = [list(x) for x in lists.values()]
        # a view's version is its base's: one of each is enough (each takes 40 ns of every step's call)
        bases = [y if y._base is None else y._base for y in flat(params, m, v, copies, m_scales, v_scales)]
        self._written = list({id(y): y for y in bases}.values())
        self.device, self._index = device, dev
        plan = ctypes.c_void_p()
        with torch.cuda.device(device):
            _un._check(_lib().un_adamw_create(arr, n, _TYPES[gt], 8 if eight else 32, ctypes.byref(plan)))
        self._plan = plan

    @staticmethod
    def state8(params):
        """Fresh 8-bit states: (m, v, m_scales, v_scales) for AdamW."""
        codes = lambda: [torch.zeros(p.numel(), dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn) for p in params]  # noqa: E731
        scales = lambda: [torch.zeros(-(-p.numel() // QBLOCK), dtype=torch.uint8, device=p.device).view(torch.float8_e8m0fnu) for p in params]  # noqa: E731
        return codes(), codes(), scales(), scales()

    def step(self, lr, step, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, key=None):
        """Step number `step` (from 1). key: with 8-bit states, a whole number of which the rounding's random numbers are made,
        another one each step; None: one made of `step`."""
        _require(self._plan is not None, "the plan is closed")
        if key is None:
            key = 0x5EED + int(step) * 0x01000193  # as for a context's models
        h = _un.un_adamw_hyper(float(lr), float(betas[0]), float(betas[1]), float(eps), float(weight_decay), int(step), int(key) & 0xFFFFFFFF)
        _call(_lib().un_adamw_step, h, self._index, self._plan)
        _written(self._written)

    def close(self):
        if self._plan:
            _un.lib().un_adamw_destroy(self._plan)
            self._plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
