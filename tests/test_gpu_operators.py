"""GPU tests of the operators on device tensors against their definitions in 64
bits (bounds: _operator_refs.py), at the sizes, strides, lengths and masks where
they can go wrong."""
import math

import pytest

torch = pytest.importorskip("torch")

import _operator_refs as R  # noqa: E402

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


def out_bound(want, bound, dtype):
    return bound + (R.half_step(dtype) * (want.abs() + bound) if dtype != F32 else 0)


# ---------------------------------------------------------------------------
# RMS norm
# ---------------------------------------------------------------------------
NORM_SIZES = [(1, 1), (3, 7), (5, 8), (1, 64), (70, 100), (9, 999), (4, 2048), (3, 2056), (2, 8191), (2, 8200), (1, 16384),
              (1100, 40), (0, 16), (33000, 40), (66000, 33), (2100, 2048)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,width", NORM_SIZES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm(ops, dtype, rows, width, residual):
    x, w = rand(1, (rows, width), dtype), rand(2, (width,), mean=1.0, std=0.3)
    r = rand(3, (rows, width), dtype, std=3.0) if residual else None
    y, s, rstd = ops.rms_norm(x, w, residual=r, eps=1e-5, keep=True)
    ws, wq, wy = R.norm_fwd(x, r, w, 1e-5)
    R.close(s, ws, torch.zeros(()), "s")
    R.close(rstd, wq[..., 0], wq[..., 0] * R.NORM_U, "rstd")
    R.close(y, wy, out_bound(wy, wy.abs() * R.NORM_U, dtype), "y")
    dy, ds = rand(4, (rows, width), dtype), rand(5, (rows, width), dtype) if residual else None
    dx, dw = ops.rms_norm_backward(dy, s, w, rstd, ds=ds)
    wdx, bdx, wdw, bdw = R.norm_bwd(dy, s, w, 1e-5, ds)
    R.close(dx, wdx, out_bound(wdx, bdx, dtype), "dx")
    R.close(dw, wdw, bdw, "dw")
    q, scale, s8 = ops.rms_norm_e4m3(x, w, residual=r, eps=1e-5)
    if rows:
        top = wy.abs().amax(-1)
        R.close(scale, top.clamp_min(1e-30) / 448, top / 448 * (R.NORM_U + 2 * R.U32) + 1e-38, "scale")
        sc = R.d(scale)[:, None]
        # half a step of e4m3: 2^-4 of the value, 2^-10 of the scale below its smallest normal
        R.close(q.float().cpu().double() * sc, wy, torch.maximum(wy.abs() * 2.0 ** -4, sc * 2.0 ** -10) + 3 * wy.abs() * R.NORM_U, "codes")
        assert torch.equal(s8, s)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_norm_strides_and_alignment(ops, dtype):
    """Rows inside a wider buffer, at every alignment of the element; neighbours stay as they are."""
    for off in (0, 1, 3):
        big = rand(off, (6, 150), dtype)
        x = big[:, off:off + 101]
        w = rand(9, (101,))
        y, s, rstd = ops.rms_norm(x, w, keep=True)
        _, _, wy = R.norm_fwd(x, None, w, 1e-6)
        R.close(y, wy, out_bound(wy, wy.abs() * R.NORM_U, dtype), "y")
        dy = rand(10, (6, 150), dtype)[:, off:off + 101]
        dx, dw = ops.rms_norm_backward(dy, s, w, rstd)
        wdx, bdx, wdw, bdw = R.norm_bwd(dy, x, w, 1e-6, None)
        R.close(dx, wdx, out_bound(wdx, bdx, dtype), "dx")
        R.close(dw, wdw, bdw, "dw")
    x3 = rand(3, (2, 3, 5, 16), dtype)
    w = rand(4, (16,))
    y = ops.rms_norm(x3, w)[0]
    assert y.shape == x3.shape and torch.equal(y.view(-1, 16), ops.rms_norm(x3.view(-1, 16), w)[0])
    xt = x3.transpose(0, 2)
    assert torch.equal(ops.rms_norm(xt, w)[0], y.transpose(0, 2))
    assert torch.equal(ops.rms_norm(x3[0, 0, 0], w)[0], y[0, 0, 0])


def test_norm_past_the_caches(ops):
    """Above 256 MiB a call's reads pass the caches: the same bits as for its first rows alone."""
    rows, less, width = 40000, 30000, 1000
    x, r, w, dy, ds = (rand(k, (rows, width), BF16) if k != 3 else rand(3, (width,), mean=1.0, std=0.3) for k in range(1, 6))
    got = []
    for k in (rows, less):
        y, s, rstd = ops.rms_norm(x[:k], w, residual=r[:k], keep=True)
        got.append((y, s, rstd, *ops.rms_norm_backward(dy[:k], s, w, rstd, ds=ds[:k])))
    for a, b in zip(got[0][:4], got[1][:4]):
        assert torch.equal(a[:less], b)
    terms = dy.double() * got[0][1].double() * got[0][2].double()[:, None]
    # dw: a rounding per term and per sum, and the two of each product
    assert ((got[0][4].double() - terms.sum(0)).abs() <= terms.abs().sum(0) * R.U32 * (rows + 40)).all()


def test_norm_special_values(ops):
    """Rows of zeros, a NaN or an infinity concern their own row alone."""
    w = torch.ones(40, device="cuda")
    x = rand(0, (6, 40))
    clean = ops.rms_norm(x, w, keep=True)
    x2 = x.clone()
    x2[1] = 0
    x2[3, 5] = float("nan")
    x2[4, 7] = float("inf")
    y, s, rstd = ops.rms_norm(x2, w, keep=True)
    keep = [0, 2, 5]
    assert torch.equal(y[keep], clean[0][keep]) and torch.equal(y[1], torch.zeros(40, device="cuda"))
    assert torch.isnan(y[3]).all() and torch.isnan(y[4, 7]) and (y[4, :7] == 0).all()
    q, scale, _ = ops.rms_norm_e4m3(x2[[0, 1]], w)
    assert (q[1].float() == 0).all() and scale[1] > 0


def test_norm_in_place_sum(ops):
    """The C call with the residual stream updated in place equals the one that allocates."""
    import ctypes
    from paper_2408_01331_amd import unifiednn as U
    x, r, w = rand(1, (33, 72), BF16), rand(2, (33, 72), BF16), rand(3, (72,))
    y, s, _ = ops.rms_norm(x, w, residual=r)
    y2, r2 = torch.empty_like(y), r.clone()
    a = U.un_rms_norm_args(type=1, width=72, rows=33, eps=1e-6, x=x.data_ptr(), ldx=72, residual=r2.data_ptr(), ldr=72,
                           weight=w.data_ptr(), sum=r2.data_ptr(), lds=72, y=y2.data_ptr(), ldy=72)
    assert U.lib().un_rms_norm(ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == U.UN_OK
    assert torch.equal(r2, s) and torch.equal(y2, y)


# ---------------------------------------------------------------------------
# Gated linear recurrence
# ---------------------------------------------------------------------------
SCAN_SIZES = [(1, 1, 1), (3, 1, 70), (2, 2, 64), (5, 15, 33), (2, 16, 130), (2, 17, 8), (1, 127, 65), (1, 128, 64), (2, 129, 66),
              (1, 257, 3), (3, 1000, 100), (1, 5000, 17), (300, 130, 128), (520, 140, 130), (130, 300, 100), (64, 300, 200)]


def check_scan(ops, gate, value, h0, lens, dh, dlast, dtype, cols=None):
    h, last, states = ops.gated_scan(gate, value, h0=h0, lens=lens, keep=True)
    dg, dv, dh0 = ops.gated_scan_backward(gate, value, states, dh, dlast=dlast, lens=lens)
    pick = (lambda x: x) if cols is None else (lambda x: None if x is None else x[:cols])
    gate, value, h0, lens, dh, dlast = map(pick, (gate, value, h0, lens, dh, dlast))
    wh, bh, wl, bl = R.scan_fwd(gate, value, h0, lens)
    R.close(pick(h), wh, out_bound(wh, bh, dtype), "h")
    R.close(pick(last), wl, bl, "last")
    (wg, bg), (wv, bv), (w0, b0) = R.scan_bwd(gate, value, h0, lens, dh, dlast)
    R.close(pick(dg), wg, out_bound(wg, bg, dtype), "dgate")
    R.close(pick(dv), wv, out_bound(wv, bv, dtype), "dvalue")
    R.close(pick(dh0), w0, b0 + 1e-38, "dh0")
    return h, last, dg, dv, dh0


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("b,n,w", SCAN_SIZES)
@pytest.mark.parametrize("ragged", [False, True])
def test_scan(ops, dtype, b, n, w, ragged):
    gate, value, dh = rand(1, (b, n, w), dtype, mean=1.5, std=2.0).clamp(-8, 8), rand(2, (b, n, w), dtype), rand(3, (b, n, w), dtype)
    h0, dlast, lens = rand(4, (b, w)), rand(5, (b, w)), None
    if ragged:
        lens = torch.randint(0, n + 1, (b,), generator=torch.Generator().manual_seed(n)).int().cuda()
        lens[-1] = 0
        if b > 1:
            lens[0] = n + 5  # clamped
    check_scan(ops, gate, value, h0 if ragged or n % 2 else None, lens, dh, dlast if n % 3 else None, dtype, cols=8)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_scan_long_split(ops, dtype):
    """A long axis split over workgroups, with lengths that end in every part."""
    b, n, w = 3, 6000, 70
    gate, value, dh = rand(1, (b, n, w), dtype, mean=4.0, std=2.0).clamp(-8, 8), rand(2, (b, n, w), dtype), rand(3, (b, n, w), dtype)
    lens = torch.tensor([6000, 2049, 129], dtype=torch.int32, device="cuda")
    check_scan(ops, gate, value, rand(4, (b, w)), lens, dh, rand(5, (b, w)), dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_scan_split_many(ops, dtype):
    """Many sequences and channels that are split all the same, with lengths of 0, 1, within, at and past a segment's end."""
    b, n, w = 8, 2100, 500
    gate, value, dh = rand(1, (b, n, w), dtype, mean=4.0, std=2.0).clamp(-8, 8), rand(2, (b, n, w), dtype), rand(3, (b, n, w), dtype)
    lens = torch.tensor([2100, 0, 1, 255, 256, 257, 1024, 2099], dtype=torch.int32, device="cuda")
    check_scan(ops, gate, value, rand(4, (b, w)), lens, dh, rand(5, (b, w)), dtype)


@pytest.mark.parametrize("n,w", [(2400, 70), (33100, 5)])
def test_scan_split_runs(ops, n, w):
    """More segments than join by their maps (runs of 32, and of 128 above 512 segments); the same bits each time."""
    gate, value, dh = rand(1, (1, n, w), BF16, mean=6.0).clamp(-8, 8), rand(2, (1, n, w), BF16), rand(3, (1, n, w), BF16)
    h0, dlast = rand(4, (1, w)), rand(5, (1, w))
    first = check_scan(ops, gate, value, h0, None, dh, dlast, BF16)
    for _ in range(10):
        h, last, states = ops.gated_scan(gate, value, h0=h0, keep=True)
        again = (h, last, *ops.gated_scan_backward(gate, value, states, dh, dlast=dlast))
        assert all(torch.equal(x, y) for x, y in zip(first, again))


def test_scan_split_values_that_are_not_finite(ops):
    """A NaN (of any bits, all ones among them) reaches every later step of its channel, and no other channel."""
    gate, value = rand(1, (2, 3000, 70), mean=3.0), rand(2, (2, 3000, 70))
    clean = ops.gated_scan(gate, value)[0]
    value.view(torch.int32)[0, 500, 3] = -1
    gate.view(torch.int32)[1, 64, 69] = -1
    value[0, 700, 4] = float("inf")
    h, last, _ = ops.gated_scan(gate, value)
    assert torch.isnan(h[0, 500:, 3]).all() and torch.isnan(h[1, 64:, 69]).all() and torch.isnan(last[0, 3]) and torch.isnan(last[1, 69])
    assert torch.isinf(h[0, 700:, 4]).all()
    for x in (h, clean):
        x[0, 500:, 3], x[1, 64:, 69], x[0, 700:, 4] = 0, 0, 0
    assert torch.equal(h, clean)


@pytest.mark.parametrize("b,n", [(2, 0), (0, 5), (0, 3000)])
def test_scan_of_nothing(ops, b, n):
    gate, h0, dlast = rand(1, (b, n, 70)), rand(2, (b, 70)), rand(3, (b, 70))
    h, last, states = ops.gated_scan(gate, gate, h0=h0, keep=True)
    assert h.shape == gate.shape and torch.equal(last, h0)
    assert torch.equal(ops.gated_scan(gate, gate)[1], torch.zeros_like(h0))
    dg, dv, dh0 = ops.gated_scan_backward(gate, gate, states, gate, dlast=dlast)
    assert dg.shape == dv.shape == gate.shape and torch.equal(dh0, dlast)


@pytest.mark.parametrize("b,less,n,w", [(1200, 600, 300, 128), (250, 150, 1500, 128), (3, 1, 125000, 128)])
def test_scan_past_the_caches(ops, b, less, n, w):
    """Above 256 MiB a call's accesses pass the caches: the same bits as for its first sequences alone."""
    z, dh = rand(1, (b, n, 2 * w), BF16, mean=1.0), rand(2, (b, n, w), BF16)
    got = []
    for k in (b, less):
        gate, value = z[:k, :, :w], z[:k, :, w:]
        h, last, states = ops.gated_scan(gate, value, keep=True)
        got.append((h, last, *ops.gated_scan_backward(gate, value, states, dh[:k])))
    assert 6 * b * n * w >= 1 << 28 > 6 * less * n * w
    for x, y in zip(*got):
        assert torch.equal(x[:less], y)


def test_scan_strides(ops):
    """Halves of one projection, and a token-major layout; what lies between stays as it is."""
    b, n, w = 4, 200, 48
    for dtype in DTYPES:
        z = rand(1, (b, n, 2 * w + 3), dtype)
        for lo in (0, 1):
            gate, value = z[..., lo:lo + w], z[..., lo + w:lo + 2 * w]
            h, last, states = ops.gated_scan(gate, value, keep=True)
            h2, last2, states2 = ops.gated_scan(gate.contiguous(), value.contiguous(), keep=True)
            assert torch.equal(h, h2) and torch.equal(last, last2) and torch.equal(states, states2)
            dh = rand(2, (n, b, w), dtype).transpose(0, 1)
            buf = torch.full((b, n, 2 * w + 3), 7.0, dtype=dtype, device="cuda")
            dh0 = ops.gated_scan_backward(gate, value, states, dh, out=(buf[..., lo:lo + w], buf[..., lo + w:lo + 2 * w]))
            dg, dv, e0 = ops.gated_scan_backward(gate.contiguous(), value.contiguous(), states, dh.contiguous())
            assert torch.equal(buf[..., lo:lo + w], dg) and torch.equal(buf[..., lo + w:lo + 2 * w], dv) and torch.equal(dh0, e0)
            assert (buf[..., :lo] == 7).all() and (buf[..., lo + 2 * w:] == 7).all()
        tm = rand(3, (n, b, w), dtype).transpose(0, 1)
        assert torch.equal(ops.gated_scan(tm, tm)[0], ops.gated_scan(tm.contiguous(), tm.contiguous())[0])


def test_scan_gates_at_their_limits(ops):
    """An infinite gate resets (-inf) or keeps (+inf) the state exactly; huge ones come near it; NaN in skipped rows is not seen."""
    b, n, w = 2, 150, 16
    for dtype in DTYPES:
        gate, value, dh = rand(1, (b, n, w), dtype), rand(2, (b, n, w), dtype), rand(3, (b, n, w), dtype)
        gate[:, 40], gate[:, 41], gate[:, 60], gate[:, 61] = float("-inf"), float("inf"), 200.0, -200.0
        lens = torch.tensor([n, 100], dtype=torch.int32, device="cuda")
        for x in (gate, value, dh):
            x[1, 100:] = float("nan")
        h, last, dg, dv, _ = check_scan(ops, gate, value, None, lens, dh, None, dtype)
        assert torch.equal(h[:, 40], value[:, 40]) and torch.equal(h[:, 41], h[:, 40])
        assert (dv[:, 41] == 0).all() and (dg[:, 40:42] == 0).all() and (h[1, 100:] == 0).all()


def test_scan_far_gates_fp32(ops):
    """fp32 gates to +-80: a and 1 - a keep their relative accuracy (a single step shows them)."""
    g = torch.linspace(-80, 80, 4001, device="cuda").view(1, 1, -1)
    h = ops.gated_scan(g, torch.ones_like(g))[0]                                   # 1 - a
    k = ops.gated_scan(g, torch.zeros_like(g), h0=torch.ones(1, 4001, device="cuda"))[1]  # a
    for got, want in ((h[0, 0], torch.sigmoid(-g[0, 0].double())), (k[0], torch.sigmoid(g[0, 0].double()))):
        R.close(got, want, want.cpu().abs() * R.SCAN_U + 1e-37, "sigmoid")


@pytest.mark.parametrize("b,n,w", [(64, 1, 100), (1, 3000, 64)])
def test_scan_state_in_place(ops, b, n, w):
    """The last state may take the start state's place, also where the axis is split."""
    gate, value, h0 = rand(1, (b, n, w), BF16, mean=5.0), rand(2, (b, n, w), BF16), rand(3, (b, w))
    h, last, _ = ops.gated_scan(gate, value, h0=h0)
    state = h0.clone()
    h2, same, _ = ops.gated_scan(gate, value, h0=state, last=state)
    assert same.data_ptr() == state.data_ptr() and torch.equal(h2, h) and torch.equal(state, last)


def test_scan_in_pieces(ops):
    """A sequence in pieces, the state handed on, is the sequence (as serving a prompt and then single tokens)."""
    b, n, w = 3, 300, 40
    gate, value = rand(1, (b, n, w)), rand(2, (b, n, w))
    want, bound, wl, bl = R.scan_fwd(gate, value, None, None)
    state, at, got = None, 0, []
    for k in (150, 100, 16, 30, 1, 1, 1, 1):
        h, state, _ = ops.gated_scan(gate[:, at:at + k], value[:, at:at + k], h0=state)
        got.append(h)
        at += k
    R.close(torch.cat(got, 1), want, bound, "h")
    R.close(state, wl, bl, "last")


def test_scan_gradient_by_differences(ops):
    """Central differences of sum(h c) + sum(last e) in 64 bits against the gradient kernels."""
    b, n, w = 1, 20, 3
    gate, value, h0, c, e = rand(1, (b, n, w)), rand(2, (b, n, w)), rand(3, (b, w)), rand(4, (b, n, w)), rand(5, (b, w))
    _, _, states = ops.gated_scan(gate, value, h0=h0, keep=True)
    dg, dv, dh0 = ops.gated_scan_backward(gate, value, states, c, dlast=e)

    def loss(g, v, s):
        h, _, last, _ = R.scan_fwd(g, v, s, None)
        return ((h * R.d(c)).sum() + (last * R.d(e)).sum()).item()

    for which, grad in ((0, dg), (1, dv), (2, dh0)):
        args = [R.d(gate), R.d(value), R.d(h0)]
        for i in range(0, args[which].numel(), 7):
            step = 1e-5
            up, down = [a.clone() for a in args], [a.clone() for a in args]
            up[which].view(-1)[i] += step
            down[which].view(-1)[i] -= step
            num = (loss(*up) - loss(*down)) / (2 * step)
            # differences: step^2 (third derivatives of order 10) and 2^-52 sums of order 100 / step
            assert abs(num - grad.reshape(-1)[i].item()) <= 1e-6 + 1e-5 * abs(num)


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
HYPER = dict(betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
COUNTS = [1, 3, 4, 255, 256, 257, 4095, 4096, 4097, 10007, 0, 5]


def params_of(seed, dtype, counts=COUNTS, shift=0):
    """Tensors of these sizes as views at odd places of one buffer."""
    out = []
    for i, n in enumerate(counts):
        out.append(rand(seed + i, (n + shift,), dtype, std=0.05)[shift:])
    return out


@pytest.mark.parametrize("gtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("copies", [False, True])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw32(ops, gtype, copies, shift):
    p, g = params_of(1, F32, shift=shift), params_of(100, gtype, shift=shift)
    m, v = params_of(200, F32, shift=shift), [x * x for x in params_of(300, F32)]
    c = [x.to(BF16) for x in p] if copies else None
    opt = ops.AdamW(p, g, m, v, copies=c)
    for t in (1, 7, 1000):
        want = [R.adamw(a, b, x, y, 0.01, HYPER["betas"], HYPER["eps"], HYPER["weight_decay"], t) for a, b, x, y in zip(p, g, m, v)]
        m0, v0 = [R.d(x) for x in m], [R.d(x) for x in v]
        opt.step(0.01, t, **HYPER)
        for i, (wp, wm, wv, up) in enumerate(want):
            b1, b2 = HYPER["betas"]
            # three roundings of each moment's terms (the constants' among them); the root and quotient of them
            bm = 4 * R.U32 * (b1 * m0[i].abs() + (1 - b1) * R.d(g[i]).abs())
            R.close(m[i], wm, bm + 1e-44, "m")
            R.close(v[i], wv, 5 * R.U32 * wv + 1e-44, "v")
            rel = torch.where(wm != 0, bm / wm.abs().clamp_min(1e-300), 0.0)
            bp = 4 * R.U32 * R.d(wp).abs() + up * (16 * R.U32 + rel)
            R.close(p[i], wp, bp + 1e-44, "p")
            if copies:
                assert torch.equal(c[i], p[i].to(BF16))


def exponent(amax):
    f, e = math.frexp(amax)
    return -127 if amax == 0 else max(-127, e - 9 + (f > 0.875))


@pytest.mark.parametrize("gtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw8(ops, gtype, shift):
    p, g = params_of(1, F32, shift=shift), params_of(100, gtype, shift=shift)
    for x in g:
        if x.numel() > 600:
            x[300:600] = 0  # whole blocks without a gradient, and values far below their block's largest
            x[0] *= 1e4
    m, v, ms, vs = ops.AdamW.state8(p)
    opt = ops.AdamW(p, g, m, v, m_scales=ms, v_scales=vs)
    for t in range(1, 4):
        m0 = [R.widen(a, b) for a, b in zip(m, ms)]
        u0 = [R.widen(a, b) for a, b in zip(v, vs)]
        want = [R.adamw(a, b, x, y * y, 0.01, HYPER["betas"], HYPER["eps"], HYPER["weight_decay"], t) for a, b, x, y in zip(p, g, m0, u0)]
        opt.step(0.01, t, key=17 * t, **HYPER)
        for i, (wp, wm, wv, up) in enumerate(want):
            b1, b2 = HYPER["betas"]
            bm = 4 * R.U32 * (b1 * m0[i].abs() + (1 - b1) * R.d(g[i]).abs())
            rel = torch.where(wm != 0, bm / wm.abs().clamp_min(1e-300), 0.0)
            R.close(p[i], wp, 4 * R.U32 * R.d(wp).abs() + up * (16 * R.U32 + rel) + 1e-44, "p")
            for codes, scales, x, slack in ((m[i], ms[i], wm, bm), (v[i], vs[i], wv.sqrt(), 6 * R.U32 * wv.sqrt())):
                got = R.widen(codes, scales)
                sc = torch.repeat_interleave(torch.pow(2.0, scales.cpu().view(torch.uint8).double() - 127), 256)[:got.numel()]
                # one of the two codes around the value: the distance is below the step of the larger one (1/8 of its
                # binade), a scale's 2^-9 at least
                lim = torch.maximum(x.abs(), got.abs())
                step = torch.maximum(torch.pow(2.0, torch.floor(torch.log2(lim.clamp_min(1e-300))) - 3), sc * 2.0 ** -9)
                R.close(got, x, step + slack, "code")
                for b in range(scales.numel()):
                    top = x[256 * b:256 * b + 256].abs().max().item()
                    near = {exponent(top * (1 + k * 8 * R.U32)) for k in (-1, 0, 1)}
                    assert scales.view(torch.uint8)[b].item() - 127 in near
            live = wv > 0
            assert (R.widen(v[i], vs[i])[live] > 0).all()


def test_adamw8_rounds_without_bias(ops):
    """Over many keys the mean of a stored moment is the moment: each draw is one of two codes a step s apart, so the mean of n
    draws is off by at most 5 s / (2 sqrt(n)) but for 6e-7 of all values (5 standard deviations of at most s / 2)."""
    n, draws = 1024, 400
    g = rand(3, (n,), std=1.0)
    sums = torch.zeros(2, n, dtype=torch.float64)
    for k in range(draws):
        p = [torch.zeros(n, device="cuda")]
        m, v, ms, vs = ops.AdamW.state8(p)
        opt = ops.AdamW(p, [g], m, v, m_scales=ms, v_scales=vs)
        opt.step(0.0, 1, key=k * 7919 + 5, **HYPER)
        sums[0] += R.widen(m[0], ms[0])
        sums[1] += R.widen(v[0], vs[0])
    _, wm, wv, _ = R.adamw(p[0], g, p[0], p[0], 0.0, HYPER["betas"], 1e-8, 0.1, 1)
    for mean, x, sc in ((sums[0] / draws, wm, ms[0]), (sums[1] / draws, wv.sqrt(), vs[0])):
        scale = torch.repeat_interleave(torch.pow(2.0, sc.cpu().view(torch.uint8).double() - 127), 256)
        step = torch.maximum(torch.pow(2.0, torch.floor(torch.log2(x.abs().clamp_min(1e-300))) - 3), scale * 2.0 ** -9)
        off = (mean - x).abs() / step
        floor = x.abs() < scale * 2.0 ** -9  # (the smallest code stands for everything below it in sqrt(v))
        assert (off[~floor] <= 2.5 / math.sqrt(draws) + 1e-4).all()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("gtype", DTYPES, ids=["f32", "bf16"])
def test_adamw_large_lists(ops, eight, gtype):
    """Above 128 MiB a step's accesses pass the caches: the same bits as for the first tensor alone, with a ragged end."""
    counts = [9_000_003, 8_000_001]
    p, g = params_of(1, F32, counts), params_of(100, gtype, counts)
    got = []
    for k in (1, 2):
        q = [x.clone() for x in p[:k]]
        c = [torch.zeros_like(x, dtype=BF16) for x in q]
        if eight:
            m, v, ms, vs = ops.AdamW.state8(q)
            opt = ops.AdamW(q, g[:k], m, v, copies=c, m_scales=ms, v_scales=vs)
            state = [m[0].view(torch.uint8), v[0].view(torch.uint8), ms[0].view(torch.uint8), vs[0].view(torch.uint8)]
        else:
            m, v = [torch.zeros_like(x) for x in q], [torch.zeros_like(x) for x in q]
            opt = ops.AdamW(q, g[:k], m, v, copies=c)
            state = [m[0], v[0]]
        for t in (1, 2):
            opt.step(0.01, t, key=t, **HYPER)
        assert all(torch.equal(a, b.to(BF16)) for a, b in zip(c, q)) and not torch.equal(q[-1], p[k - 1])
        got.append([q[0], *state])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_adamw8_depends_on_key_alone(ops):
    """The same step twice gives the same bits; another key rounds otherwise."""
    res = []
    for key in (1, 1, 2):
        p, g = params_of(1, F32), params_of(100, BF16)
        m, v, ms, vs = ops.AdamW.state8(p)
        opt = ops.AdamW(p, g, m, v, m_scales=ms, v_scales=vs)
        opt.step(0.01, 1, key=key)
        res.append(torch.cat([x.view(torch.uint8) for x in m + v]))
    assert torch.equal(res[0], res[1]) and (res[0] != res[2]).float().mean() > 0.2


def test_adamw_values_that_are_not_finite(ops):
    """A NaN or infinite gradient concerns its own element."""
    for bits in (32, 8):
        p, g = [rand(1, (600,))], [rand(2, (600,))]
        clean, q = p[0].clone(), [p[0].clone()]
        gq = [g[0].clone()]
        g[0][5], g[0][300] = float("nan"), float("inf")
        for pp, gg in ((p, g), (q, gq)):
            if bits == 32:
                opt = ops.AdamW(pp, gg, [torch.zeros(600, device="cuda")], [torch.zeros(600, device="cuda")])
            else:
                m, v, ms, vs = ops.AdamW.state8(pp)
                opt = ops.AdamW(pp, gg, m, v, m_scales=ms, v_scales=vs)
            opt.step(0.1, 1)
        bad = torch.zeros(600, dtype=torch.bool, device="cuda")
        bad[[5, 300]] = True
        assert torch.equal(p[0][~bad], q[0][~bad]) and torch.isnan(p[0][bad]).all() and not torch.equal(q[0], clean)


def test_adamw_refusals(ops):
    p = [rand(1, (10,))]
    z = lambda: [torch.zeros(10, device="cuda")]  # noqa: E731
    opt = ops.AdamW(p, z(), z(), z())
    for bad in (dict(lr=-1.0), dict(lr=float("nan")), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=0.0),
                dict(weight_decay=-1.0), dict(lr=1.0, weight_decay=1.0), dict(step=0)):
        kw = {"lr": 0.1, "step": 1, **bad}
        with pytest.raises(ops.UnError):
            opt.step(**kw)
    with pytest.raises(ValueError, match="grads"):
        ops.AdamW(p, [torch.zeros(9, device="cuda")], z(), z())
    with pytest.raises(ValueError, match="m\\["):
        ops.AdamW(p, z(), [torch.zeros(10, device="cuda", dtype=BF16)], z())
    with pytest.raises(ValueError, match="overlap"):
        ops.AdamW(p + p, z() + z(), z() + z(), z() + z())
    m = z()
    with pytest.raises(ValueError, match="overlap"):
        ops.AdamW(p, z(), m, m)
    whole = rand(1, (20,))
    with pytest.raises(ValueError, match="overlap"):
        ops.AdamW([whole[:10], whole[9:19]], z() + z(), z() + z(), z() + z())
    ops.AdamW([whole[:10], whole[10:]], z() + z(), z() + z(), z() + z(), copies=[torch.zeros(10, device="cuda", dtype=BF16) for _ in range(2)])


# ---------------------------------------------------------------------------
# Streams, graphs, all of them together
# ---------------------------------------------------------------------------
def block(ops, x, w, wz, dy):
    """A pre-norm recurrent layer forward and backward: its output and every gradient."""
    b, n, d = x.shape
    y, s, rstd = ops.rms_norm(x, w, keep=True)
    z = y @ wz.t()
    h, last, states = ops.gated_scan(z[..., :d], z[..., d:], keep=True)
    out = h + x
    dz = torch.empty_like(z)
    ops.gated_scan_backward(z[..., :d], z[..., d:], states, dy, out=(dz[..., :d], dz[..., d:]))
    dwz = dz.reshape(-1, 2 * d).t() @ y.reshape(-1, d)
    dx, dw = ops.rms_norm_backward(dz @ wz, s, w, rstd, ds=dy)
    return out, last, dx, dw, dwz


def block_args(seed, b=2, n=300, d=64):
    return rand(seed, (b, n, d)), rand(seed + 1, (d,), mean=1.0, std=0.1), rand(seed + 2, (2 * d, d), std=0.1), rand(seed + 3, (b, n, d))


def test_operators_together(ops):
    """The layer's gradients against those that torch's autograd gives for the definitions in 64 bits."""
    x, w, wz, dy = block_args(1)
    got = block(ops, x, w, wz, dy)
    X, W, Z = (R.d(t).requires_grad_() for t in (x, w, wz))
    y = X / torch.sqrt((X * X).mean(-1, keepdim=True) + 1e-6) * W
    z = y @ Z.t()
    a, v = torch.sigmoid(z[..., :64]), z[..., 64:]
    now, hs = torch.zeros(2, 64, dtype=torch.float64), []
    for t in range(300):
        now = a[:, t] * now + (1 - a[:, t]) * v[:, t]
        hs.append(now)
    out = torch.stack(hs, 1) + X
    gx, gw, gz = torch.autograd.grad(out, (X, W, Z), R.d(dy))
    # fp32 throughout: products of 64 (gradients of 600) terms, 64 u of the result's size and more by cancellation
    for g, want in zip(got, (out, now, gx, gw, gz)):
        assert (R.d(g) - want.detach()).norm() <= 2e-5 * want.norm()
    # and a step of the optimizer on these gradients
    p, g = [w.clone(), wz.clone()], [got[3], got[4]]
    m, v8, ms, vs = ops.AdamW.state8(p)
    opt = ops.AdamW(p, g, m, v8, m_scales=ms, v_scales=vs)
    opt.step(0.01, 1, weight_decay=0.1)
    for q, q0, gr in zip(p, (w, wz), g):
        wp, _, _, up = R.adamw(q0, gr, torch.zeros_like(q0), torch.zeros_like(q0), 0.01, (0.9, 0.999), 1e-8, 0.1, 1)
        R.close(q, wp, 4 * R.U32 * wp.abs() + up * 24 * R.U32, "p")


def test_another_stream(ops):
    """Work on a side stream follows that stream's order: the inputs are written there, after a long run of other work."""
    args = block_args(5)
    want = block(ops, *args)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):
            a = a @ a * 1e-2
        late = [t * 1.0 for t in args]
        got = block(ops, *late)
    s.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)


def test_two_streams_at_once(ops):
    """Two streams with calls that need workspaces do not disturb one another."""
    cases = []
    for k in range(2):
        gate, value = rand(k, (1, 20000, 64), BF16, mean=5.0), rand(k + 5, (1, 20000, 64), BF16)
        cases.append((gate, value, ops.gated_scan(gate, value)))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(10):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(ops.gated_scan(cases[k][0], cases[k][1]))
    torch.cuda.synchronize()
    for k in range(2):
        for h, last, _ in got[k]:
            assert torch.equal(h, cases[k][2][0]) and torch.equal(last, cases[k][2][1])


def test_captured(ops):
    """Captured once, replayed on new inputs with eager calls in between; the optimizer step is refused under capture."""
    sets = [block_args(10 * k, n=2000) for k in range(3)]
    gate, value = rand(77, (1, 9000, 64), BF16, mean=4.0), rand(78, (1, 9000, 64), BF16)

    def calls(x, w, dy):
        b, n, d = x.shape
        y, s, rstd = ops.rms_norm(x, w, keep=True)
        q, scale, _ = ops.rms_norm_e4m3(x, w)
        h, last, states = ops.gated_scan(y, x, keep=True)
        dg, dv, _ = ops.gated_scan_backward(y, x, states, dy)
        dx, dw = ops.rms_norm_backward(dg, s, w, rstd, ds=dv)
        return y, q.view(torch.uint8), scale, h, last, dx, dw, *ops.gated_scan(gate, value)[:2]

    want = [calls(x, w, dy) for x, w, _, dy in sets]
    x, w, _, dy = (t.clone() for t in sets[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(x, w, dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    p = [rand(1, (10,))]
    z = lambda: [torch.zeros(10, device="cuda")]  # noqa: E731
    opt = ops.AdamW(p, z(), z(), z())
    with torch.cuda.graph(graph):
        out = calls(x, w, dy)
        with pytest.raises(ops.UnError, match="captured"):
            opt.step(0.1, 1)
    for k in (0, 1, 2, 1):
        x.copy_(sets[k][0]), w.copy_(sets[k][1]), dy.copy_(sets[k][3])
        graph.replay()
        eager = calls(x, w, dy)
        torch.cuda.synchronize()
        for a, b, c in zip(out, want[k], eager):
            assert torch.equal(a, b) and torch.equal(c, b)
