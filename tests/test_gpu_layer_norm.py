"""GPU tests of the layer norm on device tensors against its definition in 64 bits
(bounds: _lm_operator_refs.py)."""
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


def rand(seed, shape, dtype=F32, mean=0.0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).cuda()


def out_bound(want, bound, dtype):
    return bound + (R.half_step(dtype) * (want.abs() + bound) if dtype != F32 else 0)


SIZES = [(1, 1), (3, 7), (5, 8), (1, 64), (70, 100), (9, 999), (4, 2048), (3, 2056), (2, 8191), (2, 8200), (1, 16384), (1100, 40),
         (0, 16), (33000, 40), (2100, 2048)]


def check(ops, x, r, w, b, dy, ds, eps, dtype):
    y, s, stats = ops.layer_norm(x, w, b, residual=r, eps=eps, keep=True)
    want = R.LayerNorm(x, r, w, b, eps)
    R.close(s, want.s, torch.zeros(()), "s")
    R.close(stats[..., 0], want.mean[..., 0], want.e_mean[..., 0], "mean")
    R.close(stats[..., 1], want.q[..., 0], (want.q * want.e_q)[..., 0], "rstd")
    R.close(y, want.y, out_bound(want.y, want.e_y, dtype), "y")
    dx, dw, db = ops.layer_norm_backward(dy, s, w, stats, ds=ds)
    wdx, edx, wdw, edw, wdb, edb = want.backward(dy, ds)
    R.close(dx, wdx, out_bound(wdx, edx, dtype), "dx")
    R.close(dw, wdw, edw, "dw")
    R.close(db, wdb, edb, "db")
    return y, s, stats, dx, dw, db


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,width", SIZES)
@pytest.mark.parametrize("residual", [False, True])
def test_layer_norm(ops, dtype, rows, width, residual):
    x, w, b = rand(1, (rows, width), dtype, mean=0.5), rand(2, (width,), mean=1.0, std=0.3), rand(6, (width,), std=0.5)
    r = rand(3, (rows, width), dtype, std=3.0) if residual else None
    dy, ds = rand(4, (rows, width), dtype), rand(5, (rows, width), dtype) if residual else None
    check(ops, x, r, w, b if residual else None, dy, ds, 1e-5, dtype)


@pytest.mark.parametrize("mean", [100.0, -3000.0])
def test_large_mean(ops, mean):
    """A mean that is large against the spread: the squares are those of the centred values."""
    x, w = rand(1, (40, 1000), F32, mean=mean), rand(2, (1000,), mean=1.0, std=0.3)
    check(ops, x, None, w, None, rand(3, (40, 1000)), None, 1e-5, F32)


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
def test_strides_and_alignment(ops, dtype):
    """Rows inside a wider buffer, at every alignment of the element; axes in another order."""
    for off in (0, 1, 3):
        x, dy = rand(off, (6, 150), dtype)[:, off:off + 101], rand(10, (6, 150), dtype)[:, off:off + 101]
        r, ds = rand(11, (6, 203), dtype)[:, off:off + 101], rand(12, (6, 101), dtype)
        check(ops, x, r, rand(9, (101,)), rand(8, (101,)), dy, ds, 1e-6, dtype)
    x3, w = rand(3, (2, 3, 5, 16), dtype), rand(4, (16,))
    y, _, stats = ops.layer_norm(x3, w, keep=True)
    assert y.shape == x3.shape and stats.shape == (2, 3, 5, 2)
    assert torch.equal(y.view(-1, 16), ops.layer_norm(x3.view(-1, 16), w)[0])
    xt = x3.transpose(0, 2)
    assert torch.equal(ops.layer_norm(xt, w)[0], y.transpose(0, 2))
    assert torch.equal(ops.layer_norm(x3[0, 0, 0], w)[0], y[0, 0, 0])


def test_past_the_caches(ops):
    """Above 256 MiB a call's reads pass the caches: the same bits as for its first rows alone."""
    rows, less, width = 40000, 30000, 1000
    x, r, dy, ds = (rand(k, (rows, width), BF16) for k in (1, 2, 4, 5))
    w, b = rand(3, (width,), mean=1.0, std=0.3), rand(6, (width,))
    got = []
    for k in (rows, less):
        y, s, stats = ops.layer_norm(x[:k], w, b, residual=r[:k], keep=True)
        got.append((y, s, stats, *ops.layer_norm_backward(dy[:k], s, w, stats, ds=ds[:k])))
    for a, c in zip(got[0][:4], got[1][:4]):
        assert torch.equal(a[:less], c)
    s, stats = got[0][1].double(), got[0][2].double()
    h = (s - stats[:, :1]) * stats[:, 1:]
    for got_sum, terms in ((got[0][4], dy.double() * h), (got[0][5], dy.double())):
        assert ((got_sum.double() - terms.sum(0)).abs() <= terms.abs().sum(0) * R.U32 * (rows + 40)).all()


def test_special_values(ops):
    """Constant rows, a NaN or an infinity concern their own row alone."""
    w, b = torch.ones(40, device="cuda"), rand(7, (40,))
    x = rand(0, (6, 40))
    clean = ops.layer_norm(x, w, b)[0]
    x2 = x.clone()
    x2[1] = 2.0
    x2[3, 5] = float("nan")
    x2[4, 7] = float("inf")
    y, _, stats = ops.layer_norm(x2, w, b, keep=True)
    keep = [0, 2, 5]
    assert torch.equal(y[keep], clean[keep]) and torch.equal(y[1], b)
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).all()
    assert torch.isfinite(stats[[0, 1, 2, 5]]).all()


def test_in_place(ops):
    """The C calls with the residual stream and the gradient updated in place equal those that allocate."""
    import ctypes
    from paper_2408_01331_amd import unifiednn as U
    x, r, w = rand(1, (33, 72), BF16), rand(2, (33, 72), BF16), rand(3, (72,))
    y, s, stats = ops.layer_norm(x, w, residual=r, eps=1e-5, keep=True)
    y2, r2 = torch.empty_like(y), r.clone()
    stream = torch.cuda.current_stream().cuda_stream
    a = U.un_layer_norm_args(type=1, width=72, rows=33, eps=1e-5, x=x.data_ptr(), ldx=72, residual=r2.data_ptr(), ldr=72,
                             weight=w.data_ptr(), sum=r2.data_ptr(), lds=72, y=y2.data_ptr(), ldy=72)
    assert U.lib().un_layer_norm(ctypes.byref(a), stream) == U.UN_OK
    assert torch.equal(r2, s) and torch.equal(y2, y)
    dy, ds = rand(4, (33, 72), BF16), rand(5, (33, 72), BF16)
    dx, dw, _ = ops.layer_norm_backward(dy, s, w, stats, ds=ds)
    need = ctypes.c_size_t()
    assert U.lib().un_layer_norm_workspace(1, 33, 72, ctypes.byref(need)) == U.UN_OK
    ws, dw2 = torch.empty(need.value, dtype=torch.uint8, device="cuda"), torch.empty_like(dw)
    for into in (ds.clone(), dy.clone()):
        own = dict(ds=into.data_ptr(), dy=dy.data_ptr()) if torch.equal(into, ds) else dict(ds=ds.data_ptr(), dy=into.data_ptr())
        a = U.un_layer_norm_grad_args(type=1, width=72, rows=33, lddy=72, s=s.data_ptr(), lds=72, weight=w.data_ptr(), stats=stats.data_ptr(),
                                      ldds=72, dx=into.data_ptr(), lddx=72, dweight=dw2.data_ptr(), workspace=ws.data_ptr(),
                                      workspace_bytes=need.value, **own)
        assert U.lib().un_layer_norm_backward(ctypes.byref(a), stream) == U.UN_OK
        assert torch.equal(into, dx) and torch.equal(dw2, dw)


def test_against_differences(ops):
    """The gradients against central differences of the definition in 64 bits, in random directions."""
    x, w, b, dy = rand(1, (7, 33), mean=0.3), rand(2, (33,), mean=1.0, std=0.2), rand(3, (33,)), rand(4, (7, 33))
    _, s, stats = ops.layer_norm(x, w, b, eps=1e-5, keep=True)
    grads = ops.layer_norm_backward(dy, s, w, stats)
    base = [R.d(t) for t in (x, w, b)]
    h = 1e-6
    for i, g in enumerate(grads):
        v = torch.randn(base[i].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64)
        f = [(R.LayerNorm(*_with(base, i, base[i] + k * h * v)).y * R.d(dy)).sum() for k in (1, -1)]
        want = (f[0] - f[1]) / (2 * h)
        # fp32 gradients: 2e-5 of the terms' magnitudes; the differences themselves are off by h^2 and 1e-16 / h of f
        assert abs((R.d(g) * v).sum() - want) <= 2e-5 * (R.d(g) * v).abs().sum() + 1e-7


def _with(base, i, t):
    x, w, b = [t if j == i else o for j, o in enumerate(base)]
    return x, None, w, b, 1e-5
