"""GPU: RMS norm and gated recurrence layers, and AdamW in 32 and 8 bits, in the
fused step: against the oracle, bit for bit against each model alone, across
active sets, graph replays and the static workspace, and resumed."""
import numpy as np
import pytest

from paper_2408_01331_amd import workloads as W
from _parity import EXTRA_FLOOR, compare_run, compare_step, run_gpu, run_oracle, theta0

pytestmark = pytest.mark.gpu

U, N, G, A, L, RELU, FLAT, RB, RE = (lambda t: ("unflatten", t)), ("rms_norm",), ("recurrence",), ("attention",), \
    (lambda n: ("linear", n)), ("relu",), ("flatten",), ("res_begin",), ("res_end",)
# No ReLU whose decision could fall either way within rounding: where a spec has
# one, the tests check that the oracle flags none.
SPECS = [
    {"layers": [U(8), G, FLAT, L(10)], "num_classes": 10},                                             # 8 tokens x 24
    {"layers": [U(24), RB, N, G, RE, N, FLAT, L(10)], "num_classes": 10},                              # 24 x 8: a skip from the input
    {"layers": [N, L(40), N, L(10)], "num_classes": 10},                                               # flat norms, the input's first
    {"layers": [L(30), RELU, N, L(10)], "num_classes": 10},                                            # a first layer that is shared
    {"layers": [U(4), L(56), RB, N, G, RE, RB, N, L(112), RELU, L(56), RE, N, L(8), FLAT, N, L(10)], "num_classes": 10},
    {"layers": [U(12), L(24), RELU, RB, N, A, RE, G, RELU, FLAT, L(10)], "num_classes": 10},           # a norm behind a ReLU
    {"layers": [L(2304), N, L(10)], "num_classes": 10},                                                # a workgroup per row
    {"layers": [L(32), RELU, L(10)], "num_classes": 10},
]


def _need_gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _bits(a):
    return np.asarray(a, dtype=np.float32).view(np.uint32)


def _wl(specs, batch, features, precision, seed=9):
    return W.Workload("recurrence", len(specs), batch, (features,), precision, specs, 0.05, 3, seed, init="torch")


def _theta(wl):
    """The generator's parameters, the norms' weights off one."""
    out = {}
    for i, s in enumerate(wl.specs):
        rng = np.random.default_rng([5, i])
        out[i] = [p if f else (p + 0.3 * rng.standard_normal(p.shape)).astype(np.float32)
                  for p, (_, f) in zip(theta0(wl, i), W.param_shapes(s, wl.in_shape))]
    return out


def _check(wl, steps, **kw):
    m = list(range(wl.n_models))
    th = _theta(wl)
    orc, spread = run_oracle(wl, steps, m, spread=True, theta=th)
    flagged = [i for i in m if any(len(v) for v in orc[i][3].values())]
    assert not flagged, f"ill-conditioned decisions in models {flagged}: take another seed"
    gpu = run_gpu(wl, steps, theta=th)
    import _parity
    real, _parity.theta0 = _parity.theta0, lambda _, i: th[i]   # the comparison's starting point
    try:
        rep = (compare_step if steps == 1 else compare_run)(wl, gpu, orc, m, spread=spread, **kw)
    finally:
        _parity.theta0 = real
    print(f"[{wl.precision} {steps} steps] " + ", ".join(f"{k}={v:.3g}" for k, v in rep.items()), flush=True)


@pytest.mark.parametrize("precision", ["f32", "bf16"])
@pytest.mark.parametrize("steps", [1, 3])
def test_models_match_the_oracle(precision, steps):
    _need_gpu()
    _check(_wl(SPECS, 37, 192, precision), steps)


@pytest.mark.parametrize("precision", ["f32", "bf16"])
@pytest.mark.parametrize("T,d", [(1, 8), (15, 16), (16, 24), (17, 136), (127, 8), (128, 72), (129, 64), (300, 8)])
def test_core_sizes(precision, T, d):
    """Tokens at the edges of a wave's steps and of a chunk, widths that fill no tile; two lengths in one launch."""
    _need_gpu()
    specs = [{"layers": [U(T), G, FLAT, L(10)], "num_classes": 10},
             {"layers": [L(64), U(4), N, G, FLAT, L(10)], "num_classes": 10}]
    _check(_wl(specs, 3, T * d, precision, seed=8), 1)


@pytest.mark.parametrize("precision", ["f32", "bf16"])
def test_model_equals_itself_alone_bitwise(precision):
    _need_gpu()
    wl = _wl(SPECS, 37, 192, precision)
    th = _theta(wl)
    merged = run_gpu(wl, 2, theta=th)
    for i in range(wl.n_models):
        one = W.Workload("alone", 1, wl.batch, wl.in_shape, precision, [wl.specs[i]], wl.lr, 2, wl.seed, init=wl.init)
        alone = run_gpu(one, 2, theta={0: th[i]})
        assert np.array_equal(_bits(merged[0][:, i]), _bits(alone[0][:, 0])), f"model {i}: losses"
        for k in (1, 2):
            for a, b in zip(merged[k][i], alone[k][0]):
                assert np.array_equal(_bits(a), _bits(b)), f"model {i}"


def test_workload():
    """The pre-norm recurrent workload at its own size. Its ReLUs may fall either way within rounding, which moves a row of
    a gradient by more than the gate: the one-step extras take the multi-step floor, and a flag anywhere frees nothing here."""
    _need_gpu()
    wl = W.get("recur8")
    m = list(range(wl.n_models))
    orc = run_oracle(wl, 1, m)
    clean = {i: orc[i][:3] + ({},) for i in m}
    rep = compare_step(wl, run_gpu(wl, 1), clean, m, extra_floor=EXTRA_FLOOR[wl.precision])
    print(f"\n[{wl.name}] " + ", ".join(f"{k}={v:.3g}" for k, v in rep.items()), flush=True)


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
OPTS = [dict(kind="adamw8", weight_decay=0.1), dict(kind="adamw", weight_decay=0.1), dict(kind="sgd"), dict(kind="adam"),
        dict(kind="adamw8", weight_decay=0.0, betas=(0.8, 0.95)), dict(kind="adamw", weight_decay=0.0), dict(kind="momentum", momentum=0.9)]


def _hybrid(wl, idx=None, opts=OPTS, keep=True):
    from paper_2408_01331_amd.unifiednn import Hybrid, flatten_params
    idx = list(range(wl.n_models)) if idx is None else idx
    h = Hybrid([wl.specs[i] for i in idx], wl.batch, wl.in_shape, wl.precision)
    th = _theta(wl) if len(wl.in_shape) == 1 else {i: theta0(wl, i) for i in range(wl.n_models)}
    for k, i in enumerate(idx):
        h.set_params(k, flatten_params(th[i]))
        h.set_optimizer(k, **opts[i % len(opts)])
    h.keep_grads(keep)
    return h


def _cnn():
    """CNNs with padded channels and pools, and a concatenated MLP-like head."""
    wl = W.shrink(W.get("lenet4"), batch=16)
    return W.Workload("lenet_bf16", wl.n_models, wl.batch, wl.in_shape, "bf16", wl.specs, wl.lr, 3, 0)


CASES = {"seq_f32": lambda: _wl(SPECS, 20, 192, "f32"), "seq_bf16": lambda: _wl(SPECS, 20, 192, "bf16"), "cnn_bf16": _cnn,
         "cnn_f32": lambda: W.shrink(W.get("lenet4"), batch=16), "mlp8": lambda: W.get("mlp8")}
LR = 0.002


def _adamw64(p, g, m, v, t, o):
    b1, b2 = (float(np.float32(b)) for b in o.get("betas", (0.9, 0.999)))
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    wd, lr = float(np.float32(o.get("weight_decay", 0.0))), float(np.float32(LR))
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    up = lr / (1 - b1 ** t) * m / (np.sqrt(v) / np.sqrt(1 - b2 ** t) + float(np.float32(1e-8)))
    return p * (1 - lr * wd) - up, m, v, np.abs(up)


@pytest.mark.parametrize("name", list(CASES))
def test_adamw_steps(name):
    """Every step of every AdamW model from the gradients that it kept and the state that it had: parameters within
    rounding of the formula in 64 bits, moments too (8 bits: within a step of their codes)."""
    _need_gpu()
    wl = CASES[name]()
    u = 2.0 ** -24
    with _hybrid(wl) as h:
        for s in range(3):
            h.load_batch(*W.make_batch(wl, s))
            before = [(h.get_params(i), h.get_opt_state(i)) for i in range(wl.n_models)]
            h.step(LR)
            for i in range(wl.n_models):
                o = OPTS[i % len(OPTS)]
                if not o["kind"].startswith("adamw"):
                    continue
                (p0, (st, t)), n = before[i], before[i][0].size
                assert t == s
                p, m, v, up = _adamw64(p0, h.get_grads(i), st[:n], st[n:], s + 1, o)
                got, (new, t2) = h.get_params(i), h.get_opt_state(i)
                assert t2 == s + 1
                b1 = o.get("betas", (0.9, 0.999))[0]
                mag = b1 * np.abs(st[:n].astype(np.float64)) + (1 - b1) * np.abs(h.get_grads(i).astype(np.float64))
                rel = np.divide(4 * u * mag, np.abs(m), out=np.zeros(n), where=m != 0)
                # fp32: the parameter's and the update's roundings, and a moment that cancels
                assert (np.abs(got - p) <= 4 * u * np.abs(p) + up * (24 * u + rel) + 1e-44).all(), f"model {i} step {s}"
                if o["kind"] == "adamw":
                    assert (np.abs(new[:n] - m) <= 4 * u * mag + 1e-44).all() and (np.abs(new[n:] - v) <= 6 * u * v + 1e-44).all()
                else:
                    # within a step of the codes: 2^-3 of the value, 2^-9 of the largest scale (at most 2^-7.8 of the largest value)
                    for a, b in ((new[:n], m), (np.sqrt(new[n:].astype(np.float64)), np.sqrt(v))):
                        assert (np.abs(a - b) <= np.maximum(np.abs(b), np.abs(a)) * 2.0 ** -3 * 1.0001 + np.abs(b).max() * 2.0 ** -16.8).all()
                    assert (new[n:][v > 0] > 0).all()


@pytest.mark.parametrize("name", list(CASES))
def test_mixed_optimizers_equal_each_model_alone_bitwise(name):
    """Steps 2 and 3 without model 0 or 1 in the set, too: the others and those two go on as alone."""
    _need_gpu()
    wl = CASES[name]()
    n = wl.n_models
    masks = [np.ones(n, bool) for _ in range(4)]
    masks[1][0] = masks[2][1] = False
    with _hybrid(wl) as h:
        losses = []
        for s in range(4):
            h.set_active(masks[s])
            h.load_batch(*W.make_batch(wl, s))
            losses.append(h.step(LR))
        want = [(h.get_params(i), *h.get_opt_state(i)) for i in range(n)]
    for i in range(n):
        with _hybrid(wl, [i], opts=[OPTS[i % len(OPTS)]] * n) as h:
            h.keep_grads(False)
            for s in range(4):
                if masks[s][i]:
                    h.load_batch(*W.make_batch(wl, s))
                    assert _bits(h.step(LR))[0] == _bits(losses[s])[i], f"model {i} step {s}"
            p, (st, t) = h.get_params(0), h.get_opt_state(0)
        assert np.array_equal(_bits(p), _bits(want[i][0])) and np.array_equal(_bits(st), _bits(want[i][1])) and t == want[i][2], i


def test_adamw8_resumes_from_a_checkpoint(tmp_path):
    """Interrupted by a checkpoint and resumed in a fresh hybrid, the run is the uninterrupted one, bit for bit; so it is after
    another model has changed its optimizer."""
    _need_gpu()
    from paper_2408_01331_amd import checkpoint as C
    wl = _wl(SPECS, 20, 192, "bf16")
    n = wl.n_models
    with _hybrid(wl) as h:
        for s in range(2):
            h.load_batch(*W.make_batch(wl, s))
            h.step(LR)
        for i in (0, 1, 4):
            C.save(h, i, str(tmp_path / f"{i}.safetensors"))
        for s in range(2, 4):
            h.load_batch(*W.make_batch(wl, s))
            h.step(LR)
        want = {i: h.get_params(i) for i in (0, 1, 4)}
        h.set_optimizer(0, "sgd")
        assert h.get_opt_state(0)[0].size == 0
        h.step(LR)
    with _hybrid(wl, opts=[dict(kind="sgd")]) as h:
        for i in (4, 0, 1):
            C.load(h, i, str(tmp_path / f"{i}.safetensors"))
        for s in range(2, 4):
            if s == 3:
                h.set_optimizer(2, "adamw8")
            h.load_batch(*W.make_batch(wl, s))
            h.step(LR)
        for i in want:
            assert np.array_equal(_bits(h.get_params(i)), _bits(want[i])), i


def test_graph_scratch_and_stream():
    """A captured step, one in the static workspace and one on another stream give the bits of the plain step."""
    _need_gpu()
    import torch
    from paper_2408_01331_amd.unifiednn import un_step_scratch
    for precision in ("f32", "bf16"):
        wl = _wl(SPECS, 37, 192, precision)
        hs = [_hybrid(wl, opts=[dict(kind="sgd")], keep=False) for _ in range(4)]
        try:
            stream = torch.cuda.Stream()
            hs[3].set_stream(stream.cuda_stream)
            hs[1].load_batch(*W.make_batch(wl, 0))
            hs[1].capture(0.05)
            for s in range(4):
                for h in hs:
                    h.load_batch(*W.make_batch(wl, s))
                a, b = hs[0].step(0.05), hs[1].replay()
                c, d = un_step_scratch(hs[2].ctx, 0.05, wl.n_models), hs[3].step(0.05)
                assert np.array_equal(_bits(a), _bits(b)) and np.array_equal(_bits(a), _bits(c)) and np.array_equal(_bits(a), _bits(d))
            for i in range(wl.n_models):
                p = [h.get_params(i) for h in hs]
                assert all(np.array_equal(_bits(p[0]), _bits(q)) for q in p[1:])
            hs[1].set_optimizer(0, "adamw8")
            from paper_2408_01331_amd.unifiednn import UnError
            with pytest.raises(UnError):
                hs[1].capture(0.05)
        finally:
            for h in hs:
                h.close()


def test_profile_classes():
    _need_gpu()
    from paper_2408_01331_amd import unifiednn as un
    wl = _wl(SPECS, 20, 192, "bf16")
    with _hybrid(wl) as h:
        h.load_batch(*W.make_batch(wl, 0))
        un.un_profile_enable(h.ctx, True)
        h.step(LR)
        got = {k: un.un_profile_read(h.ctx, j) for j, k in enumerate(un.KERNEL_CLASSES)}
    assert got["recurrence"][1] >= 2 and got["norm"][1] >= 2 and got["adamw"][1] == 1 and got["adamw"][0] > 0
