"""Pins for the oracle's RMS norm, gated recurrence and AdamW (torch modules,
autograd and torch.optim in float64, central differences), and host-side tests
of the same layers and optimizers: specs, parameter layout, checkpoint names,
8-bit states."""
import numpy as np
import pytest

import _host_hip as H
import oracle
from paper_2408_01331_amd import checkpoint as C
from paper_2408_01331_amd import workloads as W

torch = pytest.importorskip("torch")
D = torch.float64

U, N, G, A, L, RELU, FLAT, RB, RE = (lambda t: ("unflatten", t)), ("rms_norm",), ("recurrence",), ("attention",), \
    (lambda n: ("linear", n)), ("relu",), ("flatten",), ("res_begin",), ("res_end",)
SPECS = {
    "norm_flat": ({"layers": [L(12), RELU, N, L(5)], "num_classes": 5}, (8,)),
    "norm_input": ({"layers": [N, L(6), RELU, N, L(4)], "num_classes": 4}, (16,)),
    "recurrence": ({"layers": [U(6), G, FLAT, L(5)], "num_classes": 5}, (6 * 8,)),
    "pre_norm": ({"layers": [U(5), L(8), RB, N, G, RE, RB, N, L(16), RELU, L(8), RE, N, L(8), FLAT, L(3)], "num_classes": 3}, (5 * 8,)),
    "input_block": ({"layers": [U(4), RB, N, G, RE, RELU, FLAT, N, L(3)], "num_classes": 3}, (4 * 8,)),
    "with_attention": ({"layers": [U(4), N, A, RB, G, RE, RELU, FLAT, L(3)], "num_classes": 3}, (4 * 8,)),
}


class _Residual(torch.nn.Module):
    def __init__(self, inner):
        super().__init__()
        self.inner = inner

    def forward(self, x):
        return self.inner(x) + x


class _Attention(torch.nn.Module):
    def __init__(self, d):
        super().__init__()
        self.mha = torch.nn.MultiheadAttention(d, 1, batch_first=True, dtype=D)

    def forward(self, x):
        return self.mha(x, x, x, need_weights=False)[0]


class _Recurrence(torch.nn.Module):
    def __init__(self, d):
        super().__init__()
        self.inp, self.out = torch.nn.Linear(d, 2 * d, dtype=D), torch.nn.Linear(d, d, dtype=D)

    def forward(self, x):
        g, v = self.inp(x).chunk(2, -1)
        a, h, out = torch.sigmoid(g), torch.zeros_like(v[:, 0]), []
        for t in range(x.shape[1]):
            h = a[:, t] * h + (1 - a[:, t]) * v[:, t]
            out.append(h)
        return self.out(torch.stack(out, 1))


def _model(spec, in_shape, params):
    mods, stack, shape = [], [], tuple(in_shape)
    for layer in spec["layers"]:
        op = layer[0]
        if op == "res_begin":
            stack.append(mods)
            mods = []
        elif op == "res_end":
            inner = torch.nn.Sequential(*mods)
            mods = stack.pop()
            mods.append(_Residual(inner))
        elif op == "unflatten":
            mods.append(torch.nn.Unflatten(1, (layer[1], shape[0] // layer[1])))
            shape = (layer[1], shape[0] // layer[1])
        elif op == "linear":
            mods.append(torch.nn.Linear(shape[-1], layer[1], dtype=D))
            shape = shape[:-1] + (layer[1],)
        elif op == "flatten":
            mods.append(torch.nn.Flatten())
            shape = (int(np.prod(shape)),)
        else:
            mods.append({"relu": torch.nn.ReLU, "rms_norm": lambda: torch.nn.RMSNorm(shape[-1], eps=1e-6, dtype=D),
                         "recurrence": lambda: _Recurrence(shape[-1]), "attention": lambda: _Attention(shape[-1])}[op]())
    model = torch.nn.Sequential(*mods)
    with torch.no_grad():
        for tp, p in zip(model.parameters(), params):
            assert tuple(tp.shape) == np.shape(p)
            tp.copy_(torch.tensor(p))
    return model


def _setup(name, batch=5):
    spec, shape = SPECS[name]
    rng = np.random.default_rng([3, len(name)])
    params = [np.asarray(p, np.float64) + 0.1 * rng.standard_normal(np.shape(p)) for p in W.init_params(spec, shape, 3, 0, "torch")]
    x = rng.standard_normal((batch,) + shape)
    y = rng.integers(0, spec["num_classes"], batch)
    return spec, shape, params, x, y


@pytest.mark.parametrize("name", list(SPECS))
def test_forward_and_gradients_against_autograd(name):
    spec, shape, params, x, y = _setup(name)
    model = _model(spec, shape, params)
    assert sum(p.numel() for p in model.parameters()) == oracle.count_params(spec, shape)
    logits = model(torch.tensor(x))
    z, cache = oracle.forward(spec, params, x, "f64")
    assert np.max(np.abs(z - logits.detach().numpy())) <= 1e-12 * np.max(np.abs(z))
    loss = torch.nn.functional.cross_entropy(logits, torch.tensor(y))
    loss.backward()
    lo, dz = oracle.softmax_ce(z, y)
    grads = oracle.backward(spec, params, cache, dz, "f64")
    assert abs(lo - loss.item()) <= 1e-12
    for g, p in zip(grads, model.parameters()):
        assert np.max(np.abs(g - p.grad.numpy())) <= 1e-11 * max(1e-3, np.max(np.abs(g)))


@pytest.mark.parametrize("name", ["pre_norm", "input_block"])
def test_gradients_by_differences(name):
    spec, shape, params, x, y = _setup(name)
    z, cache = oracle.forward(spec, params, x, "f64")
    grads = oracle.backward(spec, params, cache, oracle.softmax_ce(z, y)[1], "f64")
    rng = np.random.default_rng(0)
    for t, g in enumerate(grads):
        for _ in range(3):
            i = tuple(rng.integers(0, n) for n in g.shape)
            p = [q.copy() for q in params]
            p[t][i] += 1e-5
            up = oracle.loss_only(spec, p, x, y)
            p[t][i] -= 2e-5
            num = (up - oracle.loss_only(spec, p, x, y)) / 2e-5
            assert abs(num - g[i]) <= 1e-7 + 1e-5 * abs(num)


def test_bf16_norm_and_recurrence_read_operands():
    """bf16 mode: every projection, norm and core reads bf16 values; the norm's
    weight, the state and the row's root are not rounded."""
    spec, shape, params, x, y = _setup("recurrence")
    params = [oracle.to_f32(p) for p in params]
    z, cache = oracle.forward(spec, params, x, "bf16")
    entry = next(e for e in cache if e[0] == "recurrence")
    for a in entry[2:6] + entry[8:]:
        assert np.array_equal(a, oracle.to_bf16(a))
    assert not np.array_equal(entry[6], oracle.to_bf16(entry[6]))


def test_adamw_against_torch():
    rng = np.random.default_rng(1)
    p = [rng.standard_normal((4, 3)), rng.standard_normal(5)]
    tp = [torch.tensor(a, requires_grad=True) for a in p]
    opt = torch.optim.AdamW(tp, lr=0.03, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.2)
    m, v = [np.zeros_like(a) for a in p], [np.zeros_like(a) for a in p]
    for t in range(1, 6):
        g = [rng.standard_normal(a.shape) for a in p]
        for q, gg in zip(tp, g):
            q.grad = torch.tensor(gg)
        opt.step()
        p, m, v = oracle.adamw_update(p, g, m, v, t, 0.03, 0.8, 0.95, 1e-6, 0.2, "f64")
        for a, q in zip(p, tp):
            assert np.max(np.abs(a - q.detach().numpy())) <= 1e-13


# ---------------------------------------------------------------------------
# The library on the host
# ---------------------------------------------------------------------------
def _plan(spec, shape, batch=4, precision="f32"):
    from paper_2408_01331_amd import unifiednn as un
    import os
    if not os.path.exists(un.LIB_PATH):
        from paper_2408_01331_amd.build import build
        build()
    try:
        un.un_plan_bytes([spec], batch, shape, precision)
    except un.UnError as e:
        return e.status, str(e)
    return 0, ""


@pytest.mark.parametrize("layers,shape,status,text", [
    ([L(16), G, L(3)], (8,), 1, "needs a sequence"),
    ([L(16), N, RELU, L(3)], (8,), 7, "must directly follow"),
    ([("conv", 8, 3, 1), N, FLAT, L(3)], (3, 4, 4), 7, "a norm"),
    ([("conv", 8, 3, 1), FLAT, N, L(3)], (3, 4, 4), 7, "a norm"),
    ([N, ("conv", 8, 3, 1), FLAT, L(3)], (3, 4, 4), 7, "a norm"),
    ([L(8), RB, L(8), N, RE, L(3)], (8,), 7, "must end with"),
    ([L(20000), RELU, N, L(3)], (8,), 7, "16384"),
    ([L(3), N], (8,), 7, "last layer"),
    ([U(4), RB, G, G, RE, L(6), FLAT, L(3)], (32,), 7, "multiple of 8"),
])
def test_specs_refused(layers, shape, status, text):
    s, msg = _plan({"layers": layers, "num_classes": 3}, shape)
    assert s == status and text in msg, msg


@pytest.mark.parametrize("name", list(SPECS))
def test_specs_accepted(name):
    spec, shape = SPECS[name]
    for precision in ("f32", "bf16"):
        assert _plan(spec, shape, 4, precision)[0] == 0
    # any number of tokens, where attention has a limit
    assert _plan({"layers": [U(4096), G, FLAT, L(3)], "num_classes": 3}, (4096 * 8,))[0] == 0


def test_checkpoint_names():
    spec, shape = SPECS["pre_norm"]
    names = C.param_names(spec)
    assert len(names) == len(W.param_shapes(spec, shape)) == len(set(names))
    assert names[2:7] == ["2.inner.0.weight", "2.inner.1.in_proj_weight", "2.inner.1.in_proj_bias", "2.inner.1.out_proj.weight",
                          "2.inner.1.out_proj.bias"]


STATES = """
spec = {"layers": [("conv", 5, 3, 1), ("relu",), ("pool",), ("flatten",), ("linear", 7), ("relu",), ("rms_norm",), ("linear", 3)],
        "num_classes": 3}
seq = {"layers": [("unflatten", 6), ("linear", 24), ("recurrence",), ("flatten",), ("rms_norm",), ("linear", 3)], "num_classes": 3}
h = U.Hybrid([spec, seq], None, None, %r, inputs=[(4, (2, 8, 8)), (4, (48,))], group_of=[0, 1])
rng = np.random.default_rng(0)
out = []
for i in range(2):
    p = rng.standard_normal(U.un_param_count(h.ctx, i)).astype(np.float32)
    h.set_params(i, p)
    out.append(bool(np.array_equal(h.get_params(i), p)))
    h.set_optimizer(i, "adamw8", weight_decay=0.1)
    z, t = h.get_opt_state(i)
    out.append(bool(z.size == 2 * p.size and not z.any() and t == 0))
    m = rng.standard_normal(p.size).astype(np.float32) * np.exp(rng.uniform(-8, 2, p.size)).astype(np.float32)
    v = (m * m).astype(np.float32)
    v[::7] = 1e-9
    h.set_opt_state(i, np.concatenate([m, v]), 12)
    s, t = h.get_opt_state(i)
    h.set_opt_state(i, s, 12)
    again = h.get_opt_state(i)[0]
    # codes within half a step, 2^-4 of the value (of v's root, so 2^-3 and its square of v), or 2^-10 of a scale of
    # at most 2^-7.8 of the largest value; what was read comes back exactly, and no second moment becomes zero
    top = np.abs(m).max() * 2.0 ** -16.8
    out.append(bool(t == 12 and np.array_equal(s, again) and (np.abs(s[:p.size] - m) <= np.maximum(2.0 ** -4 * np.abs(m), top)).all()))
    u, w = np.sqrt(s[p.size:]), np.sqrt(v)
    out.append(bool((np.abs(u - w) <= np.maximum(2.0 ** -4 * w, 2 * top)).all() and (s[p.size:] > 0).all()))
    for bad in (np.inf, np.nan):
        q = s.copy()
        q[0] = bad
        try:
            h.set_opt_state(i, q, 1)
            out.append(False)
        except U.UnError as e:
            out.append(e.status == U.UN_ERR_INVALID)
held = stub.stub_device()
h.set_optimizer(0, "sgd")
h.set_optimizer(1, "sgd")
out.append(held - stub.stub_device() == 3)  # both states, and their table
for kw in (dict(weight_decay=-1.0), dict(weight_decay=float("nan")), dict(eps=0.0), dict(betas=(1.0, 0.9))):
    for kind in ("adamw", "adamw8"):
        try:
            h.set_optimizer(0, kind, **kw)
            out.append(False)
        except U.UnError as e:
            out.append(e.status == U.UN_ERR_INVALID)
h.set_optimizer(0, "adamw", weight_decay=2.0)
h.load_batch(np.zeros((4, 2, 8, 8), np.float32), np.zeros(4, np.int32), 0)
h.load_batch(np.zeros((4, 48), np.float32), np.zeros(4, np.int32), 1)
launches()
for lr in (0.5, -0.1):
    try:
        h.step(lr)
        out.append(False)
    except U.UnError as e:
        out.append(e.status == U.UN_ERR_INVALID and not launches())
h.step([0.4, -0.5])  # model 1 is plain SGD
out.append(len(launches()) > 0)
h.close()
out.append(stub.stub_device() == 0)
result = out
"""


@pytest.mark.parametrize("precision", ["f32", "bf16"])
def test_parameters_and_8_bit_states_on_the_host(precision, tmp_path):
    """Parameters through the internal layouts and back, 8-bit states set and read, refusals, and what is given back."""
    res = H.run(STATES % precision, tmp_path)
    assert all(res), res


def test_launches_of_a_step(tmp_path):
    """One launch per level and operator for all models; short sequences on one wave, norms by their rows' plans."""
    res = H.run("""
U_, N, G = (lambda t: ("unflatten", t)), ("rms_norm",), ("recurrence",)
a = {"layers": [U_(8), N, G, ("flatten",), ("linear", 3)], "num_classes": 3}
b = {"layers": [U_(128), N, G, ("flatten",), ("linear", 3)], "num_classes": 3}
def names(specs):
    h = U.Hybrid(specs, 4, (1024,), "bf16")
    h.load_batch(np.zeros((4, 1024), np.float32), np.zeros(4, np.int32))
    h.set_optimizer(0, "adamw8")
    launches()
    h.step(0.1)
    return [l[0] + " " + str(l[2]) for l in launches() if "scan" in l[0] or "norm" in l[0] or "adamw" in l[0]]
result = [names([a]), names([a, b]), names([{"layers": [("linear", w), ("relu",), N, ("linear", 3)], "num_classes": 3} for w in (64, 4096, 128)])]
""", tmp_path)
    short, mixed, wide = res
    assert len(short) == 5 and sum("scan" in x and x.endswith(" 64") for x in short) == 2 and "adamw" in short[-1]
    assert len(mixed) == 5 and sum("scan" in x and x.endswith(" 512") for x in mixed) == 2
    assert sum("norm_fwd" in x for x in wide) == 2  # 64 and 128 features in one, 4096 in another
