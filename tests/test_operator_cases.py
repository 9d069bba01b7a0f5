"""CPU tests of the operators' cases (perf/operators.py): what a pass hands to the
operators' calls, on small states made here."""
import pytest

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("prec", ["f32", "bf16"])
@pytest.mark.parametrize("ragged", [False, True])
def test_backward_gets_both_gradients(prec, ragged, monkeypatch):
    """Every training pass of the recurrence hands the gradient at h and the one at the last state to the backward call, as
    they are in the state."""
    from paper_2408_01331_amd import operators as ops
    from perf import operators as cases
    b, n, d = 2, 5, 8
    t = cases.TYPES[prec]
    st = dict(case=cases._scan("x", b, n, d, prec, "train", ragged=ragged), gate=torch.randn(b, n, d).to(t), value=torch.randn(b, n, d).to(t),
              h0=None, lens=torch.tensor([n, 2], dtype=torch.int32) if ragged else None, dh=torch.randn(b, n, d).to(t),
              dlast=torch.randn(b, d))
    seen = []

    def forward(gate, value, h0=None, lens=None, keep=False):
        return torch.zeros_like(gate), torch.zeros(b, d), torch.zeros(1)

    def backward(gate, value, states, dh, dlast=None, lens=None, out=None):
        seen.append((dh.clone(), None if dlast is None else dlast.clone(), lens))
        return torch.zeros(b, d)

    monkeypatch.setattr(ops, "gated_scan", forward)
    monkeypatch.setattr(ops, "gated_scan_backward", backward)
    monkeypatch.setattr(cases, "own", True)
    dh, dlast = st["dh"].clone(), st["dlast"].clone()
    cases.run(st)
    assert len(seen) == 1 and torch.equal(seen[0][0], dh) and seen[0][2] is st["lens"]
    assert seen[0][1] is not None and torch.equal(seen[0][1], dlast)


@pytest.mark.parametrize("prec", ["f32", "bf16"])
@pytest.mark.parametrize("ragged", [False, True])
def test_both_passes_leave_the_same_inputs(prec, ragged, monkeypatch):
    """After a pass of either kind the state's gradient buffer holds the same values: the next pass has the same inputs."""
    from paper_2408_01331_amd import operators as ops
    from perf import operators as cases
    b, n, d = 2, 5, 8
    t = cases.TYPES[prec]
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    base = dict(gate=r(b, n, d).to(t), value=r(b, n, d).to(t), h0=None, lens=torch.tensor([n, 2], dtype=torch.int32) if ragged else None,
                dh=r(b, n, d).to(t), dlast=r(b, d))
    monkeypatch.setattr(ops, "gated_scan", lambda gate, *a, **k: (torch.zeros_like(gate), torch.zeros(b, d), torch.zeros(1)))
    monkeypatch.setattr(ops, "gated_scan_backward", lambda *a, **k: torch.zeros(b, d))
    left = []
    for own in (False, True):
        monkeypatch.setattr(cases, "own", own)
        st = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in base.items()}
        st["case"] = cases._scan("x", b, n, d, prec, "train", ragged=ragged)
        cases.run(st)
        left.append(st)
    for k in ("gate", "value", "dh", "dlast"):
        assert torch.equal(left[0][k], left[1][k]), k
