"""CPU: which kernels the operators at the ends of a language model take, recorded
from calls on a HIP runtime of the host that runs nothing. The GPU tests run at
the sizes of _lm_operator_sizes.py for the sake of these kernels; where a rule
that chooses them changes, these tests say which sizes have to follow."""
import pytest

pytest.importorskip("torch")

import _host_hip  # noqa: E402
import _lm_operator_sizes as S  # noqa: E402

CODE = """
import re
import _lm_operator_sizes as S
P = 1 << 20


def call(fn, **args):
    a = getattr(U, fn[:-9] + "_grad_args" if fn.endswith("_backward") else fn + "_args")
    status = getattr(U.lib(), fn)(ctypes.byref(a(**args)), None)
    assert status == 0, U.lib().un_last_error(None)
    return [l[0] for l in launches()]


def layer(t, rows, width):
    b = dict(type=t, width=width, rows=rows, weight=P)
    names = call("un_layer_norm", eps=1e-5, x=P, ldx=width, y=P, ldy=width, **b)
    names += call("un_layer_norm_backward", dy=P, lddy=width, s=P, lds=width, stats=P, dx=P, lddx=width, dweight=P, dbias=P, workspace=P,
                  workspace_bytes=1 << 40, **b)
    found = [re.search(r"layer_(fwd|bwd)_kernelI.Li(\\d+)ELi(\\d+)ELi(\\d+)E", n) for n in names]
    return [[m.group(1), *map(int, m.groups()[1:])] for m in found if m]


def blocks(t, rows, width):
    need = ctypes.c_size_t()
    U.lib().un_layer_norm_workspace(t, rows, width, ctypes.byref(need))
    return need.value // (8 * width)


def sorts(tokens, vocab, width):
    names = call("un_embedding_backward", type=0, width=width, vocab=vocab, index_bits=64, tokens=tokens, ids=P, dy=P, lddy=width, scale=1.0,
                 padding=-1, dweight=P, lddw=width, workspace=P, workspace_bytes=1 << 40)
    if any("sort_one_kernel" in n for n in names):
        return "one"
    moves = [int(m.group(1)) for m in (re.search(r"sort_move_kernelILi(\\d+)E", n) for n in names) if m]
    return [moves[0], len(moves)]


def head(t, rows, width, vocab, more, off, *_):
    b = dict(type=t, width=width, vocab=vocab, index_bits=64, rows=rows, x=P, ldx=width, weight=P + off * (2 if t else 4), ldw=width + more,
             targets=P, lse=P, workspace=P, workspace_bytes=1 << 50)
    names = call("un_vocab_loss", loss=P, **b)
    names += call("un_vocab_loss_backward", dloss=P, dloss_stride=1, dx=P, lddx=width, dweight=P, lddw=width, **b)
    found = [re.search(r"head_kernelILNS_8HeadKindE(\\d)ENS0_7HeadCfgILi(\\d+)ELi(\\d+)E.*Lb([01])E", n) for n in names]
    found = [list(map(int, m.groups())) for m in found if m]
    tiles = [sorted({(m, n) for kind, m, n, _ in found if kind == k}) for k in range(4)]
    regs = {r for kind, *_, r in found if kind < 3}
    joins = sum("head_join_kernel" in n for n in names)
    pieces = sum(kind == 1 for kind, *_ in found)
    return [tiles, sorted(regs), pieces, joins > 1]


result = dict(two=[layer(*c[:3]) for c in S.LAYER_TWO_ROWS], shares=[[layer(*c), blocks(*c)] for c in S.LAYER_SHARES],
              sorts=[sorts(*c[:3]) for c in S.EMBED_SORTS], heads=[head(*c) for c in S.HEADS])
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    return _host_hip.run(CODE, tmp_path_factory.mktemp("plans"))


def test_layer_norm_of_two_rows_a_thread(plans):
    for c, got in zip(S.LAYER_TWO_ROWS, plans["two"]):
        assert got[0] == ["fwd", c[3], c[4], 2], c
    assert {(t, tpr) for t, _, _, tpr, _ in S.LAYER_TWO_ROWS} == {(t, tpr) for t in (0, 1) for tpr in (16, 64, 256, 1024)}


def test_layer_norm_of_several_rows_a_workgroup(plans):
    for c, (got, blocks) in zip(S.LAYER_SHARES, plans["shares"]):
        assert got[1] == ["bwd", 1024, got[1][2], 1] and c[1] > 2 * blocks, c
        assert (got[1][2] * (8 if c[0] else 4) > 8) == (c[2] > 8192), c  # (more values of a thread than it has registers for)


def test_embedding_sorts(plans):
    for c, got in zip(S.EMBED_SORTS, plans["sorts"]):
        assert got == (c[3] if c[3] == "one" else list(c[3])), c


def test_vocabulary_losses(plans):
    for c, (tiles, regs, pieces, parts) in zip(S.HEADS, plans["heads"]):
        assert [t[0] for t in tiles] == [list(t) for t in c[6]] and all(len(t) == 1 for t in tiles), c
        assert (regs, pieces, parts) == (c[7], c[8], c[9]), c
    # every kind of tiles of every product, with the weights loaded directly (the small ones in bf16 are what other tests' sizes
    # take) and through registers
    for t, reg, kinds in ((1, False, {S.LARGE, S.MEDIUM}), (1, True, {S.MEDIUM, S.SMALL}), (0, False, {S.TERMS_LARGE, S.TERMS}),
                          (0, True, {S.TERMS})):
        for k in range(3):
            assert kinds <= {c[6][k] for c in S.HEADS if c[0] == t and c[7] == [int(reg)]}, (t, reg, k)
        assert kinds <= {c[6][3] for c in S.HEADS if c[0] == t}
