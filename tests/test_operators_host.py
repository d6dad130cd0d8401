"""Host side of the norm, the products by group, the scores and the distillation: the oracle's
formulas by hand and against differences, and the calls that are refused, none of which needs a GPU."""
import ctypes

import numpy as np
import pytest

import paper_2111_00352_amd as gs
from oracle import operators as oracle


def test_oracle_norm_by_hand():
    Y, r = oracle.rms_norm(np.array([[3.0, 4.0], [0.0, 0.0]]), np.array([1.0, 2.0]), 0.0)
    assert np.allclose(Y[0], [3 / 12.5 ** 0.5, 8 / 12.5 ** 0.5]) and np.isinf(r[1]) and np.isnan(Y[1]).all()


def test_oracle_scores_by_hand():
    s = np.log(np.array([[1.0, 2.0, 1.0], [1.0, 1.0, 2.0]]))
    s[1, 0] = -np.inf
    lp, H, every = oracle.scores(s, np.array([1, -1]))
    assert np.allclose(lp, [np.log(0.5), 0.0]) and np.allclose(H[0], 1.5 * np.log(2))
    assert np.allclose(every[1, 1:], np.log([1 / 3, 2 / 3])) and np.isneginf(every[1, 0])
    assert oracle.best(np.array([[1.0, 3.0, 3.0, np.nan, -0.0, 0.0]]), 6).tolist() == [[3, 1, 2, 0, 4, 5]]
    assert np.isnan(oracle.scores(np.full((1, 2), -np.inf), [0])[0]).all()


def test_oracle_distill_by_hand():
    s = np.zeros((3, 4))
    ids = np.array([[0, 1], [-1, -1], [2, 2]])
    loss, d, q, _, _ = oracle.distill(s, ids, np.zeros((3, 2)), 1.0)
    assert np.allclose(loss, [np.log(2), 0.0, np.log(2)])  # q is 1/2 each; two halves of one class
    assert np.allclose(d[0], [-0.25, -0.25, 0.25, 0.25]) and (d[1] == 0).all() and np.allclose(d[2], [0.25, 0.25, -0.75, 0.25])


def _differences(f, x, h=1e-6):
    d = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        d[i] = (f(up) - f(down)) / (2 * h)
    return d


def test_oracle_gradients_are_derivatives():
    rng = np.random.default_rng(0)
    s, ids = rng.standard_normal((3, 5)), np.array([4, -1, 0])
    g, e = rng.standard_normal(3), rng.standard_normal(3)
    lp, H, every = oracle.scores(s, ids)
    want = _differences(lambda x: (g * oracle.scores(x, ids)[0]).sum() + (e * oracle.scores(x, ids)[1]).sum(), s)
    assert np.allclose(oracle.scores_grad(every, H, ids, g, e), want, atol=1e-8)
    t, tid = rng.standard_normal((3, 2)), np.array([[1, 3], [0, 0], [2, -1]])
    for T in (1.0, 2.5):
        want = _differences(lambda x: oracle.distill(x, tid, t, T)[0].sum(), s)
        assert np.allclose(oracle.distill(s, tid, t, T)[1], want, atol=1e-7)
    A, W, off = rng.standard_normal((6, 3)), rng.standard_normal((2, 3, 4)), [1, 4, 5]
    G = rng.standard_normal((6, 4))
    assert np.allclose(oracle.grouped(G, W, off, True)[0], _differences(lambda x: (oracle.grouped(x, W, off, False)[0] * G).sum(), A), atol=1e-8)
    assert np.allclose(oracle.grouped_grad(A, G, off)[0], _differences(lambda x: (oracle.grouped(A, x, off, False)[0] * G).sum(), W), atol=1e-8)


def _saved(rows=4, cols=8, act=0, codes=256, scales=256):
    return ctypes.byref(gs._Saved(rows, cols, act, codes, scales))


P, BAD, NOT = 512, gs.ERR_INVALID_ARG, gs.ERR_UNSUPPORTED
P2, P3, P4 = (P + (i << 20) for i in range(1, 4))  # (apart from each other, whatever the sizes here)


def _with(args, **changes):
    names, values = args
    return [changes.get(n, v) for n, v in zip(names, values)]


NORM = ("X ldx R ldr dtype rows cols w w_dtype eps H ldh Y ldy saved rstd stream".split(),
        [P, 8, P2, 8, 0, 4, 8, P, 0, 1e-6, P3, 8, P4, 8, None, P, None])


@pytest.mark.parametrize("changes", [
    dict(X=None), dict(ldx=7), dict(X=P + 2), dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(ldr=7),
    dict(H=None), dict(ldh=7), dict(Y=None), dict(ldy=7), dict(saved=_saved()), dict(Y=None, saved=_saved(act=1)),
    dict(Y=None, saved=_saved(cols=9)), dict(Y=None, saved=_saved(codes=264)), dict(rstd=None), dict(w=P + 2), dict(w_dtype=3), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(ldx=1 << 61),
    dict(H=P + 4), dict(H=P2 + 32), dict(H=P, ldh=9), dict(Y=P), dict(Y=P2), dict(Y=P3), dict(Y=P3 + 124), dict(Y=P3 - 124)])
def test_norm_refuses(changes):
    assert gs.lib().gs_rms_norm(*_with(NORM, **changes)) == BAD


def test_norm_refuses_too_wide_and_takes_no_rows():
    big = 1 << 25
    assert gs.lib().gs_rms_norm(*_with(NORM, cols=big, ldx=big, ldr=big, ldh=big, ldy=big)) == NOT
    assert gs.lib().gs_rms_norm(*_with(NORM, rows=0, X=None, R=None, H=None, Y=None, rstd=None)) == 0


NORM_GRAD = ("H ldh rstd dY ldy dtype rows cols w w_dtype dH ldd dX ldx dw work bytes stream".split(),
             [P, 8, P, P2, 8, 0, 4, 8, P, 0, P3, 8, P4, 8, P, P, 1 << 20, None])


@pytest.mark.parametrize("changes", [
    dict(H=None), dict(ldh=7), dict(rstd=None), dict(dY=None), dict(ldy=7), dict(dtype=5), dict(rows=-1), dict(cols=0), dict(w=P + 1), dict(w_dtype=2),
    dict(ldd=7), dict(dX=None), dict(ldx=7), dict(work=None), dict(bytes=3),
    dict(dX=P), dict(dX=P2), dict(dX=P3 + 4), dict(dX=P3, ldx=9)])
def test_norm_grad_refuses(changes):
    assert gs.lib().gs_rms_norm_grad(*_with(NORM_GRAD, **changes)) == BAD


def test_workspaces():
    need = ctypes.c_uint64()
    L = gs.lib()
    assert L.gs_rms_norm_grad_workspace(100_000, 128, 0, ctypes.byref(need)) == 0 and 0 < need.value <= 32 << 20
    assert L.gs_rms_norm_grad_workspace(10, 1 << 24, 1, ctypes.byref(need)) == 0 and need.value <= 1 << 27
    assert L.gs_rms_norm_grad_workspace(10, 0, 0, ctypes.byref(need)) == BAD
    assert L.gs_rms_norm_grad_workspace(10, 8, 2, ctypes.byref(need)) == BAD
    assert L.gs_rms_norm_grad_workspace(10, 8, 0, None) == BAD
    for args in ((2_000_000, 7, 128, 128), (16_384, 16, 4096, 4096), (1_000_000, 1, 8192, 8192), (1_000_000, 60_000, 64, 64)):
        assert L.gs_grouped_weight_grad_workspace(*args, ctypes.byref(need)) == 0 and need.value <= 2 << 30
    assert L.gs_grouped_weight_grad_workspace(5, 0, 4, 4, ctypes.byref(need)) == BAD
    assert L.gs_grouped_weight_grad_workspace(5, 1 << 16, 4, 4, ctypes.byref(need)) == NOT
    assert L.gs_grouped_weight_grad_workspace(5, 1, 0, 4, ctypes.byref(need)) == BAD
    assert L.gs_grouped_weight_grad_workspace(5, 1, 4, 1 << 25, ctypes.byref(need)) == NOT
    assert L.gs_grouped_weight_grad_workspace(5, 1, 4, 4, None) == BAD


GROUPED = ("A lda dtype rows W ldw step groups k n transpose offsets bytes fill C ldc c_dtype stream".split(),
           [P, 8, 0, 4, P2, 16, 128, 3, 8, 16, 0, P, 4, 1, P3, 16, 0, None])


@pytest.mark.parametrize("changes", [
    dict(A=None), dict(lda=7), dict(dtype=2), dict(rows=-1), dict(W=None), dict(ldw=15), dict(step=-1), dict(step=1 << 61), dict(groups=0), dict(k=0),
    dict(n=0), dict(transpose=1), dict(offsets=None), dict(offsets=P + 2), dict(bytes=2), dict(bytes=8, offsets=P + 4), dict(C=None), dict(ldc=15),
    dict(c_dtype=7), dict(C=P + 2), dict(C=P), dict(C=P + 32), dict(lda=24, ldc=24, C=P + 28), dict(C=P2),
    dict(C=P2 + 1532), dict(C=P2 + 508, step=0), dict(C=P2 - 252)])
def test_grouped_matmul_refuses(changes):
    assert gs.lib().gs_grouped_matmul(*_with(GROUPED, **changes)) == BAD


def test_grouped_matmul_limits():
    L = gs.lib()
    assert L.gs_grouped_matmul(*_with(GROUPED, groups=1 << 16)) == NOT
    assert L.gs_grouped_matmul(*_with(GROUPED, k=1 << 25, lda=1 << 25)) == NOT
    assert L.gs_grouped_matmul(*_with(GROUPED, rows=0, A=None, C=None)) == 0
    args = [P, 0, 16, 128, 3, 8, 16, 0, P, 4, 1, P, 16, 0, None]
    assert L.gs_grouped_matmul_saved(None, *args) == BAD
    assert L.gs_grouped_matmul_saved(_saved(cols=9), *args) == BAD
    assert L.gs_grouped_matmul_saved(_saved(scales=None), *args) == BAD
    assert L.gs_grouped_matmul_saved(_saved(rows=0, codes=None, scales=None), *args) == 0


GROUPED_GRAD = ("A lda G ldg dtype rows a b groups offsets bytes out work work_bytes stream".split(),
                [P, 8, P, 16, 0, 4, 8, 16, 3, P, 4, P, None, 0, None])


@pytest.mark.parametrize("changes", [
    dict(A=None), dict(lda=7), dict(G=None), dict(ldg=15), dict(dtype=2), dict(rows=-1), dict(a=0), dict(b=0), dict(groups=0), dict(offsets=None),
    dict(bytes=1), dict(out=None), dict(rows=100_000)])
def test_grouped_weight_grad_refuses(changes):
    assert gs.lib().gs_grouped_weight_grad(*_with(GROUPED_GRAD, **changes)) == BAD
    assert gs.lib().gs_grouped_weight_grad_saved(None, P, 16, 0, 16, 3, P, 4, P, None, 0, None) == BAD


SCORES = ("s ld dtype n v ids bytes logp entropy stats top top_ids top_logp stream".split(),
          [P, 8, 0, 4, 8, P, 8, P, P, P, 3, P, P, None])


@pytest.mark.parametrize("changes", [
    dict(s=None), dict(ld=7), dict(dtype=2), dict(n=-1), dict(v=0), dict(ids=None), dict(bytes=2), dict(ids=P + 4), dict(top=-1), dict(top=9),
    dict(top_ids=None), dict(top_logp=None)])
def test_log_probs_refuses(changes):
    assert gs.lib().gs_log_probs(*_with(SCORES, **changes)) == BAD


def test_log_probs_limits():
    L = gs.lib()
    assert L.gs_log_probs(*_with(SCORES, v=200, ld=200, top=129)) == NOT
    assert L.gs_log_probs(*_with(SCORES, v=1 << 25, ld=1 << 25)) == NOT
    assert L.gs_log_probs(*_with(SCORES, n=0, s=None, ids=None, logp=None, top_ids=None, top_logp=None)) == 0


SCORES_GRAD = ("s ld dtype n v ids bytes stats g e entropy out ldo stream".split(), [P, 8, 0, 4, 8, P, 4, P, P, P, P, P2, 8, None])
DISTILL = ("s ld dtype n v ids bytes t t_dtype k T loss stats stream".split(), [P, 8, 0, 4, 8, P, 4, P, 0, 2, 1.0, P, P, None])
DISTILL_GRAD = ("s ld dtype n v ids bytes t t_dtype k T stats g out ldo stream".split(), [P, 8, 0, 4, 8, P, 4, P, 0, 2, 1.0, P, P, P2, 8, None])


@pytest.mark.parametrize("changes", [dict(s=None), dict(ld=7), dict(ids=None), dict(stats=None), dict(stats=P + 4), dict(entropy=None), dict(out=None),
                                     dict(ldo=7), dict(bytes=3), dict(dtype=9), dict(out=P, ldo=9), dict(out=P + 4)])
def test_log_probs_grad_refuses(changes):
    assert gs.lib().gs_log_probs_grad(*_with(SCORES_GRAD, **changes)) == BAD


@pytest.mark.parametrize("changes", [dict(s=None), dict(ld=7), dict(ids=None), dict(bytes=0), dict(t=None), dict(t=P + 2), dict(t_dtype=4), dict(k=0),
                                     dict(T=0.0), dict(T=-1.0), dict(T=float("nan")), dict(T=1e9), dict(stats=None), dict(v=0), dict(n=-1)])
def test_distill_refuses(changes):
    assert gs.lib().gs_distill_loss(*_with(DISTILL, **changes)) == BAD
    assert gs.lib().gs_distill_grad(*_with(DISTILL_GRAD, **changes)) == BAD


def test_distill_limits():
    assert gs.lib().gs_distill_loss(*_with(DISTILL, k=129)) == NOT
    assert gs.lib().gs_distill_loss(*_with(DISTILL, loss=None)) == BAD
    assert gs.lib().gs_distill_grad(*_with(DISTILL_GRAD, g=None)) == BAD
    assert gs.lib().gs_distill_grad(*_with(DISTILL_GRAD, out=None)) == BAD
    assert gs.lib().gs_distill_grad(*_with(DISTILL_GRAD, out=P, ldo=9)) == BAD
    assert gs.lib().gs_distill_grad(*_with(DISTILL_GRAD, out=P - 4)) == BAD
    assert gs.lib().gs_distill_grad(*_with(DISTILL_GRAD, n=0, s=None, out=None, ids=None, t=None, stats=None, g=None)) == 0


def test_python_refuses_cpu_tensors():
    import torch
    x, i = torch.zeros(2, 4), torch.zeros(2, dtype=torch.int64)
    for call in (lambda: gs.rms_norm(x), lambda: gs.rms_norm_grad(x, x[:, 0], x), lambda: gs.grouped_matmul(x, torch.zeros(1, 4, 4), i),
                 lambda: gs.grouped_weight_grad(x, x, i), lambda: gs.log_probs(x, i), lambda: gs.distill_loss(x, i[:, None], x[:, :1])):
        with pytest.raises(ValueError):
            call()


FAR = dict(rows=(1 << 31) - 1, A=1 << 44, W=1 << 40)  # (too many tiles: what is not refused before ends there, nothing is launched)


@pytest.mark.parametrize("changes,size", [
    (dict(step=0), 512), (dict(step=0, groups=1000), 512), (dict(step=0, groups=1), 512),  # one matrix for all
    (dict(step=16, ldw=48), 7 * 192 + 2 * 64 + 64),                                        # matrices side by side
    (dict(step=100), 2 * 400 + 512), (dict(step=128), 3 * 512), (dict(step=200), 2 * 800 + 512)])
def test_results_right_behind_the_matrices_are_taken(changes, size):
    """Only what the groups' matrices take is W's: a result may lie right behind or before them, not 4 bytes inside."""
    L = gs.lib()
    behind, before = FAR["W"] + size, FAR["W"] - 64 * FAR["rows"]
    for C in (behind, behind + 4, behind + 1024, before):
        assert L.gs_grouped_matmul(*_with(GROUPED, **FAR, **changes, C=C)) == NOT, L.gs_last_error()
        assert b"too many tiles" in L.gs_last_error()
    for C in (behind - 4, before + 4, FAR["W"]):
        assert L.gs_grouped_matmul(*_with(GROUPED, **FAR, **changes, C=C)) == BAD and b"overlaps W" in L.gs_last_error()


GROUPED_GRAD_APART = (GROUPED_GRAD[0], [P, 8, P2, 16, 0, 4, 8, 16, 3, P, 4, P3, P4, 0, None])
GRAD_BYTES, ROW_BYTES = 3 * 8 * 16 * 4, 16 * 4  # of the result, of a row of G


@pytest.mark.parametrize("changes", [
    dict(out=P), dict(out=P + 4 * 32 - 4), dict(out=P - GRAD_BYTES + 4), dict(out=P2), dict(out=P2 + 4 * ROW_BYTES - 4), dict(out=P2 - GRAD_BYTES + 4)])
def test_weight_gradients_over_their_operands_are_refused(changes):
    L = gs.lib()
    assert L.gs_grouped_weight_grad(*_with(GROUPED_GRAD_APART, **changes)) == BAD and b"out overlaps" in L.gs_last_error()


def test_workspaces_over_operands_are_refused():
    L, need, rows = gs.lib(), ctypes.c_uint64(), 100_000
    assert L.gs_grouped_weight_grad_workspace(rows, 3, 8, 16, ctypes.byref(need)) == 0 and need.value > 0
    args = dict(rows=rows, A=1 << 40, G=2 << 40, out=3 << 40, work_bytes=need.value)
    for work in (args["A"] + 32, args["A"] - need.value + 4, args["G"], args["G"] + rows * ROW_BYTES - 4, args["out"] + 4, args["out"] - 4):
        assert L.gs_grouped_weight_grad(*_with(GROUPED_GRAD_APART, **args, work=work)) == BAD and b"work overlaps" in L.gs_last_error()
    saved = ctypes.byref(gs._Saved(rows, 8, 0, 1 << 42, 1 << 43))
    for work in (args["G"], args["out"] + 4):
        assert L.gs_grouped_weight_grad_saved(saved, args["G"], 16, 0, 16, 3, P, 4, args["out"], work, need.value, None) == BAD
        assert b"work overlaps" in L.gs_last_error()
    assert L.gs_grouped_weight_grad_saved(saved, args["G"], 16, 0, 16, 3, P, 4, args["G"] + 4, 1 << 44, need.value, None) == BAD
    assert b"out overlaps" in L.gs_last_error()


@pytest.mark.parametrize("codes,scales", [(P, 1 << 40), (P + 112, 1 << 40), (P - 112, 1 << 40), (P2, 1 << 40), (P3, 1 << 40), (1 << 40, P),
                                          (1 << 40, P2 + 124), (1 << 40, P3 + 64)])
def test_norms_saved_over_their_operands_are_refused(codes, scales):
    """X, R and H are read and written while codes and scales of other rows are."""
    L = gs.lib()
    assert L.gs_rms_norm(*_with(NORM, Y=None, saved=_saved(codes=codes, scales=scales))) == BAD
    assert b"saved overlaps" in L.gs_last_error()


@pytest.mark.parametrize("work", [P, P + 124, P2, P3, P4, P4 - 28])
def test_norm_gradients_workspaces_over_operands_are_refused(work):
    L, need = gs.lib(), ctypes.c_uint64()
    assert L.gs_rms_norm_grad_workspace(4, 8, 0, ctypes.byref(need)) == 0 and need.value == 32
    assert L.gs_rms_norm_grad(*_with(NORM_GRAD, work=work, bytes=need.value)) == BAD and b"work overlaps" in L.gs_last_error()


@pytest.mark.parametrize("changes", [
    dict(A=None), dict(lda=7), dict(G=None), dict(ldg=15), dict(dtype=2), dict(rows=-1), dict(a=0), dict(b=0), dict(groups=0), dict(offsets=None),
    dict(bytes=1), dict(out=None), dict(rows=100_000)])
def test_grouped_weight_grad_refuses_for_the_reason(changes):
    """The refusals, of operands that are apart from each other."""
    L = gs.lib()
    assert L.gs_grouped_weight_grad(*_with(GROUPED_GRAD_APART, **changes)) == BAD and b"overlap" not in L.gs_last_error()


@pytest.mark.parametrize("changes", [
    dict(H=None), dict(ldh=7), dict(rstd=None), dict(dY=None), dict(ldy=7), dict(dtype=5), dict(rows=-1), dict(cols=0), dict(w=P + 1), dict(w_dtype=2),
    dict(ldd=7), dict(dX=None), dict(ldx=7), dict(work=None), dict(bytes=3)])
def test_norm_grad_refuses_for_the_reason(changes):
    L = gs.lib()
    assert L.gs_rms_norm_grad(*_with(NORM_GRAD, **dict(dict(work=1 << 40), **changes))) == BAD and b"overlap" not in L.gs_last_error()


@pytest.mark.parametrize("changes", [dict(dX=P), dict(dX=P2), dict(dX=P3 + 4), dict(dX=P3, ldx=9)])
def test_norm_grad_refuses_results_over_operands(changes):
    L = gs.lib()
    assert L.gs_rms_norm_grad(*_with(NORM_GRAD, work=1 << 40, **changes)) == BAD and b"dX overlaps" in L.gs_last_error()


def test_log_probs_refuses_statistics_that_are_not_aligned():
    L = gs.lib()
    assert L.gs_log_probs(*_with(SCORES, stats=P + 4)) == BAD and b"stats are not 8-byte aligned" in L.gs_last_error()


@pytest.mark.filterwarnings("ignore:.*torch.jit.trace.*:DeprecationWarning")
def test_operands_that_are_followed_forwards_or_traced_are_refused():
    """Every operand, not only the dense ones: a tangent would be lost, a trace replay what was in memory."""
    import torch
    from torch.autograd import forward_ad

    from paper_2111_00352_amd import operators
    x, W, off = torch.zeros(4, 3), torch.zeros(2, 3, 5), torch.tensor([0, 2, 4])
    with forward_ad.dual_level():
        for call in (lambda d: operators._array(d, "weight", (6,), operators._F32, -1), lambda d: gs.grouped_matmul(x, d.view(1, 2, 3), off)):
            with pytest.raises(RuntimeError, match="forward-mode"):
                call(forward_ad.make_dual(torch.zeros(6), torch.ones(6)))
        assert operators._array(torch.zeros(6), "weight", (6,), operators._F32, -1) == 0
        assert operators._array(off, "offsets", (3,), operators._INTS, -1) == 8
    with pytest.raises(RuntimeError, match="traced"):
        torch.jit.trace(lambda w: gs.grouped_matmul(x, w, off), W)
    with pytest.raises(RuntimeError, match="traced"):
        torch.jit.trace(lambda w: w * operators._array(w, "weight", (4,), operators._F32, -1), torch.zeros(4))


def test_captures_are_refused_where_an_eager_graph_holds_the_same_leaves(monkeypatch):
    """What the layers know of graphs recorded outside a capture, without a GPU: a function of theirs in name only."""
    import torch

    from paper_2111_00352_amd import layers

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            layers._record(ctx, x)
            return x * w

        @staticmethod
        def backward(ctx, d):
            return d, d

    def layer(x, w):
        layers._may_record(x, w)
        return Layer.apply(x, w)

    capturing = False
    monkeypatch.setattr(layers, "_capturing", lambda t: capturing)
    x, w, other = torch.ones(3), torch.ones(3, requires_grad=True), torch.ones(3, requires_grad=True)
    for eager in (lambda: layer(x, w), lambda: layer(x, w.double()), lambda: layer(layer(x, w * 2) + 1, other), lambda: layer(x, w).sum().exp()):
        kept = eager()
        capturing = True
        for call in (lambda: layer(x, w), lambda: layer(x, w.bfloat16()), lambda: layer(w.tanh(), other), lambda: layer(kept * 2, x)):
            with pytest.raises(RuntimeError, match="holds the same parameter"):
                call()
        with torch.no_grad():  # (records nothing)
            layer(x, w)
            layer(x, w.double())
        layer(x, x), layer(x, torch.ones(3, requires_grad=True))
        capturing = False
        layer(x, w).sum().backward()
        del kept, call
        capturing = True
        inside = layer(x, w)  # (what is recorded inside is no hindrance to the rest of it)
        (layer(inside, w.double()) + layer(x, w)).sum().backward()
        capturing = False
        del inside
    with torch.no_grad():
        y = layer(x, w)
    capturing = True
    layer(x, w)
    assert not y.requires_grad


def test_layers_refuse_cpu_tensors():
    import torch

    from paper_2111_00352_amd import layers
    x, i = torch.zeros(2, 4), torch.zeros(2, dtype=torch.int64)
    w, W = torch.ones(4, requires_grad=True), torch.zeros(1, 4, 4, requires_grad=True)
    for call in (lambda: layers.rms_norm(x), lambda: layers.rms_norm(x, w), lambda: layers.rms_norm([1.0], w), lambda: layers.grouped_linear(x, W, i),
                 lambda: layers.norm_grouped_linear(x, w, W, i), lambda: layers.log_probs(x * w, i), lambda: layers.distill_loss(x * w, i[:, None], x[:, :1])):
        with pytest.raises(ValueError):
            call()
