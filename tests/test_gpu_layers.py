"""The norm, the products by group, the scores and the distillation as they are used: layers
and their gradients, a run of them together, captured graphs, other streams, refusals, and
the GCN trained by distillation."""
import numpy as np
import pytest
import torch

import graphgen
import paper_2111_00352_amd as gs
from oracle import lowbit
from oracle import operators as oracle
from paper_2111_00352_amd import gcn, layers

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda"


def _np(t):
    return t.detach().cpu().double().numpy()


def _near(got, want, rel, what=""):
    """Within rel of the largest magnitude: the bounds of single operators are tested beside them."""
    got = _np(got)
    assert got.shape == want.shape and np.isfinite(got).all(), what
    assert np.abs(got - want).max() <= rel * np.abs(want).max() + 1e-30, (what, np.abs(got - want).max() / np.abs(want).max())


def _inputs(n, a, b, groups, seed):
    g = torch.Generator().manual_seed(seed)
    X, R, w = torch.randn(n, a, generator=g), torch.randn(n, a, generator=g), 1 + 0.2 * torch.randn(a, generator=g)
    W = torch.randn(groups, a, b, generator=g) / a ** 0.5
    cuts = torch.randint(0, n + 1, (groups - 1,), generator=g).sort().values
    off = torch.cat([torch.tensor([0]), cuts, torch.tensor([n])]).int()
    return X.to(DEV), R.to(DEV), w.to(DEV), W.to(DEV), off.to(DEV)


def _reference(X, R, w, W, off, ids, T8):
    """fp64 autograd of norm -> (8 bits) -> products by group -> log probabilities."""
    X, R, w, W = (t.detach().cpu().double().requires_grad_() for t in (X, R, w, W))
    H = X + R
    r = (H.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    Y = H * r * w
    if T8:  # (the values kept in 8 bits; the identity backwards)
        Y = Y + (torch.from_numpy(lowbit.save8(Y.detach().float().numpy(), False)[2]) - Y).detach()
    Z = torch.cat([Y[a:b] @ W[g] for g, (a, b) in enumerate(zip(off[:-1].tolist(), off[1:].tolist()))])
    return X, R, w, W, H, Z


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("n,a,b,groups", [(300, 64, 40, 3), (1500, 96, 130, 9), (17, 33, 7, 2)])
def test_layers_together(n, a, b, groups, eight):
    """A typed layer and its head, forwards and backwards, with a second use of the residual stream."""
    X, R, w, W, off = _inputs(n, a, b, groups, n + a)
    ids = torch.randint(-1, b, (n,), device=DEV)
    rX, rR, rw, rW, rH, rZ = _reference(X, R, w, W, off, ids, eight)
    lp = torch.log_softmax(rZ, 1)
    picked = torch.where(ids.cpu() >= 0, lp.gather(1, ids.cpu().clamp(min=0)[:, None])[:, 0], 0.0)
    want = -picked.mean() + 0.1 * (lp.exp() * lp).sum(1).mean() + 0.01 * rH.square().mean()
    want.backward()
    for t in (X, R, w, W):
        t.requires_grad_()
    if eight:
        Z, H = layers.norm_grouped_linear(X, w, W, off, residual=R)
    else:
        Y, H = layers.rms_norm(X, w, residual=R)
        Z = layers.grouped_linear(Y, W, off)
    logp, entropy = layers.log_probs(Z, ids)
    loss = -logp.mean() - 0.1 * entropy.mean() + 0.01 * H.square().mean()
    loss.backward()
    # (fp32 sums of up to 1,500 terms; an 8-bit code may differ by its last step where fp32 and fp64 fall on
    # two sides of a half: 2^-7 of one of a row's elements, within 2^-8 of the largest result)
    tol = 2.0 ** -8 if eight else 1e-5
    want = float(want.detach())
    assert abs(float(loss) - want) <= tol * abs(want)
    for got, ref, name in ((X, rX, "X"), (R, rR, "R"), (w, rw, "w"), (W, rW, "W")):
        _near(got.grad, ref.grad.numpy(), tol, name)
    assert torch.equal(X.grad, R.grad)


def test_norm_layer_without_residual_and_unused_outputs():
    X, _, w, W, off = _inputs(100, 40, 16, 2, 1)
    X.requires_grad_()
    w.requires_grad_()
    Y, H = layers.rms_norm(X, w)
    (Y.sum() + 2 * H.sum()).backward()
    d, dw, _, _ = oracle.rms_norm_grad(_np(X), oracle.rms_norm(_np(X), 1.0, 1e-6)[1], np.ones((100, 40)), _np(w))
    _near(X.grad, d + 2, 1e-5)
    _near(w.grad, dw, 1e-5)
    X.grad = None
    layers.rms_norm(X, w)[1].sum().backward()  # only H is used
    assert (X.grad == 1).all()
    X.grad = None
    Z, H = layers.norm_grouped_linear(X, w, W, off)
    H.sum().backward()
    assert (X.grad == 1).all() and torch.equal(H, X)


@pytest.mark.parametrize("lowbit_", [None, "saved8"])
@pytest.mark.parametrize("graph", [False, True])
def test_gcn_learns_from_a_teacher(lowbit_, graph):
    """The GCN's training with a Teacher in the target's place: its gradients are the formula's."""
    g = graphgen.scaled(1)
    row, col, val = (torch.from_numpy(x).to(DEV) for x in (g.row, g.col, g.val))
    X = torch.from_numpy(g.X).to(DEV)
    W1 = torch.from_numpy(graphgen.features_x(g.F, 32, 1, "normal")).to(DEV) / g.F ** 0.5
    W2 = torch.from_numpy(graphgen.features_x(32, 24, 2, "normal")).to(DEV) / 32 ** 0.5
    adj = gcn.Adjacency(row, col, val, (g.R, g.C), gs.SelectContext("fixed", fixed="csr"), key=1)
    teacher = gcn.teach(gcn.GCN2(W1, W2), X, adj, top=5, temperature=2.0)
    Out = gcn.GCN2(W1, W2).forward(X, adj)[0]
    assert np.array_equal(_np(teacher.ids), oracle.best(_np(Out), 5))
    student = gcn.GCN2(0.5 * W1, W2, lowbit_)
    So, _ = student.forward(X, adj)
    So.retain_grad()
    loss = student.loss(So, teacher)
    loss.backward()
    want, d, _, _, _ = oracle.distill(_np(So), _np(teacher.ids).astype(int), _np(teacher.logp), 2.0)
    assert abs(float(loss) - want.mean()) <= 1e-5 * want.mean()
    _near(So.grad, d / g.R, 1e-5)
    assert student.W1.grad is not None and torch.isfinite(student.W1.grad).all() and torch.isfinite(student.W2.grad).all()
    _, losses, _ = gcn.train(adj, X, teacher, 0.5 * W1, W2, 5, 0.5, graph=graph, lowbit=lowbit_)
    _, again, _ = gcn.train(adj, X, teacher, 0.5 * W1, W2, 5, 0.5, lowbit=lowbit_)
    assert losses == again and all(np.isfinite(losses))
    adj.ctx.close()


def _all_operators(X, R, w, W, off, s, ids, tid, t, g):
    Y, H, r = gs.rms_norm(X, w, R, save=True)
    Z = gs.grouped_matmul(Y, W, off)
    dY = gs.grouped_matmul(Z, W, off, transpose=True)
    dW = gs.grouped_weight_grad(Y, Z, off)
    dX, dw = gs.rms_norm_grad(H, r, dY, w, H)
    found = gs.log_probs(s, ids, top=7)
    ds = gs.log_probs_grad(s, ids, found, g, g)
    loss, stats = gs.distill_loss(s, tid, t, 1.5)
    dt = gs.distill_grad(s, tid, t, stats, g, 1.5)
    return [Y.dequantize(), H, r, Z, dY, dW, dX, dw, *found, ds, loss, stats, dt]


def _operands(n, a, v, seed):
    X, R, w, W, off = _inputs(n, a, 48, 5, seed)
    s = torch.randn(n, v, device=DEV)
    ids = torch.randint(-1, v, (n,), device=DEV)
    tid = torch.randint(-1, v, (n, 9), device=DEV)
    return X, R, w, W, off, s, ids, tid, torch.randn(n, 9, device=DEV), torch.rand(n, device=DEV)


@pytest.mark.parametrize("n,a,v", [(50, 64, 100), (3000, 200, 5000), (20_000, 64, 47)])
def test_captured_and_replayed(n, a, v):
    """A graph of every operator, replayed on other values with eager work in between, and two graphs at once."""
    ops = _operands(n, a, v, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _all_operators(*ops)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = _all_operators(*ops)
        graphs.append((graph, out))
    for seed in (4, 5, 6):
        fresh = _operands(n, a, v, seed)
        for to, of in zip(ops, fresh):
            to.copy_(of)
        want = [x.clone() for x in _all_operators(*fresh)]
        for graph, out in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for i, (x, y) in enumerate(zip(out, want)):
                assert torch.equal(x, y), i


def test_a_captured_step_and_an_eager_graph_of_the_same_leaves():
    """A capture while an eager graph of the same parameters lives is refused (PyTorch would end the
    process); without one the step is captured, and eager graphs may be made beside it."""
    X, R, w, W, off = _inputs(400, 64, 32, 4, 8)
    ids = torch.randint(0, 32, (400,), device=DEV)
    W.requires_grad_()
    w.requires_grad_()

    def step():
        Z, _ = layers.norm_grouped_linear(X, w, W, off, residual=R)
        return torch.autograd.grad(-layers.log_probs(Z, ids)[0].mean(), (w, W))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = step()
    torch.cuda.current_stream().wait_stream(side)
    eager = layers.norm_grouped_linear(X, w, W, off, residual=R)[0]
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="holds the same parameter"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            step()
    del eager
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        layers.norm_grouped_linear(X, w, W, off, residual=R)[0].sum().backward()
    assert torch.isfinite(W.grad).all()


def test_on_another_stream():
    ops = _operands(2000, 128, 300, 9)
    X, R, w, W, off, s, ids, tid, t, g = ops
    want = _all_operators(*ops)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        torch.cuda._sleep(2_000_000)
    Y, H, r = gs.rms_norm(X, w, R, save=True, stream=st)
    Z = gs.grouped_matmul(Y, W, off, stream=st)
    dY = gs.grouped_matmul(Z, W, off, transpose=True, stream=st)
    dW = gs.grouped_weight_grad(Y, Z, off, stream=st)
    dX, dw = gs.rms_norm_grad(H, r, dY, w, H, stream=st)
    found = gs.log_probs(s, ids, top=7, stream=st)
    ds = gs.log_probs_grad(s, ids, found, g, g, stream=st)
    loss, stats = gs.distill_loss(s, tid, t, 1.5, stream=st)
    dt = gs.distill_grad(s, tid, t, stats, g, 1.5, stream=st)
    V = Y.dequantize(stream=st)
    torch.cuda.current_stream().wait_stream(st)
    got = [V, H, r, Z, dY, dW, dX, dw, *found, ds, loss, stats, dt]
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), i


def test_two_threads_at_once():
    import threading
    ops = [_operands(1500, 96, 700, 20 + i) for i in range(2)]
    want = [_all_operators(*o) for o in ops]
    got = [None, None]

    def run(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(5):
                got[i] = _all_operators(*ops[i])
            torch.cuda.current_stream().synchronize()

    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_refusals():
    X, R, w, W, off, s, ids, tid, t, g = _operands(20, 64, 30, 11)
    found = gs.log_probs(s, ids)
    stats = gs.distill_loss(s, tid, t)[1]
    r = torch.ones(20, device=DEV)
    S = gs.save_activation(X, "none")[1]
    for call in (
        lambda: gs.rms_norm(X.half()), lambda: gs.rms_norm(X[0]), lambda: gs.rms_norm(X.t()), lambda: gs.rms_norm(X, w[:5]), lambda: gs.rms_norm(X, w.half()),
        lambda: gs.rms_norm(X, w, R[:5]), lambda: gs.rms_norm(X, w, R.bfloat16()), lambda: gs.rms_norm(X, w.cpu()), lambda: gs.rms_norm(X, w[::2]),
        lambda: gs.rms_norm_grad(X, r[:3], X, w), lambda: gs.rms_norm_grad(X, r, X[:3], w), lambda: gs.rms_norm_grad(X, r, X.bfloat16(), w),
        lambda: gs.rms_norm_grad(X, r, X, w, R[:, :3]),
        lambda: gs.grouped_matmul(X, W[0], off), lambda: gs.grouped_matmul(X, W.bfloat16(), off), lambda: gs.grouped_matmul(X, W, off[:3]),
        lambda: gs.grouped_matmul(X, W, off.float()), lambda: gs.grouped_matmul(X, W, off, transpose=True), lambda: gs.grouped_matmul(X, W, off.cpu()),
        lambda: gs.grouped_matmul(X, W.transpose(1, 2), off, transpose=True), lambda: gs.grouped_matmul(X, W, off, dtype=torch.half),
        lambda: gs.grouped_matmul(X, W, off, out=torch.empty(20, 5, device=DEV)), lambda: gs.grouped_matmul(S, W[:, :9], off),
        lambda: gs.grouped_weight_grad(X, R[:5], off), lambda: gs.grouped_weight_grad(X, R.bfloat16(), off), lambda: gs.grouped_weight_grad(S, R, off[:1]),
        lambda: gs.log_probs(s, ids[:4]), lambda: gs.log_probs(s, ids.float()), lambda: gs.log_probs(s, ids, top=31), lambda: gs.log_probs(s, ids, top=-1),
        lambda: gs.log_probs(torch.zeros(2, 200, device=DEV), ids[:2], top=129),
        lambda: gs.log_probs_grad(s, ids, found, g[:3]), lambda: gs.log_probs_grad(s[:3], ids, found, g), lambda: gs.log_probs_grad(s, ids, found, g.double()),
        lambda: gs.distill_loss(s, tid[:, :0], t[:, :0]), lambda: gs.distill_loss(s, tid, t[:, :3]), lambda: gs.distill_loss(s, tid.t(), t),
        lambda: gs.distill_loss(s, torch.zeros(20, 129, dtype=torch.int32, device=DEV), torch.zeros(20, 129, device=DEV)),
        lambda: gs.distill_grad(s, tid, t, g, g), lambda: gs.distill_grad(s, tid, t, found.stats, g), lambda: gs.distill_grad(s, tid, t, stats, g[:2]),
        lambda: gs.distill_grad(s, tid, t, stats, g, out=s[:, :5]),
    ):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: gs.rms_norm(torch.zeros(3, 0, device=DEV)), lambda: gs.rms_norm(X, eps=-1.0), lambda: gs.distill_loss(s, tid, t, 0.0),
                 lambda: gs.log_probs(torch.zeros(3, 0, device=DEV), ids[:3])):
        with pytest.raises(gs.GnnSpmmError):
            call()


def test_no_gradient_is_dropped_unseen():
    X, R, w, W, off, s, ids, tid, t, g = _operands(20, 64, 30, 12)
    found = gs.log_probs(s, ids)
    stats = gs.distill_loss(s, tid, t)[1]
    r = torch.ones(20, device=DEV)
    need = lambda x: x.detach().requires_grad_()  # noqa: E731
    for call in (lambda: gs.rms_norm(need(X))[0], lambda: gs.rms_norm(X, need(w))[2], lambda: gs.rms_norm(X, w, need(R))[1],
                 lambda: gs.rms_norm_grad(X, r, need(R))[0], lambda: gs.grouped_matmul(need(X), W, off), lambda: gs.grouped_matmul(X, need(W), off),
                 lambda: gs.grouped_weight_grad(X, need(R), off), lambda: gs.log_probs(need(s), ids).entropy, lambda: gs.log_probs(need(s), ids).logp,
                 lambda: gs.log_probs_grad(need(s), ids, found, g), lambda: gs.distill_loss(need(s), tid, t)[0], lambda: gs.distill_loss(s, tid, need(t))[0],
                 lambda: gs.distill_grad(s, tid, t, stats, need(g))):
        with pytest.raises(RuntimeError, match="no gradient"):
            call().sum().backward()
        with torch.no_grad():
            assert not call().requires_grad
    with pytest.raises(ValueError):
        gs.log_probs_grad(need(s), ids, found, g, out=torch.empty_like(s))
    with pytest.raises(ValueError):
        layers.distill_loss(s, tid, need(t))
    with pytest.raises(RuntimeError, match="traced"):
        torch.jit.trace(lambda x: gs.rms_norm(x)[0], X)
    with pytest.raises(RuntimeError, match="twice"):
        Y = layers.rms_norm(need(X), w)[0]
        torch.autograd.grad(Y.sum(), Y.grad_fn.next_functions[0][0].variable, create_graph=True)
    # a change in place is seen by a graph that keeps the tensor
    logits = s.clone()
    Z = need(logits) * 1.0
    lp, _ = layers.log_probs(Z, ids)
    with torch.no_grad():
        gs.log_probs_grad(Z, ids, found, g, out=Z)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        lp.sum().backward()


def test_negated_views():
    X, R, w, W, off, s, ids, tid, t, g = _operands(20, 64, 30, 13)
    neg = lambda x: torch._neg_view(x)  # noqa: E731
    assert torch.equal(gs.rms_norm(neg(X), w, neg(R))[0], gs.rms_norm(-X, w, -R)[0])
    Y, H, _ = gs.rms_norm(neg(X), w)
    assert torch.equal(H, -X)
    assert torch.equal(gs.grouped_matmul(neg(X), neg(W), off), gs.grouped_matmul(X, W, off))
    assert torch.equal(gs.log_probs(neg(s), ids).logp, gs.log_probs(-s, ids).logp)
    with pytest.raises(ValueError):
        gs.rms_norm(X, neg(w))


def test_offsets_in_a_tensor_past_32_bits():
    """Rows of a logits matrix whose elements are past 2^31 from its start."""
    n, v = 70_000, 33_000
    s = torch.empty(n, v, dtype=torch.bfloat16, device=DEV)
    s[-40:] = torch.randn(40, v, device=DEV)
    ids = torch.randint(0, v, (n,), device=DEV)
    small = gs.log_probs(s[-40:].clone(), ids[-40:], top=5)
    big = gs.log_probs(s, ids, top=5)
    # (how a row is summed depends on the number of rows; logits of at most 6, so |x| <= 12, log S <= 11, and either
    # result is within U (4 |x| + 4 log S + 2 E|x| + v / 256 + 100) <= 320 U of the formula, the sums within as much)
    for a, b in zip(big[:2] + big[4:], small[:2] + small[4:]):
        assert (a[-40:] - b).abs().max() <= 2 * 2 * 320 * U
    assert torch.equal(big.top_ids[-40:], small.top_ids) and torch.equal(big.stats[-40:, 0], small.stats[:, 0])
    assert ((big.stats[-40:, 1] / small.stats[:, 1]) - 1).abs().max() <= 2 * 320 * U
    g = torch.ones(n, device=DEV)
    d = gs.log_probs_grad(s, ids, big, g, out=s)
    assert torch.isfinite(d[-40:].float()).all() and float(d[-40:].float().sum().abs()) < 40
    del s, d
    X = torch.zeros(n, v, dtype=torch.bfloat16, device=DEV)
    X[-1] = 3.0
    Y, _, r = gs.rms_norm(X)
    assert (Y[-1] == 1).all() and (Y[-2] == 0).all()


def test_results_are_changed_in_place_and_kept_alone():
    """A loss is masked or turned in place, as any other; what is kept of a call's results holds no others' memory."""
    X, R, w, W, off, s, ids, tid, t, g = _operands(300, 64, 90, 14)
    mask = (torch.rand(300, device=DEV) < 0.5).float()
    for make in (lambda x: layers.distill_loss(x, tid, t, 1.5), lambda x: layers.log_probs(x, ids)[0]):
        grads = []
        for change in (lambda y: y * mask, lambda y: y.mul_(mask), lambda y: y.neg_().neg_() * mask):
            x = s.detach().requires_grad_()
            change(make(x)).sum().backward()
            grads.append(x.grad)
        assert torch.equal(grads[0], grads[1]) and torch.equal(grads[0], grads[2]) and (grads[0] != 0).any()
    x = s.detach().requires_grad_()
    _, entropy = layers.log_probs(x, ids)
    entropy.mul_(2.0)  # (the gradient reads it)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        entropy.sum().backward()
    found = gs.log_probs(s, ids, top=3)
    for result in (*found, *gs.distill_loss(s, tid, t)):
        assert not result._is_view() and result.untyped_storage().nbytes() == result.numel() * 4


def test_no_tangent_is_dropped_unseen():
    """A dual number in the place of any operand that has values is refused, and a trace beside 8-bit rows."""
    from torch.autograd import forward_ad
    X, R, w, W, off, s, ids, tid, t, g = _operands(20, 64, 30, 15)
    S = gs.save_activation(X, "none")[1]
    found, (_, stats) = gs.log_probs(s, ids), gs.distill_loss(s, tid, t)
    r = gs.rms_norm(X, w)[2]
    with forward_ad.dual_level():
        dual = lambda x: forward_ad.make_dual(x, torch.ones_like(x))  # noqa: E731
        for call in (lambda: gs.rms_norm(X, dual(w)), lambda: gs.rms_norm(X, w, dual(R)), lambda: gs.rms_norm_grad(X, r, R, dual(w)),
                     lambda: gs.rms_norm_grad(X, dual(r), R, w), lambda: gs.grouped_matmul(X, dual(W), off), lambda: gs.grouped_matmul(S, dual(W), off),
                     lambda: gs.log_probs_grad(s, ids, found, dual(g)), lambda: gs.log_probs_grad(s, ids, found, g, dual(g)),
                     lambda: gs.distill_loss(s, tid, dual(t)), lambda: gs.distill_grad(s, tid, dual(t), stats, g),
                     lambda: gs.distill_grad(s, tid, t, stats, dual(g)), lambda: gs.grouped_weight_grad(S, dual(R), off)):
            with pytest.raises(RuntimeError, match="forward-mode"):
                call()
        assert torch.equal(gs.grouped_matmul(S, W, off), gs.grouped_matmul(S, W, off))
    with pytest.raises(RuntimeError, match="traced"):
        torch.jit.trace(lambda x: gs.grouped_matmul(S, x, off), W)


def test_captures_beside_an_eager_graph_of_weights_of_another_type():
    """The parameters are reached through a conversion: a captured step is refused all the same, a captured forward
    pass without gradients is taken."""
    X, R, w, W, off = _inputs(400, 64, 32, 4, 16)
    ids = torch.randint(0, 32, (400,), device=DEV)
    W.requires_grad_()
    X = X.bfloat16()

    def step():
        Z = layers.grouped_linear(X, W.bfloat16(), off)
        return torch.autograd.grad(-layers.log_probs(Z, ids)[0].mean(), W)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = step()
    torch.cuda.current_stream().wait_stream(side)
    eager = layers.grouped_linear(X, W.bfloat16(), off)
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="holds the same parameter"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            step()
    with pytest.raises(RuntimeError, match="holds the same parameter"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            layers.log_probs(eager * 2, ids)
    answer = torch.cuda.CUDAGraph()
    with torch.no_grad(), torch.cuda.graph(answer):
        Z = layers.grouped_linear(X, W.bfloat16(), off)
    for _ in range(3):
        Z.zero_()
        answer.replay()
        torch.cuda.synchronize()
        assert torch.equal(Z, eager)
    del eager
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        layers.grouped_linear(X, W.bfloat16(), off).sum().backward()
