"""GPU parity of the low-bit operators (8-bit saved activations, MXFP4) against
the fp64 definitions in oracle/lowbit.py.

Codes, scale bytes and the values they stand for must be equal: every step of
the formats is exact in fp32.  Products are exact and summed in fp32, so with
u = 2^-24 a sum of c terms added one after another (an instruction adds its 16
or 64 products as one such term, rounded at most twice) is within 2 c u of its
terms' magnitudes.
"""
import numpy as np
import pytest
import torch

import graphgen
import paper_2111_00352_amd as gs
from oracle import gcn as ogcn
from oracle import lowbit
from paper_2111_00352_amd import gcn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _inside(t, left=1, right=2, above=1):
    """t as a view into a larger tensor full of NaN, at an odd element offset, and the larger one."""
    wide = torch.full((t.shape[0] + 2 * above, t.shape[1] + left + right), float("nan"), dtype=t.dtype, device=DEV)
    view = wide[above:above + t.shape[0], left:left + t.shape[1]]
    view.copy_(t)
    return view, wide


def _around_is_nan(view, wide):
    keep = view.clone()
    view.fill_(float("nan"))
    ok = bool(wide.isnan().all())
    view.copy_(keep)
    return ok


def _np(t):
    return t.detach().cpu().double().numpy()


def _data(n, a, seed, dtype, special=False):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, a)) * np.exp(2 * rng.standard_normal((n, 1)))
    x[rng.random((n, a)) < 0.05] = 0.0
    if n > 3:
        x[1] = -np.abs(x[1])
        x[2] = 0.0
    t = torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype])
    if special and n >= 16:
        t[3, a // 2] = float("nan")
        t[4, a - 1] = float("inf")
        t[5, 0] = -float("inf")
        t[6] *= 2.0 ** -140  # subnormal
        t[7] = torch.sign(t[7]) * 2.0 ** 127
        t[8] = -0.0
        t[9, :] = 1e-30
        t[9, 0] = 3e38  # everything else vanishes under the block's step
        t[10] = 2.0 ** -126
        # halves of a step: ties, and the top of the range
        ramp = torch.arange(a, dtype=torch.float32) % 32
        t[11] = (ramp * 0.25).to(t.dtype)
        t[12] = (127.5 + ramp * 4).to(t.dtype)
        t[13] = (-127.75 + ramp / 32).to(t.dtype)
        t[14] = (ramp + 0.5).to(t.dtype)
    return t


def _same(got, want):
    got = _np(got)
    return got.shape == want.shape and np.array_equal(np.nan_to_num(got, nan=12345.0), np.nan_to_num(want, nan=12345.0))


SHAPES = [(1, 1), (1, 257), (2, 31), (31, 32), (17, 33), (65, 64), (40, 100), (33, 128), (300, 129), (5, 1000)]


@pytest.mark.parametrize("n,a", SHAPES)
@pytest.mark.parametrize("act", ["relu", "none"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_save_activation_is_exact(n, a, act, dtype):
    t = _data(n, a, 11 * n + a, dtype, special=True)
    P, wide = _inside(t.to(DEV))
    q, E, v, h, _ = lowbit.save8(_np(t), act == "relu")
    H, saved = gs.save_activation(P, act)
    assert saved.shape == (n, a) and saved.act == act
    pad = -(-a // 32) * 32
    assert saved.codes.shape == (n, pad) and saved.scales.shape == (n, pad // 32)
    codes = saved.codes.cpu().numpy().astype(np.int64)
    assert np.array_equal(codes[:, :a], q & 255) and not codes[:, a:].any()
    assert np.array_equal(saved.scales.cpu().numpy().astype(np.int64), E)
    assert _same(H, h) and H.dtype == TYPES[dtype]
    for t2 in TYPES.values():
        assert _same(saved.dequantize(t2), v)
    assert _around_is_nan(P, wide)


def test_saved_values_are_within_a_step():
    t = _data(200, 320, 5, "f32")
    for act in ("relu", "none"):
        h, saved = gs.save_activation(t.to(DEV), act)
        top = h.abs().reshape(200, 10, 32).amax(2, keepdim=True).expand(-1, -1, 32).reshape(200, 320)
        step = top * 2.0 ** (-7 if act == "relu" else -6)  # (the step is at most this)
        assert bool(((saved.dequantize() - h).abs() <= step).all())


@pytest.mark.parametrize("n,a", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_relu_grad_selects(n, a, dtype):
    t = _data(n, a, 7 * n + a, "f32", special=True)
    _, saved = gs.save_activation(t.to(DEV))
    on = lowbit.save8(_np(t), True)[4]
    d = torch.from_numpy(np.random.default_rng(n).standard_normal((n, a)).astype(np.float32)).to(TYPES[dtype])
    d[torch.from_numpy(~on)] = float("nan")  # nothing of a masked place comes through
    dH, _ = _inside(d.to(DEV))
    want = np.where(on, _np(d), 0.0)
    assert _same(gs.relu_grad(saved, dH), want)
    out, wide = _inside(torch.zeros(n, a, dtype=TYPES[dtype], device=DEV), left=3, right=1)
    assert gs.relu_grad(saved, dH, out=out) is out
    assert _same(out, want) and _around_is_nan(out, wide)
    gs.relu_grad(saved, dH, out=dH)
    assert _same(dH, want)


@pytest.mark.parametrize("n", [0, 1, 15, 16, 17, 128, 129, 1000, 20_003])
@pytest.mark.parametrize("a,b", [(1, 1), (32, 33), (33, 32), (64, 64), (65, 31), (31, 65), (128, 64), (128, 128),
                                 (255, 47), (129, 5), (300, 200)])
def test_saved_weight_grad(n, a, b):
    # around the tiles (32, 64, 128 columns of A; 32, 64 of G), steps (16 rows a
    # wave, 128 a workgroup) and chunks.  A wave's chain is three terms a step of 16
    # rows, at most ceil(n / 128) steps; then the workgroup's waves and the partials.
    rng = np.random.default_rng(n * 7 + a + b)
    for act, dtype in (("relu", "f32"), ("none", "bf16"), ("none", "f32"), ("relu", "bf16")):
        P = torch.from_numpy(rng.standard_normal((n, a)).astype(np.float32))
        G = torch.from_numpy(rng.standard_normal((n, b)).astype(np.float32)).to(TYPES[dtype])
        _, saved = gs.save_activation(P.to(DEV), act)
        v = lowbit.save8(_np(P), act == "relu")[2]
        g, _ = _inside(G.to(DEV))
        got = _np(gs.saved_weight_grad(saved, g))
        want, mag = v.T @ _np(G), np.abs(v).T @ np.abs(_np(G))
        assert got.shape == (a, b)
        terms = 3 * -(-n // 128) + 16 + 64
        assert np.all(np.abs(got - want) <= 2 * terms * U * mag)


def test_saved_weight_grad_is_deterministic_and_takes_wide_ranges():
    rng = np.random.default_rng(3)
    P = torch.from_numpy((rng.standard_normal((3000, 96)) * np.exp(10 * rng.standard_normal((3000, 1)))).astype(np.float32))
    G = torch.from_numpy((rng.standard_normal((3000, 40)) * np.exp(8 * rng.standard_normal((3000, 1)))).astype(np.float32))
    _, saved = gs.save_activation(P.to(DEV))
    v, g = lowbit.save8(_np(P), True)[2], _np(G)
    first = gs.saved_weight_grad(saved, G.to(DEV))
    assert all(torch.equal(first, gs.saved_weight_grad(saved, G.to(DEV))) for _ in range(3))
    # (below 2^-100 of a gradient's size its lower parts may be subnormal in bf16)
    bound = 2 * (3 * 24 + 80) * U * (np.abs(v).T @ np.abs(g)) + 2.0 ** -100 * np.abs(v).sum(0)[:, None]
    assert np.all(np.abs(_np(first) - v.T @ g) <= bound)


def test_saved_weight_grad_of_subnormal_parts():
    # a gradient from 2^-110 on is the sum of its three bf16 parts; below that its last part
    # loses what lies under bf16's smallest subnormal, 2^-133, which large values bring back
    # into range: column j holds gradients around 2^-(105 + 2 j), values are 2^60 and more
    rng = np.random.default_rng(8)
    n, a, b = 500, 40, 23
    P = torch.from_numpy((rng.uniform(1, 2, (n, a)) * 2.0 ** rng.integers(60, 120, (1, a))).astype(np.float32))
    G = torch.from_numpy((rng.standard_normal((n, b)) * 2.0 ** -(105 + 2 * np.arange(b)))).float()
    _, saved = gs.save_activation(P.to(DEV))
    v, g = lowbit.save8(_np(P), True)[2], _np(G)
    terms = 3 * -(-n // 128) + 16 + 64
    lost = np.where(np.abs(g) < 2.0 ** -110, 2.0 ** -133, 0.0)
    got, mag = _np(gs.saved_weight_grad(saved, G.to(DEV))), v.T @ np.abs(g)
    assert np.all(np.abs(got - v.T @ g) <= 2 * terms * U * mag + v.T @ lost)
    got = _np(gs.saved_weight_grad(saved, G.bfloat16().to(DEV)))  # (one part: nothing is lost)
    g = _np(G.bfloat16())
    assert np.all(np.abs(got - v.T @ g) <= 2 * terms * U * (v.T @ np.abs(g)))


def test_saved_weight_grad_infinities_and_nan():
    # an infinite gradient gives infinity where the value is not 0 and NaN where it
    # is, as the fp32 product does; a NaN block makes its 32 columns NaN; no other
    # output is touched
    P = torch.rand(500, 70) + 0.5
    P[3, 10] = -1.0
    P[100, 40] = float("nan")
    G = torch.randn(500, 40)
    G[3, 7] = float("inf")
    G[200, 39] = -float("inf")
    G[300, 20] = float("nan")
    _, saved = gs.save_activation(P.to(DEV))
    with np.errstate(invalid="ignore"):
        want = (saved.dequantize().cpu().double().T @ G.double()).numpy()
    for g in (G, G.bfloat16()):
        got = _np(gs.saved_weight_grad(saved, g.to(DEV)))
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(np.isposinf(got), np.isposinf(want)) and np.array_equal(np.isneginf(got), np.isneginf(want))
    assert np.isnan(want[32:64]).all() and np.isposinf(want[0, 7]) and np.isnan(want[10, 7]) and np.isneginf(want[0, 39])


@pytest.mark.parametrize("a,b", [(512, 512), (40, 64)])
def test_saved_weight_grad_chains_do_not_grow_with_n(a, b):
    # every product is 1 + 2^-12 (values 1): a chain of a whole sum would lose the
    # 2^-12 once past 2^12.  A wave sums at most 8,192 rows: three terms in 512
    # steps, then 8 waves, 16 slices of partials and their tree.
    n = 500_000 if a > 100 else 3_000_000
    _, saved = gs.save_activation(torch.ones(n, a, device=DEV))
    G = torch.full((n, b), 1 + 2.0 ** -12, device=DEV)
    got = gs.saved_weight_grad(saved, G).double()
    assert float((got / (n * (1 + 2.0 ** -12)) - 1).abs().max()) <= 2 * (3 * 512 + 8 + 24) * U


@pytest.mark.parametrize("n,a", SHAPES + [(256, 40), (257, 96), (700, 70)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("axis", [1, 0])
def test_mxfp4_quantize_is_exact(n, a, dtype, axis):
    t = _data(n, a, 13 * n + a, dtype, special=True)
    X, _ = _inside(t.to(DEV))
    q = gs.mxfp4_quantize(X, axis=axis)
    ref = _np(t) if axis == 1 else _np(t).T
    code, E, v = lowbit.quant4(ref)
    rows, cols = ref.shape
    pad = -(-cols // 64) * 64 if cols <= 64 else -(-cols // 128) * 128
    assert q.shape == (rows, cols) and q.codes.shape == (rows, pad // 2) and q.scales.shape == (rows, pad // 32)
    full = np.zeros((rows, pad), dtype=np.int64)
    full[:, :cols] = code
    assert np.array_equal(q.codes.cpu().numpy().astype(np.int64), full[:, 0::2] | full[:, 1::2] << 4)
    scales = q.scales.cpu().numpy().astype(np.int64)
    assert np.array_equal(scales[:, :E.shape[1]], E) and not scales[:, E.shape[1]:].any()
    for t2 in TYPES.values():
        assert _same(q.dequantize(t2), v)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("step", [-140, -133, -131, -130, -129, -128, -127, -126, -125, 122])
def test_mxfp4_ends_of_the_range(dtype, step):
    # blocks around the smallest scale (2^-127) and near the largest, with every code and
    # every tie between two in them: inputs, scales and values may be subnormal
    ramp = torch.arange(-32, 32, dtype=torch.float64) / 4
    x = torch.stack([ramp * 2.0 ** step, ramp.flip(0) * 2.0 ** (step - 1), ramp * 2.0 ** (step - 2)]).to(TYPES[dtype])
    code, E, v = lowbit.quant4(_np(x))
    for axis, X in ((1, x), (0, x.T.contiguous())):
        q = gs.mxfp4_quantize(X.to(DEV), axis=axis)
        codes = q.codes.cpu().numpy().astype(np.int64)
        assert np.array_equal(codes[:, :32], code[:, 0::2] | code[:, 1::2] << 4)
        assert np.array_equal(q.scales[:, :2].cpu().numpy().astype(np.int64), E)
        for t2 in TYPES.values():
            assert _same(q.dequantize(t2), v)


def _check_product(A, B, mask_on, dtype, got):
    """got against value(A) value(B)^T: k / 64 instructions and, where the sum is
    split, fewer than 64 parts more; one rounding to bf16."""
    a, b = A.dequantize().cpu().double().numpy(), B.dequantize().cpu().double().numpy()
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    if mask_on is not None:
        want, mag = np.where(mask_on, want, 0.0), np.where(mask_on, mag, 0.0)
    bound = 2 * (a.shape[1] / 64 + 64) * U * mag
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
    assert got.dtype == dtype
    assert np.all(np.abs(_np(got) - want) <= bound)


MATMULS = [(1, 1, 1), (1, 64, 4096), (1, 1000, 100), (2, 33, 64), (5, 4096, 256), (16, 128, 1000), (17, 31, 65),
           (32, 257, 2048), (33, 64, 128), (64, 48, 7000), (65, 2, 16), (100, 129, 130), (128, 128, 128), (129, 256, 512),
           (200, 300, 64), (257, 511, 384), (513, 65, 96), (1000, 128, 128), (3000, 47, 257), (20_011, 64, 100),
           (256, 256, 5000), (520, 776, 1024)]
# products in slices of k (few tiles, long k), and of enough tiles for the larger ones:
# ragged, and whole with half a chunk of k at the end
MATMULS += [(150, 300, 4500), (129, 66, 8064), (700, 513, 2100), (4096, 2100, 700), (2816, 3328, 1152)]


@pytest.mark.parametrize("m,n,k", MATMULS)
@pytest.mark.parametrize("how", ["mxfp4", "f32", "bf16"])
def test_mxfp4_matmul(m, n, k, how):
    rng = np.random.default_rng(m * 31 + n * 7 + k)
    A0 = torch.from_numpy((rng.standard_normal((m, k)) * np.exp(rng.standard_normal((m, 1)))).astype(np.float32))
    B0 = torch.from_numpy(rng.standard_normal((n, k)).astype(np.float32))
    A0 = A0.to(TYPES.get(how, torch.float32))
    A, _ = _inside(A0.to(DEV))
    Aq, B = gs.mxfp4_quantize(A), gs.mxfp4_quantize(B0.to(DEV))
    operand = Aq if how == "mxfp4" else A
    _, saved = gs.save_activation(torch.from_numpy(rng.standard_normal((m, n)).astype(np.float32)).to(DEV))
    on = (saved.codes[:, :n] > 0).cpu().numpy()
    for dtype in TYPES.values():
        _check_product(Aq, B, None, dtype, gs.mxfp4_matmul(operand, B, dtype=dtype))
        out, wide = _inside(torch.zeros(m, n, dtype=dtype, device=DEV), left=3, right=2)
        assert gs.mxfp4_matmul(operand, B, mask=saved, dtype=dtype, out=out) is out
        _check_product(Aq, B, on, dtype, out)
        assert _around_is_nan(out, wide)


@pytest.mark.parametrize("m,n,k", [(16, 512, 8192), (300, 130, 256), (1024, 1024, 1024)])
def test_mxfp4_matmul_integers_are_exact(m, n, k):
    # small whole numbers: every partial sum is exact, so any misplaced element,
    # block or scale shows
    rng = np.random.default_rng(k)
    vals = np.array([0, 1, 2, 3, 4, 6, -1, -2, -3, -4, -6], dtype=np.float32)
    a, b = (torch.from_numpy(rng.choice(vals, (r, k)) * 2.0 ** rng.integers(-2, 3, (r, k // 32)).repeat(32, 1)).float()
            for r in (m, n))
    a[:, ::32] = 6.0 * torch.sign(a[:, ::32] + 0.5)  # (a full-size element, or blocks would scale differently)
    A, B = gs.mxfp4_quantize(a.to(DEV)), gs.mxfp4_quantize(b.to(DEV))
    want = A.dequantize().cpu().double() @ B.dequantize().cpu().double().T
    assert torch.equal(gs.mxfp4_matmul(A, B).cpu().double(), want)
    assert torch.equal(gs.mxfp4_matmul(a.to(DEV), B).cpu().double(), want)


# products in slices of k: of 2 chunks of 256 and more, even ones and a last one that is longer,
# with half a chunk at the end or not, of small tiles and (from 128 of them, k > 30,000) of large
# ones; and the shortest k that is made of tiles at all, in one slice of two chunks
SLICES = [(256, 256, 5000), (512, 512, 8192), (512, 512, 8500), (300, 700, 8500), (500, 520, 9100), (1000, 1000, 16000),
          (2047, 4001, 32600), (2048, 4096, 32768), (200, 600, 512), (200, 600, 450), (65, 512, 512)]


@pytest.mark.parametrize("m,n,k", SLICES)
def test_mxfp4_matmul_in_slices_of_k_is_exact(m, n, k):
    # small whole numbers under different scales: products are multiples of 2^-6 and their
    # sums' standard deviation is at most 51 sqrt(k) < 2^14, far below 2^24 of those steps, so
    # every partial sum is exact and a misplaced chunk, slice or run of scales shows
    gen = torch.Generator(device=DEV).manual_seed(m + n + k)
    vals = torch.tensor([0.0, 1, 2, 3, 4, 6, -1, -2, -3, -4, -6], device=DEV)

    def operand(rows):
        x = vals[torch.randint(len(vals), (rows, k), device=DEV, generator=gen)]
        scale = torch.exp2(torch.randint(-2, 3, (rows, -(-k // 32)), device=DEV, generator=gen).float())
        return x * scale.repeat_interleave(32, 1)[:, :k]

    a, B = operand(m), gs.mxfp4_quantize(operand(n))
    A = gs.mxfp4_quantize(a)
    want = (A.dequantize().double() @ B.dequantize().double().t()).float()
    _, saved = gs.save_activation(torch.randn(m, n, device=DEV, generator=gen))
    on = saved.codes[:, :n] > 0
    for operand in (A, a):
        assert torch.equal(gs.mxfp4_matmul(operand, B), want)
        assert torch.equal(gs.mxfp4_matmul(operand, B, mask=saved), torch.where(on, want, 0.0))
        assert torch.equal(gs.mxfp4_matmul(operand, B, dtype=torch.bfloat16), want.bfloat16())


@pytest.mark.parametrize("m", [1, 40, 300])
def test_mxfp4_matmul_nan_blocks_and_masked_nan(m):
    # a block that is not finite makes its row (A) or column (B) of the product NaN,
    # nothing else, and a masked place is 0 all the same
    k, n = 200, 70
    a, b = torch.randn(m, k), torch.randn(n, k)
    a[m - 1, 150] = float("inf")
    b[5, 199] = float("nan")
    B = gs.mxfp4_quantize(b.to(DEV))
    want = torch.zeros(m, n, dtype=torch.bool)
    want[m - 1] = True
    want[:, 5] = True
    _, saved = gs.save_activation(torch.randn(m, n, device=DEV))
    on = (saved.codes[:, :n] > 0).cpu()
    for A in (a.to(DEV), gs.mxfp4_quantize(a.to(DEV))):
        assert torch.equal(gs.mxfp4_matmul(A, B).isnan().cpu(), want)
        got = gs.mxfp4_matmul(A, B, mask=saved).cpu()
        assert torch.equal(got.isnan(), want & on) and bool((got[~on] == 0).all())


@pytest.mark.parametrize("how", ["mxfp4", "f32"])
def test_mxfp4_matmul_of_few_rows_and_very_many_columns(how):
    # more columns than one launch has workgroups for; whole numbers that e2m1 holds, so
    # products and sums are exact
    n = 2 ** 27 + 33
    vals = torch.tensor([0, 1, 2, 3, 4, 6, -1, -2, -3, -4, -6], dtype=torch.bfloat16, device=DEV)
    X = vals[torch.randint(len(vals), (n, 3), device=DEV, dtype=torch.int32)]
    A = torch.tensor([[1.0, 2.0, -3.0], [6.0, 0.0, 4.0]], device=DEV)
    C = gs.mxfp4_matmul(gs.mxfp4_quantize(A) if how == "mxfp4" else A, gs.mxfp4_quantize(X))
    for i in range(2):
        assert torch.equal(C[i], (X[:, 0] * A[i, 0] + X[:, 1] * A[i, 1] + X[:, 2] * A[i, 2]).float())


def test_mxfp4_matmul_extreme_scales():
    # scale bytes at both ends of the range meet in one product
    a = torch.zeros(40, 128)
    a[:, :32], a[:, 32:64], a[:, 64:96] = 2.0 ** 100, 2.0 ** -120, 2.0 ** -149
    b = torch.zeros(20, 128)
    b[:, :32], b[:, 32:64], b[:, 64:96] = 2.0 ** -110, 2.0 ** 118, 2.0 ** 10
    A, B = gs.mxfp4_quantize(a.to(DEV)), gs.mxfp4_quantize(b.to(DEV))
    _check_product(A, B, None, torch.float32, gs.mxfp4_matmul(A, B))


def test_empty_operands():
    for n, a in ((0, 5), (5, 0), (0, 0)):
        H, saved = gs.save_activation(torch.empty(n, a, device=DEV))
        assert H.shape == (n, a) and saved.dequantize().shape == (n, a)
        assert gs.relu_grad(saved, torch.empty(n, a, device=DEV)).shape == (n, a)
        for axis in (0, 1):
            q = gs.mxfp4_quantize(torch.empty(n, a, device=DEV), axis=axis)
            assert q.dequantize().shape == ((n, a) if axis else (a, n))
    B = gs.mxfp4_quantize(torch.empty(7, 0, device=DEV))
    assert torch.equal(gs.mxfp4_matmul(torch.empty(4, 0, device=DEV), B), torch.zeros(4, 7, device=DEV))
    assert gs.mxfp4_matmul(torch.empty(0, 64, device=DEV), gs.mxfp4_quantize(torch.ones(7, 64, device=DEV))).shape == (0, 7)
    assert gs.mxfp4_matmul(torch.ones(4, 64, device=DEV), gs.mxfp4_quantize(torch.empty(0, 64, device=DEV))).shape == (4, 0)


@pytest.mark.parametrize("n,a,b", [(6, 0, 4), (6, 4, 0), (0, 0, 0), (0, 4, 0), (0, 3, 4)])
def test_empty_weight_gradients(n, a, b):
    _, saved = gs.save_activation(torch.ones(n, a, device=DEV))
    got = gs.saved_weight_grad(saved, torch.ones(n, b, device=DEV))
    assert got.dtype == torch.float32 and torch.equal(got, torch.zeros(a, b, device=DEV))


@pytest.mark.parametrize("a", [128, 100, 64])
def test_calls_larger_than_the_caches(a):
    # more than 700 MB of operands, where loads and stores go past the caches: any rows
    # are those of a call with these rows alone
    n, b = 1_800_001 if a == 64 else 1_000_003, 70
    gen = torch.Generator(device=DEV).manual_seed(a)
    P = torch.randn(n, a, device=DEV, generator=gen)
    W = gs.mxfp4_quantize(torch.randn(b, a, device=DEV, generator=gen))
    H, saved = gs.save_activation(P)
    grad, values = gs.relu_grad(saved, P), saved.dequantize()
    q, cols, C = gs.mxfp4_quantize(P), gs.mxfp4_quantize(P, axis=0), gs.mxfp4_matmul(P, W)
    Cq, back = gs.mxfp4_matmul(q, W), q.dequantize()
    for at in (0, 31 * 32, n // 64 * 32, n // 32 * 32 - 256, n - 100):
        rows = slice(at, min(at + 256, n))
        p = P[rows].contiguous()
        h, s = gs.save_activation(p)
        assert torch.equal(H[rows], h) and torch.equal(saved.codes[rows], s.codes) and torch.equal(saved.scales[rows], s.scales)
        assert torch.equal(values[rows], s.dequantize()) and torch.equal(grad[rows], gs.relu_grad(s, p))
        x = gs.mxfp4_quantize(p)
        assert torch.equal(q.codes[rows], x.codes) and torch.equal(q.scales[rows], x.scales)
        assert torch.equal(back[rows], x.dequantize())
        c = gs.mxfp4_matmul(p, W)
        assert torch.equal(C[rows], c) and torch.equal(Cq[rows], c)
        if at % 32 == 0 and len(p) == 256:
            y = gs.mxfp4_quantize(p, axis=0)
            assert torch.equal(cols.codes[:, at // 2:at // 2 + 128], y.codes)
            assert torch.equal(cols.scales[:, at // 32:at // 32 + 8], y.scales)


def test_offsets_past_32_bits():
    # 2^31 elements and more: the last rows are those of the same rows alone
    n, a, tail = 8_400_000, 264, 100
    gen = torch.Generator(device=DEV).manual_seed(5)
    P = torch.empty(n, a, dtype=torch.bfloat16, device=DEV)
    for i in range(0, n, 1_200_000):
        P[i:i + 1_200_000] = torch.randn(min(1_200_000, n - i), a, device=DEV, generator=gen)
    assert (n - tail) * a > 2 ** 31
    H, saved = gs.save_activation(P)
    h, small = gs.save_activation(P[-tail:])
    assert torch.equal(H[-tail:], h) and torch.equal(saved.codes[-tail:], small.codes)
    assert torch.equal(saved.scales[-tail:], small.scales)
    assert torch.equal(saved.dequantize(torch.bfloat16)[-tail:], small.dequantize(torch.bfloat16))
    assert torch.equal(gs.relu_grad(saved, P)[-tail:], gs.relu_grad(small, P[-tail:]))
    del H
    G = torch.zeros(n, 40, dtype=torch.bfloat16, device=DEV)
    G[-tail:] = torch.randn(tail, 40, device=DEV, generator=gen)
    full, part = gs.saved_weight_grad(saved, G), gs.saved_weight_grad(small, G[-tail:])
    mag = small.dequantize().double().T @ G[-tail:].double().abs()
    assert bool(((full - part).abs().double() <= 2 * 100 * U * mag).all())
    del saved, G
    q, qs = gs.mxfp4_quantize(P), gs.mxfp4_quantize(P[-tail:])
    assert torch.equal(q.codes[-tail:], qs.codes) and torch.equal(q.scales[-tail:], qs.scales)
    assert torch.equal(q.dequantize(torch.bfloat16)[-tail:], qs.dequantize(torch.bfloat16))
    W = gs.mxfp4_quantize(torch.randn(270, a, device=DEV, generator=gen))
    want = gs.mxfp4_matmul(qs, W)
    for A in (q, P):
        C = gs.mxfp4_matmul(A, W, dtype=torch.bfloat16)
        assert C.shape[0] * C.shape[1] > 2 ** 31
        assert bool(((C[-tail:].float() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all())
        del C
    del q
    cols = gs.mxfp4_quantize(P, axis=0)
    last = gs.mxfp4_quantize(P[n // 32 * 32 - 96:n // 32 * 32].contiguous(), axis=0)
    assert torch.equal(cols.codes[:, (n // 32 - 3) * 16:n // 32 * 16], last.codes[:, :48])


def test_gradients_against_differences():
    # L(P, W) = |relu(P) W - T|^2 / 2: dW and dP of the fused layer against central
    # differences of L in fp64.  The weight gradient reads relu(P) within one step s
    # (2^-7 of the block's largest), so it may be off by s^T |G|; dP is exact up to
    # fp32 rounding.  L is quadratic along every direction that crosses no kink, so
    # differences are exact up to fp64 rounding.
    rng = np.random.default_rng(9)
    n, a, b = 60, 70, 20
    P0, W0, T0 = rng.standard_normal((n, a)), rng.standard_normal((a, b)) / 8, rng.standard_normal((n, b))
    P0 += np.sign(P0) * 0.01
    P, W = (torch.from_numpy(x.astype(np.float32)).to(DEV).requires_grad_(True) for x in (P0, W0))
    T = torch.from_numpy(T0.astype(np.float32)).to(DEV)
    Z = gcn._ReluLinear.apply(P, W, False)
    (0.5 * ((Z - T) ** 2).sum()).backward()
    p, w, t = _np(P), _np(W), _np(T)

    def loss(p, w):
        return 0.5 * np.sum((np.maximum(p, 0) @ w - t) ** 2)

    G = np.abs(np.maximum(p, 0) @ w - t)
    top = np.repeat(np.stack([np.maximum(p, 0)[:, i:i + 32].max(1) for i in range(0, a, 32)], 1), 32, axis=1)[:, :a]
    slack = (2.0 ** -7 * top).T @ G
    rounding = 1e-4 * (np.abs(np.maximum(p, 0)).T @ G + 1)
    for _ in range(40):
        i, j = rng.integers(a), rng.integers(b)
        d = np.zeros_like(w)
        d[i, j] = 1e-3
        diff = (loss(p, w + d) - loss(p, w - d)) / 2e-3
        assert abs(_np(W.grad)[i, j] - diff) <= slack[i, j] + rounding[i, j]
        i, j = rng.integers(n), rng.integers(a)
        d = np.zeros_like(p)
        d[i, j] = 1e-3
        diff = (loss(p + d, w) - loss(p - d, w)) / 2e-3
        assert abs(_np(P.grad)[i, j] - diff) <= 1e-4 * (G[i] @ np.abs(w[j]) + 1)


def test_relu_linear_in_mxfp4_matches_its_formula():
    rng = np.random.default_rng(10)
    n, a, b = 300, 100, 45
    P, W, G = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DEV) for s in ((n, a), (a, b), (n, b)))
    P.requires_grad_(True)
    W.requires_grad_(True)
    Z = gcn._ReluLinear.apply(P, W, True)
    Z.backward(G)
    p, w, g = _np(P), _np(W), _np(G)
    q8 = lowbit.save8(p, True)
    hv, wt, wr, gv = lowbit.quant4(np.maximum(p, 0))[2], lowbit.quant4(w.T)[2], lowbit.quant4(w)[2], lowbit.quant4(g)[2]
    assert np.all(np.abs(_np(Z) - hv @ wt.T) <= 2 * 70 * U * (np.abs(hv) @ np.abs(wt).T))
    assert np.all(np.abs(_np(P.grad) - np.where(q8[4], gv @ wr.T, 0)) <= 2 * 70 * U * (np.abs(gv) @ np.abs(wr).T))
    assert np.all(np.abs(_np(W.grad) - q8[2].T @ g) <= 2 * 100 * U * (q8[2].T @ np.abs(g)))


def test_linear_in_mxfp4_matches_its_formula():
    rng = np.random.default_rng(12)
    n, a, b = 300, 100, 45
    H, W, G = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DEV) for s in ((n, a), (a, b), (n, b)))
    H.requires_grad_(True)
    W.requires_grad_(True)
    Z = gcn._LinearMx.apply(H, W)
    Z.backward(G)
    h, w, g = _np(H), _np(W), _np(G)
    hv, wt, wr, gv = lowbit.quant4(h)[2], lowbit.quant4(w.T)[2], lowbit.quant4(w)[2], lowbit.quant4(g)[2]
    assert np.all(np.abs(_np(Z) - hv @ wt.T) <= 2 * 70 * U * (np.abs(hv) @ np.abs(wt).T))
    assert np.all(np.abs(_np(H.grad) - gv @ wr.T) <= 2 * 70 * U * (np.abs(gv) @ np.abs(wr).T))
    assert np.all(np.abs(_np(W.grad) - h.T @ g) <= 2 * n * U * (np.abs(h).T @ np.abs(g)))


@pytest.mark.parametrize("k", [2, 3])
def test_gcn_mxfp4_step_stage_by_stage(k):
    # each gradient of one step against its formula in fp64 from the gradient above it, and
    # the same step through GCN2, which runs the same kernels, bit for bit
    g, coo, X, W1, W2, T = _problem(k, 64, 32, 5400 + k)
    ctx = gs.SelectContext("fixed", fixed="csr")
    adj = gcn.Adjacency(*coo, (g.R, g.C), ctx, key=8, symmetric=g.meta["symmetric"])
    model = gcn.GCN2(W1, W2, "mxfp4")
    Z1 = gcn._LinearMx.apply(X, model.W1)
    P1 = gcn.aggregate(Z1, adj)
    Z2 = gcn._ReluLinear.apply(P1, model.W2, True)
    Out = gcn.aggregate(Z2, adj)
    for t in (Z1, P1, Z2, Out):
        t.retain_grad()
    model.loss(Out, T).backward()
    og = ogcn.Graph(g.R, g.C, g.row, g.col, g.val)
    terms = int(np.bincount(g.col, minlength=g.C).max()) + 1  # of a sum of the aggregation

    def near(got, want, mag, terms):
        assert np.all(np.abs(_np(got) - want) <= 2 * terms * U * mag)

    d = (_np(Out) - _np(T)) / g.R
    near(Out.grad, d, np.abs(d) + np.abs(_np(T)) / g.R, 4)  # (the difference, the square, the mean)
    near(Z2.grad, og.agg_t(_np(Out.grad)), og.agg_t(np.abs(_np(Out.grad)), absolute=True), terms)
    dz, p, w = _np(Z2.grad), _np(P1), _np(W2)
    gv, wv = lowbit.quant4(dz)[2], lowbit.quant4(w)[2]
    _, _, hv, _, on = lowbit.save8(p, True)
    near(P1.grad, np.where(on, gv @ wv.T, 0), np.where(on, np.abs(gv) @ np.abs(wv).T, 0), 70)
    near(model.W2.grad, hv.T @ dz, hv.T @ np.abs(dz), 3 * -(-g.R // 128) + 16 + 64)
    near(Z1.grad, og.agg_t(_np(P1.grad)), og.agg_t(np.abs(_np(P1.grad)), absolute=True), terms)
    near(model.W1.grad, _np(X).T @ _np(Z1.grad), np.abs(_np(X)).T @ np.abs(_np(Z1.grad)), g.R)
    again = gcn.GCN2(W1, W2, "mxfp4")
    again.step(X, T, adj, lr=0.0)
    ctx.close()
    assert torch.equal(again.W1.grad, model.W1.grad) and torch.equal(again.W2.grad, model.W2.grad)


@pytest.mark.parametrize("a,b", [(4130, 9), (9, 4130)])
@pytest.mark.parametrize("mx", [False, True])
def test_relu_linear_wider_than_the_weight_gradient_kernel(a, b, mx):
    rng = np.random.default_rng(a)
    n = 300
    P, W, G = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DEV) for s in ((n, a), (a, b), (n, b)))
    P.requires_grad_(True)
    W.requires_grad_(True)
    gcn._ReluLinear.apply(P, W, mx).backward(G)
    v, g = lowbit.save8(_np(P), True)[2], _np(G)
    assert np.all(np.abs(_np(W.grad) - v.T @ g) <= 2 * n * U * (v.T @ np.abs(g)))
    assert P.grad.shape == (n, a)


def _problem(k, H, O, seed):
    g = graphgen.scaled(k)
    F = g.X.shape[1]
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV)  # noqa: E731
    W1 = dev(graphgen.features_x(F, H, seed, "normal") / np.sqrt(F))
    W2 = dev(graphgen.features_x(H, O, seed + 1, "normal") / np.sqrt(H))
    T = dev(graphgen.features_x(g.R, O, seed + 2, "normal"))
    coo = tuple(torch.from_numpy(x).to(DEV) for x in (g.row, g.col, g.val))
    return g, coo, dev(g.X), W1, W2, T


@pytest.mark.parametrize("k", [2, 3])
@pytest.mark.parametrize("mode", ["saved8", "mxfp4"])
def test_gcn_lowbit_training(k, mode):
    # one step's gradients near the fp32 step's (8 bits: a step of 2^-7; 4 bits: half
    # a step of the largest elements' spacing, 1/8 of them, in each factor of three
    # products in a row), losses that fall, and for 8 bits, whose forward pass is that
    # of fp32, losses within those 2^-7 of the fp32 curve
    g, coo, X, W1, W2, T = _problem(k, 64, 32, 4800 + k)
    grads, curves = {}, {}
    for lowbit_mode in (None, mode):
        ctx = gs.SelectContext("model")
        adj = gcn.Adjacency(*coo, (g.R, g.C), ctx, key=3, symmetric=g.meta["symmetric"])
        model = gcn.GCN2(W1, W2, lowbit_mode)
        _, _, P1 = model.step(X, T, adj, lr=0.0)
        assert (P1 is None) == (lowbit_mode is not None)
        grads[lowbit_mode] = (model.W1.grad.clone(), model.W2.grad.clone())
        _, curves[lowbit_mode], _ = gcn.train(adj, X, T, W1, W2, epochs=8, lr=0.05, lowbit=lowbit_mode)
        ctx.close()
    for got, want in zip(grads[mode], grads[None]):
        rel = float((got - want).norm() / want.norm())
        assert rel <= (2.0 ** -7 if mode == "saved8" else 3 * 2 * 2.0 ** -3)
    got, want = np.array(curves[mode]), np.array(curves[None])
    assert got[-1] < got[0]
    if mode == "saved8":
        assert np.all(np.abs(got - want) <= 2.0 ** -7 * want)


@pytest.mark.parametrize("mode", ["saved8", "mxfp4"])
def test_gcn_lowbit_keeps_the_codes_and_nothing_else(mode):
    # between the passes: the output and the hidden layer's codes and scales; after them
    # the output and the gradients, though the output still holds its graph.  An
    # allocation is a multiple of 512 bytes.
    H, O = 64, 32
    g, coo, X, W1, W2, T = _problem(2, H, O, 5200)
    ctx = gs.SelectContext("fixed", fixed="csr")
    adj = gcn.Adjacency(*coo, (g.R, g.C), ctx, key=6, symmetric=g.meta["symmetric"])
    model = gcn.GCN2(W1, W2, mode)
    model.step(X, T, adj, lr=0.0)  # (formats and workspaces are made)
    model.W1.grad = model.W2.grad = None
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    Out, P1 = model.forward(X, adj)
    between = torch.cuda.memory_allocated() - before
    loss = model.loss(Out, T)
    loss.backward()
    del loss
    after = torch.cuda.memory_allocated() - before
    ctx.close()
    out, codes = g.R * O * 4, g.R * H * 33 // 32
    grads = W1.numel() * 4 + W2.numel() * 4
    assert P1 is None
    assert between <= out + codes + 256 + 2 * 511
    assert after <= out + grads + 3 * 511


@pytest.mark.parametrize("k", [2, 3])
def test_gcn_mxfp4_forward_matches_oracle(k):
    # the forward pass with its 4-bit products against the same chain in fp64.  X and
    # the weights have one MXFP4 form; the hidden activations are fp32 sums, so those
    # within their error bound eps of a rounding boundary may go either way: by what
    # the codes at +-eps differ, and by 1/2 of the block's largest where its scale may
    # change (either form is within 1/4 of it, the clamp of 8 to 6 included).
    F_H_O = (64, 32)
    g, coo, X, W1, W2, T = _problem(k, *F_H_O, 5000 + k)
    ctx = gs.SelectContext("model")
    adj = gcn.Adjacency(*coo, (g.R, g.C), ctx, key=4, symmetric=g.meta["symmetric"])
    loss, Out, _ = gcn.GCN2(W1, W2, "mxfp4").step(X, T, adj, lr=0.0)
    ctx.close()
    og = ogcn.Graph(g.R, g.C, g.row, g.col, g.val)

    def v4(t):
        return lowbit.quant4(t)[2]

    def product(a, b):  # (value, magnitude, fp32 error) of a b^T
        mag = np.abs(a) @ np.abs(b).T
        return a @ b.T, mag, 2 * (a.shape[1] / 64 + 64) * U * mag

    z1, mag1, err1 = product(v4(_np(X)), v4(_np(W1).T))
    h = np.maximum(og.agg(z1), 0)
    eps = og.agg(err1, absolute=True) + 1e-5 * og.agg(mag1 + err1, absolute=True) + 1e-6
    q = v4(h)
    amb = np.zeros_like(h)
    for c in range(0, h.shape[1], 32):
        b = slice(c, c + 32)
        s = np.exp2((lowbit.quant4(h[:, b])[1] - 127).astype(np.float64))
        near = [s * lowbit.quant4(np.concatenate([x / s, np.full((len(x), 1), 4.0)], 1))[2][:, :-1]
                for x in (np.minimum(np.maximum(h[:, b] - eps[:, b], 0), 7.9 * s), np.minimum(h[:, b] + eps[:, b], 7.9 * s))]
        amb[:, b] = np.maximum(q[:, b] - near[0], near[1] - q[:, b])
        top = h[:, b].max(1)
        lo, hi = (np.frexp(np.maximum(top + d * eps[:, b].max(1), 1e-300))[1] for d in (-1, 1))
        amb[lo != hi, b] = np.maximum(amb[lo != hi, b], 0.5 * (top + eps[:, b].max(1))[lo != hi, None])
    w2 = v4(_np(W2).T)
    z2, mag2, err2 = product(q, w2)
    err2 = err2 + 2 * amb @ np.abs(w2).T
    want, bound = og.agg(z2), og.agg(err2, absolute=True) + 1e-5 * og.agg(mag2 + err2, absolute=True) + 1e-6
    got = _np(Out)
    assert np.all(np.abs(got - want) <= bound)
    # the bound has to mean something: on average far below the values
    assert bound.mean() <= 0.05 * np.abs(want).mean()
    t = _np(T)
    ref, slack = np.sum((got - t) ** 2) / (2 * g.R), np.sum((np.abs(got) + np.abs(t)) ** 2) / (2 * g.R)
    assert abs(float(loss) - ref) <= (got.size * U + 8 * U) * slack


@pytest.mark.parametrize("mode", ["saved8", "mxfp4"])
def test_gcn_lowbit_graph_replays_match_eager(mode):
    g, coo, X, W1, W2, T = _problem(3, 32, 16, 4900)
    out = {}
    for graph in (False, True):
        ctx = gs.SelectContext("fixed", fixed="csr")
        adj = gcn.Adjacency(*coo, (g.R, g.C), ctx, key=5)
        model, losses, _ = gcn.train(adj, X, T, W1, W2, epochs=6, lr=0.05, graph=graph, lowbit=mode)
        out[graph] = (losses, model.W1.detach().clone(), model.W2.detach().clone())
        ctx.close()
    assert out[True][0] == out[False][0]
    assert torch.equal(out[True][1], out[False][1]) and torch.equal(out[True][2], out[False][2])


@pytest.mark.parametrize("handle", [False, True])
def test_calls_on_another_stream(handle):
    # the results and workspaces belong to the busy stream, and so does the memory of
    # inputs dropped right after the call, until the stream has read it
    P = torch.randn(5000, 96, device=DEV)
    G = torch.randn(5000, 64, device=DEV)
    W = gs.mxfp4_quantize(torch.randn(64, 96, device=DEV))
    _, saved = gs.save_activation(P)
    want = gs.saved_weight_grad(saved, G), gs.mxfp4_matmul(P, W), gs.relu_grad(saved, P)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    s = side.cuda_stream if handle else side
    P2, G2 = P.clone(), G.clone()
    side.wait_stream(torch.cuda.current_stream())
    _, saved2 = gs.save_activation(P2, stream=s)
    got = gs.saved_weight_grad(saved2, G2, stream=s), gs.mxfp4_matmul(P2, W, stream=s), gs.relu_grad(saved2, P2, stream=s)
    del P2, G2, saved2
    taken = [torch.full((1 << k,), float("nan"), device=DEV) for k in range(8, 22) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(bool(t.isnan().all()) for t in taken)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_refusals():
    P = torch.randn(10, 40, device=DEV)
    _, saved = gs.save_activation(P)
    _, plain = gs.save_activation(P, "none")
    q = gs.mxfp4_quantize(P)
    bad = [
        lambda: gs.save_activation(P, "gelu"), lambda: gs.save_activation(P.half()), lambda: gs.save_activation(P.cpu()),
        lambda: gs.save_activation(P[0]), lambda: gs.save_activation(P.t()), lambda: gs.save_activation(P[:, ::2]),
        lambda: gs.save_activation(P[:1].expand(10, 40)), lambda: gs.save_activation(P.to_sparse()),
        lambda: gs.relu_grad(saved, P[:9]), lambda: gs.relu_grad(saved, P, out=torch.empty(10, 41, device=DEV)),
        lambda: gs.relu_grad(saved, P, out=torch.empty(10, 40, device=DEV, dtype=torch.bfloat16)),
        lambda: gs.saved_weight_grad(saved, P[:9]), lambda: gs.saved_weight_grad(saved, P.double()),
        lambda: gs.mxfp4_quantize(P, axis=2), lambda: gs.mxfp4_quantize(P.int()),
        lambda: gs.mxfp4_matmul(P[:, :32], q), lambda: gs.mxfp4_matmul(P, P), lambda: gs.mxfp4_matmul(P, q, dtype=torch.float16),
        lambda: gs.mxfp4_matmul(P, q, mask=saved), lambda: gs.mxfp4_matmul(P, q, out=torch.empty(10, 11, device=DEV)),
        lambda: saved.dequantize(torch.float16), lambda: q.dequantize(torch.float64),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(gs.GnnSpmmError) as e:
        gs.relu_grad(plain, P)
    assert e.value.code == gs.ERR_INVALID_ARG
    with pytest.raises(gs.GnnSpmmError) as e:
        gs.saved_weight_grad(saved, torch.empty(10, 4097, device=DEV))
    assert e.value.code == gs.ERR_UNSUPPORTED
    wide = torch.randn(10, 10, device=DEV)
    _, other = gs.save_activation(wide, "none")
    with pytest.raises(gs.GnnSpmmError):
        gs.mxfp4_matmul(P, q, mask=other)
    with pytest.raises(ValueError):
        gcn.GCN2(torch.randn(3, 3), torch.randn(3, 3), lowbit="int4")


def test_views_with_other_strides():
    P = torch.randn(40, 64, device=DEV)
    want = gs.save_activation(P)[0]
    assert torch.equal(gs.save_activation(torch._neg_view(-P))[0], want)
    col = torch.randn(50, 3, device=DEV)[:, 1:2]  # one column, any strides
    assert torch.equal(gs.save_activation(col)[0], torch.relu(col))
    row = torch.randn(7, 1, device=DEV).t()  # one row whose row stride is below its width
    assert torch.equal(gs.save_activation(row)[0], torch.relu(row))


def test_no_gradient_is_dropped_unseen():
    # the operators have no derivatives: a backward pass that reaches one of their results
    # fails, as do traces, forward-mode derivatives and out= beside a gradient
    P, G = torch.randn(10, 40, device=DEV), torch.randn(10, 8, device=DEV)
    _, saved = gs.save_activation(P)
    W = gs.mxfp4_quantize(torch.randn(8, 40, device=DEV))
    calls = {"save": (lambda x: gs.save_activation(x)[0], P), "mask": (lambda x: gs.relu_grad(saved, x), P),
             "wgrad": (lambda x: gs.saved_weight_grad(saved, x), G), "matmul": (lambda x: gs.mxfp4_matmul(x, W), P)}
    for call, x in calls.values():
        want = call(x)
        assert not want.requires_grad
        p = x.clone().requires_grad_(True)
        got = call(p)
        assert torch.equal(got, want)
        with pytest.raises(RuntimeError, match="no gradient"):
            (got.sum() + p.sum()).backward()
        got = call(p.detach())
        assert torch.equal(got, want) and not got.requires_grad
        with torch.no_grad():
            got = call(p)
        assert torch.equal(got, want) and not got.requires_grad
        with pytest.raises(RuntimeError, match="traced"):
            torch.jit.trace(call, x)
        with torch.autograd.forward_ad.dual_level():
            assert torch.equal(call(x), want)
            with pytest.raises(RuntimeError, match="forward-mode"):
                call(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)))
        with torch.inference_mode():
            assert torch.equal(call(x), want)
    p = P.clone().requires_grad_(True)
    assert gs.save_activation(p, "none")[0] is p  # (the identity passes its gradient on)
    for call in (lambda: gs.relu_grad(saved, p, out=torch.empty_like(P)), lambda: gs.relu_grad(saved, P, out=p),
                 lambda: gs.mxfp4_matmul(p, W, out=torch.empty(10, 8, device=DEV)),
                 lambda: gs.mxfp4_matmul(P, W, out=torch.empty(10, 8, device=DEV, requires_grad=True))):
        with pytest.raises(ValueError):
            call()


def test_outputs_in_place_are_seen_by_autograd():
    # a tensor that a graph keeps is found changed, as by PyTorch's own in-place operations
    P = torch.randn(10, 40, device=DEV)
    _, saved = gs.save_activation(P)
    W = gs.mxfp4_quantize(torch.randn(8, 40, device=DEV))
    for shape, write in (((10, 40), lambda t: gs.relu_grad(saved, t, out=t)), ((10, 8), lambda t: gs.mxfp4_matmul(P, W, out=t)),
                         ((10, 8), lambda t: gs.mxfp4_matmul(gs.mxfp4_quantize(P), W, out=t))):
        w = torch.ones(shape, device=DEV, requires_grad=True)
        t = torch.randn(shape, device=DEV)
        loss = (w * t).sum()
        assert write(t) is t
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    with torch.inference_mode():
        t = torch.randn(10, 40, device=DEV)
        assert gs.relu_grad(saved, t, out=t) is t
