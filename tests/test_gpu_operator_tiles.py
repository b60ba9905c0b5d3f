"""The kernels that large sizes go through, with sizes that leave something over in every direction: every tile of the products, in one and in several parts and in all three orders of
operands; results that are written past the caches; updates of matrices by square tiles.

Tolerances are those of test_gpu_linear.py, test_gpu_layernorm.py and test_gpu_orthogonal.py, where they are derived."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1908_11848_amd import binding as B               # noqa: E402
import test_gpu_layernorm as norm                           # noqa: E402
import test_gpu_linear as linear                            # noqa: E402
import test_gpu_orthogonal as update                        # noqa: E402
from test_gpu_linear import BF16, F32                       # noqa: E402

# type, rows and columns of the result, the sum's length, tile: rows are y's, columns are y's, ... of each of the three products in turn.
# Aligned rows (bf16 operands as they are) and odd ones (copied), few and many parts, fp32's two larger tiles.
FORMS = [(BF16, 4090, 4070, 75, (256, 256, 1)), (BF16, 4088, 4072, 72, (256, 256, 1)), (BF16, 1030, 4090, 5003, (256, 256, 3)), (BF16, 1032, 4088, 5000, (256, 256, 3)),
         (BF16, 515, 261, 7001, (128, 128, 16)), (F32, 2050, 2060, 70, (128, 128, 1)), (F32, 1030, 1030, 1001, (128, 128, 3)), (F32, 2050, 515, 300, (128, 64, 1)),
         (F32, 1030, 195, 2003, (128, 64, 7))]
NAMES = ["%s-%dx%dx%d" % ("bf16" if f[0] == BF16 else "f32", *f[1:4]) for f in FORMS]


def slope(which, x):
    v = x.double().requires_grad_()
    return torch.autograd.grad(linear.act(which, v).sum(), v)[0]


@pytest.mark.parametrize("form", FORMS, ids=NAMES)
def test_forward(form):
    dtype, M, N, K, tile = form
    assert B.linear_form(linear.TYPE[dtype], M, N, K) == tile
    x, w, bias, res, _ = linear.inputs(M, N, K, dtype)
    which = B.DSSPK_ACT_GELU if dtype == BF16 else B.DSSPK_ACT_SILU
    y, z = linear.forward(x, w, bias, which, res)
    rz, size = x.double() @ w.double() + bias.double(), x.double().abs() @ w.double().abs() + bias.double().abs()
    assert ((z.double() - rz).abs() <= linear.sums(K, size) + linear.rounding(dtype, rz)).all()
    ry = linear.act(which, rz) + res.double()
    assert ((y.double() - ry).abs() <= 1.2 * linear.sums(K, size) + 2.0 ** -19 * (rz.abs() + 1) + linear.rounding(dtype, ry) + 2.0 ** -23 * res.abs()).all()
    for gap, shift in ((8, 0), (3, 5)):
        again = linear.forward(x, w, bias, which, res, gap=gap, shift=shift)
        assert torch.equal(again[0], y) and torch.equal(again[1], z)
    # over the residual, without z
    L, r, t = B.lib(), res.clone(), linear.TYPE[dtype]
    ws = linear.space(L.dsspk_linear_fwd_workspace_bytes(t, M, N, K))
    p = linear.ptr
    assert L.dsspk_linear_fwd(linear.stream(), t, p(x), K, p(w), p(bias), which, p(r), N, p(r), N, None, 0, M, N, K, p(ws), ws.numel()) == 0
    assert torch.equal(r, y)


@pytest.mark.parametrize("form", FORMS, ids=NAMES)
def test_gradient_of_the_input(form):
    dtype, M, K, N, tile = form
    assert B.linear_form(linear.TYPE[dtype], M, K, N) == tile
    x, w, _, dz, pre = linear.inputs(M, N, K, dtype, 1)
    which, want = B.DSSPK_ACT_GELU if dtype == BF16 else B.DSSPK_ACT_GELU_TANH, (True, False, False)
    dx, = linear.backward(x, w, dz, pre, which, want=want)
    D, W, s = dz.double(), w.double(), slope(which, pre)
    plain = D @ W.t()
    ref, size = plain * s, (D.abs() @ W.abs().t()) * s.abs()
    assert ((dx.double() - ref).abs() <= linear.sums(N, size) + 2.0 ** -19 * plain.abs() + linear.rounding(dtype, ref)).all()
    for gap, shift in ((8, 0), (3, 5)):
        assert torch.equal(linear.backward(x, w, dz, pre, which, gap=gap, shift=shift, want=want)[0], dx)


@pytest.mark.parametrize("form", FORMS, ids=NAMES)
def test_gradient_of_the_weights(form):
    dtype, K, N, M, tile = form
    assert B.linear_form(linear.TYPE[dtype], K, N, M) == tile
    x, w, _, dz, _ = linear.inputs(M, N, K, dtype, 2)
    want = (False, True, True)
    dw, db = linear.backward(x, w, dz, None, B.DSSPK_ACT_NONE, want=want)
    X, D = x.double(), dz.double()
    assert ((dw.double() - X.t() @ D).abs() <= linear.sums(M, X.abs().t() @ D.abs()) + 1e-37).all()
    assert ((db.double() - D.sum(0)).abs() <= (M / 32 + 24) * 2.0 ** -23 * D.abs().sum(0) + 1e-37).all()
    for gap, shift in ((8, 0), (3, 5)):
        again = linear.backward(x, w, dz, None, B.DSSPK_ACT_NONE, gap=gap, shift=shift, want=want)
        assert torch.equal(again[0], dw) and torch.equal(again[1], db)


@pytest.mark.parametrize("form", [f for f in FORMS if f[0] == F32], ids=[n for n in NAMES if n[0] == "f"])
@pytest.mark.parametrize("scale_a,scale_b", [(1e30, 1e-30), (1e33, 1e3), (1e20, 1e16)])
def test_all_of_single_precisions_range(form, scale_a, scale_b):
    """Sums that leave the range of the scaled bf16 terms and are computed again, in each order of operands."""
    _, R, C, S, _ = form
    g = torch.Generator(device="cuda").manual_seed(R)
    a, b = (torch.randn(*s, generator=g, device="cuda") for s in ((R, S), (S, C)))
    a, b = a * scale_a, b / S ** 0.5 * scale_b
    ref, size = a.double() @ b.double(), a.double().abs() @ b.double().abs()
    bound = linear.sums(S, size) + 2.0 ** -149 * S
    y, _ = linear.forward(a, b, None, 0, None, saves=False)
    dx, = linear.backward(torch.zeros(R, C, device="cuda"), b.t().contiguous(), a, None, 0, want=(True, False, False))
    dw, = linear.backward(a.t().contiguous(), torch.zeros(R, C, device="cuda"), b, None, 0, want=(False, True, False))
    for got in (y, dx, dw):
        assert ((got.double() - ref).abs() <= bound).all()


@pytest.mark.parametrize("form", [FORMS[0], FORMS[2], FORMS[5], FORMS[7]], ids=[NAMES[i] for i in (0, 2, 5, 7)])
def test_infinities_and_nan_stay_where_the_formula_puts_them(form):
    dtype, M, N, K, _ = form
    x, w, bias, res, _ = linear.inputs(M, N, K, dtype)
    x[3, 5], x[M - 1, K - 1], w[7, N - 2] = float("inf"), float("nan"), float("-inf")
    x[:M - 1, 7] = x[:M - 1, 7].abs() + 1           # a definite sign in front of the infinite weight
    w[5] = w[5].abs() + 1
    y, z = linear.forward(x, w, bias, 0, res)
    rows, cols = torch.arange(M, device="cuda")[:, None], torch.arange(N, device="cuda")[None]
    nan = (rows == M - 1) | ((rows == 3) & (cols == N - 2))
    inf, low = (rows == 3) & ~nan, (cols == N - 2) & ~nan
    assert torch.equal(torch.isnan(z), nan) and (z[inf] == float("inf")).all() and (z[low] == float("-inf")).all()
    assert torch.equal(torch.isnan(y), nan) and torch.isfinite(z[~nan & ~inf & ~low]).all()


# ---------------------------------------------------------------- results written past the caches: 128 MB and more

@pytest.mark.parametrize("dtype,M,N,K", [(BF16, 16400, 4099, 70), (F32, 8210, 4099, 37)])
def test_products_beyond_the_caches(dtype, M, N, K):
    assert M * N * x_bytes(dtype) >= 128 << 20
    x, w, bias, res, _ = linear.inputs(M, N, K, dtype)
    y, z = linear.forward(x, w, bias, B.DSSPK_ACT_RELU, res, gap=3, shift=5)
    rz, size = x.double() @ w.double() + bias.double(), x.double().abs() @ w.double().abs() + bias.double().abs()
    assert ((z.double() - rz).abs() <= linear.sums(K, size) + linear.rounding(dtype, rz)).all()
    ry = rz.clamp_min(0) + res.double()
    assert ((y.double() - ry).abs() <= linear.sums(K, size) + linear.rounding(dtype, ry) + 2.0 ** -23 * (rz.abs() + res.abs())).all()
    del x, w, y, z, rz, size, ry
    x, w, _, dz, pre = linear.inputs(M, K, N, dtype)        # the gradient of N inputs
    dx, = linear.backward(x, w, dz, pre, B.DSSPK_ACT_RELU, gap=3, shift=5, want=(True, False, False))
    ref, size = (dz.double() @ w.double().t()) * (pre > 0), dz.double().abs() @ w.double().abs().t()
    assert ((dx.double() - ref).abs() <= linear.sums(K, size) + linear.rounding(dtype, ref)).all()


def x_bytes(dtype):
    return torch.empty(0, dtype=dtype).element_size()


@pytest.mark.parametrize("dtype,M,C", [(BF16, 32800, 2051), (F32, 16400, 2051), (F32, 70000, 500)])
def test_layer_norms_beyond_the_caches(dtype, M, C):
    assert M * C * x_bytes(dtype) >= 128 << 20
    x, gamma, beta, dy, add = norm.inputs(M, C, dtype)
    y, stats = norm.forward(x, gamma, beta, 1e-5, C + 3, 5)
    ref, _, invstd = norm.reference(x, gamma, beta, 1e-5)
    size = x.double().abs().mean(1) * invstd
    assert ((y.double() - ref).abs() <= norm.U * (1 + size)[:, None] * gamma.double().abs() * (1 + (ref - beta).abs()) + norm.rounding(dtype, ref) + 2 ** -23 * beta.abs()).all()
    dx, dgamma, dbeta = norm.backward(x, gamma, stats, dy, add, C + 3, 5)
    rdx, rg, rb, ag, ab, q, xhat = norm.backward_reference(x, gamma, stats, dy, add)
    size = stats[:, 1:].double() * (q.abs() + q.abs().mean(1, keepdim=True) + xhat.abs() * (q * xhat).abs().mean(1, keepdim=True))
    assert ((dx.double() - rdx).abs() <= norm.U * (size + rdx.abs()) + norm.rounding(dtype, rdx)).all()
    assert ((dgamma - rg).abs() <= norm.U * ag + 1e-30).all() and ((dbeta - rb).abs() <= norm.U * ab + 1e-30).all()


# ---------------------------------------------------------------- updates

# More than 128 tiles of 128 x 128, so that halves of them would take a second round: 144 and 138 of one matrix, 420 of two, which is two rounds either way.  Reductions of 22 to 60 steps
@pytest.mark.parametrize("shapes", [[(1500, 1510)], [(1510, 1500)], [(700, 2900)], [(1700, 1900), (1900, 1700)]], ids=str)
def test_updates_by_square_tiles(shapes):
    mats, n = update.layout(shapes, 5, 3)
    w, m, g = update.vectors(n)
    got = update.call(w, m, g, mats)
    update.check(w, m, g, mats, got)
    inplace = update.call(w, m, g, mats, inplace=True)
    assert torch.equal(inplace[0], got[0]) and torch.equal(inplace[1], got[1])
