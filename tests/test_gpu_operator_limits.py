"""Sizes behind which one launch, or an offset of 32 bits, is not enough."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1908_11848_amd import binding as B               # noqa: E402

BF16 = torch.bfloat16


def stream():
    return torch.cuda.current_stream().cuda_stream


def test_layer_norm_of_more_rows_than_a_launch_has_wavefronts():
    """2^26 rows of one wavefront each would be 2^32 threads.  Rows do not depend on one another: the same bits as by calls over parts of them."""
    M, C = (1 << 26) + 5, 4
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(M, C, dtype=BF16, device="cuda").normal_(generator=g)
    gamma, beta = torch.randn(C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
    y, stats = torch.full_like(x, float("nan")), torch.full((M, 2), float("nan"), device="cuda")
    part, some = torch.empty_like(x), torch.empty_like(stats)
    L, p = B.lib(), lambda t: t.data_ptr()
    assert L.dsspk_layernorm_fwd(stream(), B.DSSPK_BF16, p(x), C, p(gamma), p(beta), p(y), C, p(stats), M, C, 1e-5) == 0
    size = 10_000_001
    for at in range(0, M, size):
        n = min(size, M - at)
        assert L.dsspk_layernorm_fwd(stream(), B.DSSPK_BF16, p(x[at:]), C, p(gamma), p(beta), p(part[at:]), C, p(some[at:]), n, C, 1e-5) == 0
    torch.cuda.synchronize()
    assert torch.equal(y, part) and torch.equal(stats, some) and torch.isfinite(y).all()


def needs(nbytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < nbytes + (4 << 30):
        pytest.skip("needs %d GB of device memory" % (nbytes >> 30))


def test_weight_gradient_of_no_rows_beyond_32_bits():
    K, N = 1 << 16, (1 << 16) + 3
    L = B.lib()
    nws = L.dsspk_linear_bwd_workspace_bytes(B.DSSPK_BF16, 0, N, K)
    needs(4 * K * N + nws)
    dw, ws, some = torch.full((K, N), float("nan"), device="cuda"), torch.empty(nws, dtype=torch.uint8, device="cuda"), torch.empty(8, device="cuda")
    p = lambda t: t.data_ptr()      # noqa: E731
    assert L.dsspk_linear_bwd(stream(), B.DSSPK_BF16, p(some), K, None, p(some), N, None, 0, None, 0, 0, p(dw), None, 0, N, K, p(ws), nws) == 0
    for part in dw.split(1 << 12):
        assert not part.any()           # a NaN is not zero
    del dw, ws
    torch.cuda.empty_cache()


def test_product_whose_copied_operand_takes_more_than_a_launch():
    """Rows of 1023 bf16 numbers are copied to aligned ones, eight numbers a lane: 2^32 lanes for 2^25 rows.  All rows are alike but for some at either end and in the middle."""
    M, K, N = (1 << 25) + 200, 1023, 8
    L = B.lib()
    nws = L.dsspk_linear_fwd_workspace_bytes(B.DSSPK_BF16, M, N, K)
    needs(2 * M * K + nws + 4 * M * N)
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    w, row = (r(K, N) / 32).to(BF16), r(K).to(BF16)
    x = torch.empty(M, K, dtype=BF16, device="cuda")
    x[:] = row
    places = [slice(0, 300), slice(M // 2, M // 2 + 300), slice(M - 300, M)]
    for at in places:
        x[at] = r(300, K).to(BF16)
    y, ws = torch.full((M, N), float("nan"), dtype=BF16, device="cuda"), torch.empty(nws, dtype=torch.uint8, device="cuda")
    p = lambda t: t.data_ptr()      # noqa: E731
    assert L.dsspk_linear_fwd(stream(), B.DSSPK_BF16, p(x), K, p(w), None, 0, None, 0, p(y), N, None, 0, M, N, K, p(ws), nws) == 0
    torch.cuda.synchronize()
    # a sum of 1023 products in 32 bits and one rounding to 8
    close = lambda got, a: ((got.double() - a.double() @ w.double()).abs() <= (K / 32 + 24) * 2.0 ** -23 * (a.double().abs() @ w.double().abs())       # noqa: E731
                            + 2.0 ** -8 * (a.double() @ w.double()).abs()).all()
    like = torch.ones(M, dtype=torch.bool, device="cuda")
    for at in places:
        like[at] = False
        assert close(y[at], x[at])
    assert close(y[1000:1001], row[None]) and (y[like] == y[1000]).all()
    del x, y, ws
    torch.cuda.empty_cache()


def test_momentum_of_more_entries_than_a_launch_takes():
    """A vector of 2^33 entries and some beside one matrix: 2^32 threads for what is not the matrix.  Without momentum of its own and with equal gradients w' = w - rest (1 + mu) g."""
    n, at = (1 << 33) + 1100, (1 << 33) + 1000
    needs(3 * 4 * n)
    w, m, g = (torch.full((n,), v, device="cuda") for v in (2.0, 0.0, 0.5))
    table, L = B.matrix_table([(at, 4, 5)]), B.lib()
    ws = torch.empty(L.dsspk_orthogonal_workspace_bytes(table, 1), dtype=torch.uint8, device="cuda")
    p = lambda t: t.data_ptr()      # noqa: E731
    assert L.dsspk_orthogonal_apply(stream(), p(w), p(w), p(m), p(m), p(g), n, table, 1, 0.5, 0.25, 0.5, 1, 5, 1e-7, p(ws), ws.numel()) == 0
    torch.cuda.synchronize()
    for part, value in ((w, 2.0 - 0.25 * 0.75), (m, 0.5)):
        for i in range(0, at, 1 << 30):
            assert (part[i:min(i + (1 << 30), at)] == value).all(), i
        assert (part[at + 20:] == value).all()
    assert (m[at:at + 20] == 0.5).all() and (w[at:at + 20] < 2.0).all() and (w[at:at + 20] > 1.0).all()
    del w, m, g
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,cols", [(33, 48), (90, 130), (130, 90)])
def test_update_whose_norm_is_beyond_single_precision(rows, cols):
    """Entries up to 3.3e38 fit fp32, their norm does not.  Bound: that of test_gpu_orthogonal.py, 2^-21 (3.4445^5 - 1) / 2.4445 of the result's norm."""
    from test_gpu_orthogonal import bound, call, orthogonal
    g = torch.Generator(device="cuda").manual_seed(rows)
    grad = (torch.rand(rows * cols, generator=g, device="cuda") * 2 - 1) * 3.3e38
    w = torch.zeros_like(grad)
    got = call(w, w, grad, [(0, rows, cols)], scale=1.0, mu=0.0)[0].double().view(rows, cols)
    want = -orthogonal(grad.view(rows, cols), 5) * max(1, cols / rows) ** 0.5
    assert (got - want).norm() <= bound(5) * want.norm()
