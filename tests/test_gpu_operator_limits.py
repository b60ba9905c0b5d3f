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
