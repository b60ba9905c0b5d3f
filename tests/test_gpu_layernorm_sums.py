"""The weights' gradients of a layer norm over many rows.

Tolerance.  A record holds r = M / 4096 rows (four of them side by side, one after the other) and three additions more, each rounded by about 0.3 2^-24 of a partial sum that grows with the
root of its rows: 0.3 2^-24 sqrt((r + 3) / 2) of the whole sum's size, below 2^-24 for r = 10; xhat has two roundings of its own, 0.6 2^-24.  Joining the records adds nothing that
counts: 2^-23 of the sums' norm."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import test_gpu_layernorm as norm            # noqa: E402


@pytest.mark.parametrize("M,C", [(42115, 48), (40000, 500)])
def test_sums_over_many_rows(M, C):
    x, gamma, beta, dy, _ = norm.inputs(M, C, torch.float32)
    _, mean, invstd = norm.reference(x, gamma, beta, 1e-5)
    stats = torch.stack([mean, invstd], 1).float()
    _, dgamma, dbeta = norm.backward(x, gamma, stats, dy, None)
    _, rg, rb, _, _, _, _ = norm.backward_reference(x, gamma, stats, dy, None)
    for got, ref in ((dgamma, rg), (dbeta, rb)):
        assert (got.double() - ref).norm() <= 2.0 ** -23 * ref.norm(), ((got.double() - ref).norm() / ref.norm()).item()
