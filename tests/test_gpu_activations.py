"""Activations and their slopes in fp32 calls, on their own: a product with a single weight, or a single gradient, of one is the other operand itself.

Tolerances.  A value is a handful of fp32 roundings of numbers no larger than itself (half a unit at most, under a third of one on average): at most 2^-22 of the larger of it and 1, and
2^-24 of the root mean square over normally distributed inputs."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1908_11848_amd import binding as B               # noqa: E402
from test_gpu_linear import act                              # noqa: E402

CURVES = [B.DSSPK_ACT_GELU, B.DSSPK_ACT_GELU_TANH, B.DSSPK_ACT_SILU]
N = 1 << 20


def stream():
    return torch.cuda.current_stream().cuda_stream


def value(which, x):
    L, one, y = B.lib(), torch.ones(1, 1, device="cuda"), torch.empty(1, N, device="cuda")
    ws = torch.empty(L.dsspk_linear_fwd_workspace_bytes(0, 1, N, 1), dtype=torch.uint8, device="cuda")
    assert L.dsspk_linear_fwd(stream(), 0, one.data_ptr(), 1, x.data_ptr(), None, which, None, 0, y.data_ptr(), N, None, 0, 1, N, 1, ws.data_ptr(), ws.numel()) == 0
    return y[0]


def slope(which, x):
    L, rows = B.lib(), 1 << 10
    K = N // rows
    dz, w, dx = torch.ones(rows, 1, device="cuda"), torch.ones(K, 1, device="cuda"), torch.empty(rows, K, device="cuda")
    ws = torch.empty(L.dsspk_linear_bwd_workspace_bytes(0, rows, 1, K), dtype=torch.uint8, device="cuda")
    assert L.dsspk_linear_bwd(stream(), 0, None, 0, w.data_ptr(), dz.data_ptr(), 1, dx.data_ptr(), K, x.data_ptr(), K, which, None, None, rows, 1, K, ws.data_ptr(), ws.numel()) == 0
    return dx.view(-1)


def exact_slope(which, x):
    v = x.double().requires_grad_()
    return torch.autograd.grad(act(which, v).sum(), v)[0]


def close(got, ref):
    e = got.double() - ref
    assert (e.abs() <= 2.0 ** -22 * ref.abs().clamp_min(1)).all(), e.abs().max().item()
    return (e.square().mean() / ref.square().mean()).sqrt().item()


@pytest.mark.parametrize("which", CURVES)
def test_errors_in_single_precision(which):
    g = torch.Generator(device="cuda").manual_seed(which)
    x = torch.randn(N, generator=g, device="cuda")
    assert close(value(which, x), act(which, x.double())) <= 2.0 ** -24
    assert close(slope(which, x), exact_slope(which, x)) <= 2.0 ** -24
    x = torch.linspace(-20, 20, N, device="cuda")
    close(value(which, x), act(which, x.double()))
    close(slope(which, x), exact_slope(which, x))


@pytest.mark.parametrize("which", CURVES)
def test_far_out(which):
    """Nothing is left of the curve: x or 0, 1 or 0; a NaN stays one."""
    x = torch.logspace(math.log10(30), 18, N // 4, device="cuda")
    x = torch.cat([x, -x, torch.full((N // 2,), float("nan"), device="cuda")])
    y, s, n = value(which, x), slope(which, x), N // 4
    assert torch.equal(y[:n], x[:n]) and (y[n:2 * n].abs() <= 1e-10).all()
    assert (s[:n] == 1).all() and (s[n:2 * n].abs() <= 1e-10).all()
    assert torch.isnan(y[2 * n:]).all() and torch.isnan(s[2 * n:]).all()


@pytest.mark.parametrize("which", CURVES)
def test_where_squares_overflow(which):
    """All finite numbers: the slope is 1 or 0 beyond 1e19 too, whose square fp32 does not hold."""
    x = torch.logspace(18, 38, N // 2, device="cuda", dtype=torch.double).float()
    s, y = slope(which, torch.cat([x, -x])), value(which, torch.cat([x, -x]))
    assert (s[:N // 2] == 1).all() and (s[N // 2:].abs() <= 1e-10).all()
    assert torch.equal(y[:N // 2], x) and (y[N // 2:].abs() <= 1e-10).all()
