"""Pushes under the orthogonalised rule that are refused: nothing of them reaches the server, and later pushes on other streams are as if they had not been."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1908_11848_amd import binding as B               # noqa: E402

MATS, N, K, LR, MLR = [(3, 40, 64), (2700, 70, 90)], 9100, 3, 0.3, 0.5


class Server:
    def __init__(self):
        g = torch.Generator(device="cuda").manual_seed(3)
        r = lambda: torch.randn(N, generator=g, device="cuda")      # noqa: E731
        self.w, self.momentum, self.grads = r(), 0.1 * r(), [r() for _ in range(K)]
        self.start = self.w.clone(), self.momentum.clone()
        self.nbytes = B.dssp_orthogonal_workspace_bytes(MATS)
        self.ws = torch.empty(self.nbytes, dtype=torch.uint8, device="cuda")
        self.space = [torch.full((N + 4,), float("nan"), device="cuda") for _ in range(K)]
        self.streams = [torch.cuda.Stream() for _ in range(K)]
        torch.cuda.synchronize()
        self.ctx = B.dssp_create(self.w, N, K, 3, 0, LR)
        for p in range(K):
            B.dssp_set_stream(self.ctx, p, self.streams[p])
        B.dssp_set_orthogonal_update(self.ctx, MATS, MLR, self.momentum, self.ws, self.nbytes, momentum=0.9, nesterov=True, steps=4, eps=1e-6)

    def snapshot(self, p, shift=0):
        return self.space[p].data_ptr() + 4 * shift

    def refused(self, call):
        with pytest.raises(B.DsspError) as e:
            call()
        assert e.value.code in (B.DSSP_EHIP, B.DSSP_EINVAL)
        torch.cuda.synchronize()
        assert torch.equal(self.w, self.start[0]) and torch.equal(self.momentum, self.start[1])
        assert B.dssp_device_stamps(self.ctx, K) == [0] * (K + 1)
        assert B.dssp_clock(self.ctx, K)[3] == 0 and B.dssp_clock(self.ctx, K)[0] == [0] * K
        assert all(torch.isnan(s).all() for s in self.space)

    def expected(self, count):
        """weights and momentum after the first `count` gradients, by the launcher called by hand"""
        (w, m), L, table = (t.clone() for t in self.start), B.lib(), B.matrix_table(MATS)
        ws, states = torch.empty(self.nbytes, dtype=torch.uint8, device="cuda"), []
        for p in range(count):
            assert L.dsspk_orthogonal_apply(torch.cuda.current_stream().cuda_stream, w.data_ptr(), w.data_ptr(), m.data_ptr(), m.data_ptr(), self.grads[p].data_ptr(), N, table,
                                            len(MATS), np.float32(MLR) / np.float32(K), np.float32(LR) / np.float32(K), 0.9, 1, 4, 1e-6, ws.data_ptr(), self.nbytes) == 0
            torch.cuda.synchronize()
            states.append((w.clone(), m.clone()))
        return states


def test_push_pull_refuses_before_anything_is_launched():
    s = Server()
    push = lambda p, grad, dst: B.dssp_push_pull(s.ctx, p, grad, 0, K, dst)       # noqa: E731
    for dst in (s.snapshot(0, 1), s.w, s.w.data_ptr() + 64, s.momentum, s.ws):
        s.refused(lambda: push(0, s.grads[0], dst))
    for grad in (s.w, s.momentum, s.momentum.data_ptr() + 4):
        s.refused(lambda: push(0, grad, s.snapshot(0)))
        s.refused(lambda: B.dssp_push(s.ctx, 0, grad, 0, K))
    # the same pushes in order, each on a stream of its own: right behind the refusals, and behind one another
    want = s.expected(K)
    for p in range(K):
        assert push(p, s.grads[p], s.snapshot(p))[4]
        with pytest.raises(B.DsspError):
            push(p, s.grads[p], s.snapshot(p, 1))
    B.dssp_synchronize(s.ctx)
    for p in range(K):
        assert torch.equal(s.space[p][:N], want[p][0])
    assert torch.equal(s.w, want[-1][0]) and torch.equal(s.momentum, want[-1][1])
    assert B.dssp_device_stamps(s.ctx, K) == [3, 1, 2, 3]
    B.dssp_destroy(s.ctx)


def test_push_many_refuses_before_anything_is_launched():
    s = Server()
    good = [s.snapshot(p) for p in range(K)]
    push = lambda grads, dst: B.dssp_push_many(s.ctx, list(range(K)), grads, 0, K, dst)       # noqa: E731
    for q, dst in ((2, s.snapshot(2, 1)), (2, s.w), (1, s.momentum), (2, s.ws), (2, good[0]), (2, good[1] + 16), (0, s.grads[2]), (0, s.grads[1]), (2, None)):
        s.refused(lambda: push(s.grads, good[:q] + [dst] + good[q + 1:]))
    for j, grad in ((2, s.w), (1, s.momentum)):
        s.refused(lambda: push(s.grads[:j] + [grad] + s.grads[j + 1:], good))
    assert all(push(s.grads, good)[0])
    B.dssp_synchronize(s.ctx)
    want = s.expected(K)
    for p in range(K):
        assert torch.equal(s.space[p][:N], want[p][0])
    assert torch.equal(s.w, want[-1][0]) and torch.equal(s.momentum, want[-1][1])
    assert B.dssp_device_stamps(s.ctx, K) == [3, 1, 2, 3]
    B.dssp_destroy(s.ctx)
