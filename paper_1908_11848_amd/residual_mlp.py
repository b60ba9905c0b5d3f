"""A pre-norm residual network over image patches, built from the raw launchers (layer norm, product with epilogue and their gradients) and trained by DSSP
pushes under either server rule: the paper's w <- w - (lr / K) g or the orthogonalised one.

Every image is cut into 64 patches of 4 x 4 pixels, the rows of all activations:

  x = patches W_in + b_in;   depth times  x <- x + gelu(norm(x) W_1 + b_1) W_2 + b_2;   logits = mean over an image's rows of norm(x), times W_out + b_out

Weights, gradients and the server stay in fp32 (Alg. 1's flat vectors); with type 'bf16' a worker works on a bf16 copy of its snapshot's matrices.

  python -m paper_1908_11848_amd.residual_mlp [--type bf16] [--rule orthogonal] [--width 256] [--hidden 1024] [--depth 2] [--batch 32] [--workers 4] [--pushes 64]
"""
import argparse
import math
import time

import numpy as np
import torch

from . import binding as B
from . import driver, inputs

PATCH, ROWS, FEATURES = 4, 64, 48
EPS = 1e-5
TYPES = {"fp32": (B.DSSPK_F32, torch.float32), "bf16": (B.DSSPK_BF16, torch.bfloat16)}


def patches(x):
    """[m][32][32][3] images -> [m * 64][48] patches"""
    m = x.shape[0]
    return np.ascontiguousarray(x.reshape(m, 8, PATCH, 8, PATCH, 3).transpose(0, 1, 3, 2, 4, 5)).reshape(m * ROWS, FEATURES)


def segments(width, hidden, depth, n_classes):
    """[(name, kind, size, fan_in)] of the flat vector, in forward order"""
    s = [("w_in", 0, FEATURES * width, FEATURES), ("b_in", 1, width, 0)]
    for i in range(depth):
        s += [("gamma%d" % i, 2, width, 0), ("beta%d" % i, 3, width, 0), ("w1_%d" % i, 0, width * hidden, width), ("b1_%d" % i, 1, hidden, 0),
              ("w2_%d" % i, 0, hidden * width, hidden), ("b2_%d" % i, 1, width, 0)]
    return s + [("gamma", 2, width, 0), ("beta", 3, width, 0), ("w_out", 0, width * n_classes, width), ("b_out", 1, n_classes, 0)]


class Step:
    """One worker's forward and backward pass: its buffers, and the launches that fill them."""

    def __init__(self, width, hidden, depth, batch, n_classes, type, device):
        self.width, self.hidden, self.depth, self.batch, self.n_classes = width, hidden, depth, batch, n_classes
        self.type, t = TYPES[type]
        self.at, at = {}, 0
        for name, _, size, _ in segments(width, hidden, depth, n_classes):
            self.at[name] = at
            at += size
        self.n = at
        L, M = B.lib(), batch * ROWS
        new = lambda *shape, dtype=t: torch.empty(*shape, dtype=dtype, device=device)       # noqa: E731
        f32 = lambda *shape: new(*shape, dtype=torch.float32)      # noqa: E731
        self.x = [new(M, width) for _ in range(depth + 1)]         # the residual stream in front of every block and behind the last
        self.norm = [new(M, width) for _ in range(depth + 1)]
        self.stats = [f32(M, 2) for _ in range(depth + 1)]
        self.z, self.h = [new(M, hidden) for _ in range(depth)], [new(M, hidden) for _ in range(depth)]
        self.dx, self.dnorm, self.dh = new(M, width), new(M, width), new(M, hidden)
        # the last norm's output and its gradient for the pooling, which is fp32: in fp32 they are these themselves
        self.wide, self.dwide = (f32(M, width), f32(M, width)) if type == "bf16" else (self.norm[depth], self.dnorm)
        self.pooled, self.dpooled = f32(batch, width), f32(batch, width)
        self.logits, self.dlogits = f32(batch, n_classes), f32(batch, n_classes)
        self.copy = new(self.n) if type == "bf16" else None
        T = self.type
        need = [L.dsspk_linear_fwd_workspace_bytes(T, M, width, FEATURES), L.dsspk_linear_bwd_workspace_bytes(T, M, width, FEATURES),
                L.dsspk_linear_fwd_workspace_bytes(B.DSSPK_F32, batch, n_classes, width), L.dsspk_linear_bwd_workspace_bytes(B.DSSPK_F32, batch, n_classes, width),
                4 * L.dsspk_layernorm_bwd_scratch_floats(M, width)]
        for n, k in ((hidden, width), (width, hidden)):
            need += [L.dsspk_linear_fwd_workspace_bytes(T, M, n, k), L.dsspk_linear_bwd_workspace_bytes(T, M, n, k)]
        self.ws = torch.empty(max(need), dtype=torch.uint8, device=device)

    def run(self, stream, x, y, w, grad, loss):
        """grad = gradient of the mean softmax cross-entropy on patches x [batch * 64][48] (of this step's type) and labels y at the fp32 weights w."""
        with torch.cuda.stream(stream):         # for the one conversion that is a torch copy: bf16 to fp32
            self._run(B.stream_handle(stream), x, y, w, grad, loss)

    def _run(self, s, x, y, w, grad, loss):
        L, T, M, W, H = B.lib(), self.type, self.batch * ROWS, self.width, self.hidden
        vec = lambda name: w.data_ptr() + 4 * self.at[name]         # noqa: E731
        grd = lambda name: grad.data_ptr() + 4 * self.at[name]      # noqa: E731
        if T == B.DSSPK_BF16:
            _ok(L.dsspk_to_bf16(s, self.copy.data_ptr(), w.data_ptr(), self.n))
            mat = lambda name: self.copy.data_ptr() + 2 * self.at[name]       # noqa: E731
        else:
            mat = vec
        ws, nws = self.ws.data_ptr(), self.ws.numel()
        p = lambda t: t.data_ptr()      # noqa: E731

        def norm(i, name):
            _ok(L.dsspk_layernorm_fwd(s, T, p(self.x[i]), W, vec("gamma" + name), vec("beta" + name), p(self.norm[i]), W, p(self.stats[i]), M, W, EPS))

        def norm_back(i, name, dy, add):
            _ok(L.dsspk_layernorm_bwd(s, T, p(self.x[i]), W, vec("gamma" + name), p(self.stats[i]), p(dy), W, B.ptr(add), W, p(self.dx), W,
                                      grd("gamma" + name), grd("beta" + name), ws, M, W))

        _ok(L.dsspk_linear_fwd(s, T, p(x), FEATURES, mat("w_in"), vec("b_in"), B.DSSPK_ACT_NONE, None, 0, p(self.x[0]), W, None, 0, M, W, FEATURES, ws, nws))
        for i in range(self.depth):
            norm(i, "%d" % i)
            _ok(L.dsspk_linear_fwd(s, T, p(self.norm[i]), W, mat("w1_%d" % i), vec("b1_%d" % i), B.DSSPK_ACT_GELU, None, 0, p(self.h[i]), H, p(self.z[i]), H,
                                   M, H, W, ws, nws))
            _ok(L.dsspk_linear_fwd(s, T, p(self.h[i]), H, mat("w2_%d" % i), vec("b2_%d" % i), B.DSSPK_ACT_NONE, p(self.x[i]), W, p(self.x[i + 1]), W, None, 0,
                                   M, W, H, ws, nws))
        norm(self.depth, "")
        bf16 = T == B.DSSPK_BF16
        if bf16:
            self.wide.copy_(self.norm[self.depth])
        _ok(L.dsspk_gap_fwd(s, p(self.wide), p(self.pooled), self.batch, ROWS, W))
        C, m = self.n_classes, self.batch
        _ok(L.dsspk_linear_fwd(s, B.DSSPK_F32, p(self.pooled), W, vec("w_out"), vec("b_out"), B.DSSPK_ACT_NONE, None, 0, p(self.logits), C, None, 0, m, C, W, ws, nws))
        _ok(L.dsspk_softmax_xent(s, p(self.logits), p(y), p(self.dlogits), p(loss), m, C))
        _ok(L.dsspk_linear_bwd(s, B.DSSPK_F32, p(self.pooled), W, vec("w_out"), p(self.dlogits), C, p(self.dpooled), W, None, 0, B.DSSPK_ACT_NONE, grd("w_out"),
                               grd("b_out"), m, C, W, ws, nws))
        _ok(L.dsspk_gap_bwd(s, p(self.dpooled), p(self.dwide), m, ROWS, W))
        if bf16:
            _ok(L.dsspk_to_bf16(s, p(self.dnorm), p(self.dwide), self.dwide.numel()))
        norm_back(self.depth, "", self.dnorm, None)
        for i in reversed(range(self.depth)):
            # through the second product and the activation in front of it, through the first, through the norm, and past all three
            _ok(L.dsspk_linear_bwd(s, T, p(self.h[i]), H, mat("w2_%d" % i), p(self.dx), W, p(self.dh), H, p(self.z[i]), H, B.DSSPK_ACT_GELU, grd("w2_%d" % i),
                                   grd("b2_%d" % i), M, W, H, ws, nws))
            _ok(L.dsspk_linear_bwd(s, T, p(self.norm[i]), W, mat("w1_%d" % i), p(self.dh), H, p(self.dnorm), W, None, 0, B.DSSPK_ACT_NONE, grd("w1_%d" % i),
                                   grd("b1_%d" % i), M, H, W, ws, nws))
            norm_back(i, "%d" % i, self.dnorm, self.dx)
        _ok(L.dsspk_linear_bwd(s, T, p(x), FEATURES, None, p(self.dx), W, None, 0, None, 0, B.DSSPK_ACT_NONE, grd("w_in"), grd("b_in"), M, W, FEATURES, ws, nws))


def _ok(rc):
    if rc:
        raise B.DsspError(rc, "a launch was refused or failed")


class Training:
    """K workers of one network on one GPU, trained by a DSSP schedule (driver.Schedule)."""

    def __init__(self, width=256, hidden=1024, depth=2, batch=32, n_classes=10, K=4, s_L=3, r_max=12, lr=0.05, type="bf16", rule="orthogonal", matrix_lr=0.04,
                 pool=2, config=4, device="cuda:0", keep=4096):
        """keep: the losses of so many iterations of every worker stay, behind that the oldest are overwritten"""
        if type not in TYPES or rule not in ("orthogonal", "sgd"):
            raise ValueError("type is 'fp32' or 'bf16', rule 'orthogonal' or 'sgd'")
        if not 1 <= batch <= 1024 or not 2 <= n_classes <= 1024 or min(width, hidden, K, pool, keep) < 1 or depth < 0:
            raise ValueError("batch in [1, 1024], n_classes in [2, 1024], width, hidden, K, pool, keep >= 1, depth >= 0")
        self.K, self.dev = K, torch.device(device)
        torch.cuda.set_device(self.dev)
        self.seg = segments(width, hidden, depth, n_classes)
        w0 = inputs.init_weights([(kind, size, fan) for _, kind, size, fan in self.seg], config)
        xs, ys = inputs.batches(config, K, pool, batch, n_classes)
        t = TYPES[type][1]
        self.xs = [[torch.from_numpy(patches(x)).to(self.dev).to(t) for x in row] for row in xs]
        self.ys = [[torch.from_numpy(y).to(self.dev) for y in row] for row in ys]
        self.w = torch.from_numpy(w0).to(self.dev)
        n = self.w.numel()
        pitch = (n + 63) // 64 * 64
        self.w_local = torch.empty((K, pitch), dtype=torch.float32, device=self.dev)[:, :n]
        self.grad = torch.zeros((K, pitch), dtype=torch.float32, device=self.dev)[:, :n]
        self.losses = torch.zeros((K, keep), dtype=torch.float32, device=self.dev)         # of each worker's iterations: n at n % keep
        self.steps = [Step(width, hidden, depth, batch, n_classes, type, self.dev) for _ in range(K)]
        self.streams = [torch.cuda.Stream(device=self.dev) for _ in range(K)]
        self.ctx = B.dssp_create(self.w, n, K, s_L, r_max, lr)
        for p in range(K):
            B.dssp_set_stream(self.ctx, p, self.streams[p])
        if rule == "orthogonal":
            matrices = B.weight_matrices([(kind, size, fan) for _, kind, size, fan in self.seg])
            nbytes = B.dssp_orthogonal_workspace_bytes(matrices)
            self.momentum = torch.zeros_like(self.w)
            self.orth_ws = torch.empty(nbytes, dtype=torch.uint8, device=self.dev)
            torch.cuda.synchronize()
            B.dssp_set_orthogonal_update(self.ctx, matrices, matrix_lr, self.momentum, self.orth_ws, nbytes)
        torch.cuda.synchronize()

    def step(self, p, n):
        j = n % len(self.xs[p])
        i = n % self.losses.shape[1]
        self.steps[p].run(self.streams[p], self.xs[p][j], self.ys[p][j], self.w_local[p], self.grad[p], self.losses[p, i:i + 1])

    def schedule(self, durations, **kw):
        return driver.Schedule(self.ctx, self.K, durations, grad_ptr=lambda p: self.grad[p], pull_dst=lambda p: self.w_local[p], step=self.step, **kw)

    def synchronize(self):
        B.dssp_synchronize(self.ctx)

    def close(self):
        if self.ctx is not None:
            B.dssp_destroy(self.ctx)
            self.ctx = None


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--type", choices=sorted(TYPES), default="bf16")
    ap.add_argument("--rule", choices=["orthogonal", "sgd"], default="orthogonal")
    for name, default in (("width", 256), ("hidden", 1024), ("depth", 2), ("batch", 32), ("workers", 4), ("pushes", 64)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    t = Training(a.width, a.hidden, a.depth, a.batch, K=a.workers, type=a.type, rule=a.rule, keep=a.pushes + 1)
    sched = t.schedule(inputs.durations(4, a.workers, a.pushes + 1), log=False, fused_pull=True)
    sched.advance(a.workers)            # everybody has pushed about once: first launches are not timed
    t.synchronize()
    t0 = time.perf_counter()
    done = sched.advance(a.pushes - a.workers)
    t.synchronize()
    per = (time.perf_counter() - t0) / max(1, done)
    first = t.losses[:, 0].mean().item()
    last = np.mean([t.losses[p, max(0, sched.count[p] - 1)].item() for p in range(a.workers)])
    print("%d parameters, %s, %s rule: %d pushes, %.0f us a push, mean loss %.3f -> %.3f" % (t.w.numel(), a.type, a.rule, a.pushes, 1e6 * per, first, last))
    assert math.isfinite(last)
    t.close()


if __name__ == "__main__":
    main()
