"""GPU parity of the layer norm (include/mux_norm.h) against the fp64 oracle, through the C ABI.

Tolerances, derived: an output is rounded once (half a step, eps / 2 of its type).  Before that, in fp32 with u = 2^-24: a
row's sums run over at most 128 elements a lane and eleven joining steps (or over as many in another split), so the mean is off by at
most 160 u max|x| and an xhat by dx = 160 u max|x| rstd + 8 u (1 + |xhat|); Y by |gamma| dx + 4 u (|Y| + |beta|).  dX is rstd times a
difference of three terms of size at most max|h| (1 + max|xhat|)^2, each off by 400 u of it, plus 3 max|h| dx (1 + max|xhat|).  A weight's gradient is a sum over
n rows in some order: (n + 64) u sum|terms| + sum|dy| dx."""
import numpy as np
import pytest

from oracle import norm as onorm
from oracle import segtab

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_02885_amd as mx
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    mx.load_library()
    return mx, torch


class Case:
    """One call's tensors: rows of padding and the columns beyond the width hold NaN, outputs and scratch start as NaN."""

    def __init__(self, env, lens, chunk, width, dtype, seed=0, pack=0, flags=0, padx=0, pady=0, shift=0, gamma=True, beta=True, offset=0.5):
        mx, torch = self.mx, self.torch = env
        self.ot = segtab.build(lens, chunk, pack, flags)
        self.st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, v) for v in lens], chunk, pack, flags)
        self.T, self.N, self.n = self.ot.T, width, len(lens)
        self.td = torch.float32 if dtype == mx.MUX_DT_F32 else torch.bfloat16
        rng = np.random.default_rng(seed)
        pad = self.pad = self.ot.row_task < 0
        self.ldx, self.ldy = width + padx, width + pady
        nan = float("nan")

        def rows(ld, values=None):       # a [T, ld] buffer that starts `shift` elements into its memory
            full = torch.full((self.T * ld + shift,), nan, dtype=self.td, device="cuda")
            v = full[shift:].view(self.T, ld)
            if values is not None:
                v[:, :width] = torch.from_numpy(values.astype(np.float32)).cuda().to(self.td)
                v[torch.from_numpy(pad).cuda()] = nan
            return v

        self.X = rows(self.ldx, rng.standard_normal((self.T, width)) * (1 + rng.random(width)) + offset)
        self.dY = rows(self.ldy, rng.standard_normal((self.T, width)))
        self.Y, self.dX = rows(self.ldy), rows(self.ldx)
        vec = lambda mean: torch.from_numpy((rng.standard_normal(width) * 0.2 + mean).astype(np.float32)).cuda().to(self.td)   # noqa: E731
        self.gamma = [vec(1.0) for _ in lens] if gamma is True else gamma
        self.beta = [vec(0.0) for _ in lens] if beta is True else beta
        self.desc = mx.NormDesc(width, dtype, self.gamma, self.beta, EPS, self.ldx, self.ldy, n_tasks=self.n)
        nb = mx.mux_segtab_device_bytes(self.st)
        self.dtab = torch.zeros(nb, dtype=torch.uint8, device="cuda")
        mx.mux_segtab_upload(self.st, self.dtab, nb)
        torch.cuda.synchronize()
        scratch = lambda b: torch.full((max(b, 256),), 0xFF, dtype=torch.uint8, device="cuda")                                   # noqa: E731
        self.saved = scratch(mx.mux_norm_saved_bytes(self.desc, self.st))
        self.wsb = mx.mux_norm_workspace_bytes(self.desc, self.st)
        self.ws = scratch(self.wsb)
        self.dg = [torch.full((width,), nan, device="cuda") for _ in lens]
        self.db = [torch.full((width,), nan, device="cuda") for _ in lens]
        print(f"norm case: T={self.T} N={width} tasks={self.n} {self.td} ld={self.ldx},{self.ldy} shift={shift}", flush=True)

    def forward(self, Y=None):
        self.mx.mux_norm_forward(self.desc, self.st, self.dtab, self.X, self.Y if Y is None else Y, self.saved, self.torch.cuda.current_stream())

    def backward(self, dX=True, dg=True, db=True, acc=0):
        pick = lambda v, own: own if v is True else v                                                                            # noqa: E731
        self.mx.mux_norm_backward(self.desc, self.st, self.dtab, self.X, self.dY, self.saved, pick(dX, self.dX), pick(dg, self.dg),
                                  pick(db, self.db), acc, self.ws, self.wsb, self.torch.cuda.current_stream())

    def host(self, t):
        return t.float().cpu().numpy().astype(np.float64)

    def reference(self):
        if not hasattr(self, "_ref"):
            x, dy = self.host(self.X)[:, :self.N], self.host(self.dY)[:, :self.N]
            g = None if self.gamma is None else [None if v is None else self.host(v) for v in self.gamma]
            b = None if self.beta is None else [None if v is None else self.host(v) for v in self.beta]
            f = onorm.forward(x, self.ot.row_task, g, b, EPS)
            r = onorm.backward(x, dy, self.ot.row_task, self.n, g, EPS)
            self._ref = x, dy, g, b, f, r
        return self._ref

    def check(self, Y=None, dX=None, grads=True, base=0.0):
        x, dy, g, b, f, r = self.reference()
        ok = ~self.pad
        half = float(self.torch.finfo(self.td).eps) / 2
        G = np.ones((self.T, self.N)) if g is None else np.array([np.ones(self.N) if t < 0 or g[t] is None else g[t] for t in self.ot.row_task]).reshape(self.T, self.N)
        B = np.zeros((self.T, self.N)) if b is None else np.array([np.zeros(self.N) if t < 0 or b[t] is None else b[t] for t in self.ot.row_task]).reshape(self.T, self.N)
        xs, dys = np.where(ok[:, None], x, 0.0), np.where(ok[:, None], dy, 0.0)
        xh = (xs - f["mean"][:, None]) * f["rstd"][:, None]
        dxh = 160 * U * np.abs(xs).max(1, initial=0)[:, None] * f["rstd"][:, None] + 8 * U * (1 + np.abs(xh))
        if Y is not None:
            got = self.host(Y)[:, :self.N]
            assert (got[self.pad] == 0).all()
            tol = half * np.abs(f["Y"]) + np.abs(G) * dxh + 4 * U * (np.abs(f["Y"]) + np.abs(B))
            assert (np.abs(got - f["Y"])[ok] <= tol[ok]).all(), float((np.abs(got - f["Y"]) / tol)[ok].max())
            sv = self.saved[:8 * self.T].view(self.torch.float32).view(2, self.T).cpu().numpy().astype(np.float64)
            assert (np.abs(sv[0] - f["mean"])[ok] <= 160 * U * np.abs(xs).max(1, initial=0)[ok] + 1e-30).all()
            assert np.allclose(sv[1][ok], f["rstd"][ok], rtol=1e-4, atol=0)
        if dX is not None:
            got = self.host(dX)[:, :self.N]
            assert (got[self.pad] == 0).all()
            h = np.abs(dys * G).max(1, initial=0)[:, None]
            big = 1 + np.abs(xh).max(1, initial=0)[:, None]
            tol = half * np.abs(r["dX"]) + f["rstd"][:, None] * (400 * U * h * big ** 2 + 3 * h * dxh * big)
            assert (np.abs(got - r["dX"])[ok] <= tol[ok]).all(), float((np.abs(got - r["dX"]) / tol)[ok].max())
        if grads:
            for t in range(self.n):
                m = self.ot.row_task == t
                slack = (m.sum() + 64) * U
                tg = slack * (np.abs(dys * xh)[m].sum(0) + abs(base)) + (np.abs(dys) * dxh)[m].sum(0) + 1e-30
                tb = slack * (np.abs(dys)[m].sum(0) + abs(base)) + 1e-30
                assert (np.abs(self.host(self.dg[t]) - base - r["dgamma"][t]) <= tg).all(), t
                assert (np.abs(self.host(self.db[t]) - base - r["dbeta"][t]) <= tb).all(), t


LENS = [[1, 2, 31], [64], [], [65, 127], [200, 5], [129]]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("width", [1, 7, 64, 513, 1605, 2048, 2560, 4096, 5120, 5128])
def test_widths(env, width, dtype):
    """Widths of one element, odd ones, whole pieces, above what one wave takes; ragged lengths and a task without tokens."""
    c = Case(env, LENS, 64, width, dtype, seed=width + dtype)
    c.forward()
    c.backward()
    c.check(c.Y, c.dX)


@pytest.mark.parametrize("width,dtype", [(8192, 0), (8191, 0), (8192, 1), (5121, 1), (16392, 0), (20000, 1), (32768, 0), (32767, 0), (32768, 1), (32765, 1)])
def test_wide_rows(env, width, dtype):
    c = Case(env, [[3], [40, 30]], 32, width, dtype, seed=width)
    c.forward()
    c.backward()
    c.check(c.Y, c.dX)


@pytest.mark.parametrize("chunk,pack,flags", [(1, 0, 0), (4, 10, 0), (16, 0, 1), (128, 200, 0), (512, 0, 0)])
@pytest.mark.parametrize("width,dtype", [(264, 0), (130, 1)])
def test_tables(env, chunk, pack, flags, width, dtype):
    """Padding inside work items, items of a few rows, tasks back to back in a chunk."""
    c = Case(env, LENS, chunk, width, dtype, seed=chunk, pack=pack, flags=flags)
    c.forward()
    c.backward()
    c.check(c.Y, c.dX)


@pytest.mark.parametrize("width,dtype,padx,pady,shift", [(256, 0, 8, 24, 0), (256, 0, 1, 0, 0), (256, 0, 0, 0, 1), (250, 0, 6, 6, 0), (256, 1, 4, 0, 0), (256, 1, 0, 3, 0), (256, 1, 0, 0, 3)])
def test_strides_and_alignment(env, width, dtype, padx, pady, shift):
    """Columns beyond the width are neither read nor written; rows that begin at places no 16-byte piece does."""
    c = Case(env, LENS, 64, width, dtype, seed=3, padx=padx, pady=pady, shift=shift)
    c.forward()
    c.backward()
    c.check(c.Y, c.dX)
    assert c.torch.isnan(c.Y[:, width:]).all() and c.torch.isnan(c.dX[:, width:]).all()


def test_many_tasks(env):
    """More tasks than one launch takes, some without tokens; tasks without weights of their own share one or none."""
    lens = [[(7 * t) % 23 + 1] if t % 5 else [] for t in range(71)]
    c = Case(env, lens, 16, 264, 0, seed=5)
    for t in (3, 34, 70):
        c.gamma[t] = c.beta[t] = None
    c.gamma[6] = c.gamma[7] = c.gamma[40]
    c.desc = c.mx.NormDesc(264, 0, c.gamma, c.beta, EPS, n_tasks=71)
    c.forward()
    c.backward()
    c.check(c.Y, c.dX)


@pytest.mark.parametrize("gamma,beta", [(None, None), (True, None), (None, True)])
def test_without_weights(env, gamma, beta):
    c = Case(env, LENS, 64, 520, 0, seed=6, gamma=gamma, beta=beta)
    c.forward()
    c.backward()
    c.check(c.Y, c.dX)


@pytest.mark.parametrize("width,dtype", [(512, 0), (517, 0), (512, 1), (9000, 1)])
def test_in_place(env, width, dtype):
    """Y over X and dX over dY or over X give the bits that separate buffers give."""
    c = Case(env, LENS, 64, width, dtype, seed=7)
    c.forward()
    c.backward()
    c.check(c.Y, c.dX)
    y, dx, dg = c.Y.clone(), c.dX.clone(), [v.clone() for v in c.dg]
    x0, dy0 = c.X.clone(), c.dY.clone()
    for target in ("dY", "X"):
        c.backward(dX=getattr(c, target))
        got = getattr(c, target)
        assert c.torch.equal(got, dx) and all(c.torch.equal(a, b) for a, b in zip(c.dg, dg)), target
        c.X.copy_(x0), c.dY.copy_(dy0)
    c.forward(Y=c.X)
    assert c.torch.equal(c.X, y)


def test_parts_and_accumulation(env):
    """Gradients left out one by one, and added to what the buffers hold."""
    c = Case(env, LENS, 64, 520, 0, seed=8)
    c.forward()
    c.backward(dg=None, db=None)
    c.check(c.Y, c.dX, grads=False)
    assert all(c.torch.isnan(v).all() for v in c.dg + c.db)
    c.dX.fill_(float("nan"))
    c.backward(dX=None)
    assert c.torch.isnan(c.dX).all()
    c.check(grads=True)
    dg, db = [v.clone() for v in c.dg], [v.clone() for v in c.db]
    some = [None if t % 2 else v for t, v in enumerate(c.dg)]
    for v in c.dg + c.db:
        v.fill_(3.0)
    c.backward(dg=some, db=None, acc=0)
    assert all(c.torch.equal(v, w if t % 2 == 0 else c.torch.full_like(v, 3.0)) for t, (v, w) in enumerate(zip(c.dg, dg)))
    for v in c.dg + c.db:
        v.fill_(3.0)
    c.backward(acc=1)
    c.check(grads=True, base=3.0)
    assert (c.dg[2] == 3.0).all()                     # a task without tokens


def test_table_without_rows(env):
    """Tasks without tokens: nothing to normalise, gradients zero or left."""
    c = Case(env, [[], []], 64, 40, 0)
    c.backward(dX=None)
    assert all((v == 0).all() for v in c.dg + c.db)
    for v in c.dg:
        v.fill_(2.0)
    c.backward(acc=1)
    assert all((v == 2).all() for v in c.dg)


def test_special_values(env):
    """A constant row is all beta; a large offset costs what fp32 costs; an infinity or a NaN stays in its row (and, as the
    sums say, in its task's gradients)."""
    c = Case(env, [[4], [5]], 16, 264, 1, seed=9, offset=1000.0)
    c.X[1] = 7.0
    c.forward()
    c.backward()
    c.check(c.Y, c.dX)
    assert c.torch.equal(c.Y[1], c.beta[0])
    c.X[2, 5], c.X[3, 0] = float("inf"), float("nan")
    before = c.Y.clone()
    c.forward()
    c.backward()
    assert c.torch.isnan(c.Y[2]).any() and c.torch.isnan(c.Y[3]).all() and c.torch.equal(c.Y[16:], before[16:])
    assert c.torch.isnan(c.dg[0]).any() and not c.torch.isnan(c.dg[1]).any() and not c.torch.isnan(c.db[0]).any()


def test_large_batch_repeats_and_streams(env):
    """Pieces of many rows; the same bits every time, on another stream too."""
    c = Case(env, [[3000, 500], [2100], [4000], [1]], 256, 1024, 0, seed=10)
    c.forward()
    c.backward()
    c.check(c.Y, c.dX)
    keep = [v.clone() for v in [c.Y, c.dX] + c.dg + c.db]
    s = c.torch.cuda.Stream()
    for _ in range(3):
        for v in [c.Y, c.dX] + c.dg + c.db:
            v.fill_(float("nan"))
        c.torch.cuda.synchronize()
        with c.torch.cuda.stream(s):
            c.forward()
            c.backward()
        c.torch.cuda.synchronize()
        assert all(c.torch.equal(a, b) for a, b in zip(keep, [c.Y, c.dX] + c.dg + c.db))


def test_captured(env):
    """Forward and backward in a captured graph, replayed between eager calls on other data."""
    c = Case(env, LENS, 64, 520, 0, seed=11)
    c.forward()
    c.backward()
    c.torch.cuda.synchronize()
    graph = c.torch.cuda.CUDAGraph()
    with c.torch.cuda.graph(graph):
        c.forward()
        c.backward()
    for k in range(3):
        c.X.copy_(c.X * (0.5 + k))
        c.forward()
        c.backward()
        want = [v.clone() for v in [c.Y, c.dX] + c.dg + c.db]
        for v in [c.Y, c.dX, c.ws, c.saved] + c.dg + c.db:
            v.fill_(0)
        c.torch.cuda.synchronize()
        graph.replay()
        c.torch.cuda.synchronize()
        assert all(c.torch.equal(a, b) for a, b in zip(want, [c.Y, c.dX] + c.dg + c.db)), k


def test_rows_far_apart(env):
    """Offsets beyond 32 bits (rows of 2^22 elements' distance): the bits of the same rows side by side, nothing else written."""
    c = Case(env, LENS, 64, 513, 0, seed=14, padx=7, pady=7)
    c.forward()
    c.backward()
    want = [t.clone() for t in (c.Y[:, :513], c.dX[:, :513], *c.dg, *c.db)]
    ld = 1 << 22
    assert c.T * ld > 1 << 31
    far = [c.torch.empty((c.T, ld), dtype=c.td, device="cuda") for _ in range(4)]
    for f, t in zip(far, (c.X, c.dY, c.Y, c.dX)):
        f[:, :513] = t[:, :513]
        f[:, 513:600] = 7.0
    c.X, c.dY, c.Y, c.dX = far
    c.desc = c.mx.NormDesc(513, 0, c.gamma, c.beta, EPS, ld, ld, n_tasks=c.n)
    for t in (c.Y, c.dX):
        t[:, :513] = float("nan")
    c.forward()
    c.backward()
    got = (c.Y[:, :513], c.dX[:, :513], *c.dg, *c.db)
    assert all(c.torch.equal(a, b) for a, b in zip(want, got))
    assert all((t[:, 513:600] == 7.0).all() for t in (c.Y, c.dX))
