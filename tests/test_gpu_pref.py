"""GPU parity of the preference loss (include/mux_pref.h) against the fp64 oracle, through the C ABI.

Tolerances, derived, with u = 2^-24: a row's sum of exponentials runs over at most 34 terms a thread and ten joining steps and
some per slab, each exponential off by (|z| + 4) u with the argument z at least -|x_label - max| - 40 where it counts: the log of the sum is off by
128 u, the row's log-probability by (|lp| + 160) u with its last rounding, a sequence's by the sum of these plus u |L|.  A loss is beta
times Lipschitz in each sum.  A gradient is c (onehot - p): p off by 320 u p, c by beta |dloss| (beta times the sums' errors) / 4 + 4 u |c|; one
rounding to the stored type (half a step)."""
import numpy as np
import pytest

from oracle import pref as opref
from oracle import segtab

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_02885_amd as mx
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    mx.load_library()
    return mx, torch


class Case:
    """Rows that do not count hold NaN, as do the columns beyond the vocabulary and every output before the call."""

    def __init__(self, env, lens, chunk, vocab, dtype, pairs, seed=0, pack=0, flags=0, pad=0, padg=0, shift=0, shiftg=0, answers=0.7, sigma=2.0):
        mx, torch = self.mx, self.torch = env
        self.ot = segtab.build(lens, chunk, pack, flags)
        self.st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, v) for v in lens], chunk, pack, flags)
        self.seqs = [(s[2], s[3]) for s in segtab.sequences(self.ot)]
        self.T, self.V, self.pairs, self.n = self.ot.T, vocab, pairs, len(pairs)
        self.td = torch.float32 if dtype == mx.MUX_DT_F32 else torch.bfloat16
        rng = np.random.default_rng(seed)
        self.ld, self.ldg = vocab + pad, vocab + padg
        labels = rng.integers(0, vocab, self.T)
        labels[rng.random(self.T) > answers] = -1
        outside = np.flatnonzero(labels < 0)
        labels[outside[::3]] = -100
        labels[outside[1::3]] = vocab
        valid = self.ot.row_task >= 0                  # (labels of padding rows stay whatever they are)
        self.on = valid & (labels >= 0) & (labels < vocab)
        x = rng.standard_normal((self.T, vocab)) * sigma
        x[np.arange(self.T)[self.on], labels[self.on]] += 4.0
        nan = float("nan")
        full = torch.full((self.T * self.ld + shift,), nan, dtype=self.td, device="cuda")
        self.x = full[shift:].view(self.T, self.ld)
        self.x[:, :vocab] = torch.from_numpy(x.astype(np.float32)).cuda().to(self.td)
        self.x[torch.from_numpy(~self.on).cuda()] = nan
        self.labels = torch.from_numpy(labels.astype(np.int32)).cuda()
        gfull = torch.full((self.T * self.ldg + shiftg,), nan, dtype=self.td, device="cuda")
        self.dx = gfull[shiftg:].view(self.T, self.ldg)
        self.ref = torch.from_numpy((rng.standard_normal(len(self.seqs)) * 3).astype(np.float32)).cuda()
        self.dloss = torch.from_numpy(rng.uniform(-1, 1, max(self.n, 1)).astype(np.float32)).cuda()
        self.desc = mx.PrefDesc(vocab, dtype, self.ld, self.ldg)
        self.layout = torch.from_numpy(mx.mux_pref_layout(self.st, pairs)).cuda()
        new = lambda n: torch.full((max(n, 1),), nan, device="cuda")                                                  # noqa: E731
        self.row_logp, self.logp, self.loss = new(self.T), new(len(self.seqs)), new(self.n)
        scratch = lambda b: torch.full((max(b, 256),), 0xFF, dtype=torch.uint8, device="cuda")                         # noqa: E731
        self.saved = scratch(mx.mux_pref_saved_bytes(self.desc, self.st, self.n))
        self.wsb = mx.mux_pref_workspace_bytes(self.desc, self.st)
        self.ws = scratch(self.wsb)
        torch.cuda.synchronize()
        print(f"pref case: T={self.T} V={vocab} seqs={len(self.seqs)} pairs={self.n} {self.td} ld={self.ld},{self.ldg} shift={shift},{shiftg}", flush=True)

    def forward(self, saved=True):
        self.mx.mux_pref_forward(self.desc, self.st, self.layout, self.n, self.x, self.labels, self.ref if self.n else None, self.row_logp,
                                 self.logp, self.loss if self.n else None, self.saved if saved else None, self.ws, self.wsb,
                                 self.torch.cuda.current_stream())

    def backward(self, dx=None):
        self.mx.mux_pref_backward(self.desc, self.st, self.layout, self.n, self.x, self.labels, self.saved, self.dloss if self.n else None,
                                  self.dx if dx is None else dx, self.torch.cuda.current_stream())

    def host(self, t):
        return t.float().cpu().numpy().astype(np.float64)

    def reference(self):
        if not hasattr(self, "_ref"):
            x, lab, ref = self.host(self.x)[:, :self.V], self.labels.cpu().numpy(), self.host(self.ref)
            self._ref = opref.forward(x, lab, self.seqs, self.pairs, ref), opref.backward(x, lab, self.seqs, self.pairs, ref, self.host(self.dloss))
        return self._ref

    def check(self, dx=None):
        f, d = self.reference()
        e_row = np.where(self.on, (np.abs(f["row_logp"]) + 160) * U, 0.0)
        got = self.host(self.row_logp)
        assert (np.abs(got - f["row_logp"]) <= e_row).all(), float(np.abs(got - f["row_logp"]).max())
        e_seq = np.array([e_row[a:a + n].sum() for a, n in self.seqs]) + U * np.abs(f["logp"])
        assert (np.abs(self.host(self.logp)[:len(self.seqs)] - f["logp"]) <= e_seq).all()
        if self.n:
            e_m = np.array([b * (e_seq[c] + e_seq[r]) for c, r, b, _ in self.pairs])
            assert (np.abs(self.host(self.loss) - f["loss"]) <= e_m + 2 * U * f["loss"]).all()
        if dx is None:
            return
        got = self.host(dx)[:, :self.V]
        half = float(self.torch.finfo(self.td).eps) / 2
        c_seq, ec_seq, used = np.zeros(len(self.seqs)), np.zeros(len(self.seqs)), np.zeros(len(self.seqs), dtype=bool)
        w = np.abs(self.host(self.dloss))
        for k, (c, r, b, _) in enumerate(self.pairs):
            for s in (c, r):
                c_seq[s] += w[k] * b
                ec_seq[s] += w[k] * b * (e_m[k] / 4 + 8 * U)
                used[s] = True
        x = self.host(self.x)[:, :self.V]
        for s, (first, n) in enumerate(self.seqs):
            for i in range(first, first + n):
                if not self.on[i] or not used[s]:
                    assert (got[i] == 0).all(), i
                    continue
                p = np.exp(x[i] - x[i].max())
                p /= p.sum()
                tol = half * np.abs(d[i]) + ec_seq[s] * p + c_seq[s] * 320 * U * p + 1e-37
                y = int(self.labels[i])
                tol[y] += ec_seq[s] + 4 * U * c_seq[s]
                assert (np.abs(got[i] - d[i]) <= tol).all(), (i, float((np.abs(got[i] - d[i]) / tol).max()))
        assert (got[self.ot.row_task < 0] == 0).all()


LENS = [[1, 2, 40, 33], [64, 65], [], [3, 130]]
PAIRS = [(0, 1, 0.1, 0.0), (2, 3, 0.5, 0.1), (5, 4, 0.2, 0.0), (6, 7, 0.1, 0.3)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("vocab", [1, 2, 9, 127, 1000, 4099, 8192, 8200, 20011, 33000])
def test_vocabularies(env, vocab, dtype):
    """One entry, a few, odd sizes, one slab, several: rows begin at every place inside 16 bytes."""
    c = Case(env, LENS, 16, vocab, dtype, PAIRS, seed=vocab)
    c.forward()
    c.backward()
    c.check(c.dx)


@pytest.mark.parametrize("chunk,pack,flags", [(1, 0, 0), (4, 50, 0), (16, 0, 1), (128, 0, 0)])
def test_tables(env, chunk, pack, flags):
    c = Case(env, LENS, chunk, 500, 0, PAIRS, seed=chunk, pack=pack, flags=flags)
    c.forward()
    c.backward()
    c.check(c.dx)


@pytest.mark.parametrize("dtype,pad,padg,shift,shiftg", [(0, 8, 0, 0, 0), (0, 3, 3, 1, 1), (0, 3, 0, 0, 0), (0, 0, 0, 1, 2), (0, 5, 13, 7, 7), (1, 1, 1, 3, 3), (1, 0, 2, 0, 0), (1, 4, 0, 1, 0)])
def test_strides_and_alignment(env, dtype, pad, padg, shift, shiftg):
    """Logits and gradients whose rows begin at the same or at different places; columns beyond the vocabulary stay."""
    c = Case(env, LENS, 16, 1003, dtype, PAIRS, seed=4, pad=pad, padg=padg, shift=shift, shiftg=shiftg)
    c.forward()
    c.backward()
    c.check(c.dx)
    assert c.torch.isnan(c.dx[:, 1003:]).all()


def test_sequences_in_many_pairs(env):
    """One sequence chosen over several, rejected by another, some in no pair; the same pair twice."""
    pairs = [(0, 1, 0.3, 0.0), (0, 2, 0.3, 0.1), (0, 3, 0.1, 0.0), (3, 2, 0.2, 1.0), (0, 1, 0.3, 0.0), (5, 4, 0.1, 0.0)]
    c = Case(env, LENS, 16, 700, 1, pairs, seed=5)
    c.forward()
    c.backward()
    c.check(c.dx)


def test_many_pairs(env):
    """More pairs than one workgroup takes, and a sequence in hundreds of them."""
    lens = [[int(v) for v in np.random.default_rng(1).integers(1, 9, 700)]]
    pairs = [(i, (i * 7 + 1) % 700, 0.1, 0.0) for i in range(0, 600, 2) if i != (i * 7 + 1) % 700] + [(3, j, 0.02, 0.0) for j in range(4, 400)]
    c = Case(env, lens, 64, 33, 1, pairs, seed=6)
    c.forward()
    c.backward()
    c.check(c.dx)


def test_reference_pass(env):
    """No pairs: log-probabilities alone, with and without what a backward would need; its gradient is zero."""
    c = Case(env, LENS, 16, 1003, 0, [], seed=7)
    c.forward(saved=False)
    c.check()
    c.forward()
    c.backward()
    assert (c.host(c.dx)[:, :1003] == 0).all()


def test_sequences_without_counted_rows(env):
    """Prompts alone: a sum of nothing is zero, its pair's loss follows from the reference."""
    c = Case(env, [[5, 6], [7, 8]], 16, 50, 1, [(0, 1, 0.5, 0.0), (2, 3, 0.5, 0.0)], seed=8)
    c.labels[:16] = -1
    c.on[:16] = False
    c.x[:16] = float("nan")
    c.forward()
    c.backward()
    c.check(c.dx)
    assert (c.logp[:2] == 0).all()


@pytest.mark.parametrize("dtype,vocab", [(0, 1000), (0, 1003), (1, 1003)])
def test_in_place(env, dtype, vocab):
    c = Case(env, LENS, 16, vocab, dtype, PAIRS, seed=9)
    c.forward()
    c.backward()
    c.check(c.dx)
    c.backward(dx=c.x)
    assert c.torch.equal(c.x, c.dx)


def test_special_values(env):
    """Masked vocabulary entries (-inf) have probability zero; a label among them costs an infinite loss when its sequence was
    chosen; logits of the type's lowest value; a NaN stays in its sequence's pair."""
    inf = float("inf")
    c = Case(env, [[4, 5], [6, 3], [2, 2]], 16, 300, 0, [(0, 1, 0.5, 0.0), (2, 3, 0.5, 0.0), (4, 5, 0.5, 0.0)], seed=10, answers=1.1)
    lab = c.labels.long()
    keep = c.x.gather(1, lab.clamp(0, 299)[:, None])
    c.x[:, ::3] = -inf
    c.x[:, 1::3] = c.torch.finfo(c.torch.bfloat16).min
    c.x.scatter_(1, lab.clamp(0, 299)[:, None], keep)
    c.forward()
    c.backward()
    c.check(c.dx)
    c.x[0, lab[0]] = -inf                                # the chosen sequence's first label becomes impossible
    c.x[16] = float("nan")                               # first row of sequence 2
    c.forward()
    c.backward()
    loss = c.host(c.loss)
    assert loss[0] == inf and np.isnan(loss[1]) and np.isfinite(loss[2]) and c.logp[0] == -inf
    d = c.host(c.dx)
    assert np.isfinite(d[:9]).all() and np.isnan(d[16:25]).all() and np.isfinite(d[32:36]).all()


def test_rows_without_a_probability(env):
    """A row that holds +inf, or nothing but -inf, makes its own sequence and its pairs NaN and nothing else."""
    inf = float("inf")
    for vocab, dtype in ((300, 0), (9001, 1)):
        c = Case(env, [[4, 5], [6, 3], [2, 2]], 16, vocab, dtype, [(0, 1, 0.5, 0.0), (2, 3, 0.5, 0.0), (4, 5, 0.5, 0.0)], seed=13, answers=1.1)
        c.x[1, vocab - 1] = inf
        c.x[17] = -inf
        c.forward()
        c.backward()
        loss, logp, d = c.host(c.loss), c.host(c.logp), c.host(c.dx)
        assert np.isnan(loss[:2]).all() and np.isfinite(loss[2])
        assert np.isnan(logp[[0, 2]]).all() and np.isfinite(logp[[1, 3, 4, 5]]).all()
        assert np.isnan(d[:9]).all() and np.isnan(d[16:25]).all() and np.isfinite(d[32:36]).all()


def test_repeats_streams_and_capture(env):
    c = Case(env, LENS, 16, 9001, 0, PAIRS, seed=11)
    c.forward()
    c.backward()
    c.check(c.dx)
    outs = [c.row_logp, c.logp, c.loss, c.dx]
    keep = [v.clone() for v in outs]
    s = c.torch.cuda.Stream()
    c.torch.cuda.synchronize()
    with c.torch.cuda.stream(s):
        c.forward()
        c.backward()
    c.torch.cuda.synchronize()
    assert all(c.torch.equal(a, b) for a, b in zip(keep, outs))
    graph = c.torch.cuda.CUDAGraph()
    with c.torch.cuda.graph(graph):
        c.forward()
        c.backward()
    for k in range(3):
        c.x.mul_(0.9)
        c.forward()
        c.backward()
        want = [v.clone() for v in outs]
        for v in outs + [c.ws, c.saved]:
            v.fill_(0)
        c.torch.cuda.synchronize()
        graph.replay()
        c.torch.cuda.synchronize()
        assert all(c.torch.equal(a, b) for a, b in zip(want, outs)), k


def test_rows_far_apart(env):
    """Offsets beyond 32 bits (rows of 2^23 elements' distance): the bits of the same rows side by side, nothing else written."""
    c = Case(env, LENS, 64, 9001, 0, PAIRS, seed=15, pad=7, padg=7)
    c.forward()
    c.backward()
    want = [t.clone() for t in (c.row_logp, c.logp, c.loss, c.dx[:, :9001])]
    ld = 1 << 23
    assert c.T * ld > 1 << 31
    far = [c.torch.empty((c.T, ld), dtype=c.td, device="cuda") for _ in range(2)]
    far[0][:, :9001] = c.x[:, :9001]
    far[1][:, :9100] = 7.0
    c.x, c.dx = far
    c.desc = c.mx.PrefDesc(9001, 0, ld, ld)
    for t in (c.row_logp, c.logp, c.loss):
        t.fill_(float("nan"))
    c.forward()
    c.backward()
    assert all(c.torch.equal(a, b) for a, b in zip(want, (c.row_logp, c.logp, c.loss, c.dx[:, :9001])))
    assert (c.dx[:, 9001:9100] == 7.0).all()
