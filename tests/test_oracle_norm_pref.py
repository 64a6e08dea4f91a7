"""Pins of the oracles of the layer norm and of the preference loss: hand-worked values, central differences, and the
layout of the pairs."""
import numpy as np
import pytest

from oracle import norm as onorm
from oracle import pref as opref


@pytest.fixture(scope="module")
def mx():
    import paper_2603_02885_amd as m
    m.load_library()
    return m


def test_norm_by_hand():
    # mean 2, squared deviations 1, 0, 1 -> variance 2/3; eps = 1/3 makes rstd 1
    X = np.array([[1.0, 2.0, 3.0], [9.0, 9.0, 9.0], [5.0, 5.0, 5.0]])
    got = onorm.forward(X, [0, -1, 1], [np.array([2.0, 3.0, 4.0]), None], [np.array([0.5, 0.0, -1.0]), None], 1.0 / 3.0)
    assert np.allclose(got["Y"], [[-1.5, 0.0, 3.0], [0, 0, 0], [0, 0, 0]], atol=1e-15)
    assert np.allclose(got["mean"], [2, 0, 5]) and np.allclose(got["rstd"], [1, 0, 3 ** 0.5])


def test_norm_gradients_by_differences():
    rng = np.random.default_rng(1)
    row_task = [0, 1, 1, -1, 0, 2]
    X, dY = rng.standard_normal((6, 5)), rng.standard_normal((6, 5))
    g = [rng.standard_normal(5), rng.standard_normal(5), None]
    b = [rng.standard_normal(5), None, None]
    eps = 1e-2
    total = lambda X, g, b: float((onorm.forward(X, row_task, g, b, eps)["Y"] * dY).sum())          # noqa: E731
    got = onorm.backward(X, dY, row_task, 3, g, eps)
    h = 1e-5
    for i in range(6):
        for n in range(5):
            E = np.zeros_like(X)
            E[i, n] = h
            assert abs((total(X + E, g, b) - total(X - E, g, b)) / (2 * h) - got["dX"][i, n]) < 1e-8
    for t in (0, 1):
        for n in range(5):
            e = np.zeros(5)
            e[n] = h
            up, down = [list(g) for _ in range(2)]
            up[t], down[t] = g[t] + e, g[t] - e
            assert abs((total(X, up, b) - total(X, down, b)) / (2 * h) - got["dgamma"][t][n]) < 1e-8
    assert np.allclose(got["dbeta"][2], dY[5]) and np.allclose(got["dbeta"][1], dY[1] + dY[2])


def test_pref_by_hand():
    # two sequences of two rows, vocabulary 2: equal logits give log 1/2 a row, a gap of log 3 gives log 3/4 and log 1/4
    l3 = np.log(3.0)
    logits = np.array([[0.0, 0.0], [l3, 0.0], [0.0, l3], [5.0, 5.0]])
    seqs, labels = [(0, 2), (2, 2)], np.array([1, 0, 0, -1])
    got = opref.forward(logits, labels, seqs, [(0, 1, 2.0, 0.0)], [0.0, 0.0])
    assert np.allclose(got["row_logp"], [np.log(0.5), np.log(0.75), np.log(0.25), 0.0])
    # m = 2 (log 3/8 - log 1/4) = 2 log 3/2 = log 9/4: sigma = 9/13
    assert np.allclose(got["loss"], [-np.log(9.0 / 13.0)])
    d = opref.backward(logits, labels, seqs, [(0, 1, 2.0, 0.0)], [0.0, 0.0], [1.0])
    c = -2.0 * 4.0 / 13.0
    assert np.allclose(d, [[-c * 0.5, c * 0.5], [c * 0.25, -c * 0.25], [-c * 0.75, c * 0.75], [0, 0]])


def test_pref_gradient_by_differences():
    rng = np.random.default_rng(2)
    seqs = [(0, 3), (3, 1), (5, 4), (9, 2)]
    logits, labels = rng.standard_normal((11, 7)), rng.integers(-1, 7, 11)
    pairs = [(0, 1, 0.5, 0.1), (0, 2, 1.5, 0.0), (2, 1, 0.7, 1.0)]
    ref, w = rng.standard_normal(4), rng.standard_normal(3)
    got = opref.backward(logits, labels, seqs, pairs, ref, w)
    for i in range(11):
        for n in range(7):
            E = np.zeros_like(logits)
            E[i, n] = 1e-5
            f = [float((opref.forward(logits + s * E, labels, seqs, pairs, ref)["loss"] * w).sum()) for s in (1, -1)]
            assert abs((f[0] - f[1]) / 2e-5 - got[i, n]) < 1e-8
    assert (got[[4, 9, 10]] == 0).all()


def test_pref_layout(mx):
    """The layout against a direct listing: rows to sequences (packs cut by chunks, padding between), pairs of each sequence."""
    from oracle import segtab
    lens = [[5, 9, 2], [], [3, 4], [30]]
    for chunk, pack, flags in ((8, 0, 0), (16, 10, 0), (4, 0, 1)):
        st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, v) for v in lens], chunk, pack, flags)
        o = segtab.build(lens, chunk, pack, flags)
        pairs = [(0, 1, 0.1, 0.0), (4, 3, 0.5, 0.25), (0, 2, 0.2, 1.0), (1, 0, 0.3, 0.0)]
        w = mx.mux_pref_layout(st, pairs)
        T, S, P = mx.mux_segtab_rows(st), 6, 4
        assert list(w[1:4]) == [T, S, P]
        want = np.full(T, -1)
        seqs = [(s[2], s[3]) for s in segtab.sequences(o)]
        for i, (first, n) in enumerate(seqs):
            want[first:first + n] = i
        assert np.array_equal(w[w[4]:w[4] + T], want)
        assert [tuple(v) for v in w[w[5]:w[5] + 2 * S].reshape(S, 2)] == seqs
        q = w[w[6]:w[6] + 4 * P].reshape(P, 4)
        assert [(int(a), int(b)) for a, b, _, _ in q] == [(c, r) for c, r, _, _ in pairs]
        assert np.array_equal(q[:, 2:].copy().view(np.float32), np.array([p[2:] for p in pairs], dtype=np.float32))
        ptr, ent = w[w[7]:w[7] + S + 1], w[w[8]:]
        by_seq = [[2 * k + side for k, p in enumerate(pairs) for side in (0, 1) if p[side] == s] for s in range(S)]
        assert [list(ent[ptr[s]:ptr[s + 1]]) for s in range(S)] == by_seq
        assert len(w) * 4 == mx.mux_pref_layout_bytes(st, P) and ptr[S] == 2 * P
    for bad in ([(0, 0, 0.1, 0.0)], [(0, 3, 0.1, 0.0)], [(0, 6, 0.1, 0.0)], [(-1, 0, 0.1, 0.0)], [(0, 1, 0.0, 0.0)],
                [(0, 1, float("nan"), 0.0)], [(0, 1, float("inf"), 0.0)], [(0, 1, 0.1, -0.1)], [(0, 1, 0.1, 1.5)]):
        with pytest.raises(mx.MuxError):
            mx.mux_pref_layout(st, bad)


def refused(mx, status, call, *a):
    with pytest.raises(mx.MuxError) as e:
        call(*a)
    assert e.value.status == status, str(e.value)


def test_norm_refusals(mx):
    """Every check happens on the host before a launch; addresses here are made up."""
    st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, [5]), mx.TaskDesc(0, 0, 1.0, [70])], 64)
    T = mx.mux_segtab_rows(st)
    M = 1 << 20
    tab, X, Y, G, sv, ws = (k * M for k in range(1, 7))

    def fwd(width=64, dtype=0, eps=1e-5, ldx=None, ldy=None, n=2, x=X, y=Y, tab=tab, g=None, s=sv):
        d = mx.NormDesc(width, dtype, [G] * n if g is None else g, None, eps, ldx, ldy)
        mx.mux_norm_forward(d, st, tab, x, y, s)

    bad = [(1, dict(dtype=7)), (1, dict(width=0)), (1, dict(eps=0.0)), (1, dict(eps=float("nan"))), (1, dict(eps=float("inf"))),
           (3, dict(width=32769)), (2, dict(ldx=63)), (2, dict(ldy=63)), (2, dict(n=1)), (1, dict(x=None)), (1, dict(y=None)),
           (1, dict(tab=None)), (3, dict(x=X + 1)), (3, dict(s=sv + 2)), (3, dict(dtype=1, y=Y + 2)), (1, dict(y=X + 128)),
           (1, dict(y=X, ldy=72)), (1, dict(s=X)), (1, dict(y=G)), (1, dict(g=[Y + 64, G])), (2, dict(ldx=1 << 41))]
    for status, kw in bad:
        refused(mx, status, lambda: fwd(**kw))

    d = mx.NormDesc(64, 0, [G, G + 128], None)
    wb = mx.mux_norm_workspace_bytes(d, st)
    dg, db, dX = [7 * M, 8 * M], [9 * M, 10 * M], 11 * M
    bwd = lambda x=X, dy=Y, s=sv, dx=dX, dg=dg, db=db, acc=0, w=ws, n=wb, tab=tab: (          # noqa: E731
        mx.mux_norm_backward(d, st, tab, x, dy, s, dx, dg, db, acc, w, n))
    bad = [(1, dict(x=None)), (1, dict(dy=None)), (1, dict(s=None)), (1, dict(w=None)), (4, dict(n=wb - 1)), (1, dict(acc=2)),
           (1, dict(tab=None)), (1, dict(dg=[7 * M, 7 * M + 128])), (1, dict(dg=[9 * M, None])), (1, dict(dg=[X, None])),
           (1, dict(dx=X + 128)), (1, dict(dx=sv)), (1, dict(dx=G)), (1, dict(w=X)), (1, dict(w=dX)), (1, dict(w=7 * M)),
           (3, dict(dg=[7 * M + 2, None])), (3, dict(w=ws + 1)), (3, dict(dx=dX + 1))]
    for status, kw in bad:
        refused(mx, status, lambda: bwd(**kw))
    assert mx.mux_norm_saved_bytes(d, st) >= 8 * T and mx.mux_norm_workspace_bytes(mx.NormDesc(0, 0, n_tasks=2), st) == 0
    empty = mx.mux_segtab_build([], 64)
    mx.mux_norm_forward(mx.NormDesc(8, 0, n_tasks=0), empty, None, None, None, None)


def test_launches_that_would_not_fit(mx):
    """A launch is held to 2^32 threads: what would take more is refused before anything runs."""
    M = 1 << 40
    st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, [(1 << 24) - 256]), mx.TaskDesc(0, 0, 1.0, [1])], 256)
    assert mx.mux_segtab_rows(st) == 1 << 24
    d = mx.NormDesc(1, 0, n_tasks=2)
    refused(mx, 2, lambda: mx.mux_norm_forward(d, st, M, 2 * M, 3 * M, None))
    refused(mx, 2, lambda: mx.mux_norm_backward(d, st, M, 2 * M, 3 * M, 4 * M, 5 * M, None, None, 0, None, 0))
    e = mx.PrefDesc(1)
    refused(mx, 2, lambda: mx.mux_pref_forward(e, st, M, 0, 2 * M, 3 * M, None, None, None, None, None, 4 * M, 1 << 60))
    refused(mx, 2, lambda: mx.mux_pref_backward(e, st, M, 0, 2 * M, 3 * M, 4 * M, None, 5 * M))
    st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, [64])], 64)
    e = mx.PrefDesc(1 << 30)                                       # 2^18 slabs of the gradient a row, 2^16 of the forward
    refused(mx, 2, lambda: mx.mux_pref_backward(e, st, M, 0, 2 * M, 3 * M, 4 * M, None, 5 * M))


def test_pref_refusals(mx):
    st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, [5, 6])], 16)
    M = 1 << 20
    lay, x, lab, ref, rl, lp, ls, sv, ws, dl, g = (k * M for k in range(1, 12))

    def fwd(V=100, dtype=0, ld=None, n=1, lay=lay, x=x, lab=lab, ref=ref, rl=rl, lp=lp, ls=ls, sv=sv, ws=ws, short=0):
        d = mx.PrefDesc(V, dtype, ld)
        mx.mux_pref_forward(d, st, lay, n, x, lab, ref, rl, lp, ls, sv, ws, mx.mux_pref_workspace_bytes(d, st) - short)

    bad = [(1, dict(dtype=3)), (1, dict(V=0)), (1, dict(n=-1)), (2, dict(ld=99)), (1, dict(lay=None)), (1, dict(x=None)),
           (1, dict(lab=None)), (1, dict(ws=None)), (1, dict(ref=None)), (1, dict(ls=None)), (4, dict(short=1)), (3, dict(x=x + 1)),
           (3, dict(lab=lab + 2)), (3, dict(sv=sv + 4)), (3, dict(ws=ws + 4)), (3, dict(dtype=1, x=x + 2)), (1, dict(rl=lp)),
           (1, dict(ls=lab)), (1, dict(ws=x)), (1, dict(sv=ws + 8)), (2, dict(ld=1 << 41)), (1, dict(rl=lay))]
    for status, kw in bad:
        refused(mx, status, lambda: fwd(**kw))

    def bwd(V=100, dtype=0, ld=None, ldg=None, n=1, lay=lay, x=x, lab=lab, sv=sv, dl=dl, g=g):
        mx.mux_pref_backward(mx.PrefDesc(V, dtype, ld, ldg), st, lay, n, x, lab, sv, dl, g)

    bad = [(2, dict(ldg=99)), (1, dict(lay=None)), (1, dict(x=None)), (1, dict(lab=None)), (1, dict(sv=None)), (1, dict(dl=None)),
           (1, dict(g=None)), (3, dict(g=g + 1)), (3, dict(sv=sv + 4)), (1, dict(g=x + 2)), (1, dict(g=x, ldg=108)),
           (1, dict(g=lab)), (1, dict(g=dl)), (1, dict(g=sv)), (1, dict(g=lay))]
    for status, kw in bad:
        refused(mx, status, lambda: bwd(**kw))
    empty = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, [])], 16)
    mx.mux_pref_forward(mx.PrefDesc(8), empty, None, 0, None, None, None, None, None, None, None, None, 0)
    refused(mx, 2, lambda: mx.mux_pref_forward(mx.PrefDesc(8), empty, lay, 1, x, lab, ref, rl, lp, ls, sv, ws, 1 << 20))
