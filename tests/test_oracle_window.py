"""Pins of the windowed attention oracle, and the refusals of the windowed entry points."""
import numpy as np
import pytest

from oracle import attention as oatt


@pytest.fixture(scope="module")
def mx():
    import paper_2603_02885_amd as m
    m.load_library()
    return m


def test_visible_by_hand():
    rows = ["".join(".x"[int(v)] for v in row) for row in oatt.visible(6, 2, 1)]
    assert rows == ["x.....", "xx....", "xxx...", "x.xx..", "x..xx.", "x...xx"]
    assert np.array_equal(oatt.visible(5, 1, 0), np.eye(5, dtype=bool))
    assert np.array_equal(oatt.visible(7, 7, 3), oatt.visible(7)) and np.array_equal(oatt.visible(7, 2, 7), oatt.visible(7))


def test_against_loops_and_differences():
    """One head, written with scalar loops; gradients by central differences."""
    rng = np.random.default_rng(0)
    seqs, d, w, z = [(1, 7), (8, 1), (10, 4)], 3, 3, 2
    Q, K, V, dO = (rng.standard_normal((15, d)) for _ in range(4))

    def loops(Q, K, V):
        O = np.zeros((15, d))
        for first, n in seqs:
            for i in range(n):
                js = [j for j in range(i + 1) if i - j < w or j < z]
                e = np.array([np.exp(Q[first + i] @ K[first + j] / d ** 0.5) for j in js])
                O[first + i] = sum(p * V[first + j] for p, j in zip(e / e.sum(), js))
        return O

    assert np.allclose(oatt.forward(Q, K, V, seqs, 1, window=w, n_sinks=z)["O"], loops(Q, K, V), atol=1e-14)
    g = oatt.backward(Q, K, V, dO, seqs, 1, window=w, n_sinks=z)
    for name, k in (("dQ", 0), ("dK", 1), ("dV", 2)):
        for i in range(15):
            for c in range(d):
                up, down = [[Q, K, V][m].copy() for m in range(3)], [[Q, K, V][m].copy() for m in range(3)]
                up[k][i, c] += 1e-5
                down[k][i, c] -= 1e-5
                diff = ((loops(*up) - loops(*down)) * dO).sum() / 2e-5
                assert abs(diff - g[name][i, c]) < 1e-8, (name, i, c)


def test_refusals(mx):
    st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, [300, 20])], 64)
    M = 1 << 20
    tab, q, k, v, o, do, sv, dq, dk, dv, ws = (i * M for i in range(1, 12))
    W = 2 * 64

    def fwd(window=40, sinks=4, d=64, ld=W, q=q, o=o, dtype=0, scale=0.0, kv=None):
        mx.mux_attn_window_forward(mx.AttnDesc(2, d, ld, ld, ld, ld, scale, kv, dtype), window, sinks, st, tab, q, k, v, o, sv)

    def bwd(window=40, sinks=4, ws=ws, short=0, dk=dk):
        desc = mx.AttnDesc(2, 64, W, W, W, W)
        n = mx.mux_attn_window_workspace_bytes(desc, window, sinks, st)
        mx.mux_attn_window_backward(desc, window, sinks, st, tab, q, k, v, o, do, sv, dq, dk, dv, ws, n - short)

    for status, call, kw in [(1, fwd, dict(window=0)), (1, fwd, dict(window=-3)), (1, fwd, dict(sinks=-1)), (3, fwd, dict(sinks=65)),
                             (3, fwd, dict(d=72, ld=144)), (3, fwd, dict(dtype=1)), (3, fwd, dict(ld=W + 4)), (2, fwd, dict(ld=W - 8)),
                             (1, fwd, dict(q=None)), (3, fwd, dict(o=o + 8)), (1, fwd, dict(scale=-1.0)), (1, fwd, dict(kv=3)),
                             (1, bwd, dict(window=0)), (3, bwd, dict(sinks=65)), (4, bwd, dict(short=1)), (1, bwd, dict(ws=None)),
                             (3, bwd, dict(ws=ws + 8)), (1, bwd, dict(dk=None))]:
        with pytest.raises(mx.MuxError) as e:
            call(**kw)
        assert e.value.status == status, (kw, str(e.value))
    desc = mx.AttnDesc(2, 64, W, W, W, W)
    base = mx.mux_attn_workspace_bytes(desc, st)
    size = lambda w, z: mx.mux_attn_window_workspace_bytes(desc, w, z, st)                       # noqa: E731
    assert size(300, 4) == base <= size(40, 0) <= size(200, 64) and size(40, 0) < size(40, 4) < size(40, 64) and size(0, 4) == 0 and size(4, 65) == 0


def test_launches_that_would_not_fit(mx):
    """A launch is held to 2^32 threads: what would take more is refused before anything runs."""
    M = 1 << 40
    st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, [1] * 65536 + [300])], 256)
    desc = lambda h, kv: mx.AttnDesc(h, 64, h * 64, kv * 64, kv * 64, h * 64, 0.0, kv)                               # noqa: E731
    for h, kv in ((256, 1), (128, 128)):
        with pytest.raises(mx.MuxError) as e:
            mx.mux_attn_window_forward(desc(h, kv), 40, 4, st, M, 2 * M, 3 * M, 4 * M, 5 * M, 6 * M)
        assert e.value.status == 2 and "too many" in str(e.value)
        with pytest.raises(mx.MuxError) as e:
            mx.mux_attn_window_backward(desc(h, kv), 40, 4, st, M, 2 * M, 3 * M, 4 * M, 5 * M, 6 * M, 7 * M, 8 * M, 9 * M, 10 * M, 11 * M, M)
        assert e.value.status == 2 and "too many" in str(e.value)


def test_workspace_where_keys_are_few(mx):
    """The partial sums of dK, dV are bounded, however long the walk."""
    for lens, h, kv, w, z in (([2048], 32, 4, 1024, 4), ([16384, 9001], 16, 4, 2048, 16), ([1 << 20], 64, 1, 1 << 19, 64), ([64, 300], 4, 1, 64, 0)):
        st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, lens)], 256)
        desc = mx.AttnDesc(h, 128, h * 128, kv * 128, kv * 128, h * 128, 0.0, kv)
        size, base = mx.mux_attn_window_workspace_bytes(desc, w, z, st), mx.mux_attn_workspace_bytes(desc, st)
        sinks = 2 * sum(-(-n // 512) for n in lens) * kv * z * 128 * 4 * (16 + 256)
        assert base < size <= base + (1024 << 17) + sinks + 1024
