"""GPU parity of the windowed attention (include/mux_attn.h) against the fp64 oracle, through the C ABI.

Tolerances, derived element by element with h = 2^-8, half a step of bf16.  O: the probabilities are rounded to bf16 as operands of the
second product and O once, e_O = h (sum p |v| + |O|).  dV likewise, h (sum p |dO| + |dV|).  dS = p (dP - delta): delta is summed from
the stored O, so off by e_delta = sum |dO| e_O, and dS is rounded as an operand: dQ off by scale sum (h |dS| + p e_delta) |k| + h |dQ|, dK by
the same over the queries.  What fp32 adds (scores, exponentials, sums: below 2^-15 of the sums of magnitudes at these lengths and
values of a few units) is covered by 1 / 64 of h on every term, and by 2^-15 sum p |dP| in dS."""
import numpy as np
import pytest

from oracle import attention as oatt
from oracle import segtab

pytestmark = pytest.mark.gpu
H2 = 2.0 ** -8 * (1 + 1 / 64)


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_02885_amd as mx
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    mx.load_library()
    return mx, torch


def bounds(Q, K, V, dO, seqs, H, G, scale, window, sinks):
    """Values of the oracle's definition and how far each may be off."""
    d, group = Q.shape[1] // H, H // G
    val = {k: np.zeros_like(Q if k in ("O", "dQ") else K) for k in ("O", "dQ", "dK", "dV")}
    mag = {k: np.zeros_like(v) for k, v in val.items()}
    for first, n in seqs:
        r = slice(first, first + n)
        for h in range(H):
            c, ck = slice(h * d, (h + 1) * d), slice(h // group * d, (h // group + 1) * d)
            q, k, v, do = Q[r, c], K[r, ck], V[r, ck], dO[r, c]
            p, _ = oatt._probabilities(q, k, scale, window, sinks)
            o, dp = p @ v, do @ v.T
            e_o = H2 * (p @ np.abs(v) + np.abs(o))
            ds = p * (dp - (dp * p).sum(1, keepdims=True))
            e_ds = H2 * np.abs(ds) + p * ((np.abs(do) * e_o).sum(1, keepdims=True) + 2.0 ** -15 * (np.abs(do) @ np.abs(v).T))
            val["O"][r, c], mag["O"][r, c] = o, e_o
            val["dQ"][r, c], mag["dQ"][r, c] = scale * (ds @ k), scale * (e_ds @ np.abs(k))
            val["dK"][r, ck] += scale * (ds.T @ q)
            mag["dK"][r, ck] += scale * (e_ds.T @ np.abs(q))
            val["dV"][r, ck] += p.T @ do
            mag["dV"][r, ck] += H2 * (p.T @ np.abs(do))
    for k in ("dQ", "dK", "dV"):
        mag[k] += H2 * np.abs(val[k])
    return val, {k: v + 1e-30 for k, v in mag.items()}


class Call:
    def __init__(self, env, lens, chunk, H, window, sinks, seed=0, G=None, d=128, pack=0, flags=0, fused=False, sigma=1.0, scale=None):
        mx, torch = self.mx, self.torch = env
        G = H if G is None else G
        self.window, self.sinks, self.H, self.G, self.d = window, sinks, H, G, d
        self.ot = segtab.build(lens, chunk, pack, flags)
        self.seqs = [(s[2], s[3]) for s in segtab.sequences(self.ot)]
        T = self.T = self.ot.T
        pad = self.pad = self.ot.row_task < 0
        rng = np.random.default_rng(seed)
        self.st = mx.mux_segtab_build([mx.TaskDesc(0, 0, 1.0, v) for v in lens], chunk, pack, flags)
        nb = mx.mux_segtab_device_bytes(self.st)
        self.dtab = torch.zeros(nb, dtype=torch.uint8, device="cuda")
        mx.mux_segtab_upload(self.st, self.dtab, nb)
        torch.cuda.synchronize()
        widths = (H * d, G * d, G * d)
        bf = lambda w: torch.from_numpy((rng.standard_normal((T, w)) * sigma).astype(np.float32)).cuda().to(torch.bfloat16)   # noqa: E731
        nan = float("nan")
        if fused:
            self.q, self.k, self.v = torch.split(bf(sum(widths)), widths, dim=1)
            self.grads = torch.split(torch.full((T, sum(widths)), nan, dtype=torch.bfloat16, device="cuda"), widths, dim=1)
            ld = (sum(widths),) * 3
        else:
            self.q, self.k, self.v = (bf(w) for w in widths)
            self.grads = [torch.full((T, w), nan, dtype=torch.bfloat16, device="cuda") for w in widths]
            ld = widths
        self.do = bf(widths[0])
        for t in (self.q, self.k, self.v, self.do):
            t[torch.from_numpy(pad).cuda()] = nan if seed % 2 else 1e30
        self.scale = 1.0 / d ** 0.5 if scale is None else scale
        self.desc = mx.AttnDesc(H, d, ld[0], ld[1], ld[2], widths[0], scale or 0.0, G)
        self.o = torch.full((T, widths[0]), nan, dtype=torch.bfloat16, device="cuda")
        scratch = lambda b: torch.full((max(b, 256),), 0xFF, dtype=torch.uint8, device="cuda")                                 # noqa: E731
        self.saved = scratch(mx.mux_attn_saved_bytes(self.desc, self.st))
        self.wsb = mx.mux_attn_window_workspace_bytes(self.desc, window, sinks, self.st)
        self.ws = scratch(self.wsb)
        torch.cuda.synchronize()
        print(f"window case: T={T} H={H}/{G} d={d} window={window} sinks={sinks} longest={max(n for _, n in self.seqs)}", flush=True)

    def forward(self, saved=True):
        self.mx.mux_attn_window_forward(self.desc, self.window, self.sinks, self.st, self.dtab, self.q, self.k, self.v, self.o,
                                        self.saved if saved else None, self.torch.cuda.current_stream())

    def backward(self):
        self.mx.mux_attn_window_backward(self.desc, self.window, self.sinks, self.st, self.dtab, self.q, self.k, self.v, self.o, self.do,
                                         self.saved, *self.grads, self.ws, self.wsb, self.torch.cuda.current_stream())

    def both(self):
        self.forward()
        self.backward()
        self.torch.cuda.synchronize()
        return self

    def outputs(self):
        return [self.o, *self.grads]

    def check(self):
        host = lambda t: t.float().cpu().numpy().astype(np.float64)                                                            # noqa: E731
        clean = lambda t: np.where(self.pad[:, None], 0.0, host(t))                                                            # noqa: E731
        val, tol = bounds(clean(self.q), clean(self.k), clean(self.v), clean(self.do), self.seqs, self.H, self.G, self.scale, self.window, self.sinks)
        for name, t in zip(("O", "dQ", "dK", "dV"), self.outputs()):
            got = host(t)
            assert (got[self.pad] == 0).all(), name
            off = np.abs(got - val[name]) / tol[name]
            assert (off <= 1).all(), (name, float(np.nanmax(off)), np.argwhere(~(off <= 1))[:4].tolist())


SHORT = [[1, 2, 31, 32, 33], [63, 64, 65], [127, 128, 129], [200, 5], []]


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (32, 0), (48, 33), (64, 64), (100, 3)])
def test_around_every_boundary(env, window, sinks, d):
    """Lengths around waves, tiles and blocks, windows around the same; windows of the token alone; first tokens inside it."""
    Call(env, SHORT, 64, 2, window, sinks, seed=window + d, d=d).both().check()


@pytest.mark.parametrize("window,sinks", [(1, 5), (50, 4), (64, 1), (65, 0), (128, 40), (129, 64), (300, 16), (513, 4), (699, 2)])
def test_long_sequences(env, window, sinks):
    """Several blocks: tiles between the first tokens and the window are passed over; spans of far queries, whole and ragged."""
    Call(env, [[700], [300, 260], [1300]], 128, 2, window, sinks, seed=window).both().check()


@pytest.mark.parametrize("d,H,G", [(64, 4, 1), (80, 8, 2), (96, 3, 1), (128, 8, 8), (128, 6, 2)])
def test_heads(env, d, H, G):
    Call(env, [[600, 70], [129, 64, 30]], 64, H, 90, 5, seed=d + H, G=G, d=d, fused=True).both().check()
    Call(env, [[64] * 5, [128] * 3, [100]], 64, H, 20, 2, seed=d + H + 1, G=G, d=d).both().check()


@pytest.mark.parametrize("lens,H,G,d,window,sinks", [([[700], [650, 300]], 48, 48, 64, 90, 5), ([[2000]], 16, 1, 64, 1000, 4),
                                                     ([[1, 900, 3], [770]], 10, 2, 80, 333, 64), ([[1100], [300]], 5, 5, 128, 500, 0)])
def test_key_blocks_many_and_few(env, lens, H, G, d, window, sinks):
    """A workgroup a key block; sixteen that share one's walk over a large group; runs that end inside a head and a ragged last block."""
    Call(env, lens, 64, H, window, sinks, seed=window + H, G=G, d=d).both().check()


@pytest.mark.parametrize("chunk,pack,flags", [(1, 0, 0), (16, 500, 0), (64, 0, 1)])
def test_tables(env, chunk, pack, flags):
    Call(env, [[140, 700], [3], [90, 333]], chunk, 2, 77, 9, seed=3, pack=pack, flags=flags, d=64).both().check()


@pytest.mark.parametrize("seed,sigma,scale", [(4, 3.0, None), (5, 1.0, 0.3), (6, 0.05, None)])
def test_scores(env, seed, sigma, scale):
    """Nearly one-hot and nearly uniform rows; a scale of the caller's."""
    Call(env, [[500], [130, 40]], 64, 2, 100, 4, seed=seed, sigma=sigma, scale=scale, d=64).both().check()


def test_window_that_hides_nothing(env):
    """As long as the longest sequence: the bits of the attention without a window."""
    c = Call(env, SHORT + [[450]], 64, 2, 450, 3, seed=7)
    c.both()
    keep = [t.clone() for t in c.outputs()]
    for t in c.outputs():
        t.fill_(0)
    mx = c.mx
    mx.mux_attn_forward(c.desc, c.st, c.dtab, c.q, c.k, c.v, c.o, c.saved)
    mx.mux_attn_backward(c.desc, c.st, c.dtab, c.q, c.k, c.v, c.o, c.do, c.saved, *c.grads, c.ws, mx.mux_attn_workspace_bytes(c.desc, c.st))
    c.torch.cuda.synchronize()
    assert all(c.torch.equal(a, b) for a, b in zip(keep, c.outputs()))
    c.window = 2 ** 31 - 1
    c.both()
    assert all(c.torch.equal(a, b) for a, b in zip(keep, c.outputs()))


def test_hidden_keys_do_not_matter(env):
    """Keys and values that no later query sees: changing them changes nothing behind their window, bit for bit."""
    c = Call(env, [[600]], 64, 2, 70, 4, seed=8, d=64)
    c.both()
    o, dq = c.o.clone(), c.grads[0].clone()
    c.k[100:150] *= -37.0
    c.v[100:150] += 5.0
    c.both()
    assert c.torch.equal(c.o[220:600], o[220:600]) and c.torch.equal(c.grads[0][220:600], dq[220:600])
    assert not c.torch.equal(c.o[100:219], o[100:219]) and c.torch.equal(c.o[:100], o[:100])


def test_repeats_streams_and_capture(env):
    c = Call(env, [[1500], [64, 128], [260]], 128, 4, 200, 20, seed=9, G=2)
    c.both().check()
    keep = [t.clone() for t in c.outputs()]
    s = c.torch.cuda.Stream()
    for _ in range(2):
        for t in c.outputs():
            t.fill_(float("nan"))
        c.torch.cuda.synchronize()
        with c.torch.cuda.stream(s):
            c.both()
        assert all(c.torch.equal(a, b) for a, b in zip(keep, c.outputs()))
    graph = c.torch.cuda.CUDAGraph()
    with c.torch.cuda.graph(graph):
        c.forward()
        c.backward()
    for k in range(3):
        c.q.mul_(0.8)
        c.both()
        want = [t.clone() for t in c.outputs()]
        for t in c.outputs() + [c.ws, c.saved]:
            t.fill_(0)
        c.torch.cuda.synchronize()
        graph.replay()
        c.torch.cuda.synchronize()
        assert all(c.torch.equal(a, b) for a, b in zip(want, c.outputs())), k


def test_forward_alone(env):
    """Without `saved`, as an evaluation calls it."""
    c = Call(env, [[37], [1, 129], [700]], 64, 4, 100, 4, seed=10, G=2, fused=True)
    c.both().check()
    o = c.o.clone()
    c.o.fill_(float("nan"))
    c.forward(saved=False)
    c.torch.cuda.synchronize()
    assert c.torch.equal(c.o, o)


def test_rows_far_apart(env):
    """Offsets beyond 32 bits (all tensors columns of one buffer of 2^22 a row): the bits of the same rows side by side."""
    c = Call(env, [[600, 40], [300], [129]], 64, 4, 100, 5, seed=12, G=2, d=80).both()
    want = [t.clone() for t in c.outputs()]
    ld, at, far = 1 << 22, 0, []
    big = c.torch.empty((c.T, ld), dtype=c.torch.bfloat16, device="cuda")
    assert c.T * ld > 1 << 31
    for t in (c.q, c.k, c.v, c.do, *c.outputs()):
        v = big[:, at:at + t.shape[1]]
        v.copy_(t)
        far.append(v)
        at += t.shape[1] + 8
    c.q, c.k, c.v, c.do, c.o = far[:5]
    c.grads = far[5:]
    for t in c.outputs():
        t.fill_(float("nan"))
    c.desc = c.mx.AttnDesc(4, 80, ld, ld, ld, ld, 0.0, 2)
    c.both()
    assert all(c.torch.equal(a, b) for a, b in zip(want, c.outputs()))
