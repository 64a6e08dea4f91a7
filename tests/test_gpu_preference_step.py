"""The operators of a preference step together, as a trainer runs them: per-task layer norm -> multiplexed q / k / v
projections -> attention in a sliding window -> multiplexed o projection and residual -> per-task layer norm -> multiplexed
output head -> preference loss, and the whole chain backwards, through the C ABI -- against the same chain built from the
oracles.  The reference's log-probabilities come from the same backbone with the adapters off.  What the GPU path stores in
bf16 between the stages is rounded at the same places in the oracle chain; every stage then adds its own error, of the size that
the single stages' tests allow: max |gpu - ref| <= 2e-2 max |ref| per tensor, as in the other chain's test."""
import numpy as np
import pytest

import mux_workloads as wlm
from oracle import attention as oatt
from oracle import norm as onorm
from oracle import pref as opref
from oracle import segtab
from tests import mux_harness as hz
from tests.test_gpu_attention import bf16_round

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_02885_amd as mx
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    mx.load_library()
    return mx, torch


def test_preference_step(env):
    import oracle
    mx, torch = env
    H, d, V, window, sinks, eps = 4, 64, 515, 40, 3, 1e-5
    C = H * d
    tasks = [wlm.Task(wlm.KIND_LORA, 16, 2.0, [100, 37]), wlm.Task(wlm.KIND_IA3, 0, 1.0, [70, 129, 64]),
             wlm.Task(wlm.KIND_LORA, 8, 1.0, [5, 200]), wlm.Task(wlm.KIND_ADAPTER, 8, 0.5, [64, 90])]
    pairs = [(0, 1, 0.1, 0.0), (2, 3, 0.2, 0.1), (2, 4, 0.2, 0.0), (6, 5, 0.1, 0.0), (7, 8, 0.1, 0.05)]
    VP = (V + 7) // 8 * 8                                  # the head's width in memory; its last columns are no vocabulary
    names = [("q", C, C), ("k", C, C), ("v", C, C), ("o", C, C), ("head", C, VP)]
    wl = wlm.Workload(name="pref", layers=names, tasks=tasks, chunk=64, sigma_w=0.06, sigma_ab=0.06)
    ot = segtab.build([t.seq_lens for t in tasks], wl.chunk)
    seqs = [(s[2], s[3]) for s in segtab.sequences(ot)]
    T, M, pad = ot.T, len(tasks), ot.row_task < 0
    kinds, ranks, scales = [t.kind for t in tasks], [t.rank for t in tasks], [t.scale for t in tasks]
    lts = [wlm.layer_tensors(wl, li, T, seed=60 + li, bf16=True) for li in range(5)]
    rng = np.random.default_rng(5)
    X = bf16_round(rng.standard_normal((T, C)))
    X[pad] = np.nan
    gam = [[bf16_round(1 + 0.2 * rng.standard_normal(C)) for _ in tasks] for _ in range(2)]
    bet = [[bf16_round(0.2 * rng.standard_normal(C)) for _ in tasks] for _ in range(2)]
    labels = rng.integers(0, V, T).astype(np.int32)
    labels[rng.random(T) < 0.4] = -1
    dloss = rng.uniform(0.1, 0.3, len(pairs)).astype(np.float32)

    # ---- oracle chain
    r = lambda a: bf16_round(a).astype(np.float64)                                                   # noqa: E731
    zero = lambda a: np.where(pad[:, None], 0.0, a)                                                  # noqa: E731

    def forward(off):
        ks = [wlm.KIND_NONE] * M if off else kinds
        none = [None] * M
        lay = lambda li, x: oracle.forward(x, lts[li].W, ot.row_task, ks, ranks, scales, none if off else lts[li].A,   # noqa: E731
                                           none if off else lts[li].B, none if off else lts[li].L)["Y"]
        n1 = r(onorm.forward(zero(X), ot.row_task, gam[0], bet[0], eps)["Y"])
        q, k, v = (r(lay(li, n1)) for li in range(3))
        o = r(oatt.forward(q, k, v, seqs, H, window=window, n_sinks=sinks)["O"])
        h = r(zero(X) + r(lay(3, o)))
        n2 = r(onorm.forward(h, ot.row_task, gam[1], bet[1], eps)["Y"])
        return n1, q, k, v, o, h, n2, r(lay(4, n2))

    ref_logp = opref.forward(forward(True)[-1][:, :V], labels, seqs, [], None)["logp"]
    n1, q, k, v, o, h, n2, logits = forward(False)
    want = opref.forward(logits[:, :V], labels, seqs, pairs, ref_logp)
    dlog = np.zeros((T, VP))
    dlog[:, :V] = r(opref.backward(logits[:, :V], labels, seqs, pairs, ref_logp, dloss))
    back = lambda li, x, g: oracle.backward(x, g, lts[li].W, ot.row_task, kinds, ranks, scales, lts[li].A, lts[li].B, lts[li].L)   # noqa: E731
    b4 = back(4, n2, dlog)
    bn2 = onorm.backward(h, r(b4["dX"]), ot.row_task, M, gam[1], eps)
    dh = r(bn2["dX"])
    b3 = back(3, o, dh)
    ba = oatt.backward(q, k, v, r(b3["dX"]), seqs, H, window=window, n_sinks=sinks)
    bq = [back(li, n1, r(ba[n])) for li, n in enumerate(("dQ", "dK", "dV"))]
    dn1 = r(sum(r(b["dX"]) for b in bq))
    bn1 = onorm.backward(zero(X), dn1, ot.row_task, M, gam[0], eps)

    # ---- the same chain through the library
    dev, bf, stream = "cuda:0", torch.bfloat16, torch.cuda.current_stream()
    up = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dev).to(bf).contiguous()   # noqa: E731
    scratch = lambda n: torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device=dev)              # noqa: E731
    buf = lambda w: torch.full((T, w), float("nan"), dtype=bf, device=dev)                           # noqa: E731
    f32 = lambda ts: [None if t is None else torch.full(t.shape, float("nan"), device=dev) for t in ts]                              # noqa: E731

    def table(descs):
        st = mx.mux_segtab_build(descs, wl.chunk, 0, 0)
        nb = mx.mux_segtab_device_bytes(st)
        dt = torch.zeros(nb, dtype=torch.uint8, device=dev)
        mx.mux_segtab_upload(st, dt, nb)
        torch.cuda.synchronize()
        return st, dt

    Xg = up(X)
    norms = [mx.NormDesc(C, mx.MUX_DT_BF16, [up(g) for g in gam[i]], [up(b) for b in bet[i]], eps) for i in range(2)]
    adesc = mx.AttnDesc(H, d, C, C, C, C)
    pdesc = mx.PrefDesc(V, mx.MUX_DT_BF16, VP, VP)
    lab = torch.from_numpy(labels).to(dev)
    ref = torch.full((len(seqs),), float("nan"), device=dev)

    def run(off):
        """The forward with the adapters on, or off as the reference runs it; returns what a backward needs."""
        descs = [mx.TaskDesc(0, 0, 1.0, t.seq_lens) for t in tasks] if off else hz.task_descs(mx, wl)
        st, dt = table(descs)
        s = {"st": st, "dt": dt, "layers": []}
        for li, (_, K, N) in enumerate(names):
            A, B, L = ([None] * M,) * 3 if off else ([up(a) for a in lts[li].A], [up(b) for b in lts[li].B], [up(x) for x in lts[li].L])
            desc = mx.LayerDesc(K, N, mx.MUX_DT_BF16, up(lts[li].W), M, A, B, L)
            wsb = mx.mux_lora_workspace_bytes(desc, st)
            s["layers"].append(dict(desc=desc, saved=scratch(mx.mux_lora_saved_bytes(desc, st)), wsb=wsb, ws=scratch(wsb), dA=f32(A), dB=f32(B), dL=f32(L)))
        lay = lambda li, x, y: mx.mux_lora_forward(s["layers"][li]["desc"], st, dt, x, y, s["layers"][li]["saved"],                   # noqa: E731
                                                   s["layers"][li]["ws"], s["layers"][li]["wsb"], stream)
        s["ns"] = [scratch(mx.mux_norm_saved_bytes(n, st)) for n in norms]
        s["n1"], s["q"], s["k"], s["v"], s["o"], s["y"], s["n2"], s["logits"] = (buf(w) for w in (C, C, C, C, C, C, C, VP))
        mx.mux_norm_forward(norms[0], st, dt, Xg, s["n1"], s["ns"][0], stream)
        for li, n in enumerate("qkv"):
            lay(li, s["n1"], s[n])
        s["lse"] = scratch(mx.mux_attn_saved_bytes(adesc, st))
        mx.mux_attn_window_forward(adesc, window, sinks, st, dt, s["q"], s["k"], s["v"], s["o"], s["lse"], stream)
        lay(3, s["o"], s["y"])
        s["h"] = torch.where(torch.from_numpy(pad).to(dev)[:, None], torch.zeros_like(Xg), Xg + s["y"])
        mx.mux_norm_forward(norms[1], st, dt, s["h"], s["n2"], s["ns"][1], stream)
        lay(4, s["n2"], s["logits"])
        use = [] if off else pairs
        s["layout"] = torch.from_numpy(mx.mux_pref_layout(st, use)).to(dev)
        s["psaved"] = scratch(mx.mux_pref_saved_bytes(pdesc, st, len(use)))
        wsb = mx.mux_pref_workspace_bytes(pdesc, st)
        s["loss"], s["logp"] = torch.empty(len(pairs), device=dev), ref if off else torch.empty(len(seqs), device=dev)
        mx.mux_pref_forward(pdesc, st, s["layout"], len(use), s["logits"], lab, None if off else ref, None, s["logp"],
                            None if off else s["loss"], s["psaved"], scratch(wsb), wsb, stream)
        return s

    run(True)
    s = run(False)
    st, dt, L = s["st"], s["dt"], s["layers"]
    logits_kept = s["logits"].clone()                      # (the gradient takes the logits' place)
    s["logits"][:, V:] = 0                                 # columns that are no vocabulary have no gradient
    mx.mux_pref_backward(pdesc, st, s["layout"], len(pairs), s["logits"], lab, s["psaved"], torch.from_numpy(dloss).to(dev), s["logits"], stream)

    def back_g(li, x, g):
        dx = buf(C)
        mx.mux_lora_backward(L[li]["desc"], st, dt, x, g, L[li]["saved"], dx, L[li]["dA"], L[li]["dB"], L[li]["dL"], 0, L[li]["ws"], L[li]["wsb"], stream)
        return dx

    wsb = mx.mux_norm_workspace_bytes(norms[0], st)
    nws = scratch(wsb)
    dg, db = [f32(norms[i]._keep[0]) for i in range(2)], [f32(norms[i]._keep[1]) for i in range(2)]
    dn2 = back_g(4, s["n2"], s["logits"])
    mx.mux_norm_backward(norms[1], st, dt, s["h"], dn2, s["ns"][1], dn2, dg[1], db[1], 0, nws, wsb, stream)
    do = back_g(3, s["o"], dn2)
    dq, dk, dv = buf(C), buf(C), buf(C)
    awsb = mx.mux_attn_window_workspace_bytes(adesc, window, sinks, st)
    mx.mux_attn_window_backward(adesc, window, sinks, st, dt, s["q"], s["k"], s["v"], s["o"], do, s["lse"], dq, dk, dv, scratch(awsb), awsb, stream)
    dxs = [back_g(li, s["n1"], g) for li, g in enumerate((dq, dk, dv))]
    dn1g = (dxs[0].float() + dxs[1].float() + dxs[2].float()).to(bf)
    dX = buf(C)
    mx.mux_norm_backward(norms[0], st, dt, Xg, dn1g, s["ns"][0], dX, dg[0], db[0], 0, nws, wsb, stream)
    torch.cuda.synchronize()

    # ---- compare
    f = lambda t: t.float().cpu().numpy().astype(np.float64)                                         # noqa: E731
    errs = {"ref": hz.norm_err(f(ref), ref_logp), "n1": hz.norm_err(f(s["n1"]), n1), "o": hz.norm_err(f(s["o"]), o), "h": hz.norm_err(f(s["h"]), h),
            "n2": hz.norm_err(f(s["n2"]), n2), "logits": hz.norm_err(f(logits_kept), logits), "logp": hz.norm_err(f(s["logp"]), want["logp"]),
            "loss": hz.norm_err(f(s["loss"]), want["loss"]), "dlogits": hz.norm_err(f(s["logits"]), dlog), "dh": hz.norm_err(f(dn2), dh),
            "dq": hz.norm_err(f(dq), ba["dQ"]), "dk": hz.norm_err(f(dk), ba["dK"]), "dv": hz.norm_err(f(dv), ba["dV"]), "dX": hz.norm_err(f(dX), bn1["dX"])}
    for i, b in enumerate((bn1, bn2)):
        for t in range(M):
            errs[f"dgamma[{i}][{t}]"] = hz.norm_err(f(dg[i][t]), b["dgamma"][t])
            errs[f"dbeta[{i}][{t}]"] = hz.norm_err(f(db[i][t]), b["dbeta"][t])
    for li, b in enumerate(bq + [b3, b4]):
        for name in ("dA", "dB", "dL"):
            for t, want_t in enumerate(b[name]):
                if want_t is not None:
                    errs[f"{name}[{li}][{t}]"] = hz.norm_err(f(L[li][name][t]), want_t)
    print({k: float(f"{e:.2e}") for k, e in errs.items()}, flush=True)
    bad = {k: e for k, e in errs.items() if not (e <= hz.TOL_BF16)}
    assert not bad, bad
