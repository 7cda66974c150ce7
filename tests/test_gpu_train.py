"""The router's training calls against their formulas in 64 bits, and those against differences.

u = 2^-24.  Where a reference starts from the fp32 probabilities and gates that the forward call left, they are exact inputs, and what is
left are the kernels' own roundings, each bounded by a few u of the sum of its terms' magnitudes; sums of n terms by n u of it.
"""
import numpy as np
import pytest
import torch

import fp8_ref
from oracle import harness, zeda_oracle as orc
from paper_2605_18643_amd import synth, zeda

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ALPHA, W = 0.25, 1.5
GATES = [zeda.GATE_SOFTMAX, zeda.GATE_TOPK_NORM, zeda.GATE_REAL_RENORM]


def _new(*shape, dtype=torch.float32, fill=None):
    t = torch.empty(*shape, dtype=dtype, device="cuda")
    return t if fill is None else t.fill_(fill)


def _np(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy().astype(np.int64)


def _workload(T, H, N, Z, K, dtype, seed=5):
    return synth.Workload("train", T=T, H=H, I=64, N=N, Z=Z, K=K, dtype=dtype, seed=seed, recipe="zero_bias" if Z else "plain", x_std=1.0, w_std=0.02,
                          wr_std=1.0 / np.sqrt(H), zero_bias=0.4 if Z else 0.0)


def _mask(T, kind):
    if kind == "none":
        return None
    m = np.ones(T, np.uint8) if kind == "all" else np.zeros(T, np.uint8) if kind == "nothing" else (np.random.default_rng(T).random(T) < 0.6).astype(np.uint8) * 7
    return torch.from_numpy(m).cuda()


class Forward:
    def __init__(self, w, L, gate, mask, ws_fill=0x7f):
        NE = w.N + w.Z
        self.w, self.L, self.mask, self.gate = w, L, mask, gate
        self.d = zeda.make_desc(w.T, w.H, w.I, w.N, w.Z, w.K, w.dtype, gate)
        self.ids, self.g, self.p = _new(w.T, w.K, dtype=torch.int32, fill=-3), _new(w.T, w.K, fill=np.nan), _new(w.T, NE, fill=np.nan)
        self.counts, self.P, self.summary = _new(NE, dtype=torch.int32, fill=-1), _new(NE, fill=np.nan), _new(7, fill=np.nan)
        self.ws = _new(zeda.route_train_workspace_bytes(self.d), dtype=torch.uint8, fill=ws_fill)
        self.run()

    def run(self, stream=None):
        zeda.zeda_route_train(self.d, self.L["x"], self.L["w_router"], self.L["router_bias"], self.mask, ALPHA, W, self.ids, self.g, self.p, self.counts,
                              self.P, self.summary, self.ws, stream=stream)

    def outputs(self):
        return self.ids, self.g, self.p, self.counts, self.P, self.summary


def _batch_sums(p, ids, on, N, K):
    n, NE = max(1, int(on.sum())), p.shape[1]
    counts = np.bincount(ids[on].ravel(), minlength=NE)
    f, P = counts / n, p[on].sum(0) / n
    fE, PE, fZ, PZ, Z = f[:N].sum(), P[:N].sum(), f[N:].sum(), P[N:].sum(), NE - N
    return counts, P, np.array([fE, PE, fZ, PZ, fZ / K, ALPHA * NE / K * (f * P).sum(),
                                ALPHA * (N + Z * W) / K * (fE * PE / N + (fZ * PZ / (Z * W) if Z else 0.0))])


SHAPES = [(1, 128, 8, 4, 2, "bf16"), (15, 256, 3, 0, 3, "bf16"), (16, 128, 20, 12, 6, "bf16"), (17, 384, 24, 8, 3, "bf16"), (64, 2048, 128, 32, 8, "bf16"),
          (65, 128, 1, 0, 1, "bf16"), (333, 512, 64, 32, 4, "bf16"), (1500, 256, 128, 64, 8, "bf16"), (130, 128, 250, 6, 16, "bf16"),
          (2, 64, 8, 4, 2, "f32"), (77, 260, 33, 7, 5, "f32"), (513, 1024, 32, 8, 4, "f32"), (40, 36, 200, 56, 16, "f32"), (5000, 128, 16, 8, 2, "bf16"),
          (8201, 128, 60, 4, 4, "bf16"), (8500, 128, 224, 32, 8, "bf16"), (4099, 256, 100, 28, 8, "bf16")]


@pytest.mark.parametrize("T, H, N, Z, K, dtype", SHAPES)
@pytest.mark.parametrize("masked", ["none", "some", "nothing"])
def test_forward(T, H, N, Z, K, dtype, masked):
    print(T, H, N, Z, K, dtype, masked, flush=True)
    w = _workload(T, H, N, Z, K, dtype)
    L = harness.gapped_layer(w, "cuda")
    a, mask = harness.to_arrays(L), _mask(T, masked)
    on = np.ones(T, bool) if mask is None else mask.cpu().numpy() != 0
    for gate in GATES:
        f = Forward(w, L, gate, mask)
        ids, gates, logits = orc.route(a["x"], a["w_router"], a["router_bias"], N, Z, K, gate, want_logits=True)
        assert np.array_equal(_np(f.ids), ids)
        # a logit is an fp32 sum of H products: about sqrt(H) u of its terms' root sum of squares, 4 sqrt(H) u max|logit| at most here;
        # probabilities and gates take its error as a relative one, twice, and a few u of exp, sum and division
        rel = 8 * np.sqrt(H) * U * max(1.0, np.abs(logits).max()) + 2e-6
        np.testing.assert_allclose(_np(f.g), gates, rtol=rel, atol=1e-30)
        e = np.exp(logits - logits.max(1, keepdims=True))
        p = e / e.sum(1, keepdims=True)
        np.testing.assert_allclose(_np(f.p), p, rtol=rel, atol=1e-30)
        counts, P, summary = _batch_sums(_np(f.p), ids, on, N, K)
        assert np.array_equal(_np(f.counts), counts)
        # sums of 16 in fp32, then 64 bits, rounded once
        np.testing.assert_allclose(_np(f.P), P, rtol=20 * U)
        np.testing.assert_allclose(_np(f.summary), summary, rtol=20 * U)
        if masked == "nothing":
            assert not bool(f.counts.any()) and not bool(f.P.any()) and not bool(f.summary.any())
    # the same experts and gates as the inference router, bit for bit
    ids2, g2 = torch.empty_like(f.ids), torch.empty_like(f.g)
    n = zeda.route_workspace_bytes(f.d)
    zeda.zeda_route(f.d, L["x"], L["w_router"], L["router_bias"], ids2, g2, _new(n, dtype=torch.uint8) if n else None)
    assert torch.equal(ids2, f.ids)
    # (its softmax denominators may be added in another order: a few u)
    np.testing.assert_allclose(_np(f.g), _np(g2), rtol=16 * U)
    if masked == "none":
        F, P2, s2 = zeda.zeda_routing_stats(f.d, L["x"], L["w_router"], L["router_bias"], alpha=ALPHA, w=W)
        np.testing.assert_allclose(_np(F), _np(f.counts) / T, rtol=4 * U)
        np.testing.assert_allclose(_np(P2), _np(f.P), rtol=(64 + T / 16) * U)
        np.testing.assert_allclose(_np(s2), _np(f.summary), rtol=(64 + T / 16) * U)


def test_no_token():
    w = _workload(0, 128, 6, 2, 2, "bf16")
    L = {"x": _new(1, 128, dtype=torch.bfloat16, fill=1.0), "w_router": _new(8, 128, dtype=torch.bfloat16, fill=1.0), "router_bias": None}
    f = Forward(w, L, zeda.GATE_TOPK_NORM, None)
    assert not bool(f.counts.any()) and not bool(f.P.any()) and not bool(f.summary.any())
    dw, db = _new(8, 128, fill=3.0), _new(8, fill=3.0)
    zeda.zeda_route_backward(f.d, L["x"], L["w_router"], _new(1, 8), _new(1, 2, dtype=torch.int32), _new(1, 2), None, f.counts, ALPHA, W, _new(2, fill=1.0), None,
                             None, dw, db, _new(zeda.route_backward_workspace_bytes(f.d), dtype=torch.uint8))
    assert not bool(dw.any()) and not bool(db.any())


def _slopes(counts, d_loss, N, Z, K, n):
    """n times the derivative of the losses by P."""
    f = counts / n
    return ALPHA / K * (d_loss[0] * (N + Z) * f + d_loss[1] * (N + Z * W) * np.concatenate([np.full(N, f[:N].sum() / N), np.full(Z, f[N:].sum() / max(Z * W, 1e-300))]))


def _logit_grad(p, ids, g, on, counts, d_loss, d_gates, N, gate):
    """(gradient of the logits, sum of the magnitudes that it is made of), token by token."""
    T, NE = p.shape
    K = ids.shape[1]
    n = max(1.0, counts.sum() / K)
    a = np.zeros(NE) if d_loss is None else _slopes(counts, d_loss, N, NE - N, K, n) / n
    a = a - a.mean()
    dl, mag = np.zeros((T, NE)), np.zeros((T, NE))
    for t in np.nonzero(on)[0]:
        u = np.abs(a).copy() * 0 + a
        extra, m = np.zeros(NE), np.zeros(NE)
        if d_gates is not None:
            s = ma = 0.0
            for j in range(K):
                if 0 <= ids[t, j] < NE:
                    s += g[t, j] * d_gates[t, j]
                    ma += abs(g[t, j] * d_gates[t, j])
            for j in range(K):
                e = ids[t, j]
                if not 0 <= e < NE:
                    continue
                if gate == zeda.GATE_SOFTMAX:
                    u[e] += d_gates[t, j]
                else:
                    within = gate == zeda.GATE_TOPK_NORM or e < N
                    extra[e] += g[t, j] * (d_gates[t, j] - (s if within else 0.0))
                    m[e] += g[t, j] * (abs(d_gates[t, j]) + ma)
        ub = np.abs(a) + np.abs(u - a)
        dl[t] = p[t] * (u - (p[t] * u).sum()) + extra
        mag[t] = p[t] * (ub + (p[t] * ub).sum()) + m
    return dl, mag


class Backward:
    def __init__(self, f, d_loss, d_gates, dx=True, dw=True, db=True):
        w, NE = f.w, f.w.N + f.w.Z
        self.f, self.d_loss, self.d_gates = f, d_loss, d_gates
        self.dx = torch.full_like(f.L["x"], float("nan")) if dx else None
        self.dw = _new(NE, w.H, fill=np.nan) if dw else None
        self.db = _new(NE, fill=np.nan) if db else None
        self.ws = _new(zeda.route_backward_workspace_bytes(f.d), dtype=torch.uint8, fill=0xff)
        self.run()

    def run(self, stream=None):
        f = self.f
        zeda.zeda_route_backward(f.d, f.L["x"], f.L["w_router"], f.p, f.ids, f.g, f.mask, f.counts, ALPHA, W, self.d_loss, self.d_gates, self.dx, self.dw,
                                 self.db, self.ws, stream=stream)

    def check(self):
        f, w = self.f, self.f.w
        on = np.ones(w.T, bool) if f.mask is None else f.mask.cpu().numpy() != 0
        d_loss = None if self.d_loss is None else _np(self.d_loss)
        d_gates = None if self.d_gates is None else _np(self.d_gates)
        p = np.where(on[:, None], _np(f.p), 0.0)
        dl, mag = _logit_grad(p, _np(f.ids), _np(f.g), on, _np(f.counts), d_loss, d_gates, w.N, f.gate)
        x, wr = np.where(on[:, None], _np(f.L["x"]), 0.0), _np(f.L["w_router"])
        NE = w.N + w.Z
        own = (NE + 2 * w.K + 16) * U * mag  # dl itself: sums over the pool and the slots
        if self.dx is not None:
            want, tol = dl @ wr, own @ np.abs(wr) + 1e-38
            # two bf16 parts leave 2^-15 of dl at most behind
            tol = tol + (2.0 ** -15 + NE * U) * (np.abs(dl) @ np.abs(wr)) + 2.0 ** -8 * np.abs(want) if w.dtype == "bf16" else tol + (NE + 2) * U * (np.abs(dl) @ np.abs(wr))
            got = _np(self.dx)
            assert (np.abs(got - want) <= tol).all(), "dx"
            assert not got[~on].any(), "dx of tokens that do not count"
        if self.dw is not None:
            want, tol = dl.T @ x, own.T @ np.abs(x) + (w.T + 8) * U * (np.abs(dl).T @ np.abs(x)) + 1e-38
            assert (np.abs(_np(self.dw) - want) <= tol).all(), "dw"
        if self.db is not None:
            assert (np.abs(_np(self.db) - dl.sum(0)) <= own.sum(0) + 4 * U * np.abs(dl).sum(0) + 1e-38).all(), "dbias"
        return dl


def _grads(f, seed=1):
    g = torch.Generator().manual_seed(seed)
    return torch.rand(2, generator=g).add_(0.5).cuda(), (torch.randn(f.w.T, f.w.K, generator=g) / f.w.T).cuda()


@pytest.mark.parametrize("T, H, N, Z, K, dtype", SHAPES)
@pytest.mark.parametrize("masked", ["none", "some", "nothing"])
def test_backward(T, H, N, Z, K, dtype, masked):
    print(T, H, N, Z, K, dtype, masked, flush=True)
    w = _workload(T, H, N, Z, K, dtype)
    L = harness.gapped_layer(w, "cuda")
    for gate in GATES:
        f = Forward(w, L, gate, _mask(T, masked))
        d_loss, d_gates = _grads(f)
        Backward(f, d_loss, d_gates).check()
    Backward(f, d_loss, None, dw=False, db=False).check()
    Backward(f, None, d_gates, dx=False, db=False).check()
    Backward(f, None, d_gates, dx=False, dw=False).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_that_do_not_count_may_hold_anything(dtype):
    T = 150
    w = _workload(T, 128, 12, 4, 3, dtype)
    L = dict(harness.gapped_layer(w, "cuda"))
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    mask[[0, 63, 64, 100, 149]] = 0
    for gate in GATES:
        f = Forward(w, L, gate, mask)
        d_loss, d_gates = _grads(f)
        clean = Backward(f, d_loss, d_gates)
        clean.check()
        x = L["x"].clone()
        x[0], x[63, 5], x[64], x[100, 127], x[149] = float("nan"), float("inf"), -float("inf"), float("nan"), 3e38
        g = Forward(w, dict(L, x=x), gate, mask)
        on = mask != 0
        assert all(torch.equal(a[on], b[on]) for a, b in zip(f.outputs()[:3], g.outputs()[:3]))
        assert all(torch.equal(a, b) for a, b in zip(f.outputs()[3:], g.outputs()[3:]))
        dg = d_gates.clone()
        dg[~on] = float("nan")
        b = Backward(g, d_loss, dg)
        assert torch.equal(b.dx, clean.dx) and torch.equal(b.dw, clean.dw) and torch.equal(b.db, clean.db)


def test_masked_experts_and_foreign_ids():
    """An expert whose bias is -inf has no probability and no gradient; ids outside the pool are left out; an id that a caller lists
    twice counts twice."""
    w = _workload(70, 128, 10, 4, 3, "bf16")
    L = dict(harness.gapped_layer(w, "cuda"))
    L["router_bias"] = L["router_bias"].clone()
    L["router_bias"][[2, 12]] = -float("inf")
    for gate in GATES:
        f = Forward(w, L, gate, _mask(70, "some"))
        assert not bool(f.p[:, [2, 12]].any()) and not bool(f.counts[[2, 12]].any()) and bool(torch.isfinite(f.p).all())
        d_loss, d_gates = _grads(f)
        b = Backward(f, d_loss, d_gates)
        b.check()
        assert not bool(b.dw[[2, 12]].any()) and not bool(b.db[[2, 12]].any())
        f.ids[3, 1], f.ids[4, 0], f.ids[5, 2] = 0x7fffffff, -1, 14
        f.ids[6, 1] = f.ids[6, 0]
        Backward(f, d_loss, d_gates).check()


def _total_loss(logits, ids, on, f_const, d_loss, d_gates, N, gate):
    """What is differentiated, as a function of the logits in 64 bits: sets and f are constants."""
    e = np.exp(logits - logits.max(1, keepdims=True))
    p = e / e.sum(1, keepdims=True)
    NE, K, n = p.shape[1], ids.shape[1], max(1, int(on.sum()))
    P, Z = p[on].sum(0) / n, p.shape[1] - N
    la = ALPHA * NE / K * (f_const * P).sum()
    lga = ALPHA * (N + Z * W) / K * (f_const[:N].sum() * P[:N].sum() / N + (f_const[N:].sum() * P[N:].sum() / (Z * W) if Z else 0.0))
    g = np.take_along_axis(p, ids, 1)
    if gate == zeda.GATE_TOPK_NORM:
        g = g / g.sum(1, keepdims=True)
    if gate == zeda.GATE_REAL_RENORM:
        den = np.where(ids < N, g, 0.0).sum(1, keepdims=True)
        g = np.where(den > 0, g / np.where(den > 0, den, 1.0), 0.0)
    return d_loss[0] * la + d_loss[1] * lga + (d_gates * g)[on].sum()


@pytest.mark.parametrize("gate", GATES)
def test_gradients_against_differences(gate):
    T, H, N, Z, K = 45, 128, 10, 6, 4
    w = _workload(T, H, N, Z, K, "f32")
    L = harness.gapped_layer(w, "cuda")
    mask = _mask(T, "some")
    f = Forward(w, L, gate, mask)
    d_loss, d_gates = _grads(f)
    b = Backward(f, d_loss, d_gates)
    x, wr, bias, ids, on = _np(L["x"]), _np(L["w_router"]), _np(L["router_bias"]), _np(f.ids), mask.cpu().numpy() != 0
    fc = _np(f.counts) / on.sum()
    loss = lambda x, wr, bias: _total_loss(x @ wr.T + bias, ids, on, fc, _np(d_loss), _np(d_gates), N, gate)  # noqa: E731
    g = np.random.default_rng(0)
    h = 1e-5
    for name, grad, at in (("x", b.dx, 0), ("w_router", b.dw, 1), ("bias", b.db, 2)):
        for _ in range(4):
            v = [x, wr, bias]
            r = g.standard_normal(v[at].shape)
            up, down = list(v), list(v)
            up[at], down[at] = v[at] + h * r, v[at] - h * r
            slope = (loss(*up) - loss(*down)) / (2 * h)
            got = (_np(grad) * r).sum()
            # the difference's own error: h^2 / 6 of the third derivative and 1e-16 / h of the loss, 1e-10 of it; the gradient: fp32
            scale = np.sqrt((_np(grad) ** 2).sum())
            assert abs(slope - got) <= 1e-5 * scale + 1e-9, (name, slope, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, H, N, Z, K", [(1, 128, 4, 2, 1), (33, 256, 6, 3, 5), (150, 1152, 10, 0, 3), (64, 2048, 20, 12, 16), (7, 8192, 3, 1, 2)])
@pytest.mark.parametrize("copy", [False, True])
def test_combine_backward(T, H, N, Z, K, dtype, copy):
    print(T, H, N, Z, K, dtype, copy, flush=True)
    g = torch.Generator().manual_seed(T)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    d = zeda.make_desc(T, H, 64, N, Z, K, dtype, free_expert=zeda.EXPERT_COPY if copy else zeda.EXPERT_ZERO)
    ids = torch.stack([torch.randperm(N + Z, generator=g)[:K] for _ in range(T)]).int().cuda()
    if T > 3:
        ids[1], ids[2, 0] = max(N, N + Z - 1), 0x7fffffff  # only free experts (if there are any); no expert
    off, ss, sr = (_new(n, dtype=torch.int32, fill=-9) for n in (N + 1, T * K, T * K))
    nr = _new(1, dtype=torch.int32)
    zeda.zeda_dispatch(d, ids, off, ss, sr, nr, _new(max(16, zeda.dispatch_workspace_bytes(d)), dtype=torch.uint8))
    R = int(nr.item())
    gates, y, d_out, x = (torch.randn(*s, generator=g).to(t).cuda() for s, t in (((T, K), torch.float32), ((T * K, H), dt), ((T, H), dt), ((T, H), dt)))
    y[R:] = float("nan")
    for want_dy, want_dx in ((True, copy), (False, False)):
        dg, dy, dx = _new(T, K, fill=np.nan), (_new(T * K, H, dtype=dt, fill=5.0) if want_dy else None), (_new(T, H, dtype=dt, fill=np.nan) if want_dx else None)
        zeda.zeda_combine_backward(d, d_out, y, ids, gates, sr, x if copy else None, dg, dy, dx)
        do, yy, gg, ii, rows = _np(d_out), _np(y), _np(gates), _np(ids), _np(sr).reshape(T, K)
        want, mag, wdy = np.zeros((T, K)), np.zeros((T, K)), np.full((T * K, H), 5.0)
        for t in range(T):
            for j in range(K):
                if rows[t, j] >= 0:
                    want[t, j], mag[t, j] = do[t] @ yy[rows[t, j]], np.abs(do[t]) @ np.abs(yy[rows[t, j]])
                    wdy[rows[t, j]] = gg[t, j] * do[t]
                elif copy and N <= ii[t, j] < N + Z:
                    want[t, j], mag[t, j] = do[t] @ _np(x)[t], np.abs(do[t]) @ np.abs(_np(x)[t])
        half = 2.0 ** -8 if dtype == "bf16" else U
        assert (np.abs(_np(dg) - want) <= (H / 64 + 16) * U * mag).all()
        if want_dy:
            assert (np.abs(_np(dy) - wdy) <= half * np.abs(wdy) * (1 + 2 * U)).all()
        if want_dx:
            gz = (gg * ((ii >= N) & (ii < N + Z))).sum(1, keepdims=True)
            size = (np.abs(gg) * ((ii >= N) & (ii < N + Z))).sum(1, keepdims=True)
            assert (np.abs(_np(dx) - gz * do) <= (half * np.abs(gz) + K * U * size) * np.abs(do) * (1 + 2 * half)).all()


def test_the_same_bits_again_on_another_stream_and_in_a_graph():
    w = _workload(200, 256, 24, 8, 4, "bf16")
    L = dict(harness.gapped_layer(w, "cuda"))
    L["x"] = L["x"].clone()
    f = Forward(w, L, zeda.GATE_TOPK_NORM, _mask(200, "some"))
    d_loss, d_gates = _grads(f)
    b = Backward(f, d_loss, d_gates)
    torch.cuda.synchronize()
    keep = [t.clone() for t in (*f.outputs(), b.dx, b.dw, b.db)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    f.run(stream=s)
    b.run(stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(keep, (*f.outputs(), b.dx, b.dw, b.db)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f.run()
        b.run()
    for rep in range(4):
        L["x"].copy_(torch.randn(200, 256, generator=torch.Generator().manual_seed(rep)).bfloat16())
        d_loss.fill_(0.5 + rep)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*f.outputs(), b.dx, b.dw, b.db)]
        f.run()
        b.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (*f.outputs(), b.dx, b.dw, b.db))), rep
        (L["x"].float() @ L["x"].float().t()).sum().item()


@pytest.mark.parametrize("gate, copy", [(zeda.GATE_TOPK_NORM, False), (zeda.GATE_SOFTMAX, True), (zeda.GATE_REAL_RENORM, False)])
def test_a_training_step_over_frozen_8_bit_experts(gate, copy):
    """Forward with experts in 8 bits, a loss <v, out> + balance losses, back to the router: against differences of that loss in 64 bits,
    the experts' outputs being constants."""
    T, H, I, N, Z, K = 160, 256, 192, 12, 4, 4
    w = synth.Workload("step", T=T, H=H, I=I, N=N, Z=Z, K=K, dtype="bf16", seed=8, recipe="zero_bias", x_std=1.0, w_std=0.08, wr_std=0.06, zero_bias=0.4)
    L = harness.gapped_layer(w, "cuda")
    mask = _mask(T, "some")
    f = Forward(w, L, gate, mask)
    d = f.d
    d.free_expert = zeda.EXPERT_COPY if copy else zeda.EXPERT_ZERO
    experts = zeda.zeda_pack_expert_weights_fp8(d, *[t for k in ("w_gate", "w_up", "w_down") for t in zeda.zeda_quantize_weights_fp8(L[k].contiguous())])
    off, ss, sr = (_new(n, dtype=torch.int32) for n in (N + 1, T * K, T * K))
    nr = _new(1, dtype=torch.int32)
    zeda.zeda_dispatch(d, f.ids, off, ss, sr, nr, _new(max(16, zeda.dispatch_workspace_bytes(d)), dtype=torch.uint8))
    y, out = _new(T * K, H, dtype=torch.bfloat16, fill=0.0), _new(T, H, dtype=torch.bfloat16)
    zeda.zeda_expert_ffn_fp8(d, L["x"], experts, off, ss, nr, y, _new(zeda.expert_ffn_workspace_bytes_fp8(d), dtype=torch.uint8))
    zeda.zeda_combine(d, y, f.ids, f.g, sr, out, x=L["x"] if copy else None)
    v = (torch.randn(T, H, generator=torch.Generator().manual_seed(2)) / T).bfloat16().cuda()
    v[mask == 0] = 0.0
    d_gates, dx_copy = _new(T, K), _new(T, H, dtype=torch.bfloat16) if copy else None
    zeda.zeda_combine_backward(d, v, y, f.ids, f.g, sr, L["x"] if copy else None, d_gates, None, dx_copy)
    d_loss = torch.tensor([0.7, 1.3], device="cuda")
    b = Backward(f, d_loss, d_gates)
    b.check()
    # the loss in 64 bits as a function of the router
    rows, ids, on = _np(sr).reshape(T, K), _np(f.ids), mask.cpu().numpy() != 0
    yy = np.where((rows >= 0)[..., None], _np(y)[np.maximum(rows, 0)], 0.0)
    x, wr, bias = _np(L["x"]), _np(L["w_router"]), _np(L["router_bias"])
    if copy:
        yy = np.where((ids >= N)[..., None], x[:, None, :], yy)
    slot = np.einsum("th,tkh->tk", _np(v), yy)
    fc = _np(f.counts) / on.sum()
    loss = lambda wr, bias: _total_loss(x @ wr.T + bias, ids, on, fc, _np(d_loss), slot, N, gate)  # noqa: E731
    # the kernels' combine is that sum, rounded once
    e = np.exp(x @ wr.T + bias)
    p = e / e.sum(1, keepdims=True)
    got, want = _np(out), np.einsum("tk,tkh->th", _np(f.g), yy)
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 32 * U * np.einsum("tk,tkh->th", _np(f.g), np.abs(yy))).all() and np.isfinite(p).all()
    g, h = np.random.default_rng(1), 1e-5
    for _ in range(4):
        r, q = g.standard_normal(wr.shape), g.standard_normal(bias.shape)
        slope = (loss(wr + h * r, bias + h * q) - loss(wr - h * r, bias - h * q)) / (2 * h)
        grad = (_np(b.dw) * r).sum() + (_np(b.db) * q).sum()
        # differences 1e-9 of the loss; gates and probabilities come from fp32 logits (sqrt(H) u each, some 1e-5 of a gradient)
        assert abs(slope - grad) <= 1e-4 * np.sqrt((_np(b.dw) ** 2).sum()) + 1e-8
    assert fp8_ref.TABLE[126] == 448.0
