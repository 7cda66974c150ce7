"""8-bit experts on the GPU against the definition in 64 bits (fp8_ref.py) and the oracle's router.

Tolerance of an expert output y_j = sum_k h_k D_jk, h rounded to e4m3 from fp32: the kernel's h differs from the 64-bit one by the
matrix instruction's additions (about 1e-4 of the root mean square of the sums at worst), so an h_k that lies that close to the middle
of two e4m3 values may be rounded to the other one: a step of at most 2^-3 |h_k|.  The steps are no wider than 2^-3 of the value, so
a share of at most 2 * 2e-4 / 2^-4 < 1 % of the h_k is that close, and at most 8 + I / 64 of a row are allowed to be, each at its
worst: (8 + I / 64) 2^-3 max|h| max|D|.  bf16 outputs add half a step, 2^-8 |y|.  By norms: 2^-8, and 2^-3 sqrt(0.01) for the
flips, 1.7e-2 together.  Between the whole layer's kernels outputs keep 11 bits, and its gates are fp32: 2^-11 of every term.
"""
import numpy as np
import pytest
import torch

import fp8_ref as ref
from oracle import harness, zeda_oracle as orc
from paper_2605_18643_amd import synth, zeda
from paper_2605_18643_amd.stack import EPS, MoeStack

pytestmark = pytest.mark.gpu

SPECIAL = [0.0, -0.0, 448.0, -448.0, 449.0, 464.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 1e-38, 3e38, 1e30, np.inf, -np.inf, np.nan]


def _cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows, cols", [(1, 8), (3, 128), (5, 136), (17, 448), (64, 2048), (300, 1152)])
def test_quantized_rows_bit_for_bit(rows, cols, dtype):
    g = np.random.default_rng(rows * 10000 + cols)
    x = g.standard_normal((rows, cols)) * 2.0 ** g.integers(-140, 120, (rows, 1))
    x[g.random((rows, cols)) < 0.1] = 0.0
    x.ravel()[: len(SPECIAL)] = SPECIAL[: x.size]
    x[-1] = 0.0
    t = _cuda(x.astype(np.float32), dtype)
    q, s = zeda.zeda_quantize_rows_fp8(t)
    wq, ws = ref.quantize(t.double().cpu().numpy())
    assert np.array_equal(s.cpu().numpy(), ws)
    got = q.view(torch.uint8).cpu().numpy()
    nan = (wq & 127) == 127
    assert np.array_equal((got & 127) == 127, nan) and np.array_equal(got[~nan], wq[~nan])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("count, rows, cols", [(1, 1, 8), (2, 128, 128), (3, 130, 136), (2, 448, 1152), (1, 64, 200)])
def test_quantized_weights_bit_for_bit(count, rows, cols, dtype):
    g = np.random.default_rng(rows)
    w = g.standard_normal((count, rows, cols)) * 2.0 ** g.integers(-100, 100, (count, 1, 1))
    w.ravel()[: len(SPECIAL)] = SPECIAL[: w.size]
    t = _cuda(w.astype(np.float32), dtype)
    q, s = zeda.zeda_quantize_weights_fp8(t)
    for i in range(count):
        wq, ws = ref.quantize(t[i].double().cpu().numpy(), 128)
        got = q[i].view(torch.uint8).cpu().numpy()
        nan = (wq & 127) == 127
        assert np.array_equal(s[i].cpu().numpy(), ws)
        assert np.array_equal((got & 127) == 127, nan) and np.array_equal(got[~nan], wq[~nan])


def _packed(m):
    """[rows, cols] bytes to units of 32 x 64: piece p of lane l = row l % 32, columns 32 p + 16 (l / 32) of the unit."""
    r, c = m.shape
    u = m.reshape(r // 32, 32, c // 64, 2, 2, 16)  # row block, row, column block, p, half, byte
    return u.transpose(0, 2, 3, 4, 1, 5).reshape(-1)


@pytest.mark.parametrize("N, H, I", [(1, 128, 64), (3, 256, 192), (2, 1152, 448)])
def test_packed_layout(N, H, I):
    g = np.random.default_rng(I)
    q = [g.integers(0, 256, s).astype(np.uint8) for s in ((N, I, H), (N, I, H), (N, H, I))]
    Ib, Hb, Ip = -(-I // 128), H // 128, -(-I // 128) * 128
    s = [g.integers(0, 255, v).astype(np.uint8) for v in ((N, Ib, Hb), (N, Ib, Hb), (N, Hb, Ib))]
    d = zeda.make_desc(0, H, I, N, 0, 1, "bf16")
    e = zeda.zeda_pack_expert_weights_fp8(d, *[_cuda(v) for p in zip(q, s) for v in p])
    gu, dn, sgu, sdn = [b.cpu().numpy() for b in e.buffers]
    up = [np.pad(m, ((0, 0), (0, Ip - I), (0, 0))).reshape(N, Ip // 16, 16, H) for m in q[:2]]
    want = np.concatenate([_packed(np.concatenate([up[0][n], up[1][n]], axis=1).reshape(2 * Ip, H)) for n in range(N)])
    assert np.array_equal(gu, want)
    assert np.array_equal(dn, np.concatenate([_packed(np.pad(q[2][n], ((0, 0), (0, Ip - I)))) for n in range(N)]))
    word = lambda n: -(-n // 4) * 4  # noqa: E731
    assert np.array_equal(sgu.reshape(N, Ib, 2, word(Hb))[..., :Hb], np.stack([s[0], s[1]], axis=2))
    assert np.array_equal(sdn.reshape(N, Hb, word(Ib))[..., :Ib], s[2])


def _layer(T, H, I, N, Z, K, seed=3, gate=zeda.GATE_TOPK_NORM, copy=False, x_std=1.0):
    w = synth.Workload("fp8", T=T, H=H, I=I, N=N, Z=Z, K=K, dtype="bf16", seed=seed, recipe="zero_bias" if Z else "plain", x_std=x_std, w_std=0.05,
                       wr_std=0.05, zero_bias=0.4 if Z else 0.0)
    return w, zeda.make_desc(T, H, I, N, Z, K, "bf16", gate, 0, zeda.EXPERT_COPY if copy else zeda.EXPERT_ZERO)


class Experts:
    def __init__(self, d, L):
        mats = [L[k].contiguous() for k in ("w_gate", "w_up", "w_down")]
        qs = [zeda.zeda_quantize_weights_fp8(m) for m in mats]
        self.packed = zeda.zeda_pack_expert_weights_fp8(d, *[t for p in qs for t in p])
        self.host = [[ref.dequantize(q[n].view(torch.uint8).cpu().numpy(), s[n].cpu().numpy(), 128) for n in range(d.N)] for q, s in qs]

    def rows(self, x, expert_of):
        """(outputs, elementwise tolerance before the rounding to bf16) of rows of x, each by its expert."""
        y, tol = np.zeros((len(x), self.host[2][0].shape[0])), np.zeros((len(x), 1))
        xq = ref.rounded(x)
        for e in np.unique(expert_of):
            r = expert_of == e
            g, u, d = (m[e] for m in self.host)
            y[r], h = ref.expert(xq[r], g, u, d)
            tol[r] = (8 + h.shape[1] / 64) * 2.0 ** -3 * np.abs(h).max(1, keepdims=True) * np.abs(d).max()
        return y, tol


def _dispatch(d, ids):
    off = torch.empty(d.N + 1, dtype=torch.int32, device="cuda")
    ss, sr = (torch.full((d.T * d.K,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    nr = torch.zeros(1, dtype=torch.int32, device="cuda")
    zeda.zeda_dispatch(d, ids, off, ss, sr, nr, torch.empty(max(16, zeda.dispatch_workspace_bytes(d)), dtype=torch.uint8, device="cuda"))
    return off, ss, sr, nr


def _close(got, want, tol, what):
    assert np.isfinite(got).all(), what
    worst = (np.abs(got - want) - (tol + 2.0 ** -8 * np.abs(want))).max()
    assert worst <= 0, f"{what}: {worst:.3e} past the tolerance"
    assert harness.rel_l2(got, want) <= 1.7e-2, what


# rows per expert: none, one, around the 16-, 32- and 128-row edges of the kernels' tiles; widths inside and at the 128-blocks
LOADS = [[1], [0, 1, 0], [15, 16, 17], [31, 32, 33, 0], [63, 64, 65], [127, 128, 129], [96, 97, 200, 1], [300, 2]]
WIDTHS = [(128, 64), (256, 128), (384, 192), (1152, 448), (2048, 768), (512, 1536)]


@pytest.mark.parametrize("loads", LOADS, ids=str)
@pytest.mark.parametrize("H, I", WIDTHS)
def test_expert_ffn_loads_and_widths(loads, H, I):
    N, T = len(loads) + 1, sum(loads) + 3
    print(f"loads {loads} H {H} I {I}", flush=True)
    w, d = _layer(T, H, I, N, 2, 1)
    L = {**dict(zip(("w_gate", "w_up", "w_down"), synth.draw_experts(w, "cuda"))), "x": synth.draw_tokens(w, "cuda")}
    ids = np.repeat(np.arange(N + 2), loads + [0, 2, 1])  # the last expert has none, three tokens are on zero experts
    ids = np.random.default_rng(H + I).permutation(ids).astype(np.int32).reshape(T, 1)
    off, ss, _, nr = _dispatch(d, _cuda(ids))
    R = int(nr.item())
    assert R == sum(loads)
    ex = Experts(d, L)
    y = torch.full((T, H), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((zeda.expert_ffn_workspace_bytes_fp8(d) + 256,), 0xa5, dtype=torch.uint8, device="cuda")
    zeda.zeda_expert_ffn_fp8(d, L["x"], ex.packed, off, ss, nr, y, ws[:-256])
    slots = ss[:R].cpu().numpy()
    want, tol = ex.rows(L["x"].double().cpu().numpy()[slots], ids[slots, 0])
    _close(y[:R].double().cpu().numpy(), want, tol, "y_slot")
    assert bool((y[R:] == 7.0).all()), "rows behind the last normal slot were written"
    assert bool((ws[-256:] == 0xa5).all()), "written past the workspace"


def _forward(d, L, packed, ws=None, stream=None):
    ws = torch.full((zeda.workspace_bytes_fp8(d),), 0x7f, dtype=torch.uint8, device="cuda") if ws is None else ws
    out = torch.full((d.T, d.H), float("nan"), dtype=torch.bfloat16, device="cuda")
    nr = torch.full((1,), -5, dtype=torch.int32, device="cuda")
    zeda.zeda_moe_forward_fp8(d, L["x"], L["w_router"], L["router_bias"], packed, out, nr, ws, stream=stream)
    return out, nr


def _reference(d, L, ex, gate, copy):
    x = L["x"].double().cpu().numpy()
    a = harness.to_arrays(L)
    ids, gates = orc.route(a["x"], a["w_router"], a["router_bias"], d.N, d.Z, d.K, gate)[:2]
    t, j = np.nonzero(ids < d.N)
    y, tol = ex.rows(x[t], ids[t, j])
    out, bound = np.zeros((d.T, d.H)), np.zeros((d.T, d.H))
    np.add.at(out, t, y * gates[t, j][:, None])
    np.add.at(bound, t, (tol + 2.0 ** -11 * np.abs(y)) * gates[t, j][:, None])
    if copy:
        out += (gates * (ids >= d.N)).sum(1, keepdims=True) * x
    return out, bound, ids


SHAPES = [(1, 256, 128, 8, 4, 2), (1, 2048, 768, 12, 4, 8), (3, 256, 64, 4, 0, 4), (16, 512, 192, 20, 8, 6), (17, 1152, 448, 24, 8, 3), (64, 2048, 768, 40, 12, 8),
          (130, 384, 320, 3, 2, 2), (301, 1152, 448, 24, 8, 3), (700, 256, 128, 6, 2, 4), (2000, 128, 64, 2, 1, 1)]


@pytest.mark.parametrize("T, H, I, N, Z, K", SHAPES)
@pytest.mark.parametrize("gate, copy", [(zeda.GATE_TOPK_NORM, False), (zeda.GATE_SOFTMAX, True), (zeda.GATE_REAL_RENORM, False)])
def test_whole_layer(T, H, I, N, Z, K, gate, copy):
    print(T, H, I, N, Z, K, gate, copy, flush=True)
    w, d = _layer(T, H, I, N, Z, K, gate=gate, copy=copy)
    L = harness.gapped_layer(w, "cuda")
    ex = Experts(d, L)
    out, nr = _forward(d, L, ex.packed)
    want, tol, ids = _reference(d, L, ex, gate, copy)
    assert int(nr.item()) == int((ids < N).sum())
    got = out.double().cpu().numpy()
    _close(got, want, tol, "out")
    assert copy or not got[(ids >= N).all(1)].any(), "tokens without an expert are zero"


def test_no_token_and_no_normal_slot():
    w, d = _layer(40, 256, 128, 4, 4, 2)
    L = harness.gapped_layer(w, "cuda")
    ex = Experts(d, L)
    d0 = zeda.make_desc(0, 256, 128, 4, 4, 2, "bf16")
    nr = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    out = torch.full((1, 256), 3.0, dtype=torch.bfloat16, device="cuda")
    zeda.zeda_moe_forward_fp8(d0, L["x"], L["w_router"], L["router_bias"], ex.packed, out, nr, torch.empty(zeda.workspace_bytes_fp8(d0), dtype=torch.uint8, device="cuda"))
    assert int(nr.item()) == 0 and bool((out == 3.0).all())
    bias = L["router_bias"].clone()
    bias[4:] = 1e4  # every slot on a zero expert
    out, nr = _forward(d, dict(L, router_bias=bias), ex.packed)
    assert int(nr.item()) == 0 and not bool(out.any())
    bias[:4], bias[4:] = -float("inf"), 0.0  # and with the normal experts masked
    out, nr = _forward(d, dict(L, router_bias=bias), ex.packed)
    assert int(nr.item()) == 0 and not bool(out.any())


@pytest.mark.parametrize("T", [7, 200])
def test_bad_tokens_stay_by_themselves(T):
    w, d = _layer(T, 256, 128, 4, 2, 2)
    L = harness.gapped_layer(w, "cuda")
    ex = Experts(d, L)
    good, _ = _forward(d, L, ex.packed)
    x = L["x"].clone()
    x[2, 5], x[5, 200] = float("inf"), float("nan")
    # (their router logits are no numbers either: look at the expert stage, with the good tokens' routing)
    ids = torch.from_numpy(np.arange(2 * T, dtype=np.int32).reshape(T, 2) % 4).cuda()
    off, ss, sr, nr = _dispatch(d, ids)
    y = [torch.zeros(2 * T, 256, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ws = torch.empty(zeda.expert_ffn_workspace_bytes_fp8(d), dtype=torch.uint8, device="cuda")
    for t, o in ((L["x"], y[0]), (x, y[1])):
        zeda.zeda_expert_ffn_fp8(d, t, ex.packed, off, ss, nr, o, ws)
    bad = torch.isin(ss // 2, torch.tensor([2, 5], device="cuda"))
    assert bool(torch.isnan(y[1][bad]).all()) and torch.equal(y[0][~bad], y[1][~bad]) and bool(torch.isfinite(y[0]).all())
    out, _ = _forward(d, dict(L, x=x), ex.packed)
    keep = torch.ones(T, dtype=torch.bool)
    keep[[2, 5]] = False
    assert torch.equal(out.cpu()[keep], good.cpu()[keep])


@pytest.mark.parametrize("x_std, w_scale", [(1e-30, 1.0), (1e12, 1.0), (1.0, 2.0 ** -40), (1.0, 2.0 ** 30), (2.0 ** -100, 2.0 ** 50)])
@pytest.mark.parametrize("T", [5, 150])
def test_magnitudes(T, x_std, w_scale):
    """Scales far from one: the outputs are as near as at ordinary magnitudes, down to where fp32 ends."""
    w, d = _layer(T, 256, 128, 4, 2, 2)
    L = dict(harness.gapped_layer(w, "cuda"))
    ids = torch.from_numpy(np.arange(2 * T, dtype=np.int32).reshape(T, 2) % 4).cuda()
    off, ss, sr, nr = _dispatch(d, ids)
    gates = torch.rand(T, 2, device="cuda")
    L["x"] = (L["x"].float() * x_std).bfloat16()
    L["w_down"] = (L["w_down"].float() * w_scale).bfloat16()
    ex = Experts(d, L)
    y = torch.zeros(2 * T, 256, dtype=torch.bfloat16, device="cuda")
    zeda.zeda_expert_ffn_fp8(d, L["x"], ex.packed, off, ss, nr, y, torch.empty(zeda.expert_ffn_workspace_bytes_fp8(d), dtype=torch.uint8, device="cuda"))
    slots = ss.cpu().numpy()
    want, tol = ex.rows(L["x"].double().cpu().numpy()[slots // 2], ids.cpu().numpy().ravel()[slots])
    keep = np.abs(want) < 3e38
    got = np.where(keep, y.double().cpu().numpy(), 0.0)
    want = np.where(keep, want, 0.0)
    assert (np.abs(got - want) <= tol + 2.0 ** -8 * np.abs(want) + 2.0 ** -126).all()
    # the whole layer (scaled 16-bit expert outputs between the kernels): token 0's output is finite wherever the sums are
    out, _ = _forward(d, L, ex.packed)
    ref_out, bound, _ = _reference(d, L, ex, zeda.GATE_TOPK_NORM, False) if x_std <= 1.0 else (None, None, None)
    if ref_out is not None:
        err = np.abs(out.double().cpu().numpy() - ref_out)
        assert (err <= bound + 2.0 ** -8 * np.abs(ref_out) + 2.0 ** -126).all()


def test_the_same_bits_again_on_another_stream_and_in_a_graph():
    w, d = _layer(90, 512, 320, 12, 4, 4)
    L = harness.gapped_layer(w, "cuda")
    ex = Experts(d, L)
    first, n0 = _forward(d, L, ex.packed)
    again, _ = _forward(d, L, ex.packed)
    torch.cuda.synchronize()
    assert torch.equal(first, again)
    # two calls at once, each on a stream and a workspace of its own
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append(_forward(d, L, ex.packed))
    outs.append(_forward(d, L, ex.packed, stream=torch.cuda.current_stream()))
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) and int(n.item()) == int(n0.item()) for o, n in outs)
    # captured: replays on new inputs, with eager calls between them on the same buffers
    ws = torch.empty(zeda.workspace_bytes_fp8(d), dtype=torch.uint8, device="cuda")
    x, out, nr = L["x"].clone(), torch.empty_like(L["x"]), torch.zeros(1, dtype=torch.int32, device="cuda")
    x_res, xn = torch.zeros_like(x), torch.empty_like(x)

    def step():
        zeda.zeda_moe_forward_fp8(d, x, L["w_router"], L["router_bias"], ex.packed, out, nr, ws)
        zeda.zeda_moe_block_forward_fp8(d, x, x_res, L["w_router"], L["router_bias"], ex.packed, None, EPS, xn, nr, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        x.copy_(torch.randn(90, 512, generator=torch.Generator().manual_seed(rep)).bfloat16())
        x_res.fill_(0.5 * rep)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, x_res, xn, nr)]
        x_res.fill_(0.5 * rep)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, x_res, xn, nr)))
        (x.float() @ x.float().t()).sum().item()


@pytest.mark.parametrize("H, I", [(512, 256), (640, 384), (1024, 704), (2048, 768)])
def test_tiles_of_all_sizes_keep_their_bits_after_other_data(H, I):
    """Rows of one to four 32-row blocks per tile, and between the runs the same kernels on data whose every value is a NaN: what a workgroup
    finds in its shared memory must not reach the result."""
    loads = [1, 20, 40, 64, 70, 96, 100, 128, 5, 33, 129, 160] * 4
    if H == 512:  # enough work items for tiles of 160 rows
        loads += [161, 320, 2000] + [30000] * 7
    N, T = len(loads), sum(loads)
    w, d = _layer(T, H, I, N, 1, 1)
    qs = [zeda.zeda_quantize_weights_fp8(m.contiguous()) for m in synth.draw_experts(w, "cuda")]
    packed, x = zeda.zeda_pack_expert_weights_fp8(d, *[t for p in qs for t in p]), synth.draw_tokens(w, "cuda")
    ids = torch.tensor(np.repeat(np.arange(N), loads), dtype=torch.int32, device="cuda").view(T, 1)
    off, ss, _, nr = _dispatch(d, ids)
    bad = torch.full_like(x, float("nan"))
    ws = torch.empty(zeda.expert_ffn_workspace_bytes_fp8(d), dtype=torch.uint8, device="cuda")

    def run(rows):
        y = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
        zeda.zeda_expert_ffn_fp8(d, rows, packed, off, ss, nr, y, ws)
        return y

    first = run(x)
    assert torch.isfinite(first).all()
    for rep in range(12):
        assert torch.isnan(run(bad)).all()
        assert torch.equal(run(x), first), rep


def test_tiles_of_160_rows_give_what_tiles_of_128_give():
    """Twice the experts' rows from one call with many work items (other tiles) against calls with few."""
    loads = [159, 160, 161, 300, 128, 31, 0, 45]
    H, I, N, many = 256, 128, len(loads), 60000
    w, d = _layer(sum(loads), H, I, N + 1, 0, 1)
    big = zeda.make_desc(sum(loads) + 8 * many, H, I, N + 1, 0, 1, "bf16")
    assert big.T * 1 >= 128 * 3072
    qs = [zeda.zeda_quantize_weights_fp8(m.contiguous()) for m in synth.draw_experts(w, "cuda")]
    packed = zeda.zeda_pack_expert_weights_fp8(d, *[t for p in qs for t in p])
    x = torch.randn(big.T, H, device="cuda").bfloat16()
    outs = []
    for desc, extra in ((d, 0), (big, 8 * many)):
        ids = torch.tensor(np.repeat(np.arange(N + 1), loads + [extra]), dtype=torch.int32, device="cuda").view(desc.T, 1)
        off, ss, _, nr = _dispatch(desc, ids)
        y = torch.empty(desc.T, H, dtype=torch.bfloat16, device="cuda")
        zeda.zeda_expert_ffn_fp8(desc, x, packed, off, ss, nr, y, torch.empty(zeda.expert_ffn_workspace_bytes_fp8(desc), dtype=torch.uint8, device="cuda"))
        outs.append(y[: sum(loads)])
    torch.cuda.synchronize()
    assert torch.equal(*outs)


def test_token_rows_past_4_gib():
    """T * H >= 2^32: offsets of the quantised rows pass 32 bits; the last tokens against a call of their own."""
    H, I, N, T = 16384, 64, 3, (1 << 18) + 700
    x = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    last = 1500
    x[-last:] = torch.randn(last, H, device="cuda").bfloat16()
    w, d = _layer(last, H, I, N, 0, 1)
    qs = [zeda.zeda_quantize_weights_fp8(m.contiguous()) for m in synth.draw_experts(w, "cuda")]
    packed = zeda.zeda_pack_expert_weights_fp8(d, *[t for p in qs for t in p])
    ids = torch.tensor(np.arange(last) % N, dtype=torch.int32, device="cuda").view(last, 1)

    def run(T, x, ids):
        desc = zeda.make_desc(T, H, I, N, 0, 1, "bf16")
        off, ss, sr, nr = _dispatch(desc, ids)
        y = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
        zeda.zeda_expert_ffn_fp8(desc, x, packed, off, ss, nr, y, torch.empty(zeda.expert_ffn_workspace_bytes_fp8(desc), dtype=torch.uint8, device="cuda"))
        return y[sr.long()[-last:]]

    want = run(last, x[-last:].contiguous(), ids)
    got = run(T, x, torch.cat([torch.zeros(T - last, 1, dtype=torch.int32, device="cuda"), ids]))
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_slot_out_of_range_is_some_token():
    """Rows of one expert whose slots do not exist (few rows and a tile's worth): the other experts' rows are what they were."""
    for loads in ([3, 5], [300, 900, 1000, 700]):
        T, N = sum(loads), len(loads)
        w, d = _layer(T, 256, 192, N, 1, 1)
        qs = [zeda.zeda_quantize_weights_fp8(m.contiguous()) for m in synth.draw_experts(w, "cuda")]
        packed, x = zeda.zeda_pack_expert_weights_fp8(d, *[t for p in qs for t in p]), synth.draw_tokens(w, "cuda")
        off, ss, _, nr = _dispatch(d, torch.tensor(np.repeat(np.arange(N), loads), dtype=torch.int32, device="cuda").view(T, 1))
        ws = torch.empty(zeda.expert_ffn_workspace_bytes_fp8(d), dtype=torch.uint8, device="cuda")
        want, got = (torch.empty(T, 256, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        zeda.zeda_expert_ffn_fp8(d, x, packed, off, ss, nr, want, ws)
        ss[: loads[0]] = torch.tensor([2 ** 31 - 1, -(2 ** 31), T], dtype=torch.int32, device="cuda").repeat(loads[0] // 3)
        zeda.zeda_expert_ffn_fp8(d, x, packed, off, ss, nr, got, ws)
        torch.cuda.synchronize()
        assert torch.equal(got[loads[0]:], want[loads[0]:])


def test_stack_whose_workspace_is_smaller_than_the_bf16_layers():
    """The ids for the per-token counters lie where the 8-bit layout says; views by the bf16 layout would end past it."""
    w, d = _layer(3000, 128, 1024, 3, 3, 4)
    assert zeda.workspace_bytes_fp8(d) < zeda.workspace_layout(d).y_slot + 3000 * 4 * 128 * 2
    stack = MoeStack(w, 2, fp8=True)
    zero = torch.zeros(3000, dtype=torch.int32, device="cuda")
    stack.forward(synth.draw_tokens(w, "cuda"), token_zero=zero)
    torch.cuda.synchronize()
    assert int(zero.sum()) == 2 * 3000 * 4 - int(stack.num_real.sum())


@pytest.mark.parametrize("T", [1, 24, 333])
def test_residual_block_and_stack(T):
    w, d = _layer(T, 256, 192, 6, 3, 3)
    w = w.with_(K=3)
    x0 = synth.draw_tokens(w, "cuda")
    stack = MoeStack(w, 3, fp8=True)
    zero = torch.zeros(T, dtype=torch.int32, device="cuda")
    for fused in (True, False):
        y = stack.forward(x0.clone(), fused=fused, token_zero=zero)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(y).all()) and int(zero.sum()) == 3 * T * 3 - int(stack.num_real.sum())
    # one layer against its parts
    stack = MoeStack(w, 1, fp8=True)
    x = x0.clone()
    stack.forward(x)
    xn = torch.empty_like(x0)
    zeda.zeda_rmsnorm(x0, None, EPS, xn)
    p = stack.weights[0]
    out = torch.empty_like(x0)
    zeda.zeda_moe_forward_fp8(d, xn, p["w_router"], p["router_bias"], p["experts"], out, None, stack.ws)
    torch.cuda.synchronize()
    want = x0.double() + out.double()
    # the layer's output is rounded apart from the sum here: half a step of each
    tol = 2.0 ** -8 * (out.double().abs() + want.abs()) * 1.01
    assert bool(((x.double() - want).abs() <= tol).all())
    assert bool(((stack.forward(x0.clone(), fused=False).double() - want).abs() <= tol).all())
    twin = stack.static_twin()
    twin.forward(x0.clone())
    torch.cuda.synchronize()
    assert int(twin.num_real[0]) == T * 3
    with pytest.raises(ValueError):
        MoeStack(w, 1, tiled=True, fp8=True)
