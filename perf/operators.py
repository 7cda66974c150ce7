"""Performance cases of the layer's 8-bit experts and of the router's training operators.

Four kinds of call:
  layer     one zeda_moe_forward_fp8: the whole layer with expert weights in 8-bit floating point, a power-of-two scale for every
            block of 128 (serving)
  route     one zeda_route_train: ids, gates, probabilities, per-expert counts and the balance losses of a training batch
  backward  one zeda_route_backward: gradients of the balance losses and of the gates, down to x, w_router and router_bias
  combine   one zeda_combine_backward: gradients of the gates and of the expert outputs from the layer output's gradient

A case is a dict of plain values.  With `own` the calls are the library's, without it elementary torch operations in 32 bits.
Layer shapes are those of the package's own configurations and tests: H=2048, I=768, N=128, K=8 with 32 zero experts; H=2048,
I=1536, N=64, K=4 with 32; and small layers whose widths are not multiples of the large tiles.
"""
from __future__ import annotations

import math

import torch

own = False

WIDE = dict(H=2048, I=768, N=128, Z=32, K=8)
WIDE64 = dict(H=2048, I=768, N=128, Z=64, K=8)
FEW = dict(H=2048, I=1536, N=64, Z=32, K=4)
# bias on every zero expert's logit that puts about half of the slots on zero experts (logits of standard deviation 0.905)
ZERO_BIAS = {(128, 32, 8): 0.6468, (128, 64, 8): 0.2991, (64, 32, 4): 0.3092}
LOGIT_STD = 0.905
MIN_GAP = 1e-4  # between a token's neighbouring top logits: sums in any order then select the same experts in the same order
GATES = ("softmax", "topk_norm", "real_renorm")
ALPHA, GROUP_W = 0.01, 2.0


def listed():
    layer = lambda name, T, shape, **kw: dict(name=name, kind="layer", T=T, gate="topk_norm", copy=False, skew=0.0, dtype="bf16", **shape) | kw  # noqa: E731
    train = lambda kind, name, T, shape, **kw: dict(name=name, kind=kind, T=T, gate="topk_norm", padded=True, dtype="bf16", **shape) | kw  # noqa: E731
    return [
        # decode of one sequence: the smallest serving call, a few experts' weights
        layer("layer_1", 1, WIDE),
        # decode at concurrency 64: streams nearly every expert's weights
        layer("layer_64", 64, WIDE),
        # small model whose widths end inside the 128-blocks, copy experts, weights renormalised over the normal experts
        layer("layer_301_ragged", 301, dict(H=1152, I=448, N=24, Z=8, K=3), gate="real_renorm", copy=True),
        # a prefill chunk of odd length, wide experts
        layer("layer_997_few", 997, FEW, gate="softmax"),
        # prefill of 4096 tokens
        layer("layer_4096", 4096, WIDE),
        # a long prefill with uneven expert popularity: loads from a handful to thousands of rows
        layer("layer_16381_skewed", 16381, WIDE, skew=1.0),
        # a small fp32 training batch, packed without padding
        train("route", "route_513_f32", 513, dict(H=1024, I=512, N=32, Z=8, K=4), dtype="f32", padded=False),
        # a training batch of 8192 tokens with padding
        train("route", "route_8192", 8192, WIDE),
        # the second router's batch of odd length, gates as plain softmax
        train("backward", "backward_997_few", 997, FEW, gate="softmax"),
        # a training batch of 8192 tokens with padding
        train("backward", "backward_8192", 8192, WIDE),
        # the small fp32 batch
        train("combine", "combine_513_f32", 513, dict(H=1024, I=512, N=32, Z=8, K=4), dtype="f32", padded=False),
        # a training batch of 4096 tokens
        train("combine", "combine_4096", 4096, WIDE, padded=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _small(rng):
    N = rng.randint(8, 48)
    return dict(H=128 * rng.randint(2, 12), I=64 * rng.randint(2, 12), N=N, Z=rng.randint(0, 16), K=rng.randint(1, 6))


def draw(rng):
    kind = rng.choice(["layer", "layer", "layer", "route", "backward", "combine"])
    small = rng.random() < 0.4
    shape = _small(rng) if small else dict(rng.choice([WIDE, WIDE64, FEW]))
    c = dict(kind=kind, gate=rng.choice(GATES), **shape)
    if kind == "layer":
        return dict(c, T=_log_int(rng, 1, 12288), copy=rng.random() < 0.3, skew=rng.choice([0.0, 0.0, 0.5, 1.0]), dtype="bf16")
    dtype = rng.choice(["bf16", "bf16", "f32"])
    return dict(c, T=_log_int(rng, 1, 4096 if dtype == "f32" or kind == "combine" else 8192), padded=rng.random() < 0.6, dtype=dtype)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    """Tokens and router; only tokens whose K + 1 largest logits are MIN_GAP apart are taken (and one alone has work to do)."""
    T, H, N, Z, K = (case[k] for k in ("T", "H", "N", "Z", "K"))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    wr = (torch.randn(N + Z, H, generator=g, device="cuda") * (LOGIT_STD / math.sqrt(H))).to(_dt(case))
    bias = torch.zeros(N + Z, device="cuda")
    bias[:N] = torch.randn(N, generator=g, device="cuda") * case.get("skew", 0.0)
    bias[N:] = ZERO_BIAS.get((N, Z, K), 0.4) + case.get("skew", 0.0)
    x = torch.randn(T + T // 8 + 128, H, generator=g, device="cuda").to(_dt(case))
    top = torch.sort(x.double() @ wr.double().t() + bias.double(), dim=1, descending=True)
    ok = (top.values[:, :-1] - top.values[:, 1:])[:, :K].min(1).values > MIN_GAP
    if T == 1:
        ok &= (top.indices[:, :K] < N).any(1)
    x = x[torch.nonzero(ok).view(-1)[:T]].contiguous()
    return {"x": x, "w_router": wr, "router_bias": bias}, g


def _mask(case, g):
    """Sequences of a few lengths, padded behind their ends: 1 for a token that counts."""
    T = case["T"]
    if not case["padded"]:
        return None
    length = max(1, T // 8)
    valid = (torch.rand(T // length + 1, generator=g, device="cuda") * 0.6 + 0.4) * length
    t = torch.arange(T, device="cuda")
    return ((t % length) < valid[t // length]).to(torch.uint8)


def _blocks_scaled(w):
    """[N, F, D] -> e4m3 values and the bytes of the scales 2^(s - 127) of their blocks of 128 x 128: the least power of two that
    keeps a block's largest value within 448."""
    N, F, D = w.shape
    p = torch.nn.functional.pad(w, (0, -D % 128, 0, -F % 128)).view(N, -(-F // 128), 128, -(-D // 128), 128)
    m, e = torch.frexp(p.abs().amax((2, 4)))
    s = (e - 9 + (m > 0.875)).clamp(-126, 127)
    q = torch.ldexp(p, -s[:, :, None, :, None]).view(N, -(-F // 128) * 128, -1)[:, :F, :D].contiguous().to(torch.float8_e4m3fn)
    return q, (s + 127).to(torch.uint8)


def _desc(case):
    from paper_2605_18643_amd import zeda

    gate = {"softmax": zeda.GATE_SOFTMAX, "topk_norm": zeda.GATE_TOPK_NORM, "real_renorm": zeda.GATE_REAL_RENORM}[case["gate"]]
    return zeda.make_desc(case["T"], case["H"], case["I"], case["N"], case["Z"], case["K"], case["dtype"], gate, zeda.WEIGHTS_ROW_MAJOR,
                          zeda.EXPERT_COPY if case.get("copy") else zeda.EXPERT_ZERO)


def _prepare_layer(case, seed):
    st, g = _inputs(case, seed)
    H, I, N = case["H"], case["I"], case["N"]
    draw = lambda F, D, std: _blocks_scaled(torch.randn(N, F, D, generator=g, device="cuda") * std)  # noqa: E731
    for name, F, D, std in (("gate", I, H, LOGIT_STD / math.sqrt(H)), ("up", I, H, LOGIT_STD / math.sqrt(H)), ("down", H, I, 0.55 / math.sqrt(I))):
        st["q_" + name], st["s_" + name] = draw(F, D, std)
    if own:  # packed once, when the weights are loaded
        from paper_2605_18643_amd import zeda

        st["desc"] = _desc(case)
        names = ("q_gate", "s_gate", "q_up", "s_up", "q_down", "s_down")
        st["experts"] = zeda.zeda_pack_expert_weights_fp8(st["desc"], *[st.pop(n) for n in names])
        st["ws"] = torch.empty(zeda.workspace_bytes_fp8(st["desc"]), dtype=torch.uint8, device="cuda")
        st["out"] = torch.empty_like(st["x"])
        st["num_real"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return st


def prepare(case, seed):
    kind, T, H, N, NE, K = case["kind"], case["T"], case["H"], case["N"], case["N"] + case["Z"], case["K"]
    if kind == "layer":
        return dict(_prepare_layer(case, seed), case=case)
    st, g = _inputs(case, seed)
    st.update(case=case, mask=_mask(case, g))
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if kind == "route":
        if own:
            from paper_2605_18643_amd import zeda

            st.update(desc=_desc(case), topk_ids=new(T, K, dtype=torch.int32), topk_gates=new(T, K), probs=new(T, NE),
                      counts=new(NE, dtype=torch.int32), mean_probs=new(NE), summary=new(7))
            st["ws"] = new(zeda.route_train_workspace_bytes(st["desc"]), dtype=torch.uint8)
        return st
    # the backward calls start from what the forward pass has left
    st.update(dict(zip(("topk_ids", "topk_gates", "probs", "counts"), _route(st))))
    if kind == "backward":
        st["d_loss"] = torch.rand(2, generator=g, device="cuda") + 0.5  # gradients of L_A and L_GA
        st["d_gates"] = torch.randn(T, K, generator=g, device="cuda") * (0.1 / T)
        if own:
            from paper_2605_18643_amd import zeda

            st.update(desc=_desc(case), dx=torch.empty_like(st["x"]), dw_router=new(NE, H), dbias=new(NE))
            st["ws"] = new(zeda.route_backward_workspace_bytes(st["desc"]), dtype=torch.uint8)
        return st
    real = (st["topk_ids"] < N).view(-1)
    order = torch.sort(torch.where(real, st["topk_ids"].view(-1), NE), stable=True).indices
    row = torch.empty_like(order)
    row[order] = torch.arange(T * K, device="cuda")
    st["slot_to_row"] = torch.where(real, row, -1).to(torch.int32)
    st["y_slot"] = torch.randn(T * K, H, generator=g, device="cuda").to(_dt(case))
    st["d_out"] = (torch.randn(T, H, generator=g, device="cuda") / T).to(_dt(case))
    st["d_y_slot"] = torch.zeros(T * K, H, dtype=_dt(case), device="cuda")  # rows behind the last normal slot stay as they are
    if own:
        st.update(desc=_desc(case), d_gates=new(T, K))
    return st


# ---------------------------------------------------------------------------------------------------------------------
# the operators in their plain form
# ---------------------------------------------------------------------------------------------------------------------
def _select(logits, N, K, gate):
    """(ids, gates, probabilities): ties go to the lower index."""
    top = torch.sort(logits, dim=1, descending=True, stable=True)
    ids, p = top.indices[:, :K], torch.softmax(logits, dim=1)
    if gate == "softmax":
        return ids, p.gather(1, ids), p
    e = torch.exp(top.values[:, :K] - top.values[:, :1])
    den = (e if gate == "topk_norm" else e * (ids < N)).sum(1, keepdim=True)
    return ids, torch.where(den > 0, e / den, torch.zeros_like(e)), p


def _logits(st):
    return st["x"].float() @ st["w_router"].float().t() + st["router_bias"]


def _route(st):
    c = st["case"]
    N, NE, K, n = c["N"], c["N"] + c["Z"], c["K"], float(c["T"])
    ids, gates, p = _select(_logits(st), N, K, c["gate"])
    f, P = torch.nn.functional.one_hot(ids, NE).sum(1), p
    if st["mask"] is not None:
        m = (st["mask"] != 0)[:, None]
        f, P, n = torch.where(m, f, 0), torch.where(m, p, torch.zeros_like(p)), m.sum().clamp(min=1)
    counts = f.sum(0)
    f, P = counts.double() / n, P.sum(0, dtype=torch.float64) / n
    fE, PE, fZ, PZ, Zw = f[:N].sum(), P[:N].sum(), f[N:].sum(), P[N:].sum(), c["Z"] * GROUP_W
    la = ALPHA * NE / K * (f * P).sum()
    lga = ALPHA * (N + Zw) / K * (fE * PE / N + (fZ * PZ / Zw if c["Z"] else 0.0))
    return ids.int(), gates, p, counts.int(), P.float(), torch.stack([fE, PE, fZ, PZ, fZ / K, la, lga]).float()


def _backward(st):
    c = st["case"]
    N, Z, NE, K, p, ids, gates = c["N"], c["Z"], c["N"] + c["Z"], c["K"], st["probs"], st["topk_ids"].long(), st["topk_gates"]
    on = torch.ones_like(p[:, :1], dtype=torch.bool) if st["mask"] is None else (st["mask"] != 0)[:, None]
    n = on.sum().clamp(min=1)
    # dL/dP of both losses, in 64 bits and with its mean taken off (which the softmax's gradient does not see)
    f = st["counts"].double() / n
    group = torch.cat([(f[:N].sum() / N).expand(N), (f[N:].sum() / max(Z * GROUP_W, 1e-30)).expand(Z)])
    a = ALPHA / K * (st["d_loss"][0] * NE * f + st["d_loss"][1] * (N + Z * GROUP_W) * group)
    a = ((a - a.mean()) / n).float()
    d = p * (a - (p * a).sum(1, keepdim=True))
    # the gates'
    dg, g = st["d_gates"], gates
    if c["gate"] == "softmax":
        dg = dg * p.gather(1, ids)
        d = d - p * dg.sum(1, keepdim=True)
    else:
        s = (dg * g).sum(1, keepdim=True)
        dg = dg * g - s * g * (1 if c["gate"] == "topk_norm" else ids < N)
    d = torch.where(on, d.scatter_add(1, ids, dg), torch.zeros_like(d))
    x = torch.where(on, st["x"].float(), torch.zeros_like(st["x"], dtype=torch.float32))
    return (d @ st["w_router"].float()).to(st["x"].dtype), d.t() @ x, d.sum(0)


def _combine_backward(st):
    K, rows = st["case"]["K"], st["slot_to_row"].long()
    slots = torch.nonzero(rows >= 0).view(-1)
    r, d = rows[slots], st["d_out"].float()[slots // K]
    dg = torch.zeros(rows.numel(), device="cuda")
    dg[slots] = (d * st["y_slot"].float()[r]).sum(1)
    dy = st["d_y_slot"].clone()
    dy[r] = (d * st["topk_gates"].view(-1)[slots, None]).to(dy.dtype)
    return dg.view(-1, K), dy


def _rows_8bit(x):
    """Rows as the values that 8 bits hold: e4m3 with a power-of-two scale for every 128 columns."""
    p = torch.nn.functional.pad(x, (0, -x.shape[-1] % 128)).view(*x.shape[:-1], -1, 128)
    m, e = torch.frexp(p.abs().amax(-1, keepdim=True))
    s = (e - 9 + (m > 0.875)).clamp(-126, 127)
    q = torch.ldexp(torch.ldexp(p, -s).to(torch.float8_e4m3fn).float(), s)
    return q.flatten(-2)[..., : x.shape[-1]]


def _weights(st, name, of):
    """The matrices of the experts `of`, out of 8 bits: each expert's once, or only those that are asked for where they are fewer."""
    few = of.numel() < st["case"]["N"]
    q, s = st["q_" + name], st["s_" + name]
    if few:
        q, s = q.view(torch.uint8)[of].view(q.dtype), s[of]
    q, s = q.float(), torch.ldexp(torch.ones((), device="cuda"), s.int() - 127)
    w = q * s.repeat_interleave(128, 1)[:, : q.shape[1]].repeat_interleave(128, 2)[:, :, : q.shape[2]]
    return w if few else w[of]


def _layer(st):
    c, x = st["case"], st["x"].float()
    T, H, N, K = c["T"], c["H"], c["N"], c["K"]
    ids, gates, _ = _select(_logits(st), N, K, c["gate"])
    # the slots on normal experts, sorted by expert and padded to blocks of b rows of one expert
    e, order = torch.sort(ids.reshape(-1), stable=True)
    real = int((ids < N).sum())
    e, order = e[:real], order[:real]
    b = min(128, 1 << max(0, math.ceil(math.log2(max(1.0, real / N)))))
    rows = torch.bincount(e, minlength=N)
    nb = (rows + b - 1) // b
    dest = (nb.cumsum(0) - nb)[e] * b + torch.arange(real, device="cuda") - (rows.cumsum(0) - rows)[e]
    of = torch.repeat_interleave(torch.arange(N, device="cuda"), nb)
    xb = torch.zeros(of.numel() * b, H, device="cuda")
    xb[dest] = _rows_8bit(x)[order // K]
    xb = xb.view(-1, b, H).transpose(1, 2).contiguous()
    gate = torch.bmm(_weights(st, "gate", of), xb)
    up = torch.bmm(_weights(st, "up", of), xb)
    act = _rows_8bit((gate / (1.0 + torch.exp(-gate)) * up).transpose(1, 2)).transpose(1, 2).contiguous()
    y = torch.bmm(_weights(st, "down", of), act).transpose(1, 2).reshape(-1, H)
    slots = torch.zeros(T * K, H, device="cuda")
    slots[order] = y[dest]
    out = (slots.view(T, K, H) * gates[:, :, None]).sum(1)
    if c["copy"]:
        out = out + (gates * (ids >= N)).sum(1, keepdim=True) * x
    return out.to(torch.bfloat16), (ids < N).sum().int().view(1)


def run(st):
    c = st["case"]
    if not own:
        return {"layer": _layer, "route": _route, "backward": _backward, "combine": _combine_backward}[c["kind"]](st)
    from paper_2605_18643_amd import zeda

    if c["kind"] == "layer":
        zeda.zeda_moe_forward_fp8(st["desc"], st["x"], st["w_router"], st["router_bias"], st["experts"], st["out"], st["num_real"], st["ws"])
        return st["out"], st["num_real"]
    if c["kind"] == "route":
        zeda.zeda_route_train(st["desc"], st["x"], st["w_router"], st["router_bias"], st["mask"], ALPHA, GROUP_W, st["topk_ids"],
                              st["topk_gates"], st["probs"], st["counts"], st["mean_probs"], st["summary"], st["ws"])
        return tuple(st[k] for k in ("topk_ids", "topk_gates", "probs", "counts", "mean_probs", "summary"))
    if c["kind"] == "backward":
        zeda.zeda_route_backward(st["desc"], st["x"], st["w_router"], st["probs"], st["topk_ids"], st["topk_gates"], st["mask"], st["counts"],
                                 ALPHA, GROUP_W, st["d_loss"], st["d_gates"], st["dx"], st["dw_router"], st["dbias"], st["ws"])
        return st["dx"], st["dw_router"], st["dbias"]
    zeda.zeda_combine_backward(st["desc"], st["d_out"], st["y_slot"], st["topk_ids"], st["topk_gates"], st["slot_to_row"], None,
                               st["d_gates"], st["d_y_slot"], None)
    return st["d_gates"], st["d_y_slot"]


def work(case):
    kind, T, H, I, N, Z, K = (case[k] for k in ("kind", "T", "H", "I", "N", "Z", "K"))
    s, NE = 2.0 if case["dtype"] == "bf16" else 4.0, N + Z
    R = T * K * (0.5 if Z else 1.0)  # slots on normal experts
    if kind == "layer":  # e4m3 weights of the experts that are hit, tokens in and out, the router
        hit = N * (1.0 - (1.0 - 1.0 / N) ** R)
        return {"bytes": hit * 3.0 * H * I + NE * H * s + 2.0 * T * H * s, "flops": 6.0 * H * I * R + 2.0 * T * NE * H}
    if kind == "route":
        return {"bytes": (T + NE) * H * s + T * NE * 4.0 + T * K * 8.0, "flops": 2.0 * T * NE * H}
    if kind == "backward":  # tokens, router, probabilities in; the gradients of tokens and router out
        return {"bytes": (2.0 * T + NE) * H * s + NE * H * 4.0 + T * NE * 4.0 + T * K * 12.0, "flops": 4.0 * T * NE * H}
    return {"bytes": (T + 2.0 * R) * H * s + T * K * 12.0, "flops": 3.0 * R * H}


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, token by token and expert by expert from the definitions
# ---------------------------------------------------------------------------------------------------------------------
def _exact_8bit(v):
    """e4m3's nearest values (ties to even) under the scale of every 128 columns, in 64 bits."""
    n = v.shape[1]
    p = torch.cat([v, v.new_zeros(v.shape[0], -n % 128)], 1).reshape(v.shape[0], -1, 128)
    top = p.abs().amax(2, keepdim=True)
    scale = 2.0 ** torch.ceil(torch.log2(top.clamp(min=448 * 2.0 ** -126) / 448))
    scale = torch.where(scale * 224 >= top, scale / 2, scale)  # (where the logarithm was rounded up past a whole number)
    q = p / scale
    step = 2.0 ** (torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(q / step) * step * scale).reshape(v.shape[0], -1)[:, :n]


def _exact_router(case, st):
    logit = st["x"].double() @ st["w_router"].double().t() + st["router_bias"].double()
    order = torch.argsort(-logit, dim=1, stable=True)[:, : case["K"]]
    ex = torch.exp(logit - logit.max(1, keepdim=True).values)
    p = ex / ex.sum(1, keepdim=True)
    g = torch.gather(p, 1, order)
    if case["gate"] == "topk_norm":
        g = g / g.sum(1, keepdim=True)
    if case["gate"] == "real_renorm":
        among = torch.where(order < case["N"], g, 0.0).sum(1, keepdim=True)
        g = torch.where(among > 0, g / among, 0.0)
    return order, g, p


def _exact_layer(case, seed):
    own_before = globals()["own"]
    globals()["own"] = False
    try:
        st = _prepare_layer(case, seed)
    finally:
        globals()["own"] = own_before
    order, g, _ = _exact_router(case, st)
    x, out = st["x"].double(), torch.zeros(st["x"].shape, dtype=torch.float64, device="cuda")
    xq = _exact_8bit(x)

    def matrix(name, i):
        q, s = st["q_" + name][i].double(), st["s_" + name][i].double() - 127
        return q * torch.kron(2.0 ** s, torch.ones(128, 128, dtype=torch.float64, device="cuda"))[: q.shape[0], : q.shape[1]]

    for i in range(case["N"]):
        t, j = torch.nonzero(order == i, as_tuple=True)
        if len(t):
            a = xq[t] @ matrix("gate", i).t()
            h = _exact_8bit(a * torch.sigmoid(a) * (xq[t] @ matrix("up", i).t()))
            out[t] += (h @ matrix("down", i).t()) * g[t, j, None]
    if case["copy"]:
        out += torch.where(order >= case["N"], g, 0.0).sum(1, keepdim=True) * x
    return out, None


def exact(case, seed):
    kind, N, Z, K = case["kind"], case["N"], case["Z"], case["K"]
    if kind == "layer":
        return _exact_layer(case, seed)
    st, g = _inputs(case, seed)
    mask = _mask(case, g)
    order, gates, p = _exact_router(case, st)
    keep = torch.arange(case["T"], device="cuda") if mask is None else torch.nonzero(mask).view(-1)
    n = max(1, len(keep))
    f = torch.zeros(N + Z, dtype=torch.float64, device="cuda").index_add_(0, order[keep].reshape(-1), torch.ones(len(keep) * K, dtype=torch.float64, device="cuda")) / n
    P = p[keep].sum(0) / n
    tokens, weight = [N, Z], [N, Z * GROUP_W]
    fs, Ps = torch.stack([v.sum() for v in f.split(tokens)]), torch.stack([v.sum() for v in P.split(tokens)])
    inv = torch.tensor([1.0 / v if v else 0.0 for v in weight], dtype=torch.float64, device="cuda")
    kA, kGA = ALPHA * (N + Z) / K, ALPHA * sum(weight) / K
    if kind == "route":
        summary = torch.stack([fs[0], Ps[0], fs[1], Ps[1], fs[1] / K, kA * f.dot(P), kGA * (fs * Ps * inv).sum()])
        return None, gates, p, None, P, summary
    if kind == "combine":
        real = (order < N).reshape(-1)
        place = torch.argsort(torch.where(real, order.reshape(-1), N + Z), stable=True)[: int(real.sum())]  # the slot of every row
        y = torch.randn(case["T"] * K, case["H"], generator=g, device="cuda").to(_dt(case)).double()
        d = (torch.randn(case["T"], case["H"], generator=g, device="cuda") / case["T"]).to(_dt(case)).double()
        dg, dy = torch.zeros(case["T"] * K, dtype=torch.float64, device="cuda"), torch.zeros_like(y)
        dg[place] = torch.linalg.vecdot(d[place // K], y[: len(place)])
        dy[: len(place)] = gates.reshape(-1)[place][:, None] * d[place // K]
        return dg.reshape(-1, K), dy
    d_loss = (torch.rand(2, generator=g, device="cuda") + 0.5).double()
    d_gates = (torch.randn(case["T"], K, generator=g, device="cuda") * (0.1 / case["T"])).double()
    # through the softmaxes' Jacobians: the whole pool's for the probabilities, the selected experts' for the gates
    slope = (d_loss[0] * kA * f + d_loss[1] * kGA * (fs * inv).repeat_interleave(torch.tensor(tokens, device="cuda"))) / n
    chosen = torch.zeros_like(p).scatter_(1, order, 1.0) > 0
    up = torch.zeros_like(p).scatter_(1, order, d_gates)
    if case["gate"] == "softmax":
        dl = p * (slope + up) - p * (p * (slope + up)).sum(1, keepdim=True)
    else:
        gate = torch.zeros_like(p).scatter_(1, order, gates)
        shared = chosen if case["gate"] == "topk_norm" else chosen & (torch.arange(N + Z, device="cuda") < N)
        dl = p * slope - p * (p * slope).sum(1, keepdim=True) + gate * (up - torch.where(shared, (gate * up).sum(1, keepdim=True), 0.0))
    dx = torch.zeros(st["x"].shape, dtype=torch.float64, device="cuda")
    dx[keep] = dl[keep] @ st["w_router"].double()
    return dx, dl[keep].t() @ st["x"][keep].double(), dl[keep].sum(0)
