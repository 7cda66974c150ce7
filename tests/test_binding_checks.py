"""What the C side cannot see of a tensor, refused by the binding before anything is launched (no GPU)."""
import ctypes

import pytest
import torch

from paper_2605_18643_amd import zeda

F, I32, BF = torch.float32, torch.int32, torch.bfloat16


def _refused(call):
    with pytest.raises(zeda.ZedaError) as e:
        call()
    return e.value.status == zeda.ZEDA_EINVAL


def _wrong(t):
    """The same buffer of another type, one entry short, and with gaps."""
    return t.to(torch.float64), t.reshape(-1)[:-1], torch.stack([t, t], -1)[..., 0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_combine_backward_looks_at_the_expert_outputs(dtype):
    dt, other = (BF, F) if dtype == "bf16" else (F, BF)
    d = zeda.make_desc(6, 128, 64, 3, 2, 2, dtype)
    t = dict(d_out=torch.zeros(6, 128, dtype=dt), ids=torch.zeros(6, 2, dtype=I32), gates=torch.zeros(6, 2), s2r=torch.zeros(12, dtype=I32), d_gates=torch.zeros(6, 2),
             dy=torch.zeros(12, 128, dtype=dt))
    y = torch.zeros(12, 128, dtype=dt)
    for bad in (*_wrong(y), y.to(other), y[:6]):
        assert _refused(lambda: zeda.zeda_combine_backward(d, t["d_out"], bad, t["ids"], t["gates"], t["s2r"], None, t["d_gates"], t["dy"], None))


def _experts(d, short=None, **kw):
    sizes = (ctypes.c_size_t * 4)()
    assert zeda.lib().zeda_fp8_expert_bytes(ctypes.byref(d), sizes) == zeda.ZEDA_OK
    return zeda.Fp8Experts([torch.zeros(n - (i == short), dtype=torch.uint8) for i, n in enumerate(sizes)], **kw)


def _layer(T=6, H=256, I=128, N=3, Z=2, K=2):
    d = zeda.make_desc(T, H, I, N, Z, K, "bf16")
    experts = _experts(d)
    t = dict(x=torch.zeros(T, H, dtype=BF), wr=torch.zeros(N + Z, H, dtype=BF), bias=torch.zeros(N + Z), out=torch.zeros(T, H, dtype=BF), nr=torch.zeros(1, dtype=I32),
             x_res=torch.zeros(T, H, dtype=BF), gamma=torch.zeros(H, dtype=BF), xn=torch.zeros(T, H, dtype=BF), off=torch.zeros(N + 1, dtype=I32),
             ss=torch.zeros(T * K, dtype=I32), y=torch.zeros(T * K, H, dtype=BF), ws=torch.zeros(zeda.workspace_bytes_fp8(d), dtype=torch.uint8))

    def calls(d=d, experts=experts, **kw):
        a = {**t, **kw}
        return {"ffn": lambda: zeda.zeda_expert_ffn_fp8(d, a["x"], experts, a["off"], a["ss"], a["nr"], a["y"], a["ws"]),
                "forward": lambda: zeda.zeda_moe_forward_fp8(d, a["x"], a["wr"], a["bias"], experts, a["out"], a["nr"], a["ws"]),
                "block": lambda: zeda.zeda_moe_block_forward_fp8(d, a["x"], a["x_res"], a["wr"], a["bias"], experts, a["gamma"], 1e-6, a["xn"], a["nr"], a["ws"])}

    return d, t, calls


TAKES = {"ffn": ("x", "off", "ss", "nr", "y"), "forward": ("x", "wr", "bias", "out", "nr"), "block": ("x", "x_res", "wr", "bias", "gamma", "xn", "nr")}


@pytest.mark.parametrize("call", TAKES)
def test_8_bit_layer_calls_look_at_their_tensors(call):
    _, t, calls = _layer()
    for n in TAKES[call]:
        for bad in _wrong(t[n])[: 2 if t[n].numel() == 1 else 3]:
            assert _refused(calls(**{n: bad})[call]), n


@pytest.mark.parametrize("call", TAKES)
def test_experts_packed_for_another_layer_are_refused(call):
    d, t, calls = _layer()
    # buffers that a caller has kept: by their sizes
    for short in range(4):
        assert _refused(calls(experts=_experts(d, short=short))[call])
    assert _refused(calls(experts=_experts(zeda.make_desc(0, 128, 128, 3, 0, 1, "bf16")))[call])
    assert _refused(calls(experts=zeda.Fp8Experts([]))[call])
    # packed by the binding: by the layer's shape, where sizes are alike too
    for N, H, I in ((4, 256, 128), (3, 256, 192), (3, 384, 128), (3, 128, 256), (1, 256, 384)):
        other = zeda.make_desc(0, H, I, N, 0, 1, "bf16")
        assert _refused(calls(experts=_experts(other, desc=other))[call]), (N, H, I)


def test_buffers_too_small_for_the_descriptor_make_no_experts():
    d = zeda.make_desc(0, 256, 128, 3, 0, 1, "bf16")
    for short in range(4):
        assert _refused(lambda: _experts(d, short=short, desc=d))
    e = _experts(d, desc=d)
    assert e.shape == (3, 256, 128) and e.w_gateup == e.buffers[0].data_ptr()


def test_fp32_layers_are_unsupported_not_ill_typed(monkeypatch):
    """8-bit calls with an fp32 descriptor and fp32 tensors: what the header says of the descriptor."""
    monkeypatch.setattr(zeda, "_stream", lambda stream: 0)  # (the library refuses before it looks at the stream)
    d, t, calls = _layer()
    f32 = zeda.make_desc(6, 256, 128, 3, 2, 2, "f32")
    wide = {n: v.float() for n, v in t.items() if v.dtype == BF}
    for call in calls(d=f32, experts=_experts(d, desc=d), **wide).values():
        with pytest.raises(zeda.ZedaError) as e:
            call()
        assert e.value.status == zeda.ZEDA_EUNSUPPORTED
