"""8-bit experts without a GPU: sizes, and every refusal before anything is launched."""
import ctypes

import pytest
import torch

from paper_2605_18643_amd import zeda

OK, EINVAL, EUNSUPPORTED, EWORKSPACE = zeda.ZEDA_OK, zeda.ZEDA_EINVAL, zeda.ZEDA_EUNSUPPORTED, zeda.ZEDA_EWORKSPACE
P, ODD = 4096, 4097  # plausible device addresses (never touched), aligned and not


def _desc(**kw):
    return zeda.make_desc(**{**dict(T=4096, H=2048, I=768, N=128, Z=32, K=8, dtype="bf16"), **kw})


def _experts(**kw):
    e = zeda.Fp8Experts([])
    for n in ("w_gateup", "w_down", "s_gateup", "s_down"):
        setattr(e, n, kw.get(n, P))
    return e


def test_sizes():
    b = (ctypes.c_size_t * 4)()
    assert zeda.lib().zeda_fp8_expert_bytes(ctypes.byref(_desc()), b) == OK
    assert list(b) == [128 * 2 * 768 * 2048, 128 * 768 * 2048, 128 * 6 * 2 * 16, 128 * 16 * 8]
    # I is filled up to whole blocks of 128, scale rows to whole words
    assert zeda.lib().zeda_fp8_expert_bytes(ctypes.byref(_desc(H=1152, I=448, N=24)), b) == OK
    assert list(b) == [24 * 2 * 512 * 1152, 24 * 512 * 1152, 24 * 4 * 2 * 12, 24 * 9 * 4]
    d = _desc()
    L = zeda.workspace_layout_fp8(d)
    assert zeda.workspace_bytes_fp8(d) == L.total
    assert L.y_slot - L.act >= zeda.expert_ffn_workspace_bytes_fp8(d) >= 4096 * (2048 + 16) + 4096 * 8 * (768 + 8)
    # the tables in front of it lie where the bf16 layer has them (MoeStack reads the ids there)
    M = zeda.workspace_layout(d)
    assert all(getattr(L, n) == getattr(M, n) for n in ("topk_ids", "topk_gates", "expert_offsets", "sorted_slot", "slot_to_row", "num_real"))
    # the layout of the row-major weights does not matter
    assert zeda.workspace_bytes_fp8(_desc(weight_layout=zeda.WEIGHTS_TILED)) == L.total
    assert zeda.workspace_bytes_fp8(_desc(T=0)) > 0


@pytest.mark.parametrize("kw, code", [
    (dict(dtype="f32"), EUNSUPPORTED), (dict(H=16512), EUNSUPPORTED), (dict(I=16448), EUNSUPPORTED), (dict(H=2112), EUNSUPPORTED),
    (dict(I=800), EUNSUPPORTED), (dict(K=17), EUNSUPPORTED), (dict(N=0), EINVAL), (dict(T=-1), EINVAL), (dict(gate_norm=3), EINVAL)])
def test_descriptors_that_are_refused(kw, code):
    d, b, out = _desc(**kw), (ctypes.c_size_t * 4)(), zeda.WsLayout()
    L, e = zeda.lib(), _experts()
    assert zeda.workspace_bytes_fp8(d) == 0 and zeda.expert_ffn_workspace_bytes_fp8(d) == 0
    assert L.zeda_workspace_layout_fp8(ctypes.byref(d), ctypes.byref(out)) == code
    big = 1 << 40
    assert L.zeda_expert_ffn_fp8(ctypes.byref(d), P, ctypes.byref(e), P, P, P, P, P, big, None) == code
    assert L.zeda_moe_forward_fp8(ctypes.byref(d), P, P, None, ctypes.byref(e), P, None, P, big, None) == code
    assert L.zeda_moe_block_forward_fp8(ctypes.byref(d), P, 2 * P, P, None, ctypes.byref(e), None, 1e-6, P, None, P, big, None) == code
    if "T" not in kw:
        assert L.zeda_fp8_expert_bytes(ctypes.byref(d), b) == code
        assert L.zeda_pack_expert_weights_fp8(ctypes.byref(d), P, P, P, P, P, P, ctypes.byref(e), None) == code


def test_pointers_that_are_refused():
    d, L = _desc(), zeda.lib()
    big = zeda.workspace_bytes_fp8(d)

    def forward(x=P, wr=P, bias=None, e=_experts(), out=P, ws=P, n=big):
        return L.zeda_moe_forward_fp8(ctypes.byref(d), x, wr, bias, None if e is None else ctypes.byref(e), out, None, ws, n, None)

    for kw in (dict(x=None), dict(wr=None), dict(e=None), dict(out=None), dict(ws=None), dict(x=ODD), dict(bias=ODD), dict(out=ODD),
               dict(e=_experts(w_gateup=None)), dict(e=_experts(s_down=None)), dict(e=_experts(w_down=ODD)), dict(e=_experts(s_gateup=ODD))):
        assert forward(**kw) == EINVAL, kw
    assert forward(n=big - 1) == EWORKSPACE

    def ffn(x=P, e=_experts(), off=P, ss=P, nr=P, y=P, ws=P, n=big):
        return L.zeda_expert_ffn_fp8(ctypes.byref(d), x, None if e is None else ctypes.byref(e), off, ss, nr, y, ws, n, None)

    for kw in (dict(x=None), dict(e=None), dict(off=None), dict(ss=None), dict(nr=None), dict(y=None), dict(ws=None), dict(ss=ODD), dict(y=ODD)):
        assert ffn(**kw) == EINVAL, kw
    assert ffn(n=zeda.expert_ffn_workspace_bytes_fp8(d) - 1) == EWORKSPACE
    # the residual block: x_res apart from its input and its next one, rows that fit
    def block(xn=P, xr=2 * P, nx=3 * P, eps=1e-6, desc=d):
        return L.zeda_moe_block_forward_fp8(ctypes.byref(desc), xn, xr, P, None, ctypes.byref(_experts()), None, eps, nx, None, P, 1 << 40, None)

    assert block(xr=P) == EINVAL and block(nx=2 * P) == EINVAL and block(eps=-1.0) == EINVAL and block(xr=None) == EINVAL
    assert block(desc=_desc(H=16384)) == EUNSUPPORTED


def test_quantisation_and_packing_refusals():
    L = zeda.lib()
    rows, weights = L.zeda_quantize_rows_fp8, L.zeda_quantize_weights_fp8
    assert rows(0, 128, 1, P, P, P, None) == OK and weights(0, 8, 8, 0, P, P, P, None) == OK
    assert rows(-1, 128, 1, P, P, P, None) == EINVAL and rows(1, 0, 1, P, P, P, None) == EINVAL and rows(1, 128, 2, P, P, P, None) == EINVAL
    assert rows(1, 12, 1, P, P, P, None) == EUNSUPPORTED and weights(1, 4, 12, 1, P, P, P, None) == EUNSUPPORTED
    assert rows(1, 128, 1, None, P, P, None) == EINVAL and rows(1, 128, 1, P, ODD, P, None) == EINVAL and rows(1, 128, 1, P, P, None, None) == EINVAL
    assert weights(1, 0, 8, 1, P, P, P, None) == EINVAL and weights(1, 8, 8, 1, ODD, P, P, None) == EINVAL and weights(-1, 8, 8, 1, P, P, P, None) == EINVAL
    d, e = _desc(), _experts(w_gateup=1 << 44, w_down=1 << 45, s_gateup=1 << 46, s_down=1 << 47)
    q = [1 << 33, 1 << 34, 1 << 35, 1 << 36, 1 << 37, 1 << 38]
    pack = lambda q, e: L.zeda_pack_expert_weights_fp8(ctypes.byref(d), *q, ctypes.byref(e), None)  # noqa: E731
    for i in range(6):
        assert pack(q[:i] + [None] + q[i + 1:], e) == EINVAL
    for i in (0, 2, 4):
        assert pack(q[:i] + [q[i] + 1] + q[i + 1:], e) == EINVAL
    for i in range(6):  # every input against every output
        for n in ("w_gateup", "w_down", "s_gateup", "s_down"):
            o = _experts(w_gateup=1 << 44, w_down=1 << 45, s_gateup=1 << 46, s_down=1 << 47)
            setattr(o, n, q[i])
            assert pack(q, o) == EINVAL, (i, n)


def test_binding_refuses_what_the_library_cannot_see():
    d = _desc(T=4, H=256, I=128, N=2, Z=0, K=1)
    bad = [lambda: zeda.zeda_quantize_rows_fp8(torch.zeros(4, 128, dtype=torch.float16)),
           lambda: zeda.zeda_quantize_rows_fp8(torch.zeros(128, 4, dtype=torch.bfloat16).t()),
           lambda: zeda.zeda_quantize_rows_fp8(torch.zeros(1, 4, 128)),
           lambda: zeda.zeda_quantize_weights_fp8(torch.zeros(4, 128)),
           lambda: zeda.zeda_quantize_weights_fp8(torch.zeros(1, 4, 128, dtype=torch.float64))]
    u = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    good = [u(2, 128, 256), u(2, 1, 2), u(2, 128, 256), u(2, 1, 2), u(2, 256, 128), u(2, 2, 1)]
    for i, other in ((0, u(2, 128, 128)), (1, u(2, 2, 1)), (2, torch.zeros(2, 128, 256)), (4, u(2, 128, 256)), (5, u(2, 1, 2)),
                     (0, u(2, 256, 128).transpose(1, 2))):
        bad.append(lambda i=i, other=other: zeda.zeda_pack_expert_weights_fp8(d, *good[:i], other, *good[i + 1:]))
    for f in bad:
        with pytest.raises(zeda.ZedaError) as err:
            f()
        assert err.value.status == EINVAL


def test_a_longer_batch_never_needs_less():
    for kw in (dict(), dict(N=64, I=1536, K=4), dict(N=12, I=192, H=256, K=2), dict(N=2, Z=0, I=64, H=128, K=1)):
        sizes = [zeda.expert_ffn_workspace_bytes_fp8(zeda.make_desc(**{**dict(T=T, H=2048, I=768, N=128, Z=32, K=8, dtype="bf16"), **kw}))
                 for T in list(range(1, 300)) + list(range(301, 20000, 97))]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), kw
