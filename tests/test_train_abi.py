"""The router's training calls without a GPU: sizes, and every refusal before anything is launched."""
import ctypes

import pytest
import torch

from paper_2605_18643_amd import zeda

OK, EINVAL, EUNSUPPORTED, EWORKSPACE = zeda.ZEDA_OK, zeda.ZEDA_EINVAL, zeda.ZEDA_EUNSUPPORTED, zeda.ZEDA_EWORKSPACE
BIG = 1 << 44
A = {n: (i + 1) << 33 for i, n in enumerate(("x", "wr", "ids", "gates", "probs", "counts", "P", "summary", "ws", "d_loss", "d_gates", "dx", "dw",
                                             "dbias", "d_out", "y", "s2r", "dy", "bias", "mask"))}  # 8 GiB apart, never touched


def _desc(**kw):
    return zeda.make_desc(**{**dict(T=4096, H=2048, I=768, N=128, Z=32, K=8, dtype="bf16"), **kw})


def _train(d, n=BIG, w=2.0, **kw):
    a = {**A, **kw}
    return zeda.lib().zeda_route_train(ctypes.byref(d), a["x"], a["wr"], a["bias"], a["mask"], 0.01, w, a["ids"], a["gates"], a["probs"], a["counts"],
                                       a["P"], a["summary"], a["ws"], n, None)


def _back(d, n=BIG, w=2.0, **kw):
    a = {**A, **kw}
    return zeda.lib().zeda_route_backward(ctypes.byref(d), a["x"], a["wr"], a["probs"], a["ids"], a["gates"], a["mask"], a["counts"], 0.01, w,
                                          a["d_loss"], a["d_gates"], a["dx"], a["dw"], a["dbias"], a["ws"], n, None)


def _combine(d, **kw):
    a = {**A, "dx": None, **kw}
    return zeda.lib().zeda_combine_backward(ctypes.byref(d), a["d_out"], a["y"], a["ids"], a["gates"], a["s2r"], a["x"], a["d_gates"], a["dy"],
                                            a["dx"], None)


@pytest.mark.parametrize("kw, code", [(dict(T=-1), EINVAL), (dict(K=0), EINVAL), (dict(N=4, Z=2, K=7), EINVAL), (dict(K=17), EUNSUPPORTED),
                                      (dict(N=250, Z=7), EUNSUPPORTED), (dict(H=2112), EUNSUPPORTED), (dict(dtype="f32", H=2050), EUNSUPPORTED),
                                      (dict(gate_norm=5), EINVAL)])
def test_descriptors_that_are_refused(kw, code):
    d = _desc(**kw)
    assert zeda.route_train_workspace_bytes(d) == 0 and zeda.route_backward_workspace_bytes(d) == 0
    assert _train(d) == code and _back(d) == code and _combine(d) == code


@pytest.mark.parametrize("kw", [dict(), dict(T=1), dict(T=0), dict(dtype="f32"), dict(N=1, Z=0, K=1), dict(N=250, Z=6, H=128)])
def test_workspaces(kw):
    d = _desc(**kw)
    for size, call in ((zeda.route_train_workspace_bytes, _train), (zeda.route_backward_workspace_bytes, _back)):
        n = size(d)
        assert n > 0 and call(d, n=n - 1) == EWORKSPACE


def test_pointers_that_are_refused():
    d = _desc()
    for n in ("x", "wr", "ids", "gates", "probs", "counts", "P", "summary", "ws"):
        assert _train(d, **{n: None}) == EINVAL, n
    for n in ("x", "wr", "ids", "gates", "probs", "ws", "bias"):
        assert _train(d, **{n: A[n] + 4}) == EINVAL, n
    for n in ("counts", "P", "summary"):
        assert _train(d, **{n: A[n] + 2}) == EINVAL, n
    for n in ("x", "wr", "ids", "gates", "probs", "counts", "ws"):
        assert _back(d, **{n: None}) == EINVAL, n
    for n in ("x", "wr", "ids", "gates", "probs", "ws", "d_gates", "dx", "dw"):
        assert _back(d, **{n: A[n] + 4}) == EINVAL, n
    for n in ("counts", "d_loss", "dbias"):
        assert _back(d, **{n: A[n] + 2}) == EINVAL, n
    for n in ("d_out", "y", "ids", "gates", "s2r", "d_gates"):
        assert _combine(d, **{n: None}) == EINVAL, n
    for n in ("d_out", "y", "ids", "gates", "s2r", "d_gates", "dy"):
        assert _combine(d, **{n: A[n] + 4}) == EINVAL, n
    copy = _desc(free_expert=zeda.EXPERT_COPY)
    assert _combine(copy, x=None) == EINVAL and _combine(copy, x=A["x"] + 4) == EINVAL and _combine(copy, dx=A["dx"] + 4) == EINVAL
    assert _combine(d, dx=A["dx"]) == EINVAL  # only copy experts have a share of x


def test_group_weight_and_empty_gradients():
    d = _desc()
    for w in (0.0, -1.0, float("nan")):
        assert _train(d, w=w) == EINVAL and _back(d, w=w) == EINVAL
    assert _back(d, d_loss=None, d_gates=None) == EINVAL
    assert _back(d, dx=None, dw=None, dbias=None) == EINVAL


def test_outputs_over_inputs_are_refused():
    d, copy = _desc(), _desc(free_expert=zeda.EXPERT_COPY)
    nx = 4096 * 2048 * 2
    assert _back(d, dx=A["x"]) == EINVAL and _back(d, dx=A["x"] + nx - 16) == EINVAL and _back(d, dx=A["wr"] - nx + 16) == EINVAL
    assert _back(d, dw=A["x"] + 64) == EINVAL and _back(d, dw=A["wr"]) == EINVAL
    assert _combine(d, dy=A["y"]) == EINVAL and _combine(d, dy=A["d_out"]) == EINVAL
    for o in ("d_out", "y", "x", "dy"):
        assert _combine(copy, dx=A[o]) == EINVAL, o
    assert _combine(copy, dy=A["x"]) == EINVAL
    assert _combine(_desc(T=0)) == OK


def test_a_longer_batch_never_needs_less():
    """Workspaces are sized once, for the longest batch."""
    for kw in (dict(), dict(N=64, K=4), dict(H=1024, N=12, Z=4, K=3), dict(H=7168, N=250, Z=6), dict(dtype="f32", H=1152)):
        for size in (zeda.route_train_workspace_bytes, zeda.route_backward_workspace_bytes):
            sizes = [size(_desc(T=T, **kw)) for T in list(range(0, 300)) + list(range(301, 20000, 97))]
            assert all(a <= b for a, b in zip(sizes, sizes[1:])), (kw, size.__name__)


def test_tensors_of_another_type_or_size_are_refused():
    """What a pointer does not say."""
    d = _desc(T=6, H=128, N=3, Z=2, K=2)
    f, i = torch.float32, torch.int32
    shapes = dict(x=((6, 128), torch.bfloat16), wr=((5, 128), torch.bfloat16), ids=((6, 2), i), gates=((6, 2), f), probs=((6, 5), f), counts=((5,), i), P=((5,), f),
                  summary=((7,), f), ws=((64,), torch.uint8), mask=((6,), torch.uint8), d_loss=((2,), f), d_gates=((6, 2), f), dx=((6, 128), torch.bfloat16),
                  dw=((5, 128), f), dbias=((5,), f), d_out=((6, 128), torch.bfloat16), y=((12, 128), torch.bfloat16), s2r=((12,), i), dy=((12, 128), torch.bfloat16))
    t = {n: torch.zeros(s, dtype=k) for n, (s, k) in shapes.items()}

    def calls(**kw):
        a = {**t, **kw}
        return (lambda: zeda.zeda_route_train(d, a["x"], a["wr"], None, a["mask"], 0.01, 2.0, a["ids"], a["gates"], a["probs"], a["counts"], a["P"], a["summary"], a["ws"]),
                lambda: zeda.zeda_route_backward(d, a["x"], a["wr"], a["probs"], a["ids"], a["gates"], a["mask"], a["counts"], 0.01, 2.0, a["d_loss"],
                                                 a["d_gates"], a["dx"], a["dw"], a["dbias"], a["ws"]),
                lambda: zeda.zeda_combine_backward(d, a["d_out"], a["y"], a["ids"], a["gates"], a["s2r"], None, a["d_gates"], a["dy"], None))

    for which, names in enumerate((("x", "wr", "mask", "ids", "gates", "probs", "counts", "P", "summary"),
                                   ("x", "wr", "mask", "probs", "ids", "gates", "counts", "d_loss", "d_gates", "dx", "dw", "dbias"),
                                   ("d_out", "ids", "gates", "s2r", "d_gates", "dy"))):
        for n in names:
            for bad in (t[n].to(torch.float64), t[n][:-1]):
                with pytest.raises(zeda.ZedaError) as e:
                    calls(**{n: bad})[which]()
                assert e.value.status == EINVAL, n
