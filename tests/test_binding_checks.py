"""What the C side cannot see of a tensor, refused by the binding before anything is launched (no GPU)."""
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
