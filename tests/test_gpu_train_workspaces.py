"""Training batches whose router splits the hidden dimension into more than 4096 rows of logit tables: against the formulas in 64 bits, with
bytes behind both workspaces that must stay as they are.  Tolerances as derived in test_gpu_train.py."""
import numpy as np
import pytest
import torch

import test_gpu_train as tt
from oracle import harness, zeda_oracle as orc
from paper_2605_18643_amd import zeda

pytestmark = pytest.mark.gpu

GUARD, BYTE = 1 << 16, 0xa5


class _Guarded:
    """The scratch of exactly the size that the library asks for, in front of GUARD bytes."""

    def run(self, stream=None):
        if not hasattr(self, "whole"):
            self.whole = torch.full((self.ws.numel() + GUARD,), BYTE, dtype=torch.uint8, device="cuda")
            self.ws = self.whole[:-GUARD]
        super().run(stream)

    def untouched(self):
        return bool((self.whole[-GUARD:] == BYTE).all())


class Forward(_Guarded, tt.Forward):
    pass


class Backward(_Guarded, tt.Backward):
    pass


@pytest.mark.parametrize("T, H, N, Z, K, masked", [(2048, 2048, 32, 8, 4, "some"), (4096, 4096, 128, 32, 8, "none"), (1396, 1536, 48, 10, 6, "some"), (2006, 2048, 40, 0, 4, "none"),
                                                   (4080, 1536, 200, 28, 8, "some"), (1000, 4096, 24, 8, 4, "none"), (1536, 2560, 128, 32, 8, "some")])
def test_wide_splits_stay_in_their_scratch(T, H, N, Z, K, masked):
    print(T, H, N, Z, K, masked, flush=True)
    w = tt._workload(T, H, N, Z, K, "bf16")
    L = harness.gapped_layer(w, "cuda")
    a, mask = harness.to_arrays(L), tt._mask(T, masked)
    on = np.ones(T, bool) if mask is None else mask.cpu().numpy() != 0
    gate = zeda.GATE_TOPK_NORM
    f = Forward(w, L, gate, mask)
    torch.cuda.synchronize()
    assert f.untouched(), "written past the workspace"
    ids, gates, logits = orc.route(a["x"], a["w_router"], a["router_bias"], N, Z, K, gate, want_logits=True)
    assert np.array_equal(tt._np(f.ids), ids)
    rel = 8 * np.sqrt(H) * tt.U * max(1.0, np.abs(logits).max()) + 2e-6
    np.testing.assert_allclose(tt._np(f.g), gates, rtol=rel, atol=1e-30)
    e = np.exp(logits - logits.max(1, keepdims=True))
    np.testing.assert_allclose(tt._np(f.p), e / e.sum(1, keepdims=True), rtol=rel, atol=1e-30)
    counts, P, summary = tt._batch_sums(tt._np(f.p), ids, on, N, K)
    assert np.array_equal(tt._np(f.counts), counts)
    np.testing.assert_allclose(tt._np(f.P), P, rtol=20 * tt.U)
    np.testing.assert_allclose(tt._np(f.summary), summary, rtol=20 * tt.U)
    keep = [t.clone() for t in f.outputs()]
    f.run()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(keep, f.outputs()))
    b = Backward(f, *tt._grads(f))
    b.check()
    assert b.untouched() and f.untouched()
