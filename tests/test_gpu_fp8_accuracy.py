"""How near the 8-bit layer comes to its definition in 64 bits, by norms: the choices of precision that its kernels make.

The result's rounding to bf16 is uniform in a step of 2^-8 to 2^-7 of the value, half a step at most: relative to the value it has a root
mean square of 2^-8 / sqrt(3) * sqrt(mean of 1 / m^2 over mantissas m in 1..2), 1.6e-3 to 1.8e-3 by the mantissas' distribution.  To that, in
squares:
  - expert outputs in 11 bits between the kernels: an eighth of that, 2.2e-4 (in bf16 it would be as large again, 2.4e-3 and more in all);
  - activations that fall on the other side of the middle between two e4m3 values, each by a step of 2^-4 to 2^-3 of its value, 9e-2 on
    average: a share s of them adds 9e-2 sqrt(s).  Sums with relative errors d have s = about 2 d / 2^-4.  With fp32's d = 1e-7 that is less than
    one of the some 6000 activations of a token; with the 8-bit instruction's d = 1.4e-5 of the root mean square of sums, s = 1 / 5000 to 1 / 2000, it
    adds 1.3e-3 to 2e-3 over many tokens.
So 2.1e-3 bounds short batches (one token: a tenth of H = 2048 columns' standard error is below 2 %), whose sums are as exact as fp32's, and
sqrt(1.8^2 + 2.0^2 + 0.2^2) e-3 = 2.7e-3, with a tenth to spare 3e-3, long ones."""
import numpy as np
import pytest

import test_gpu_fp8 as tf
from oracle import harness
from paper_2605_18643_amd import zeda

pytestmark = pytest.mark.gpu


def _error(T, H, I, N, Z, K, seed):
    w, d = tf._layer(T, H, I, N, Z, K, seed=seed)
    L = harness.gapped_layer(w, "cuda")
    ex = tf.Experts(d, L)
    out, _ = tf._forward(d, L, ex.packed)
    want, _, _ = tf._reference(d, L, ex, zeda.GATE_TOPK_NORM, False)
    return harness.rel_l2(out.double().cpu().numpy(), want)


@pytest.mark.parametrize("T, seeds", [(1, 8), (8, 3)])
def test_short_batches_are_as_exact_as_fp32_sums(T, seeds):
    errors = [_error(T, 2048, 768, 24, 8, 8, seed) for seed in range(10, 10 + seeds)]
    print(T, errors, flush=True)
    assert max(errors) <= 2.1e-3, errors


@pytest.mark.parametrize("T, H, I, N, Z, K", [(1200, 1152, 448, 24, 8, 3), (1500, 2048, 768, 12, 4, 4)])
def test_long_batches(T, H, I, N, Z, K):
    errors = [_error(T, H, I, N, Z, K, seed) for seed in (10, 11)]
    print(T, errors, flush=True)
    assert max(errors) <= 3e-3 and np.isfinite(errors).all(), errors
