"""Quantisation of nothing: an empty tensor has no address."""
import pytest
import torch

from paper_2605_18643_amd import zeda

P = 4096  # a plausible device address, never touched


def test_no_rows_and_no_matrices_are_no_ops():
    L = zeda.lib()
    assert L.zeda_quantize_rows_fp8(0, 128, zeda.ZEDA_BF16, None, None, None, None) == zeda.ZEDA_OK
    assert L.zeda_quantize_weights_fp8(0, 8, 128, zeda.ZEDA_F32, None, None, None, None) == zeda.ZEDA_OK


def test_what_is_wrong_without_rows_too():
    rows, weights = zeda.lib().zeda_quantize_rows_fp8, zeda.lib().zeda_quantize_weights_fp8
    assert rows(0, 0, 1, None, None, None, None) == zeda.ZEDA_EINVAL and rows(0, 128, 2, None, None, None, None) == zeda.ZEDA_EINVAL
    assert weights(0, 0, 8, 1, None, None, None, None) == zeda.ZEDA_EINVAL and weights(0, 8, 8, 3, None, None, None, None) == zeda.ZEDA_EINVAL
    assert rows(0, 12, 1, None, None, None, None) == zeda.ZEDA_EUNSUPPORTED and weights(0, 4, 12, 1, None, None, None, None) == zeda.ZEDA_EUNSUPPORTED
    # one row needs all its pointers
    for i in range(3):
        p = [P] * i + [None] + [P] * (2 - i)
        assert rows(1, 128, 1, *p, None) == zeda.ZEDA_EINVAL and weights(1, 8, 128, 1, *p, None) == zeda.ZEDA_EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_empty_tensors(dtype):
    q, s = zeda.zeda_quantize_rows_fp8(torch.empty(0, 256, dtype=dtype, device="cuda"))
    assert q.shape == (0, 256) and s.shape == (0, 2)
    q, s = zeda.zeda_quantize_weights_fp8(torch.empty(0, 64, 256, dtype=dtype, device="cuda"))
    assert q.shape == (0, 64, 256) and s.shape == (0, 1, 2)
