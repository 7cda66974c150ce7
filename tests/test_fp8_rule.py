"""Which kernels an 8-bit layer takes (no GPU): the rule's answers at sizes where both sides have been measured, and no jumps between them."""
import ctypes

import pytest

from paper_2605_18643_amd import zeda


def _slots(N, Z, H, I):
    f = zeda.lib()["_ZN4zeda13fp8_few_slotsEPK15zeda_layer_desc"]  # zeda::fp8_few_slots: slots up to which the kernels of few rows are taken
    f.restype, f.argtypes = ctypes.c_int64, [ctypes.POINTER(zeda.LayerDesc)]
    return f(ctypes.byref(zeda.make_desc(1, H, I, N, Z, 1, "bf16")))


# (N, Z, H, I, slots where the kernels of few rows took at most 0.92 of the tile kernels' time, slots where they took at least 1.05 of it)
MEASURED = [(16, 4, 4096, 1024, 16, 80), (16, 4, 4096, 256, 120, 800), (24, 8, 4096, 448, 60, 288), (32, 8, 4096, 1024, 4, 120), (64, 16, 1024, 512, 8, 320),
            (24, 8, 1152, 448, 192, None), (128, 32, 2048, 768, 128, 640), (64, 32, 2048, 1536, 4, None), (12, 4, 1664, 320, 180, None), (1, 1, 2048, 2048, 35, None),
            (2, 1, 4352, 4352, 7, None), (30, 10, 256, 256, 400, 2280), (64, 16, 128, 128, 8, 8800), (200, 40, 128, 64, 8, 2000)]


@pytest.mark.parametrize("N, Z, H, I, few, tile", MEASURED)
def test_measured_sides(N, Z, H, I, few, tile):
    assert few <= _slots(N, Z, H, I) and (tile is None or _slots(N, Z, H, I) < tile)


@pytest.mark.parametrize("H, I", [(4096, 1024), (4096, 256), (2560, 768), (1024, 512), (512, 256)])
def test_one_more_expert_is_no_other_layer(H, I):
    """As long as the weights are small, the slots do not depend on how many experts there are."""
    assert len({_slots(N, 4, H, I) for N in range(14, 36)}) == 1


def test_wider_rows_never_get_more_slots():
    for N, I in ((16, 256), (16, 1024), (24, 448)):
        s = [_slots(N, 4, H, I) for H in range(128, 4608, 128)]
        assert all(a >= b for a, b in zip(s, s[1:]))
