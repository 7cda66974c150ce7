"""The training calls' scratch without a GPU: what the kernels write there fits into what callers are told to bring."""
import ctypes
import random

import pytest

from paper_2605_18643_amd import zeda


class Tables(ctypes.Structure):
    """RouteTables: the split of the bf16 router's product that a launch takes."""

    _fields_ = [(n, ctypes.c_int) for n in ("slices", "Tpad", "E", "tokens")]


def _tables(d):
    f = zeda.lib()["_ZN4zeda12route_tablesEPK15zeda_layer_desc"]  # zeda::route_tables
    f.restype, f.argtypes = Tables, [ctypes.POINTER(zeda.LayerDesc)]
    return f(ctypes.byref(d))


def _desc(T, H, N, Z, K, dtype="bf16"):
    return zeda.make_desc(T, H, 768, N, Z, K, dtype)


def _align(n):
    return -(-max(n, 1) // 256) * 256


def _need(d):
    """Bytes of the logit tables of all slices (a bf16 router without a split writes none) and of the batch sums' parts behind them."""
    t, NE, blocks = _tables(d), d.N + d.Z, -(-d.T // 16)
    assert t.Tpad >= d.T and t.E >= NE
    return _align(t.slices * t.Tpad * t.E * 4 if t.slices > 1 or d.dtype != zeda.ZEDA_BF16 else 0) + _align(blocks * NE * 4) + _align(blocks * (NE + 1) * 4) + 4


# (T, H, N, Z, K) whose splits write more than 4096 rows of logits
WIDE_SPLITS = [(2048, 2048, 32, 8, 4), (2048, 1536, 48, 16, 4), (1536, 2560, 128, 32, 8), (4096, 4096, 128, 32, 8), (4096, 2048, 224, 32, 8), (1000, 4096, 24, 8, 4),
               (1396, 1536, 48, 10, 6), (2006, 2048, 40, 0, 4), (2006, 2048, 200, 53, 8)]


@pytest.mark.parametrize("shape", WIDE_SPLITS, ids=str)
def test_scratch_holds_the_splits_tables(shape):
    d = _desc(*shape)
    assert zeda.route_train_workspace_bytes(d) >= _need(d)


@pytest.mark.parametrize("H", [128, 512, 1024, 1536, 2048, 2560, 4096, 5120, 6144, 7168, 8192])
def test_scratch_holds_every_split(H):
    """All batch lengths near the ends of blocks and plans, for pools of every number of 32-expert blocks."""
    rng = random.Random(H)
    lengths = sorted({1, 2, 15, 16, 17} | {t + o for t in range(32, 8321, 32) for o in (0, 1, rng.randrange(2, 32))})
    for NE in (1, 24, 32, 33, 40, 64, 65, 96, 128, 136, 160, 192, 193, 224, 253, 256):
        for T in lengths:
            d = _desc(T, H, NE, 0, 1)
            assert zeda.route_train_workspace_bytes(d) >= _need(d), (T, H, NE)


@pytest.mark.parametrize("dtype, H", [("bf16", 2048), ("bf16", 4096), ("f32", 1152)])
def test_scratch_of_a_long_batch_does_for_shorter_ones(dtype, H):
    for N, Z in ((32, 8), (128, 32), (224, 32)):
        sizes = [zeda.route_train_workspace_bytes(_desc(T, H, N, Z, 4, dtype)) for T in range(0, 9000, 7)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), (N, Z)
