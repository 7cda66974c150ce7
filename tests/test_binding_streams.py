"""Buffers that the binding allocates belong to the stream that fills them: torch hands a block freed on one stream to that stream's next
allocation at once, while work on it may still be queued there, so a kernel on another stream must not be given it."""
import contextlib

import pytest
import torch

from paper_2605_18643_amd import zeda

D = zeda.make_desc(40, 256, 128, 3, 2, 2, "bf16")
BF, U8 = torch.bfloat16, torch.uint8
# name: (inputs' shapes and types, call of the inputs on a stream)
CALLS = {
    "quantize_rows": ([((64, 256), BF)], lambda a, s: zeda.zeda_quantize_rows_fp8(*a, stream=s)),
    "quantize_weights": ([((2, 64, 256), BF)], lambda a, s: zeda.zeda_quantize_weights_fp8(*a, stream=s)),
    "pack_fp8": ([((3, 128, 256), U8), ((3, 1, 2), U8)] * 2 + [((3, 256, 128), U8), ((3, 2, 1), U8)], lambda a, s: zeda.zeda_pack_expert_weights_fp8(D, *a, stream=s)),
    "pack": ([((3, 128, 256), BF), ((3, 128, 256), BF), ((3, 256, 128), BF)], lambda a, s: zeda.zeda_pack_expert_weights(D, *a, stream=s)),
    "stats": ([((40, 256), BF), ((5, 256), BF)], lambda a, s: zeda.zeda_routing_stats(D, *a, None, stream=s)),
    "init_rows": ([((5, 256), BF), ((2, 256), torch.float32)], lambda a, s: zeda.zeda_init_zero_expert_rows(D, *a, stream=s)),
}


def _inputs(call, device):
    g = torch.Generator().manual_seed(1)
    return [(torch.randint(0, 127, n, generator=g) if dt == U8 else torch.randn(n, generator=g)).to(dt).to(device) for n, dt in CALLS[call][0]]


@pytest.mark.parametrize("call", CALLS)
def test_allocations_are_made_on_the_callers_stream(call, monkeypatch):
    """On the CPU, with the library's calls and the stream's context replaced by recorders."""
    inside, where = [], []

    @contextlib.contextmanager
    def on(stream):
        inside.append(stream)
        yield
        inside.pop()

    class Library:
        def __getattr__(self, name):
            own = getattr(zeda_lib, name)
            return own if "bytes" in name else lambda *a: zeda.ZEDA_OK

    class Stream:
        cuda_stream = 0

    zeda_lib, side, args = zeda.lib(), Stream(), _inputs(call, "cpu")
    monkeypatch.setattr(zeda, "lib", Library)
    monkeypatch.setattr(zeda, "_stream", lambda stream: 0)
    monkeypatch.setattr(torch.cuda, "stream", on)
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, lambda *a, _f=getattr(torch, name), **k: (where.append(inside[-1] if inside else None), _f(*a, **k))[1])
    CALLS[call][1](args, side)
    assert where and all(w is side for w in where)
    where.clear()
    CALLS[call][1](args, None)  # the current stream: as torch allocates
    assert where and all(w is None for w in where)


@pytest.mark.gpu
@pytest.mark.parametrize("call", CALLS)
def test_results_on_another_stream(call):
    """The same results as on the current stream, in blocks that the current stream has not had."""
    def tensors(r):
        return [r] if isinstance(r, torch.Tensor) else list(r.buffers) if isinstance(r, zeda.Fp8Experts) else list(r)

    args, again = _inputs(call, "cuda"), _inputs(call, "cuda")  # (one of the calls writes into an input)
    want = [t.clone() for t in tensors(CALLS[call][1](args, None))]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    before = [torch.empty_like(t) for t in want]
    had = {t.untyped_storage().data_ptr() for t in before}
    del before
    side.wait_stream(torch.cuda.current_stream())
    got = tensors(CALLS[call][1](again, side))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g.view(torch.uint8), w.view(torch.uint8)) and g.untyped_storage().data_ptr() not in had
