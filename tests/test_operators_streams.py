"""Buffers that a call with stream= makes for itself: taken from that stream's memory, kept until the current stream has read them.
The allocator is watched on the CPU; the last test runs on a GPU."""
import contextlib
import types

import pytest
import torch

import paper_2503_00392_amd as psa
from paper_2503_00392_amd import binding as pb

B, H, G = 3, 2, 4


def tensors(device):
    new = lambda *shape: torch.randn(shape).bfloat16().to(device)   # noqa: E731
    table = torch.arange(2 * B, dtype=torch.int32, device=device).view(B, 2)
    lens = torch.tensor([20, 32, 1], dtype=torch.int32, device=device)
    kv = psa.KvCache(new(2 * B, H, 16, 128), new(2 * B, H, 16, 128), table, lens, H * G)
    packed = psa.PackedCache(psa.PackedCache.empty_pool(2 * B, H, device=device), table, lens, H * G, torch.bfloat16)
    freq = torch.ones(64, device=device)
    q, k = new(B, H * G, 128), new(B, H, 128)
    return {"window": lambda **kw: psa.window_attention(kv, q, 20, 1, **kw), "packed": lambda **kw: psa.packed_attention(packed, q, **kw),
            "rotate": lambda **kw: psa.norm_rotate(q, k, lens, freq, **kw)}


@pytest.mark.parametrize("name", ["window", "packed", "rotate"])
@pytest.mark.parametrize("given", [True, False])
def test_buffers_come_from_the_stream_that_writes_them(monkeypatch, name, given):
    side, here = (types.SimpleNamespace(device=types.SimpleNamespace(index=-1)) for _ in range(2))      # (as CPU tensors say)
    at_work, made, kept, launched = [here], [], [], []

    @contextlib.contextmanager
    def on(stream):
        at_work.append(stream)
        yield
        at_work.pop()

    plain = torch.empty

    def empty(shape, dtype, device):
        made.append(at_work[-1])
        return plain(shape, dtype=dtype)

    call = tensors("cpu")[name]
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: at_work[-1])
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: kept.append(stream))
    monkeypatch.setattr(pb, "_device_of", lambda t: -1)
    monkeypatch.setattr(pb, "_launch", lambda call, at, stream, *args: launched.append(stream))
    call(stream=side if given else None)
    assert launched == [side if given else None]
    assert len(made) == (2 if name == "rotate" else 3) and all(s is (side if given else here) for s in made)
    assert len(kept) == (len(made) if given else 0) and all(s is here for s in kept)
    made.clear()
    side.device = types.SimpleNamespace(index=5)             # a stream of another GPU: refused before anything is made
    if given:
        with pytest.raises(ValueError, match="the stream is of"):
            call(stream=side)
        assert not made


def test_the_error_word_is_read_behind_the_calls_of_its_own_gpu(monkeypatch):
    """The calls run on the current stream of the tensors' GPU, whichever GPU is the current one; so does the read of their error word."""
    asked = []

    def current_stream(device=None):
        asked.append(device)
        return types.SimpleNamespace(cuda_stream=1)

    class Library:
        psa_read_device_error = staticmethod(lambda workspace, flags, stream: pb.PSA_OK)

    monkeypatch.setattr(torch.cuda, "current_stream", current_stream)
    monkeypatch.setattr(pb, "load_library", lambda: Library)
    workspace = torch.empty(256, dtype=torch.uint8, device="meta")
    assert psa.read_device_error(workspace) == 0 and asked == [workspace.device]


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["window", "packed", "rotate"])
def test_memory_let_go_behind_running_work_is_not_written(name):
    """Buffers of the results' sizes are in use by work queued on the current stream and let go by the host: a call on another
    stream that makes its own leaves them alone, and its results are those of a call on the current stream."""
    call = tensors("cuda")[name]
    want = [x.clone() for x in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    old = [torch.full_like(x, 7) for x in want for _ in range(3)]
    seen = [torch.empty_like(x) for x in old]
    addresses = {x.data_ptr() for x in old}
    torch.cuda._sleep(20_000_000)                             # some 10 ms
    for x, y in zip(old, seen):
        y.copy_(x)
    del old, x
    got = call(stream=side)
    assert not addresses & {x.data_ptr() for x in got}
    torch.cuda.synchronize()
    assert all(bool((y == 7).all()) for y in seen)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
