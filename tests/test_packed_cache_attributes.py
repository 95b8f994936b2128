"""A PackedCache whose attributes are assigned anew: calls see what it holds now.  The descriptor on the CPU, results on a GPU."""
import copy

import pytest
import torch

import paper_2503_00392_amd as psa
from paper_2503_00392_amd import binding as pb


def make(device="cpu", B=2, P=8, H=2, Hq=8):
    table, lens = torch.zeros((B, 4), dtype=torch.int32, device=device), torch.zeros(B, dtype=torch.int32, device=device)
    return psa.PackedCache(psa.PackedCache.empty_pool(P, H, device=device), table, lens, Hq, torch.bfloat16)


def launched(monkeypatch, call):
    """The arguments that a call would have handed to the library."""
    got = []
    monkeypatch.setattr(pb, "_device_of", lambda t: -1)
    monkeypatch.setattr(pb, "_launch", lambda call, at, stream, *args: got.append(args))
    call()
    return got[0]


def attend(cache):
    B, Hq = cache.block_table.shape[0], cache.num_q_heads
    q = torch.zeros((B, Hq, 128), dtype=cache.dtype)
    return lambda: psa.packed_attention(cache, q, 4, 1, workspace=torch.empty(1 << 16, dtype=torch.uint8), out=torch.empty(q.shape), lse=torch.empty(q.shape[:2]))


def append(cache):
    k = torch.zeros((cache.block_table.shape[0], cache.num_kv_heads, 128), dtype=cache.dtype)
    return lambda: psa.append_kv_packed(cache, k, k)


@pytest.mark.parametrize("call", [attend, append])
def test_calls_use_what_was_assigned_last(monkeypatch, call):
    cache = make()
    before = launched(monkeypatch, call(cache))
    assert launched(monkeypatch, call(cache))[0] is before[0]            # (made once)
    cache.ctx_lens = torch.ones(2, dtype=torch.int32)
    cache.block_table = torch.zeros((2, 9), dtype=torch.int32)
    cache.pool = psa.PackedCache.empty_pool(5, 4, device="cpu")
    cache.num_q_heads, cache.dtype = 16, torch.float16
    d, pool, *_ = launched(monkeypatch, call(cache))
    assert (d.ctx_lens, d.block_table, pool) == (cache.ctx_lens.data_ptr(), cache.block_table.data_ptr(), cache.pool.data_ptr())
    assert (d.batch, d.max_blocks_per_seq, d.num_pages, d.num_kv_heads, d.num_q_heads, d.dtype) == (2, 9, 5, 4, 16, pb.PSA_F16)
    assert cache.num_kv_heads == 4
    cache.block_table, cache.ctx_lens = torch.zeros((3, 9), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)      # another batch
    assert launched(monkeypatch, call(cache))[0].batch == 3


def test_workspaces_follow_assignments():
    cache = make()
    small = psa.packed_workspace_bytes(cache)
    cache.block_table = torch.zeros((2, 8000), dtype=torch.int32)
    assert psa.packed_workspace_bytes(cache) > small
    assert psa.packed_workspace_bytes(cache) == psa.packed_workspace_bytes(psa.PackedCache(cache.pool, cache.block_table, cache.ctx_lens, 8, torch.bfloat16))


@pytest.mark.parametrize("name,value,error", [
    ("pool", torch.zeros((8, 2, 2175), dtype=torch.uint8), "pool"), ("pool", torch.zeros((8, 2176), dtype=torch.uint8), "pool"),
    ("pool", torch.zeros((8, 2, 2176), dtype=torch.int8), "pool"), ("block_table", torch.zeros((2, 4)), "block_table"),
    ("block_table", torch.zeros((4, 2), dtype=torch.int32).t(), "block_table"), ("block_table", torch.zeros((3, 4), dtype=torch.int32), "ctx_lens"),
    ("ctx_lens", torch.zeros(3, dtype=torch.int32), "ctx_lens"), ("ctx_lens", torch.zeros(2, dtype=torch.int64), "ctx_lens")])
def test_assignments_that_do_not_fit_are_refused_by_the_next_call(monkeypatch, name, value, error):
    cache = make()
    setattr(cache, name, value)
    k = torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    for call in (attend(cache), lambda: psa.append_kv_packed(cache, k, k), lambda: psa.packed_workspace_bytes(cache)):
        with pytest.raises(ValueError, match=error):
            launched(monkeypatch, call)


def test_copies_are_assigned_apart_and_heads_follow_the_pool():
    cache = make()
    other = copy.copy(cache)
    other.ctx_lens = torch.ones(2, dtype=torch.int32)
    assert cache._desc is not None and cache._made().ctx_lens == cache.ctx_lens.data_ptr() and other._made().ctx_lens == other.ctx_lens.data_ptr()
    with pytest.raises(AttributeError):
        cache.num_kv_heads = 4
    cache.layer = 3                                           # (what a program keeps beside it is its own)
    assert cache._desc is not None


@pytest.mark.gpu
def test_results_follow_assignments():
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *shape: torch.randn(shape, generator=gen, device="cuda").half()   # noqa: E731
    none = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    pools = [psa.pack_pages(psa.KvCache(new(12, 2, 16, 128), new(12, 2, 16, 128), none, none[0], 4), psa.PackedCache.empty_pool(12, 2)) for _ in range(2)]
    tables = [torch.randperm(12, generator=gen, device="cuda").view(2, 6).to(torch.int32) for _ in range(2)]
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([90, 17], [3, 96])]
    q = new(2, 4, 128)
    cache = psa.PackedCache(pools[0], tables[0], lens[0], 4, torch.float16)
    psa.packed_attention(cache, q)
    for i in range(8):
        cache.pool, cache.block_table, cache.ctx_lens = pools[i & 1], tables[i >> 1 & 1], lens[i >> 2]
        got = psa.packed_attention(cache, q)
        want = psa.packed_attention(psa.PackedCache(pools[i & 1], tables[i >> 1 & 1], lens[i >> 2], 4, torch.float16), q)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
