"""The paged cache in 4 bits: records against a plain numpy packer bit by bit, attention against binary64 over the values
that the records stand for."""
import numpy as np
import pytest
import torch

import packed_reference as pr
import window_reference as wr

pytestmark = pytest.mark.gpu
INT_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def psa():
    import paper_2503_00392_amd as psa
    psa.load_library()
    assert torch.cuda.is_available()
    return psa


def sixteen(psa, k, v):
    none = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    return psa.KvCache(k, v, none, none[0], k.shape[1])


def awkward(dtype, seed, pages=3, H=2):
    """Blocks of every size of number that the type has, with ties, saturation, zeros, infinities and NaN among them."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((pages, H, 16, 4, 32))
    lowest, highest = (-24, 15) if dtype == torch.float16 else (-133, 127)
    x *= 2.0 ** rng.integers(lowest - 2, highest - 1, size=x.shape[:-1])[..., None].astype(float)
    x[0, 0, 0, 0] = 0
    x[0, 0, 1, 0, :16] = [7, 6.5, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25, -0.75, -5, -7, -0.0, 6, 0.1]
    x[0, 0, 1, 0, 16:] = 0
    x[0, 0, 2, 1, :4] = [7.0625, -7, 3.5, 1.5]
    x[0, 0, 2, 1, 4:] = 0
    x[0, 1, 3, 2, 7], x[0, 1, 4, 3, 0], x[0, 1, 5, 0, 31] = np.inf, -np.inf, np.nan
    x[0, 1, 6, 1] = float(torch.finfo(dtype).max)
    x[0, 1, 7, 1] = -float(torch.finfo(dtype).tiny) * 2.0 ** (-10 if dtype == torch.float16 else -7)     # the least subnormal
    return torch.from_numpy(x.reshape(pages, H, 16, 128)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_records_are_what_the_definition_says(psa, dtype):
    k, v = awkward(dtype, 1), awkward(dtype, 2)
    pool = psa.PackedCache.empty_pool(3, 2).fill_(0x5a)
    psa.pack_pages(sixteen(psa, k, v), pool)
    got = pool.cpu().numpy()
    kd, vd = k.double().cpu().numpy(), v.double().cpu().numpy()
    for p in range(3):
        for h in range(2):
            want = pr.pack_record(kd[p, h], vd[p, h])
            bad = np.flatnonzero(got[p, h] != want)
            assert bad.size == 0, (p, h, bad[:8], got[p, h][bad[:8]], want[bad[:8]])
    back = [torch.zeros_like(k), torch.zeros_like(v)]
    psa.unpack_pages(sixteen(psa, *back), pool)
    for x, y in zip(back, pr.unpack(got)):
        y = torch.from_numpy(y).to(dtype).cuda()
        # bfloat16's subnormals (below 2^-126) may come back as zeros
        same = (x == y) | (torch.isnan(x) & torch.isnan(y))
        if dtype == torch.bfloat16:
            same |= (x == 0) & (y.abs() < 2.0 ** -126)
        assert same.all(), (x[~same][:5], y[~same][:5])


def test_lists_and_fills(psa):
    k, v = (torch.randn((9, 3, 16, 128), device="cuda").half() for _ in range(2))
    whole = psa.pack_pages(sixteen(psa, k, v), psa.PackedCache.empty_pool(9, 3))
    some = psa.PackedCache.empty_pool(9, 3).fill_(0x77)
    lst = torch.tensor([4, 0, 4, -1, 9, 7], dtype=torch.int32, device="cuda")          # one twice, two outside the pool
    psa.pack_pages(sixteen(psa, k, v), some, page_list=lst)
    for p in range(9):
        assert torch.equal(some[p], whole[p]) if p in (4, 0, 7) else bool((some[p] == 0x77).all())
    kb, vb = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
    psa.unpack_pages(sixteen(psa, kb, vb), whole, page_list=lst)
    full = [x.numpy() for x in (kb.cpu(), vb.cpu())]
    for got, want in zip(full, pr.unpack(whole.cpu().numpy())):
        for p in range(9):
            assert np.array_equal(got[p], want[p].astype(np.float16)) if p in (4, 0, 7) else (got[p] == 9).all()
    fill = torch.tensor([16, 0, 5, 1, 15, 99, -4, 16, 8], dtype=torch.int32, device="cuda")
    zeroed = [x.clone() for x in (k, v)]
    dirty = [x.clone() for x in (k, v)]
    for p, n in enumerate(fill.clamp(0, 16).tolist()):
        for x in zeroed:
            x[p, :, n:] = 0
        for x in dirty:
            x[p, :, n:] = float("nan")
    want = psa.pack_pages(sixteen(psa, *zeroed), psa.PackedCache.empty_pool(9, 3))
    assert torch.equal(psa.pack_pages(sixteen(psa, *dirty), psa.PackedCache.empty_pool(9, 3), page_fill=fill), want)


@pytest.mark.parametrize("dtype,H", [(torch.float16, 1), (torch.bfloat16, 8), (torch.bfloat16, 5), (torch.float16, 24)])
def test_appended_tokens_are_packed_as_pages_are(psa, dtype, H):
    """Three requests, tokens one by one over page borders; one row of the table fills up, one entry is outside the pool."""
    width, steps = 3, 37
    start = [0, 12, 11]
    table = torch.tensor([[5, 2, 7], [1, 6, 8], [0, 99, 4]], dtype=torch.int32, device="cuda")
    k, v = (torch.zeros((9, H, 16, 128), dtype=dtype, device="cuda") for _ in range(2))
    cache = psa.PackedCache(psa.PackedCache.empty_pool(9, H), table, torch.tensor(start, dtype=torch.int32, device="cuda"), H, dtype)
    status = torch.full((3,), -1, dtype=torch.int32, device="cuda")
    n = list(start)
    for step in range(steps):
        kn, vn = (torch.randn((3, H, 128), device="cuda").mul_(2.0 ** (step % 9)).to(dtype) for _ in range(2))
        psa.append_kv_packed(cache, kn, vn, status)
        want = []
        for r in range(3):
            page = int(table[r, n[r] // 16]) if n[r] < 16 * width else None
            if page is None or page == 99:
                want.append(2 if page is None else 1)
                continue
            k[page, :, n[r] % 16], v[page, :, n[r] % 16] = kn[r], vn[r]
            n[r] += 1
            want.append(0)
        assert status.tolist() == want
    assert cache.ctx_lens.tolist() == n == [37, 48, 16]
    got = cache.pool.clone()
    expect = psa.pack_pages(sixteen(psa, k, v), psa.PackedCache.empty_pool(9, H))
    back = [pr.unpack(x.cpu().numpy()) for x in (got, expect)]
    for a, b in zip(*back):
        assert np.array_equal(a, b)
    for r in range(3):                                        # pages appended whole: the very bytes (in a pool that was
        for b in range((start[r] + 15) // 16, n[r] // 16):    # never written a zero block's power byte is 0, packed it is 1)
            assert torch.equal(got[int(table[r, b])], expect[int(table[r, b])])


def cache(psa, lens, H, G, dtype, seed, spare=2):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, width = len(lens), max(1, (max(lens) + 15) // 16)
    pages = B * width + spare
    k, v = (torch.randn((pages, H, 16, 128), generator=gen, device="cuda") for _ in range(2))
    k[:, :, :, ::17] *= 4
    v *= torch.exp2(torch.randint(-3, 4, (pages, H, 16, 4), generator=gen, device="cuda").float()).repeat_interleave(32, -1)
    pool = psa.pack_pages(sixteen(psa, k.to(dtype), v.to(dtype)), psa.PackedCache.empty_pool(pages, H))
    table = torch.randperm(pages, generator=gen, device="cuda")[: B * width].view(B, width).to(torch.int32)
    q = torch.randn((B, H * G, 128), generator=gen, device="cuda").to(dtype)
    return psa.PackedCache(pool, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), H * G, dtype), q


def reference(kv, q, lens, window, sinks):
    table = kv.block_table.cpu().long()
    raw = kv.pool

    def rows(which):
        def get(r, at):
            pages, inverse = torch.unique(table[r, at // 16], return_inverse=True)
            x = torch.from_numpy(pr.unpack(raw[pages.cuda()].cpu().numpy())[which])
            return x[inverse, :, at % 16].transpose(0, 1)
        return get
    return wr.attention(q, rows(0), rows(1), lens, window, sinks)


def check(psa, kv, q, lens, window, sinks, where=""):
    out, lse = psa.packed_attention(kv, q, window, sinks)
    torch.cuda.synchronize()
    assert psa.read_device_error(out._workspace) == 0, where
    wr.close(out, lse, *reference(kv, q, lens, window, sinks), where=(where, window, sinks))


LENS = [0, 1, 15, 16, 17, 31, 64, 100, 333, 1000]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("H", [1, 3])
def test_attention_over_records(psa, dtype, G, H):
    kv, q = cache(psa, LENS, H, G, dtype, seed=G * 10 + H)
    for window, sinks in [(INT_MAX, 0), (0, 0), (0, 5), (1, 0), (15, 16), (16, 17), (17, 0), (50, 33), (999, 0), (500, 500)]:
        check(psa, kv, q, LENS, window, sinks)


@pytest.mark.parametrize("dtype,G", [(torch.float16, 8), (torch.bfloat16, 8), (torch.bfloat16, 4), (torch.float16, 1)])
def test_many_splits_and_one(psa, dtype, G):
    kv, q = cache(psa, [20011], 1, G, dtype, seed=5)
    for window, sinks in [(INT_MAX, 0), (9000, 70), (129, 4)]:
        check(psa, kv, q, [20011], window, sinks)
    lens = [(37 * i) % 150 for i in range(400)]
    kv, q = cache(psa, lens, 6, G, dtype, seed=6)
    for window, sinks in [(INT_MAX, 0), (33, 2)]:
        check(psa, kv, q, lens, window, sinks)


@pytest.mark.parametrize("few", [True, False])
def test_what_is_not_visible_is_not_looked_at(psa, few):
    """All ones (elements -6 under a power of NaN) in every token that is not visible, no page where a block holds none."""
    lens, window, sinks = ([700, 1603] if few else [90 + i % 40 for i in range(300)]), 45, 20
    kv, q = cache(psa, lens, 2 if few else 8, 4, torch.bfloat16, seed=7)
    want = reference(kv, q, lens, window, sinks)
    table = kv.block_table.cpu()
    for r, ctx in enumerate(lens if few else lens[:4]):
        seen = wr.visible(ctx, window, sinks)
        for b in range(table.shape[1]):
            part = seen[16 * b:16 * b + 16].tolist()
            page = int(table[r, b])
            if not any(part):
                kv.block_table[r, b] = -12345
                continue
            for t in range(16):
                if t >= len(part) or not part[t]:
                    rec = kv.pool[page]
                    rec[:, t * 64:t * 64 + 64] = 255
                    rec[:, 1024:2048].view(-1, 4, 16, 4, 4)[:, t // 4, :, t % 4] = 255
                    rec[:, 2048 + 4 * t:2052 + 4 * t] = 255
                    rec[:, 2112 + t::16] = 255
    out, lse = psa.packed_attention(kv, q, window, sinks)
    torch.cuda.synchronize()
    assert psa.read_device_error(out._workspace) == 0
    wr.close(out, lse, *want)


def test_blocks_that_are_no_numbers(psa):
    """A NaN power of a visible key makes its heads' rows NaN, one of a visible value 32 channels of them."""
    lens = [1, 200, 200]
    kv, q = cache(psa, lens, 2, 2, torch.float16, seed=8)
    table = kv.block_table.cpu().long()
    kv.pool[table[0, 0], 0, 2048 + 2] = 255                   # key, token 0, channels 64 .. 95
    kv.pool[table[1, 12], 1, 2112 + 3 * 16 + 5] = 255         # value, token 5, channels 96 .. 127
    for window in (INT_MAX, 20):
        out, lse = psa.packed_attention(kv, q, window)
        want = reference(kv, q, lens, window, 0)
        assert torch.isnan(out[0, :2]).all() and torch.isnan(lse[0, :2]).all() and not torch.isnan(out[0, 2:]).any()
        assert torch.isnan(out[1, 2:, 96:]).all() and int(torch.isnan(out[1]).sum()) == 64 and not torch.isnan(lse[1]).any()
        wr.close(out[2:], lse[2:], want[0][2:], want[1][2:])


@pytest.mark.parametrize("many", [False, True])
def test_bad_pages_and_lengths_are_reported(psa, many):
    lens = [40, 100] if not many else [40, 100] * 600
    kv, q = cache(psa, lens, 2, 4, torch.float16, seed=11)
    good = kv.block_table.clone(), kv.ctx_lens.clone()
    ws = torch.empty(psa.packed_workspace_bytes(kv, 30, 0), dtype=torch.uint8, device="cuda")
    def word():
        psa.packed_attention(kv, q, 30, 0, workspace=ws)
        return psa.read_device_error(ws)
    assert word() == 0
    kv.block_table[1, 6] = kv.pool.shape[0]
    assert word() == 1
    kv.block_table.copy_(good[0])
    kv.block_table[1, 0] = -1                                 # not visible
    assert word() == 0
    kv.ctx_lens[0] = 16 * kv.block_table.shape[1] + 1
    assert word() == 2
    kv.block_table[len(lens) - 1, 5] = -7
    assert word() == 3
    kv.block_table.copy_(good[0]); kv.ctx_lens.copy_(good[1])
    assert word() == 0


def test_a_pool_without_pages(psa):
    kv = psa.PackedCache(psa.PackedCache.empty_pool(0, 2), torch.zeros((3, 2), dtype=torch.int32, device="cuda"),
                         torch.tensor([0, 5, 0], dtype=torch.int32, device="cuda"), 8, torch.bfloat16)
    out, lse = psa.packed_attention(kv, torch.randn((3, 8, 128), device="cuda").bfloat16(), 4, 4)
    torch.cuda.synchronize()
    assert psa.read_device_error(out._workspace) == 1 and not out.any() and torch.isneginf(lse).all()


def test_a_cache_beyond_4_gib(psa):
    pages = (1 << 32) // (8 * 2176) + 64
    small, q = cache(psa, [150, 160], 8, 2, torch.float16, seed=14, spare=0)
    pool = torch.empty((pages, 8, 2176), dtype=torch.uint8, device="cuda")
    pool[:64] = 255
    pool[pages - 20:] = small.pool
    big = psa.PackedCache(pool, (small.block_table + (pages - 20)).contiguous(), small.ctx_lens, 16, torch.float16)
    check(psa, big, q, [150, 160], 100, 3)
    kn, vn = (torch.randn((2, 8, 128), device="cuda").half() for _ in range(2))
    status = torch.full((2,), -1, dtype=torch.int32, device="cuda")
    psa.append_kv_packed(big, kn, vn, status)
    assert status.tolist() == [0, 2] and big.ctx_lens.tolist() == [151, 160]
    check(psa, big, q, [151, 160], 100, 3)


def test_repeats_bit_for_bit(psa):
    kv, q = cache(psa, [5000, 17, 2048], 4, 8, torch.bfloat16, seed=12)
    first = psa.packed_attention(kv, q)
    again = psa.packed_attention(kv, q)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("B,H,G", [(5, 8, 4), (64, 2, 8), (65, 1, 1), (300, 3, 2)])
def test_one_long_request_among_short_ones(psa, B, H, G):
    lens = [(i * 31) % 97 for i in range(B)]
    lens[B // 2], lens[-1] = 9000, 2307
    small, _ = cache(psa, [16 * 64], H, 1, torch.float16, seed=B)
    gen = torch.Generator(device="cuda").manual_seed(B)
    table = torch.randint(0, small.pool.shape[0], (B, 563), generator=gen, device="cuda", dtype=torch.int32)
    q = torch.randn((B, H * G, 128), generator=gen, device="cuda").half()
    kv = psa.PackedCache(small.pool, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), H * G, torch.float16)
    for window, sinks in [(INT_MAX, 0), (2500, 100)]:
        check(psa, kv, q, lens, window, sinks)
    table[B // 2, 562] = small.pool.shape[0]
    kv.ctx_lens[0] = -1
    out, _ = psa.packed_attention(kv, q)
    assert psa.read_device_error(out._workspace) == 3
