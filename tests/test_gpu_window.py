"""Decode attention with a window and sinks over the 16-bit cache, against its definition in binary64."""
import pytest
import torch

import window_reference as wr

pytestmark = pytest.mark.gpu
INT_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def psa():
    import paper_2503_00392_amd as psa
    psa.load_library()
    assert torch.cuda.is_available()
    return psa


def cache(psa, lens, H, G, dtype, seed, width=None, spare=2):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B = len(lens)
    width = width or max(1, (max(lens) + 15) // 16)
    pages = B * width + spare
    k = torch.randn((pages, H, 16, 128), generator=gen, device="cuda")
    k[:, :, :, ::17] *= 4                                     # a few strong channels
    v = torch.randn((pages, H, 16, 128), generator=gen, device="cuda")
    table = torch.randperm(pages, generator=gen, device="cuda")[: B * width].view(B, width).to(torch.int32)
    q = torch.randn((B, H * G, 128), generator=gen, device="cuda").to(dtype)
    return psa.KvCache(k.to(dtype), v.to(dtype), table, torch.tensor(lens, dtype=torch.int32, device="cuda"), H * G), q


def reference(kv, q, lens, window, sinks, table=None):
    table = (kv.block_table if table is None else table).cpu().long()

    def rows(pool):
        return lambda r, at: pool[table[r, at // 16].cuda(), :, (at % 16).cuda()].transpose(0, 1)
    return wr.attention(q, rows(kv.k_pool), rows(kv.v_pool), lens, window, sinks)


def check(psa, kv, q, lens, window, sinks, where=""):
    out, lse = psa.window_attention(kv, q, window, sinks)
    torch.cuda.synchronize()
    assert psa.read_device_error(out._workspace) == 0, where
    wr.close(out, lse, *reference(kv, q, lens, window, sinks), where=(where, window, sinks))
    return out, lse


LENS = [0, 1, 15, 16, 17, 31, 64, 100, 333, 1000]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("H", [1, 3])
def test_windows_and_sinks(psa, dtype, G, H):
    kv, q = cache(psa, LENS, H, G, dtype, seed=G * 10 + H)
    for window, sinks in [(0, 0), (0, 5), (0, INT_MAX), (1, 0), (1, 1), (15, 16), (16, 17), (17, 0), (50, 33), (100, 400), (999, 0), (1000, 3),
                          (500, 500), (INT_MAX, 0), (INT_MAX, INT_MAX)]:
        check(psa, kv, q, LENS, window, sinks)


@pytest.mark.parametrize("dtype,G", [(torch.float16, 8), (torch.bfloat16, 8), (torch.bfloat16, 4), (torch.float16, 1)])
def test_many_splits_and_one(psa, dtype, G):
    """One long request (as many splits as there are), and more (request, KV head) pairs than are ever split."""
    kv, q = cache(psa, [20011], 1, G, dtype, seed=5)
    for window, sinks in [(INT_MAX, 0), (9000, 70), (129, 4)]:
        check(psa, kv, q, [20011], window, sinks)
    lens = [(37 * i) % 150 for i in range(400)]
    kv, q = cache(psa, lens, 6, G, dtype, seed=6)
    for window, sinks in [(INT_MAX, 0), (33, 2)]:
        check(psa, kv, q, lens, window, sinks)


@pytest.mark.parametrize("few", [True, False])
def test_what_is_not_visible_is_not_looked_at(psa, few):
    """NaN in every token that is not visible, no page at all where a block holds none."""
    lens, window, sinks = ([700, 1603] if few else [90 + i % 40 for i in range(300)]), 45, 20
    kv, q = cache(psa, lens, 2 if few else 8, 4, torch.bfloat16, seed=7)
    want = reference(kv, q, lens, window, sinks)
    table = kv.block_table.clone()
    for r, ctx in enumerate(lens if few else lens[:4]):
        seen = wr.visible(ctx, window, sinks)
        for b in range(table.shape[1]):
            inside = torch.zeros(16, dtype=torch.bool)
            part = seen[16 * b:16 * b + 16]
            inside[: part.numel()] = part
            if not inside.any():
                table[r, b] = -12345
            else:
                page = int(kv.block_table[r, b])
                kv.k_pool[page, :, ~inside.cuda()] = float("nan")
                kv.v_pool[page, :, ~inside.cuda()] = float("inf")
    kv.block_table = table
    out, lse = psa.window_attention(kv, q, window, sinks)
    torch.cuda.synchronize()
    assert psa.read_device_error(out._workspace) == 0
    wr.close(out, lse, *want)


def test_numbers_that_are_none(psa):
    """A visible NaN shows in the heads of its KV head and nowhere else, whether it is the only token or one of many; logits
    of -inf count for nothing."""
    lens = [1, 200, 200, 200]
    kv, q = cache(psa, lens, 2, 2, torch.float16, seed=8)
    table = kv.block_table.cpu().long()
    kv.k_pool[table[0, 0], 0, 0, 3] = float("nan")
    kv.v_pool[table[1, 12], 1, 5, 9] = float("nan")
    q[3, 0] = float("nan")
    for window, sinks in [(INT_MAX, 0), (20, 0)]:
        out, lse = psa.window_attention(kv, q, window, sinks)
        want = reference(kv, q, lens, window, sinks)
        assert torch.isnan(out[0, :2]).all() and torch.isnan(lse[0, :2]).all() and not torch.isnan(out[0, 2:]).any()
        assert torch.isnan(out[1, 2:, 9]).all() and int(torch.isnan(out[1]).sum()) == 2 and not torch.isnan(lse[1]).any()
        assert torch.isnan(out[3, 0]).all() and torch.isnan(lse[3, 0]) and not torch.isnan(out[3, 1:]).any()
        wr.close(out[2:3], lse[2:3], want[0][2:3], want[1][2:3])
    big = torch.zeros((1, 4, 128), dtype=torch.float16, device="cuda")
    one, _ = cache(psa, [48], 2, 2, torch.float16, seed=9)
    big[:] = 60000.0
    one.k_pool[:] = -60000.0                                  # logits of -4e10: finite
    one.k_pool[one.block_table[0, 1].long(), :, 4] = 0.0
    out, lse = psa.window_attention(one, big, INT_MAX)
    assert torch.equal(out.view(2, 2, 128), one.v_pool[one.block_table[0, 1].long(), :, 4].float()[:, None].expand(2, 2, 128))
    assert not lse.any()


@pytest.mark.parametrize("many", [False, True])
def test_bad_pages_and_lengths_are_reported(psa, many):
    """Both ways of a call (with and without a launch that joins splits); the word is of the last call."""
    lens = [40, 100] if not many else [40, 100] * 600
    kv, q = cache(psa, lens, 2, 4, torch.float16, seed=11)
    good = kv.block_table.clone(), kv.ctx_lens.clone()
    ws = torch.empty(psa.window_workspace_bytes(kv, 30, 0), dtype=torch.uint8, device="cuda")
    def word():
        psa.window_attention(kv, q, 30, 0, workspace=ws)
        return psa.read_device_error(ws)
    assert word() == 0
    kv.block_table[1, 6] = kv.k_pool.shape[0]
    assert word() == 1
    kv.block_table.copy_(good[0])
    kv.block_table[1, 0] = -1                                 # not visible
    assert word() == 0
    kv.ctx_lens[0] = -3
    assert word() == 2
    kv.ctx_lens[0] = 16 * kv.block_table.shape[1] + 1
    assert word() == 2
    kv.block_table[len(lens) - 1, 5] = -7
    assert word() == 3
    kv.block_table.copy_(good[0]); kv.ctx_lens.copy_(good[1])
    assert word() == 0


def test_a_pool_without_pages(psa):
    empty = torch.empty((0, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    kv = psa.KvCache(empty, empty, torch.zeros((3, 2), dtype=torch.int32, device="cuda"),
                     torch.tensor([0, 5, 0], dtype=torch.int32, device="cuda"), 8)
    out, lse = psa.window_attention(kv, torch.randn((3, 8, 128), device="cuda").bfloat16(), 4, 4)
    torch.cuda.synchronize()
    assert psa.read_device_error(out._workspace) == 1 and not out.any() and torch.isneginf(lse).all()


def test_a_cache_beyond_4_gib(psa):
    pages = (1 << 32) // (8 * 4096) + 64
    k, v = (torch.empty((pages, 8, 16, 128), dtype=torch.float16, device="cuda") for _ in range(2))
    table = torch.arange(pages - 20, pages, device="cuda", dtype=torch.int32).view(2, 10)
    k[pages - 20:].normal_(); v[pages - 20:].normal_()
    k[:64] = float("nan")
    kv = psa.KvCache(k, v, table, torch.tensor([150, 160], dtype=torch.int32, device="cuda"), 16)
    check(psa, kv, torch.randn((2, 16, 128), device="cuda").half(), [150, 160], 100, 3)


def test_agrees_with_the_dense_control_and_repeats_bit_for_bit(psa):
    lens = [5000, 17, 2048]
    kv, q = cache(psa, lens, 4, 4, torch.bfloat16, seed=12)
    dense, dense_lse = psa.dense_attention(kv, q)
    out, lse = psa.window_attention(kv, q, 5000)
    again, again_lse = psa.window_attention(kv, q, 5000)
    assert torch.equal(out, again) and torch.equal(lse, again_lse)
    assert ((out - dense).norm(dim=-1) / dense.norm(dim=-1)).max() <= 2e-5 and (lse - dense_lse).abs().max() <= 2e-5


def test_host_tier(psa):
    """Pools in pinned host memory: read from where they are."""
    kv, q = cache(psa, [200, 33], 2, 4, torch.float16, seed=13)
    want = psa.window_attention(kv, q, 64, 5)
    host = psa.KvCache(kv.k_pool.cpu().pin_memory(), kv.v_pool.cpu().pin_memory(), kv.block_table, kv.ctx_lens, 8,
                       tier=psa.Tier(kv.k_pool.shape[0] * 2, 8))
    got = psa.window_attention(host, q, 64, 5)
    torch.cuda.synchronize()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("B,H,G", [(5, 8, 4), (64, 2, 8), (65, 1, 1), (70, 5, 2), (256, 1, 4), (257, 3, 8), (600, 1, 4), (1030, 1, 2)])
def test_one_long_request_among_short_ones(psa, B, H, G):
    """Pieces: a long request is cut into many, the others are one each, some requests are empty; batches about the sizes where a
    workgroup finds its piece in another way."""
    lens = [(i * 31) % 97 for i in range(B)]
    lens[B // 2], lens[-1] = 6000, 2307
    kv, q = cache(psa, lens[:1], H, G, torch.bfloat16, seed=B, width=1)
    gen = torch.Generator(device="cuda").manual_seed(B)
    k, v = (torch.randn((700, H, 16, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    table = torch.randint(0, 700, (B, 375), generator=gen, device="cuda", dtype=torch.int32)
    q = torch.randn((B, H * G, 128), generator=gen, device="cuda").bfloat16()
    kv = psa.KvCache(k, v, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), H * G)
    for window, sinks in [(INT_MAX, 0), (2500, 100)]:
        out, lse = check(psa, kv, q, lens, window, sinks)
        again = psa.window_attention(kv, q, window, sinks)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    table[B // 2, 374] = -1                                   # in the long one's last piece
    kv.ctx_lens[0] = -1                                       # of a request without a piece
    out, _ = psa.window_attention(kv, q, INT_MAX)
    assert psa.read_device_error(out._workspace) == 3


def test_so_many_requests_that_no_pieces_are_listed(psa):
    B, width = 66000, 40
    gen = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn((64, 1, 16, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    table = torch.randint(0, 64, (B, width), generator=gen, device="cuda", dtype=torch.int32)
    lens = torch.randint(0, 40, (B,), generator=gen, device="cuda", dtype=torch.int32)
    lens[-3:] = torch.tensor([640, 0, 333])
    q = torch.randn((B, 1, 128), generator=gen, device="cuda").bfloat16()
    out, lse = psa.window_attention(psa.KvCache(k, v, table, lens, 1), q, INT_MAX)
    assert psa.read_device_error(out._workspace) == 0
    for part in (slice(0, 50), slice(B - 50, B)):
        some = psa.KvCache(k, v, table[part], lens[part], 1)
        wr.close(out[part], lse[part], *reference(some, q[part], lens[part].tolist(), INT_MAX, 0))


def test_so_many_requests_that_no_workgroup_checks_the_tables(psa):
    B = 9000
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((50, 1, 16, 128), generator=gen, device="cuda").half() for _ in range(2))
    table = torch.randint(0, 50, (B, 1), generator=gen, device="cuda", dtype=torch.int32)
    lens = torch.randint(0, 17, (B,), generator=gen, device="cuda", dtype=torch.int32)
    q = torch.randn((B, 2, 128), generator=gen, device="cuda").half()
    kv = psa.KvCache(k, v, table, lens, 2)
    out, lse = psa.window_attention(kv, q, 9, 2)
    assert psa.read_device_error(out._workspace) == 0
    for part in (slice(0, 60), slice(B - 60, B)):
        some = psa.KvCache(k, v, table[part], lens[part], 2)
        wr.close(out[part], lse[part], *reference(some, q[part], lens[part].tolist(), 9, 2))
    table[8765] = 50
    lens[8765] = 5
    assert psa.read_device_error(psa.window_attention(kv, q, 9, 2, workspace=out._workspace)[0]._workspace) == 1
    table[8765] = 0
    lens[17] = 99
    assert psa.read_device_error(psa.window_attention(kv, q, 9, 2, workspace=out._workspace)[0]._workspace) == 2
    lens[17] = 3
    assert psa.read_device_error(psa.window_attention(kv, q, 9, 2, workspace=out._workspace)[0]._workspace) == 0
