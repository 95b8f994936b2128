"""Attention with a window and sinks over keys and values that are infinite."""
import pytest
import torch

import paper_2503_00392_amd as psa
import window_reference as wr

pytestmark = pytest.mark.gpu
INF = float("inf")


def cache(dtype, lens, H, G, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, width = len(lens), (max(lens) + 15) // 16
    k, v = (torch.randn((B * width, H, 16, 128), generator=gen, device="cuda").to(dtype) for _ in range(2))
    q = (0.1 + torch.rand((B, H * G, 128), generator=gen, device="cuda")).to(dtype)       # positive: times -inf it is -inf
    table = torch.arange(B * width, device="cuda", dtype=torch.int32).view(B, width)
    return psa.KvCache(k, v, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), H * G), q


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_logits_of_minus_infinity_count_for_nothing(dtype, G):
    """All of a request's, all but one, every other one, a first block's (before any finite one): in one launch and in pieces."""
    lens = [40, 40, 40, 70, 5000]
    kv, q = cache(dtype, lens, 2, G, seed=G)
    width = kv.block_table.shape[1]
    off = [torch.zeros(width * 16, dtype=torch.bool) for _ in lens]
    off[0][:] = True
    off[1][:] = True
    off[1][33] = False
    off[2][::2] = True
    off[3][:64] = True
    off[4][:4096] = True
    for r, x in enumerate(off):
        kv.k_pool[r * width:(r + 1) * width, :, :, 5] = torch.where(x.view(width, 1, 16).cuda(), -INF, kv.k_pool[r * width:(r + 1) * width, :, :, 5])
    table = kv.block_table.cpu().long()

    def rows(pool):
        return lambda r, at: pool[table[r + 1, at // 16].cuda(), :, (at % 16).cuda()].transpose(0, 1)       # (without the first)
    for window, sinks in [(2 ** 31 - 1, 0), (4900, 30), (36, 2)]:
        out, lse = psa.window_attention(kv, q, window, sinks)
        assert not out[0].any() and torch.isneginf(lse[0]).all()
        want = wr.attention(q[1:], rows(kv.k_pool), rows(kv.v_pool), lens[1:], window, sinks)
        wr.close(out[1:], lse[1:], *want, where=(window, sinks))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_infinite_values_show_in_their_channel_alone(dtype):
    kv, q = cache(dtype, [100], 2, 4, seed=3)
    kv.v_pool[kv.block_table[0, 2].long(), 1, 3, 77] = -INF
    out, lse = psa.window_attention(kv, q, 2 ** 31 - 1)
    bad = ~torch.isfinite(out[0])
    assert bad[4:, 77].all() and int(bad.sum()) == 4 and torch.isfinite(lse).all()
    out, _ = psa.window_attention(kv, q, 40)                  # token 35 is not visible
    assert torch.isfinite(out).all()
