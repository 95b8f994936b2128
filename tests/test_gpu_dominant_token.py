"""Attention with a window and sinks where one token holds nearly all of the weight and its value is small: what the output is made
of are the other tokens' weights, many octaves below the largest."""
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


# Every query is a sign pattern u times 1/4 and a little noise, the dominant key 16 / sqrt(128) * nats * u / 4 and the others N(0, 1/4):
# logits of about `nats` and within 1 of 0.  Sum |q_c k_c| / sqrt(128) is nats (and a few) for the one and below 3 for the others; a
# logit's error is at most 8 * 2^-24 of that (window_reference.py has it), 1.2e-5 at 25 nats, and shows once in an output
# whose numerator the dominant token adds nothing to, so the bounds there (2e-5) hold.
def dominated(psa, ctx, H, G, dtype, nats, at, scale, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    width = (ctx + 15) // 16
    table = torch.randperm(width + 1, generator=gen, device="cuda")[:width].view(1, width).to(torch.int32)
    k = 0.5 * torch.randn((width + 1, H, 16, 128), generator=gen, device="cuda")
    v = 0.5 + torch.randn((width + 1, H, 16, 128), generator=gen, device="cuda")
    u = torch.randint(0, 2, (H, 128), generator=gen, device="cuda") * 2.0 - 1
    page = int(table[0, at // 16])
    k[page, :, at % 16] = u * (nats * 4 / 128 ** 0.5)
    v[page, :, at % 16] *= scale
    q = (u[:, None] / 4 + 0.02 * torch.randn((H, G, 128), generator=gen, device="cuda")).view(1, H * G, 128).to(dtype)
    kv = psa.KvCache(k.to(dtype), v.to(dtype), table, torch.tensor([ctx], dtype=torch.int32, device="cuda"), H * G)

    def rows(pool):
        return lambda r, i: pool[table[r, i.cuda() // 16].long(), :, (i % 16).cuda()].transpose(0, 1)
    return kv, q, (rows(kv.k_pool), rows(kv.v_pool))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("nats", [8, 12, 16, 25])
def test_a_first_token_that_holds_nearly_everything(psa, dtype, G, nats):
    for ctx, H, window, sinks, scale in [(4112, 2, 4096, 16, 0.0), (4112, 2, 4096, 16, 1.0), (9000, 1, 4096, 16, 2.0 ** -14),
                                         (65536, 1, INT_MAX, 0, 0.0), (65536, 1, INT_MAX, 0, 1.0), (333, 3, 100, 1, 0.0)]:
        kv, q, (keys, values) = dominated(psa, ctx, H, G, dtype, nats, 0, scale, seed=ctx + nats)
        out, lse = psa.window_attention(kv, q, window, sinks)
        wr.close(out, lse, *wr.attention(q, keys, values, [ctx], window, sinks), where=(ctx, window, scale))
        assert (lse > nats - 4).all()                         # (it does dominate)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("at", [17, 2047, 4110, 4111])
def test_wherever_the_token_stands(psa, dtype, at):
    kv, q, (keys, values) = dominated(psa, 4112, 2, 4, dtype, 16, at, 0.0, seed=at)
    out, lse = psa.window_attention(kv, q, INT_MAX)
    wr.close(out, lse, *wr.attention(q, keys, values, [4112], INT_MAX, 0))


def test_values_of_every_size(psa):
    """Binary16 values from the least subnormal to the largest number keep all their bits beside a weight of one."""
    ctx, H = 32, 1
    kv, q, (keys, values) = dominated(psa, ctx, H, 2, torch.float16, 16, 5, 1.0, seed=1)
    page = int(kv.block_table[0, 0])
    least = 2.0 ** -24
    special = torch.tensor([least, 3 * least, 1023 * least, 2.0 ** -14, 65504.0, -65504.0, 1 + 2.0 ** -10, -1 - 2.0 ** -10, 0.0, 2047 * 2.0 ** -11])
    kv.v_pool[:] = 0
    kv.v_pool[page, 0, 5, :special.numel()] = special.half().cuda()
    out, lse = psa.window_attention(kv, q, INT_MAX)
    want, want_lse = wr.attention(q, keys, values, [ctx], INT_MAX, 0)
    # the token's own weight: its logit and the sum of weights are off by 2e-5 at most, each element relative to itself
    assert ((out.double().cpu() - want).abs() <= wr.OUT * want.abs()).all()
    assert (lse.double().cpu() - want_lse).abs().max() <= wr.LSE
