"""The 4-bit cache at the ends of the 16-bit types' ranges: what is read back, and what attention sees."""
import pytest
import torch

import paper_2503_00392_amd as psa

pytestmark = pytest.mark.gpu
INF = float("inf")

# (largest number of a block, what it is held as, what unpacking gives): 7/8 of the power of two beyond the range is the border
ENDS = {torch.float16: [(65504.0, 65536.0, INF), (57376.0, 65536.0, INF), (57344.0, 49152.0, 49152.0), (49152.0, 49152.0, 49152.0)],
        torch.bfloat16: [((2 - 2.0 ** -7) * 2.0 ** 127, INF, INF), ((1.75 + 2.0 ** -7) * 2.0 ** 127, INF, INF), (1.75 * 2.0 ** 127, 1.5 * 2.0 ** 127, 1.5 * 2.0 ** 127)]}


def packed(k, v):
    none = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    return psa.pack_pages(psa.KvCache(k, v, none, none[0], k.shape[1]), psa.PackedCache.empty_pool(k.shape[0], k.shape[1]))


def unpacked(pool, dtype):
    k, v = (torch.zeros((pool.shape[0], pool.shape[1], 16, 128), dtype=dtype, device="cuda") for _ in range(2))
    none = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    psa.unpack_pages(psa.KvCache(k, v, none, none[0], pool.shape[1]), pool)
    return k, v


@pytest.mark.parametrize("dtype,top,held,back", [(t, *x) for t, xs in ENDS.items() for x in xs])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_the_top_of_the_range(dtype, top, held, back, sign):
    x = torch.zeros((1, 1, 16, 128), dtype=torch.float64)
    x[0, 0, 3, 40] = sign * top
    x[0, 0, 3, 41] = top / 4                                  # beside it in its block of 32
    x[0, 0, 5, 100] = 1.0
    x16 = x.to(dtype).cuda()
    assert float(x16[0, 0, 3, 40]) == sign * top
    for got in unpacked(packed(x16, x16), dtype):
        assert float(got[0, 0, 3, 40]) == sign * back
        assert torch.isfinite(got[0, 0, 3, 41]) and abs(float(got[0, 0, 3, 41]) / (top / 4) - 1) <= 1 / 4 and float(got[0, 0, 5, 100]) == 1.0
        assert int((got == 0).sum()) == 16 * 128 - 3          # (nothing else, and no NaN)
    # one visible token: its value as the record holds it, with a weight of one
    none = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    cache = psa.PackedCache(packed(torch.zeros_like(x16), x16), none, torch.tensor([4], dtype=torch.int32, device="cuda"), 2, dtype)
    out, lse = psa.packed_attention(cache, torch.ones((1, 2, 128), dtype=dtype, device="cuda"), window=1)
    assert not lse.any()
    if held != INF:
        assert (out[0, :, 40] == sign * held).all() and torch.isfinite(out).all()
    else:       # an infinity: infinite or NaN (the weight of one is 1 + 0 + 0 in its parts, and 0 times an infinity is NaN), there alone
        assert not torch.isfinite(out[0, :, 40]).any() and int(torch.isfinite(out).sum()) == 2 * 127


def test_the_bottom_of_the_range():
    """Numbers of 2^-126 and more come back exactly where an element stands for them; below they keep their size or are zeros."""
    x = torch.zeros((1, 1, 16, 128), dtype=torch.float64)
    x[0, 0, 0, :8] = torch.tensor([0.5, 1, 1.5, 2, 3, 4, 6, -1]) * 2.0 ** -126
    x16 = x.to(torch.bfloat16).cuda()
    for got in unpacked(packed(x16, x16), torch.bfloat16):
        assert torch.equal(got[0, 0, 0, 1:8], x16[0, 0, 0, 1:8]) and float(got[0, 0, 0, 0]) in (0.0, 2.0 ** -127)
        assert int((got != 0).sum()) in (7, 8)
    least = torch.zeros((1, 1, 16, 128), dtype=torch.float16, device="cuda")
    least[0, 0, 0, :3] = torch.tensor([2.0 ** -24, -3 * 2.0 ** -24, 2.0 ** -22])
    for got in unpacked(packed(least, least), torch.float16):
        assert torch.equal(got, least)
