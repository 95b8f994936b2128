"""RMS norm and rotation of rows whose squares leave binary32's range, against binary64."""
import pytest
import torch

from test_gpu_rotate import check, frequencies, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("weighted", [False, True])
def test_large_and_small_rows(interleaved, weighted):
    """Rows of every size beside each other in a wave; the smallest only where eps does not swallow them (eps 0 and 1e-38)."""
    import paper_2503_00392_amd as psa
    gen = torch.Generator().manual_seed(3)
    powers = [0, 60, 62, 64, 90, 100, 126, -40, -47, -49, -60, -63, -64, -75, -100, -124, 0, 127]
    x = torch.randn((3, len(powers), 128), generator=gen).clamp(-1.9, 1.9).double()
    x = (x * 2.0 ** torch.tensor(powers, dtype=torch.float64)[:, None]).to(torch.bfloat16)
    assert torch.isfinite(x).all()
    q, k = x.cuda(), x.flip(1).contiguous().cuda()
    w = (1 + 0.3 * torch.randn(128, generator=gen)).bfloat16().cuda() if weighted else None
    pos, freq = torch.tensor([0, 7, 100000], dtype=torch.int32).cuda(), frequencies(96)
    for eps in (0.0, 1e-38, 1e-30, 1e-6, 1.0):
        got = psa.norm_rotate(q, k, pos, freq, q_weight=w, k_weight=w, eps=eps, interleaved=interleaved)
        # (eps as the call has it, in binary32)
        for y, z in zip(got, (q, k)):
            check(y, *reference(z, w, pos, freq, float(torch.tensor(eps, dtype=torch.float32)), True, interleaved))


def test_subnormal_rows_and_what_is_no_number():
    import paper_2503_00392_amd as psa
    x = torch.zeros((1, 5, 128), dtype=torch.bfloat16, device="cuda")
    x[0, 0] = 2.0 ** -133                                     # bfloat16's least
    x[0, 1, ::2] = -2.0 ** -130
    x[0, 2], x[0, 2, 5] = 2.0 ** 100, float("inf")
    x[0, 3], x[0, 3, 5] = 2.0 ** 100, float("nan")
    pos, freq = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    got, _ = psa.norm_rotate(x, x, pos, freq, eps=0.0)
    check(got[:, :2], *reference(x[:, :2], None, pos, freq, 0.0, True, False))
    assert torch.isnan(got[0, 2, 5]) and int(torch.isnan(got[0, 2]).sum()) == 1 and int((got[0, 2] == 0).sum()) == 127
    assert torch.isnan(got[0, 3]).all() and torch.isnan(got[0, 4]).all()                   # (zeros: 0 / 0)
