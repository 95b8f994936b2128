"""RMS norm and rotation of queries and keys against binary64."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def psa():
    import paper_2503_00392_amd as psa
    psa.load_library()
    assert torch.cuda.is_available()
    return psa


def reference(x, weight, positions, inv_freq, eps, normalize, interleaved):
    """The result in binary64, and what bounds the computation's error: the size of the numbers that a sum is made of."""
    y = x.double().cpu()
    if normalize:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        if weight is not None:
            y = y * weight.double().cpu()
    half = inv_freq.numel()
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    u = positions.double().cpu()[:, None, None] * inv_freq.double().cpu()
    z, size = y.clone(), y.abs()
    z[..., a] = y[..., a] * torch.cos(u) - y[..., b] * torch.sin(u)
    z[..., b] = y[..., a] * torch.sin(u) + y[..., b] * torch.cos(u)
    size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
    return z, size


def check(got, want, size):
    # one rounding to the type: half a step; before it some ten roundings in binary32 and sine and cosine to a few
    # units of 2^-24: 16 * 2^-24 = 2^-20 of the sizes; and half of the least subnormal
    eps = torch.finfo(got.dtype).eps
    least = torch.finfo(got.dtype).tiny * eps / 2
    off = (got.double().cpu() - want).abs()
    assert (off <= eps / 2 * want.abs() + 2.0 ** -20 * size + least).all(), float((off / (size + 1e-30)).max())


def frequencies(rot, base=10000.0):
    return (base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().cuda()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 8, 24, 64, 96, 120, 128])
def test_against_the_definition(psa, dtype, interleaved, rot):
    gen = torch.Generator().manual_seed(rot + 1000 * interleaved)
    for T, Hq, H in [(1, 32, 8), (1, 1, 1), (3, 5, 0), (2, 0, 7), (33, 7, 3), (257, 8, 1), (64, 24, 24)]:
        q, k = ((3 * torch.randn((T, n, 128), generator=gen)).to(dtype).cuda() for n in (Hq, H))
        qw, kw = ((1 + 0.3 * torch.randn(128, generator=gen)).to(dtype).cuda() for _ in range(2))
        pos = torch.randint(0, 1 << 20, (T,), generator=gen).to(torch.int32).cuda()
        pos[0] = [0, 1, (1 << 31) - 1, -5][T % 4]
        freq = frequencies(rot)
        for normalize, weighted in [(True, True), (True, False), (False, True)]:
            w = (qw, kw) if weighted else (None, None)
            got = psa.norm_rotate(q, k, pos, freq, q_weight=w[0], k_weight=w[1], eps=1e-5, normalize=normalize, interleaved=interleaved)
            for x, y, weight in zip(got, (q, k), w):
                check(x, *reference(y, weight, pos, freq, 1e-5, normalize, interleaved))


@pytest.mark.parametrize("in_place", [False, True])
def test_views_of_one_projection(psa, in_place):
    """Queries and keys as slices of [T][(Hq + 2 H) 128], results anywhere; the values beside them stay as they were."""
    T, Hq, H = 70, 12, 4
    qkv = torch.randn((T, (Hq + 2 * H) * 128 + 64), device="cuda").bfloat16()
    before = qkv.clone()
    q, k = qkv[:, : Hq * 128].view(T, Hq, 128), qkv[:, Hq * 128:(Hq + H) * 128].view(T, H, 128)
    pos, freq = torch.arange(T, device="cuda", dtype=torch.int32) + 100000, frequencies(128, 5e5)
    want = [reference(x, None, pos, freq, 1e-6, True, False) for x in (q, k)]
    store = torch.full((T, Hq + H + 3, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    outs = (q, k) if in_place else (store[:, :Hq], store[:, Hq + 1:Hq + 1 + H])
    got = psa.norm_rotate(q, k, pos, freq, q_out=outs[0], k_out=outs[1])
    for x, w in zip(got, want):
        check(x.contiguous(), *w)
    if in_place:
        assert torch.equal(qkv[:, (Hq + H) * 128:], before[:, (Hq + H) * 128:])
    else:
        assert torch.equal(qkv, before) and bool((store[:, Hq] == 7).all()) and bool((store[:, Hq + 1 + H:] == 7).all())


def test_tokens_that_share_a_row_and_rows_that_share_a_frequency(psa):
    """One row for all tokens (a stride of 0) at different positions; frequencies of 0."""
    row = torch.randn((1, 4, 128), device="cuda").half()
    q = row.expand(9, 4, 128)
    pos, freq = torch.arange(9, device="cuda", dtype=torch.int32), torch.zeros(32, device="cuda")
    got, _ = psa.norm_rotate(q, q, pos, freq, normalize=False)
    assert torch.equal(got, q.contiguous())
    freq[3] = 0.5
    got, _ = psa.norm_rotate(q, q, pos, freq, normalize=False)
    check(got, *reference(q, None, pos, freq, 0, False, False))


def test_extremes(psa):
    """Zero rows, tiny and large rows, infinities in channels that are not rotated, NaN staying in its row."""
    x = torch.zeros((1, 6, 128), dtype=torch.bfloat16, device="cuda")
    x[0, 1] = 2.0 ** -40
    x[0, 2] = 2.0 ** 40
    x[0, 3, 100] = float("inf")
    x[0, 4, 5] = float("nan")
    x[0, 5, ::2] = 1.0
    pos, freq = torch.tensor([17], dtype=torch.int32, device="cuda"), frequencies(64)
    raw, _ = psa.norm_rotate(x, x, pos, freq, normalize=False)
    assert torch.isinf(raw[0, 3, 100]) and int(torch.isnan(raw[0, 3]).sum()) == 0
    assert torch.isnan(raw[0, 4, [5, 37]]).all() and int(torch.isnan(raw).sum()) == 2
    normed, _ = psa.norm_rotate(x, x, pos, freq, eps=0.0)
    assert torch.isnan(normed[0, 0]).all()                    # 0 / 0, as the formula has it
    normed, _ = psa.norm_rotate(x, x, pos, freq, eps=1e-30)
    assert not normed[0, 0].any() and torch.isnan(normed[0, 4]).all()
    rows = [1, 2, 5]
    check(normed[:, rows], *reference(x[:, rows], None, pos, freq, 1e-30, True, False))


def test_norm_alone_needs_no_positions(psa):
    """At the C boundary: without rotation the positions and frequencies may be NULL."""
    import ctypes as C
    from paper_2503_00392_amd import binding as pb
    x = torch.randn((3, 5, 128), device="cuda").half()
    y = torch.zeros_like(x)
    d = pb._RotateDesc(3, 5, 0, 128, 0, 0, 1, 0, 640, 0, 640, 0, 1e-6)
    assert psa.load_library().psa_norm_rotate(C.byref(d), x.data_ptr(), None, y.data_ptr(), None, None, None, None, None, None) == 0
    torch.cuda.synchronize()
    none = torch.empty(0, device="cuda")
    check(y, *reference(x, None, torch.zeros(3), none, 1e-6, True, False))
