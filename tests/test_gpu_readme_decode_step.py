"""The README's decode step of a layer with a window and a layer in 4 bits, run as it stands there."""
import os
import re

import pytest
import torch

import packed_reference as pr
import window_reference as wr

pytestmark = pytest.mark.gpu
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def test_each_cache_gets_the_token_once():
    import paper_2503_00392_amd as psa
    text, = [x for x in re.findall(r"```python\n(.*?)```", open(README).read(), re.S) if "norm_rotate" in x]
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()   # noqa: E731
    B, heads, pages, start = 3, 8, 40, [0, 31, 100]
    table = [torch.randperm(pages, generator=gen, device="cuda")[: B * 8].view(B, 8).to(torch.int32) for _ in range(2)]
    lens = [torch.tensor(start, dtype=torch.int32, device="cuda") for _ in range(2)]
    pools = [[new(pages, heads, 16, 128) for _ in range(2)] for _ in range(2)]
    kv, prompt = psa.KvCache(*pools[0], table[0], lens[0], 32), psa.KvCache(*pools[1], table[1], lens[1], 32)
    names = dict(psa=psa, torch=torch, kv=kv, meta=psa.build_block_metadata(kv), ctx_lens=lens[0], block_table=table[0], kv_prompt=prompt,
                 block_table_4bit=table[1], ctx_lens_4bit=lens[1], num_pages=pages, num_kv_heads=heads, q_proj=new(B, 32, 128),
                 k_proj=new(B, heads, 128), v=new(B, heads, 128), wq=new(128), wk=new(128),
                 inv_freq=(10000.0 ** (-torch.arange(0, 128, 2, device="cuda") / 128)).float())
    # (both calls call their results out, lse there)
    exec(re.sub(r"out, lse = (psa.window_attention)", r"window_out, window_lse = \1", text), names)
    torch.cuda.synchronize()
    after = [n + 1 for n in start]
    assert lens[0].tolist() == after and lens[1].tolist() == after
    tables = [x.cpu().long() for x in table]

    def rows(pool, which):
        return lambda r, at: pool[tables[which][r, at // 16].cuda(), :, (at % 16).cuda()].transpose(0, 1)
    for r, n in enumerate(start):                             # the new token, where it belongs and as it was made
        page = tables[0][r, n // 16]
        assert torch.equal(kv.k_pool[page, :, n % 16], names["k"][r]) and torch.equal(kv.v_pool[page, :, n % 16], names["v"][r])
    wr.close(names["window_out"], names["window_lse"], *wr.attention(names["q"], rows(kv.k_pool, 0), rows(kv.v_pool, 0), after, 4096, 4))
    values = [torch.from_numpy(x).cuda() for x in pr.unpack(names["pool"].cpu().numpy())]
    wr.close(names["out"], names["lse"], *wr.attention(names["q"], rows(values[0], 1), rows(values[1], 1), after, 2 ** 31 - 1, 0))
