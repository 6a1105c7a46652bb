"""Growing cache: the largest numbers of tiles that the library takes."""
import math

import pytest
import torch

import paper_2406_02069_b200 as pkv

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_every_sequence_is_answered_at_the_largest_number_of_tiles():
    """1024 sequences of 2097151 tiles: with what the plan counts on top of each sequence the sum passes 2^31.  All pages of a
    sequence are one page, of which one row is early enough to be seen: every weight is 1, every sum a whole number below 2^24,
    so that the output is that row's value to the bit."""
    batch, page, max_pages, d = 1024, 56896, 2359, 64
    assert page * max_pages // 64 == 2097151 and page % 64 == 0
    cfg = pkv.make_config(num_layers=1, num_q_heads=1, num_kv_heads=1, head_dim=d, window=1, pool_kernel=1, dtype="bf16", avg_budget=1)
    k, v = (torch.full((3, page, d), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    positions = torch.full((3, page), 9, dtype=torch.int32, device=DEV)
    values = torch.randint(-100, 100, (3, d), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    for i, row in enumerate((0, 30001, page - 1)):
        k[i, row], v[i, row], positions[i, row] = 0.0, values[i].to(DEV), 3
    which = (torch.arange(batch) % 3).to(torch.int32)
    tables = which.to(DEV).view(1, batch, 1, 1).expand(1, batch, 1, max_pages).contiguous()
    cache = pkv.PagedCache(cfg, k, v, tables, torch.full((1, batch), page * max_pages, dtype=torch.int32, device=DEV), positions=positions)
    ws = pkv.new_cache_workspace(cfg, cache)
    out, lse = torch.full((batch, 1, d), 7.0, device=DEV), torch.full((batch, 1), 7.0, device=DEV)
    q = torch.randn(batch, 1, d, device=DEV).to(torch.bfloat16)
    pkv.decode_attention_cache(cfg, cache, 0, q, out, ws, q_positions=torch.full((batch,), 5, dtype=torch.int32, device=DEV), lse=lse)
    pkv.check_status(ws)
    assert torch.equal(out[:, 0].cpu(), values[which.long()].float())
    assert torch.all((lse.cpu() - math.log(max_pages)).abs() <= 8 * 2.0 ** -24 * 8)          # (a logarithm and a product, of 8 at most)
    # one tile more in every table: refused
    more = torch.zeros(1, batch, 1, max_pages + 1, dtype=torch.int32, device=DEV)
    long = pkv.PagedCache(cfg, k, v, more, cache.lens, positions=positions)
    assert pkv.cache_workspace_bytes(cfg, long) == 0
    with pytest.raises(pkv.PkvError):
        pkv.decode_attention_cache(cfg, long, 0, q, out, ws)
