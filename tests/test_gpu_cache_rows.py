"""Rows behind the page calls: what can still be read through the cache that a fork started from."""
import pytest
import torch

import paper_2406_02069_b200 as pkv
from test_gpu_cache_pages import Pool, add_tensor, bits, config

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rows_of(cache, layer, b):
    """Keys, values and positions of a sequence as its tables name them: [heads][rows]."""
    n, page = int(cache.lens[layer, b]), cache.page_size
    r = torch.arange(n)
    slot = cache.tables[layer, b].cpu()[:, r // page].long() * page + r % page
    return [t.cpu().reshape(-1, *t.shape[2:])[slot] for t in (cache.k_pool, cache.v_pool, cache.positions)]


@pytest.mark.parametrize("dtype,d,page", [("bf16", 64, 4), ("fp32", 128, 16), ("fp16", 64, 1)])
def test_parents_can_be_read_through_the_cache_that_a_fork_started_from(dtype, d, page):
    """Sequence 1 is dropped and its pages, the lowest of the pool, are dealt out again by the same call; the rows of the others, as
    `from` names them, are as they were."""
    lens, parents = [[5 * page + 1, 40, 3, page], [1, 4 * page, 2 * page + 1, 0]], [0, 2, 0, 3, 2, 0]
    x = Pool(config(2, d, dtype), lens, page, 900, 64 // page + 60)
    # the lowest pages to sequence 1
    order = torch.argsort(torch.cat([x.cache.tables[:, 1].flatten(), x.cache.tables[:, [0, 2, 3]].flatten()]).cpu().eq(-1).int(), stable=True)
    flat = torch.cat([x.cache.tables[:, 1].flatten(), x.cache.tables[:, [0, 2, 3]].flatten()]).cpu()
    live = flat[order][: int(flat.ne(-1).sum())]
    place = torch.arange(900)
    place[live.long()] = torch.arange(len(live))                     # a new number for every page in use
    tables = torch.where(x.cache.tables.cpu() >= 0, place[x.cache.tables.cpu().clamp(min=0).long()].to(torch.int32), -1)
    refs = torch.zeros(900, dtype=torch.int32)
    refs[: len(live)] = 1
    x.cache.tables.copy_(tables)
    x.cache.refs.copy_(refs)
    before = [[rows_of(x.cache, l, b) for b in range(4)] for l in range(2)]
    to = x.other(len(parents))
    dropped = set(x.cache.tables[:, 1].flatten().tolist()) - {-1}
    pkv.cache_fork(x.cfg, x.cache, add_tensor(parents), x.ws, add=add_tensor([3] * len(parents)), to=to)
    pkv.check_status(x.ws)
    named = set(to.tables.flatten().tolist())
    assert dropped & named                                           # (some of the dropped pages have new rows)
    for l in range(2):
        for b in (0, 2, 3):
            assert all(torch.equal(bits(u), bits(w)) for u, w in zip(rows_of(x.cache, l, b), before[l][b]))
        for c, p in enumerate(parents):                              # and every child starts with them
            n = lens[l][p]
            assert all(torch.equal(bits(u[:, :n]), bits(w)) for u, w in zip(rows_of(to, l, c), before[l][p]))
