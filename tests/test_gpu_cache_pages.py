"""Pages of a growing cache: reserve, fork, compact against lists, in place and into another cache, and a decode run of all
the calls together."""
import random

import pytest
import torch

import paper_2406_02069_b200 as pkv
from cache_oracle import ListCache, attend, frequencies, rotate

pytestmark = pytest.mark.gpu
DEV = "cuda"


def config(heads=2, d=64, dtype="bf16", group=1, layers=1):
    return pkv.make_config(num_layers=layers, num_q_heads=heads * group, num_kv_heads=heads, head_dim=d, window=1, pool_kernel=1, dtype=dtype, avg_budget=1)


def bits(t):
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


class Pool:
    """A cache whose pages are dealt out at random, its lists beside it."""

    def __init__(self, cfg, lens, page, pages, max_pages, seed=0, positions=True):
        g = torch.Generator().manual_seed(seed)
        heads, d = cfg.num_kv_heads, cfg.head_dim
        self.cfg, self.page, self.layers, self.batch = cfg, page, len(lens), len(lens[0])
        t = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}[cfg.dtype]
        tables = torch.full((self.layers, self.batch, heads, max_pages), -1, dtype=torch.int32)
        refs = torch.zeros(pages, dtype=torch.int32)
        order = torch.randperm(pages, generator=g).tolist()
        for l in range(self.layers):
            for b in range(self.batch):
                for h in range(heads):
                    for j in range(-(-lens[l][b] // page)):
                        tables[l, b, h, j] = order.pop()
                        refs[tables[l, b, h, j]] = 1
        lens = torch.tensor(lens, dtype=torch.int32)
        self.lists = ListCache(tables, lens, refs, page)
        k, v = (torch.randn(pages, page, d, generator=g).to(t) for _ in range(2))
        pos = torch.randint(0, 10 ** 6, (pages, page), generator=g).to(torch.int32) if positions else None
        self.pools = [k, v, pos]
        dev = [x.to(DEV) if x is not None else None for x in (k, v, tables, lens, pos, refs)]
        self.cache = pkv.PagedCache(cfg, dev[0], dev[1], dev[2], dev[3], positions=dev[4], refs=dev[5])
        self.ws = pkv.new_cache_workspace(cfg, self.cache)

    def other(self, batch=None):
        """A second set of tables over the same pools."""
        c = self.cache
        batch = batch or c.batch
        to = pkv.PagedCache(self.cfg, c.k_pool, c.v_pool, torch.full((c.layers, batch, c.heads_kv, c.max_pages), -1, dtype=torch.int32, device=DEV),
                            torch.full((c.layers, batch), -1, dtype=torch.int32, device=DEV), positions=c.positions,
                            refs=torch.full_like(c.refs, -1))
        self.ws = pkv.new_cache_workspace(self.cfg, c, to)
        return to

    def check_pools(self, moves):
        """moves: (source page, page, rows) that were copied since the pools were last looked at."""
        for got, want in zip((self.cache.k_pool, self.cache.v_pool, self.cache.positions), self.pools):
            if want is None:
                continue
            old = want.clone()
            for s, t, rows in moves:
                want[t, :rows] = old[s, :rows]
            same = torch.equal(got.cpu(), want) if want.dtype == torch.int32 else torch.equal(bits(got.cpu()), bits(want))
            assert same


def add_tensor(add):
    return torch.tensor(add, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("dtype,heads,d,page,pages,max_pages,lens,add", [
    ("bf16", 2, 64, 4, 60, 6, [[3, 4, 5, 0]], [[1, 1, 0, 1]]),
    ("fp32", 1, 64, 1, 40, 20, [[7, 0], [2, 9]], [[3, 0], [1, 5]]),
    ("fp16", 8, 128, 16, 3000, 12, [[30, 100, 16, 15], [17, 1, 0, 64], [5, 5, 5, 5]], [[50, 1, 1, 1], [1, 40, 100, 0], [-3, 0, 11, 12]]),
    ("bf16", 1, 64, 5, 1, 3, [[0]], [[5]]),                           # the only page
])
def test_reserve_deals_out_the_lowest_free_pages(in_place, dtype, heads, d, page, pages, max_pages, lens, add):
    x = Pool(config(heads, d, dtype), lens, page, pages, max_pages)
    before = [t.clone() for t in (x.cache.tables, x.cache.lens, x.cache.refs)]
    to = x.cache if in_place else x.other()
    granted = torch.full((x.layers, x.batch), 9, dtype=torch.int32, device=DEV)
    pkv.cache_reserve(x.cfg, x.cache, add_tensor(add), x.ws, granted=granted, to=None if in_place else to)
    pkv.check_status(x.ws)
    counts, copies = x.lists.fork(list(range(x.batch)), add)
    assert not copies and granted.flatten().tolist() == counts
    x.lists.check(to.tables.cpu(), to.lens.cpu(), to.refs.cpu())
    # entries behind the last page are as they were
    for l in range(x.layers):
        for b in range(x.batch):
            n = x.lists.pages(x.lists.lens[l][b])
            assert torch.all(to.tables[l, b, :, n:] == -1)
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(before, (x.cache.tables, x.cache.lens, x.cache.refs)))
    x.check_pools([])


def test_reserve_takes_one_list_for_all_layers():
    x = Pool(config(2), [[3, 4, 5], [8, 1, 2]], 4, 60, 6)
    pkv.cache_reserve(x.cfg, x.cache, add_tensor([1, 0, 6]), x.ws)
    x.lists.fork([0, 1, 2], [[1, 0, 6]] * 2)
    x.lists.check(x.cache.tables.cpu(), x.cache.lens.cpu(), x.cache.refs.cpu())
    pkv.cache_reserve(x.cfg, x.cache, add_tensor([2, 1, 0]).expand(2, 3), x.ws)
    x.lists.fork([0, 1, 2], [[2, 1, 0]] * 2)
    x.lists.check(x.cache.tables.cpu(), x.cache.lens.cpu(), x.cache.refs.cpu())
    pkv.check_status(x.ws)


@pytest.mark.parametrize("call", ["reserve", "fork"])
@pytest.mark.parametrize("why", ["no room", "table too short", "huge", "bad parent"])
def test_a_call_that_cannot_be_met_changes_nothing(call, why):
    if call == "reserve" and why == "bad parent":
        return
    lens = [[3, 4, 5, 9], [8, 1, 2, 0]]
    x = Pool(config(2), lens, 4, 2 * (1 + 1 + 2 + 3 + 2 + 1 + 1) + 3, 6)
    add = {"no room": [[1, 1, 0, 1], [0, 4, 0, 0]], "table too short": [[0, 0, 0, 16], [0] * 4], "huge": [[2 ** 31 - 1] * 4, [2 ** 31 - 1] * 4], "bad parent": [[0] * 4] * 2}[why]
    parents = [0, 1, 2, 3] if why != "bad parent" else [1, 4, 0, -2]
    before = [t.clone() for t in (x.cache.tables, x.cache.lens, x.cache.refs)]
    granted = torch.full((2, 4), 9, dtype=torch.int32, device=DEV)
    assert x.lists.fork(parents, add) is None
    if call == "reserve":
        pkv.cache_reserve(x.cfg, x.cache, add_tensor(add), x.ws, granted=granted)
    else:
        pkv.cache_fork(x.cfg, x.cache, add_tensor(parents), x.ws, add=add_tensor(add), granted=granted)
    with pytest.raises(pkv.PkvError, match="0x8" if why == "bad parent" else "0x10"):
        pkv.check_status(x.ws)
    assert all(torch.equal(a, b) for a, b in zip(before, (x.cache.tables, x.cache.lens, x.cache.refs)))
    assert torch.all(granted == 0)
    x.check_pools([])
    # into another cache: this one is as good as before, and goes on
    to = x.other()
    if call == "fork":
        pkv.cache_fork(x.cfg, x.cache, add_tensor(parents), x.ws, add=add_tensor(add), to=to)
    else:
        pkv.cache_reserve(x.cfg, x.cache, add_tensor(add), x.ws, to=to)
    assert all(torch.equal(a, b) for a, b in zip(before, (x.cache.tables, x.cache.lens, x.cache.refs)))
    x.check_pools([])
    x.ws.zero_()
    pkv.cache_reserve(x.cfg, x.cache, add_tensor([1, 0, 0, 0]), x.ws)
    x.lists.fork([0, 1, 2, 3], [[1, 0, 0, 0]] * 2)
    x.lists.check(x.cache.tables.cpu(), x.cache.lens.cpu(), x.cache.refs.cpu())
    pkv.check_status(x.ws)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("dtype,d,page,lens,parents,add", [
    ("bf16", 64, 4, [[3, 4, 5]], [0, 0, 0], 0),                       # everyone goes on with one, the others are freed
    ("fp16", 128, 4, [[3, 4, 5], [8, 7, 0]], [2, 0, 2], 1),
    ("fp32", 64, 5, [[9, 4, 5], [8, 7, 12]], [-1, -1, -1], 3),        # all freed
    ("bf16", 128, 16, [[30, 47, 16], [1, 100, 33]], [1, -1, 1], 17),
    ("bf16", 64, 1, [[3, 4, 5]], [1, 1, 0], 2),                       # pages of one row are always full
])
def test_fork_shares_full_pages_and_copies_the_rest(in_place, dtype, d, page, lens, parents, add):
    x = Pool(config(2, d, dtype), lens, page, 200, 12)
    more = [[add] * len(parents)] * len(lens)
    to = x.cache if in_place else x.other()
    pkv.cache_fork(x.cfg, x.cache, add_tensor(parents), x.ws, add=add_tensor(more) if add else None, to=to if not in_place else None)
    pkv.check_status(x.ws)
    _, copies = x.lists.fork(parents, more)
    x.lists.check(to.tables.cpu(), to.lens.cpu(), to.refs.cpu())
    x.check_pools(copies)


@pytest.mark.parametrize("batch", [1, 2, 7, 30])
def test_fork_into_another_number_of_sequences(batch):
    x = Pool(config(3, 64), [[30, 47, 16], [1, 100, 33]], 8, 900, 20)
    r = random.Random(batch)
    parents = [r.randrange(-1, 3) for _ in range(batch)]
    add = [[r.randrange(0, 10) for _ in range(batch)] for _ in range(2)]
    to = x.other(batch)
    granted = torch.zeros(2, batch, dtype=torch.int32, device=DEV)
    pkv.cache_fork(x.cfg, x.cache, add_tensor(parents), x.ws, add=add_tensor(add), granted=granted, to=to)
    pkv.check_status(x.ws)
    counts, copies = x.lists.fork(parents, add)
    x.lists.check(to.tables.cpu(), to.lens.cpu(), to.refs.cpu())
    assert granted.flatten().tolist() == counts
    x.check_pools(copies)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("dtype,heads,d,page,pages,layers,batch,hi,seed", [
    ("bf16", 2, 64, 4, 100, 1, 3, 20, 0), ("fp32", 1, 128, 3, 5000, 2, 5, 200, 1), ("fp16", 4, 64, 16, 9001, 3, 10, 700, 2), ("bf16", 1, 64, 1, 7, 1, 1, 7, 3),
    ("bf16", 1, 64, 2, 50, 1, 2, 0, 4),                                # nothing in use
])
def test_compact_moves_pages_to_the_lowest_places(in_place, dtype, heads, d, page, pages, layers, batch, hi, seed):
    r = random.Random(seed)
    lens = [[r.randint(0, hi) for _ in range(batch)] for _ in range(layers)]
    x = Pool(config(heads, d, dtype), lens, page, pages, hi // page + 2, seed, positions=seed != 1)
    to = x.cache if in_place else x.other()
    used = torch.full((1,), -1, dtype=torch.int32, device=DEV)
    before = [t.clone() for t in (x.cache.tables, x.cache.lens, x.cache.refs)]
    pkv.cache_compact(x.cfg, x.cache, x.ws, used=used, to=None if in_place else to)
    pkv.check_status(x.ws)
    count, moves = x.lists.compact()
    assert int(used) == count
    x.lists.check(to.tables.cpu(), to.lens.cpu(), to.refs.cpu())
    x.check_pools([(s, t, page) for s, t in moves])
    assert torch.all(to.refs[count:] == 0) and torch.all(to.refs[:count] > 0)
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(before, (x.cache.tables, x.cache.lens, x.cache.refs)))


@pytest.mark.parametrize("seed", range(6))
def test_page_calls_one_after_another(seed):
    """Forks, reserves and compactions at random, in place and into a second cache in turn; every look at the lists agrees."""
    r = random.Random(seed)
    page, layers, batch = r.choice([1, 3, 8, 16]), r.choice([1, 3]), r.choice([2, 5, 9])
    lens = [[r.randint(0, 40) for _ in range(batch)] for _ in range(layers)]
    x = Pool(config(r.choice([1, 2, 3])), lens, page, 40 * batch * layers * 3 // page + 50, 60 // page + 1, seed)
    home, away = x.cache, x.other()
    ws, failed = x.ws, 0
    for step in range(30):
        inside = r.random() < 0.5
        to = home if inside else away
        kind = r.choice(["reserve", "fork", "fork", "compact"])
        copies = []
        if kind == "compact":
            pkv.cache_compact(x.cfg, home, ws, to=None if inside else to)
            copies = [(s, t, page) for s, t in x.lists.compact()[1]]
            done = True
        else:
            parents = list(range(batch)) if kind == "reserve" else [r.randrange(-1 if r.random() < 0.3 else 0, batch) for _ in range(batch)]
            add = [[r.choice([0, 1, 1, 3, 10]) for _ in range(batch)] for _ in range(layers)]
            got = x.lists.fork(parents, add)
            done = got is not None
            if kind == "reserve":
                pkv.cache_reserve(x.cfg, home, add_tensor(add), ws, to=None if inside else to)
            else:
                pkv.cache_fork(x.cfg, home, add_tensor(parents), ws, add=add_tensor(add), to=None if inside else to)
            if done:
                copies = got[1]
        if done:
            pkv.check_status(ws)
            if not inside:
                home, away = away, home
        else:
            failed += 1
            with pytest.raises(pkv.PkvError, match="0x10"):
                pkv.check_status(ws)
            ws[:256].zero_()
            parents = [-1] * (batch // 2) + list(range(batch // 2, batch))      # let go of half of them
            pkv.cache_fork(x.cfg, home, add_tensor(parents), ws)
            copies = x.lists.fork(parents, [[0] * batch] * layers)[1]
        x.lists.check(home.tables.cpu(), home.lens.cpu(), home.refs.cpu())
        x.check_pools(copies)


@pytest.mark.parametrize("pages", [4095, 4097, 300001])
def test_large_pools(pages):
    """More pages than a pass of the cluster takes, page counts that divide into nothing, refs at an odd address."""
    cfg = config(1, 64, "fp16")
    g = torch.Generator().manual_seed(pages)
    batch, max_pages = 3, pages // 3 + 2
    k = torch.zeros(pages, 1, 64, dtype=torch.float16, device=DEV)
    k[:, 0, 0] = torch.arange(pages, device=DEV).half()
    v = torch.arange(pages, device=DEV).to(torch.int32)[:, None, None].expand(pages, 1, 64).to(torch.float16).contiguous()
    rows = [pages // 4, pages // 3, 1000]
    order = torch.randperm(pages, generator=g).to(torch.int32)
    tables = torch.full((1, batch, 1, max_pages), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(rows):
        tables[0, b, 0, :n] = order[at:at + n]
        at += n
    refs = torch.zeros(pages + 1, dtype=torch.int32)
    refs[1:][order[:at].long()] = 1
    refs = refs.to(DEV)[1:]                                          # contiguous, four bytes behind a 16-byte border
    cache = pkv.PagedCache(cfg, k, v, tables.to(DEV), torch.tensor([rows], dtype=torch.int32, device=DEV), refs=refs)
    ws = pkv.new_cache_workspace(cfg, cache)
    lists = ListCache(tables, torch.tensor([rows]), refs.cpu(), 1)
    pkv.cache_reserve(cfg, cache, add_tensor([7, 0, pages // 3 - 1100]), ws)
    pkv.check_status(ws)
    lists.fork([0, 1, 2], [[7, 0, pages // 3 - 1100]])
    lists.check(cache.tables.cpu(), cache.lens.cpu(), cache.refs.cpu())
    pkv.cache_fork(cfg, cache, add_tensor([-1, 1, 2]), ws)
    lists.fork([-1, 1, 2], [[0] * 3])
    pkv.cache_compact(cfg, cache, ws)
    pkv.check_status(ws)
    old = k.clone()
    _, moves = lists.compact()
    lists.check(cache.tables.cpu(), cache.lens.cpu(), cache.refs.cpu())
    assert moves
    with pytest.raises(ValueError):                                  # a pool of another size
        pkv.PagedCache(cfg, k, v[:-1], cache.tables, cache.lens, refs=refs)
    assert torch.equal(old, k)


def test_page_calls_need_refs_and_fitting_tensors():
    x = Pool(config(2), [[3, 4]], 4, 20, 6)
    c = x.cache
    bare = pkv.PagedCache(x.cfg, c.k_pool, c.v_pool, c.tables, c.lens, positions=c.positions)
    for f in (lambda: pkv.cache_reserve(x.cfg, bare, add_tensor([1, 1]), x.ws), lambda: pkv.cache_fork(x.cfg, bare, add_tensor([1, 1]), x.ws),
              lambda: pkv.cache_compact(x.cfg, bare, x.ws), lambda: pkv.cache_reserve(x.cfg, c, add_tensor([1]), x.ws),
              lambda: pkv.cache_reserve(x.cfg, c, add_tensor([1, 1]).long(), x.ws), lambda: pkv.cache_fork(x.cfg, c, add_tensor([1]), x.ws),
              lambda: pkv.cache_fork(x.cfg, c, add_tensor([1, 1]).cpu(), x.ws), lambda: pkv.cache_reserve(x.cfg, c, add_tensor([1, 1]), x.ws, granted=add_tensor([1, 1])),
              lambda: pkv.cache_compact(x.cfg, c, x.ws, used=add_tensor([1, 1])),
              lambda: pkv.cache_compact(config(2, dtype="fp16"), c, x.ws)):
        with pytest.raises(ValueError):
            f()
    half = pkv.PagedCache(x.cfg, c.k_pool, c.v_pool, c.tables, c.lens.clone(), positions=c.positions, refs=c.refs)
    with pytest.raises(pkv.PkvError):
        pkv.cache_compact(x.cfg, c, x.ws, to=half)                   # shares some arrays, not all
    for bad in (dict(tables=c.tables.long()), dict(lens=c.lens[:, :1]), dict(v_pool=c.v_pool.half()), dict(positions=c.positions[:3]), dict(refs=c.refs[1:]),
                dict(tables=c.tables.cpu()), dict(k_pool=c.k_pool[:, :, :32], v_pool=c.v_pool[:, :, :32])):
        kw = {**dict(k_pool=c.k_pool, v_pool=c.v_pool, tables=c.tables, lens=c.lens), **bad}
        with pytest.raises(ValueError):
            pkv.PagedCache(x.cfg, kw.pop("k_pool"), kw.pop("v_pool"), kw.pop("tables"), kw.pop("lens"), **kw)


def test_positions_of_kept_rows_follow_the_block_table():
    cfg = pkv.make_config(num_layers=1, num_q_heads=2, num_kv_heads=2, head_dim=64, window=4, pool_kernel=1, dtype="bf16", avg_budget=8)
    lens, kl, page = [30, 6, 100], 9, 4
    counts = [pkv.kept_count(cfg, kl, n) for n in lens]
    pages = [pkv.pages_needed(cfg, kl, n, page) for n in lens]
    g = torch.Generator().manual_seed(4)
    table = torch.randperm(2 * sum(pages) + 3, generator=g)[:2 * sum(pages)].to(torch.int32)
    idx = torch.cat([torch.randint(0, n, (2 * c,), generator=g) for n, c in zip(lens, counts)]).to(torch.int32)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)

    def check(bad_pages=(), bad_rows=()):
        t, i = table.clone(), idx.clone()
        for e in bad_pages:
            t[e] = 10 ** 6
        for r in bad_rows:
            i[r] = 100
        got = torch.full((2 * sum(pages) + 3, page), -7, dtype=torch.int32, device=DEV)
        want = got.cpu()
        pkv.cache_positions(cfg, i.to(DEV), lens, kl, t.to(DEV), got, ws)
        entry = row = 0
        for b, c in enumerate(counts):
            for h in range(2):
                for r in range(c):
                    if entry + r // page not in bad_pages and row + r not in bad_rows:
                        want[int(table[entry + r // page]), r % page] = idx[row + r]
                entry += pages[b]
                row += c
        assert torch.equal(got.cpu(), want)
    check()
    pkv.check_status(ws)
    check(bad_pages=(1, len(table) - 1))
    with pytest.raises(pkv.PkvError, match="0x4"):
        pkv.check_status(ws)
    ws.zero_()
    check(bad_rows=(0, len(idx) - 1))
    with pytest.raises(pkv.PkvError, match="0x8"):
        pkv.check_status(ws)
    for bad in (dict(indices=idx[:-1].to(DEV)), dict(table=table[:-1].to(DEV)), dict(positions=torch.zeros(4, page, device=DEV))):
        with pytest.raises(ValueError):
            kw = {**dict(indices=idx.to(DEV), table=table.to(DEV), positions=torch.zeros(99, page, dtype=torch.int32, device=DEV)), **bad}
            pkv.cache_positions(cfg, kw["indices"], lens, kl, kw["table"], kw["positions"], ws)


# ------------------------------------------------------------------------------------------------ all of it together
class Rows:
    """What a sequence's head holds: (key as stored, value, position), oldest first."""

    def __init__(self, k, v, pos):
        self.k, self.v, self.pos = k, v, pos

    def __add__(self, other):
        return Rows(torch.cat([self.k, other.k]), torch.cat([self.v, other.v]), torch.cat([self.pos, other.pos]))


@pytest.mark.parametrize("dtype,group,layout,graph", [("bf16", 4, "half", False), ("fp16", 8, "interleaved", True), ("fp32", 2, "half", True)])
def test_a_decode_run_behind_compressed_prompts(dtype, group, layout, graph):
    """Two prompts are rotated and compressed into pages; they decode three tokens, fork into five branches that decode two
    more each with a bias on the distance and a window over original positions, one branch ends, the pool is compacted, and
    the rest decodes on (captured into a graph where `graph`).  Every output against 64 bits on the rows kept so far."""
    heads, d, layers, page, lens, window = 2, 128, 2, 4, [150, 90], 4
    cfg = pkv.make_config(num_layers=layers, num_q_heads=heads * group, num_kv_heads=heads, head_dim=d, window=window, pool_kernel=5, dtype=dtype, avg_budget=24)
    t = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[dtype]
    g = torch.Generator().manual_seed(31)
    plan = pkv.make_rotary(64, layout=layout, scaling="llama3", factor=8.0, original_positions=512)
    freq, magnitude = frequencies(64, scaling="llama3", factor=8.0, original=512)
    budgets = pkv.layer_budgets(cfg)
    pages = 400
    k_pool, v_pool = (torch.full((pages, page, d), float("nan"), dtype=t, device=DEV) for _ in range(2))
    pos_pool = torch.full((pages, page), -1, dtype=torch.int32, device=DEV)

    def new_cache(batch):
        return pkv.PagedCache(cfg, k_pool, v_pool, torch.full((layers, batch, heads, 24), -1, dtype=torch.int32, device=DEV),
                              torch.zeros(layers, batch, dtype=torch.int32, device=DEV), positions=pos_pool,
                              refs=torch.zeros(pages, dtype=torch.int32, device=DEV))
    cache, branches = new_cache(2), new_cache(5)
    ws = pkv.new_cache_workspace(cfg, cache, branches)
    prompt_ws = pkv.new_workspace(cfg, 2, max(lens), DEV)
    # ---- the prompts: rotary positions, room for the kept rows, compression into them
    kept = [[pkv.kept_count(cfg, kl, n) for n in lens] for kl in budgets]
    pkv.cache_reserve(cfg, cache, add_tensor(kept), ws)
    model = [[[None] * heads for _ in lens] for _ in range(layers)]
    for l in range(layers):
        q, k, v = (torch.randn(2, h, max(lens), d, generator=g).to(t).to(DEV) for h in (heads * group, heads, heads))
        positions = torch.arange(max(lens), dtype=torch.int32, device=DEV).expand(2, -1)
        pkv.rotary(cfg, plan, positions, q, k)
        q_win = torch.stack([q[b, :, n - window:n] for b, n in enumerate(lens)])
        table = cache.block_table(l, [pkv.pages_needed(cfg, budgets[l], n, page) for n in lens])
        idx = torch.zeros(heads * sum(kept[l]), dtype=torch.int32, device=DEV)
        pkv.compress_layer_paged(cfg, l, q_win, k, v, lens, table, k_pool, v_pool, idx, prompt_ws)
        pkv.cache_positions(cfg, idx, lens, budgets[l], table, pos_pool, prompt_ws)
        pkv.check_status(prompt_ws)
        at = 0
        for b in range(2):
            for h in range(heads):
                i = idx[at:at + kept[l][b]].cpu()
                at += kept[l][b]
                model[l][b][h] = Rows(k[b, h].cpu()[i.long()], v[b, h].cpu()[i.long()], i)
    # ---- decode steps
    slopes = (2.0 ** -torch.arange(2, 2 + heads * group).float())
    at_position = torch.tensor(lens, dtype=torch.int32, device=DEV)

    def buffers(batch):
        make = lambda h: torch.zeros(layers, batch, h, 1, d, dtype=t, device=DEV)  # noqa: E731
        return dict(q=make(heads * group), k=make(heads), v=make(heads), out=torch.zeros(layers, batch, heads * group, d, device=DEV),
                    add=torch.zeros(batch, dtype=torch.int32, device=DEV), granted=torch.zeros(layers, batch, dtype=torch.int32, device=DEV))

    def step(c, x, positions, far):
        pkv.cache_reserve(cfg, c, x["add"], ws, granted=x["granted"])
        for l in range(layers):
            pkv.append_cache(cfg, c, l, positions[:, None], x["k"][l], x["v"][l], ws, q=x["q"][l], rotary=plan, counts=x["granted"][l])
            pkv.decode_attention_cache(cfg, c, l, x["q"][l], x["out"][l], ws, q_positions=positions if far else None,
                                       slopes=dev_slopes if far else None, window=40 if far else 0, prefix=5 if far else 0)

    dev_slopes = slopes.to(DEV)

    def check(c, x, given, positions, far, live):
        for l in range(layers):
            for b in range(c.batch):
                if b not in live:
                    assert torch.all(x["out"][l, b] == 0)
                    continue
                p = positions[b:b + 1].cpu()
                turned = lambda y: rotate(y, p, freq, magnitude, layout)[0]  # noqa: E731
                q = x["q"][l, b, :, 0].cpu()
                assert torch.all((q.double() - turned(given["q"][l, b])[:, 0]).abs() <= 0.04)      # (rotary's own test is the exact one)
                for h in range(heads):
                    slot = [int(c.tables[l, b, h, r // page]) * page + r % page for r in range(int(c.lens[l, b]))]
                    stored = k_pool.view(-1, d)[slot[-1]].cpu()
                    model[l][b][h] = model[l][b][h] + Rows(stored[None], given["v"][l, b, h], p)
                    rows = model[l][b][h]
                    assert torch.equal(k_pool.view(-1, d)[slot].cpu(), rows.k) and torch.equal(v_pool.view(-1, d)[slot].cpu(), rows.v)
                    assert torch.equal(pos_pool.view(-1)[slot].cpu(), rows.pos)
                    hq = slice(h * group, (h + 1) * group)
                    want, _, size = attend(q[hq], rows.k, rows.v, **(dict(positions=rows.pos, q_position=int(p), slopes=slopes[hq], window=40, prefix=5) if far else {}))
                    assert torch.all((x["out"][l, b, hq].cpu().double() - want).abs() <= 1e-4 * size + 1e-7), (l, b, h)

    def decode(c, x, positions, far, live, run):
        given = {n: torch.randn(x[n].shape, generator=g).to(t) for n in ("q", "k", "v")}
        for n in given:
            x[n].copy_(given[n])
        x["add"].copy_(torch.tensor([1 if b in live else 0 for b in range(c.batch)]))
        run()
        check(c, x, given, positions, far, live)
        positions += 1
        pkv.check_status(ws)

    x = buffers(2)
    for _ in range(3):
        decode(cache, x, at_position, False, {0, 1}, lambda: step(cache, x, at_position, False))
    parents = [1, 0, 1, 1, 0]
    pkv.cache_fork(cfg, cache, add_tensor(parents), ws, to=branches)
    model = [[[Rows(r.k, r.v, r.pos) for r in model[l][p]] for p in parents] for l in range(layers)]
    positions = at_position[torch.tensor(parents, device=DEV)].contiguous()
    y = buffers(5)
    run = lambda: step(branches, y, positions, True)  # noqa: E731
    for _ in range(2):
        decode(branches, y, positions, True, {0, 1, 2, 3, 4}, run)
    parents = [0, -1, 2, 3, 4]
    pkv.cache_fork(cfg, branches, add_tensor(parents), ws)
    used = torch.zeros(1, dtype=torch.int32, device=DEV)
    pkv.cache_compact(cfg, branches, ws, used=used)                   # (the first cache's tables name pages that have moved: it is not used again)
    pkv.check_status(ws)
    assert int(branches.refs.gt(0).sum()) == int(used) and torch.all(branches.refs[int(used):] == 0)
    if graph:
        captured = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        y["add"].zero_()
        with torch.cuda.stream(side):
            step(branches, y, positions, True)                        # (nothing is added: a warm-up that leaves the cache alone)
        torch.cuda.current_stream().wait_stream(side)
        with torch.cuda.graph(captured):
            step(branches, y, positions, True)
        run = captured.replay
    for _ in range(6):                                                # over a page's border
        decode(branches, y, positions, True, {0, 2, 3, 4}, run)
