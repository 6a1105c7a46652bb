"""Rows behind the page calls and the appends: what can still be read through the cache that a fork started from, the rows of large pools
that a compaction moves, keys of a decode run against the rotation of what was given."""
import pytest
import torch

import paper_2406_02069_b200 as pkv
from cache_oracle import ListCache, assert_rotated, attend, frequencies, rotate
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


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("pages", [4097, 300001])
def test_rows_of_large_pools_move_with_their_pages(pages, in_place):
    """Pages marked with the halves of their numbers, exact in fp16, in every row of K and V."""
    cfg = config(1, 64, "fp16")
    g = torch.Generator().manual_seed(pages)
    number = torch.arange(pages, device=DEV)
    k = torch.zeros(pages, 2, 64, dtype=torch.float16, device=DEV)
    k[:, 0, 0], k[:, 0, 63], k[:, 1, 8], k[:, 1, 9] = number % 1024, number // 1024, number // 1024, number % 1024
    v = -k
    used = pages * 2 // 3
    order = torch.randperm(pages, generator=g).to(torch.int32)[:used]
    tables = torch.full((1, 2, 1, used), -1, dtype=torch.int32)
    tables[0, 0, 0, : used // 4], tables[0, 1, 0, : used - used // 4] = order[: used // 4], order[used // 4:]
    lens = torch.tensor([[2 * (used // 4) - 1, 2 * (used - used // 4)]], dtype=torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[order.long()] = 1
    cache = pkv.PagedCache(cfg, k, v, tables.to(DEV), lens.to(DEV), refs=refs.to(DEV))
    to = cache if in_place else pkv.PagedCache(cfg, k, v, torch.zeros_like(cache.tables), torch.zeros_like(cache.lens), refs=torch.zeros_like(cache.refs))
    ws = pkv.new_cache_workspace(cfg, cache)
    lists = ListCache(tables, lens, refs, 2)
    old_k, old_v = k.clone(), v.clone()
    pkv.cache_compact(cfg, cache, ws, to=None if in_place else to)
    pkv.check_status(ws)
    count, moves = lists.compact()
    lists.check(to.tables.cpu(), to.lens.cpu(), to.refs.cpu())
    assert count == used and len(moves) > pages // 8
    source, target = (torch.tensor(m, device=DEV) for m in zip(*moves))
    assert not torch.equal(k[target], old_k[target])
    old_k[target], old_v[target] = old_k[source], old_v[source]
    assert torch.equal(bits(k), bits(old_k)) and torch.equal(bits(v), bits(old_v))
    where = to.tables[0, 1, 0, : used - used // 4].long()            # a sequence's rows are those that it had
    assert torch.equal((k[where, 0, 0] + 1024 * k[where, 0, 63].float()).int().cpu(), order[used // 4:])


@pytest.mark.parametrize("dtype,group,layout,rotary_dim,native", [("bf16", 4, "half", 128, True), ("fp16", 8, "interleaved", 64, True), ("fp32", 2, "half", 64, True),
                                                                  ("bf16", 1, "interleaved", 20, True), ("bf16", 4, "half", 128, False)])
def test_keys_of_a_decode_run_are_the_rotated_ones(dtype, group, layout, rotary_dim, native, monkeypatch):
    """Steps of reserve, append and attention, a fork between them, eagerly and then replayed from a graph: every stored key and every
    rotated query is compared with the rotation, in 64 bits, of what was given at its position.  native: through the native half of the
    binding, or without it."""
    if not native:
        monkeypatch.setattr(pkv.cache, "_native", WithoutNative())
    heads, d, layers, page, batch = 2, 128, 2, 4, 3
    x = Pool(config(heads, d, dtype, group, layers), [[0, 5, 9], [3, 0, 7]], page, 200, 12)
    t = x.cache.k_pool.dtype
    g = torch.Generator().manual_seed(7)
    plan = pkv.make_rotary(rotary_dim, layout=layout, scaling="yarn", factor=4.0, original_positions=4096)
    freq, magnitude = frequencies(rotary_dim, scaling="yarn", factor=4.0, original=4096, high=32.0)
    make = lambda h: torch.zeros(layers, batch, h, 1, d, dtype=t, device=DEV)  # noqa: E731
    q, k, v, q_out = make(heads * group), make(heads), make(heads), make(heads * group)
    out, lse = torch.zeros(layers, batch, heads * group, d, device=DEV), torch.zeros(layers, batch, heads * group, device=DEV)
    add, granted = add_tensor([0] * batch), torch.zeros(layers, batch, dtype=torch.int32, device=DEV)
    positions, parents = add_tensor([[100], [20000], [131071]]), add_tensor([0, 1, 2])
    model = [[[r.clone() for r in rows_of(x.cache, l, b)] for b in range(batch)] for l in range(layers)]

    def step():
        pkv.cache_fork(x.cfg, x.cache, parents, x.ws)
        pkv.cache_reserve(x.cfg, x.cache, add, x.ws, granted=granted)
        for l in range(layers):
            pkv.append_cache(x.cfg, x.cache, l, positions, k[l], v[l], x.ws, q=q[l], q_out=q_out[l], rotary=plan, counts=granted[l])
            pkv.decode_attention_cache(x.cfg, x.cache, l, q_out[l], out[l], x.ws, lse=lse[l])
        pkv.cache_compact(x.cfg, x.cache, x.ws)

    def given(parent, more):
        for y in (q, k, v):
            y.copy_((2 * torch.randn(y.shape, generator=g)).to(t))
        parents.copy_(add_tensor(parent))
        add.copy_(add_tensor(more))
        positions.copy_(positions[torch.tensor(parent, device=DEV)] + 1)

    def check(parent, more):
        pkv.check_status(x.ws)
        for l in range(layers):
            model[l] = [[r.clone() for r in model[l][p]] for p in parent]
            for b in range(batch):
                p = positions[b].cpu()
                rows = rows_of(x.cache, l, b)
                if more[b]:
                    want, size = rotate(k[l, b].cpu(), p, freq, magnitude, layout)
                    assert_rotated(rows[0][:, -1:], want, size, "keys")
                    want, size = rotate(q[l, b].cpu(), p, freq, magnitude, layout)
                    assert_rotated(q_out[l, b].cpu(), want, size, "queries")
                    new = (rows[0][:, -1:], v[l, b].cpu(), p.expand(heads, 1))
                    model[l][b] = [torch.cat([a, n], 1) for a, n in zip(model[l][b], new)]
                assert all(torch.equal(bits(a), bits(w)) for a, w in zip(rows, model[l][b])), (l, b)
                for h in range(heads):
                    hq = slice(h * group, (h + 1) * group)
                    want, want_lse, size = attend(q_out[l, b, hq, 0].cpu(), rows[0][h], rows[1][h])
                    assert torch.all((out[l, b, hq].cpu().double() - want).abs() <= 1e-4 * size + 1e-7), (l, b, h)
                    assert torch.all((lse[l, b, hq].cpu().double() - want_lse).abs() <= 1e-4) or rows[0].shape[1] == 0

    steps = [([0, 1, 2], [1, 1, 1]), ([0, 1, 2], [1, 0, 1]), ([1, 1, 2], [1, 1, 0]), ([0, 2, 2], [1, 1, 1]), ([0, 1, 2], [1, 1, 1])]
    for parent, more in steps:
        given(parent, more)
        step()
        check(parent, more)
    given([0, 1, 2], [0, 0, 0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    check([0, 1, 2], [0, 0, 0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for parent, more in steps:
        given(parent, more)
        graph.replay()
        check(parent, more)


class WithoutNative:
    """The binding where its native half is not there: every call is left to the checks and the marshalling in Python."""

    def __getattr__(self, name):
        return lambda *args: pkv.binding._NOT_TAKEN


@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_without_the_native_half_gives_the_same_bits(inverse, monkeypatch):
    cfg, plan = config(2, 128, "bf16", 4), pkv.make_rotary(64, layout="interleaved")
    q = torch.randn(2, 8, 33, 128, device=DEV).to(torch.bfloat16)
    k = torch.randn(2, 33, 2, 128, device=DEV).to(torch.bfloat16).transpose(1, 2)        # (tokens first)
    positions = torch.arange(50, 83, dtype=torch.int32, device=DEV).expand(2, -1)
    got = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(pkv.cache, "_native", WithoutNative())
        q_out, k_out = torch.zeros_like(q), k.clone()
        pkv.rotary(cfg, plan, positions, q, k_out, q_out, None, inverse)
        got.append((q_out, k_out))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and not torch.equal(got[0][0], q)
    with pytest.raises(ValueError):
        pkv.rotary(cfg, plan, positions[:1], q)


def test_a_direction_that_is_neither_true_nor_false_is_refused():
    cfg, plan = config(1, 64, "bf16"), pkv.make_rotary(64)
    q = torch.randn(1, 1, 3, 64, device=DEV).to(torch.bfloat16)
    before, positions = q.clone(), torch.arange(3, dtype=torch.int32, device=DEV)[None]
    with pytest.raises(RuntimeError, match="ambiguous"):
        pkv.rotary(cfg, plan, positions, q, inverse=torch.tensor([True, False]))
    assert torch.equal(q, before)
