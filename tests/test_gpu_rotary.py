"""Rotary positions and appends to a paged cache against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2406_02069_b200 as pkv
from cache_oracle import TYPES, assert_rotated, frequencies, rotate

pytestmark = pytest.mark.gpu
DEV = "cuda"


def config(heads, d, dtype):
    return pkv.make_config(num_layers=1, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=d, window=1, pool_kernel=1, dtype=dtype, avg_budget=1)


def randn(g, *shape, dtype, scale=1.0):
    return (scale * torch.randn(*shape, generator=g)).to(dtype)


# (query heads, KV heads), d, dtype, rotary_dim, layout, scaling, batch, tokens, first position
CASES = [
    ((4, 2), 64, "fp32", 64, "half", {}, 1, 1, 0),                              # one token at position 0
    ((4, 2), 64, "fp32", 64, "interleaved", {}, 1, 1, 131071),
    ((32, 8), 128, "bf16", 128, "half", dict(scaling="llama3", factor=8.0, original=8192), 1, 1, 1000000),
    ((32, 32), 128, "fp16", 128, "interleaved", dict(scaling="linear", factor=4.0), 2, 3, 5),
    ((5, 1), 128, "bf16", 32, "half", dict(scaling="yarn", factor=4.0, original=4096, high=32.0), 3, 77, 4000),
    ((6, 3), 64, "fp16", 16, "interleaved", dict(scaling="ntk", factor=8.0), 2, 130, 2 ** 31 - 200),
    ((3, 3), 64, "fp32", 20, "half", {}, 2, 9, -4),                             # part of the head, not in 16-byte pieces
    ((3, 1), 128, "bf16", 20, "interleaved", {}, 1, 33, 77),
    ((2, 1), 64, "fp16", 2, "half", {}, 1, 5, 100),
    ((2, 1), 64, "bf16", 2, "interleaved", {}, 1, 5, 100),
    ((7, 7), 128, "fp32", 120, "interleaved", {}, 1, 11, 9),                    # 4-element pieces
    ((16, 8), 64, "bf16", 64, "half", {}, 2, 1501, 0),                          # enough rows for a warp per token
    ((40, 8), 128, "bf16", 128, "half", {}, 1, 1801, 3),
    ((8, 2), 128, "fp16", 100, "half", {}, 3, 1203, 10),                        # ... two pairs at a time
    ((8, 2), 128, "bf16", 98, "interleaved", {}, 3, 1203, 10),                  # ... pair by pair
    ((4, 2), 64, "fp32", 30, "half", {}, 2, 9, 50),
    ((8, 8), 128, "fp32", 128, "interleaved", {}, 1, 1203, 10),
]
IDS = ["%dx%d_d%d_%s_r%d_%s_%dx%d" % (c[0][0], c[0][1], c[1], c[2], c[3], c[4], c[6], c[7]) for c in CASES]


def plan_of(case):
    s = case[5]
    low, high = s.get("low"), s.get("high")
    plan = pkv.make_rotary(case[3], layout=case[4], scaling=s.get("scaling", "none"), factor=s.get("factor", 1.0), original_positions=s.get("original", 0),
                           low=low, high=high)
    return plan, frequencies(case[3], **s)


@pytest.mark.parametrize("where", ["out", "in place", "inverse", "views"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_rotary_against_the_definition(case, where):
    heads, d, dtype, dim, layout, _, batch, tokens, first = case
    t = TYPES[dtype]
    g = torch.Generator().manual_seed(3)
    q, k = randn(g, batch, heads[0], tokens, d, dtype=t, scale=3.0), randn(g, batch, heads[1], tokens, d, dtype=t)
    positions = (first + torch.arange(tokens) + 11 * torch.arange(batch)[:, None]).to(torch.int32)
    plan, (freq, magnitude) = plan_of(case)
    cfg = config(heads, d, dtype)
    dp = positions.to(DEV)
    if where == "views":                                             # one buffer [batch][token][head][d], as a fused projection leaves it
        both = torch.full((batch, tokens, heads[0] + heads[1] + 1, d), 5.0, dtype=t, device=DEV)
        dq, dk = both[:, :, :heads[0]].transpose(1, 2), both[:, :, heads[0]:-1].transpose(1, 2)
        dq.copy_(q)
        dk.copy_(k)
        oq, ok = dq, dk
        dp = torch.stack([dp, dp + 1])[0] if batch > 1 else dp[0].expand(1, tokens)
        pkv.rotary(cfg, plan, dp, dq, dk)
        assert torch.all(both[:, :, -1] == 5.0)
    else:
        dq, dk = q.to(DEV), k.to(DEV)
        oq, ok = (dq, dk) if where == "in place" else (torch.full_like(dq, 9.0), torch.full_like(dk, 9.0))
        pkv.rotary(cfg, plan, dp, dq, dk, oq, ok, inverse=where == "inverse")
    for name, got, x in (("q", oq, q), ("k", ok, k)):
        want, size = rotate(x, positions[:, None], freq, magnitude, layout, where == "inverse")
        assert_rotated(got.cpu(), want, size, name)
        assert torch.equal(got.cpu()[..., dim:], x[..., dim:])
    if where in ("out", "inverse"):
        assert torch.equal(dq.cpu(), q) and torch.equal(dk.cpu(), k)


def test_one_tensor_alone_and_shared_positions():
    cfg, plan = config((4, 2), 64, "bf16"), pkv.make_rotary(64)
    g = torch.Generator().manual_seed(4)
    q, k = randn(g, 3, 4, 5, 64, dtype=torch.bfloat16).to(DEV), randn(g, 3, 2, 5, 64, dtype=torch.bfloat16).to(DEV)
    positions = torch.arange(100, 105, dtype=torch.int32, device=DEV).expand(3, 5)
    a, b, c, d = (torch.empty_like(x) for x in (q, k, q, k))
    pkv.rotary(cfg, plan, positions, q, k, a, b)
    pkv.rotary(cfg, plan, positions, q, None, c)
    pkv.rotary(cfg, plan, positions, None, k, None, d)
    assert torch.equal(a, c) and torch.equal(b, d)
    none = torch.empty(3, 4, 0, 64, dtype=torch.bfloat16, device=DEV)
    pkv.rotary(cfg, plan, positions[:, :0], none)                    # no tokens: nothing to do


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_inverse_is_the_gradient(layout):
    """The rotation is linear, so <y', R x> has the gradient R^T y' for x: by autograd of the definition in 64 bits, and by a
    difference of two rotations along a direction."""
    cfg = config((2, 1), 64, "fp32")
    plan = pkv.make_rotary(48, layout=layout, scaling="yarn", factor=4.0, original_positions=4096)
    freq, magnitude = frequencies(48, scaling="yarn", factor=4.0, original=4096, high=32.0)
    g = torch.Generator().manual_seed(5)
    x, dy, way = (torch.randn(2, 2, 7, 64, generator=g) for _ in range(3))
    positions = (1000 + torch.arange(7)).expand(2, 7).to(torch.int32)
    leaf = x.double().requires_grad_()
    r = 48
    a, b = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    angle = positions[:, None].double()[..., None] * torch.tensor(freq, dtype=torch.float64)
    p, q = leaf[..., a], leaf[..., b]
    w = dy.double()
    loss = (magnitude * ((p * angle.cos() - q * angle.sin()) * w[..., a] + (q * angle.cos() + p * angle.sin()) * w[..., b])).sum()
    loss = loss + (leaf[..., r:] * w[..., r:]).sum()
    loss.backward()
    got = torch.empty_like(dy, device=DEV)
    dp = positions.contiguous().to(DEV)
    pkv.rotary(cfg, plan, dp, dy.to(DEV), None, got, inverse=True)
    _, size = rotate(dy, positions[:, None], freq, magnitude, layout, True)
    assert_rotated(got.cpu(), leaf.grad, size)
    up, down = torch.empty_like(got), torch.empty_like(got)
    step = 0.5                                                        # linear: any step gives the derivative
    pkv.rotary(cfg, plan, dp, (x + step * way).to(DEV), None, up)
    pkv.rotary(cfg, plan, dp, (x - step * way).to(DEV), None, down)
    slope = ((up - down).double().cpu() / (2 * step) * w).sum()
    # each of the 1792 products is off by at most 1e-6 (|x| + |way|) |dy|, all below 5
    assert math.isclose(float(slope), float((got.cpu().double() * way.double()).sum()), abs_tol=1792 * 1e-6 * 50)


# ------------------------------------------------------------------------------------------------ appends
def empty_cache(cfg, dtype, lens, page, g, spare=3, positions=True):
    """A cache with garbage in every slot (NaN among it) and pages dealt out at random."""
    heads, d = cfg.num_kv_heads, cfg.head_dim
    need = [-(-n // page) for n in lens]
    width = max(1, max(need)) + 1
    total = heads * sum(need) + spare
    order = torch.randperm(total, generator=g).to(torch.int32)
    tables = torch.full((1, len(lens), heads, width), -7, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        for h in range(heads):
            tables[0, b, h, :n] = order[at:at + n]
            at += n
    pools = [torch.randn(total, page, d, generator=g).to(TYPES[dtype]) for _ in range(2)]
    for p in pools:
        p[:, :, 1] = math.nan
    pos = torch.full((total, page), -5, dtype=torch.int32) if positions else None
    lens_t = torch.tensor([lens], dtype=torch.int32)
    dev = [x.to(DEV) if x is not None else None for x in (*pools, tables, lens_t, pos)]
    return pkv.PagedCache(cfg, dev[0], dev[1], dev[2], dev[3], positions=dev[4]), pools, tables, pos


def bits(t):
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


# heads, d, dtype, rotary_dim (0: no plan), layout, page, lens, counts (None: all), tokens
APPENDS = [
    ((4, 2), 64, "fp32", 64, "half", 16, [1], None, 1),
    ((32, 8), 128, "bf16", 128, "half", 16, [17, 16, 1, 400], None, 1),
    ((8, 8), 64, "fp16", 32, "interleaved", 5, [3, 9, 40], [3, 0, 2], 3),
    ((6, 2), 128, "bf16", 0, "half", 1, [5, 7], [2, 2], 2),
    ((5, 1), 128, "fp16", 20, "half", 7, [30, 100, 64], [30, 1, 33], 33),
    ((6, 2), 64, "bf16", 26, "interleaved", 7, [30, 100, 64], [30, 1, 33], 33),
    ((8, 2), 64, "bf16", 64, "interleaved", 64, [700, 650], [600, 513], 600),
    ((4, 4), 128, "fp32", 128, "half", 32, [0, 5], [0, 5], 5),
    ((4, 1), 64, "bf16", 64, "half", 16, [20], [99], 4),                       # a count beyond the tokens: as if all
]


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: "%dx%d_d%d_%s_r%d_p%d_t%d" % (c[0][0], c[0][1], c[1], c[2], c[3], c[5], c[8]))
@pytest.mark.parametrize("with_q", [True, False])
def test_append_against_the_definition(case, with_q):
    heads, d, dtype, dim, layout, page, lens, counts, tokens = case
    t, cfg, batch = TYPES[dtype], config(heads, d, dtype), len(lens)
    g = torch.Generator().manual_seed(6)
    cache, pools, tables, pos = empty_cache(cfg, dtype, lens, page, g)
    k, v, q = (randn(g, batch, h, tokens, d, dtype=t) for h in (heads[1], heads[1], heads[0]))
    positions = torch.randint(0, 200000, (batch, tokens), generator=g).to(torch.int32)
    plan = pkv.make_rotary(dim, layout=layout) if dim else None
    ws = pkv.new_cache_workspace(cfg, cache)
    q_out = torch.full_like(q, 3.0, device=DEV)
    pkv.append_cache(cfg, cache, 0, positions.to(DEV), k.to(DEV), v.to(DEV), ws, q=q.to(DEV) if with_q else None, q_out=q_out if with_q else None,
                     rotary=plan, counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV))
    pkv.check_status(ws)
    freq = frequencies(dim)[0] if dim else []
    want_k, size_k = rotate(k, positions[:, None], freq, 1.0, layout)
    want_q, size_q = rotate(q, positions[:, None], freq, 1.0, layout)
    got_k, got_v, got_pos = cache.k_pool.cpu().view(-1, d), cache.v_pool.cpu().view(-1, d), cache.positions.cpu().view(-1)
    touched = torch.zeros(got_pos.numel(), dtype=torch.bool)
    for b, n in enumerate(lens):
        count = tokens if counts is None else min(max(counts[b], 0), tokens)
        for h in range(heads[1]):
            slots = torch.tensor([int(tables[0, b, h, r // page]) * page + r % page for r in range(n - count, n)], dtype=torch.long)
            touched[slots] = True
            assert_rotated(got_k[slots], want_k[b, h, :count], size_k[b, h, :count], (b, h))
            assert torch.equal(got_k[slots][:, dim:], k[b, h, :count, dim:])
            assert torch.equal(bits(got_v[slots]), bits(v[b, h, :count]))
            assert torch.equal(got_pos[slots], positions[b, :count])
        if with_q:
            assert_rotated(q_out[b, :, :count].cpu(), want_q[b, :, :count], size_q[b, :, :count], (b, "q"))
            assert torch.all(q_out[b, :, count:] == 3.0)
    # everything else is as it was
    assert torch.equal(bits(got_k)[~touched], bits(pools[0]).view(-1, d)[~touched])
    assert torch.equal(bits(got_v)[~touched], bits(pools[1]).view(-1, d)[~touched])
    assert torch.equal(got_pos[~touched], pos.view(-1)[~touched])


def test_append_reports_bad_pages_and_rows_outside_the_table():
    cfg = config((2, 2), 64, "bf16")
    g = torch.Generator().manual_seed(7)
    cache, pools, tables, pos = empty_cache(cfg, "bf16", [9, 9, 9, 9], 4, g)
    tables[0, 1, 0, 2], tables[0, 2, 1, 2] = cache.num_pages, -1     # behind the pool, and none
    cache.tables.copy_(tables)
    cache.lens.copy_(torch.tensor([[9, 9, 9, 0]], dtype=torch.int32))  # the last sequence: row -1
    ws = pkv.new_cache_workspace(cfg, cache)
    k, v = (torch.randn(4, 2, 1, 64, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    pkv.append_cache(cfg, cache, 0, torch.zeros(4, 1, dtype=torch.int32, device=DEV), k, v, ws)
    with pytest.raises(pkv.PkvError, match="0x4"):
        pkv.check_status(ws)
    new = {(0, 0), (0, 1), (1, 1), (2, 0)}
    slots = {int(tables[0, b, h, 2]) * 4: (b, h) for b, h in new}
    got = bits(cache.k_pool.cpu()).view(-1, 64)
    for s in range(got.shape[0]):
        want = bits(k[slots[s]].cpu())[0] if s in slots else bits(pools[0]).view(-1, 64)[s]
        assert torch.equal(got[s], want), s
    # a sequence longer than its table
    cache.lens.fill_(cache.max_pages * 4 + 1)
    ws.zero_()
    before = cache.k_pool.clone()
    pkv.append_cache(cfg, cache, 0, torch.zeros(4, 1, dtype=torch.int32, device=DEV), k, v, ws)
    with pytest.raises(pkv.PkvError, match="0x4"):
        pkv.check_status(ws)
    assert torch.equal(bits(cache.k_pool), bits(before))


def test_appends_without_positions_take_keys_as_they_are():
    cfg = config((2, 2), 64, "fp16")
    g = torch.Generator().manual_seed(8)
    cache, _, tables, _ = empty_cache(cfg, "fp16", [3], 4, g, positions=False)
    k, v = (torch.randn(1, 2, 3, 64, generator=g).to(torch.float16) for _ in range(2))
    ws = pkv.new_cache_workspace(cfg, cache)
    pkv.append_cache(cfg, cache, 0, None, k.to(DEV), v.to(DEV), ws)
    pkv.check_status(ws)
    for h in range(2):
        assert torch.equal(cache.k_pool[int(tables[0, 0, h, 0]), :3].cpu(), k[0, h])


def test_tensors_that_do_not_fit_are_refused():
    cfg = config((4, 2), 64, "bf16")
    g = torch.Generator().manual_seed(9)
    cache, _, _, _ = empty_cache(cfg, "bf16", [3, 4], 4, g)
    ws = pkv.new_cache_workspace(cfg, cache)
    plan = pkv.make_rotary(64)
    k = torch.zeros(2, 2, 1, 64, dtype=torch.bfloat16, device=DEV)
    q = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16, device=DEV)
    p = torch.zeros(2, 1, dtype=torch.int32, device=DEV)
    for bad in (dict(k=k.half()), dict(k=k[:1]), dict(k=k[:, :1]), dict(v=k.cpu()), dict(q=k), dict(q=q[..., ::2]), dict(positions=p.long()), dict(positions=p[:1]),
                dict(positions=None), dict(counts=p), dict(counts=p[:, 0].long()), dict(ws=ws.float()), dict(q_out=q)):
        kw = {**dict(k=k, v=k, positions=p, ws=ws), **bad}
        with pytest.raises(ValueError):
            pkv.append_cache(cfg, cache, 0, kw.pop("positions"), kw.pop("k"), kw.pop("v"), kw.pop("ws"), rotary=plan, **kw)
    with pytest.raises(pkv.PkvError):
        pkv.append_cache(cfg, cache, 1, p, k, k, ws)                 # no such layer
    with pytest.raises(pkv.PkvError):
        pkv.append_cache(cfg, cache, 0, p, k, k, ws[:256])           # a workspace that is too small
    for bad in (dict(q=None, k=None), dict(q=q.float(), k=None), dict(q=q, k=k[:1]), dict(q=None, k=k, q_out=q), dict(q=q.cpu(), k=None)):
        with pytest.raises(ValueError):
            pkv.rotary(cfg, plan, p, bad["q"], bad["k"], bad.get("q_out"))
    with pytest.raises(ValueError):
        pkv.append_cache(config((4, 2), 64, "fp16"), cache, 0, p, k, k, ws)      # another configuration's cache
    for call in (lambda: pkv.rotary(cfg, None, p, q), lambda: pkv.append_cache(cfg, cache, 0, p, k, k, ws, rotary=128)):
        with pytest.raises(ValueError):                              # no plan
            call()
