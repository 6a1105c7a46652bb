"""Growing cache: calls on several streams, captured calls that share a workspace, calls behind and ahead of the library's others."""
import random

import pytest
import torch

import paper_2406_02069_b200 as pkv
from paper_2406_02069_b200 import binding
from cache_oracle import attend
from test_gpu_cache_attention import Data
from test_gpu_cache_pages import Pool, add_tensor

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_calls_on_a_given_stream_are_ordered_there():
    """Everything of a decode step on one side stream, behind a slow kernel that makes its inputs."""
    x = Data((8, 2), 128, "bf16", 16, [200, 33])
    want, want_lse = x.run()
    side = torch.cuda.Stream()
    q, out, lse = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 8, 128, device=DEV), torch.zeros(2, 8, device=DEV)
    src = x.q.to(DEV)
    torch.cuda.synchronize()
    binding.slow_copy(q, src, stream=side)
    pkv.decode_attention_cache(x.cfg, x.cache, 0, q, out, x.ws, lse=lse, stream=side)
    side.synchronize()
    assert torch.equal(out.cpu(), want) and torch.equal(lse.cpu(), want_lse)
    # rotary, append and attention in a row: the rotation in place is what the append sees
    plan = pkv.make_rotary(128)
    k = torch.zeros(2, 2, 1, 128, dtype=torch.bfloat16, device=DEV)
    fresh = torch.randn(2, 2, 1, 128, device=DEV).to(torch.bfloat16)
    positions = torch.full((2, 1), 77, dtype=torch.int32, device=DEV)
    turned = torch.empty_like(fresh)
    pkv.rotary(x.cfg, plan, positions, None, fresh, None, turned)
    torch.cuda.synchronize()
    binding.slow_copy(k, fresh, stream=side)
    pkv.append_cache(x.cfg, x.cache, 0, positions, k, k, x.ws, rotary=plan, stream=side)
    side.synchronize()
    for b, n in enumerate((200, 33)):
        for h in range(2):
            page, slot = int(x.tables[0, b, h, (n - 1) // 16]), (n - 1) % 16
            assert torch.equal(x.cache.k_pool[page, slot], turned[b, h, 0]) and torch.equal(x.cache.v_pool[page, slot], fresh[b, h, 0])


def test_streams_with_workspaces_of_their_own_run_side_by_side():
    a, b = Data((8, 2), 128, "bf16", 16, [3000, 100, 7], seed=1), Data((4, 4), 64, "fp16", 7, [900, 1500], seed=2)
    want = [x.run() for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[torch.zeros_like(w, device=DEV) for w in ws] for ws in want]
    qs = [x.q.to(DEV) for x in (a, b)]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, q, s, (out, lse) in zip((a, b), qs, streams, got):
            pkv.decode_attention_cache(x.cfg, x.cache, 0, q, out, x.ws, lse=lse, stream=s)
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(u, v.cpu()) for u, v in zip(w, g))


def capture(call):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    return graph


def test_two_graphs_share_a_workspace_one_after_the_other():
    a, b = Data((8, 1), 128, "bf16", 16, [6000], seed=1), Data((4, 4), 64, "fp32", 7, [900, 1500, 3], seed=2)
    want = [x.run() for x in (a, b)]
    ws = max((a.ws, b.ws), key=lambda w: w.numel())                  # one workspace for caches of other shapes and types
    ws.zero_()
    got = [[torch.zeros_like(w, device=DEV) for w in one] for one in want]
    qs = [x.q.to(DEV) for x in (a, b)]
    graphs = [capture(lambda x=x, q=q, o=o: pkv.decode_attention_cache(x.cfg, x.cache, 0, q, o[0], ws, lse=o[1])) for x, q, o in zip((a, b), qs, got)]
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for o in got:
            o[0].fill_(3.0)
        for i in order:
            graphs[i].replay()
        for w, g in zip(want, got):
            assert all(torch.equal(u, v.cpu()) for u, v in zip(w, g))
    pkv.check_status(ws)


def test_captured_page_calls_follow_the_device():
    """A reserve captured once grows the cache at every replay; a fork and a compaction captured once follow their inputs."""
    x = Pool(pkv.make_config(num_layers=1, num_q_heads=2, num_kv_heads=2, head_dim=64, window=1, pool_kernel=1, dtype="bf16", avg_budget=1),
             [[3, 4, 5], [8, 1, 2]], 4, 400, 12)
    add, parents = add_tensor([0, 0, 0]), add_tensor([0, 1, 2])
    reserve = capture(lambda: pkv.cache_reserve(x.cfg, x.cache, add, x.ws))
    fork = capture(lambda: pkv.cache_fork(x.cfg, x.cache, parents, x.ws))
    compact = capture(lambda: pkv.cache_compact(x.cfg, x.cache, x.ws))
    x.check_pools([(s, t, 4) for s, t in x.lists.compact()[1]])      # (the warm-up's)
    r = random.Random(1)
    for _ in range(6):
        more, new = [r.choice([0, 1, 3]) for _ in range(3)], [r.randrange(3) for _ in range(3)]
        add.copy_(add_tensor(more))
        parents.copy_(add_tensor(new))
        reserve.replay()
        fork.replay()
        compact.replay()
        x.lists.fork([0, 1, 2], [more] * 2)
        copies = x.lists.fork(new, [[0] * 3] * 2)[1]
        moves = x.lists.compact()[1]
        pkv.check_status(x.ws)
        x.lists.check(x.cache.tables.cpu(), x.cache.lens.cpu(), x.cache.refs.cpu())
        for m in (copies, [(s, t, 4) for s, t in moves]):
            for pool in x.pools:
                old = pool.clone()
                for s, t, rows in m:
                    pool[t, :rows] = old[s, :rows]
        x.check_pools([])


def test_scores_of_final_inputs_wait_for_the_rotation():
    """Keys that pyramidkv_rotary is still to write are not read early, even where the caller calls its inputs final, and even
    with many small calls of the library between."""
    cfg = pkv.make_config(num_layers=2, num_q_heads=8, num_kv_heads=2, head_dim=128, window=8, pool_kernel=5, dtype="bf16", avg_budget=64, inputs_final=True)
    n = 900
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(1, h, n, 128, generator=g).to(torch.bfloat16).to(DEV) for h in (8, 2, 2))
    plan = pkv.make_rotary(128)
    positions = torch.arange(n, dtype=torch.int32, device=DEV)[None]
    ws = pkv.new_workspace(cfg, 1, n, DEV)
    rows = pkv.total_rows(cfg, pkv.layer_budgets(cfg)[0], [n])
    small = torch.randn(1, 2, 1, 128, device=DEV).to(torch.bfloat16)
    filler, slow = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV), torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)

    def step(between):
        qr, kr = q.clone(), k.clone()
        out = [torch.zeros(rows, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)] + [torch.zeros(rows, dtype=torch.int32, device=DEV)]
        torch.cuda.synchronize()
        if between:
            binding.slow_copy(slow, filler, steps=256)               # lets the calls behind it start at once
        pkv.rotary(cfg, plan, positions, qr, kr)
        for _ in range(30 if between else 0):
            pkv.rotary(cfg, plan, positions[:, :1], None, small)
        pkv.compress_layer(cfg, 0, qr[:, :, n - 8:], kr, v, [n], out[0], out[1], out[2], ws)
        torch.cuda.synchronize()
        return out
    want, got = step(False), step(True)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("seed", range(12))
def test_attention_at_random(seed):
    r = random.Random(100 + seed)
    kv = r.choice([1, 2, 3, 8])
    group, d, dtype = r.choice([1, 2, 4, 5, 8, 9]), r.choice([64, 128]), r.choice(["bf16", "fp16", "fp32"])
    batch = r.choice([1, 2, 5, 33, 140])
    top = r.choice([1, 20, 90, 400] + ([3000] if batch < 5 else []))
    lens = [r.randint(0, top) for _ in range(batch)]
    x = Data((group * kv, kv), d, dtype, r.choice([1, 3, 16, 32, 100]), lens, seed=seed)
    positions = r.random() < 0.6
    kw = dict(use_positions=positions, softcap=r.choice([0.0, 5.0, 50.0]))
    if positions:
        kw.update(window=r.choice([0, 1, 30, 500]), prefix=r.choice([0, 2, 50]))
        if r.random() < 0.5:
            kw["slopes"] = torch.rand(group * kv) * 0.3
        x.q_pos = x.q_pos - torch.tensor([r.choice([0, 0, 0, 5, 100]) for _ in lens], dtype=torch.int32)   # some rows are later than the query
    out, lse = x.run(**kw)
    x.check(out, lse, **kw)


def test_inactive_sequences_of_a_batch_are_left_alone():
    """A slot without rows, a slot that takes no new token: zeros out, nothing written for it."""
    x = Data((4, 2), 64, "bf16", 4, [9, 0, 6, 5])
    plan = pkv.make_rotary(64)
    before = [t.clone() for t in (x.cache.k_pool, x.cache.v_pool, x.cache.positions)]
    q = torch.randn(4, 4, 1, 64, device=DEV).to(torch.bfloat16)
    q0 = q.clone()
    k = torch.randn(4, 2, 1, 64, device=DEV).to(torch.bfloat16)
    counts = add_tensor([1, 0, 0, 1])
    pkv.append_cache(x.cfg, x.cache, 0, add_tensor([[50], [51], [52], [53]]), k, k, x.ws, q=q, rotary=plan, counts=counts)
    out = torch.full((4, 4, 64), 9.0, device=DEV)
    pkv.decode_attention_cache(x.cfg, x.cache, 0, q, out, x.ws)
    pkv.check_status(x.ws)
    assert torch.equal(q[1:3], q0[1:3]) and not torch.equal(q[0], q0[0])
    assert torch.all(out[1] == 0)
    changed = (x.cache.positions != before[2]).nonzero().tolist()
    want = sorted([int(x.tables[0, b, h, (n - 1) // 4]), (n - 1) % 4] for b, n in ((0, 9), (3, 5)) for h in range(2))
    assert sorted(changed) == want
    for h in range(2):                                               # a sequence that took nothing still attends to what it has
        w, _, size = attend(q[2, 2 * h:2 * h + 2, 0].cpu(), x.k[2][h], x.v[2][h])
        assert torch.all((out[2, 2 * h:2 * h + 2].cpu().double() - w).abs() <= 1e-4 * size + 1e-7)


@pytest.mark.parametrize("page", [1, 4])
def test_a_long_run_of_steps_with_nothing_waited_for(page):
    """Reserve, append and attend sixty times in a row without looking: every step sees the lengths, pages and rows of the ones
    ahead of it, although its kernels are on the device before those have finished."""
    heads, group, d, steps, layers = 2, 4, 64, 60, 2
    x = Pool(pkv.make_config(num_layers=layers, num_q_heads=heads * group, num_kv_heads=heads, head_dim=d, window=1, pool_kernel=1, dtype="bf16", avg_budget=1),
             [[3, 0, 7]] * layers, page, 4 * (steps + 10) * 3 * heads * layers // page, steps // page + 12)
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(steps, layers, 3, h, 1, d, generator=g).to(torch.bfloat16) for h in (heads * group, heads, heads))
    dq, dk, dv = q.to(DEV), k.to(DEV), v.to(DEV)
    r = random.Random(page)
    adds = [[1, r.choice([0, 1]), 1] for _ in range(steps)]
    dadd = add_tensor(adds)
    granted = torch.zeros(steps, layers, 3, dtype=torch.int32, device=DEV)
    out = torch.zeros(steps, layers, 3, heads * group, d, device=DEV)
    positions = torch.zeros(3, 1, dtype=torch.int32, device=DEV)
    rows = [[[[p[x.lists.row(l, b, h, i) // page, x.lists.row(l, b, h, i) % page] for i in range(x.lists.lens[l][b])] for p in x.pools[:2]]
             for b in range(3) for h in range(heads)] for l in range(layers)]
    torch.cuda.synchronize()
    for s in range(steps):
        pkv.cache_reserve(x.cfg, x.cache, dadd[s], x.ws, granted=granted[s])
        for l in range(layers):
            pkv.append_cache(x.cfg, x.cache, l, positions, dk[s, l], dv[s, l], x.ws, counts=granted[s, l])
            pkv.decode_attention_cache(x.cfg, x.cache, l, dq[s, l], out[s, l], x.ws)
    pkv.check_status(x.ws)
    got = out.cpu()
    for s in range(steps):
        for l in range(layers):
            for b in range(3):
                for h in range(heads):
                    ks, vs = rows[l][b * heads + h]
                    if adds[s][b]:
                        ks.append(k[s, l, b, h, 0])
                        vs.append(v[s, l, b, h, 0])
                    hq = slice(h * group, (h + 1) * group)
                    if not ks:
                        assert torch.all(got[s, l, b, hq] == 0)
                        continue
                    want, _, size = attend(q[s, l, b, hq, 0], torch.stack(ks), torch.stack(vs))
                    assert torch.all((got[s, l, b, hq].double() - want).abs() <= 1e-4 * size + 1e-7), (s, l, b, h)


def test_the_largest_batch():
    lens = [(7 * i) % 5 for i in range(1024)]
    x = Data((2, 1), 64, "fp16", 2, lens)
    out, lse = x.run(use_positions=True, window=6)
    x.check(out, lse, use_positions=True, window=6)
    # one sequence goes on as 1024
    p = Pool(pkv.make_config(num_layers=1, num_q_heads=1, num_kv_heads=1, head_dim=64, window=1, pool_kernel=1, dtype="bf16", avg_budget=1), [[6, 9]], 4, 3000, 4)
    to = p.other(1024)
    parents, add = [1] * 600 + [0] * 400 + [-1] * 24, [[i % 3 for i in range(1024)]]
    pkv.cache_fork(p.cfg, p.cache, add_tensor(parents), p.ws, add=add_tensor(add), to=to)
    pkv.check_status(p.ws)
    copies = p.lists.fork(parents, add)[1]
    p.lists.check(to.tables.cpu(), to.lens.cpu(), to.refs.cpu())
    p.check_pools(copies)
