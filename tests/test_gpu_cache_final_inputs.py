"""Scores of inputs that the caller calls final: what calls of the library are still to write is waited for, however many other calls
of the library come between, run on another stream or are captured meanwhile."""
import pytest
import torch

import paper_2406_02069_b200 as pkv
from paper_2406_02069_b200 import binding
from test_gpu_cache_pages import Pool

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Decoding:
    """Appends of one token with queries, to a cache of its own."""

    def __init__(self):
        self.x = Pool(pkv.make_config(num_layers=1, num_q_heads=4, num_kv_heads=2, head_dim=64, window=1, pool_kernel=1, dtype="bf16", avg_budget=1), [[5]], 4, 20, 4)
        self.q, self.k = (torch.randn(1, h, 1, 64, device=DEV).to(torch.bfloat16) for h in (4, 2))
        self.q_out, self.plan = torch.zeros_like(self.q), pkv.make_rotary(64)
        self.positions = torch.zeros(1, 1, dtype=torch.int32, device=DEV)

    def append(self, stream=None):
        pkv.append_cache(self.x.cfg, self.x.cache, 0, self.positions, self.k, self.k, self.x.ws, q=self.q, q_out=self.q_out, rotary=self.plan, stream=stream)


@pytest.mark.parametrize("where,calls", [("same stream", 90), ("other stream", 90), ("other stream", 400), ("captured", 200), ("none", 0)])
def test_scores_wait_for_the_rotation_behind_many_appends(where, calls):
    cfg = pkv.make_config(num_layers=2, num_q_heads=4, num_kv_heads=1, head_dim=128, window=8, pool_kernel=5, dtype="bf16", avg_budget=24, inputs_final=True)
    n = 300                                                          # (few CTAs of the rotation, so that the scores find room beside it)
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(1, h, n, 128, generator=g).to(torch.bfloat16).to(DEV) for h in (4, 1, 1))
    qr, kr = (torch.zeros(8 << 20, dtype=torch.uint8, device=DEV)[: t.numel() * 2].view(torch.bfloat16).view(t.shape) for t in (q, k))   # (memory that no output had before)
    plan = pkv.make_rotary(128)
    positions = torch.arange(n, dtype=torch.int32, device=DEV)[None]
    ws = pkv.new_workspace(cfg, 1, n, DEV)
    rows = pkv.total_rows(cfg, pkv.layer_budgets(cfg)[0], [n])
    filler, slow = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV), torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    decoding, main, side = Decoding(), torch.cuda.Stream(), torch.cuda.Stream()

    def step(held):
        qr.copy_(q)
        kr.copy_(k)
        out = [torch.zeros(rows, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)] + [torch.zeros(rows, dtype=torch.int32, device=DEV)]
        torch.cuda.synchronize()
        with torch.cuda.stream(main):
            if held:
                binding.slow_copy(slow, filler, steps=2048)          # lets the calls behind it start at once
            pkv.rotary(cfg, plan, positions, qr, kr)
            if held and where == "captured":                         # (nothing of it runs)
                graph = torch.cuda.CUDAGraph()
                graph.capture_begin(capture_error_mode="thread_local")
            for _ in range(calls if held else 0):
                decoding.append(side if where == "other stream" else None)
            if held and where == "captured":
                graph.capture_end()
            pkv.compress_layer(cfg, 0, qr[:, :, n - 8:], kr, v, [n], out[0], out[1], out[2], ws)
        torch.cuda.synchronize()
        return out
    want = step(False)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(want, step(True)))


@pytest.mark.parametrize("first", ["graph", "call"])
def test_graphs_and_calls_are_ordered_at_their_borders(first):
    """A rotation that is held, replayed from a graph with the scores called behind it, or called with the scores replayed behind
    it: neither side has the other's outputs in its record."""
    cfg = pkv.make_config(num_layers=2, num_q_heads=4, num_kv_heads=1, head_dim=128, window=8, pool_kernel=5, dtype="bf16", avg_budget=24, inputs_final=True)
    n = 300
    g = torch.Generator().manual_seed(6)
    q, k, v = (torch.randn(1, h, n, 128, generator=g).to(torch.bfloat16).to(DEV) for h in (4, 1, 1))
    qr, kr = (torch.zeros(8 << 20, dtype=torch.uint8, device=DEV)[: t.numel() * 2].view(torch.bfloat16).view(t.shape) for t in (q, k))
    plan, positions = pkv.make_rotary(128), torch.arange(n, dtype=torch.int32, device=DEV)[None]
    ws = pkv.new_workspace(cfg, 1, n, DEV)
    rows = pkv.total_rows(cfg, pkv.layer_budgets(cfg)[0], [n])
    out = [torch.zeros(rows, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)] + [torch.zeros(rows, dtype=torch.int32, device=DEV)]
    filler, slow = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV), torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)

    def rotate_late():
        binding.slow_copy(slow, filler, steps=512)
        pkv.rotary(cfg, plan, positions, qr, kr)

    def compress():
        pkv.compress_layer(cfg, 0, qr[:, :, n - 8:], kr, v, [n], out[0], out[1], out[2], ws)
    main = torch.cuda.Stream()
    with torch.cuda.stream(main):
        rotate_late()
        compress()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        (rotate_late if first == "graph" else compress)()
    ends = []
    for wait in (True, False, False):
        qr.copy_(q)
        kr.copy_(k)
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(main):
            graph.replay() if first == "graph" else rotate_late()
            if wait:
                torch.cuda.synchronize()
            compress() if first == "graph" else graph.replay()
        torch.cuda.synchronize()
        ends.append([t.clone() for t in out])
    assert all(torch.equal(a, b) for end in ends[1:] for a, b in zip(ends[0], end))
