"""Decode attention over a paged cache whose lengths live on the device, against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2406_02069_b200 as pkv
from cache_oracle import TYPES, attend

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Data:
    """Rows of a batch, and the cache that holds them: garbage (NaN among it) in every slot that no row has."""

    def __init__(self, heads, d, dtype, page, lens, seed=1, spare_pages=1, q_scale=2.0, start=None):
        self.heads, self.d, self.page, self.lens, self.t = heads, d, page, lens, TYPES[dtype]
        self.cfg = pkv.make_config(num_layers=1, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=d, window=1, pool_kernel=1, dtype=dtype, avg_budget=1)
        g = self.g = torch.Generator().manual_seed(seed)
        batch, kv = len(lens), heads[1]
        need = [-(-n // page) for n in lens]
        total = kv * sum(need) + 2
        order = torch.randperm(total, generator=g).to(torch.int32)
        self.tables = torch.full((1, batch, kv, max(1, max(need) + spare_pages)), -9, dtype=torch.int32)
        self.k_pool, self.v_pool = (torch.full((total, page, d), math.nan).to(self.t) for _ in range(2))
        self.pos_pool = torch.full((total, page), -3, dtype=torch.int32)
        self.q = (q_scale * torch.randn(batch, heads[0], d, generator=g)).to(self.t)
        self.k, self.v, self.pos = [], [], []
        at = 0
        for b, n in enumerate(lens):
            gaps = torch.randint(1, 6, (kv, n), generator=g)
            self.pos.append((gaps.cumsum(1) - gaps[:, :1]).to(torch.int32))      # ascending from 0, another list per head
            self.k.append(torch.randn(kv, n, d, generator=g).to(self.t))
            self.v.append(torch.randn(kv, n, d, generator=g).to(self.t))
            for h in range(kv):
                self.tables[0, b, h, :need[b]] = order[at:at + need[b]]
                at += need[b]
        self.q_pos = torch.tensor([int(p[:, -1].max()) if p.numel() else 7 for p in self.pos], dtype=torch.int32)
        self.fill()

    def fill(self):
        for b, n in enumerate(self.lens):
            for h in range(self.heads[1]):
                for j in range(-(-n // self.page)):
                    lo, hi = j * self.page, min(n, (j + 1) * self.page)
                    p = int(self.tables[0, b, h, j])
                    self.k_pool[p, :hi - lo], self.v_pool[p, :hi - lo] = self.k[b][h, lo:hi], self.v[b][h, lo:hi]
                    self.pos_pool[p, :hi - lo] = self.pos[b][h, lo:hi]
        lens = torch.tensor([self.lens], dtype=torch.int32)
        dev = [x.to(DEV) for x in (self.k_pool, self.v_pool, self.tables, lens, self.pos_pool)]
        self.cache = pkv.PagedCache(self.cfg, dev[0], dev[1], dev[2], dev[3], positions=dev[4])
        self.ws = pkv.new_cache_workspace(self.cfg, self.cache)

    def run(self, use_positions=False, status=True, **kw):
        out = torch.full((len(self.lens), self.heads[0], self.d), 7.0, device=DEV)
        lse = torch.full((len(self.lens), self.heads[0]), 7.0, device=DEV)
        if kw.get("slopes") is not None:
            kw["slopes"] = kw["slopes"].to(DEV)
        pkv.decode_attention_cache(self.cfg, self.cache, 0, self.q.to(DEV), out, self.ws, lse=lse,
                                   q_positions=self.q_pos.to(DEV) if use_positions else None, **kw)
        if status:
            pkv.check_status(self.ws)
        return out.cpu(), lse.cpu()

    def check(self, out, lse, use_positions=False, tolerance=1e-4, **kw):
        """tolerance: exponents x = q.k log2(e)/sqrt(d) take d + 8 roundings at most of terms whose absolute sum is below 40
        here (they come in groups of 16 products: d / 16 + 8 of sums below that), at most 16 * 2^-24 * 40 = 4e-5 in x and in
        a weight's factor 2^x; a cap or a bias of up to 300 rounds by 300 * 2^-24 = 2e-5 more, exponential and sums by 1e-6 each."""
        group = self.heads[0] // self.heads[1]
        for b in range(len(self.lens)):
            for h in range(self.heads[1]):
                hq = slice(h * group, (h + 1) * group)
                more = dict(kw)
                if more.get("slopes") is not None:
                    more["slopes"] = more["slopes"][hq]
                want, want_lse, size = attend(self.q[b, hq], self.k[b][h], self.v[b][h], positions=self.pos[b][h],
                                              q_position=int(self.q_pos[b]) if use_positions else None, **more)
                off = (out[b, hq].double() - want).abs() - tolerance * size
                assert torch.all(off <= 1e-7), (b, h, float(off.max()))
                assert torch.equal(torch.isinf(lse[b, hq]), torch.isinf(want_lse)), (b, h)
                fine = ~torch.isinf(want_lse)
                assert torch.all((lse[b, hq].double() - want_lse)[fine].abs() <= tolerance), (b, h)


# (query heads, KV heads), d, dtype, page, lens
CASES = [
    ((4, 2), 64, "fp32", 16, [64]),
    ((2, 2), 128, "bf16", 16, [1, 0, 2]),                            # a single row, none
    ((3, 1), 128, "fp16", 1, [15, 16, 17]),
    ((8, 2), 64, "bf16", 5, [63, 64, 65, 66]),                       # around a tile
    ((5, 1), 128, "bf16", 16, [127, 129, 700]),                      # a block of eight with five heads
    ((8, 1), 128, "bf16", 64, [5000]),                               # split over many CTAs
    ((8, 1), 64, "fp16", 7, [3001, 1]),
    ((12, 1), 128, "fp16", 16, [900, 33]),                           # two blocks, the second of four heads
    ((40, 2), 64, "bf16", 16, [300]),                                # three blocks of eight
    ((32, 32), 128, "bf16", 16, [100, 513, 64, 1, 9]),
    ((32, 8), 128, "fp16", 33, [4097, 129, 1000]),
    ((1, 1), 128, "fp32", 16, [1]),
    ((7, 7), 128, "fp32", 3, [65, 64, 200]),
    ((10, 2), 64, "fp32", 16, [2000, 0, 31]),
    ((8, 1), 128, "fp32", 64, [3000]),
    ((16, 1), 128, "fp32", 8, [257]),
    ((4, 1), 64, "bf16", 16, [(37 * i) % 130 for i in range(300)]),  # many short ones, several to a CTA
    ((8, 8), 64, "fp32", 4, [(29 * i) % 70 for i in range(70)]),
]
IDS = ["%dx%d_d%d_%s_p%d_n%d" % (c[0][0], c[0][1], c[1], c[2], c[3], c[4][0]) for c in CASES]
WAYS = {"plain": {}, "causal": dict(use_positions=True), "scale": dict(scale=0.03),
        "cap": dict(softcap=3.0), "window": dict(use_positions=True, window=40), "window and prefix": dict(use_positions=True, window=100, prefix=9),
        "all": dict(use_positions=True, window=700, prefix=3, softcap=20.0, slopes=True)}


@pytest.mark.parametrize("way", list(WAYS))
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_attention_against_the_definition(case, way):
    x = Data(*case)
    kw = dict(WAYS[way])
    if kw.get("slopes"):
        kw["slopes"] = 2.0 ** (-8.0 * torch.arange(1, case[0][0] + 1) / case[0][0])
    out, lse = x.run(**kw)
    x.check(out, lse, **kw)
    again = x.run(**kw)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])           # the same bits every time


@pytest.mark.parametrize("dtype,group", [("bf16", 4), ("fp16", 8), ("fp32", 2)])
def test_a_query_that_sees_nothing_gets_zeros(dtype, group):
    x = Data((group * 2, 2), 128, dtype, 16, [200, 90, 0, 500])
    x.q_pos = torch.tensor([-1, 0, 5, 100000], dtype=torch.int32)              # before all rows, only the first, no rows, far behind
    kw = dict(use_positions=True, window=50)
    out, lse = x.run(**kw)
    x.check(out, lse, **kw)
    assert torch.all(out[0] == 0) and torch.all(out[2:] == 0) and torch.all(lse[[0, 2, 3]] == -math.inf)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_rows_that_are_not_seen_may_hold_anything(dtype):
    x = Data((4, 1), 64, dtype, 16, [300, 40])
    kw = dict(use_positions=True, window=60, prefix=1)
    for b in range(2):
        far = int(x.q_pos[b]) - x.pos[b][0].long()
        hidden = (far >= 60) & (x.pos[b][0] >= 1)
        assert hidden.any()
        x.k[b][0][hidden], x.v[b][0][hidden] = math.nan, math.inf
    x.fill()
    out, lse = x.run(**kw)
    x.check(out, lse, **kw)


@pytest.mark.parametrize("what", ["inf", "-inf", "both signs", "nan"])
@pytest.mark.parametrize("dtype,d,group", [("fp32", 128, 4), ("bf16", 128, 4), ("fp16", 128, 5), ("bf16", 64, 8), ("fp16", 64, 2)])
def test_infinities_and_nan_in_the_values_stay_in_their_channel(dtype, d, group, what):
    x = Data((2 * group, 2), d, dtype, 16, [700, 90], q_scale=1.5)
    inf = math.inf
    v = x.v[0][1]
    if what == "both signs":
        v[10, 3], v[600, 3], v[10, 40] = inf, -inf, -inf
    else:
        v[10, 3], v[699, d - 1] = float(what), float(what)
    x.fill()
    out, _ = x.run(softcap=30.0)
    for b in range(2):
        for h in range(2):
            hq = slice(h * group, (h + 1) * group)
            want, _, _ = attend(x.q[b, hq], x.k[b][h], x.v[b][h], softcap=30.0)
            got = out[b, hq].double()
            assert torch.equal(torch.isnan(got), torch.isnan(want)), (b, h)
            special = ~torch.isfinite(want)
            assert torch.equal(got[special & ~torch.isnan(want)], want[special & ~torch.isnan(want)]), (b, h)
            w = torch.softmax(30 * torch.tanh(x.q[b, hq].double() @ x.k[b][h].double().T / math.sqrt(d) / 30), -1)
            size = (w[:, :, None] * x.v[b][h].double().abs()).sum(1)
            assert torch.all((got - want).abs()[~special] <= 1e-4 * size[~special] + 1e-7), (b, h)


def test_nan_and_infinities_in_keys_reach_only_their_heads():
    x = Data((8, 2), 128, "bf16", 16, [300])
    x.k[0][1][17, 5] = math.nan
    x.fill()
    out, lse = x.run()
    assert torch.all(torch.isnan(out[0, 4:])) and torch.all(torch.isnan(lse[0, 4:]))
    want, _, size = attend(x.q[0, :4], x.k[0][0], x.v[0][0])
    assert torch.all((out[0, :4].double() - want).abs() <= 1e-4 * size + 1e-7)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bad_pages_are_left_out_and_reported(dtype):
    x = Data((4, 2), 64, dtype, 16, [100, 70])
    tables = x.tables.clone()
    tables[0, 0, 1, 2], tables[0, 1, 0, 4] = x.cache.num_pages, -1
    x.cache.tables.copy_(tables)
    out, lse = x.run(status=False)
    with pytest.raises(pkv.PkvError, match="0x4"):
        pkv.check_status(x.ws)
    keep = torch.ones(100, dtype=torch.bool)
    keep[32:48] = False
    x.k[0], x.v[0] = x.k[0].clone(), x.v[0].clone()
    want, _, size = attend(x.q[0, 2:], x.k[0][1][keep], x.v[0][1][keep])
    assert torch.all((out[0, 2:].double() - want).abs() <= 1e-4 * size + 1e-7)
    want, _, size = attend(x.q[1, :2], x.k[1][0][:64], x.v[1][0][:64])
    assert torch.all((out[1, :2].double() - want).abs() <= 1e-4 * size + 1e-7)


def test_lengths_beyond_the_table_and_below_zero_are_clamped():
    x = Data((4, 1), 64, "bf16", 16, [64, 64], spare_pages=0)
    want, want_lse = x.run()
    x.cache.lens.copy_(torch.tensor([[2 ** 31 - 1, 65]], dtype=torch.int32))
    out, lse = x.run()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    x.cache.lens.copy_(torch.tensor([[-5, 64]], dtype=torch.int32))
    out, lse = x.run()
    assert torch.all(out[0] == 0) and torch.all(lse[0] == -math.inf) and torch.equal(out[1], want[1])


def test_strided_queries_and_no_lse():
    x = Data((8, 2), 128, "fp16", 16, [200, 300, 10])
    want, _ = x.run()
    fused = torch.zeros(3, 12, 128, dtype=torch.float16, device=DEV)          # [batch][H_q + 2 H_kv][d]
    fused[:, :8] = x.q.to(DEV)
    out = torch.zeros(3, 8, 128, device=DEV)
    pkv.decode_attention_cache(x.cfg, x.cache, 0, fused[:, :8], out, x.ws)
    assert torch.equal(out.cpu(), want)
    out.zero_()
    tokens_first = x.q.to(DEV).transpose(0, 1).contiguous().transpose(0, 1)   # heads far apart
    pkv.decode_attention_cache(x.cfg, x.cache, 0, tokens_first.unsqueeze(2), out, x.ws)
    assert torch.equal(out.cpu(), want)


def test_outputs_need_no_more_than_a_float_s_alignment():
    for lens in ([200, 3], [6000]):                                  # whole heads, and heads that are joined
        x = Data((8, 1), 64, "bf16", 16, lens)
        want, want_lse = x.run()
        flat = torch.full((len(lens) * 8 * 64 + 2,), 5.0, device=DEV)
        out = flat[1:-1].view(len(lens), 8, 64)
        pkv.decode_attention_cache(x.cfg, x.cache, 0, x.q.to(DEV), out, x.ws)
        assert torch.equal(out.cpu(), want) and flat[0] == 5.0 and flat[-1] == 5.0


def test_captured_calls_follow_the_lengths_on_the_device():
    """A graph captured once is replayed as the cache grows; calls of several sizes share the workspace, one after another."""
    x = Data((8, 2), 64, "bf16", 16, [900, 500, 64])
    out, lse = torch.zeros(3, 8, 64, device=DEV), torch.zeros(3, 8, device=DEV)
    q = x.q.to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pkv.decode_attention_cache(x.cfg, x.cache, 0, q, out, x.ws, lse=lse)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkv.decode_attention_cache(x.cfg, x.cache, 0, q, out, x.ws, lse=lse)
    full = (x.k, x.v, x.pos)
    for lens in ([900, 500, 64], [1, 2, 3], [64, 65, 0], [800, 0, 17]):
        x.cache.lens.copy_(torch.tensor([lens], dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        x.k, x.v, x.pos = ([t[:, :n] for t, n in zip(ts, lens)] for ts in full)
        x.check(out.cpu(), lse.cpu())
    pkv.check_status(x.ws)


def test_parts_of_a_cache_join_through_their_logarithms():
    x = Data((4, 1), 128, "bf16", 16, [640])
    whole, whole_lse = x.run()
    parts = []
    for lo, hi in ((0, 320), (320, 640)):
        y = Data((4, 1), 128, "bf16", 16, [320])
        y.q, y.k, y.v = x.q, [x.k[0][:, lo:hi]], [x.v[0][:, lo:hi]]
        y.fill()
        parts.append(y.run())
    lse = torch.logaddexp(parts[0][1], parts[1][1])
    joined = sum(o * torch.exp(l - lse)[..., None] for o, l in parts)
    assert torch.all((joined - whole).abs() <= 3e-4) and torch.all((lse - whole_lse).abs() <= 2e-4)


def test_far_rows_of_a_large_pool():
    """Slots whose elements lie behind 2^31 of the pool."""
    page, d, pages = 64, 128, 2 ** 31 // (64 * 128) + 64
    cfg = pkv.make_config(num_layers=1, num_q_heads=4, num_kv_heads=1, head_dim=d, window=1, pool_kernel=1, dtype="bf16", avg_budget=1)
    k_pool, v_pool = (torch.zeros(pages, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    tables = torch.tensor([pages - 1, 3, pages - 40], dtype=torch.int32, device=DEV).view(1, 1, 1, 3)
    cache = pkv.PagedCache(cfg, k_pool, v_pool, tables, torch.tensor([[150]], dtype=torch.int32, device=DEV))
    ws = pkv.new_cache_workspace(cfg, cache)
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(1, 1, 150, d, generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(1, 4, d, generator=g).to(torch.bfloat16)
    pkv.append_cache(cfg, cache, 0, None, k.to(DEV), v.to(DEV), ws)
    assert torch.equal(k_pool[pages - 40, :22].cpu(), k[0, 0, 128:]) and torch.equal(v_pool[pages - 1].cpu(), v[0, 0, :64])
    out = torch.zeros(1, 4, d, device=DEV)
    pkv.decode_attention_cache(cfg, cache, 0, q.to(DEV), out, ws)
    pkv.check_status(ws)
    want, _, size = attend(q[0], k[0, 0], v[0, 0])
    assert torch.all((out[0].cpu().double() - want).abs() <= 1e-4 * size + 1e-7)


def test_tensors_that_do_not_fit_are_refused():
    x = Data((4, 2), 64, "bf16", 16, [10, 20])
    q, out = x.q.to(DEV), torch.zeros(2, 4, 64, device=DEV)
    good = dict(q=q, out=out, workspace=x.ws)
    for bad in (dict(q=q.half()), dict(q=q[:1]), dict(q=q[..., ::2]), dict(q=q.cpu()), dict(out=out.half()), dict(out=out[:1]), dict(out=out.cpu()),
                dict(lse=out), dict(slopes=out[0, 0], q_positions=x.q_pos.to(DEV)), dict(q_positions=x.q_pos), dict(q_positions=x.q_pos.long().to(DEV)),
                dict(workspace=x.ws.float())):
        with pytest.raises(ValueError):
            kw = {**good, **bad}
            pkv.decode_attention_cache(x.cfg, x.cache, 0, kw.pop("q"), kw.pop("out"), kw.pop("workspace"), **kw)
    for bad in (dict(window=3), dict(prefix=1), dict(slopes=torch.zeros(4, device=DEV)), dict(softcap=-1.0), dict(layer=1), dict(window=-1, q_positions=x.q_pos.to(DEV))):
        with pytest.raises(pkv.PkvError):
            kw = dict(bad)
            pkv.decode_attention_cache(x.cfg, x.cache, kw.pop("layer", 0), q, out, x.ws, **kw)
