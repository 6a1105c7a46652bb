"""The operators of a cache that goes on growing behind a compressed prompt, as measurable cases.

A prompt's layers are compressed into pages (`compress_layer_paged`); every new token is then given its rotary positions
(`rotary`), appended to the pages (`append_cache`) and attends to what they hold (`decode_attention_cache`), and the pages
are dealt out, shared between the branches of a search (`cache_fork`, `cache_reserve`) and moved together (`cache_compact`).

Each operator stands here in its plain form too: elementary torch operations in 32 bits, angles in 64.  A cache is
  k_pool, v_pool  [num_pages][page_size][d]          positions  int32 [num_pages][page_size], a row's position in its text
  tables          int32 [layers][batch][H_kv][max_pages]        lens  int32 [layers][batch], rows a head holds
  refs            int32 [num_pages], how many table entries name a page
and row r of head h of sequence b in layer l lies in page tables[l][b][h][r / page_size] at slot r % page_size.
"""
import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
WORD = {2: torch.int16, 4: torch.int32}
TINY, MHA, GQA4, GQA8, GQA4_64 = (4, 2, 64), (32, 32, 128), (32, 8, 128), (64, 8, 128), (32, 8, 64)

BLANK = {"batch": 1, "dtype": "bf16", "layers": 1, "page": 16, "lens_seed": 1,
         # rotary positions
         "tokens": 1, "layout": "half", "rot_dim": 128, "base": 500000.0, "scaling": "none", "factor": 1.0, "inverse": False,
         "start": 0, "counts_lo": 1,
         # rows of a sequence
         "n_lo": 1, "n_hi": 1,
         # logits
         "softcap": 0.0, "window": 0, "prefix": 0, "slopes": False,
         # pages
         "children": 0, "add": 0, "shared": 0.0, "filled": 0.5}


def _case(name, op, heads, **more):
    """A case dict: heads = (query heads, KV heads, head size)."""
    case = {"name": name, "op": op, "heads_q": heads[0], "heads_kv": heads[1], "dim": heads[2], **BLANK}
    unknown = set(more) - set(BLANK)
    if unknown:
        raise ValueError("unknown fields %s" % sorted(unknown))
    case.update(more)
    case["rot_dim"] = min(case["rot_dim"], heads[2])
    return case


def listed():
    return [
        # queries and keys of a whole prompt, one layer, positions scaled for a long context
        _case("rotary_prompt_32k", "rotary", GQA4, tokens=32768, scaling="llama3", factor=8.0),
        # two prompts of odd length in fp16, interleaved pairs in half of the head, rotated back (as for a gradient)
        _case("rotary_back_partial", "rotary", GQA4_64, dtype="fp16", batch=2, tokens=7001, layout="interleaved", rot_dim=32,
              base=10000.0, scaling="yarn", factor=4.0, start=90000, inverse=True),
        # the smallest call: one token of one sequence of a toy model in fp32
        _case("append_tiny_token", "append", TINY, dtype="fp32", n_lo=65, n_hi=65, base=10000.0, start=512),
        # a serving step takes in pieces of new prompts of different lengths behind what their caches hold
        _case("append_chunks", "append", GQA4, batch=16, tokens=257, counts_lo=1, n_lo=300, n_hi=1500, page=32,
              scaling="llama3", factor=8.0, start=20000),
        # one token of one sequence of a toy model in fp32: latency is all there is
        _case("decode_tiny_fp32", "decode", TINY, dtype="fp32", n_lo=64, n_hi=64),
        # one sequence whose cache was never compressed: the longest context
        _case("decode_one_128k", "decode", GQA8, n_lo=131072, n_hi=131072, page=64),
        # a full batch of compressed caches of different lengths; capped logits, a sliding window behind the first rows
        _case("decode_ragged_capped", "decode", GQA4, batch=64, n_lo=129, n_hi=4096, softcap=30.0, window=12000, prefix=4),
        # eight sequences of a model with a bias on the distance, fp16, head size 64
        _case("decode_distance_bias", "decode", GQA4_64, dtype="fp16", batch=8, n_lo=512, n_hi=2048, page=32, slopes=True),
        # a beam search over eight prompts opens four branches each and makes room for their next token
        _case("fork_beams", "fork", GQA4, layers=32, batch=8, n_lo=100, n_hi=200, children=32, add=1),
        # a serving step makes room for a token of each of 64 sequences
        _case("reserve_step", "fork", GQA4, layers=32, batch=64, n_lo=100, n_hi=200, add=1),
        # a toy model's pool after some sequences have gone, pages of odd size
        _case("compact_tiny", "compact", TINY, dtype="fp32", layers=2, batch=3, n_lo=30, n_hi=90, page=5, filled=0.3),
        # a served model's pool, half of it in use, pages of some sequences shared
        _case("compact_pool", "compact", GQA4, layers=32, batch=32, n_lo=100, n_hi=500, shared=0.5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["rotary", "append", "decode", "decode", "fork", "compact"])
    heads = rng.choice([TINY, MHA, GQA4, GQA4, GQA8, GQA4_64])
    more = {"dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "lens_seed": rng.randrange(1000), "page": rng.choice([1, 5, 16, 16, 32, 64])}
    if op in ("rotary", "append"):
        scaling = rng.choice(["none", "linear", "ntk", "llama3", "yarn"])
        more.update(layout=rng.choice(["half", "interleaved"]), rot_dim=rng.choice([heads[2], heads[2], heads[2] // 2, heads[2] // 4, 20]),
                    base=rng.choice([10000.0, 500000.0]), scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]))
    if op == "rotary":
        more.update(batch=rng.choice([1, 1, 2, 3]), inverse=rng.random() < 0.3, start=rng.choice([0, 77, 120001]))
        more["tokens"] = _log_int(rng, 1, 32768 * 40 * 128 * 2 // ((heads[0] + heads[1]) * heads[2] * 4 * more["batch"]) // 2)
    elif op == "append":
        more.update(batch=_log_int(rng, 1, 16), tokens=rng.choice([1, 1, 1, 4, 33, 257]), n_lo=300, n_hi=rng.choice([301, 900, 1500]),
                    start=rng.choice([0, 20000, 500000]))
        more["counts_lo"] = rng.choice([1, more["tokens"]])
    elif op == "decode":
        more["batch"] = _log_int(rng, 1, 64)
        room = 131072 * 8 * 128 * 2 // (heads[1] * heads[2] * (4 if more["dtype"] == "fp32" else 2)) // 2
        more["n_hi"] = _log_int(rng, 1, min(131072, max(1, room // more["batch"])))
        more["n_lo"] = rng.choice([1, max(1, more["n_hi"] // 3), more["n_hi"]])
        more.update(softcap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.random() < 0.3, window=rng.choice([0, 0, 1, 500, 4096]))
        more["prefix"] = rng.choice([0, 4]) if more["window"] else 0
    elif op == "fork":
        more.update(layers=rng.choice([2, 32]), batch=_log_int(rng, 1, 32), n_lo=rng.choice([1, 40]), n_hi=rng.choice([41, 160, 200]), add=rng.choice([0, 1, 1, 7]))
        more["children"] = rng.choice([0, more["batch"], 32])
        more["page"] = rng.choice([5, 16, 32])
        more["dtype"] = rng.choice(["bf16", "fp16"])
    else:
        more.update(layers=rng.choice([2, 8, 16]), batch=_log_int(rng, 1, 24), n_lo=1, n_hi=rng.choice([41, 160, 400]), shared=rng.choice([0.0, 0.5]),
                    filled=rng.choice([0.2, 0.5, 0.9]), dtype=rng.choice(["bf16", "fp16"]))
        more["page"] = rng.choice([5, 16, 32])
    if op in ("fork", "compact") and heads[1] > 8:
        heads = GQA4
    case = _case("", op, heads, **more)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------ sizes of a case
def _lens(case):
    """Rows that every layer holds of every sequence."""
    r = random.Random(case["lens_seed"])
    return [[r.randint(case["n_lo"], case["n_hi"]) for _ in range(case["batch"])] for _ in range(case["layers"])]


def _counts(case):
    """New tokens of every sequence: the first one has them all."""
    r = random.Random(case["lens_seed"] + 1)
    return [case["tokens"]] + [r.randint(min(case["counts_lo"], case["tokens"]), case["tokens"]) for _ in range(case["batch"] - 1)]


def _parents(case):
    """The sequence that each new sequence goes on from; most have children, one slot stays empty where there are many."""
    r = random.Random(case["lens_seed"] + 2)
    n, batch = case["children"], case["batch"]
    p = [i % batch for i in range(n)]
    if n <= batch:
        p = [r.randrange(batch) for _ in range(n)]
    r.shuffle(p)
    if n >= 8:
        p[r.randrange(n)] = -1
    return p


def _pages(rows, page):
    return -(-rows // page)


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    d, row = case["dim"], case["dim"] * size
    hq, hkv = case["heads_q"], case["heads_kv"]
    if case["op"] == "rotary":
        rows = case["batch"] * case["tokens"] * (hq + hkv)
        return {"bytes": 2 * rows * row + 4 * case["batch"] * case["tokens"], "flops": 3 * rows * case["rot_dim"]}
    if case["op"] == "append":
        new = sum(_counts(case))
        return {"bytes": 2 * new * (hq + 2 * hkv) * row + 4 * new * (1 + hkv) + 8 * case["batch"], "flops": 3 * new * (hq + hkv) * case["rot_dim"]}
    lens = _lens(case)
    if case["op"] == "decode":
        rows, page = 0, case["page"]
        pos = 4 if case["window"] or case["slopes"] else 0
        for n in lens[0]:
            # rows that a window leaves out are not needed; the gaps between positions are 4 on average
            seen = min(n, case["prefix"] + _pages(case["window"], 4)) if case["window"] else n
            rows += hkv * seen * (2 * row + pos) + 4 * hkv * _pages(n, page)
        q = case["batch"] * hq
        return {"bytes": rows + q * row + q * (d + 1) * 4, "flops": 4 * d * (hq // hkv) * hkv * sum(lens[0])}
    page = case["page"]
    if case["op"] == "fork":
        parents = _parents(case) if case["children"] else list(range(case["batch"]))
        entries = copied = taken = 0
        for n in lens:
            seen = set()
            for p in parents:
                if p < 0:
                    continue
                rows = n[p] + case["add"]
                entries += _pages(rows, page)
                taken += _pages(rows, page) - n[p] // page
                if n[p] % page and p in seen:
                    copied += n[p] % page
                elif n[p] % page:
                    taken -= 1
                seen.add(p)
        old = sum(_pages(x, page) for n in lens for x in n)
        moved = hkv * (copied * (2 * row + 4) * 2 + 4 * (old + entries)) + 8 * (hkv * (old + taken))
        return {"bytes": moved + 4 * case["layers"] * (case["batch"] + 2 * len(parents)), "flops": 0}
    used, total = _compact_sizes(case)
    moves = used * (total - used) // total                           # pages in use above the border, dealt out at random
    return {"bytes": moves * page * (2 * row + 4) * 2 + 8 * total + 8 * hkv * sum(_pages(x, page) for n in lens for x in n), "flops": 0}


def _compact_sizes(case):
    """Pages in use and pages of the pool."""
    used = 0
    for n in _lens(case):
        for b, x in enumerate(n):
            pages = _pages(x, case["page"])
            if b % 2 and case["shared"]:
                pages -= min(int(case["shared"] * (x // case["page"])), n[b - 1] // case["page"])
            used += pages * case["heads_kv"]
    return used, max(used + 1, int(used / case["filled"]))


# ------------------------------------------------------------------------------------------------ inputs
def _frequencies(case):
    """Angle of each pair per position, and the factor on the rotated values, in 64 bits."""
    r, base, factor = case["rot_dim"], case["base"], case["factor"]
    i = torch.arange(r // 2, dtype=torch.float64)
    if case["scaling"] == "ntk":
        base = base * factor ** (r / (r - 2))
    f = base ** (-2.0 * i / r)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "llama3":                                  # trained on 8192 positions, factors 1 and 4
        turns = 8192 * f / (2 * math.pi)
        blend = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
        return (1 - blend) * f / factor + blend * f, 1.0
    if case["scaling"] == "yarn":                                    # trained on 4096 positions, 32 turns and 1 turn
        edge = [r * math.log(4096 / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (32.0, 1.0)]
        lo, hi = max(math.floor(edge[0]), 0), min(math.ceil(edge[1]), r - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _randn(g, *shape, dtype):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def _deal(lens, heads, page, room, rng, pool):
    """Tables [layers][batch][H_kv][max_pages] with the pool's pages dealt out in random order, as an allocator in use would
    have them; -1 behind a sequence's last page."""
    need = [[_pages(n, page) for n in row] for row in lens]
    width = max(max(row) for row in need) + _pages(room, page)
    held = torch.tensor(need).view(len(need), -1, 1, 1) > torch.arange(width)
    held = held.expand(len(need), len(need[0]), heads, width)
    tables = torch.full(held.shape, -1, dtype=torch.int32)
    total = int(held.sum())
    order = torch.randperm(pool(total), generator=rng)[:total].to(torch.int32)
    tables[held] = order
    return tables.contiguous().cuda(), pool(total)


def _slots(tables, rows, page):
    """Pool row of each of the rows 0 .. rows - 1 of every head, by a layer's tables; entries of -1 count as page 0."""
    r = torch.arange(rows, device=tables.device)
    entry = tables.long().clamp_min(0).index_select(-1, torch.div(r, page, rounding_mode="floor"))
    return entry * page + r % page


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = torch.Generator()
    rng.manual_seed(seed + 17)
    s = {"case": case, "op": case["op"]}
    {"rotary": _prepare_rotary, "append": _prepare_append, "decode": _prepare_decode, "fork": _prepare_fork, "compact": _prepare_compact}[case["op"]](case, s, g, rng)
    if own:
        _prepare_own(case, s)
    return s


def _prepare_rotary(case, s, g, rng):
    dtype = TYPES[case["dtype"]]
    batch, tokens, d = case["batch"], case["tokens"], case["dim"]
    s["q"] = _randn(g, batch, case["heads_q"], tokens, d, dtype=dtype)
    s["k"] = _randn(g, batch, case["heads_kv"], tokens, d, dtype=dtype)
    s["q_out"], s["k_out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
    first = case["start"] + torch.randint(0, 1000, (batch, 1), generator=rng)
    s["positions"] = (first + torch.arange(tokens)).to(torch.int32).cuda()
    f, s["magnitude"] = _frequencies(case)
    s["frequencies"] = f.cuda()


def _prepare_append(case, s, g, rng):
    _prepare_rotary(case, s, g, rng)
    dtype = TYPES[case["dtype"]]
    heads, page, d = case["heads_kv"], case["page"], case["dim"]
    counts, lens = _counts(case), _lens(case)[0]
    s["v"] = _randn(g, case["batch"], heads, case["tokens"], d, dtype=dtype)
    s["counts"] = torch.tensor(counts, dtype=torch.int32).cuda()
    s["tables"], pages = _deal([lens], heads, page, 0, rng, lambda n: n + 7)
    s["lens"] = torch.tensor([lens], dtype=torch.int32).cuda()
    s["k_pool"], s["v_pool"] = (_randn(g, pages, page, d, dtype=dtype) for _ in range(2))
    s["pos_pool"] = torch.zeros(pages, page, dtype=torch.int32, device="cuda")


def _prepare_decode(case, s, g, rng):
    dtype = TYPES[case["dtype"]]
    heads, page, d, batch = case["heads_kv"], case["page"], case["dim"], case["batch"]
    lens = _lens(case)[0]
    s["tables"], pages = _deal([lens], heads, page, 1, rng, lambda n: n + 7)
    s["lens"] = torch.tensor([lens], dtype=torch.int32).cuda()
    s["k_pool"], s["v_pool"] = (_randn(g, pages, page, d, dtype=dtype) for _ in range(2))
    s["pos_pool"] = torch.zeros(pages, page, dtype=torch.int32, device="cuda")
    # queries lean towards a direction that the first rows of a sequence's heads share
    toward = torch.nn.functional.normalize(torch.randn(d, generator=g, device="cuda"), dim=0)
    s["q"] = (torch.randn(batch, case["heads_q"], d, generator=g, device="cuda") + 2.0 * toward).to(dtype)
    first = s["tables"][0, :, :, 0].long().flatten()
    s["k_pool"][first, 0] += (math.sqrt(d) * toward).to(dtype)
    # the first rows are a text's first ones; positions of the others rise by 4 on average and end at the query's own
    rows = max(lens)
    gaps = torch.randint(1, 8, (batch, heads, rows), generator=g, device="cuda").cumsum(-1)
    n = s["lens"][0].long().view(-1, 1, 1)
    s["q_pos"] = (8 * s["lens"][0] + 100).to(torch.int32)
    pos = s["q_pos"].long().view(-1, 1, 1) - (gaps.gather(-1, (n - 1).expand(batch, heads, 1)) - gaps)
    r = torch.arange(rows, device="cuda")
    pos = torch.where(r < torch.div(n, 2, rounding_mode="floor").clamp_max(4), r, pos)
    live = (r < n).expand_as(pos)
    s["pos_pool"].view(-1)[_slots(s["tables"][0], rows, page)[live]] = pos[live].to(torch.int32)
    s["rows"] = rows
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, case["heads_q"] + 1, device="cuda") / case["heads_q"]) if case["slopes"] else None
    s["out"] = torch.zeros(batch, case["heads_q"], d, device="cuda")
    s["lse"] = torch.zeros(batch, case["heads_q"], device="cuda")


def _count_refs(tables, lens, page, pages):
    held = torch.arange(tables.shape[-1], device="cuda") < ((lens.long() + page - 1) // page)[:, :, None, None]
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    named = tables[held.expand_as(tables)].long()
    return refs.scatter_add_(0, named, torch.ones_like(named, dtype=torch.int32))


def _prepare_fork(case, s, g, rng):
    dtype = TYPES[case["dtype"]]
    heads, page, d, layers = case["heads_kv"], case["page"], case["dim"], case["layers"]
    lens, parents = _lens(case), _parents(case) if case["children"] else list(range(case["batch"]))
    # each new sequence may need the pages of a whole one's last rows, of the copied page and of the added rows
    spare = layers * heads * len(parents) * (1 + _pages(case["add"], page))
    s["tables"], pages = _deal(lens, heads, page, case["add"] + 1, rng, lambda n: n + spare + 7)
    s["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    s["refs"] = _count_refs(s["tables"], s["lens"], page, pages)
    s["k_pool"], s["v_pool"] = (_randn(g, pages, page, d, dtype=dtype) for _ in range(2))
    s["pos_pool"] = torch.randint(0, 100000, (pages, page), generator=g, device="cuda", dtype=torch.int32)
    s["parents"] = torch.tensor(parents, dtype=torch.int32).cuda() if case["children"] else None
    s["add"] = torch.full((layers, len(parents)), case["add"], dtype=torch.int32, device="cuda")
    s["to_tables"] = torch.full((layers, len(parents), heads, s["tables"].shape[-1]), -1, dtype=torch.int32, device="cuda")
    s["to_lens"] = torch.zeros(layers, len(parents), dtype=torch.int32, device="cuda")
    s["to_refs"] = torch.zeros_like(s["refs"])
    s["granted"] = torch.zeros(layers, len(parents), dtype=torch.int32, device="cuda")


def _prepare_compact(case, s, g, rng):
    dtype = TYPES[case["dtype"]]
    heads, page, d = case["heads_kv"], case["page"], case["dim"]
    lens = _lens(case)
    pages = _compact_sizes(case)[1]
    s["tables"], most = _deal(lens, heads, page, 1, rng, lambda n: n)
    s["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    t = s["tables"]
    if case["shared"] and case["batch"] > 1:                         # every second sequence shares full pages with the one ahead
        full = torch.div(s["lens"], page, rounding_mode="floor")
        odd = t[:, 1::2]
        even = t[:, 0:2 * odd.shape[1]:2]
        both = torch.minimum((case["shared"] * full[:, 1::2]).int(), full[:, 0:2 * odd.shape[1]:2])
        t[:, 1::2] = torch.where(torch.arange(t.shape[-1], device="cuda") < both[:, :, None, None], even, odd)
    # the pages named are spread over the whole pool
    named = torch.unique(t[t >= 0]).long()
    spread = torch.full((most,), -1, dtype=torch.int32, device="cuda")
    spread[named] = torch.randperm(pages, generator=rng)[:named.numel()].to(torch.int32).cuda()
    s["tables"] = torch.where(t >= 0, spread[t.long().clamp_min(0)], t)
    s["refs"] = _count_refs(s["tables"], s["lens"], page, pages)
    s["k_pool"], s["v_pool"] = (_randn(g, pages, page, d, dtype=dtype) for _ in range(2))
    s["pos_pool"] = torch.randint(0, 100000, (pages, page), generator=g, device="cuda", dtype=torch.int32)
    s["to_tables"] = torch.full_like(s["tables"], -1)
    s["to_lens"], s["to_refs"] = torch.zeros_like(s["lens"]), torch.zeros_like(s["refs"])
    s["used"] = torch.zeros(1, dtype=torch.int32, device="cuda")


def _prepare_own(case, s):
    """What a program keeps between calls: the configuration, the rotary plan, the cache's handle and a workspace."""
    import paper_2406_02069_b200 as pkv
    cfg = s["cfg"] = pkv.make_config(num_layers=case["layers"], num_q_heads=case["heads_q"], num_kv_heads=case["heads_kv"],
                                     head_dim=case["dim"], window=8, pool_kernel=5, dtype=case["dtype"], avg_budget=64)
    s["pkv"] = pkv
    if case["op"] in ("rotary", "append"):
        s["rotary"] = pkv.make_rotary(case["rot_dim"], layout=case["layout"], base=case["base"], scaling=case["scaling"], factor=case["factor"],
                                      original_positions={"llama3": 8192, "yarn": 4096}.get(case["scaling"], 0))
    if case["op"] != "rotary":
        s["cache"] = pkv.PagedCache(cfg, s["k_pool"], s["v_pool"], s["tables"], s["lens"], positions=s["pos_pool"], refs=s.get("refs"))
        s["to"] = pkv.PagedCache(cfg, s["k_pool"], s["v_pool"], s["to_tables"], s["to_lens"], positions=s["pos_pool"],
                                 refs=s["to_refs"]) if "to_tables" in s else None
        s["workspace"] = pkv.new_cache_workspace(cfg, *[c for c in (s["cache"], s["to"]) if c is not None])


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return (_own if own else _plain)[s["op"]](s)


def _own_rotary(s):
    s["pkv"].rotary(s["cfg"], s["rotary"], s["positions"], s["q"], s["k"], s["q_out"], s["k_out"], inverse=s["case"]["inverse"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_append(s):
    s["pkv"].append_cache(s["cfg"], s["cache"], 0, s["positions"], s["k"], s["v"], s["workspace"], q=s["q"], q_out=s["q_out"],
                          rotary=s["rotary"], counts=s["counts"])
    return _appended(s)


def _own_decode(s):
    case = s["case"]
    by_distance = case["slopes"] or case["window"] > 0               # otherwise positions play no part
    s["pkv"].decode_attention_cache(s["cfg"], s["cache"], 0, s["q"], s["out"], s["workspace"], lse=s["lse"], softcap=case["softcap"],
                                    q_positions=s["q_pos"] if by_distance else None, slopes=s["slopes"], window=case["window"],
                                    prefix=case["prefix"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_fork(s):
    if s["parents"] is None:
        s["pkv"].cache_reserve(s["cfg"], s["cache"], s["add"], s["workspace"], granted=s["granted"], to=s["to"])
    else:
        s["pkv"].cache_fork(s["cfg"], s["cache"], s["parents"], s["workspace"], add=s["add"], granted=s["granted"], to=s["to"])
    return _bookkeeping(s, s["granted"])


def _own_compact(s):
    s["pkv"].cache_compact(s["cfg"], s["cache"], s["workspace"], used=s["used"], to=s["to"])
    return _bookkeeping(s, s["used"])


def _appended(s):
    return {"k_pool": s["k_pool"], "v_pool": _bits(s["v_pool"]), "positions": s["pos_pool"], "q": s["q_out"]}


def _bookkeeping(s, more):
    return {"tables": s["to_tables"], "lens": s["to_lens"], "refs": s["to_refs"], "more": more, "k_pool": _bits(s["k_pool"]),
            "v_pool": _bits(s["v_pool"]), "positions": s["pos_pool"]}


def _bits(t):
    return t.view(WORD[t.element_size()])


def _rotate(s, x):
    """x [batch][heads][tokens][d] rotated pair by pair in 32 bits, its angles formed in 64."""
    case = s["case"]
    r = case["rot_dim"]
    angle = s["positions"].double()[:, None, :, None] * s["frequencies"]
    cos = (angle.cos() * s["magnitude"]).float()
    sin = (angle.sin() * s["magnitude"]).float() * (-1.0 if case["inverse"] else 1.0)
    f = x.float()
    if case["layout"] == "half":
        a, b = f[..., :r // 2], f[..., r // 2:r]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, f[..., r:]], -1).to(x.dtype)
    a, b = f[..., 0:r:2], f[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), f[..., r:]], -1).to(x.dtype)


def _plain_rotary(s):
    s["q_out"].copy_(_rotate(s, s["q"]))
    s["k_out"].copy_(_rotate(s, s["k"]))
    return {"q": s["q_out"], "k": s["k_out"]}


def _plain_append(s):
    case = s["case"]
    batch, heads, tokens, page = case["batch"], case["heads_kv"], case["tokens"], case["page"]
    t = torch.arange(tokens, device="cuda")
    real = t < s["counts"][:, None]                                                          # [batch][tokens]
    row = (s["lens"][0] - s["counts"])[:, None] + t
    row = torch.where(real, row, 0).long()[:, None, :].expand(batch, heads, tokens)
    entry = s["tables"][0].long().gather(-1, torch.div(row, page, rounding_mode="floor"))
    slot = (entry * page + row % page).flatten()
    real_kv = real[:, None, :].expand(batch, heads, tokens).flatten()
    # tokens behind a sequence's count write what the first one (always there) writes
    pick = torch.where(real_kv, torch.arange(slot.numel(), device="cuda"), 0)
    d = case["dim"]
    s["k_pool"].view(-1, d)[slot[pick]] = _rotate(s, s["k"]).reshape(-1, d)[pick]
    s["v_pool"].view(-1, d)[slot[pick]] = s["v"].reshape(-1, d)[pick]
    s["pos_pool"].view(-1)[slot[pick]] = s["positions"][:, None, :].expand(batch, heads, tokens).flatten()[pick]
    s["q_out"].copy_(torch.where(real[:, None, :, None], _rotate(s, s["q"]), s["q_out"]))
    return _appended(s)


def _plain_decode(s):
    case = s["case"]
    batch, heads, d = case["batch"], case["heads_kv"], case["dim"]
    slot = _slots(s["tables"][0], s["rows"], case["page"])                                   # [batch][H_kv][rows]
    seen = torch.arange(s["rows"], device="cuda") < s["lens"][0][:, None, None]
    q = s["q"].float().view(batch, heads, -1, d)
    x = q @ s["k_pool"].view(-1, d)[slot].float().transpose(-1, -2) / math.sqrt(d)           # [batch][H_kv][group][rows]
    if case["softcap"]:
        x = case["softcap"] * torch.tanh(x / case["softcap"])
    far = s["q_pos"][:, None, None] - s["pos_pool"].view(-1)[slot]
    seen = seen & (far >= 0)
    if case["window"]:
        seen = seen & ((far < case["window"]) | (s["pos_pool"].view(-1)[slot] < case["prefix"]))
    if case["slopes"]:
        x = x - s["slopes"].view(heads, -1, 1) * far[:, :, None].float()
    x = x.masked_fill(~seen[:, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    z = e.sum(-1, keepdim=True)
    o = e @ s["v_pool"].view(-1, d)[slot].float() / torch.where(z == 0, 1.0, z)
    s["out"].copy_(o.view(batch, -1, d))
    s["lse"].copy_((m + torch.log(z)).view(batch, -1))
    return {"out": s["out"], "lse": s["lse"]}


def _plain_fork(s):
    case = s["case"]
    page, width = case["page"], s["tables"].shape[-1]
    parents = s["parents"] if s["parents"] is not None else torch.arange(case["batch"], device="cuda", dtype=torch.int32)
    named, goes_on = parents.clamp_min(0).long(), parents >= 0
    n = torch.where(goes_on, s["lens"][:, named], 0)                                         # [layers][children]
    full, part = torch.div(n, page, rounding_mode="floor"), n % page
    again = torch.tril(parents[:, None] == parents[None, :], -1).any(-1)                     # not its parent's first child
    keeps = full + ((part > 0) & ~again)                                                     # pages it shares or takes over
    add = s["add"].clamp_min(0)
    pages = torch.div(n + add + page - 1, page, rounding_mode="floor")
    j = torch.arange(width, device="cuda")
    old = s["tables"][:, named]
    kept = (j < keeps[:, :, None, None]).expand_as(old)
    fresh = ((j < pages[:, :, None, None]) & ~kept).expand_as(old)
    # a page is named once more for every child that keeps it and once less for every sequence that had it
    had = (j < torch.div(s["lens"] + page - 1, page, rounding_mode="floor")[:, :, None, None]).expand_as(s["tables"])
    refs = s["refs"].long()
    refs = refs.scatter_add(0, old.long().clamp_min(0).flatten(), kept.long().flatten())
    refs = refs.scatter_add(0, s["tables"].long().clamp_min(0).flatten(), -had.long().flatten())
    free = torch.argsort((refs > 0).byte(), stable=True)                                     # the free pages first, ascending
    rank = (fresh.flatten().long().cumsum(0) - 1).clamp_min(0).view(old.shape)
    new = free[rank]
    s["to_refs"].copy_(refs.scatter_add(0, torch.where(fresh, new, 0).flatten(), fresh.long().flatten()))
    tables = torch.where(kept, old, torch.where(fresh, new.int(), s["to_tables"]))
    s["to_tables"].copy_(tables)
    s["to_lens"].copy_(n + add)
    s["granted"].copy_(add)
    # rows of a page that is not full: children behind the first have them copied into pages of their own
    moves = ((part > 0) & again)[:, :, None].expand(old.shape[:3])
    at = full[:, :, None, None].long().clamp_max(width - 1).expand(*old.shape[:3], 1)
    rows = torch.arange(page, device="cuda")
    src = (old.gather(-1, at).long().clamp_min(0) * page + rows).flatten()
    dst = (tables.gather(-1, at).long().clamp_min(0) * page + rows).flatten()
    real = (moves[..., None] & (rows < part[:, :, None, None])).flatten()
    stays = torch.argmax(real.byte())
    any_moves = real.any()
    pick = torch.where(real, torch.arange(real.numel(), device="cuda"), stays)
    src, dst = src[pick], dst[pick]
    dst = torch.where(any_moves, dst, src)
    _move_rows(s, src, dst)
    return _bookkeeping(s, s["granted"])


def _move_rows(s, src, dst):
    d = s["case"]["dim"]
    k, v, p = s["k_pool"].view(-1, d), s["v_pool"].view(-1, d), s["pos_pool"].view(-1)
    k[dst], v[dst], p[dst] = k[src], v[src], p[src]


def _plain_compact(s):
    case = s["case"]
    page, refs = case["page"], s["refs"]
    pages = refs.numel()
    ids = torch.arange(pages, device="cuda")
    used = refs > 0
    border = used.sum()
    hole, mover = ~used & (ids < border), used & (ids >= border)
    n = mover.sum()
    most = (pages + 1) // 2                                                                  # there cannot be more pairs
    real = ids[:most] < n
    src, dst = (torch.argsort((~w).byte(), stable=True)[:most] for w in (mover, hole))
    src = torch.where(real, src, torch.where(n > 0, src[0], 0))                              # no pair: the first one once more
    dst = torch.where(real, dst, torch.where(n > 0, dst[0], 0))
    moved = ids.scatter(0, src, dst)
    held = torch.arange(s["tables"].shape[-1], device="cuda") < torch.div(s["lens"] + page - 1, page, rounding_mode="floor")[:, :, None, None]
    s["to_tables"].copy_(torch.where(held, moved[s["tables"].long().clamp_min(0)].int(), s["to_tables"]))
    s["to_lens"].copy_(s["lens"])
    s["to_refs"].copy_(refs.scatter(0, src, 0).scatter(0, dst, refs[src]))
    s["used"].copy_(border.view(1))
    _move_pages(s, src, dst)
    return _bookkeeping(s, s["used"])


def _move_pages(s, src, dst):
    s["k_pool"][dst], s["v_pool"][dst], s["pos_pool"][dst] = s["k_pool"][src], s["v_pool"][src], s["pos_pool"][src]


_own = {"rotary": _own_rotary, "append": _own_append, "decode": _own_decode, "fork": _own_fork, "compact": _own_compact}
_plain = {"rotary": _plain_rotary, "append": _plain_append, "decode": _plain_decode, "fork": _plain_fork, "compact": _plain_compact}


# ------------------------------------------------------------------------------------------------ the same in 64 bits
def _exact_frequency(case, i):
    r, base, factor, kind = case["rot_dim"], case["base"], case["factor"], case["scaling"]
    if kind == "ntk":
        return math.pow(base * math.pow(factor, r / (r - 2)), -2 * i / r)
    f = math.pow(base, -2 * i / r)
    if kind == "linear":
        return f / factor
    if kind == "llama3":
        wave = 2 * math.pi / f
        if wave < 8192 / 4:
            return f
        if wave > 8192:
            return f / factor
        smooth = (8192 / wave - 1) / (4 - 1)
        return (1 - smooth) * f / factor + smooth * f
    if kind == "yarn":
        def pair_of(turns):
            return r * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair_of(32)), 0), min(math.ceil(pair_of(1)), r - 1)
        scaled = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
        return f * (1 - scaled) + f / factor * scaled
    return f


def _exact_rotation(case, positions, x):
    """x [heads][tokens][d] of one sequence: each pair as a complex number, turned by its angle."""
    r = case["rot_dim"]
    f = torch.tensor([_exact_frequency(case, i) for i in range(r // 2)], dtype=torch.float64, device=x.device)
    angle = positions.double()[:, None] * f * (-1 if case["inverse"] else 1)
    size = 0.1 * math.log(case["factor"]) + 1 if case["scaling"] == "yarn" else 1.0
    turn = torch.polar(torch.full_like(angle, size), angle)
    y = x.double().clone()
    first, second = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    if case["op"] in ("fork", "compact"):
        return None                                                  # whole numbers and copied bits
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return {x: torch.stack([_exact_rotation(case, s["positions"][b], s[x][b]) for b in range(case["batch"])]) for x in ("q", "k")}
    if case["op"] == "append":
        k_pool, q = s["k_pool"].double(), s["q_out"].double()
        lens, counts, page = _lens(case)[0], _counts(case), case["page"]
        tables = s["tables"][0].tolist()
        for b in range(case["batch"]):
            k_new = _exact_rotation(case, s["positions"][b], s["k"][b])
            q[b, :, :counts[b]] = _exact_rotation(case, s["positions"][b], s["q"][b])[:, :counts[b]]
            rows = range(lens[b] - counts[b], lens[b])
            for h in range(case["heads_kv"]):
                slots = torch.tensor([tables[b][h][r // page] * page + r % page for r in rows], device="cuda")
                k_pool.view(-1, case["dim"])[slots] = k_new[h, :counts[b]]
        return {"k_pool": k_pool, "v_pool": None, "positions": None, "q": q}
    group, page, d = case["heads_q"] // case["heads_kv"], case["page"], case["dim"]
    out, lse = s["out"].double(), s["lse"].double()
    k_rows, v_rows, at = s["k_pool"].view(-1, d), s["v_pool"].view(-1, d), s["pos_pool"].view(-1)
    for b, n in enumerate(_lens(case)[0]):
        r = torch.arange(n, device="cuda")
        for h in range(case["heads_kv"]):
            slots = s["tables"][0, b, h].long()[r // page] * page + r % page
            q = s["q"][b, h * group:(h + 1) * group].double()
            logit = k_rows[slots].double() @ q.T / math.sqrt(d)                              # [n][group]
            if case["softcap"]:
                logit = case["softcap"] * torch.tanh(logit / case["softcap"])
            apart = (s["q_pos"][b] - at[slots]).double()
            if case["slopes"]:
                logit = logit - apart[:, None] * s["slopes"][h * group:(h + 1) * group].double()
            keep = apart >= 0
            if case["window"]:
                keep = keep & ((apart < case["window"]) | (at[slots] < case["prefix"]))
            logit, v = logit[keep], v_rows[slots[keep]].double()
            lse[b, h * group:(h + 1) * group] = torch.logsumexp(logit, 0)
            out[b, h * group:(h + 1) * group] = torch.softmax(logit, 0).T @ v
    return {"out": out, "lse": lse}
