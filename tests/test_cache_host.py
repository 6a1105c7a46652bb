"""Growing cache: what the C boundary decides on the host.  Plans of rotary positions, workspace sizes, refused arguments (a
refused call enqueues nothing, so these need no GPU; the pointers are never followed)."""
import ctypes
import math

import pytest

import paper_2406_02069_b200 as pkv
from paper_2406_02069_b200 import binding, cache as cache_mod
import cache_oracle

INVALID, UNSUPPORTED, WORKSPACE = binding.PKV_ERR_INVALID_ARG, binding.PKV_ERR_UNSUPPORTED, binding.PKV_ERR_WORKSPACE
P = 1 << 20                                                          # an aligned address that nothing reads


@pytest.mark.parametrize("dim", [2, 20, 64, 128])
@pytest.mark.parametrize("scaling,kw", [("none", {}), ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0)),
                                        ("llama3", dict(factor=8.0, original=8192)), ("llama3", dict(factor=8.0, original=100, low=0.5, high=3.0)),
                                        ("yarn", dict(factor=4.0, original=4096, high=32.0)), ("yarn", dict(factor=2.0, original=64, low=2.0, high=2.5))])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_plans_follow_the_definitions(dim, scaling, kw, base):
    if scaling == "ntk" and dim == 2:
        with pytest.raises(pkv.PkvError):
            pkv.make_rotary(dim, base=base, scaling=scaling, factor=8.0)
        return
    plan = pkv.make_rotary(dim, base=base, scaling=scaling, factor=kw.get("factor", 1.0), original_positions=kw.get("original", 0),
                           low=kw.get("low"), high=kw.get("high"))
    want, magnitude = cache_oracle.frequencies(dim, base, scaling, **{"high": 4.0, **kw})
    assert plan.rotary_dim == dim and plan.layout == 0
    assert math.isclose(plan.magnitude, magnitude, rel_tol=1e-14)
    for i, f in enumerate(want):
        assert math.isclose(plan.frequency[i], f, rel_tol=1e-12), i
    assert all(plan.frequency[i] == 0.0 for i in range(dim // 2, 64))


@pytest.mark.parametrize("dim,kw", [(0, {}), (3, {}), (130, {}), (-2, {}), (64, dict(base=1.0)), (64, dict(base=math.nan)), (64, dict(base=math.inf)),
                                    (64, dict(scaling="linear", factor=0.5)), (64, dict(scaling="linear", factor=math.inf)),
                                    (64, dict(scaling="llama3", factor=2.0)), (64, dict(scaling="llama3", factor=2.0, original_positions=100, low=4.0, high=1.0)),
                                    (64, dict(scaling="yarn", factor=2.0, original_positions=100, low=0.0)),
                                    (64, dict(scaling="yarn", factor=2.0, original_positions=100, high=math.inf))])
def test_plans_that_make_no_sense_are_refused(dim, kw):
    with pytest.raises(pkv.PkvError) as e:
        pkv.make_rotary(dim, **kw)
    assert e.value.status == INVALID


def test_plan_names():
    with pytest.raises(ValueError):
        pkv.make_rotary(64, layout="quarter")
    with pytest.raises(ValueError):
        pkv.make_rotary(64, scaling="dynamic")


def config(**kw):
    return pkv.make_config(**{**dict(num_layers=2, num_q_heads=8, num_kv_heads=2, head_dim=64, window=4, pool_kernel=5, dtype="bf16", avg_budget=16), **kw})


def cache(**kw):
    return cache_mod.PkvCache(**{**dict(k_pool=P, v_pool=P, positions=P, tables=P, lens=P, refs=P, num_pages=10, page_size=4, layers=2, batch=3, max_pages=5), **kw})


def tensor(ptr=P, sb=4096, sh=1024, st=64):
    return binding.PkvTensor(ptr, sb, sh, st)


NONE = binding.PkvTensor(None, 0, 0, 0)
BIG = 1 << 40


def call(name, *args):
    return getattr(binding._lib, name)(*args)


def append(cfg=None, c=None, layer=0, plan=True, positions=P, tokens=1, q=None, q_out=None, k=None, v=None, counts=None, ws=P, size=BIG):
    cfg, c = cfg or config(), c or cache()
    p = pkv.make_rotary(64) if plan is True else plan
    return call("pyramidkv_append_cache", ctypes.byref(cfg), ctypes.byref(c), layer, ctypes.byref(p) if p is not None else None, positions, 1, tokens,
                q or NONE, q_out or NONE, k or tensor(), v or tensor(), counts, ws, size, None)


def attend(cfg=None, c=None, layer=0, q=None, out=P, lse=None, ws=P, size=BIG, **options):
    cfg, c = cfg or config(), c or cache()
    o = cache_mod.PkvAttendOptions(**options)
    return call("pyramidkv_decode_attention_cache", ctypes.byref(cfg), ctypes.byref(c), layer, ctypes.byref(o), q or tensor(), out, lse, ws, size, None)


def rotary(cfg=None, plan=None, positions=P, batch=1, tokens=1, q=None, q_out=None, k=None, k_out=None):
    cfg, plan = cfg or config(), plan or pkv.make_rotary(64)
    return call("pyramidkv_rotary", ctypes.byref(cfg), ctypes.byref(plan), positions, 1, batch, tokens, q or NONE, q_out or NONE, k or NONE, k_out or NONE, 0, None)


def fork(c=None, to=None, parents=P, add=None, ws=P, size=BIG):
    c = c or cache()
    return call("pyramidkv_cache_fork", ctypes.byref(config()), ctypes.byref(c), ctypes.byref(to or c), parents, add, 0, None, ws, size, None)


def reserve(c=None, to=None, add=P, ws=P, size=BIG):
    c = c or cache()
    return call("pyramidkv_cache_reserve", ctypes.byref(config()), ctypes.byref(c), ctypes.byref(to or c), add, 0, None, ws, size, None)


def compact(c=None, to=None, used=None, ws=P, size=BIG):
    c = c or cache()
    return call("pyramidkv_cache_compact", ctypes.byref(config()), ctypes.byref(c), ctypes.byref(to or c), used, ws, size, None)


BAD_CACHES = [(dict(k_pool=None), INVALID), (dict(v_pool=P + 8), INVALID), (dict(tables=None), INVALID), (dict(lens=P + 2), INVALID),
              (dict(positions=P + 1), INVALID), (dict(refs=P + 3), INVALID), (dict(num_pages=0), INVALID), (dict(page_size=0), INVALID),
              (dict(layers=0), INVALID), (dict(batch=0), INVALID), (dict(max_pages=-1), INVALID), (dict(batch=1025), UNSUPPORTED),
              (dict(layers=65536), UNSUPPORTED), (dict(num_pages=(1 << 27) + 1), UNSUPPORTED), (dict(num_pages=1 << 27, page_size=16), UNSUPPORTED), (dict(max_pages=1 << 20, page_size=1025), UNSUPPORTED),
              (dict(max_pages=1 << 30, page_size=1, batch=512), UNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD_CACHES, ids=lambda x: "_".join(x) if isinstance(x, dict) else str(x))
def test_caches_that_make_no_sense_are_refused_by_every_call(bad, status):
    c = cache(**bad)
    assert append(c=c) == status and attend(c=c) == status and fork(c=c) == status and reserve(c=c) == status and compact(c=c) == status
    assert call("pyramidkv_cache_workspace_bytes", ctypes.byref(config()), ctypes.byref(c)) == 0


def test_configurations_are_checked_first():
    for bad, status in ((config(num_q_heads=7), INVALID), (config(head_dim=96), UNSUPPORTED), (config(window=0), INVALID)):
        assert append(cfg=bad) == status and attend(cfg=bad) == status
        assert rotary(cfg=bad, k=tensor(), k_out=tensor()) == status
    wide = config(num_q_heads=65536, num_kv_heads=1)
    assert append(cfg=wide) == UNSUPPORTED and attend(cfg=wide) == UNSUPPORTED and rotary(cfg=wide, k=tensor(), k_out=tensor()) == UNSUPPORTED
    many = config(num_q_heads=1024, num_kv_heads=256)
    assert attend(cfg=many, c=cache(batch=257)) == UNSUPPORTED              # more blocks of query heads than counters


def test_workspaces_are_checked():
    need = call("pyramidkv_cache_workspace_bytes", ctypes.byref(config()), ctypes.byref(cache()))
    assert need > 0
    for f in (append, attend, fork, reserve, compact):
        assert f(ws=None) == WORKSPACE and f(ws=P + 128) == WORKSPACE and f(size=need - 1) == WORKSPACE
    bigger = cache(batch=900, tables=P + 4096, lens=P + 4096, refs=P + 4096)
    assert fork(to=bigger, size=need) == WORKSPACE                          # the larger side's size is needed
    for more in (dict(num_pages=100), dict(batch=30), dict(layers=9), dict(max_pages=400)):
        assert call("pyramidkv_cache_workspace_bytes", ctypes.byref(config()), ctypes.byref(cache(**more))) >= need


@pytest.mark.parametrize("kw", [dict(layer=-1), dict(layer=2), dict(tokens=0), dict(tokens=-1), dict(tokens=1 << 30), dict(positions=None),
                                dict(positions=None, plan=None), dict(positions=P + 2), dict(counts=P + 1), dict(q=tensor()), dict(q_out=tensor()),
                                dict(k=tensor(ptr=P + 8)), dict(v=NONE), dict(k=tensor(st=60)), dict(k=tensor(st=68)), dict(v=tensor(sh=1028)),
                                dict(k=tensor(sb=0)), dict(v=tensor(sh=-64)), dict(q=tensor(), q_out=tensor(sb=-4096))],
                         ids=lambda kw: "_".join(kw))
def test_appends_that_make_no_sense_are_refused(kw):
    assert append(**kw) == INVALID


def test_plans_are_checked_by_the_calls():
    wide, odd, nan, layout, mag = (pkv.make_rotary(64) for _ in range(5))
    wide.rotary_dim, odd.rotary_dim, nan.frequency[31], layout.layout, mag.magnitude = 128, 33, math.nan, 2, math.inf
    for plan in (wide, odd, nan, layout, mag):
        assert append(plan=plan) == INVALID
        assert rotary(plan=plan, k=tensor(), k_out=tensor()) == INVALID


@pytest.mark.parametrize("kw", [dict(), dict(q=tensor()), dict(k_out=tensor()), dict(k=tensor(), k_out=tensor(), positions=None),
                                dict(k=tensor(), k_out=tensor(), batch=0), dict(k=tensor(), k_out=tensor(), tokens=0),
                                dict(k=tensor(), k_out=tensor(), batch=1 << 16, tokens=1 << 16), dict(k=tensor(ptr=P + 4), k_out=tensor()),
                                dict(k=tensor(), k_out=tensor(st=32)), dict(k=tensor(), k_out=tensor(sb=0), batch=2)], ids=lambda kw: "_".join(kw) or "nothing")
def test_rotations_that_make_no_sense_are_refused(kw):
    assert rotary(**kw) == INVALID


@pytest.mark.parametrize("kw", [dict(layer=2), dict(out=None), dict(out=P + 2), dict(lse=P + 1), dict(q=NONE), dict(q=tensor(ptr=P + 2)),
                                dict(q=tensor(sh=68)), dict(scale=math.nan), dict(softcap=-1.0), dict(softcap=math.inf), dict(softcap=1e-40), dict(window=-1, q_positions=P),
                                dict(window=5), dict(prefix=1), dict(slopes=P), dict(slopes=P + 1, q_positions=P), dict(q_positions=P + 2),
                                dict(q_positions=P, c=cache(positions=None))], ids=lambda kw: "_".join(kw))
def test_attention_that_makes_no_sense_is_refused(kw):
    assert attend(**kw) == INVALID


def test_page_calls_that_make_no_sense_are_refused():
    other = dict(tables=P + 4096, lens=P + 4096, refs=P + 4096)
    assert fork(c=cache(refs=None)) == INVALID and reserve(c=cache(refs=None)) == INVALID and compact(c=cache(refs=None)) == INVALID
    assert fork(parents=None) == INVALID and fork(parents=P + 2) == INVALID and fork(add=P + 1) == INVALID
    assert reserve(add=None) == INVALID and compact(used=P + 2) == INVALID
    for bad in (dict(k_pool=P + 4096), dict(v_pool=P + 4096), dict(positions=None), dict(num_pages=11), dict(page_size=5), dict(layers=1), dict(max_pages=6)):
        for f in (fork, reserve, compact):
            assert f(to=cache(**{**other, **bad})) == INVALID               # not the same pools
    for part in ("tables", "lens", "refs"):                                  # neither in place nor all of its own
        for f in (fork, reserve, compact):
            assert f(to=cache(**{part: P + 4096})) == INVALID
    assert reserve(to=cache(**other, batch=4)) == INVALID and compact(to=cache(**other, batch=4)) == INVALID
    assert fork(to=cache(batch=4)) == INVALID                                # in place with another batch


def test_position_lists_that_make_no_sense_are_refused():
    lens = (ctypes.c_int32 * 2)(40, 9)

    def call_positions(cfg=None, indices=P, batch=2, k_layer=3, table=P, page=4, pages=10, positions=P, ws=P, size=256, seq=lens):
        return call("pyramidkv_cache_positions", ctypes.byref(cfg or config()), indices, seq, batch, k_layer, table, page, pages, positions, ws, size, None)
    for bad in (dict(indices=None), dict(table=None), dict(positions=None), dict(page=0), dict(pages=0), dict(batch=0), dict(k_layer=-1), dict(seq=None)):
        assert call_positions(**bad) == INVALID, bad
    assert call_positions(batch=65) == UNSUPPORTED and call_positions(cfg=config(head_dim=96)) == UNSUPPORTED
    assert call_positions(ws=None) == WORKSPACE and call_positions(size=255) == WORKSPACE and call_positions(ws=P + 64) == WORKSPACE
