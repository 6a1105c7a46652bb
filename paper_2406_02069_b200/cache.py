"""A cache that grows behind the compressed prompt: rotary positions, appends, decode attention, pages.

Same names as the C boundary (include/pyramidkv.h, "A cache that grows behind the compressed prompt"); this module checks
the tensors and marshals the arguments.  A decode step of one model looks like this:

    cache_reserve(cfg, cache, add, ws, granted=counts)                      # once: room for the new rows of every layer
    for layer in range(layers):
        append_cache(cfg, cache, layer, positions, k, v, ws, q=q, q_out=q, rotary=plan, counts=counts[layer])
        decode_attention_cache(cfg, cache, layer, q, out, ws)

and nothing in it waits for the device, so it can be captured into a CUDA graph.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import binding
from .binding import PkvConfig, PkvError, PkvTensor, _check, _lib, _lens, _native, _NOT_TAKEN, _stream, _TORCH_DTYPE, _want

MAX_CACHE_BATCH = 1024


class PkvCache(ctypes.Structure):
    """The C boundary's pkv_cache, and behind it what the cache was made for (which the C side does not look at)."""
    _fields_ = [("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("tables", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("layers", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("_end", ctypes.c_int32),
                ("heads_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("device", ctypes.c_int32)]


class PkvRotary(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("magnitude", ctypes.c_double),
                ("frequency", ctypes.c_double * 64)]


class PkvAttendOptions(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("softcap", ctypes.c_float), ("window", ctypes.c_int32),
                ("prefix", ctypes.c_int32), ("slopes", ctypes.c_void_p), ("q_positions", ctypes.c_void_p)]


LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "llama3": 3, "yarn": 4}


def make_rotary(rotary_dim: int, *, layout: str = "half", base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                original_positions: int = 0, low: Optional[float] = None, high: Optional[float] = None) -> PkvRotary:
    """Plan of rotary positions.  low and high: turns within original_positions between which frequencies are blended
    (default 1 and 4 for "llama3", 1 and 32 for "yarn")."""
    if layout not in LAYOUTS or scaling not in SCALINGS:
        raise ValueError("layout is one of %s, scaling one of %s" % (sorted(LAYOUTS), sorted(SCALINGS)))
    plan = PkvRotary()
    _check(_lib.pyramidkv_rotary_plan(int(rotary_dim), LAYOUTS[layout], SCALINGS[scaling], float(base), float(factor),
                                      int(original_positions), 1.0 if low is None else float(low),
                                      {"yarn": 32.0}.get(scaling, 4.0) if high is None else float(high), ctypes.byref(plan)),
           "pyramidkv_rotary_plan")
    return plan


def _plan(plan: PkvRotary) -> None:
    _want(isinstance(plan, PkvRotary), "a plan of rotary positions is what make_rotary gives")


def _same_device(tensors) -> None:
    """The library launches on the current device: the tensors have to be its."""
    current = torch.cuda.current_device()
    for name, t in tensors:
        _want(t is None or (t.is_cuda and t.device.index == current), "%s must live on the current CUDA device" % name)


def _int32(name: str, t: torch.Tensor, shape) -> None:
    _want(t.dtype == torch.int32 and tuple(t.shape) == tuple(shape) and t.is_contiguous(),
          "%s must be a contiguous int32 tensor of shape %s, not %s %s" % (name, tuple(shape), t.dtype, tuple(t.shape)))


class PagedCache:
    """The rows of `layers` layers and `batch` sequences in a pool of pages: the tensors, and the struct that the calls take.

    k_pool, v_pool [num_pages][page_size][d]; tables int32 [layers][batch][H_kv][max_pages]; lens int32 [layers][batch];
    positions int32 [num_pages][page_size] or None; refs int32 [num_pages] (table entries that name a page, 0 = free) or None,
    which only the page calls need.  The tensors are the caller's; the cache keeps them alive and reads their addresses once."""

    def __init__(self, cfg: PkvConfig, k_pool: torch.Tensor, v_pool: torch.Tensor, tables: torch.Tensor, lens: torch.Tensor, *,
                 positions: Optional[torch.Tensor] = None, refs: Optional[torch.Tensor] = None):
        for name, t in (("k_pool", k_pool), ("v_pool", v_pool)):
            _want(t.dim() == 3 and t.shape[2] == cfg.head_dim and t.is_contiguous() and t.dtype == _TORCH_DTYPE[cfg.dtype],
                  "%s must be a contiguous [num_pages][page_size][%d] tensor of type %s" % (name, cfg.head_dim, _TORCH_DTYPE[cfg.dtype]))
        _want(k_pool.shape == v_pool.shape, "k_pool and v_pool must have one shape")
        _want(tables.dim() == 4 and tables.shape[2] == cfg.num_kv_heads, "tables must be [layers][batch][%d][max_pages]" % cfg.num_kv_heads)
        _int32("tables", tables, tables.shape)
        _int32("lens", lens, tables.shape[:2])
        if positions is not None:
            _int32("positions", positions, k_pool.shape[:2])
        if refs is not None:
            _int32("refs", refs, k_pool.shape[:1])
        for name, t in (("v_pool", v_pool), ("tables", tables), ("lens", lens), ("positions", positions), ("refs", refs)):
            _want(t is None or t.device == k_pool.device, "%s must live where k_pool does" % name)
        _want(k_pool.is_cuda, "the cache must live on a CUDA device")
        _want(max(k_pool.shape[0], k_pool.shape[1], *tables.shape) <= 2 ** 31 - 1, "too many pages")
        self.k_pool, self.v_pool, self.tables, self.lens, self.positions, self.refs = k_pool, v_pool, tables, lens, positions, refs
        self.heads_kv, self.head_dim, self.dtype = cfg.num_kv_heads, cfg.head_dim, cfg.dtype
        self.layers, self.batch, self.max_pages = tables.shape[0], tables.shape[1], tables.shape[3]
        self.num_pages, self.page_size = k_pool.shape[0], k_pool.shape[1]
        ptr = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
        self.struct = PkvCache(ptr(k_pool), ptr(v_pool), ptr(positions), ptr(tables), ptr(lens), ptr(refs), self.num_pages,
                               self.page_size, self.layers, self.batch, self.max_pages, 0, self.heads_kv, self.head_dim, self.dtype,
                               k_pool.device.index)

    def fits(self, cfg: PkvConfig) -> bool:
        return (self.heads_kv, self.head_dim, self.dtype) == (cfg.num_kv_heads, cfg.head_dim, cfg.dtype)

    def block_table(self, layer: int, pages: Sequence[int]) -> torch.Tensor:
        """The packed block table that pyramidkv_compress_layer_paged takes, of the first pages[b] pages of each head of
        sequence b in a layer."""
        _want(len(pages) == self.batch, "one number of pages per sequence")
        return torch.cat([self.tables[layer, b, :, :n].reshape(-1) for b, n in enumerate(pages)])


def _check_cache(cfg: PkvConfig, cache: PagedCache, workspace: torch.Tensor) -> None:
    _want(isinstance(cache, PagedCache) and cache.fits(cfg), "the cache does not fit the configuration (KV heads, head size, type)")
    binding._check_workspace(workspace)
    _same_device((("the cache", cache.k_pool), ("the workspace", workspace)))


def cache_workspace_bytes(cfg: PkvConfig, cache: PagedCache) -> int:
    return int(_lib.pyramidkv_cache_workspace_bytes(ctypes.byref(cfg), ctypes.byref(cache.struct)))


def new_cache_workspace(cfg: PkvConfig, *caches: PagedCache) -> torch.Tensor:
    """A zeroed workspace that is large enough for every one of the caches."""
    sizes = [cache_workspace_bytes(cfg, c) for c in caches]
    if not sizes or min(sizes) == 0:
        raise PkvError(binding.PKV_ERR_INVALID_ARG, "pyramidkv_cache_workspace_bytes")
    return torch.zeros(max(sizes), dtype=torch.uint8, device=caches[0].k_pool.device)


def _rows(cfg: PkvConfig, name: str, t: torch.Tensor, batch: int, heads: int, tokens: int) -> None:
    _want(t.dim() == 4 and tuple(t.shape) == (batch, heads, tokens, cfg.head_dim) and t.stride(3) == 1 and t.dtype == _TORCH_DTYPE[cfg.dtype],
          "%s must be a [%d][%d][%d][%d] tensor of type %s with a contiguous last dimension, not %s %s" %
          (name, batch, heads, tokens, cfg.head_dim, _TORCH_DTYPE[cfg.dtype], t.dtype, tuple(t.shape)))


def _strides(t: Optional[torch.Tensor]) -> PkvTensor:
    """A [batch][heads][tokens][d] view.  A dimension of one entry has no say in where rows lie: it gets a stride that the
    checks of the C side accept, whatever torch left there."""
    if t is None:
        return PkvTensor(None, 0, 0, 0)
    st = t.stride(2) if t.shape[2] > 1 else t.shape[3]
    sh = t.stride(1) if t.shape[1] > 1 else t.shape[3]
    sb = t.stride(0) if t.shape[0] > 1 else t.shape[3]
    return PkvTensor(t.data_ptr(), sb, sh, st)


def _positions(positions: torch.Tensor, batch: int, tokens: int) -> int:
    """Stride between sequences of positions [batch][tokens] (a broadcast batch dimension is fine)."""
    _want(positions.dtype == torch.int32 and tuple(positions.shape) == (batch, tokens) and (tokens == 1 or positions.stride(1) == 1),
          "positions must be an int32 [%d][%d] tensor with a contiguous last dimension" % (batch, tokens))
    return positions.stride(0) if batch > 1 else 0


def rotary(cfg: PkvConfig, plan: PkvRotary, positions: torch.Tensor, q: Optional[torch.Tensor], k: Optional[torch.Tensor] = None,
           q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, inverse: bool = False, stream=None) -> None:
    """Rotary positions on q [batch][H_q][tokens][d] and k [batch][H_kv][tokens][d] (either may be None), into q_out and k_out
    or, where those are None, in place.  inverse: turned back, which is also what takes a gradient of the outputs to one of
    the inputs."""
    st = _native.rotary(cfg, plan, positions, q, k, q if q_out is None else q_out, k if k_out is None else k_out, inverse, stream) \
        if (q is not None or q_out is None) and (k is not None or k_out is None) else _NOT_TAKEN
    if st != _NOT_TAKEN:
        _check(st, "pyramidkv_rotary")
        return
    _plan(plan)
    _want(q is not None or k is not None, "rotary needs q or k")
    _want((q is not None or q_out is None) and (k is not None or k_out is None), "an output without its input")
    q_out, k_out = (q if q_out is None else q_out), (k if k_out is None else k_out)
    batch, tokens = (q if q is not None else k).shape[0], (q if q is not None else k).shape[2]
    for name, t, heads in (("q", q, cfg.num_q_heads), ("q_out", q_out, cfg.num_q_heads), ("k", k, cfg.num_kv_heads), ("k_out", k_out, cfg.num_kv_heads)):
        if t is not None:
            _rows(cfg, name, t, batch, heads, tokens)
    _same_device((("positions", positions), ("q", q), ("q_out", q_out), ("k", k), ("k_out", k_out)))
    stride = _positions(positions, batch, tokens)
    if batch == 0 or tokens == 0:
        return
    _check(_lib.pyramidkv_rotary(ctypes.byref(cfg), ctypes.byref(plan), positions.data_ptr(), stride, batch, tokens, _strides(q), _strides(q_out),
                                 _strides(k), _strides(k_out), 1 if inverse else 0, _stream(stream)), "pyramidkv_rotary")


def append_cache(cfg: PkvConfig, cache: PagedCache, layer: int, positions: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
                 workspace: torch.Tensor, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 rotary: Optional[PkvRotary] = None, counts: Optional[torch.Tensor] = None, stream=None) -> None:
    """New rows of a layer into their pages: k, v [batch][H_kv][tokens][d] become the last counts[b] (None: tokens) rows of
    their sequences, keys and q given their rotary positions if there is a plan.  q_out None: q in place."""
    st = _native.append_cache(cfg, getattr(cache, "struct", None), layer, positions, k, v, workspace, q, q if q_out is None else q_out, rotary,
                              counts, stream) if q is not None or q_out is None else _NOT_TAKEN
    if st != _NOT_TAKEN:
        _check(st, "pyramidkv_append_cache")
        return
    _check_cache(cfg, cache, workspace)
    _want(k.dim() == 4, "k must be [batch][H_kv][tokens][d]")
    tokens = k.shape[2]
    _rows(cfg, "k", k, cache.batch, cfg.num_kv_heads, tokens)
    _rows(cfg, "v", v, cache.batch, cfg.num_kv_heads, tokens)
    _want(q is not None or q_out is None, "q_out without q")
    q_out = q if q_out is None else q_out
    if q is not None:
        _rows(cfg, "q", q, cache.batch, cfg.num_q_heads, tokens)
        _rows(cfg, "q_out", q_out, cache.batch, cfg.num_q_heads, tokens)
    if rotary is not None:
        _plan(rotary)
    _want(positions is not None or (rotary is None and cache.positions is None), "positions are needed for the rotation and for the cache's positions")
    stride = _positions(positions, cache.batch, tokens) if positions is not None else 0
    if counts is not None:
        _int32("counts", counts, (cache.batch,))
    _same_device((("positions", positions), ("k", k), ("v", v), ("q", q), ("q_out", q_out), ("counts", counts)))
    if tokens == 0:
        return
    _check(_lib.pyramidkv_append_cache(ctypes.byref(cfg), ctypes.byref(cache.struct), int(layer), ctypes.byref(rotary) if rotary is not None else None,
                                       positions.data_ptr() if positions is not None else None, stride, tokens, _strides(q), _strides(q_out),
                                       _strides(k), _strides(v), counts.data_ptr() if counts is not None else None, workspace.data_ptr(),
                                       workspace.numel(), _stream(stream)), "pyramidkv_append_cache")


def cache_positions(cfg: PkvConfig, indices: torch.Tensor, seq_lens: Sequence[int], k_layer: int, block_table: torch.Tensor,
                    positions: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    """Positions of a compressed layer's rows from the packed list that compress_layer_paged wrote, into positions
    [num_pages][page_size] at the rows' slots."""
    lens, batch = _lens(seq_lens)
    binding._check_rows(cfg, binding.total_rows(cfg, k_layer, seq_lens), None, None, indices)
    binding._check_workspace(workspace)
    _want(positions.dim() == 2, "positions must be [num_pages][page_size]")
    _int32("positions", positions, positions.shape)
    entries = cfg.num_kv_heads * sum(binding.pages_needed(cfg, k_layer, n, positions.shape[1]) for n in seq_lens)
    _want(block_table.dtype == torch.int32 and block_table.is_contiguous() and block_table.numel() >= entries,
          "block_table must be a contiguous int32 tensor of at least %d entries" % entries)
    _same_device((("indices", indices), ("block_table", block_table), ("positions", positions), ("the workspace", workspace)))
    _check(_lib.pyramidkv_cache_positions(ctypes.byref(cfg), indices.data_ptr(), lens, batch, int(k_layer), block_table.data_ptr(),
                                          int(positions.shape[1]), int(positions.shape[0]), positions.data_ptr(), workspace.data_ptr(),
                                          workspace.numel(), _stream(stream)), "pyramidkv_cache_positions")


def decode_attention_cache(cfg: PkvConfig, cache: PagedCache, layer: int, q: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor,
                           q_positions: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, *, scale: float = 0.0,
                           softcap: float = 0.0, slopes: Optional[torch.Tensor] = None, window: int = 0, prefix: int = 0, stream=None) -> None:
    """One new token per sequence attends to the rows of a layer: q [batch][H_q][d] (any strides of 16 bytes; or
    [batch][H_q][1][d] as append_cache leaves it) -> out [batch][H_q][d] float32.  With q_positions [batch] int32 rows at later
    positions are not seen; window leaves out rows at a distance of window and more unless their position is below prefix;
    slopes [H_q] float32 times the distance is taken off the logits; softcap caps them.  lse: the logarithm of the sums."""
    st = _native.decode_attention_cache(cfg, getattr(cache, "struct", None), layer, q, out, workspace, q_positions, lse, scale, softcap, slopes,
                                        window, prefix, stream)
    if st != _NOT_TAKEN:
        _check(st, "pyramidkv_decode_attention_cache")
        return
    _check_cache(cfg, cache, workspace)
    if q.dim() == 4 and q.shape[2] == 1:
        q = q[:, :, 0]
    _want(q.dim() == 3 and tuple(q.shape) == (cache.batch, cfg.num_q_heads, cfg.head_dim) and q.stride(2) == 1 and q.dtype == _TORCH_DTYPE[cfg.dtype],
          "q must be a [%d][%d][%d] tensor of type %s with a contiguous last dimension" % (cache.batch, cfg.num_q_heads, cfg.head_dim, _TORCH_DTYPE[cfg.dtype]))
    _want(out.dtype == torch.float32 and out.is_contiguous() and tuple(out.shape) == (cache.batch, cfg.num_q_heads, cfg.head_dim),
          "out must be a contiguous float32 [batch][H_q][d] tensor")
    if lse is not None:
        _want(lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == (cache.batch, cfg.num_q_heads),
              "lse must be a contiguous float32 [batch][H_q] tensor")
    if slopes is not None:
        _want(slopes.dtype == torch.float32 and slopes.is_contiguous() and tuple(slopes.shape) == (cfg.num_q_heads,),
              "slopes must be a contiguous float32 [H_q] tensor")
    if q_positions is not None:
        _int32("q_positions", q_positions, (cache.batch,))
    _same_device((("q", q), ("out", out), ("lse", lse), ("slopes", slopes), ("q_positions", q_positions)))
    options = PkvAttendOptions(scale, softcap, int(window), int(prefix), slopes.data_ptr() if slopes is not None else None,
                               q_positions.data_ptr() if q_positions is not None else None)
    view = PkvTensor(q.data_ptr(), q.stride(0) if cache.batch > 1 else 0, q.stride(1) if cfg.num_q_heads > 1 else 0, 0)
    _check(_lib.pyramidkv_decode_attention_cache(ctypes.byref(cfg), ctypes.byref(cache.struct), int(layer), ctypes.byref(options), view,
                                                 out.data_ptr(), lse.data_ptr() if lse is not None else None, workspace.data_ptr(),
                                                 workspace.numel(), _stream(stream)), "pyramidkv_decode_attention_cache")


def _page_call(cfg: PkvConfig, cache: PagedCache, to: Optional[PagedCache], workspace: torch.Tensor) -> PagedCache:
    _check_cache(cfg, cache, workspace)
    to = cache if to is None else to
    if to is not cache:
        _check_cache(cfg, to, workspace)
    _want(cache.refs is not None and to.refs is not None, "the page calls need the cache's refs")
    return to


def _add(add: torch.Tensor, layers: int, batch: int) -> int:
    """Entries between the layers of add, int32 [batch] or [layers][batch] (expanded over the layers is fine)."""
    _want(add.dtype == torch.int32 and tuple(add.shape) in ((batch,), (layers, batch)) and (batch == 1 or add.stride(-1) == 1),
          "add must be an int32 [%d] or [%d][%d] tensor with a contiguous last dimension" % (batch, layers, batch))
    return add.stride(0) if add.dim() == 2 and layers > 1 else 0


def cache_reserve(cfg: PkvConfig, cache: PagedCache, add: torch.Tensor, workspace: torch.Tensor, granted: Optional[torch.Tensor] = None,
                  to: Optional[PagedCache] = None, stream=None) -> None:
    """Room for add (int32 [batch] or [layers][batch]) more rows: lens grow, new pages are dealt out.  granted [layers][batch]
    int32 gets what was made room for: add, or zeros where the pool had too few pages and nothing changed.  to: another
    cache over the same pools that takes the result; None: in place."""
    st = _native.cache_reserve(cfg, getattr(cache, "struct", None), getattr(cache if to is None else to, "struct", None), add, granted, workspace, stream)
    if st != _NOT_TAKEN:
        _check(st, "pyramidkv_cache_reserve")
        return
    to = _page_call(cfg, cache, to, workspace)
    stride = _add(add, cache.layers, cache.batch)
    if granted is not None:
        _int32("granted", granted, (cache.layers, to.batch))
    _same_device((("add", add), ("granted", granted)))
    _check(_lib.pyramidkv_cache_reserve(ctypes.byref(cfg), ctypes.byref(cache.struct), ctypes.byref(to.struct), add.data_ptr(), stride,
                                        granted.data_ptr() if granted is not None else None, workspace.data_ptr(), workspace.numel(),
                                        _stream(stream)), "pyramidkv_cache_reserve")


def cache_fork(cfg: PkvConfig, cache: PagedCache, parents: torch.Tensor, workspace: torch.Tensor, add: Optional[torch.Tensor] = None,
               granted: Optional[torch.Tensor] = None, to: Optional[PagedCache] = None, stream=None) -> None:
    """Sequence c goes on from sequence parents[c] (int32), or starts empty for -1: full pages are shared, a part-filled last page
    is copied for every child behind the first, pages that nobody goes on with are freed, and add more rows are made room
    for as by cache_reserve.  to: another cache over the same pools, with any number of sequences; None: in place.  With another
    one the parents' rows can still be read through `cache`; those of sequences that nobody goes on with cannot, their pages
    may hold other rows already."""
    st = _native.cache_fork(cfg, getattr(cache, "struct", None), getattr(cache if to is None else to, "struct", None), parents, add, granted, workspace, stream)
    if st != _NOT_TAKEN:
        _check(st, "pyramidkv_cache_fork")
        return
    to = _page_call(cfg, cache, to, workspace)
    _int32("parents", parents, (to.batch,))
    stride = _add(add, cache.layers, to.batch) if add is not None else 0
    if granted is not None:
        _int32("granted", granted, (cache.layers, to.batch))
    _same_device((("parents", parents), ("add", add), ("granted", granted)))
    _check(_lib.pyramidkv_cache_fork(ctypes.byref(cfg), ctypes.byref(cache.struct), ctypes.byref(to.struct), parents.data_ptr(),
                                     add.data_ptr() if add is not None else None, stride, granted.data_ptr() if granted is not None else None,
                                     workspace.data_ptr(), workspace.numel(), _stream(stream)), "pyramidkv_cache_fork")


def cache_compact(cfg: PkvConfig, cache: PagedCache, workspace: torch.Tensor, used: Optional[torch.Tensor] = None,
                  to: Optional[PagedCache] = None, stream=None) -> None:
    """Moves the pages in use to the lowest numbers; used (int32, one entry) gets how many there are."""
    st = _native.cache_compact(cfg, getattr(cache, "struct", None), getattr(cache if to is None else to, "struct", None), used, workspace, stream)
    if st != _NOT_TAKEN:
        _check(st, "pyramidkv_cache_compact")
        return
    to = _page_call(cfg, cache, to, workspace)
    if used is not None:
        _int32("used", used, (1,))
    _same_device((("used", used),))
    _check(_lib.pyramidkv_cache_compact(ctypes.byref(cfg), ctypes.byref(cache.struct), ctypes.byref(to.struct),
                                        used.data_ptr() if used is not None else None, workspace.data_ptr(), workspace.numel(),
                                        _stream(stream)), "pyramidkv_cache_compact")
