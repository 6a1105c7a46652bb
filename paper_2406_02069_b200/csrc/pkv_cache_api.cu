// Host side of the growing cache: rotary plans, argument checks, workspace carving and launches of the calls that include/pyramidkv.h
// lists under "A cache that grows behind the compressed prompt".
#include <atomic>
#include <cmath>
#include <cstring>

#include "pkv_cache_attend.cuh"
#include "pkv_cache_pages.cuh"
#include "pkv_common.cuh"
#include "pkv_host.cuh"
#include "pkv_rotary.cuh"

namespace pkv {
namespace {

constexpr int64_t kMaxRows = int64_t{1} << 30;                   // of a sequence: row numbers and what is added to them fit 32 bits
constexpr int64_t kMaxPages = int64_t{1} << 27;                  // of a pool: eight times as many requests are counted in 32 bits

constexpr int64_t kMaxUnits = 65536;                             // blocks of query heads of a batch, each with a counter in the workspace

int elem_bytes(const pkv_config* c) { return c->dtype == PKV_DTYPE_FP32 ? 4 : 2; }

bool pointer_ok(const void* p, size_t align) { return p && reinterpret_cast<uintptr_t>(p) % align == 0; }

// Query heads that a CTA of the attention takes.  16-bit rows: four cost what one does (they are rows of one product); fp32: each has
// its own instructions (three sequences of up to 1231 rows, 32 heads of their own: 35 us four at a time, 28 one at a time).
int heads_per_cta(const pkv_config* c) {
  const int group = c->num_q_heads / c->num_kv_heads;
  if (group >= 5) return 8;
  return c->dtype == PKV_DTYPE_FP32 && group < 3 ? group : 4;
}
int head_blocks(const pkv_config* c) {
  const int group = c->num_q_heads / c->num_kv_heads, gt = heads_per_cta(c);
  return (group + gt - 1) / gt;
}

int cache_check(const pkv_config* c, const pkv_cache* x) {
  if (!config_ok(c) || !x) return PKV_ERR_INVALID_ARG;
  if (const int st = config_supported(c)) return st;
  if (!pointer_ok(x->k_pool, 16) || !pointer_ok(x->v_pool, 16) || !pointer_ok(x->tables, 4) || !pointer_ok(x->lens, 4)) return PKV_ERR_INVALID_ARG;
  if ((x->positions && !pointer_ok(x->positions, 4)) || (x->refs && !pointer_ok(x->refs, 4))) return PKV_ERR_INVALID_ARG;
  if (x->num_pages < 1 || x->page_size < 1 || x->layers < 1 || x->batch < 1 || x->max_pages < 1) return PKV_ERR_INVALID_ARG;
  const int64_t rows = static_cast<int64_t>(x->max_pages) * x->page_size;
  if (x->batch > PKV_MAX_CACHE_BATCH || x->layers > 65535 || c->num_q_heads > 65535 || x->num_pages > kMaxPages || rows > kMaxRows ||
      static_cast<int64_t>(x->num_pages) * x->page_size > INT32_MAX)
    return PKV_ERR_UNSUPPORTED;
  if ((rows + kCaTile - 1) / kCaTile * x->batch > INT32_MAX) return PKV_ERR_UNSUPPORTED;      // tiles of a head
  if (static_cast<int64_t>(x->batch) * c->num_kv_heads * head_blocks(c) > kMaxUnits) return PKV_ERR_UNSUPPORTED;
  static_assert(int64_t{PKV_MAX_CACHE_BATCH} * 65535 < INT32_MAX, "sequences of all layers are counted in 32 bits");
  return PKV_OK;
}

struct CacheWorkspace {
  uint32_t* status;
  int32_t* counters;
  int32_t* group_counters;
  int32_t* state;
  float* partials;
  int32_t* list;
  int32_t* second;
  int32_t* place;
  PageArrays staged;
  size_t bytes;
};

CacheWorkspace carve_cache(const pkv_config* c, const pkv_cache* x, void* base) {
  CacheWorkspace w{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    void* p = base ? static_cast<char*>(base) + at : nullptr;
    at += align_up(bytes);
    return p;
  };
  const size_t units = static_cast<size_t>(x->layers) * x->batch, pages = static_cast<size_t>(x->num_pages);
  w.status = static_cast<uint32_t*>(take(256));
  w.state = static_cast<int32_t*>(take(256));
  // the counters, which have to be zero between calls, lie at the same place for every cache: a workspace may serve several
  w.counters = static_cast<int32_t*>(take(kMaxUnits * 4));
  w.group_counters = static_cast<int32_t*>(take(size_t{2} * kCaMaxGrid * 4));
  w.partials = static_cast<float*>(take(size_t{2} * kCaMaxGrid * kCaPartial * sizeof(float)));
  w.list = static_cast<int32_t*>(take(pages * 4));
  w.second = static_cast<int32_t*>(take(pages * 4));
  w.place = static_cast<int32_t*>(take(pages * 4));
  w.staged.tables = static_cast<int32_t*>(take(units * c->num_kv_heads * x->max_pages * 4));
  w.staged.lens = static_cast<int32_t*>(take(units * 4));
  w.staged.refs = static_cast<int32_t*>(take(pages * 4));
  w.bytes = at;
  return w;
}

int cache_workspace(const pkv_config* c, const pkv_cache* x, void* ws, size_t bytes, CacheWorkspace* out) {
  if (!ws || reinterpret_cast<uintptr_t>(ws) % kAlign) return PKV_ERR_WORKSPACE;
  *out = carve_cache(c, x, ws);
  return out->bytes <= bytes ? PKV_OK : PKV_ERR_WORKSPACE;
}

size_t pool_bytes(const pkv_config* c, const pkv_cache* x) {
  return static_cast<size_t>(x->num_pages) * x->page_size * c->head_dim * elem_bytes(c);
}

Output rows_of(const pkv_tensor& t, int64_t batch, int heads, int64_t tokens, int d, int elem) {
  return {t.ptr, static_cast<size_t>((batch - 1) * t.stride_batch + (heads - 1) * t.stride_head + (tokens - 1) * t.stride_token + d) * elem};
}

// ---------------------------------------------------------------- rotary positions
bool plan_ok(const pkv_config* c, const pkv_rotary* r) {
  if (r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > c->head_dim) return false;
  if (r->layout != PKV_ROTARY_HALF && r->layout != PKV_ROTARY_INTERLEAVED) return false;
  if (!std::isfinite(r->magnitude)) return false;
  for (int i = 0; i < r->rotary_dim / 2; ++i)
    if (!std::isfinite(r->frequency[i])) return false;
  return true;
}

template <typename T, int VEC, bool APPEND>
void launch_rotary_units(RotaryParams& p, int d, cudaStream_t st) {
  p.units = d / (2 * VEC);
  p.rot_units = p.half / VEC;
  p.unit_lanes = p.units;
  const int heads = p.heads_q + p.heads_kv * (APPEND ? 2 : 1);
  const int64_t tokens = static_cast<int64_t>(p.batch) * p.tokens;
  const int room = kRotThreads / p.units;
  int splits = 1;
  // Enough rows to fill the device: at most a warp's lanes, four to a head's unit, stay with a token and go through its heads, so
  // that its sines are formed four times over.  Fewer: lanes for every row, so that nothing is done in turn.
  const int sms = std::max(1, device_sm_count());
  if (tokens * heads * p.units > static_cast<int64_t>(sms) * 4096) {
    p.head_lanes = std::max(1, std::min(4, 32 / p.units));
  } else {
    p.head_lanes = 1;
    while (p.head_lanes < heads && p.head_lanes < room) p.head_lanes *= 2;
    splits = (heads + p.head_lanes - 1) / p.head_lanes;
  }
  const int block_tokens = room / p.head_lanes;
  // (counted with the outputs: a call of few rows is bound by its host time)
  launch_uncounted(rotary_kernel<T, VEC, APPEND>, dim3(static_cast<unsigned>((tokens + block_tokens - 1) / block_tokens), splits), dim3(kRotThreads), 0, st, p);
}

template <typename T, bool APPEND>
void launch_rotary_type(RotaryParams& p, int d, cudaStream_t st) {
  constexpr int VEC = 16 / static_cast<int>(sizeof(T));
  // 16-byte pieces need both halves of the rotated part (interleaved: its end) at multiples of 16 bytes
  if (p.half % VEC == 0) launch_rotary_units<T, VEC, APPEND>(p, d, st);
  else if (p.half % 2 == 0) launch_rotary_units<T, 2, APPEND>(p, d, st);
  else launch_rotary_units<T, 1, APPEND>(p, d, st);
}

template <bool APPEND>
int launch_rotary(const pkv_config* c, const pkv_rotary* plan, int inverse, RotaryParams& p, cudaStream_t st) {
  p.half = plan ? plan->rotary_dim / 2 : 0;
  p.interleaved = plan && plan->layout == PKV_ROTARY_INTERLEAVED;
  p.magnitude_cos = plan ? static_cast<float>(plan->magnitude) : 1.f;
  p.magnitude_sin = inverse ? -p.magnitude_cos : p.magnitude_cos;
  for (int i = 0; i < p.half; ++i) p.turns[i] = plan->frequency[i] / 6.283185307179586476925;
  switch (c->dtype) {
    case PKV_DTYPE_FP32: launch_rotary_type<float, APPEND>(p, c->head_dim, st); break;
    case PKV_DTYPE_BF16: launch_rotary_type<__nv_bfloat16, APPEND>(p, c->head_dim, st); break;
    default: launch_rotary_type<__half, APPEND>(p, c->head_dim, st); break;
  }
  return check_launch();
}

// Tokens of a call: what the grid can hold.
bool tokens_ok(int64_t batch, int64_t tokens) { return batch >= 1 && tokens >= 1 && batch * tokens <= INT32_MAX; }

// ---------------------------------------------------------------- attention
template <typename T, int D, int GT, int POS>
int launch_cache_attend(CacheAttendParams& p, int64_t max_rows, cudaStream_t st) {
  constexpr size_t kSmem = kCaWarps<T> * CaWarp<T, D, GT, POS>::kRing + 2 * GT * (sizeof(T) == 4 ? (D + 4) * 4 : D * 2 + 64);
  static std::atomic<int> per_sm[64];      // CTAs that an SM holds, once the kernel's shared memory is set up on a device
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return PKV_ERR_CUDA;
  int fit = per_sm[dev].load(std::memory_order_acquire);
  if (!fit) {
    if (cudaFuncSetAttribute(cache_attend_kernel<T, D, GT, POS>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem)) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, cache_attend_kernel<T, D, GT, POS>, kCaThreads<T>, kSmem) != cudaSuccess || fit < 1)
      return PKV_ERR_CUDA;
    per_sm[dev].store(fit, std::memory_order_release);
  }
  const int sms = device_sm_count();
  if (sms <= 0) return PKV_ERR_CUDA;
  const int64_t units = static_cast<int64_t>(p.batch) * p.num_kv_heads * p.head_blocks;
  // no more CTAs than there can be tiles
  const int grid = static_cast<int>(std::min<int64_t>(std::min(kCaMaxGrid, sms * fit), (max_rows + kCaTile - 1) / kCaTile * units));
  launch_pdl(cache_attend_kernel<T, D, GT, POS>, dim3(grid), dim3(kCaThreads<T>), kSmem, st, p);
  return check_launch();
}

template <typename T, int D, int GT>
int dispatch_positions(CacheAttendParams& p, int64_t max_rows, cudaStream_t st) {
  if (!p.q_pos) return launch_cache_attend<T, D, GT, 0>(p, max_rows, st);
  return p.slopes ? launch_cache_attend<T, D, GT, 2>(p, max_rows, st) : launch_cache_attend<T, D, GT, 1>(p, max_rows, st);
}

template <typename T, int D>
int dispatch_cache_attend(CacheAttendParams& p, int gt, int64_t max_rows, cudaStream_t st) {
  if constexpr (sizeof(T) == 4) {
    if (gt == 1) return dispatch_positions<T, D, 1>(p, max_rows, st);
    if (gt == 2) return dispatch_positions<T, D, 2>(p, max_rows, st);
  }
  return gt == 4 ? dispatch_positions<T, D, 4>(p, max_rows, st) : dispatch_positions<T, D, 8>(p, max_rows, st);
}

// ---------------------------------------------------------------- pages
int launch_cluster(void (*kernel)(PagesParams), const PagesParams& p, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(kPgCluster);
  cfg.blockDim = dim3(kPgThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kPgCluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) return PKV_ERR_CUDA;
  note_launch(st);
  return check_launch();
}

// Blocks for a grid-stride loop over n items.
unsigned stride_grid(int64_t n, int threads, int sms, int per_sm) {
  return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((n + threads - 1) / threads, static_cast<int64_t>(sms) * per_sm)));
}

// Checks of a page call and the part of its parameters that all three share.
int pages_setup(const pkv_config* c, const pkv_cache* from, const pkv_cache* to, void* workspace, size_t workspace_bytes, PagesParams* p) {
  if (!from || !to) return PKV_ERR_INVALID_ARG;
  if (const int st = cache_check(c, from)) return st;
  if (const int st = cache_check(c, to)) return st;
  if (!from->refs || !to->refs) return PKV_ERR_INVALID_ARG;
  if (from->k_pool != to->k_pool || from->v_pool != to->v_pool || from->positions != to->positions || from->num_pages != to->num_pages ||
      from->page_size != to->page_size || from->layers != to->layers || from->max_pages != to->max_pages)
    return PKV_ERR_INVALID_ARG;
  const int same = (from->tables == to->tables) + (from->lens == to->lens) + (from->refs == to->refs);
  if (same != 0 && same != 3) return PKV_ERR_INVALID_ARG;
  if (same == 3 && from->batch != to->batch) return PKV_ERR_INVALID_ARG;
  CacheWorkspace w, other;
  if (const int st = cache_workspace(c, from, workspace, workspace_bytes, &w)) return st;
  if (const int st = cache_workspace(c, to, workspace, workspace_bytes, &other)) return st;
  if (to->batch > from->batch) w = other;                        // the larger one's arrays
  std::memset(p, 0, sizeof *p);
  p->home = PageArrays{from->tables, from->lens, from->refs};
  p->from = p->home;
  p->to = PageArrays{to->tables, to->lens, to->refs};
  p->in_place = same == 3;
  p->k_pool = from->k_pool;
  p->v_pool = from->v_pool;
  p->pos_pool = from->positions;
  p->layers = from->layers;
  p->from_batch = from->batch;
  p->to_batch = to->batch;
  p->num_kv_heads = c->num_kv_heads;
  p->max_pages = from->max_pages;
  p->page_size = from->page_size;
  p->num_pages = from->num_pages;
  p->row_pieces = c->head_dim * elem_bytes(c) / 16;
  p->status = w.status;
  p->state = w.state;
  p->list = w.list;
  p->second = w.second;
  p->place = w.place;
  p->staged = w.staged;
  return PKV_OK;
}

int run_fork(const pkv_config* c, const pkv_cache* from, const pkv_cache* to, PagesParams& p, cudaStream_t st) {
  const int sms = device_sm_count();
  if (sms <= 0) return PKV_ERR_CUDA;
  if (p.in_place && p.parents) {           // sequences change places: the old tables are set aside
    p.from = p.staged;
    const int64_t entries = static_cast<int64_t>(p.layers) * p.from_batch * p.num_kv_heads * p.max_pages;
    launch_pdl(pages_stage_kernel, dim3(stride_grid(std::max<int64_t>(entries, p.num_pages), kPgCarryThreads, sms, 8)), dim3(kPgCarryThreads), 0, st, p);
  } else if (!p.in_place && p.parents) {
    launch_pdl(pages_refs_kernel, dim3(stride_grid(p.num_pages, kPgCarryThreads, sms, 8)), dim3(kPgCarryThreads), 0, st, p);
  }
  if (p.parents || !p.in_place)
    launch_pdl(pages_carry_kernel, dim3(p.to_batch + (p.parents ? p.from_batch : 0), p.layers), dim3(kPgCarryThreads), 0, st, p);
  if (const int rc = launch_cluster(pages_deal_kernel, p, st)) return rc;
  if (p.parents) {
    launch_pdl(pages_copy_kernel, dim3(p.to_batch, p.layers), dim3(kPgCarryThreads), 0, st, p);
    note_outputs(st, {{from->k_pool, pool_bytes(c, from)}, {from->v_pool, pool_bytes(c, from)}});
  }
  return check_launch();
}

}  // namespace
}  // namespace pkv

using namespace pkv;

extern "C" {

size_t pyramidkv_cache_workspace_bytes(const pkv_config* cfg, const pkv_cache* cache) {
  return cache_check(cfg, cache) == PKV_OK ? carve_cache(cfg, cache, nullptr).bytes : 0;
}

int pyramidkv_rotary_plan(int32_t rotary_dim, int32_t layout, int32_t scaling, double base, double factor, int32_t original_positions,
                          double low, double high, pkv_rotary* out) {
  constexpr double kTwoPi = 6.283185307179586476925;
  if (!out || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > 128) return PKV_ERR_INVALID_ARG;
  if (layout != PKV_ROTARY_HALF && layout != PKV_ROTARY_INTERLEAVED) return PKV_ERR_INVALID_ARG;
  if (scaling < PKV_ROTARY_SCALE_NONE || scaling > PKV_ROTARY_SCALE_YARN) return PKV_ERR_INVALID_ARG;
  if (!(base > 1.0) || !std::isfinite(base) || !(factor >= 1.0) || !std::isfinite(factor)) return PKV_ERR_INVALID_ARG;
  if (scaling == PKV_ROTARY_SCALE_NTK && rotary_dim < 4) return PKV_ERR_INVALID_ARG;
  if (scaling == PKV_ROTARY_SCALE_LLAMA3 || scaling == PKV_ROTARY_SCALE_YARN)
    if (original_positions < 1 || !(low > 0.0) || !(high > low) || !std::isfinite(high)) return PKV_ERR_INVALID_ARG;
  std::memset(out, 0, sizeof *out);
  out->rotary_dim = rotary_dim;
  out->layout = layout;
  out->magnitude = scaling == PKV_ROTARY_SCALE_YARN ? 0.1 * std::log(factor) + 1.0 : 1.0;
  const double dim = rotary_dim;
  if (scaling == PKV_ROTARY_SCALE_NTK) base *= std::pow(factor, dim / (dim - 2.0));
  // pair that makes `turns` turns within the original positions
  auto pair_of = [&](double turns) { return dim * std::log(original_positions / (turns * kTwoPi)) / (2.0 * std::log(base)); };
  double first = 0.0, width = 1.0;
  if (scaling == PKV_ROTARY_SCALE_YARN) {
    first = std::max(std::floor(pair_of(high)), 0.0);
    width = std::max(std::min(std::ceil(pair_of(low)), dim - 1.0) - first, 0.001);
  }
  for (int i = 0; i < rotary_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / dim);
    double blend = 1.0;                    // share of the unscaled frequency
    if (scaling == PKV_ROTARY_SCALE_LINEAR) blend = 0.0;
    if (scaling == PKV_ROTARY_SCALE_LLAMA3) blend = (original_positions * f / kTwoPi - low) / (high - low);
    if (scaling == PKV_ROTARY_SCALE_YARN) blend = 1.0 - (i - first) / width;
    blend = std::min(std::max(blend, 0.0), 1.0);
    out->frequency[i] = blend * f + (1.0 - blend) * f / factor;
  }
  return PKV_OK;
}

int pyramidkv_rotary(const pkv_config* cfg, const pkv_rotary* plan, const int32_t* positions, int64_t positions_stride, int32_t batch,
                     int32_t tokens, pkv_tensor q, pkv_tensor q_out, pkv_tensor k, pkv_tensor k_out, int32_t inverse, void* stream) {
  if (!config_ok(cfg) || !plan || !positions || reinterpret_cast<uintptr_t>(positions) % 4) return PKV_ERR_INVALID_ARG;
  if (const int st = config_supported(cfg)) return st;
  if (!plan_ok(cfg, plan) || !tokens_ok(batch, tokens)) return PKV_ERR_INVALID_ARG;
  if (cfg->num_q_heads > 65535) return PKV_ERR_UNSUPPORTED;
  const int d = cfg->head_dim, e = elem_bytes(cfg);
  if (!q.ptr != !q_out.ptr || !k.ptr != !k_out.ptr || (!q.ptr && !k.ptr)) return PKV_ERR_INVALID_ARG;
  RotaryParams p{};
  if (q.ptr) {
    if (!tensor_ok(q, d, e, batch, cfg->num_q_heads) || !tensor_ok(q_out, d, e, batch, cfg->num_q_heads)) return PKV_ERR_INVALID_ARG;
    p.q = view(q);
    p.q_out = view(q_out);
    p.heads_q = cfg->num_q_heads;
  }
  if (k.ptr) {
    if (!tensor_ok(k, d, e, batch, cfg->num_kv_heads) || !tensor_ok(k_out, d, e, batch, cfg->num_kv_heads)) return PKV_ERR_INVALID_ARG;
    p.k = view(k);
    p.k_out = view(k_out);
    p.heads_kv = cfg->num_kv_heads;
  }
  p.positions = positions;
  p.positions_stride = positions_stride;
  p.batch = batch;
  p.tokens = tokens;
  const int st = launch_rotary<false>(cfg, plan, inverse, p, static_cast<cudaStream_t>(stream));
  note_outputs(static_cast<cudaStream_t>(stream),
               {rows_of(q_out, batch, cfg->num_q_heads, tokens, d, e), rows_of(k_out, batch, cfg->num_kv_heads, tokens, d, e)}, st == PKV_OK);
  return st;
}

int pyramidkv_append_cache(const pkv_config* cfg, const pkv_cache* cache, int32_t layer, const pkv_rotary* plan_or_null,
                           const int32_t* positions, int64_t positions_stride, int32_t tokens, pkv_tensor q, pkv_tensor q_out,
                           pkv_tensor k, pkv_tensor v, const int32_t* counts_or_null, void* workspace, size_t workspace_bytes,
                           void* stream) {
  if (const int st = cache_check(cfg, cache)) return st;
  if (layer < 0 || layer >= cache->layers || !tokens_ok(cache->batch, tokens)) return PKV_ERR_INVALID_ARG;
  if (plan_or_null && !plan_ok(cfg, plan_or_null)) return PKV_ERR_INVALID_ARG;
  if (!positions && (plan_or_null || cache->positions)) return PKV_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(positions) % 4 || reinterpret_cast<uintptr_t>(counts_or_null) % 4) return PKV_ERR_INVALID_ARG;
  const int d = cfg->head_dim, e = elem_bytes(cfg), batch = cache->batch;
  if (!q.ptr != !q_out.ptr) return PKV_ERR_INVALID_ARG;
  if (!tensor_ok(k, d, e, batch, cfg->num_kv_heads) || !tensor_ok(v, d, e, batch, cfg->num_kv_heads)) return PKV_ERR_INVALID_ARG;
  if (q.ptr && (!tensor_ok(q, d, e, batch, cfg->num_q_heads) || !tensor_ok(q_out, d, e, batch, cfg->num_q_heads))) return PKV_ERR_INVALID_ARG;
  CacheWorkspace w;
  if (const int st = cache_workspace(cfg, cache, workspace, workspace_bytes, &w)) return st;
  RotaryParams p{};
  if (q.ptr) {
    p.q = view(q);
    p.q_out = view(q_out);
    p.heads_q = cfg->num_q_heads;
  }
  p.k = view(k);
  p.v = view(v);
  p.heads_kv = cfg->num_kv_heads;
  p.positions = positions;
  p.positions_stride = positions_stride;
  p.batch = batch;
  p.tokens = tokens;
  p.counts = counts_or_null;
  p.lens = cache->lens + static_cast<int64_t>(layer) * batch;
  p.table = cache->tables + static_cast<int64_t>(layer) * batch * cfg->num_kv_heads * cache->max_pages;
  p.max_pages = cache->max_pages;
  p.page_size = cache->page_size;
  p.num_pages = cache->num_pages;
  p.k_pool = cache->k_pool;
  p.v_pool = cache->v_pool;
  p.pos_pool = cache->positions;
  p.status = w.status;
  const int st = launch_rotary<true>(cfg, plan_or_null, 0, p, static_cast<cudaStream_t>(stream));
  note_outputs(static_cast<cudaStream_t>(stream), {rows_of(q_out, batch, cfg->num_q_heads, tokens, d, e),
                                                   {cache->k_pool, pool_bytes(cfg, cache)}, {cache->v_pool, pool_bytes(cfg, cache)}}, st == PKV_OK);
  return st;
}

int pyramidkv_decode_attention_cache(const pkv_config* cfg, const pkv_cache* cache, int32_t layer, const pkv_attend_options* options_or_null,
                                     pkv_tensor q, float* out, float* lse_or_null, void* workspace, size_t workspace_bytes, void* stream) {
  if (const int st = cache_check(cfg, cache)) return st;
  if (layer < 0 || layer >= cache->layers || !pointer_ok(out, 4) || reinterpret_cast<uintptr_t>(lse_or_null) % 4) return PKV_ERR_INVALID_ARG;
  const int64_t per16 = 16 / elem_bytes(cfg);
  if (!pointer_ok(q.ptr, 16) || q.stride_batch % per16 || q.stride_head % per16) return PKV_ERR_INVALID_ARG;
  pkv_attend_options o{};
  if (options_or_null) o = *options_or_null;
  if (!std::isfinite(o.scale) || !std::isfinite(o.softcap) || o.softcap < 0.f || o.window < 0) return PKV_ERR_INVALID_ARG;
  if (!o.q_positions && (o.slopes || o.window > 0 || o.prefix != 0)) return PKV_ERR_INVALID_ARG;
  if (o.q_positions && !cache->positions) return PKV_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(o.slopes) % 4 || reinterpret_cast<uintptr_t>(o.q_positions) % 4) return PKV_ERR_INVALID_ARG;
  CacheWorkspace w;
  if (const int st = cache_workspace(cfg, cache, workspace, workspace_bytes, &w)) return st;
  CacheAttendParams p{};
  p.q = q.ptr;
  p.q_sb = q.stride_batch;
  p.q_sh = q.stride_head;
  p.k_pool = cache->k_pool;
  p.v_pool = cache->v_pool;
  p.pos_pool = cache->positions;
  p.table = cache->tables + static_cast<int64_t>(layer) * cache->batch * cfg->num_kv_heads * cache->max_pages;
  p.lens = cache->lens + static_cast<int64_t>(layer) * cache->batch;
  p.q_pos = o.q_positions;
  p.slopes = o.slopes;
  p.out = out;
  p.lse = lse_or_null;
  p.status = w.status;
  p.counters = w.counters;
  p.group_counters = w.group_counters;
  p.partials = w.partials;
  p.batch = cache->batch;
  p.num_kv_heads = cfg->num_kv_heads;
  p.group = cfg->num_q_heads / cfg->num_kv_heads;
  p.head_blocks = head_blocks(cfg);
  p.max_pages = cache->max_pages;
  p.page_size = cache->page_size;
  p.num_pages = cache->num_pages;
  p.page_shift = -1;
  for (int i = 0; i < 31; ++i)
    if (cache->page_size == 1 << i) p.page_shift = i;
  p.window = o.window;
  p.prefix = o.prefix;
  const double log2e = 1.4426950408889634, scale = o.scale == 0.f ? 1.0 / std::sqrt(static_cast<double>(cfg->head_dim)) : o.scale;
  p.cap_log2 = static_cast<float>(o.softcap * log2e);
  p.scale_log2 = static_cast<float>(o.softcap > 0.f ? scale / o.softcap : scale * log2e);
  if (!std::isfinite(p.cap_log2) || !std::isfinite(p.scale_log2)) return PKV_ERR_INVALID_ARG;  // a cap too close to zero for fp32
  const int gt = heads_per_cta(cfg);
  const bool wide = cfg->head_dim == 128;
  const int64_t rows = static_cast<int64_t>(cache->max_pages) * cache->page_size;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  switch (cfg->dtype) {
    case PKV_DTYPE_FP32: return wide ? dispatch_cache_attend<float, 128>(p, gt, rows, st) : dispatch_cache_attend<float, 64>(p, gt, rows, st);
    case PKV_DTYPE_FP16: return wide ? dispatch_cache_attend<__half, 128>(p, gt, rows, st) : dispatch_cache_attend<__half, 64>(p, gt, rows, st);
    default:
      return wide ? dispatch_cache_attend<__nv_bfloat16, 128>(p, gt, rows, st) : dispatch_cache_attend<__nv_bfloat16, 64>(p, gt, rows, st);
  }
}

int pyramidkv_cache_fork(const pkv_config* cfg, const pkv_cache* from, const pkv_cache* to, const int32_t* parents, const int32_t* add_or_null,
                         int64_t add_stride, int32_t* granted_or_null, void* workspace, size_t workspace_bytes, void* stream) {
  PagesParams p;
  if (!pointer_ok(parents, 4) || reinterpret_cast<uintptr_t>(add_or_null) % 4 || reinterpret_cast<uintptr_t>(granted_or_null) % 4) return PKV_ERR_INVALID_ARG;
  if (const int st = pages_setup(cfg, from, to, workspace, workspace_bytes, &p)) return st;
  p.parents = parents;
  p.add = add_or_null;
  p.add_stride = add_stride;
  p.granted = granted_or_null;
  return run_fork(cfg, from, to, p, static_cast<cudaStream_t>(stream));
}

int pyramidkv_cache_reserve(const pkv_config* cfg, const pkv_cache* from, const pkv_cache* to, const int32_t* add, int64_t add_stride,
                            int32_t* granted_or_null, void* workspace, size_t workspace_bytes, void* stream) {
  PagesParams p;
  if (!pointer_ok(add, 4) || reinterpret_cast<uintptr_t>(granted_or_null) % 4) return PKV_ERR_INVALID_ARG;
  if (const int st = pages_setup(cfg, from, to, workspace, workspace_bytes, &p)) return st;
  if (from->batch != to->batch) return PKV_ERR_INVALID_ARG;
  p.add = add;
  p.add_stride = add_stride;
  p.granted = granted_or_null;
  return run_fork(cfg, from, to, p, static_cast<cudaStream_t>(stream));
}

int pyramidkv_cache_compact(const pkv_config* cfg, const pkv_cache* from, const pkv_cache* to, int32_t* used_or_null, void* workspace,
                            size_t workspace_bytes, void* stream) {
  PagesParams p;
  if (reinterpret_cast<uintptr_t>(used_or_null) % 4) return PKV_ERR_INVALID_ARG;
  if (const int st = pages_setup(cfg, from, to, workspace, workspace_bytes, &p)) return st;
  if (from->batch != to->batch) return PKV_ERR_INVALID_ARG;
  p.used = used_or_null;
  const int sms = device_sm_count();
  if (sms <= 0) return PKV_ERR_CUDA;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (const int rc = launch_cluster(pages_pair_kernel, p, st)) return rc;
  const int64_t units = static_cast<int64_t>(p.layers) * p.from_batch;
  launch_pdl(pages_move_kernel, dim3(stride_grid(std::max<int64_t>(p.num_pages / 2, units), 1, sms, 16)), dim3(kPgCopyThreads), 0, st, p);
  note_outputs(st, {{from->k_pool, pool_bytes(cfg, from)}, {from->v_pool, pool_bytes(cfg, from)}});
  return check_launch();
}

}  // extern "C"
