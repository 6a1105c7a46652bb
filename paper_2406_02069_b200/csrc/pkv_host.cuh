// Host helpers that the files behind the C boundary share: checks of configurations and tensors, launches, the record of
// outputs still in flight, the number of SMs.
#pragma once

#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <initializer_list>
#include <mutex>
#include <utility>

#include "pkv_common.cuh"

namespace pkv {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

inline bool config_ok(const pkv_config* c) {
  if (!c) return false;
  if (c->num_layers < 1 || c->num_kv_heads < 1 || c->num_q_heads < 1) return false;
  if (c->num_q_heads % c->num_kv_heads != 0) return false;
  if (c->window < 1 || c->avg_budget < c->window) return false;
  if (c->pool_kernel < 1 || (c->pool_kernel % 2) == 0) return false;
  if (!(c->beta >= 1.0) || c->beta > 1.0e6) return false;
  if (c->schedule != PKV_SCHEDULE_LINEAR && c->schedule != PKV_SCHEDULE_GEOMETRIC) return false;
  if ((c->flags & ~PKV_FLAG_INPUTS_FINAL) != 0 || c->sweep_ctas > 1024) return false;
  return true;
}

inline int config_supported(const pkv_config* c) {
  if (c->dtype != PKV_DTYPE_FP32 && c->dtype != PKV_DTYPE_BF16 && c->dtype != PKV_DTYPE_FP16)
    return PKV_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return PKV_ERR_UNSUPPORTED;
  if (c->pool_kind != PKV_POOL_MAX && c->pool_kind != PKV_POOL_AVG) return PKV_ERR_UNSUPPORTED;
  return PKV_OK;
}

// A [batch][heads][token][d] view the kernels can take: 16-byte aligned base and strides, rows that do not
// overlap, and a positive stride along every dimension that has more than one entry (a broadcast or reversed
// view has no tensor map and would be mis-sized by the overlap test below).
inline bool tensor_ok(const pkv_tensor& t, int d, int elem_bytes, int batch = 1, int heads = 1) {
  if (!t.ptr || t.stride_token < d) return false;
  if (reinterpret_cast<uintptr_t>(t.ptr) % 16) return false;
  if ((batch > 1 && t.stride_batch <= 0) || (heads > 1 && t.stride_head <= 0)) return false;
  const int64_t q = 16 / elem_bytes;
  return t.stride_token % q == 0 && t.stride_head % q == 0 && t.stride_batch % q == 0;
}

inline TensorView view(const pkv_tensor& t) { return TensorView{t.ptr, t.stride_batch, t.stride_head, t.stride_token}; }

inline int check_launch() { return cudaPeekAtLastError() == cudaSuccess ? PKV_OK : PKV_ERR_CUDA; }

// ---------------------------------------------------------------- outputs still in flight
// The tensor-core sweeps start reading Q and K before the kernels ahead of them in the stream have finished.
// That is only right for tensors those kernels do not write, so the library remembers where its calls put K/V rows (packed
// caches, page pools, rotated keys and queries) and a sweep whose Q or K overlaps one of them waits like any other kernel.
//   How long: a kernel starts when all CTAs of the one ahead in its stream have started, and every kernel of the library stays
// until the one ahead of it has finished.  So whatever is between a kernel that still writes and a sweep is on the device with
// both, and a device holds kResidentGrids grids: what has as many launches behind it in its own stream is complete.  Every stream has
// ranges of its own, since launches on another one say nothing about it; a sweep looks at all of them.
//   A range that is written again is taken once, by its last writer; ranges whose stream makes room for another one (more than
// kOutStreams of them) stay for good, as parts of one range.
constexpr unsigned kResidentGrids = 128;   // compute capability 10.0
constexpr int kOutRanges = 3 * kResidentGrids;                  // no launch has more than three outputs
constexpr int kOutStreams = 64;

struct Output { const void* ptr; size_t bytes; };

struct OutputRecord {
  struct Range { uintptr_t lo, hi; uint64_t at; };              // at: launches of the stream when it was written
  struct Stream {
    cudaStream_t stream;
    int device;
    uint64_t thread;                       // of the per-thread stream, whose handle is the same in all threads
    uint64_t launches, used;
    int count;
    Range range[kOutRanges];
    bool live(const Range& r) const { return launches - r.at < kResidentGrids; }
  };
  std::mutex mutex;
  Stream streams[kOutStreams];
  int known = 0;
  uint64_t clock = 0;
  Range rest = {};                         // hi 0: none

  static uint64_t this_thread() {
    static std::atomic<uint64_t> next{1};
    static thread_local const uint64_t id = next.fetch_add(1);
    return id;
  }
  void stays(const Range& r) {
    rest.lo = rest.hi ? std::min(rest.lo, r.lo) : r.lo;
    rest.hi = std::max(rest.hi, r.hi);
  }
  Stream& of(cudaStream_t st) {
    int dev = -1;                          // only the default streams have the same handles on all devices
    if (reinterpret_cast<uintptr_t>(st) <= reinterpret_cast<uintptr_t>(cudaStreamPerThread) && cudaGetDevice(&dev) != cudaSuccess) dev = -1;
    const uint64_t thread = st == cudaStreamPerThread ? this_thread() : 0;
    ++clock;
    Stream* oldest = streams;
    for (int i = 0; i < known; ++i) {
      Stream& s = streams[i];
      if (s.stream == st && s.device == dev && s.thread == thread) {
        s.used = clock;
        return s;
      }
      if (s.used < oldest->used) oldest = &s;
    }
    Stream& s = known < kOutStreams ? streams[known++] : *oldest;
    for (int i = 0; i < s.count; ++i)
      if (s.live(s.range[i])) stays(s.range[i]);
    s.stream = st;
    s.device = dev;
    s.thread = thread;
    s.launches = 0;
    s.used = clock;
    s.count = 0;
    return s;
  }
  void launched(cudaStream_t st) {
    std::lock_guard<std::mutex> lock(mutex);
    ++of(st).launches;
  }
  void wrote(cudaStream_t st, std::initializer_list<Output> outputs) {
    std::lock_guard<std::mutex> lock(mutex);
    Stream& s = of(st);
    for (const Output& o : outputs)
      if (o.ptr && o.bytes) wrote(s, reinterpret_cast<uintptr_t>(o.ptr), reinterpret_cast<uintptr_t>(o.ptr) + o.bytes);
  }
  void wrote(Stream& s, uintptr_t lo, uintptr_t hi) {
    int n = 0;
    for (int i = 0; i < s.count; ++i) {    // what is complete goes, and what this range takes in
      const Range r = s.range[i];
      if (s.live(r) && !(lo <= r.lo && r.hi <= hi)) s.range[n++] = r;
    }
    if (n == kOutRanges) stays(s.range[--n]);
    s.range[n] = Range{lo, hi, s.launches};
    s.count = n + 1;
  }
  bool overlaps(uintptr_t lo, uintptr_t hi) {
    std::lock_guard<std::mutex> lock(mutex);
    if (lo < rest.hi && rest.lo < hi) return true;
    for (int i = 0; i < known; ++i)
      for (int j = 0; j < streams[i].count; ++j) {
        const Range& r = streams[i].range[j];
        if (lo < r.hi && r.lo < hi && streams[i].live(r)) return true;
      }
    return false;
  }
};
inline OutputRecord g_outputs;

inline void note_launch(cudaStream_t st) { g_outputs.launched(st); }
inline void note_outputs(cudaStream_t st, std::initializer_list<Output> outputs) { g_outputs.wrote(st, outputs); }

inline bool overlaps_recent_output(const pkv_tensor& t, int batch, int heads, int tokens, int d, int elem_bytes) {
  const int64_t last = (batch - 1) * std::max<int64_t>(t.stride_batch, 0) +
                       (heads - 1) * std::max<int64_t>(t.stride_head, 0) + (tokens - 1) * t.stride_token + d;
  const uintptr_t lo = reinterpret_cast<uintptr_t>(t.ptr), hi = lo + static_cast<uintptr_t>(last) * elem_bytes;
  return g_outputs.overlaps(lo, hi);
}

// Launch with programmatic stream serialisation: the kernel may be scheduled while its predecessor in
// the stream drains; the kernels order themselves with pdl_wait() (pkv_common.cuh).
template <typename... KArgs, typename... Args>
void launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...) == cudaSuccess) note_launch(st);
}

// SMs the persistent score kernels may count on: the device's, or fewer while a call runs them on a lane that
// owns only a group of the SMs (pyramidkv_compress_model_lanes sets the limit for its own thread).
inline thread_local int tl_sm_limit = 0;

inline int device_sm_count() {
  static int sms[64] = {};
  if (tl_sm_limit > 0) return tl_sm_limit;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  if (!sms[dev]) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    sms[dev] = n;
  }
  return sms[dev];
}

}  // namespace pkv
