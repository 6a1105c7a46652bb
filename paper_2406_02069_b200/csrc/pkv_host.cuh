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
// Launches that are captured into a graph run later, and a graph's start waits for all that is ahead of it in the stream as
// what follows waits for its end: a capture keeps a record of its own, and only its own sweeps look at it.
//   A range that is written again is taken once, by its last writer; ranges whose stream makes room for another one (more than
// kOutStreams of them) stay for good, as parts of one range.
constexpr unsigned kResidentGrids = 128;   // compute capability 10.0
constexpr int kOutRanges = 3 * kResidentGrids;                  // no launch has more than three outputs
constexpr int kOutStreams = 64;

struct Output { const void* ptr; size_t bytes; };

struct StreamKey {
  cudaStream_t stream;
  int device;                              // of a default stream, whose handle is the same on all devices
  uint64_t thread;                         // of the per-thread one, whose handle is the same in all threads
  uint64_t capture;                        // 0: not being captured
};

inline StreamKey stream_key(cudaStream_t st) {
  static std::atomic<uint64_t> next_thread{1};
  static thread_local const uint64_t this_thread = next_thread.fetch_add(1);
  StreamKey k{st, -1, st == cudaStreamPerThread ? this_thread : 0, 0};
  if (reinterpret_cast<uintptr_t>(st) <= reinterpret_cast<uintptr_t>(cudaStreamPerThread) && cudaGetDevice(&k.device) != cudaSuccess) k.device = -1;
  if (st && st != cudaStreamLegacy) {      // (that one cannot be captured)
    cudaStreamCaptureStatus status;
    unsigned long long id = 0;
    if (cudaStreamGetCaptureInfo(st, &status, &id) == cudaSuccess && status == cudaStreamCaptureStatusActive) k.capture = id;
  }
  return k;
}

struct OutputRecord {
  struct Range { uintptr_t lo, hi; uint64_t at; };              // at: launches of the stream when it was written
  struct Stream {
    StreamKey key;
    uint64_t launches, used;
    int count;
    Range range[kOutRanges];
    bool live(const Range& r) const { return launches - r.at < kResidentGrids; }
  };
  std::mutex mutex;
  Stream streams[kOutStreams];
  int known = 0;
  uint64_t clock = 0;
  Range rest[2] = {};                      // without and with a capture; hi 0: none

  void stays(const Stream& s, const Range& r) {
    Range& to = rest[s.key.capture != 0];
    to.lo = to.hi ? std::min(to.lo, r.lo) : r.lo;
    to.hi = std::max(to.hi, r.hi);
  }
  Stream& of(const StreamKey& k) {
    ++clock;
    Stream* at = nullptr;
    Stream* oldest = streams;
    for (int i = 0; i < known && !at; ++i) {
      Stream& s = streams[i];
      if (s.key.stream == k.stream && s.key.device == k.device && s.key.thread == k.thread && !s.key.capture == !k.capture) {
        if (s.key.capture == k.capture) {
          s.used = clock;
          return s;
        }
        at = &s;                           // a stream is in one capture at a time: the one ahead has ended
      }
      if (s.used < oldest->used) oldest = &s;
    }
    if (!at) {
      at = known < kOutStreams ? &streams[known++] : oldest;
      for (int i = 0; i < at->count; ++i)
        if (at->live(at->range[i])) stays(*at, at->range[i]);
    }
    at->key = k;
    at->launches = 0;
    at->used = clock;
    at->count = 0;
    return *at;
  }
  void launched(const StreamKey& k) {
    std::lock_guard<std::mutex> lock(mutex);
    ++of(k).launches;
  }
  // launches: of those that wrote, how many have not been counted
  void wrote(const StreamKey& k, std::initializer_list<Output> outputs, int launches = 0) {
    std::lock_guard<std::mutex> lock(mutex);
    Stream& s = of(k);
    s.launches += launches;
    for (const Output& o : outputs)
      if (o.ptr && o.bytes) wrote(s, reinterpret_cast<uintptr_t>(o.ptr), reinterpret_cast<uintptr_t>(o.ptr) + o.bytes);
  }
  void wrote(Stream& s, uintptr_t lo, uintptr_t hi) {
    int n = 0;
    for (int i = 0; i < s.count; ++i) {    // what is complete goes, and what this range takes in
      const Range r = s.range[i];
      if (s.live(r) && !(lo <= r.lo && r.hi <= hi)) s.range[n++] = r;
    }
    if (n == kOutRanges) stays(s, s.range[--n]);
    s.range[n] = Range{lo, hi, s.launches};
    s.count = n + 1;
  }
  bool overlaps(uint64_t capture, uintptr_t lo, uintptr_t hi) {
    std::lock_guard<std::mutex> lock(mutex);
    const Range& kept = rest[capture != 0];
    if (lo < kept.hi && kept.lo < hi) return true;
    for (int i = 0; i < known; ++i) {
      const Stream& s = streams[i];
      if (s.key.capture != capture) continue;
      for (int j = 0; j < s.count; ++j)
        if (lo < s.range[j].hi && s.range[j].lo < hi && s.live(s.range[j])) return true;
    }
    return false;
  }
};
inline OutputRecord g_outputs;

inline void note_launch(cudaStream_t st) { g_outputs.launched(stream_key(st)); }
inline void note_outputs(cudaStream_t st, std::initializer_list<Output> outputs, int launches = 0) { g_outputs.wrote(stream_key(st), outputs, launches); }

// Whether a call on stream st may find an output in flight in a tensor.
inline bool overlaps_recent_output(const pkv_tensor& t, int batch, int heads, int tokens, int d, int elem_bytes, cudaStream_t st) {
  const int64_t last = (batch - 1) * std::max<int64_t>(t.stride_batch, 0) +
                       (heads - 1) * std::max<int64_t>(t.stride_head, 0) + (tokens - 1) * t.stride_token + d;
  const uintptr_t lo = reinterpret_cast<uintptr_t>(t.ptr), hi = lo + static_cast<uintptr_t>(last) * elem_bytes;
  return g_outputs.overlaps(stream_key(st).capture, lo, hi);
}

// Launch with programmatic stream serialisation: the kernel may be scheduled while its predecessor in
// the stream drains; the kernels order themselves with pdl_wait() (pkv_common.cuh).
template <typename... KArgs, typename... Args>
bool launch_uncounted(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
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
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...) == cudaSuccess;
}
template <typename... KArgs, typename... Args>
void launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
  if (launch_uncounted(kernel, grid, block, smem, st, std::forward<Args>(args)...)) note_launch(st);
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
