// Host helpers that the files behind the C boundary share: checks of configurations and tensors, launches, the record of
// outputs still in flight, the number of SMs.
#pragma once

#include <cuda_runtime.h>

#include <algorithm>
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
  cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

// ---------------------------------------------------------------- outputs still in flight
// The tensor-core sweeps start reading Q and K before the kernels ahead of them in the stream have finished.
// That is only right for tensors those kernels do not write, so the library remembers where its last calls put
// K/V rows (packed caches, page pools, rotated keys and queries) and a sweep whose Q or K overlaps one of them waits like any other kernel.
struct ByteRange { uintptr_t lo, hi; };
inline std::mutex g_out_mutex;
constexpr unsigned kRecentOut = 256;       // a kernel can wait behind as many as fit on the device at once
inline ByteRange g_recent_out[kRecentOut];
inline unsigned g_recent_out_next = 0;

inline void note_output(const void* ptr, size_t bytes) {
  if (!ptr || !bytes) return;
  std::lock_guard<std::mutex> lock(g_out_mutex);
  const uintptr_t lo = reinterpret_cast<uintptr_t>(ptr);
  g_recent_out[g_recent_out_next++ % kRecentOut] = ByteRange{lo, lo + bytes};
}

inline bool overlaps_recent_output(const pkv_tensor& t, int batch, int heads, int tokens, int d, int elem_bytes) {
  const int64_t last = (batch - 1) * std::max<int64_t>(t.stride_batch, 0) +
                       (heads - 1) * std::max<int64_t>(t.stride_head, 0) + (tokens - 1) * t.stride_token + d;
  const uintptr_t lo = reinterpret_cast<uintptr_t>(t.ptr), hi = lo + static_cast<uintptr_t>(last) * elem_bytes;
  std::lock_guard<std::mutex> lock(g_out_mutex);
  for (const ByteRange& r : g_recent_out)
    if (r.hi > r.lo && lo < r.hi && r.lo < hi) return true;
  return false;
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
