// Rotary positions on queries and keys, and the append of a growing cache's new rows (rotary positions on the way).
//
// A pair (x, y) of a row at position p is turned by the angle p f: x' = m (x cos - y sin), y' = m (y cos + x sin).  Nothing is
// summed, so the floor is one read and one write of every row.
//   * A thread owns a unit of a row, two pieces of VEC elements: VEC pairs in the half layout (a piece of either half), VEC
//     pairs in the interleaved one (2 VEC elements in a row).  Its sines serve every head of its token.
//   * The angle is formed in turns and in fp64, p * (f / 2 pi), and loses its whole turns there: in fp32 a position of 100000
//     would leave an error of 4e-3 rad.  sincospif then sees at most half a turn.
//   * VEC elements make 16 bytes where the pieces of the rotated part start at multiples of 16 bytes; a rotated part of another
//     size is taken pair by pair (VEC = 1).
#pragma once

#include "pkv_common.cuh"

namespace pkv {

constexpr int kRotThreads = 256;
constexpr int kRotUnroll = 4;              // heads whose rows a thread has on their way at a time

struct RotaryParams {
  TensorView q, q_out, k, k_out, v;        // k_out: not used by an append, its keys go into pages
  const int32_t* positions;                // null: everything at position 0 (no plan, no positions)
  int64_t positions_stride;
  int32_t batch, tokens;
  int32_t heads_q, heads_kv;               // 0 where a tensor is not given
  int32_t units, rot_units;                // units of a row; those of the rotated part
  int32_t unit_lanes, head_lanes;          // threads of a block: unit, then head, then token; powers of two
  int32_t half;                            // rotary_dim / 2
  int32_t interleaved;
  float magnitude_cos, magnitude_sin;      // the factor on cosines and on sines (negative angles: its negative)
  // append
  const int32_t* counts;                   // or null
  const int32_t* lens;                     // of the layer
  const int32_t* table;
  int32_t max_pages, page_size, num_pages;
  void* k_pool;
  void* v_pool;
  int32_t* pos_pool;                       // or null
  uint32_t* status;
  double turns[64];                        // per position, of each pair
};

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) RotPiece {
  T x[VEC];
};

// grid (ceil(tokens of the batch / tokens of a block), head splits).
template <typename T, int VEC, bool APPEND>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const __grid_constant__ RotaryParams p) {
  using Piece = RotPiece<T, VEC>;
  __shared__ double s_turns[64];
  pdl_trigger();
  if (threadIdx.x < 64) s_turns[threadIdx.x] = p.turns[threadIdx.x];
  __syncthreads();
  const int u = threadIdx.x % p.unit_lanes, hl = threadIdx.x / p.unit_lanes % p.head_lanes;
  const int block_tokens = kRotThreads / (p.unit_lanes * p.head_lanes);
  const int64_t token = static_cast<int64_t>(blockIdx.x) * block_tokens + threadIdx.x / (p.unit_lanes * p.head_lanes);
  if (token >= static_cast<int64_t>(p.batch) * p.tokens) return;
  const int b = static_cast<int>(token / p.tokens), t = static_cast<int>(token - static_cast<int64_t>(b) * p.tokens);
  pdl_wait();
  int page_at = 0, slot_in_page = 0;
  bool inside = true;
  if (APPEND) {
    const int count = p.counts ? min(max(__ldg(p.counts + b), 0), p.tokens) : p.tokens;
    if (t >= count) return;
    const int64_t row = static_cast<int64_t>(__ldg(p.lens + b)) - count + t;
    inside = row >= 0 && row < static_cast<int64_t>(p.max_pages) * p.page_size;
    page_at = inside ? static_cast<int>(row / p.page_size) : 0;
    slot_in_page = inside ? static_cast<int>(row - static_cast<int64_t>(page_at) * p.page_size) : 0;
  }
  const int pos = p.positions ? __ldg(p.positions + b * p.positions_stride + t) : 0;
  const bool rotated = u < p.rot_units;
  float cs[VEC], sn[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    cs[i] = 1.f;
    sn[i] = 0.f;
    if (rotated) {
      double turn = static_cast<double>(pos) * s_turns[u * VEC + i];
      turn -= rint(turn);
      sincospif(2.f * static_cast<float>(turn), &sn[i], &cs[i]);
      cs[i] *= p.magnitude_cos;
      sn[i] *= p.magnitude_sin;
    }
  }
  // elements at which the unit's two pieces start
  const int r = 2 * p.half;
  const int e0 = !rotated ? r + (u - p.rot_units) * 2 * VEC : (p.interleaved ? u * 2 * VEC : u * VEC);
  const int e1 = rotated && !p.interleaved ? p.half + u * VEC : e0 + VEC;

  const int heads = p.heads_q + p.heads_kv * (APPEND ? 2 : 1);
  const int step = gridDim.y * p.head_lanes;
  for (int h0 = blockIdx.y * p.head_lanes + hl; h0 < heads; h0 += step * kRotUnroll) {
    Piece a[kRotUnroll], c[kRotUnroll];
    T* to[kRotUnroll];
#pragma unroll
    for (int i = 0; i < kRotUnroll; ++i) {
      const int h = h0 + i * step;
      to[i] = nullptr;
      if (h >= heads) continue;
      const bool is_q = h < p.heads_q, is_v = APPEND && h >= p.heads_q + p.heads_kv;
      const int hh = is_q ? h : (is_v ? h - p.heads_q - p.heads_kv : h - p.heads_q);
      const TensorView& in = is_q ? p.q : (is_v ? p.v : p.k);
      const T* from = static_cast<const T*>(in.ptr) + b * in.sb + hh * in.sh + t * in.st;
      if (APPEND && !is_q) {
        const int page = inside ? __ldg(p.table + (static_cast<int64_t>(b) * p.heads_kv + hh) * p.max_pages + page_at) : -1;
        if (page < 0 || page >= p.num_pages) {
          if (u == 0) atomicOr(p.status, kStatusBadPage);
          continue;
        }
        const int64_t slot = static_cast<int64_t>(page) * p.page_size + slot_in_page;
        to[i] = static_cast<T*>(is_v ? p.v_pool : p.k_pool) + slot * (p.units * 2 * VEC);
        if (!is_v && u == 0 && p.pos_pool) p.pos_pool[slot] = pos;
      } else {
        const TensorView& out = is_q ? p.q_out : p.k_out;
        to[i] = static_cast<T*>(const_cast<void*>(out.ptr)) + b * out.sb + hh * out.sh + t * out.st;
        if (to[i] == from && !rotated) { to[i] = nullptr; continue; }         // in place, not part of the rotation
      }
      a[i] = *reinterpret_cast<const Piece*>(from + (is_v ? u * 2 * VEC : e0));
      c[i] = *reinterpret_cast<const Piece*>(from + (is_v ? u * 2 * VEC + VEC : e1));
    }
#pragma unroll
    for (int i = 0; i < kRotUnroll; ++i) {
      if (!to[i]) continue;
      const bool is_v = APPEND && h0 + i * step >= p.heads_q + p.heads_kv;
      if (rotated && !is_v) {
        if (VEC == 1 || !p.interleaved) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float x = to_float(a[i].x[e]), y = to_float(c[i].x[e]);
            a[i].x[e] = from_float<T>(fmaf(x, cs[e], -(y * sn[e])));
            c[i].x[e] = from_float<T>(fmaf(y, cs[e], x * sn[e]));
          }
        } else {
#pragma unroll
          for (int e = 0; e + 1 < VEC; e += 2) {
            const float x = to_float(a[i].x[e]), y = to_float(a[i].x[e + 1]);
            a[i].x[e] = from_float<T>(fmaf(x, cs[e / 2], -(y * sn[e / 2])));
            a[i].x[e + 1] = from_float<T>(fmaf(y, cs[e / 2], x * sn[e / 2]));
            const float z = to_float(c[i].x[e]), w = to_float(c[i].x[e + 1]);
            c[i].x[e] = from_float<T>(fmaf(z, cs[VEC / 2 + e / 2], -(w * sn[VEC / 2 + e / 2])));
            c[i].x[e + 1] = from_float<T>(fmaf(w, cs[VEC / 2 + e / 2], z * sn[VEC / 2 + e / 2]));
          }
        }
      }
      *reinterpret_cast<Piece*>(to[i] + (is_v ? u * 2 * VEC : e0)) = a[i];
      *reinterpret_cast<Piece*>(to[i] + (is_v ? u * 2 * VEC + VEC : e1)) = c[i];
    }
  }
}

}  // namespace pkv
