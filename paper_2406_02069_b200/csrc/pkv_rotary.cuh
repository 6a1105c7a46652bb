// Rotary positions on queries and keys, and the append of a growing cache's new rows (rotary positions on the way).
//
// A pair (x, y) of a row at position p is turned by the angle p f: x' = m (x cos - y sin), y' = m (y cos + x sin).  Nothing is
// summed, so the floor is one read and one write of every row.
//   * A thread owns a unit of a row, two pieces of VEC elements: VEC pairs in the half layout (a piece of either half), VEC
//     pairs in the interleaved one (2 VEC elements in a row).  Its sines serve every head of its token.
//   * The angle is formed in turns and in fp64, p * (f / 2 pi), and loses its whole turns there: in fp32 a position of 100000
//     would leave an error of 4e-3 rad.  sincospif then sees at most half a turn.
//   * VEC elements make 16 bytes where the pieces of the rotated part start at multiples of 16 bytes; a rotated part of another
//     size is taken two pairs at a time (8192 tokens of 40 heads, 20 of 128 elements rotated: 44 us, 59 % of the rate of a copy), or
//     pair by pair (18 of 128: 64 us, 40 %).
//   * 16-bit elements are taken apart and put together two to a word (one by one: 185 us for 32 / 8 heads x 32768 tokens, this way
//     105, 98 % of the rate of a copy; in fp32 206, 99 %).  The rows come while the sines are formed, and while the page tables are read.
#pragma once

#include "pkv_common.cuh"
#include "pkv_mma16.cuh"

namespace pkv {

constexpr int kRotThreads = 256;
// Heads whose rows a thread has on their way at a time, and CTAs that an SM shall hold.  32 / 8 heads x 32768 tokens in bf16: two
// and four 109 us, four and two 118, one and four 118, two and two 132.  An append of 2000 rows in pieces: four and two 13.4 us,
// two and three 15.7, two and four 18.7 (its look-ups need the registers).
template <int VEC, bool APPEND>
constexpr int kRotUnroll = VEC > 2 && !APPEND ? 2 : 4;
template <int VEC, bool APPEND>
constexpr int kRotPerSm = VEC > 2 && !APPEND ? 4 : 2;

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

// VEC elements of a row, and the rotation of two of them (half layout: x and y of VEC pairs; interleaved: VEC / 2 pairs each).
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) RotPiece {
  T x[VEC];
};

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ void rot_pair(float& x, float& y, float c, float s) {
  const float t = fmaf(x, c, -(y * s));
  y = fmaf(y, c, x * s);
  x = t;
}

template <typename T, int VEC>
__device__ __forceinline__ void rot_pieces(RotPiece<T, VEC>& a, RotPiece<T, VEC>& b, const float (&cs)[VEC], const float (&sn)[VEC], bool interleaved) {
  if constexpr (sizeof(T) == 2 && VEC > 1) {                     // two elements to a word
    uint32_t* aw = reinterpret_cast<uint32_t*>(&a);
    uint32_t* bw = reinterpret_cast<uint32_t*>(&b);
#pragma unroll
    for (int w = 0; w < VEC / 2; ++w) {
      float2 x = Dec16<T>::unpack(aw[w]), y = Dec16<T>::unpack(bw[w]);
      if (interleaved) {
        rot_pair(x.x, x.y, cs[w], sn[w]);
        rot_pair(y.x, y.y, cs[VEC / 2 + w], sn[VEC / 2 + w]);
      } else {
        rot_pair(x.x, y.x, cs[2 * w], sn[2 * w]);
        rot_pair(x.y, y.y, cs[2 * w + 1], sn[2 * w + 1]);
      }
      aw[w] = Dec16<T>::pack(x.x, x.y);
      bw[w] = Dec16<T>::pack(y.x, y.y);
    }
  } else if constexpr (VEC > 1) {
    if (interleaved) {
#pragma unroll
      for (int e = 0; e < VEC / 2; ++e) {
        rot_pair(a.x[2 * e], a.x[2 * e + 1], cs[e], sn[e]);
        rot_pair(b.x[2 * e], b.x[2 * e + 1], cs[VEC / 2 + e], sn[VEC / 2 + e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) rot_pair(a.x[e], b.x[e], cs[e], sn[e]);
    }
  } else {
    float x = to_float(a.x[0]), y = to_float(b.x[0]);
    rot_pair(x, y, cs[0], sn[0]);
    a.x[0] = from_float<T>(x);
    b.x[0] = from_float<T>(y);
  }
}

// grid (ceil(tokens of the batch / tokens of a block), head splits).
template <typename T, int VEC, bool APPEND>
__global__ void __launch_bounds__(kRotThreads, kRotPerSm<VEC, APPEND>) rotary_kernel(const __grid_constant__ RotaryParams p) {
  using Piece = RotPiece<T, VEC>;
  constexpr int UNROLL = kRotUnroll<VEC, APPEND>;
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
    const int count = p.counts ? min(max(p.counts[b], 0), p.tokens) : p.tokens;
    if (t >= count) return;
    const int64_t row = static_cast<int64_t>(p.lens[b]) - count + t;
    inside = row >= 0 && row < static_cast<int64_t>(p.max_pages) * p.page_size;
    page_at = inside ? static_cast<int>(row / p.page_size) : 0;
    slot_in_page = inside ? static_cast<int>(row - static_cast<int64_t>(page_at) * p.page_size) : 0;
  }
  const int pos = p.positions ? p.positions[b * p.positions_stride + t] : 0;
  const bool rotated = u < p.rot_units;
  // elements at which the unit's two pieces start
  const int r = 2 * p.half;
  const int e0 = !rotated ? r + (u - p.rot_units) * 2 * VEC : (p.interleaved ? u * 2 * VEC : u * VEC);
  const int e1 = rotated && !p.interleaved ? p.half + u * VEC : e0 + VEC;

  const int heads = p.heads_q + p.heads_kv * (APPEND ? 2 : 1);
  const int step = gridDim.y * p.head_lanes;
  const T* q_in = static_cast<const T*>(p.q.ptr) + b * p.q.sb + t * p.q.st;
  const T* k_in = static_cast<const T*>(p.k.ptr) + b * p.k.sb + t * p.k.st;
  const T* v_in = static_cast<const T*>(p.v.ptr) + b * p.v.sb + t * p.v.st;
  T* q_to = static_cast<T*>(const_cast<void*>(p.q_out.ptr)) + b * p.q_out.sb + t * p.q_out.st;
  T* k_to = static_cast<T*>(const_cast<void*>(p.k_out.ptr)) + b * p.k_out.sb + t * p.k_out.st;
  Piece a[UNROLL], c[UNROLL];
  int page[UNROLL];                        // of a key or value that is appended
  // What a head index stands for: a query's, a key's or a value's head.
  auto is_query = [&](int h) { return h < p.heads_q; };
  auto is_value = [&](int h) { return APPEND && h >= p.heads_q + p.heads_kv; };
  auto number = [&](int h) { return is_query(h) ? h : (is_value(h) ? h - p.heads_q - p.heads_kv : h - p.heads_q); };
  auto source = [&](int h) -> const T* {
    return is_query(h) ? q_in + number(h) * p.q.sh : (is_value(h) ? v_in + number(h) * p.v.sh : k_in + number(h) * p.k.sh);
  };
  // Rows of the heads h0, h0 + step .. on their way to a and c, their pages beside them.
  auto fetch = [&](int h0) {
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      const int h = h0 + i * step;
      if (h >= heads) continue;
      const T* from = source(h);
      const bool is_v = is_value(h);
      a[i] = *reinterpret_cast<const Piece*>(from + (is_v ? u * 2 * VEC : e0));
      c[i] = *reinterpret_cast<const Piece*>(from + (is_v ? u * 2 * VEC + VEC : e1));
      if (APPEND && !is_query(h))
        page[i] = inside ? p.table[(static_cast<int64_t>(b) * p.heads_kv + number(h)) * p.max_pages + page_at] : -1;
    }
  };
  const int first = blockIdx.y * p.head_lanes + hl;
  fetch(first);                            // (the sines are formed while they come)
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
  for (int h0 = first; h0 < heads;) {
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      const int h = h0 + i * step;
      if (h >= heads) continue;
      const bool is_v = is_value(h);
      T* to;
      if (APPEND && !is_query(h)) {
        if (page[i] < 0 || page[i] >= p.num_pages) {
          if (u == 0) atomicOr(p.status, kStatusBadPage);
          continue;
        }
        const int64_t slot = static_cast<int64_t>(page[i]) * p.page_size + slot_in_page;
        to = static_cast<T*>(is_v ? p.v_pool : p.k_pool) + slot * (p.units * 2 * VEC);
        if (!is_v && u == 0 && p.pos_pool) p.pos_pool[slot] = pos;
      } else {
        to = is_query(h) ? q_to + h * p.q_out.sh : k_to + number(h) * p.k_out.sh;
        if (!rotated && to == source(h)) continue;                // in place, not part of the rotation
      }
      if (rotated && !is_v) rot_pieces<T, VEC>(a[i], c[i], cs, sn, p.interleaved);
      *reinterpret_cast<Piece*>(to + (is_v ? u * 2 * VEC : e0)) = a[i];
      *reinterpret_cast<Piece*>(to + (is_v ? u * 2 * VEC + VEC : e1)) = c[i];
    }
    h0 += step * UNROLL;
    if (h0 < heads) fetch(h0);
  }
}

}  // namespace pkv
