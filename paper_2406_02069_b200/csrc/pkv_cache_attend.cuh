// Attention of one new token per sequence over a cache that grows: out[b][g] = softmax(x[g][r]) V over the rows r of sequence b,
// whose number, pages and positions are read on the device.
//
//   s = q . k_r scale,   x = cap tanh(s / cap) - slope_g (p - p_r),   row seen if p_r <= p and (p - p_r < window or p_r < prefix)
//
// What bounds it: every seen row is read once, 2 d elements for 4 d operations per query head, so the floor is the bytes of
// the cache over the memory bandwidth; a call with few rows is a chain of latencies (lengths, table, rows, join).
//   * The lengths are not known on the host, so the grid does not depend on them: as many CTAs as fit on the device at once,
//     and the tiles (64 rows of one KV head and block of query heads) of the whole batch are dealt out to them in equal
//     consecutive ranges.  A long sequence is then split over many CTAs, and a CTA takes many short ones in turn.
//   * A CTA that has all tiles of a head writes its output; otherwise it leaves (exponent, sum, weighted sum) in the workspace, and
//     the last CTA of the head to arrive joins them in the order of the rows, so that equal calls give equal bits.
//   * A warp takes tiles of 16 rows, kStages of them in shared memory or on their way by asynchronous copies.  A row that is
//     not seen is filled with zeros instead of read; a tile without a seen row costs its positions only.
//   * 16-bit rows go through mma.sync, fp32 accumulation, the query heads as M: GT = 4 heads with the high, middle and low
//     16-bit parts of their softmax weights in rows 0-3, 4-7 and 8-11, GT = 8 with high and middle parts in one product and
//     the low ones in a second.  The parts carry 24 bits, so the weights stay fp32 in effect.
//   * fp32 rows: a lane has half a row's dot products, then a few channels of all rows.
#pragma once

#include "pkv_common.cuh"
#include "pkv_mma16.cuh"

namespace pkv {

constexpr int kCaWarps = 4;
constexpr int kCaThreads = kCaWarps * 32;
constexpr int kCaTile = kCaWarps * 16;     // rows of a tile: 16 to a warp
constexpr int kCaStages = 3;               // a warp's tiles in shared memory or on their way
constexpr int kCaMaxGrid = 2 * 160;        // CTAs at most (sizes the partial sums in the workspace)
constexpr int kCaMaxHeads = 8;             // query heads of a CTA at most
// Floats of one partial result: sums, then exponents, then weights' sums.
constexpr int kCaPartial = kCaMaxHeads * (128 + 2);

struct CacheAttendParams {
  const void* q;
  int64_t q_sb, q_sh;
  const void* k_pool;
  const void* v_pool;
  const int32_t* pos_pool;                 // with POS
  const int32_t* table;                    // of the layer: [batch][H_kv][max_pages]
  const int32_t* lens;                     // of the layer
  const int32_t* q_pos;                    // with POS
  const float* slopes;                     // or null
  float* out;
  float* lse;                              // or null
  uint32_t* status;
  int32_t* counters;                       // [batch * H_kv * head_blocks], zero between calls
  float* partials;                         // [2 * gridDim.x][kCaPartial]
  int32_t batch, num_kv_heads, group, head_blocks;
  int32_t max_pages, page_size, num_pages;
  int32_t window, prefix;
  float scale_log2;                        // log2(e) scale; with a cap scale / cap
  float cap_log2;                          // log2(e) cap, 0: no cap
};

// Logit in powers of two from a dot product; far: p - p_r where there is a bias.
__device__ __forceinline__ float ca_logit(const CacheAttendParams& p, float dot, float slope_log2, float far) {
  float x = dot * p.scale_log2;
  if (p.cap_log2 != 0.f) x = p.cap_log2 * tanhf(x);
  return fmaf(-slope_log2, far, x);
}

// The rows of one KV head of one sequence, as a warp looks them up.
template <bool POS>
struct CaRows {
  const int32_t* table;
  int32_t rows;                            // that the segment goes up to
  int32_t q_pos;
};

// Where row r lies (in rows of the pool), -1 if it is not seen; *far: p - p_r.
template <bool POS>
__device__ __forceinline__ int64_t ca_look_up(const CacheAttendParams& p, const CaRows<POS>& s, int r, bool report, uint32_t* far) {
  *far = 0;
  if (r >= s.rows) return -1;
  const int page = __ldg(s.table + r / p.page_size);
  if (page < 0 || page >= p.num_pages) {
    if (report) atomicOr(p.status, kStatusBadPage);
    return -1;
  }
  const int64_t at = static_cast<int64_t>(page) * p.page_size + r % p.page_size;
  if (POS) {
    const int pos = __ldg(p.pos_pool + at);
    *far = static_cast<uint32_t>(s.q_pos) - static_cast<uint32_t>(pos);       // positions may be 2^31 apart and more
    if (pos > s.q_pos) return -1;
    if (p.window > 0 && *far >= static_cast<uint32_t>(p.window) && pos >= p.prefix) return -1;
  }
  return at;
}

// Sums of one query head over the warp's rows on the fp32 pipe, for rows that hold infinities or NaN:
// in the matrix product every part of a weight meets every value, and a part that is zero or negative makes NaN of an infinity.
template <typename T, int D, bool POS>
__device__ __noinline__ void ca_sum_special(const CacheAttendParams& p, const CaRows<POS>& s, const T* q, int first, float slope, float ref,
                                            float* acc) {
  constexpr int PER = D / 32;
  const int lane = threadIdx.x & 31;
  float qv[PER], a[PER];
#pragma unroll
  for (int c = 0; c < PER; ++c) {
    qv[c] = to_float(q[lane * PER + c]);
    a[c] = 0.f;
  }
#pragma unroll 1
  for (int t0 = first; t0 < s.rows; t0 += kCaTile)
#pragma unroll 1
    for (int r = t0; r < min(t0 + 16, s.rows); ++r) {
      uint32_t far;
      const int64_t at = ca_look_up<POS>(p, s, r, false, &far);
      if (at < 0) continue;
      const T* k = static_cast<const T*>(p.k_pool) + at * D + lane * PER;
      const T* v = static_cast<const T*>(p.v_pool) + at * D + lane * PER;
      float dot = 0.f;
#pragma unroll
      for (int c = 0; c < PER; ++c) dot = fmaf(qv[c], to_float(k[c]), dot);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
      const float w = exp2f(ca_logit(p, dot, slope, __uint2float_rn(far)) - ref);
#pragma unroll
      for (int c = 0; c < PER; ++c) a[c] = fmaf(w, to_float(v[c]), a[c]);
    }
#pragma unroll
  for (int c = 0; c < PER; ++c) acc[lane * PER + c] = a[c];
}

// One warp's sums over rows first .. first + 15, first + kCaTile .. of a segment: weights' sums to z[GT], exponents that they
// are relative to (-infinity: no seen row) to m[GT], weighted sums of V to acc[GT][D + 4], all in shared memory; acc is the warp's own
// ring, whose rows are used up by then.
template <typename T, int D, int GT, bool POS>
struct CaWarp {
  static constexpr uint32_t ROW = D * sizeof(T), TILE = 16 * ROW;
  static constexpr int PIECES = ROW / 16;                        // 16-byte pieces of a row: 8, 16 or 32
  static constexpr int ROWS_AT_ONCE = 32 / PIECES;
  static constexpr int HEAD = D + 4;                             // floats from a head's sums to the next one's
  static constexpr size_t kRing = kCaStages * 2 * TILE;          // bytes of a warp's ring

  // A piece's place in its row: eight lanes that read together touch every bank once.
  __device__ __forceinline__ static uint32_t k_place(int r, int piece) {
    if constexpr (sizeof(T) == 4) return (piece ^ (r & 7)) << 4;
    return (piece ^ ((r & 1) << 2)) << 4;
  }
  __device__ __forceinline__ static uint32_t v_place(int r, int piece) {
    if constexpr (sizeof(T) == 4) return piece << 4;
    return (piece ^ (((r >> 1) & 3) << 1)) << 4;
  }

  __device__ __forceinline__ static void copy_tile(const CacheAttendParams& p, uint32_t to_tile, int64_t mine) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int s = 0; s < 16 / ROWS_AT_ONCE; ++s) {
      const int r = s * ROWS_AT_ONCE + lane / PIECES, piece = lane % PIECES;
      const int64_t at = __shfl_sync(0xffffffffu, mine, r);
      const int64_t from = (at >= 0 ? at : 0) * D + piece * (16 / static_cast<int>(sizeof(T)));
      const uint32_t to = to_tile + r * ROW;
      dec_copy16(to + k_place(r, piece), static_cast<const T*>(p.k_pool) + from, at >= 0);
      dec_copy16(to + TILE + v_place(r, piece), static_cast<const T*>(p.v_pool) + from, at >= 0);
    }
  }
};

// State of the sums of a warp, and one step over a tile; 16-bit rows.
template <typename T, int D, int GT, bool POS>
struct CaSums {
  using W = CaWarp<T, D, GT, POS>;
  using X = Dec16<T>;
  static constexpr int KC = D / 32, VC = D / 64;
  uint4 q[KC];
  float o[VC * 8][4];
  float m, z;                              // of head g % GT: m over the warp's rows, z over this lane's
  float slope;

  __device__ __forceinline__ void start(const CacheAttendParams& p, const T* q0, int heads, int hq) {
    const int lane = threadIdx.x & 31, g = (lane >> 2) % GT, c = lane & 3;
    const bool there = g < heads;
#pragma unroll
    for (int j = 0; j < KC; ++j)
      q[j] = there ? *reinterpret_cast<const uint4*>(q0 + g * p.q_sh + j * 32 + c * 8) : make_uint4(0, 0, 0, 0);
    slope = POS && p.slopes && there ? __ldg(p.slopes + hq + g) * 1.4426950408889634f : 0.f;
#pragma unroll
    for (int i = 0; i < VC * 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    m = -INFINITY;
    z = 0.f;
  }

  // seen: bit r for row r of the tile; far: lane r (and r + 16) has row r's distance.
  __device__ __forceinline__ void step(const CacheAttendParams& p, uint32_t k_at, uint32_t v_at, uint32_t seen, uint32_t far) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    float x[2][2];
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        const uint4 k = dec_lds16(k_at + (t * 8 + g) * W::ROW + W::k_place(g, j * 4 + c));
        X::mma(s0, q[j].x, q[j].x, q[j].y, q[j].y, k.x, k.y);
        X::mma(s1, q[j].z, q[j].z, q[j].w, q[j].w, k.z, k.w);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = t * 8 + 2 * c + i;
        float d = 0.f;
        if (POS) d = __uint2float_rn(__shfl_sync(0xffffffffu, far, r));
        x[t][i] = (seen >> r) & 1u ? ca_logit(p, s0[i] + s1[i], slope, d) : -INFINITY;
        mx = fmaxf(mx, x[t][i]);
      }
    }
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    const float mn = fmaxf(m, mx);
    const float ref = mn == -INFINITY ? 0.f : mn - X::kShift;
    if (__any_sync(0xffffffffu, mn > m)) {
      const float corr = m == -INFINITY ? 0.f : ex2(m - mn);
      z *= corr;
#pragma unroll
      for (int i = 0; i < VC * 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] *= corr;
    }
    m = mn;
    uint32_t a[2][2], low8[2];             // [rows 2c.. / 2c + 8..][fragment row g / g + 8]
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float w0 = ex2(x[t][0] - ref), w1 = ex2(x[t][1] - ref);
      z += w0 + w1;
      const uint32_t high = X::pack(w0, w1);
      const float2 hf = X::unpack(high);
      const uint32_t mid = X::pack(w0 - hf.x, w1 - hf.y);
      const float2 mf = X::unpack(mid);
      const uint32_t low = X::pack(w0 - hf.x - mf.x, w1 - hf.y - mf.y);
      if (GT == 4) {
        a[t][0] = g < 4 ? high : mid;
        a[t][1] = g < 4 ? low : 0u;
      } else {
        a[t][0] = high;
        a[t][1] = mid;
        low8[t] = low;
      }
    }
#pragma unroll
    for (int j = 0; j < VC; ++j) {
      uint4 v[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {        // row (t / 2) * 8 + 2c + t % 2
        const int r = (t >> 1) * 8 + 2 * c + (t & 1);
        v[t] = dec_lds16(v_at + r * W::ROW + W::v_place(2 * c, j * 8 + g));
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t v0 = reinterpret_cast<const uint32_t*>(&v[0])[w], v1 = reinterpret_cast<const uint32_t*>(&v[1])[w];
        const uint32_t v2 = reinterpret_cast<const uint32_t*>(&v[2])[w], v3 = reinterpret_cast<const uint32_t*>(&v[3])[w];
        const uint32_t e0 = __byte_perm(v0, v1, 0x5410), e1 = __byte_perm(v2, v3, 0x5410);
        const uint32_t f0 = __byte_perm(v0, v1, 0x7632), f1 = __byte_perm(v2, v3, 0x7632);
        X::mma(o[j * 8 + 2 * w], a[0][0], a[0][1], a[1][0], a[1][1], e0, e1);
        X::mma(o[j * 8 + 2 * w + 1], a[0][0], a[0][1], a[1][0], a[1][1], f0, f1);
        if (GT == 8) {
          X::mma(o[j * 8 + 2 * w], low8[0], 0u, low8[1], 0u, e0, e1);
          X::mma(o[j * 8 + 2 * w + 1], low8[0], 0u, low8[1], 0u, f0, f1);
        }
      }
    }
  }

  __device__ __forceinline__ void finish(const CacheAttendParams& p, const CaRows<POS>& s, const T* q0, int heads, int first, float* acc,
                                         float* m_out, float* z_out) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    z += __shfl_xor_sync(0xffffffffu, z, 1);
    z += __shfl_xor_sync(0xffffffffu, z, 2);
    float special = 0.f;                   // NaN once a sum is not finite
    __syncwarp();
    if (GT == 4) {
      // Lanes g and g + 4 hold parts of the same sums: each keeps one of the channel octets 64 j + 8 (2c + e) + 0 .. 7 of head g % 4
      const bool upper = g >= 4;
#pragma unroll
      for (int j = 0; j < VC; ++j) {
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float s0 = o[j * 8 + i][0] + o[j * 8 + i][2], s1 = o[j * 8 + i][1] + o[j * 8 + i][3];
          t[i] = (upper ? s1 : s0) + __shfl_xor_sync(0xffffffffu, upper ? s0 : s1, 16);
          special = fmaf(t[i], 0.f, special);
        }
        float4* to = reinterpret_cast<float4*>(acc + (g & 3) * W::HEAD + j * 64 + (2 * c + (upper ? 1 : 0)) * 8);
        to[0] = make_float4(t[0], t[1], t[2], t[3]);
        to[1] = make_float4(t[4], t[5], t[6], t[7]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < VC; ++j) {
        float t[2][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          t[0][i] = o[j * 8 + i][0] + o[j * 8 + i][2];
          t[1][i] = o[j * 8 + i][1] + o[j * 8 + i][3];
          special = fmaf(t[0][i], 0.f, special);
          special = fmaf(t[1][i], 0.f, special);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float4* to = reinterpret_cast<float4*>(acc + g * W::HEAD + j * 64 + (2 * c + e) * 8);
          to[0] = make_float4(t[e][0], t[e][1], t[e][2], t[e][3]);
          to[1] = make_float4(t[e][4], t[e][5], t[e][6], t[e][7]);
        }
      }
    }
    const float ref = m == -INFINITY ? m : m - X::kShift;
    if (__any_sync(0xffffffffu, special != 0.f)) {
      __syncwarp();
#pragma unroll 1
      for (int j = 0; j < heads; ++j) {
        const float rj = __shfl_sync(0xffffffffu, ref, j * 4);
        const float sj = __shfl_sync(0xffffffffu, slope, j * 4);
        ca_sum_special<T, D, POS>(p, s, q0 + j * p.q_sh, first, sj, rj == -INFINITY ? 0.f : rj, acc + j * W::HEAD);
      }
    }
    if (g < GT && c == 0) {
      m_out[g] = ref;
      z_out[g] = z;
    }
  }
};

// fp32 rows.  Lane l has channels of half l / 16 of row l % 16 for the dot products, and channels 4 (l % PIECES) .. of the rows of
// parity l / PIECES (all rows where a row has 32 pieces) for the weighted sums.
template <int D, int GT, bool POS>
struct CaSums<float, D, GT, POS> {
  using W = CaWarp<float, D, GT, POS>;
  static constexpr int PIECES = W::PIECES, VR = W::ROWS_AT_ONCE;
  const float* q0;                         // shared memory: [GT][D], zeros for heads that are not there
  float o[GT][4];
  float m[GT], z[GT];                      // m the same in all lanes; z of this lane's row
  float slope[GT];

  __device__ __forceinline__ void start(const CacheAttendParams& p, const float* q_shared, int heads, int hq) {
    q0 = q_shared;
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      slope[g] = POS && p.slopes && g < heads ? __ldg(p.slopes + hq + g) * 1.4426950408889634f : 0.f;
      o[g][0] = o[g][1] = o[g][2] = o[g][3] = 0.f;
      m[g] = -INFINITY;
      z[g] = 0.f;
    }
  }

  __device__ __forceinline__ void step(const CacheAttendParams& p, uint32_t k_at, uint32_t v_at, uint32_t seen, uint32_t far) {
    const int lane = threadIdx.x & 31, row = lane & 15, part = lane >> 4;
    unsigned long long d2[GT][2];
#pragma unroll
    for (int g = 0; g < GT; ++g) d2[g][0] = d2[g][1] = 0ull;
#pragma unroll
    for (int j = 0; j < PIECES / 2; ++j) {
      const int piece = part * (PIECES / 2) + j;
      const uint4 raw = dec_lds16(k_at + row * W::ROW + W::k_place(row, piece));
      const unsigned long long k0 = pack2(__uint_as_float(raw.x), __uint_as_float(raw.y));
      const unsigned long long k1 = pack2(__uint_as_float(raw.z), __uint_as_float(raw.w));
#pragma unroll
      for (int g = 0; g < GT; ++g) {
        const float4 qv = *reinterpret_cast<const float4*>(q0 + g * D + piece * 4);
        d2[g][0] = fma2(pack2(qv.x, qv.y), k0, d2[g][0]);
        d2[g][1] = fma2(pack2(qv.z, qv.w), k1, d2[g][1]);
      }
    }
    const bool live = (seen >> row) & 1u;
    const float d = POS ? __uint2float_rn(far) : 0.f;             // lane l has row l % 16's
    float w[GT];
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      float a, b;
      unpack2(add2(d2[g][0], d2[g][1]), a, b);
      float dot = a + b;
      dot += __shfl_xor_sync(0xffffffffu, dot, 16);
      const float x = live ? ca_logit(p, dot, slope[g], d) : -INFINITY;
      float mx = x;
#pragma unroll
      for (int s = 8; s > 0; s >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
      const float mn = fmaxf(m[g], mx);
      if (mn > m[g]) {                     // the same in all lanes
        const float corr = m[g] == -INFINITY ? 0.f : exp2f(m[g] - mn);
        z[g] *= corr;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[g][e] *= corr;
        m[g] = mn;
      }
      w[g] = exp2f(x - (mn == -INFINITY ? 0.f : mn));
      z[g] += w[g];
    }
#pragma unroll
    for (int r0 = 0; r0 < 16; r0 += VR) {
      const int r = r0 + lane / PIECES;
      const uint4 raw = dec_lds16(v_at + r * W::ROW + W::v_place(r, lane % PIECES));
      const float v[4] = {__uint_as_float(raw.x), __uint_as_float(raw.y), __uint_as_float(raw.z), __uint_as_float(raw.w)};
#pragma unroll
      for (int g = 0; g < GT; ++g) {
        const float wr = __shfl_sync(0xffffffffu, w[g], r);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[g][e] = fmaf(wr, v[e], o[g][e]);
      }
    }
  }

  __device__ __forceinline__ void finish(const CacheAttendParams&, const CaRows<POS>&, const float*, int, int, float* acc, float* m_out,
                                         float* z_out) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int g = 0; g < GT; ++g) {
#pragma unroll
      for (int s = 8; s > 0; s >>= 1) z[g] += __shfl_xor_sync(0xffffffffu, z[g], s);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (VR == 2) o[g][e] += __shfl_xor_sync(0xffffffffu, o[g][e], 16);
      if (lane < PIECES) *reinterpret_cast<float4*>(acc + g * W::HEAD + lane * 4) = make_float4(o[g][0], o[g][1], o[g][2], o[g][3]);
      if (lane == 0) {
        m_out[g] = m[g];
        z_out[g] = z[g];
      }
    }
  }
};

// Factor of sums that are relative to 2^m in sums relative to 2^largest.
__device__ __forceinline__ float ca_factor(float m, float largest) { return m == -INFINITY ? 0.f : exp2f(m - largest); }

// Writes a head's output: acc and z are relative to 2^m.  A sum of zero means that no row was seen.
__device__ __forceinline__ void ca_write(const CacheAttendParams& p, int64_t head, int D, int channel, float m, float z, float acc) {
  p.out[head * D + channel] = z == 0.f ? 0.f : acc / z;
  if (channel == 0 && p.lse) p.lse[head] = z == 0.f ? -INFINITY : (m + log2f(z)) * 0.6931471805599453f;
}

// grid: any number of CTAs up to kCaMaxGrid; block kCaThreads; dynamic shared memory kCaWarps rings (+ GT * D floats in fp32).
template <typename T, int D, int GT, bool POS>
__global__ void __launch_bounds__(kCaThreads) cache_attend_kernel(const __grid_constant__ CacheAttendParams p) {
  using W = CaWarp<T, D, GT, POS>;
  using Sums = CaSums<T, D, GT, POS>;
  static_assert(GT * W::HEAD * 4 <= W::kRing, "a warp's sums fit its ring");
  extern __shared__ __align__(128) uint8_t ca_smem[];
  __shared__ int32_t s_off[PKV_MAX_CACHE_BATCH + 1];             // tiles of a head of the sequences ahead
  __shared__ int32_t s_scan[kCaWarps];
  __shared__ float s_m[kCaWarps][GT], s_z[kCaWarps][GT];
  __shared__ int32_t s_last;
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int most = static_cast<int>(min(static_cast<int64_t>(p.max_pages) * p.page_size, static_cast<int64_t>(INT32_MAX - kCaTile)));
  pdl_wait();

  // ---- tiles of every sequence (at least one, whose rows may be none) and their running sum
  {
    constexpr int PER = PKV_MAX_CACHE_BATCH / kCaThreads;
    int mine[PER], sum = 0;
    const int per = (p.batch + kCaThreads - 1) / kCaThreads;     // consecutive sequences of a thread
    for (int i = 0; i < PER; ++i) {
      const int b = tid * per + i;
      mine[i] = 0;
      if (i < per && b < p.batch) mine[i] = max(1, (min(max(__ldg(p.lens + b), 0), most) + kCaTile - 1) / kCaTile);
      sum += mine[i];
    }
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += x;
    }
    if (lane == 31) s_scan[warp] = run;
    __syncthreads();
    for (int w = 0; w < warp; ++w) run += s_scan[w];
    run -= sum;
    for (int i = 0; i < PER; ++i) {
      const int b = tid * per + i;
      if (i < per && b < p.batch) s_off[b] = run;
      run += mine[i];
    }
    if (tid == kCaThreads - 1) s_off[p.batch] = run;
    __syncthreads();
  }
  const int per_seq = p.num_kv_heads * p.head_blocks;
  const int64_t total = static_cast<int64_t>(s_off[p.batch]) * per_seq;
  const int64_t ctas = min(static_cast<int64_t>(gridDim.x), total);
  if (blockIdx.x >= ctas) return;
  auto range_begin = [&](int64_t cta) { return total * cta / ctas; };
  auto owner = [&](int64_t tile) { return ((tile + 1) * ctas - 1) / total; };
  const int64_t begin = range_begin(blockIdx.x), end = range_begin(blockIdx.x + 1);
  const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(ca_smem)) + warp * static_cast<uint32_t>(W::kRing);
  float* acc = reinterpret_cast<float*>(ca_smem + warp * W::kRing);

  int b = 0;
  for (int64_t at = begin; at < end;) {
    // ---- the segment: tiles tile0 .. tile1 - 1 of one block of query heads
    while (at >= static_cast<int64_t>(s_off[b + 1]) * per_seq) ++b;
    const int tiles = s_off[b + 1] - s_off[b];
    const int64_t in_seq = at - static_cast<int64_t>(s_off[b]) * per_seq;
    const int unit = static_cast<int>(in_seq / tiles), tile0 = static_cast<int>(in_seq - static_cast<int64_t>(unit) * tiles);
    const int tile1 = static_cast<int>(min(static_cast<int64_t>(tiles), tile0 + (end - at)));
    const int h = unit / p.head_blocks, g0 = (unit - h * p.head_blocks) * GT;
    const int heads = min(GT, p.group - g0);
    const int hq = h * p.group + g0;
    const T* q0 = static_cast<const T*>(p.q) + b * p.q_sb + hq * p.q_sh;
    const int n = min(max(__ldg(p.lens + b), 0), most);
    CaRows<POS> rows;
    rows.table = p.table + (static_cast<int64_t>(b) * p.num_kv_heads + h) * p.max_pages;
    rows.rows = min(n, tile1 * kCaTile);
    rows.q_pos = POS ? __ldg(p.q_pos + b) : 0;
    const int first = tile0 * kCaTile + warp * 16;

    // ---- copies of the first tiles
    uint32_t seen[kCaStages], far[kCaStages];
    {
      int64_t mine[kCaStages];
#pragma unroll
      for (int s = 0; s < kCaStages; ++s) mine[s] = ca_look_up<POS>(p, rows, first + s * kCaTile + (lane & 15), lane < 16, &far[s]);
#pragma unroll
      for (int s = 0; s < kCaStages; ++s) {
        seen[s] = __ballot_sync(0xffffffffu, mine[s] >= 0);
        if (seen[s]) W::copy_tile(p, ring + s * (2 * W::TILE), mine[s]);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
    }
    uint32_t far_next;
    int64_t next = ca_look_up<POS>(p, rows, first + kCaStages * kCaTile + (lane & 15), lane < 16, &far_next);
    const float* q_f = nullptr;
    if constexpr (sizeof(T) == 4) {
      float* q_shared = reinterpret_cast<float*>(ca_smem + kCaWarps * W::kRing);
      for (int i = tid; i < GT * D; i += kCaThreads) q_shared[i] = i / D < heads ? q0[(i / D) * p.q_sh + i % D] : 0.f;
      __syncthreads();
      q_f = q_shared;
    }
    Sums sums;
    if constexpr (sizeof(T) == 4) sums.start(p, q_f, heads, hq);
    else sums.start(p, q0, heads, hq);

    // ---- the warp's rows
    for (int t0 = first; t0 < rows.rows;) {
#pragma unroll
      for (int slot = 0; slot < kCaStages; ++slot) {
        if (t0 >= rows.rows) break;        // (uniform over the warp)
        asm volatile("cp.async.wait_group %0;" ::"n"(kCaStages - 1) : "memory");
        __syncwarp();
        const uint32_t k_at = ring + slot * (2 * W::TILE);
        if (seen[slot]) sums.step(p, k_at, k_at + W::TILE, seen[slot], far[slot]);
        __syncwarp();                      // the tile has been read
        seen[slot] = __ballot_sync(0xffffffffu, next >= 0);
        far[slot] = far_next;
        if (seen[slot]) W::copy_tile(p, k_at, next);
        asm volatile("cp.async.commit_group;" ::: "memory");
        t0 += kCaTile;
        next = ca_look_up<POS>(p, rows, t0 + kCaStages * kCaTile + (lane & 15), lane < 16, &far_next);
      }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    sums.finish(p, rows, q0, heads, first, acc, s_m[warp], s_z[warp]);
    __syncthreads();

    // ---- the warps' sums; then the output, or a partial result that the head's last CTA joins with the others
    const int64_t head0 = static_cast<int64_t>(b) * p.num_kv_heads * p.group + hq;
    const bool whole = tile0 == 0 && tile1 == tiles;
    float* part = p.partials + (2 * static_cast<int64_t>(blockIdx.x) + (at > begin ? 1 : 0)) * kCaPartial;
    for (int o = tid; o < heads * D; o += kCaThreads) {
      const int g = o / D, channel = o - g * D;
      float m = s_m[0][g];
#pragma unroll
      for (int w = 1; w < kCaWarps; ++w) m = fmaxf(m, s_m[w][g]);
      float z = 0.f, a = 0.f;
#pragma unroll
      for (int w = 0; w < kCaWarps; ++w) {
        const float f = ca_factor(s_m[w][g], m);
        z = fmaf(s_z[w][g], f, z);
        a = fmaf(reinterpret_cast<const float*>(ca_smem + w * W::kRing)[g * W::HEAD + channel], f, a);
      }
      if (whole) {
        ca_write(p, head0 + g, D, channel, m, z, a);
      } else {
        __stcg(part + o, a);
        if (channel == 0) {
          __stcg(part + GT * D + g, m);
          __stcg(part + GT * D + GT + g, z);
        }
      }
    }
    if (!whole) {
      const int64_t unit0 = at - tile0, c0 = owner(unit0), c1 = owner(unit0 + tiles - 1);
      int32_t* counter = p.counters + static_cast<int64_t>(b) * per_seq + unit;
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const int before = atomicAdd(counter, 1);
        s_last = before == static_cast<int>(c1 - c0);
        if (s_last) *counter = 0;          // everybody has arrived: ready for the next call
        __threadfence();
      }
      __syncthreads();
      if (s_last) {
        for (int o = tid; o < heads * D; o += kCaThreads) {
          const int g = o / D, channel = o - g * D;
          float m = -INFINITY, z = 0.f, a = 0.f;
          for (int64_t c = c0; c <= c1; ++c) {                   // in the order of the rows
            const float* other = p.partials + (2 * c + (range_begin(c) < unit0 ? 1 : 0)) * kCaPartial;
            const float mo = __ldcg(other + GT * D + g);
            const float mn = fmaxf(m, mo);
            const float f = ca_factor(m, mn), fo = ca_factor(mo, mn);
            z = fmaf(z, f, __ldcg(other + GT * D + GT + g) * fo);
            a = fmaf(a, f, __ldcg(other + o) * fo);
            m = mn;
          }
          ca_write(p, head0 + g, D, channel, m, z, a);
        }
      }
    }
    __syncthreads();                       // the sums have been read: the rings may be filled again
    at += tile1 - tile0;
  }
}

}  // namespace pkv
