// Attention of one new token per sequence over a cache that grows: out[b][g] = softmax(x[g][r]) V over the rows r of sequence b,
// whose number, pages and positions are read on the device.
//
//   s = q . k_r scale,   x = cap tanh(s / cap) - slope_g (p - p_r),   row seen if p_r <= p and (p - p_r < window or p_r < prefix)
//
// What bounds it: every seen row is read once for eight query heads at most, 2 d elements for 4 d operations per head, so the floor is
// the bytes of the cache over the memory bandwidth (64 sequences of 129 to 4096 rows, 32 / 8 heads, bf16: 93 us, 89 % of the rate of
// a copy; 131072 rows of one, 64 / 8 heads: 99, 83 %).  Sixteen query heads to a KV head are two blocks, each with its own loads: 142
// us for 131072 rows, 128 / 8 heads.  A call with few rows is a chain of latencies (64 rows: 5.2 us, of which lengths and plan
// 1.5, table and queries 0.7, rows and products 1.0, merge and output 0.6; 512 rows in eight parts: 8.2).
//   * The lengths are not known on the host, so the grid does not depend on them: as many CTAs as fit on the device at once,
//     which deal the batch's tiles (64 rows of one KV head and block of query heads) out among themselves (CaPlan).  A long
//     sequence is split over many CTAs, and a CTA takes many short ones in turn, the next one's rows on their way while
//     it finishes the one ahead.
//   * A CTA that has all tiles of a head writes its output; otherwise it leaves (exponent, sum, weighted sum) in the workspace, and
//     the last CTA of the head to arrive joins them in the order of the rows (many of them in groups first), so that equal calls
//     give equal bits.
//   * A warp takes tiles of 16 rows (fp32: 8), kCaStages of them in shared memory or on their way by asynchronous copies.  A row that is
//     not seen is filled with zeros instead of read; a tile without a seen row costs its positions only.
//   * 16-bit rows go through mma.sync, fp32 accumulation, the query heads as M: GT = 4 heads with the high, middle and low
//     16-bit parts of their softmax weights in rows 0-3, 4-7 and 8-11, GT = 8 with high and middle parts in one product (rows 0-7
//     and 8-15) and the low ones in a second, added to the middle ones.  The parts carry the 24 bits of an fp32 weight (fp16: of
//     weights down to 2^-27 of the largest, Dec16).
//   * fp32 rows: a lane has a quarter of a row's dot products, then four channels of all rows; GT = 1, 2, 4 or 8.
#pragma once

#include "pkv_common.cuh"
#include "pkv_mma16.cuh"

namespace pkv {

constexpr int kCaTile = 64;                // rows of a tile, shared by the warps of a CTA
constexpr int kCaStages = 2;               // a warp's tiles in shared memory or on their way
// Warps of a CTA: four with 16 rows each of 16-bit types, eight with 8 rows each in fp32, where a row takes twice the bytes and
// several times the instructions.
template <typename T>
constexpr int kCaWarps = sizeof(T) == 4 ? 8 : 4;
template <typename T>
constexpr int kCaThreads = kCaWarps<T> * 32;
template <typename T>
constexpr int kCaRows = kCaTile / kCaWarps<T>;
// CTAs to an SM: twelve warps hide more of a tile's chain of products, shuffles and exponentials than eight with all registers
// (131072 rows x 8 KV heads x 8 query heads: two CTAs 114 us, three 102; 64 sequences of 129 to 4096 rows, capped, window: 123, 106).
constexpr int kCaPerSm = 3;
constexpr int kCaMaxGrid = kCaPerSm * 160; // CTAs at most (sizes the partial sums in the workspace)
constexpr int kCaMaxHeads = 8;             // query heads of a CTA at most
constexpr int kCaDirect = 32;              // parts of a unit that one CTA joins at once
// Floats of one partial result: sums, then exponents, then weights' sums.
constexpr int kCaPartial = kCaMaxHeads * (128 + 2);

// POS of the templates: 0 positions play no part, 1 they say which rows are seen, 2 and give a bias.
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
  int32_t* group_counters;                 // [2 * gridDim.x], too
  float* partials;                         // [2 * gridDim.x][kCaPartial]
  int32_t batch, num_kv_heads, group, head_blocks;
  int32_t max_pages, page_size, num_pages;
  int32_t page_shift;                      // log2(page_size), -1 if it is no power of two
  int32_t window, prefix;
  float scale_log2;                        // log2(e) scale; with a cap scale / cap
  float cap_log2;                          // log2(e) cap, 0: no cap
};

// Logit in powers of two from a dot product; far: p - p_r where there is a bias.
template <int POS>
__device__ __forceinline__ float ca_logit(const CacheAttendParams& p, float dot, float slope_log2, float far) {
  float x = dot * p.scale_log2;
  if (p.cap_log2 != 0.f) x = p.cap_log2 * tanhf(x);
  return POS == 2 ? fmaf(-slope_log2, far, x) : x;
}

// The rows of one KV head of one sequence, as a warp looks them up.
template <int POS>
struct CaRows {
  const int32_t* table;
  int32_t rows;                            // that the segment goes up to
  int32_t q_pos;
};

// Row r's place in the pool, counted in rows (the host keeps those below 2^31); -1 if it has none.
template <int POS>
__device__ __forceinline__ int ca_place(const CacheAttendParams& p, const CaRows<POS>& s, int r, bool report) {
  if (r >= s.rows) return -1;
  const int j = p.page_shift >= 0 ? r >> p.page_shift : r / p.page_size;
  const int page = s.table[j];
  if (page < 0 || page >= p.num_pages) {
    if (report) atomicOr(p.status, kStatusBadPage);
    return -1;
  }
  return page * p.page_size + (r - j * p.page_size);
}

// Whether the row at a place is seen, by its position; *far: p - p_r.
template <int POS>
__device__ __forceinline__ bool ca_seen(const CacheAttendParams& p, const CaRows<POS>& s, int pos, uint32_t* far) {
  *far = static_cast<uint32_t>(s.q_pos) - static_cast<uint32_t>(pos);         // positions may be 2^31 apart and more
  return pos <= s.q_pos && (p.window == 0 || *far < static_cast<uint32_t>(p.window) || pos < p.prefix);
}

// Sums of one query head over the warp's rows on the fp32 pipe, for rows that hold infinities or NaN:
// in the matrix product every part of a weight meets every value, and a part that is zero or negative makes NaN of an infinity.
template <typename T, int D, int POS>
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
    for (int r = t0; r < min(t0 + kCaRows<T>, s.rows); ++r) {
      uint32_t far = 0;
      const int at = ca_place<POS>(p, s, r, false);
      if (at < 0 || (POS && !ca_seen<POS>(p, s, p.pos_pool[at], &far))) continue;
      const T* k = static_cast<const T*>(p.k_pool) + static_cast<int64_t>(at) * D + lane * PER;
      const T* v = static_cast<const T*>(p.v_pool) + static_cast<int64_t>(at) * D + lane * PER;
      float dot = 0.f;
#pragma unroll
      for (int c = 0; c < PER; ++c) dot = fmaf(qv[c], to_float(k[c]), dot);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
      const float w = exp2f(ca_logit<POS>(p, dot, slope, __uint2float_rn(far)) - ref);
#pragma unroll
      for (int c = 0; c < PER; ++c) a[c] = fmaf(w, to_float(v[c]), a[c]);
    }
#pragma unroll
  for (int c = 0; c < PER; ++c) acc[lane * PER + c] = a[c];
}

// One warp's sums over rows first .. first + kCaRows - 1, first + kCaTile .. of a segment: weights' sums to z[GT], exponents that they
// are relative to (-infinity: no seen row) to m[GT], weighted sums of V to acc[GT][D + 4], all in shared memory.
template <typename T, int D, int GT, int POS>
struct CaWarp {
  static constexpr int TR = kCaRows<T>;                          // rows of the warp's tile
  static constexpr uint32_t ROW = D * sizeof(T), TILE = TR * ROW;
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

  __device__ __forceinline__ static void copy_tile(const CacheAttendParams& p, uint32_t to_tile, int mine) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int s = 0; s < TR / ROWS_AT_ONCE; ++s) {
      const int r = s * ROWS_AT_ONCE + lane / PIECES, piece = lane % PIECES;
      const int at = __shfl_sync(0xffffffffu, mine, r);
      const int64_t from = static_cast<int64_t>(max(at, 0)) * D + piece * (16 / static_cast<int>(sizeof(T)));
      const uint32_t to = to_tile + r * ROW;
      dec_copy16(to + k_place(r, piece), static_cast<const T*>(p.k_pool) + from, at >= 0);
      dec_copy16(to + TILE + v_place(r, piece), static_cast<const T*>(p.v_pool) + from, at >= 0);
    }
  }
};

// State of the sums of a warp, and one step over a tile; 16-bit rows.
template <typename T, int D, int GT, int POS>
struct CaSums {
  using W = CaWarp<T, D, GT, POS>;
  using X = Dec16<T>;
  static constexpr int KC = D / 32, VC = D / 64;
  // Queries in shared memory, rows of kQ bytes: eight lanes that read 16 bytes each touch every bank once.
  static constexpr uint32_t kQ = D * 2 + 64;
  uint32_t q;
  // [channel octet's element][fragment rows g, g + 8]: channels of two of the octets.  Each tile's products are added to
  // them on the fp32 pipe, which rounds to nearest; the tensor core's own accumulation cuts off, and over 131072 rows that
  // came to 2e-6 of the output (2.2e-7 this way).
  unsigned long long o[VC * 8][2];
  float m, z;                              // of head g % GT: m over the warp's rows, z over this lane's
  float slope;

  __device__ __forceinline__ void start(const CacheAttendParams& p, uint32_t q_shared, int heads, int hq) {
    const int lane = threadIdx.x & 31, g = (lane >> 2) % GT, c = lane & 3;
    const bool there = g < heads;
    q = q_shared + g * kQ + c * 16;
    slope = POS == 2 && there ? p.slopes[hq + g] * 1.4426950408889634f : 0.f;
#pragma unroll
    for (int i = 0; i < VC * 8; ++i) o[i][0] = o[i][1] = 0ull;
    m = -INFINITY;
    z = 0.f;
  }

  // seen: bit r for row r of the tile; far: lane r (and r + 16) has row r's distance.
  __device__ __forceinline__ void step(const CacheAttendParams& p, uint32_t k_at, uint32_t v_at, uint32_t seen, uint32_t far) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    float x[2][2], mx;
    float s0[2][4], s1[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) s0[t][e] = s1[t][e] = 0.f;
#pragma unroll
    for (int j = 0; j < KC; ++j) {
      const uint4 qj = dec_lds16(q + j * 64);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint4 k = dec_lds16(k_at + (t * 8 + g) * W::ROW + W::k_place(g, j * 4 + c));
        X::mma(s0[t], qj.x, qj.x, qj.y, qj.y, k.x, k.y);
        X::mma(s1[t], qj.z, qj.z, qj.w, qj.w, k.z, k.w);
      }
    }
    auto logit = [&](int t, int i) {
      const int r = t * 8 + 2 * c + i;
      float d = 0.f;
      if (POS == 2) d = __uint2float_rn(__shfl_sync(0xffffffffu, far, r));
      const float dot = t == 0 ? s0[0][i] + s1[0][i] : s0[1][i] + s1[1][i];
      return (seen >> r) & 1u ? ca_logit<POS>(p, dot, slope, d) : -INFINITY;
    };
    if (GT == 4 && p.cap_log2 != 0.f) {    // lanes g and g + 4 have the same dot products: each caps half of them
      const bool upper = g >= 4;
      const float y0 = logit(upper, 0), y1 = logit(upper, 1);
      const float o0 = __shfl_xor_sync(0xffffffffu, y0, 16), o1 = __shfl_xor_sync(0xffffffffu, y1, 16);
      x[0][0] = upper ? o0 : y0;
      x[0][1] = upper ? o1 : y1;
      x[1][0] = upper ? y0 : o0;
      x[1][1] = upper ? y1 : o1;
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) x[t][i] = logit(t, i);
    }
    mx = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1]));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    const float mn = fmaxf(m, mx);
    const float ref = mn == -INFINITY ? 0.f : mn - X::kShift;
    if (__any_sync(0xffffffffu, mn > m)) {
      const float corr = m == -INFINITY ? 0.f : ex2(m - mn);
      z *= corr;
      const unsigned long long corr2 = pack2(corr, corr);
#pragma unroll
      for (int i = 0; i < VC * 8; ++i) {
        o[i][0] = mul2(o[i][0], corr2);
        o[i][1] = mul2(o[i][1], corr2);
      }
    }
    m = mn;
    uint32_t a[2][2], low8[2];             // [rows 2c.. / 2c + 8..][fragment row g / g + 8]
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float w0 = ex2(x[t][0] - ref), w1 = ex2(x[t][1] - ref);
      z += w0 + w1;
      const uint32_t high = X::pack(w0, w1);
      const float2 hf = X::unpack(high);
      constexpr float kUp = 1 << X::kFine;
      const float r0 = (w0 - hf.x) * kUp, r1 = (w1 - hf.y) * kUp;
      const uint32_t mid = X::pack(r0, r1);
      const float2 mf = X::unpack(mid);
      const uint32_t low = X::pack(r0 - mf.x, r1 - mf.y);
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
        float d0[4] = {0.f, 0.f, 0.f, 0.f}, d1[4] = {0.f, 0.f, 0.f, 0.f};
        X::mma(d0, a[0][0], a[0][1], a[1][0], a[1][1], e0, e1);
        X::mma(d1, a[0][0], a[0][1], a[1][0], a[1][1], f0, f1);
        if (GT == 8) {
          X::mma(d0, 0u, low8[0], 0u, low8[1], e0, e1);
          X::mma(d1, 0u, low8[0], 0u, low8[1], f0, f1);
        }
        unsigned long long* to = o[j * 8 + 2 * w];
        to[0] = add2(to[0], pack2(d0[0], d0[1]));
        to[1] = add2(to[1], pack2(d0[2], d0[3]));
        to = o[j * 8 + 2 * w + 1];
        to[0] = add2(to[0], pack2(d1[0], d1[1]));
        to[1] = add2(to[1], pack2(d1[2], d1[3]));
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
    // fragment rows g and g + 8 together, the middle and low parts with their factor taken off
    constexpr float kDown = 1.f / (1 << X::kFine);
    const float top = GT == 4 && g >= 4 ? kDown : 1.f;
    auto join = [&](const unsigned long long (&x)[2]) {
      if (X::kFine == 0) return add2(x[0], x[1]);
      return fma2(x[1], pack2(kDown, kDown), mul2(x[0], pack2(top, top)));
    };
    if (GT == 4) {
      // Lanes g and g + 4 hold parts of the same sums: each keeps one of the channel octets 64 j + 8 (2c + e) + 0 .. 7 of head g % 4
      const bool upper = g >= 4;
#pragma unroll
      for (int j = 0; j < VC; ++j) {
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float s0, s1;
          unpack2(join(o[j * 8 + i]), s0, s1);
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
          unpack2(join(o[j * 8 + i]), t[0][i], t[1][i]);
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

// fp32 rows.  Lane l has channels of quarter l / 8 of row l % 8 for the dot products, and channels 4 (l % PIECES) .. of the rows of
// parity l / PIECES (all rows where a row has 32 pieces) for the weighted sums.
template <int D, int GT, int POS>
struct CaSums<float, D, GT, POS> {
  using W = CaWarp<float, D, GT, POS>;
  static constexpr int PIECES = W::PIECES, VR = W::ROWS_AT_ONCE;
  static_assert(W::TR == 8, "");
  const float* q0;                         // shared memory: [GT][D], zeros for heads that are not there
  unsigned long long o[GT][2];
  float m[GT], z[GT];                      // m the same in all lanes; z of this lane's row

  __device__ __forceinline__ void start(const CacheAttendParams&, const float* q_shared, int, int) {
    q0 = q_shared;
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      o[g][0] = o[g][1] = 0ull;
      m[g] = -INFINITY;
      z[g] = 0.f;
    }
  }

  __device__ __forceinline__ void step(const CacheAttendParams& p, uint32_t k_at, uint32_t v_at, uint32_t seen, uint32_t far) {
    const int lane = threadIdx.x & 31, row = lane & 7, part = lane >> 3;
    unsigned long long d2[GT][2];
#pragma unroll
    for (int g = 0; g < GT; ++g) d2[g][0] = d2[g][1] = 0ull;
#pragma unroll
    for (int j = 0; j < PIECES / 4; ++j) {
      const int piece = part * (PIECES / 4) + j;
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
    const float d = POS == 2 ? __uint2float_rn(far) : 0.f;        // lane l has row l % 8's
    float w[GT];
#pragma unroll
    for (int g = 0; g < GT; ++g) {
      float a, b;
      unpack2(add2(d2[g][0], d2[g][1]), a, b);
      float dot = a + b;
      dot += __shfl_xor_sync(0xffffffffu, dot, 8);
      dot += __shfl_xor_sync(0xffffffffu, dot, 16);
      const float slope = POS == 2 ? q0[GT * D + g] : 0.f;        // (behind the queries)
      const float x = live ? ca_logit<POS>(p, dot, slope, d) : -INFINITY;
      float mx = x;
#pragma unroll
      for (int s = 4; s > 0; s >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
      const float mn = fmaxf(m[g], mx);
      if (mn > m[g]) {                     // the same in all lanes
        const float corr = m[g] == -INFINITY ? 0.f : exp2f(m[g] - mn);
        const unsigned long long corr2 = pack2(corr, corr);
        z[g] *= corr;
        o[g][0] = mul2(o[g][0], corr2);
        o[g][1] = mul2(o[g][1], corr2);
        m[g] = mn;
      }
      w[g] = exp2f(x - (mn == -INFINITY ? 0.f : mn));
      z[g] += w[g];
    }
#pragma unroll
    for (int r0 = 0; r0 < W::TR; r0 += VR) {
      const int r = r0 + lane / PIECES;
      const uint4 raw = dec_lds16(v_at + r * W::ROW + W::v_place(r, lane % PIECES));
      const unsigned long long v0 = pack2(__uint_as_float(raw.x), __uint_as_float(raw.y));
      const unsigned long long v1 = pack2(__uint_as_float(raw.z), __uint_as_float(raw.w));
#pragma unroll
      for (int g = 0; g < GT; ++g) {
        const float wr = __shfl_sync(0xffffffffu, w[g], r);
        const unsigned long long w2 = pack2(wr, wr);
        o[g][0] = fma2(w2, v0, o[g][0]);
        o[g][1] = fma2(w2, v1, o[g][1]);
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
      for (int s = 4; s > 0; s >>= 1) z[g] += __shfl_xor_sync(0xffffffffu, z[g], s);
      float t[4];
      unpack2(o[g][0], t[0], t[1]);
      unpack2(o[g][1], t[2], t[3]);
      if (VR == 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] += __shfl_xor_sync(0xffffffffu, t[e], 16);
      if (lane < PIECES) *reinterpret_cast<float4*>(acc + g * W::HEAD + lane * 4) = make_float4(t[0], t[1], t[2], t[3]);
      if (lane == 0) {
        m_out[g] = m[g];
        z_out[g] = z[g];
      }
    }
  }
};

// Factor of sums that are relative to 2^m in sums relative to 2^largest.
__device__ __forceinline__ float ca_factor(float m, float largest) { return m == -INFINITY ? 0.f : exp2f(m - largest); }

// Writes four channels of a head's output: acc and z are relative to 2^m.  A sum of zero means that no row was seen.
__device__ __forceinline__ void ca_write(const CacheAttendParams& p, int64_t head, int D, int channel, float m, float z, float4 acc) {
  float* to = p.out + head * D + channel;
  const float4 v = z == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(acc.x / z, acc.y / z, acc.z / z, acc.w / z);
  if (reinterpret_cast<uintptr_t>(p.out) % 16 == 0) {
    *reinterpret_cast<float4*>(to) = v;
  } else {                                 // (the output is as aligned as a float)
    to[0] = v.x;
    to[1] = v.y;
    to[2] = v.z;
    to[3] = v.w;
  }
  if (channel == 0 && p.lse) p.lse[head] = z == 0.f ? -INFINITY : (m + log2f(z)) * 0.6931471805599453f;
}
__device__ __forceinline__ void ca_add(float4& a, const float4& x, float f) {
  a.x = fmaf(x.x, f, a.x);
  a.y = fmaf(x.y, f, a.y);
  a.z = fmaf(x.z, f, a.z);
  a.w = fmaf(x.w, f, a.w);
}

// A unit's partial results: where they lie, in the order of its rows.
struct CaParts {
  int first, rest, count;                  // the first one, then rest + 2, rest + 4 ..
  __device__ __forceinline__ int at(int i) const { return i == 0 ? first : rest + 2 * i; }
  // More than kCaDirect are joined in groups first, each by its own last CTA: the parts of a group, and of the unit's joined groups.
  __device__ __forceinline__ int group() const { return count <= kCaDirect ? count : static_cast<int>(ceilf(sqrtf(static_cast<float>(count)))); }
};

// Parts i0, i0 + stride .. (count of them) of a unit -> its output, or (part) one partial result that takes the place of the
// first.  By one CTA.  The factors go to shared memory, to the last slots of the warps' rings in turn.  A warp finds the factors
// of a head; then every thread has four channels of a head and adds up the parts in the order of the rows, kAhead loads on their
// way at a time.  (One channel and one load at a time: 120 us for the 37 parts of 8 heads x 128 channels; 55 of them 20 us this
// way; 131072 rows x 8 KV heads x 8 query heads in all 102 us, in groups 98.)
template <typename T, int D, int GT>
__device__ __forceinline__ void ca_join(const CacheAttendParams& p, uint8_t* last_slots, uint32_t ring, const CaParts& parts, int i0, int stride,
                                        int count, int heads, int64_t head0, bool part) {
  constexpr int kAhead = 8;
  __shared__ float s_jm[GT], s_jz[GT];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto factor = [&](int i) -> float* { return reinterpret_cast<float*>(last_slots + (i % kCaWarps<T>) * ring) + i / kCaWarps<T> * GT; };
  auto partial = [&](int i) { return p.partials + static_cast<int64_t>(parts.at(i0 + i * stride)) * kCaPartial; };
  float4 x[kAhead];
  auto fetch = [&](int i, int o) {         // (the last one again behind it: loads without a condition go out together)
#pragma unroll
    for (int j = 0; j < kAhead; ++j) x[j] = __ldcg(reinterpret_cast<const float4*>(partial(min(i + j, count - 1)) + o));
  };
  fetch(0, min(static_cast<int>(threadIdx.x) * 4, heads * D - 4));               // on their way while the factors are found
  for (int g = warp; g < heads; g += kCaWarps<T>) {
    float m = -INFINITY, z0 = 0.f;
    for (int i = lane; i < count; i += 32) {
      const float mi = __ldcg(partial(i) + GT * D + g);
      if (i == lane) z0 = __ldcg(partial(i) + GT * D + GT + g);
      factor(i)[g] = mi;
      m = fmaxf(m, mi);
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
    float z = 0.f;
    for (int i = lane; i < count; i += 32) {
      const float f = ca_factor(factor(i)[g], m);
      factor(i)[g] = f;
      z = fmaf(i == lane ? z0 : __ldcg(partial(i) + GT * D + GT + g), f, z);
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) z += __shfl_xor_sync(0xffffffffu, z, s);
    if (lane == 0) {
      s_jm[g] = m;
      s_jz[g] = z;
    }
  }
  __syncthreads();
  for (int o = threadIdx.x * 4; o < heads * D; o += kCaThreads<T> * 4) {
    const int g = o / D;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < count; i += kAhead) {
      if (i > 0 || o >= kCaThreads<T> * 4) fetch(i, o);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (i + j < count) ca_add(a, x[j], factor(i + j)[g]);
      }
    }
    if (part) {
      __stcg(reinterpret_cast<float4*>(partial(0) + o), a);
    } else {
      ca_write(p, head0 + g, D, o - g * D, s_jm[g], s_jz[g], a);
    }
  }
  if (part && threadIdx.x < heads) {
    __stcg(partial(0) + GT * D + threadIdx.x, s_jm[threadIdx.x]);
    __stcg(partial(0) + GT * D + GT + threadIdx.x, s_jz[threadIdx.x]);
  }
}

// Whether this CTA is the last of `of` to arrive at a counter, which is zero again then.  Everything that the CTA wrote ahead is
// there for the last one to read.
__device__ __forceinline__ bool ca_last(int32_t* counter, int of, int32_t* s_last) {
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();                       // for the whole CTA, which the barrier has ordered before it
    *s_last = atomicAdd(counter, 1) == of - 1;
    if (*s_last) *counter = 0;             // everybody has arrived: ready for the next call
    __threadfence();
  }
  __syncthreads();
  return *s_last != 0;
}

// How the tiles of a call are dealt out.  A unit is a block of query heads of one KV head of one sequence; s_off has the tiles of
// a unit of the sequences ahead (at least one per sequence, whose rows may be none).
//   * Where there are fewer units than CTAs (and it costs next to nothing): every unit in equal parts of at most `most` tiles, one part to a
//     CTA, `most` as small as it can be.
//   * Else equal consecutive ranges of all tiles.  Starting on a unit and handing over its sums takes a CTA about as long as kCaStart
//     tiles, so that many are counted on top of each unit's own.
// (64 sequences of 129 to 4096 rows, 32 / 8 heads: 120 us without the count, equal lengths 95.  Eight sequences of 300 to 700 rows:
// 14.6 us in equal ranges, where nearly every CTA has the end of one unit and the start of another.)
constexpr int kCaStart = 2;
constexpr int kCaSpare = 3;                // tiles that parts may have more than equal ranges would
// A split has to save so many tiles in turn: handing sums over and joining them takes 2.8 us, a tile about 1 (one sequence, 8 KV
// heads, while every call took 1.1 us longer than now: 128 rows 8.8 us in two parts, 7.4 in one; 512 rows 9.2 in eight, 10.0 in
// four, 11.5 in two).
constexpr int kCaSplit = 3;

struct CaSegment {
  int b, unit;                             // sequence (-1: no segment) and unit of it: KV head * head_blocks + block
  int tile0, tile1;
  bool whole;                              // the unit's only segment
  int slot;                                // where this segment's partial result goes
  int first, rest, more;                   // where the unit's are: the first one, and rest + 2 .. rest + 2 more
};

// Lies in shared memory: one thread works it out while the others are at the sums.
struct CaPlan {
  int batch, per_seq;                      // sequences, units of each
  int b;
  int64_t begin, end, total;               // this CTA's range, and all of it
  int64_t at;                              // of the next segment; end with parts

  __device__ __forceinline__ int64_t start_of(int64_t cta) const { return total * cta / gridDim.x; }
  __device__ __forceinline__ int64_t owner(int64_t tile) const { return ((tile + 1) * gridDim.x - 1) / total; }
  // Counted tiles of the sequences ahead (the sum passes 2^31 where off comes near it).
  __host__ __device__ __forceinline__ int64_t ahead(const int32_t* off, int s) const {
    return (static_cast<int64_t>(off[s]) + int64_t{kCaStart} * s) * per_seq;
  }
};

// The next segment of this CTA's range.  One thread.
__device__ __noinline__ void ca_next(const int32_t* off, CaPlan* plan, CaSegment* s) {
  CaPlan p = *plan;
  s->b = -1;
  while (p.at < p.end) {
    while (p.at >= p.ahead(off, p.b + 1)) ++p.b;
    const int tiles = off[p.b + 1] - off[p.b], counted = tiles + kCaStart;
    const int64_t in_seq = p.at - p.ahead(off, p.b);
    const int unit = static_cast<int>(in_seq / counted);
    const int v0 = static_cast<int>(in_seq - static_cast<int64_t>(unit) * counted);
    const int v1 = static_cast<int>(min(static_cast<int64_t>(counted), v0 + (p.end - p.at)));
    const int64_t unit0 = p.at - v0;
    p.at += v1 - v0;
    const int tile0 = max(0, v0 - kCaStart), tile1 = max(0, v1 - kCaStart);
    if (tile0 == tile1) continue;
    s->b = p.b;
    s->unit = unit;
    s->tile0 = tile0;
    s->tile1 = tile1;
    s->whole = tile0 == 0 && tile1 == tiles;
    if (!s->whole) {
      // a CTA has at most one unit that it did not start (place 0) and one that it does not finish (place 1)
      const int64_t c0 = p.owner(unit0 + kCaStart);
      s->more = static_cast<int>(p.owner(unit0 + counted - 1) - c0);
      s->slot = 2 * blockIdx.x + (p.begin <= unit0 ? 1 : 0);
      s->rest = static_cast<int>(2 * c0);
      s->first = s->rest + (p.start_of(c0) <= unit0 ? 1 : 0);
    }
    break;
  }
  plan->at = p.at;
  plan->b = p.b;
}

// The plan of a call and this CTA's first two segments.  One warp.
__device__ __noinline__ void ca_plan(const int32_t* off, int batch, int per_seq, CaPlan* plan, CaSegment* seg) {
  const int lane = threadIdx.x & 31;
  const unsigned ctas = gridDim.x;
  const int64_t all = static_cast<int64_t>(off[batch]) * per_seq;
  if (lane == 0) {
    seg[0].b = seg[1].b = -1;
    plan->batch = batch;
    plan->per_seq = per_seq;
    plan->at = plan->end = 0;
    plan->b = 0;
  }
  int most = 0;                            // tiles of a part, 0: equal ranges
  if (static_cast<int64_t>(batch) * per_seq <= ctas && all < (1 << 30)) {
    int longest = 0;
    for (int s = lane; s < batch; s += 32) longest = max(longest, off[s + 1] - off[s]);
    longest = __reduce_max_sync(0xffffffffu, longest);
    if (longest <= kCaSplit) most = longest;                       // no split saves enough
    const unsigned units = batch * per_seq, tiles = static_cast<unsigned>(all);
    auto parts = [&](unsigned most) {
      unsigned sum = 0;
      for (int s = lane; s < batch; s += 32) sum += (off[s + 1] - off[s] + most - 1) / most;
      return __reduce_add_sync(0xffffffffu, sum) * per_seq;
    };
    unsigned lo = (tiles + ctas - 1) / ctas, hi = units < ctas ? (tiles + ctas - units - 1) / (ctas - units) : off[batch];
    hi = max(lo, hi);                      // parts of hi tiles fit: there are fewer than tiles / hi + units of them
    while (most == 0 && lo < hi) {
      const unsigned mid = (lo + hi) / 2;
      if (parts(mid) <= ctas) hi = mid;
      else lo = mid + 1;
    }
    if (most == 0 && static_cast<int64_t>(hi) * ctas <= all + static_cast<int64_t>(kCaSpare) * ctas)
      most = longest < static_cast<int>(hi) + kCaSplit ? longest : static_cast<int>(hi);
  }
  __syncwarp();
  if (most == 0) {
    if (lane) return;
    plan->total = plan->ahead(off, batch);
    plan->at = plan->begin = plan->start_of(blockIdx.x);
    plan->end = plan->start_of(blockIdx.x + 1);
    int b = 0;
    for (int step = PKV_MAX_CACHE_BATCH / 2; step > 0; step >>= 1)   // the last sequence that starts at or before `at`
      if (b + step < batch && plan->ahead(off, b + step) <= plan->at) b += step;
    plan->b = b;
    ca_next(off, plan, &seg[0]);
    ca_next(off, plan, &seg[1]);
    return;
  }
  const int cta = static_cast<int>(blockIdx.x);
  int run = 0;                             // parts of the sequences ahead
  for (int s0 = 0; s0 < batch; s0 += 32) {
    const int x = s0 + lane < batch ? (off[s0 + lane + 1] - off[s0 + lane] + most - 1) / most : 0;
    int sum = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    const unsigned past = __ballot_sync(0xffffffffu, (run + sum) * per_seq > cta);
    if (past) {
      if (lane == __ffs(past) - 1) {
        const int b = s0 + lane, tiles = off[b + 1] - off[b], in_seq = cta - (run + sum - x) * per_seq;
        const int unit = in_seq / x, k = in_seq - unit * x;
        seg[0].b = b;
        seg[0].unit = unit;
        const int each = tiles / x, longer = tiles - each * x;   // the first ones have a tile more
        seg[0].tile0 = k * each + min(k, longer);
        seg[0].tile1 = seg[0].tile0 + each + (k < longer ? 1 : 0);
        seg[0].whole = x == 1;
        seg[0].slot = 2 * cta;
        seg[0].first = seg[0].rest = 2 * (cta - k);
        seg[0].more = x - 1;
      }
      return;
    }
    run += __shfl_sync(0xffffffffu, sum, 31);
  }
}

// grid: any number of CTAs up to kCaMaxGrid; block kCaThreads; dynamic shared memory: a ring per warp, and twice a segment's
// queries (GT rows of 2 D + 64 bytes; fp32: GT * (D + 4) floats, slopes behind them).
template <typename T, int D, int GT, int POS>
__global__ void __launch_bounds__(kCaThreads<T>, sizeof(T) == 4 ? 1 : kCaPerSm) cache_attend_kernel(const __grid_constant__ CacheAttendParams p) {
  using W = CaWarp<T, D, GT, POS>;
  using Sums = CaSums<T, D, GT, POS>;
  constexpr uint32_t kSlot = 2 * W::TILE;
  constexpr int WARPS = kCaWarps<T>, THREADS = kCaThreads<T>;
  static_assert(GT * W::HEAD * 4 <= kSlot, "a warp's sums fit the last slot of its ring");
  static_assert((kCaMaxGrid + WARPS - 1) / WARPS * GT * 4 <= kSlot, "and the factors of a join all warps' last slots");
  extern __shared__ __align__(128) uint8_t ca_smem[];
  __shared__ int32_t s_off[PKV_MAX_CACHE_BATCH + 1];             // tiles of a unit of the sequences ahead
  __shared__ int32_t s_scan[WARPS];
  __shared__ float s_m[WARPS][GT], s_z[WARPS][GT];
  __shared__ int32_t s_last;
  __shared__ CaPlan s_plan;
  __shared__ CaSegment s_seg[3];         // the segment that is worked on, the next one and the one after it, in turn
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int most = static_cast<int>(static_cast<int64_t>(p.max_pages) * p.page_size);      // the host keeps it below 2^30
  pdl_wait();

  // ---- tiles of every sequence and their running sum
  auto tiles_of = [&](int b) { return max(1, (min(max(p.lens[b], 0), most) + kCaTile - 1) / kCaTile); };
  if (p.batch <= 32) {                     // every warp for itself: all write the same
    const int x = lane < p.batch ? tiles_of(lane) : 0;
    int run = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += y;
    }
    if (lane < p.batch) s_off[lane + 1] = run;
    if (lane == 0) s_off[0] = 0;
    __syncwarp();
  } else {
    const int per = (p.batch + THREADS - 1) / THREADS;           // consecutive sequences of a thread
    int sum = 0;
    for (int i = 0, b = tid * per; i < per && b < p.batch; ++i, ++b) sum += tiles_of(b);
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += y;
    }
    if (lane == 31) s_scan[warp] = run;
    __syncthreads();
    for (int w = 0; w < warp; ++w) run += s_scan[w];
    run -= sum;
    for (int i = 0, b = tid * per; i < per && b < p.batch; ++i, ++b) {
      s_off[b] = run;
      run += tiles_of(b);
    }
    if (tid == THREADS - 1) s_off[p.batch] = run;
    __syncthreads();
  }
  if (warp == 0) ca_plan(s_off, p.batch, p.num_kv_heads * p.head_blocks, &s_plan, s_seg);
  __syncthreads();
  if (s_seg[0].b < 0) return;

  const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(ca_smem)) + warp * static_cast<uint32_t>(W::kRing);
  constexpr uint32_t kAcc = (kCaStages - 1) * kSlot;             // the warp's sums: in the last slot of its ring
  CaRows<POS> rows;
  const T* q0;
  int first, heads, which = 0;
  uint32_t seen[kCaStages], far[kCaStages];                      // of the tiles in the ring, oldest first
  int mine_last, next;                                           // where the rows of the last slot's tile lie, and the next one's
  int next_pos;
  int q_buffer = 0;
  Sums sums;
  // Rows are looked up in two steps, a tile apart: a row's place, then its position.  Lane l has row l % TR.
  auto place = [&](int t0) { return ca_place<POS>(p, rows, t0 + lane % W::TR, lane < W::TR); };
  auto position = [&](int at) { return POS && at >= 0 ? p.pos_pool[at] : 0; };
  auto check = [&](int at, int pos, uint32_t* f) -> int {                          // the place, -1 if the row is not seen
    *f = 0;
    return POS && at >= 0 && !ca_seen<POS>(p, rows, pos, f) ? -1 : at;
  };
  constexpr uint32_t kRowBits = W::TR == 32 ? 0xffffffffu : (1u << W::TR) - 1u;
  auto copy_in = [&](uint32_t slot, uint32_t there, int mine) {
    if (there) W::copy_tile(p, ring + slot, mine);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // Starts on a segment: the tiles of all slots but the last one are on their way.
  auto begin = [&](const CaSegment& seg) {
    const int h = seg.unit / p.head_blocks, g0 = (seg.unit - h * p.head_blocks) * GT;
    const int hq = h * p.group + g0;
    heads = min(GT, p.group - g0);
    q0 = static_cast<const T*>(p.q) + seg.b * p.q_sb + hq * p.q_sh;
    rows.table = p.table + (static_cast<int64_t>(seg.b) * p.num_kv_heads + h) * p.max_pages;
    rows.rows = min(min(max(p.lens[seg.b], 0), most), seg.tile1 * kCaTile);
    rows.q_pos = POS ? p.q_pos[seg.b] : 0;
    first = seg.tile0 * kCaTile + warp * W::TR;
    // the queries: a 16-byte piece to a thread, on its way while the rows are looked up
    constexpr int kPiece = 16 / static_cast<int>(sizeof(T)), kPieces = GT * D / kPiece;
    static_assert(kPieces <= THREADS, "");
    const int q_head = tid / (D / kPiece), q_piece = tid % (D / kPiece);
    uint4 q_mine = make_uint4(0, 0, 0, 0);
    if (q_head < heads) q_mine = *reinterpret_cast<const uint4*>(q0 + q_head * p.q_sh + q_piece * kPiece);
    int mine[kCaStages];
    int pos[kCaStages];
#pragma unroll
    for (int s = 0; s < kCaStages; ++s) mine[s] = place(first + s * kCaTile);
    next = place(first + kCaStages * kCaTile);
#pragma unroll
    for (int s = 0; s < kCaStages; ++s) pos[s] = position(mine[s]);
    next_pos = position(next);
#pragma unroll
    for (int s = 0; s < kCaStages; ++s) {
      mine[s] = check(mine[s], pos[s], &far[s]);
      seen[s] = __ballot_sync(0xffffffffu, mine[s] >= 0) & kRowBits;
      if (s < kCaStages - 1) copy_in(s * kSlot, seen[s], mine[s]);
    }
    mine_last = mine[kCaStages - 1];
    q_buffer ^= 1;
    if constexpr (sizeof(T) == 4) {
      float* q_shared = reinterpret_cast<float*>(ca_smem + WARPS * W::kRing) + q_buffer * (GT * (D + 4));
      if (tid < kPieces) reinterpret_cast<uint4*>(q_shared)[tid] = q_mine;
      if (POS == 2 && tid < GT) q_shared[GT * D + tid] = tid < heads ? p.slopes[hq + tid] * 1.4426950408889634f : 0.f;
      sums.start(p, q_shared, heads, hq);
    } else {
      uint8_t* q_shared = ca_smem + WARPS * W::kRing + q_buffer * (GT * Sums::kQ);
      if (tid < kPieces) *reinterpret_cast<uint4*>(q_shared + q_head * Sums::kQ + q_piece * 16) = q_mine;
      sums.start(p, static_cast<uint32_t>(__cvta_generic_to_shared(q_shared)), heads, hq);
    }
  };
  begin(s_seg[0]);
  __syncthreads();                         // the queries are there
  while (true) {
    copy_in(kAcc, seen[kCaStages - 1], mine_last);
    const int next_seg = which == 2 ? 0 : which + 1;
    if (tid == THREADS - 1) ca_next(s_off, &s_plan, &s_seg[3 - which - next_seg]);       // (while the rows come)
    int second = place(first + (kCaStages + 1) * kCaTile);   // one tile further

    // ---- the warp's rows
    uint32_t slot = 0;
    for (int t0 = first; t0 < rows.rows; t0 += kCaTile) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kCaStages - 1) : "memory");
      __syncwarp();
      if (seen[0]) sums.step(p, ring + slot, ring + slot + W::TILE, seen[0], far[0]);
      __syncwarp();                        // the tile has been read
#pragma unroll
      for (int s = 0; s + 1 < kCaStages; ++s) {
        seen[s] = seen[s + 1];
        far[s] = far[s + 1];
      }
      const int mine = check(next, next_pos, &far[kCaStages - 1]);
      seen[kCaStages - 1] = __ballot_sync(0xffffffffu, mine >= 0) & kRowBits;
      copy_in(slot, seen[kCaStages - 1], mine);
      next = second;
      next_pos = position(next);
      second = place(t0 + (kCaStages + 2) * kCaTile);
      slot = slot == kAcc ? 0 : slot + kSlot;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    sums.finish(p, rows, q0, heads, first, reinterpret_cast<float*>(ca_smem + warp * W::kRing + kAcc), s_m[warp], s_z[warp]);

    // ---- the next segment's rows start on their way, then the warps' sums meet
    const CaSegment& was = s_seg[which];
    const int heads_was = heads;
    const bool have = s_seg[next_seg].b >= 0;
    if (have) begin(s_seg[next_seg]);
    __syncthreads();
    const int h_was = was.unit / p.head_blocks;
    const int64_t head0 = (static_cast<int64_t>(was.b) * p.num_kv_heads + h_was) * p.group + (was.unit - h_was * p.head_blocks) * GT;
    // the output, or a partial result that the unit's last CTA joins with the others
    float* part = p.partials + static_cast<int64_t>(was.slot) * kCaPartial;
    for (int o = tid * 4; o < heads_was * D; o += THREADS * 4) {
      const int g = o / D, channel = o - g * D;
      float m = s_m[0][g];
#pragma unroll
      for (int w = 1; w < WARPS; ++w) m = fmaxf(m, s_m[w][g]);
      float z = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float f = ca_factor(s_m[w][g], m);
        z = fmaf(s_z[w][g], f, z);
        ca_add(a, *reinterpret_cast<const float4*>(ca_smem + w * W::kRing + kAcc + (g * W::HEAD + channel) * 4), f);
      }
      if (was.whole) {
        ca_write(p, head0 + g, D, channel, m, z, a);
      } else {
        __stcg(reinterpret_cast<float4*>(part + o), a);
        if (channel == 0) {
          __stcg(part + GT * D + g, m);
          __stcg(part + GT * D + GT + g, z);
        }
      }
    }
    if (!was.whole) {
      const CaParts parts{was.first, was.rest, was.more + 1};
      const int group = parts.group(), groups = (parts.count + group - 1) / group;
      const int mine = was.slot == was.first ? 0 : (was.slot - was.rest) / 2, i0 = mine / group * group;
      const uint32_t ring_bytes = static_cast<uint32_t>(W::kRing);
      int32_t* unit_counter = p.counters + static_cast<int64_t>(was.b) * s_plan.per_seq + was.unit;
      if (groups == 1) {
        if (ca_last(unit_counter, parts.count, &s_last))
          ca_join<T, D, GT>(p, ca_smem + kAcc, ring_bytes, parts, 0, 1, parts.count, heads_was, head0, false);
      } else if (ca_last(p.group_counters + parts.at(i0), min(group, parts.count - i0), &s_last)) {
        ca_join<T, D, GT>(p, ca_smem + kAcc, ring_bytes, parts, i0, 1, min(group, parts.count - i0), heads_was, head0, true);
        if (ca_last(unit_counter, groups, &s_last))
          ca_join<T, D, GT>(p, ca_smem + kAcc, ring_bytes, parts, 0, group, groups, heads_was, head0, false);
      }
    }
    if (!have) return;
    __syncthreads();                       // the sums have been read: the last slot may be filled
    which = next_seg;
  }
}

}  // namespace pkv
