// What the kernels of decode attention share: mma.sync on 16-bit rows, softmax weights in 16-bit parts, asynchronous copies.
#pragma once

#include "pkv_common.cuh"

namespace pkv {

// 16-bit types of the matrix products.  A softmax weight w 2^kShift (w <= 1) is taken apart into a high part and, of what that leaves
// times 2^kFine, a middle and a low one; sums of the latter two are multiplied by 2^-kFine at the end.
//   bfloat16: the range of fp32, so that the three parts carry 24 bits of every weight.
//   fp16: its smallest step is 2^-24, and without a factor of their own the lower parts of small weights would be subnormal (11 bits
//   left of a weight of 2^-27).  With 2^13 on the weight and 2^13 more on what the high part leaves (at most 2^1, so 2^14 of
//   the largest 2^16) the parts are off by 2^-25 of the weight or 2^-51 of the largest one, whichever is more: 24 bits of weights
//   down to 2^-27.
template <typename T>
struct Dec16;
template <>
struct Dec16<__nv_bfloat16> {
  static constexpr float kShift = 0.f;
  static constexpr int kFine = 0;
  __device__ __forceinline__ static uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  __device__ __forceinline__ static float2 unpack(uint32_t u) {
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  }
  __device__ __forceinline__ static void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};
template <>
struct Dec16<__half> {
  static constexpr float kShift = 13.f;
  static constexpr int kFine = 13;
  __device__ __forceinline__ static uint32_t pack(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  __device__ __forceinline__ static float2 unpack(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
  __device__ __forceinline__ static void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};

// Bytes from global to shared memory past the registers, zeros where `there` is false.
__device__ __forceinline__ void dec_copy16(uint32_t to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16u : 0u) : "memory");
}
__device__ __forceinline__ uint4 dec_lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

}  // namespace pkv
