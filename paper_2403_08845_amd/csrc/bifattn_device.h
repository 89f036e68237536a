// Device helpers shared by the library's HIP kernels: vector types, the bf16
// matrix instructions, reductions across a wave and raw buffer loads.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace bifattn {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;  // LDS-qualified operand slot

constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ f32x4 mfma_bf16(const u32x4& a, const u32x4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  bf16x2 v = {(__bf16)lo, (__bf16)hi};  // round to nearest even
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Cross-row exchanges without a trip through LDS: v_permlane16_swap and
// v_permlane32_swap of a register with itself return, in their two results,
// the lane's own value and the value of lane l^16 (l^32), in an order that
// depends on the row; max / sum of the two is the same in every lane. The
// two vector elements are copied to scalars before the float reinterpret:
// __builtin_bit_cast applied to an element of the result vector reads
// element 0 whatever the index.
template <bool kWide>
__device__ __forceinline__ void swap_halves(float x, float& a, float& b) {
  const unsigned u = __float_as_uint(x);
  const auto r = kWide ? __builtin_amdgcn_permlane32_swap(u, u, false, false)
                       : __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const unsigned r0 = r[0], r1 = r[1];
  a = __uint_as_float(r0);
  b = __uint_as_float(r1);
}
__device__ __forceinline__ float xor16_max(float x) {
  float a, b;
  swap_halves<false>(x, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float xor32_max(float x) {
  float a, b;
  swap_halves<true>(x, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float xor16_sum(float x) {
  float a, b;
  swap_halves<false>(x, a, b);
  return a + b;
}
__device__ __forceinline__ float xor32_sum(float x) {
  float a, b;
  swap_halves<true>(x, a, b);
  return a + b;
}
// Whole-wave reductions: permlane swaps across rows, then shuffles in a row.
__device__ __forceinline__ float wave_max(float x) {
  x = xor32_max(xor16_max(x));
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
  x = xor32_sum(xor16_sum(x));
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// Wave index within the work-group, as a wave-uniform (scalar) value so that
// branches on it and on tile bounds derived from it stay scalar.
__device__ __forceinline__ int wave_id() {
  return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}

__device__ __forceinline__ u32x4 load16(const uint16_t* p) {
  return *reinterpret_cast<const u32x4*>(p);
}

// Byte offsets into a buffer resource are formed in 32-bit unsigned
// arithmetic: prefetches past the end of a cache near the 2^31-byte limit may
// wrap, which is well defined here and lands outside the resource's range
// (or inside it, on bytes that are never consumed), where a raw buffer load
// returns zeros or valid memory and never faults.
__device__ __forceinline__ int boff(uint32_t x) { return __builtin_bit_cast(int, x); }

// Cache policy of the loads that stream a cache: every byte of the decode
// cache, and of the context on the few-row path, is read exactly once per
// step, so those loads are non-temporal (the nt bit: streamed past the caches
// instead of displacing lines). Measured on MI355X over 402 MB of loads-only
// regions: 6.0 TB/s with the default policy, 6.7 TB/s with nt.
constexpr int kAuxStream = 2;

// N bytes a lane loads with one buffer instruction (cache policy AUX), and
// 32-bit word w of them.
template <int N> struct Raw;
template <> struct Raw<16> {
  typedef u32x4 type;
  template <int AUX = 0>
  static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, int off) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, AUX);
  }
  static __device__ __forceinline__ type zero() { return u32x4{0, 0, 0, 0}; }
  static __device__ __forceinline__ uint32_t word(const type& v, int w) { return v[w]; }
};
template <> struct Raw<8> {
  typedef u32x2 type;
  template <int AUX = 0>
  static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, int off) {
    return __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, AUX);
  }
  static __device__ __forceinline__ type zero() { return u32x2{0, 0}; }
  static __device__ __forceinline__ uint32_t word(const type& v, int w) { return v[w]; }
};
template <> struct Raw<4> {
  typedef uint32_t type;
  template <int AUX = 0>
  static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, int off) {
    return __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, AUX);
  }
  static __device__ __forceinline__ type zero() { return 0u; }
  static __device__ __forceinline__ uint32_t word(const type& v, int) { return v; }
};
template <> struct Raw<2> {
  typedef uint32_t type;
  template <int AUX = 0>
  static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, int off) {
    return __builtin_amdgcn_raw_buffer_load_b16(r, off, 0, AUX);
  }
  static __device__ __forceinline__ type zero() { return 0u; }
  static __device__ __forceinline__ uint32_t word(const type& v, int) { return v; }
};

}  // namespace
}  // namespace bifattn
