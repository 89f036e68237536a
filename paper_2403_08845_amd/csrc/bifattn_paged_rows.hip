// Rows in and out of paged caches for gfx950: the append of new tokens (the
// position rotation of queries and keys, the encoding of keys and values, the
// scatter into pages) and the read-out of rows as bf16.
#include <hip/hip_ext.h>

#include "bifattn_device.h"
#include "bifattn_paged.h"

namespace bifattn {
namespace {

constexpr int kAppendThreads = 256;

// x rounded to odd: to fp32 toward zero, with the last bit set when anything
// was cut off. Rounding that to a type of at most 22 significant bits gives
// the rounding of x itself, ties and borders included.
__device__ __forceinline__ float odd_f32(double x) {
  const float f = (float)x;
  const double back = (double)f;
  if (back == x || !(fabs(x) <= 3.4e38)) return f;
  const uint32_t u = __float_as_uint(f) - (fabs(back) > fabs(x) ? 1u : 0u);
  return __uint_as_float(u | 1u);
}

__device__ __forceinline__ u32x4 to_bf16(const float* f) {
  u32x4 r;
#pragma unroll
  for (int w = 0; w < 4; ++w) r[w] = pack_bf16(f[2 * w], f[2 * w + 1]);
  return r;
}

// cos and sin of an angle, each as a part of 16 significant bits and the rest
// (about 40 bits together): ch, cl, sh, sl; and in 64 bits.
typedef f32x4 Turn;
typedef double FullTurn __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void two_parts(double v, float& hi, float& lo) {
  hi = __uint_as_float(__float_as_uint((float)v) & 0xffffff00u);
  lo = (float)(v - (double)hi);
}
// (x cos - y sin, x sin + y cos) of bf16 values. x * ch and y * sh have at most
// 24 bits, so y * sh is exact and the fused product rounds the exact main part
// once: the result is off by 2^-22 of itself and, which shows where the terms
// cancel, by 2^-37 of |x| + |y|: the rest (2^-15 of the terms) is cut and formed
// with 24 bits, and the main part may exceed the result by as much. The rest of
// an infinite element has no meaning; it is kept finite (a finite element's is
// below 2^113), so that the main part decides.
__device__ __forceinline__ float finite_rest(float r) { return __builtin_amdgcn_fmed3f(r, -0x1p120f, 0x1p120f); }
__device__ __forceinline__ void rotate(float& x, float& y, const Turn& a) {
  const float p = __builtin_fmaf(x, a[0], -(y * a[2])) + finite_rest(__builtin_fmaf(x, a[1], -(y * a[3])));
  y = __builtin_fmaf(x, a[2], y * a[0]) + finite_rest(__builtin_fmaf(x, a[3], y * a[1]));
  x = p;
}
// The same in 64 bits, then rounded to odd, for codes: an element next
// to a border between two codes falls on its side, where it is 2^-50 of |x| + |y| or
// more away from it.
template <typename R> __device__ __forceinline__ void rotate_odd(float& x, float& y, const FullTurn& a, const R& rounded) {
  const double u = x, v = y;
  x = rounded(u * a[0] - v * a[1]);
  y = rounded(u * a[1] + v * a[0]);
}
// x / scale, rounded to odd: the fp32 value f near x times the rounded reciprocal
// is compared with the quotient itself by f * scale (48 bits, exact), which that
// product misses where it is short (147 / 49 is 3). Past fp32's range the largest
// value, which saturates as a code; NaN stays.
struct OddQuotient {
  double scale, inv;
  __device__ __forceinline__ float operator()(double x) const {
    const float f = (float)(x * inv);
    const double back = (double)f * scale;
    if (back == x) return f;
    const uint32_t u = __float_as_uint(f) - (fabs(back) > fabs(x) ? 1u : 0u);
    return __uint_as_float(u | 1u);
  }
};
// Two chunks of 8 whose elements rotate with `turn`: with each other, or in
// neighbouring pairs.
template <typename T, typename F>
__device__ __forceinline__ void rotate_chunks(float* x, float* y, const T* a, bool neighbours, F&& turn) {
  if (neighbours) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      turn(x[2 * e], x[2 * e + 1], a[e]);
      turn(y[2 * e], y[2 * e + 1], a[4 + e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) turn(x[e], y[e], a[e]);
  }
}

// Eight OCP E4M3 codes, saturated at +-448 (NaN stays NaN).
__device__ __forceinline__ u32x2 to_fp8(const float* x) {
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = x[e] > 448.f ? 448.f : (x[e] < -448.f ? -448.f : x[e]);
  u32x2 r;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * w], f[4 * w + 1], 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * w + 2], f[4 * w + 3], v, true);
    r[w] = (uint32_t)v;
  }
  return r;
}

// Biased exponent of the largest of 8 magnitudes, 255 when one is not finite.
__device__ __forceinline__ int top_exponent(const float* f) {
  uint32_t t = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) t = max(t, __float_as_uint(f[e]) & 0x7fffffffu);
  return (int)(t >> 23);
}
// Scale byte of a block whose largest magnitude has that exponent: 2^(byte -
// 127) with byte - 127 = floor(log2(largest)) - 2 within [-126, 127] (the
// largest E2M1 value is 1.5 * 2^2), 255 for a block that is not finite.
__device__ __forceinline__ uint32_t scale_byte(int top) { return top == 255 ? 255u : (uint32_t)max(1, top - 2); }
// Eight E2M1 codes of f 2^(127 - byte), to nearest even, saturated at 6.
__device__ __forceinline__ uint32_t to_mx4(const float* f, uint32_t byte) {
  const float s = __uint_as_float(byte << 23);
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[0], f[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[2], f[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[4], f[5], s, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[6], f[7], s, 3);
  return r;
}
__device__ __forceinline__ void widen8(const u32x4& r, float* f) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[2 * w] = __uint_as_float(r[w] << 16);
    f[2 * w + 1] = __uint_as_float(r[w] & 0xffff0000u);
  }
}

// Append. Work-group: sample i, tokens_per_block tokens, heads_per_block of the
// h query rows, g key rows and g value rows of each. A row is d/16 threads'
// work, each two chunks of 8 elements that rotate with each other.
//
// The angle of a pair is position * freq in 64 bits, off by 2^-51 of itself
// (positions reach 2^30 and an fp32 product is off by 2^-24 of a turn per turn: 0.06
// of a radian at 10^6), formed once per token and pair and kept in LDS. Rotated
// queries and bf16 keys are off by 2^-22 of themselves and 2^-37 of |x| + |y| before
// their one rounding, codes are formed from 64 bits.
//
// Byte work where the batch is large (8192 tokens of 32 + 8 heads into MXFP4:
// 46 us for 177 MB, 3.8 TB/s, of which a copy takes 35); a step of some tokens is
// one launch's latency (a chain of loads: length, table entry, row; 32 samples of
// 32 heads 4.4 us).
template <int D, int KV>
__global__ __launch_bounds__(kAppendThreads) __attribute__((amdgpu_waves_per_eu(4))) void append_kernel(PagedAppendParams A) {
  constexpr int TPR = D / 16;                       // threads of a row
  constexpr int ROWS = kAppendThreads / TPR;        // rows in flight
  constexpr int RB = paged_row_bytes(D, KV), EB = D / kMxBlock;
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn[];
  Turn* turn = reinterpret_cast<Turn*>(dyn);  // [tokens_per_block][rot/2]
  FullTurn* full = reinterpret_cast<FullTurn*>(dyn) + A.tokens_per_block * (A.rot / 2);  // the same, for codes
  __shared__ int tops[ROWS][D / 8];
  const int per = A.token_blocks * A.head_blocks;
  const int i = blockIdx.x / per, in = blockIdx.x - i * per;
  const int tb = in / A.head_blocks, hb = in - tb * A.head_blocks;
  const int raw = A.lens[i];
  const int start = raw < 0 ? 0 : min(raw, A.max_rows);
  const int rawn = A.counts ? A.counts[i] : A.n;
  const int count = rawn < 0 ? 0 : min(rawn, A.n);
  const int fit = min(count, A.max_rows - start);
  if (in == 0 && threadIdx.x == 0 && (raw != start || rawn != count || fit != count)) atomicOr(A.status, kStatusLens);
  const int t0 = tb * A.tokens_per_block, t1 = min(min(A.n, t0 + A.tokens_per_block), count);
  const int half = A.rot / 2;
  for (int k = threadIdx.x; k < (t1 - t0) * half; k += kAppendThreads) {
    const int t = k / half, j = k - t * half;
    // turns: the product with 1/(2 pi) and the fraction in 64 bits
    const double rev = (double)((int64_t)A.position0 + start + t0 + t) * ((double)A.freqs[j] * 0.15915494309189533577);
    double s, c;
    sincospi(2.0 * (rev - rint(rev)), &s, &c);
    float ch, cl, sh, sl;
    two_parts(c, ch, cl);
    two_parts(s, sh, sl);
    turn[k] = Turn{ch, cl, sh, sl};
    if constexpr (KV != kPagedBf16) full[k] = FullTurn{c, s};
  }
  __syncthreads();  // also: every thread has read lens and counts
  if (threadIdx.x == 0) {
    if (!A.in_place) {
      if (in == 0) A.lens_out[i] = start + fit;
    } else if (per == 1) {
      A.lens_out[i] = start + fit;
    } else if (atomicAdd(A.tickets + i, 1) == per - 1) {  // the others have read theirs
      A.tickets[i] = 0;
      A.lens_out[i] = start + fit;
    }
  }
  const int heads = A.h + 2 * A.g;
  const int h0 = hb * A.heads_per_block, nh = min(heads, h0 + A.heads_per_block) - h0;
  const int slot = threadIdx.x / TPR, t = threadIdx.x % TPR;
  const int mask = (1 << A.pool.shift) - 1;
  const int items = max(0, t1 - t0) * nh;
  // The chunks of a thread. Within each of the maps parts of a row: `halves`
  // pairs chunk c with c + rot/16, else both elements of a pair are neighbours.
  const int part_threads = TPR / A.maps, u = t % part_threads, base = t / part_threads * (D / 8 / A.maps);
  const int rc = A.rot / 16;  // threads with rotated chunks
  const bool turns = u < rc;
  const int c0 = base + (turns && !A.neighbours ? u : 2 * u), c1 = turns && !A.neighbours ? c0 + rc : c0 + 1;
  // Row `slot` of every pass: r-th token, head h0 + hd (kept without divisions).
  int r = slot / nh, hd = slot % nh;
  const int dr = ROWS / nh, dh = ROWS % nh;
  for (int item = slot; item < items; item += ROWS, r += dr, hd += dh) {
    if (hd >= nh) hd -= nh, ++r;
    const int head = h0 + hd, token = t0 + r;
    const bool is_q = head < A.h, is_k = !is_q && head < A.h + A.g;
    const int gam = is_q ? 0 : (is_k ? head - A.h : head - A.h - A.g);
    const int64_t* st = is_q ? A.qs : (is_k ? A.ks : A.vs);
    const uint16_t* src = (is_q ? A.q : (is_k ? A.k : A.v)) + (int64_t)i * st[0] + (is_q ? head : gam) * st[1] + token * st[2];
    const u32x4 rx = load16(src + 8 * c0), ry = load16(src + 8 * c1);
    const int first = r * half + 8 * u;  // of the pairs' angles
    float fx[8], fy[8];
    widen8(rx, fx);
    widen8(ry, fy);
    if (is_q) {
      if (turns) rotate_chunks(fx, fy, turn + first, A.neighbours, rotate);
      uint16_t* dst = A.q_out + (((size_t)i * A.h + head) * A.n + token) * D;
      *reinterpret_cast<u32x4*>(dst + 8 * c0) = to_bf16(fx);
      *reinterpret_cast<u32x4*>(dst + 8 * c1) = to_bf16(fy);
      continue;
    }
    const int row = start + token;
    if (token >= fit) continue;
    const int id = A.table[(size_t)i * A.table_pages + (row >> A.pool.shift)];
    if ((unsigned)id >= (unsigned)A.pool.num_pages) {
      if (t == 0) atomicOr(A.status, kStatusPage);
      continue;
    }
    const size_t at = ((size_t)((int64_t)id * A.g + gam) << A.pool.shift) + (row & mask);
    uint8_t* dst = (is_k ? A.pool.K : A.pool.V) + at * RB;
    const bool rotates = is_k && turns;
    if constexpr (KV == kPagedBf16) {
      if (rotates) rotate_chunks(fx, fy, turn + first, A.neighbours, rotate);
      *reinterpret_cast<u32x4*>(dst + 16 * c0) = to_bf16(fx);
      *reinterpret_cast<u32x4*>(dst + 16 * c1) = to_bf16(fy);
    } else if constexpr (KV == kPagedFp8) {
      const float* sc = is_k ? A.pool.k_scale : A.pool.v_scale;
      const float s = sc ? sc[gam] : 1.f;
      if (t == 0 && !(s >= __FLT_MIN__ && s <= __FLT_MAX__)) atomicOr(A.status, kStatusScale);
      const OddQuotient over = {(double)s, 1.0 / (double)s};
      if (rotates) {
        rotate_chunks(fx, fy, full + first, A.neighbours,
                      [&](float& x, float& y, const FullTurn& a) { rotate_odd(x, y, a, over); });
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) fx[e] = over(fx[e]), fy[e] = over(fy[e]);
      }
      *reinterpret_cast<u32x2*>(dst + 8 * c0) = to_fp8(fx);
      *reinterpret_cast<u32x2*>(dst + 8 * c1) = to_fp8(fy);
    } else {
      if (rotates)
        rotate_chunks(fx, fy, full + first, A.neighbours,
                      [&](float& x, float& y, const FullTurn& a) { rotate_odd(x, y, a, odd_f32); });
      // A block is four chunks, of several of the row's threads: their
      // exponents meet in LDS. A row's threads are neighbours in one wave,
      // whose LDS accesses execute in order.
      volatile int* ts = tops[slot];
      ts[c0] = top_exponent(fx);
      ts[c1] = top_exponent(fy);
      __builtin_amdgcn_wave_barrier();
      const int b0 = c0 / 4, b1 = c1 / 4;
      const uint32_t s0 = scale_byte(max(max(ts[4 * b0], ts[4 * b0 + 1]), max(ts[4 * b0 + 2], ts[4 * b0 + 3])));
      const uint32_t s1 = scale_byte(max(max(ts[4 * b1], ts[4 * b1 + 1]), max(ts[4 * b1 + 2], ts[4 * b1 + 3])));
      __builtin_amdgcn_wave_barrier();
      uint8_t* exps = (is_k ? A.pool.K_exp : A.pool.V_exp) + at * EB;
      *reinterpret_cast<uint32_t*>(dst + 4 * c0) = to_mx4(fx, s0);
      *reinterpret_cast<uint32_t*>(dst + 4 * c1) = to_mx4(fy, s1);
      if (c0 % 4 == 0) exps[b0] = (uint8_t)s0;
      if (c1 % 4 == 0) exps[b1] = (uint8_t)s1;
    }
  }
}

// Read-out: a thread's 8 elements of a row, widened (times the group's scale)
// to bf16, rounded once. Rows at or past a sample's length are not written. Bytes alone: 8192
// rows of 8 heads from MXFP4 9.3 us for 43 MB, 4.6 TB/s.
template <int D, int KV>
__global__ __launch_bounds__(256) void gather_kernel(PagedGatherParams P) {
  constexpr int C = D / 8, RB = paged_row_bytes(D, KV), EB = D / kMxBlock;
  const int64_t items = (int64_t)P.samples * P.pool.g * P.rows * C;
  const int mask = (1 << P.pool.shift) - 1;
  for (int64_t k = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; k < items; k += (int64_t)gridDim.x * blockDim.x) {
    const int c = (int)(k % C);
    const int64_t line = k / C;
    const int r = (int)(line % P.rows);
    const int unit = (int)(line / P.rows);
    const int i = unit / P.pool.g, gam = unit - i * P.pool.g;
    const int raw = P.lens[i], from = P.first ? P.first[i] : 0;
    const int len = raw < 0 ? 0 : min(raw, P.max_rows);
    if (c == 0 && r == 0 && gam == 0 && (raw != len || from < 0)) atomicOr(P.status, kStatusLens);
    const int64_t row = (int64_t)from + r;
    if (from < 0 || row >= len) continue;
    const int id = P.table[(size_t)i * P.table_pages + (row >> P.pool.shift)];
    if ((unsigned)id >= (unsigned)P.pool.num_pages) {
      if (c == 0) atomicOr(P.status, kStatusPage);
      continue;
    }
    const size_t at = ((size_t)((int64_t)id * P.pool.g + gam) << P.pool.shift) + ((int)row & mask);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint8_t* src = (u ? P.pool.V : P.pool.K) + at * RB;
      u32x4 w;
      if constexpr (KV == kPagedBf16) {
        w = *reinterpret_cast<const u32x4*>(src + 16 * c);
      } else if constexpr (KV == kPagedFp8) {
        const u32x2 b = *reinterpret_cast<const u32x2*>(src + 8 * c);
        const float* sc = u ? P.pool.v_scale : P.pool.k_scale;
        const float s = sc ? sc[gam] : 1.f;
        if (c == 0 && !(s >= __FLT_MIN__ && s <= __FLT_MAX__)) atomicOr(P.status, kStatusScale);
        // Code times scale has 28 bits. Rounded to fp32 first, it goes to another bf16
        // value than at once only where it meets the middle between two: then (1 in
        // 2^16) formed in 64 bits and rounded to odd.
        float f[8], p[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)b[e], false);
          const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)b[e], true);
          f[4 * e] = lo[0], f[4 * e + 1] = lo[1], f[4 * e + 2] = hi[0], f[4 * e + 3] = hi[1];
        }
        uint32_t off = 0xffffu;  // 0: a product in the middle
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = f[e] * s;
          off = min(off, (__float_as_uint(p[e]) & 0xffffu) ^ 0x8000u);
        }
        if (off == 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = odd_f32((double)f[e] * (double)s);
        }
        w = to_bf16(p);
      } else {
        const uint32_t b = *reinterpret_cast<const uint32_t*>(src + 4 * c);
        const float s = __uint_as_float((uint32_t)((u ? P.pool.V_exp : P.pool.K_exp) + at * EB)[c / 4] << 23);
        w = u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b, s, 0)),
                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b, s, 1)),
                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b, s, 2)),
                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b, s, 3))};
      }
      *reinterpret_cast<u32x4*>((u ? P.v_out : P.k_out) + (size_t)line * D + 8 * c) = w;
    }
  }
}

template <typename Prm>
hipError_t go(void (*kernel)(Prm), int grid, int block, int lds, hipStream_t stream, hipEvent_t stop, const Prm& p) {
  if (stop)
    hipExtLaunchKernelGGL(kernel, dim3(grid), dim3(block), lds, stream, nullptr, stop, 0, p);
  else
    kernel<<<grid, block, lds, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendParams& A, int kv, hipStream_t s, hipEvent_t stop) {
  const int grid = A.samples * A.token_blocks * A.head_blocks;
  const int lds = A.tokens_per_block * (A.rot / 2) * (int)(sizeof(Turn) + (kv == kPagedBf16 ? 0 : sizeof(FullTurn)));
  auto run = [&](auto kernel) { return go(kernel, grid, kAppendThreads, lds, s, stop, A); };
  if (A.d == 128) {
    if (kv == kPagedBf16) return run(append_kernel<128, kPagedBf16>);
    if (kv == kPagedFp8) return run(append_kernel<128, kPagedFp8>);
    if (kv == kPagedMxfp4) return run(append_kernel<128, kPagedMxfp4>);
  } else if (A.d == 64) {
    if (kv == kPagedBf16) return run(append_kernel<64, kPagedBf16>);
    if (kv == kPagedFp8) return run(append_kernel<64, kPagedFp8>);
    if (kv == kPagedMxfp4) return run(append_kernel<64, kPagedMxfp4>);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_paged_gather(const PagedGatherParams& P, int kv, hipStream_t s, hipEvent_t stop) {
  const int64_t items = (int64_t)P.samples * P.pool.g * P.rows * (P.d / 8);
  const int grid = (int)((items + 255) / 256 < 16384 ? (items + 255) / 256 : 16384);
  auto run = [&](auto kernel) { return go(kernel, grid, 256, 0, s, stop, P); };
  if (P.d == 128) {
    if (kv == kPagedBf16) return run(gather_kernel<128, kPagedBf16>);
    if (kv == kPagedFp8) return run(gather_kernel<128, kPagedFp8>);
    if (kv == kPagedMxfp4) return run(gather_kernel<128, kPagedMxfp4>);
  } else if (P.d == 64) {
    if (kv == kPagedBf16) return run(gather_kernel<64, kPagedBf16>);
    if (kv == kPagedFp8) return run(gather_kernel<64, kPagedFp8>);
    if (kv == kPagedMxfp4) return run(gather_kernel<64, kPagedMxfp4>);
  }
  return hipErrorInvalidValue;
}

}  // namespace bifattn
