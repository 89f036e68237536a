// Attention over paged caches for gfx950: the context that all samples share
// and every sample's own rows lie in pages of one pool, named by tables.
//
// The split is that of the contiguous kernels: work-groups turn one key range
// into an online-softmax partial (m, l, acc) per query row, the combine merges
// a row's partials. Differential heads (maps = 2) are query rows of their own:
// map u multiplies half u of q with half u of k, both maps share the value
// rows, and the combine subtracts them.
//
// MFMA layouts (lane l): 16x16x32, n = l & 15, G = l >> 4: A holds
// A[n][8G..8G+7], B holds B[8G..8G+7][n], C holds C[4G..4G+3][n]; 32x32x16,
// j = l & 31, h = l >> 5: A holds A[j][8h..8h+7], C element v is
// C[8(v/4) + 4h + v%4][j]. Logits are computed transposed, S^T = K Q^T, so the
// weights a lane holds are its own B operand of O^T = V^T P^T; V^T operands
// come from key-major rows in LDS by transposing reads.
//
// The weights enter the value product as two bf16 terms (15 bits together): the
// output is bf16, and one bf16 term alone would add an error as large as the
// output's own rounding (1.7e-3 against 1e-5). Sums, statistics and
// accumulators are fp32.
#include <hip/hip_ext.h>

#include "bifattn_device.h"
#include "bifattn_paged.h"

namespace bifattn {
namespace {

typedef __attribute__((address_space(3))) unsigned char lds_u8;
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(3))) u32x2 lds_u32x2;

constexpr int cmax(int a, int b) { return a > b ? a : b; }

// Four consecutive keys (of the 16 lanes' chunks) of one dimension: in each
// group of 16 lanes, lane i' addresses 4 elements of key i'/4, dims
// 4(i'%4).., and lane i receives dim i of the four keys.
__device__ __forceinline__ u32x2 read_tr(const unsigned char* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p));
}
__device__ __forceinline__ u32x4 read128(const unsigned char* p) { return *(const lds_u32x4*)p; }
__device__ __forceinline__ void write128(unsigned char* p, const u32x4& v) { *(lds_u32x4*)p = v; }

// Codecs, and the widening of 8 elements to bf16
// (exact: an E4M3 value has 4 significant bits, an E2M1 value 2, and MXFP4
// scales are powers of two).
struct PgBf16 {
  static constexpr int BITS = 16;
  static constexpr bool MX = false;
};
struct PgFp8 {
  static constexpr int BITS = 8;
  static constexpr bool MX = false;
};
struct PgMx4 {
  static constexpr int BITS = 4;
  static constexpr bool MX = true;
};
__device__ __forceinline__ u32x4 widen_fp8(uint32_t a, uint32_t b) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true))};
}
// Eight E2M1 codes times 2^(e - 127), e a scale byte (255: NaN). The
// conversion reads the exponent bits of its scale operand alone and takes 0 as
// 2^-127 (verified over all bytes), which is the scale byte's own meaning.
__device__ __forceinline__ u32x4 widen_mx4(uint32_t w, uint32_t e) {
  const float s = __uint_as_float(e << 23);
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3))};
}
// The same to fp16, which holds E4M3 values exactly, and E2M1 values whose
// scale is within its range.
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ u32x4 widen_fp8_f16(uint32_t a, uint32_t b) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true))};
}
__device__ __forceinline__ u32x4 widen_mx4_f16(uint32_t w, uint32_t e) {
  const float s = __uint_as_float(e << 23);
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3))};
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  f16x2 v = {(_Float16)lo, (_Float16)hi};  // round to nearest even
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ f32x16 mfma32_f16(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int AUX> __device__ __forceinline__ uint32_t load_u8(__amdgpu_buffer_rsrc_t r, int off) {
  return (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, off, 0, AUX);
}

// A value that is the same in all lanes, in a scalar register. The statement
// hides that it is: the compiler drops a readfirstlane of a value it knows to be
// uniform and then, where a vector instruction made it (a vector load, a
// three-way median), builds every buffer resource that depends on it lane by
// lane, in a loop around each load.
__device__ __forceinline__ int scalar(int x) {
  asm("" : "+v"(x));
  return __builtin_amdgcn_readfirstlane(x);
}

// Padded rows in LDS: 16 key rows of an operand read start in different
// 16-byte bank groups, the 4 value rows of a transposing read in different
// 32-byte ones.
template <int D> struct PageRow {
  static constexpr int KROW = 2 * D + 16;
  static constexpr int VROW = 2 * D + 32;
};

// Buffer resource over n rows of row_bytes from `base`; past them loads return
// zeros without a memory access.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t half_rsrc(const uint8_t* base, int n, int row_bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), (short)0, n * row_bytes, 0x00020000);
}

// A 32-key tile in a wave's registers. Pages hold at least 16 rows, so the
// tile's two halves of 16 keys lie in one page each: every load instruction
// reads within one half, whose page is wave-uniform.
//   bf16, fp8: instruction e reads 1 KB of consecutive rows of K and of V;
//   MXFP4: V likewise (d = 64: 512 bytes); K straight as operands: lane (n, G)
//     holds quarter G of row n of each half (with d = 128 one scale block),
//     k-step s of the logits is then elements (d/4)G + 8s.. of the row, the
//     order that Q^T operands take too, and keys need no LDS.
template <int D, typename KV> struct PageTile {
  static constexpr int RB = D * KV::BITS / 8;      // bytes of a row
  static constexpr int EB = D / kMxBlock;          // scale bytes of a row (MXFP4)
  static constexpr int HALF = 16 * RB;             // bytes of half a tile
  static constexpr int LB = HALF >= 1024 ? 16 : HALF / 64;  // bytes a lane loads
  static constexpr int HI = HALF / (64 * LB);      // instructions for a half
  typedef Raw<LB> L;
  typename L::type k[2][HI], v[2][HI];
  uint32_t ke[2], ve[2];

  // AUX: cache policy (rows that are read once stream past the caches).
  template <int AUX>
  __device__ __forceinline__ void load(const PagePool& P, int gam, int id0, int id1, int key0, int k1,
                                       int lane) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      const int id = a ? id1 : id0, key = key0 + 16 * a;
      const int n = scalar(min(16, max(0, k1 - key)));
      const size_t row = ((size_t)((int64_t)id * P.g + gam) << P.shift) + (key & ((1 << P.shift) - 1));
      const __amdgpu_buffer_rsrc_t rk = half_rsrc(P.K + row * RB, n, RB);
      const __amdgpu_buffer_rsrc_t rv = half_rsrc(P.V + row * RB, n, RB);
#pragma unroll
      for (int e = 0; e < HI; ++e) {
        const int at = KV::MX ? (lane & 15) * RB + (lane >> 4) * LB : (64 * e + lane) * LB;
        k[a][e] = L::template load<AUX>(rk, at);
        v[a][e] = L::template load<AUX>(rv, (64 * e + lane) * LB);
      }
      if constexpr (KV::MX) {
        const __amdgpu_buffer_rsrc_t re = half_rsrc(P.K_exp + row * EB, n, EB);
        const __amdgpu_buffer_rsrc_t rf = half_rsrc(P.V_exp + row * EB, n, EB);
        ke[a] = load_u8<AUX>(re, (lane & 15) * EB + ((lane >> 4) * EB) / 4);
        ve[a] = load_u8<AUX>(rf, (lane * EB) / 4);
      }
    }
  }
  // Write the widened rows into the wave's LDS tiles (K only where its
  // operands are read from there). A wave's LDS instructions execute in order;
  // the wave barriers keep the compiler from moving other tiles' reads across.
  __device__ __forceinline__ void stage(unsigned char* kl, unsigned char* vl, int lane) const {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int e = 0; e < HI; ++e) {
        const int at = (64 * e + lane) * LB;  // byte of the half
        const int row = 16 * a + at / RB, col = (at % RB) * (16 / KV::BITS);
        unsigned char* vd = vl + row * PageRow<D>::VROW + col;
        if constexpr (KV::BITS == 16) {
          write128(kl + row * PageRow<D>::KROW + col, k[a][e]);
          write128(vd, v[a][e]);
        } else if constexpr (KV::BITS == 8) {
          unsigned char* kd = kl + row * PageRow<D>::KROW + col;
          write128(kd, widen_fp8(k[a][e][0], k[a][e][1]));
          write128(kd + 16, widen_fp8(k[a][e][2], k[a][e][3]));
          write128(vd, widen_fp8(v[a][e][0], v[a][e][1]));
          write128(vd + 16, widen_fp8(v[a][e][2], v[a][e][3]));
        } else {
#pragma unroll
          for (int w = 0; w < LB / 4; ++w) write128(vd + 16 * w, widen_mx4(L::word(v[a][e], w), ve[a]));
        }
      }
    __builtin_amdgcn_wave_barrier();
  }
  // K operand of sub-tile a, k-step s: key 16a + n.
  __device__ __forceinline__ u32x4 kop(const unsigned char* kl, int a, int s, int lane) const {
    if constexpr (KV::MX)
      return widen_mx4(L::word(k[a][0], s), ke[a]);
    else
      return read128(kl + (16 * a + (lane & 15)) * PageRow<D>::KROW + 64 * s + 16 * (lane >> 4));
  }
  // V^T operand of dims 16t..16t+15: k-slots 8G + 4a + j are keys 16a + 4G + j.
  static __device__ __forceinline__ u32x4 vop(const unsigned char* vl, int t, int lane) {
    const unsigned char* p = vl + (4 * (lane >> 4) + ((lane & 15) >> 2)) * PageRow<D>::VROW + 32 * t + 8 * (lane & 3);
    const u32x2 lo = read_tr(p), hi = read_tr(p + 16 * PageRow<D>::VROW);
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  }
  // First element of the 8 that lane group G holds of k-step s.
  static __device__ __forceinline__ int qdim(int s, int G) { return KV::MX ? (D / 4) * G + 8 * s : 32 * s + 8 * G; }
};

// Running state of NT query tiles of 16 rows: lane (n, G) holds dims
// 16t + 4G + j of row n in acc[nt][t][j].
template <int D, int NT> struct PageState {
  float mref[NT], thr[NT], l[NT];
  f32x4 acc[NT][D / 16];
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      mref[nt] = thr[nt] = kNegInf;
      l[nt] = 0.f;
#pragma unroll
      for (int t = 0; t < D / 16; ++t) acc[nt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
};

// The two bf16 terms of 2 NW weights, as B operands: the weight cut to 8 bits
// and the rest rounded to 8, together off by at most 2^-15 of it. The rest is
// formed from the weight plus 2^-23 of it, so that it is above 0 wherever the
// weight is: an infinite value times it stays infinite (times 0, or a negative
// rest, it would give NaN).
template <int NW>
__device__ __forceinline__ void split_weights(const float* pr, uint32_t* hi, uint32_t* lo) {
  constexpr float kUp = 1.f + 0x1p-23f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const uint32_t a = __float_as_uint(pr[2 * w]), b = __float_as_uint(pr[2 * w + 1]);
    hi[w] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    lo[w] = pack_bf16(__builtin_fmaf(pr[2 * w], kUp, -__uint_as_float(a & 0xffff0000u)),
                      __builtin_fmaf(pr[2 * w + 1], kUp, -__uint_as_float(b & 0xffff0000u)));
  }
}

// Whether a staged value tile holds an infinity or a NaN: the sum carries past
// an exponent of all ones.
template <int D> __device__ __forceinline__ bool has_odd_values(const unsigned char* vl, int lane) {
  uint32_t odd = 0;
#pragma unroll
  for (int u = 0; u < kTileKeys * D / 512; ++u) {
    const int at = 64 * u + lane;
    const u32x4 v = *(volatile const lds_u32x4*)(vl + at / (D / 8) * PageRow<D>::VROW + at % (D / 8) * 16);
#pragma unroll
    for (int w = 0; w < 4; ++w) odd |= (v[w] & 0x7f807f80u) + 0x00800080u;
  }
  return __any((odd & 0x80008000u) != 0);
}

// Keys of the tile that hold such values and that later tokens alone see (row r
// sees those below all + r % ntok): their weight in the rows before is 0, which the
// products would turn into NaN. They enter the rows that see them one by one,
// whatever the weight, and leave the tile.
template <int D, int NT>
__device__ __forceinline__ void take_odd_values(PageState<D, NT>& st, unsigned char* vl, const u32x4* hi, const u32x4* lo,
                                             int all, int ntok, int lane) {
#pragma unroll 1
  for (int key = max(0, all); key < kTileKeys; ++key) {
    unsigned char* row = vl + key * PageRow<D>::VROW;
    const u32x4 own = *(volatile const lds_u32x4*)(row + 16 * (lane % (D / 8)));
    bool odd = false;
#pragma unroll
    for (int w = 0; w < 4; ++w) odd |= ((((own[w] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0);
    if (!__any(odd)) continue;
    const int e = 4 * (key / 16) + key % 4, from = (lane & 15) + 16 * (key % 16 / 4);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      uint32_t a = 0, b = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        if (w == e / 2) a = hi[nt][w], b = lo[nt][w];
      const int up = e % 2 ? 0 : 16;
      const float p = __shfl(__uint_as_float(a << up & 0xffff0000u) + __uint_as_float(b << up & 0xffff0000u), from);
      if (key < all + (nt * kRowsPerTile + (lane & 15)) % ntok)
#pragma unroll
        for (int t = 0; t < D / 16; ++t) {
          const u32x2 v = *(volatile const lds_u32x2*)(row + 32 * t + 8 * (lane >> 4));
          st.acc[nt][t] += p * f32x4{__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xffff0000u),
                                     __uint_as_float(v[1] << 16), __uint_as_float(v[1] & 0xffff0000u)};
        }
    }
    if (lane < D / 8) write128(row + 16 * lane, u32x4{0, 0, 0, 0});
    __builtin_amdgcn_wave_barrier();
  }
}

// One staged tile against NT query tiles. rem: keys from the tile's first to
// the end of the sequence; row r sees keys < rem - (ntok - 1) + r % ntok. second:
// the first row of the second map, 0 with one map.
template <int D, int NT, typename KV, typename QAt>
__device__ __forceinline__ void page_update(PageState<D, NT>& st, const PageTile<D, KV>& A,
                                            const unsigned char* kl, unsigned char* vl, QAt&& q_at,
                                            int rem, int ntok, int second, float scale_log2, int lane) {
  constexpr int KS = D / 32, DV = D / 16;
  const int G = lane >> 4;
  f32x4 sacc[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) sacc[nt][0] = sacc[nt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const u32x4 k0 = A.kop(kl, 0, s, lane), k1 = A.kop(kl, 1, s, lane);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const u32x4 qo = q_at(nt, s);
      sacc[nt][0] = mfma_bf16(k0, qo, sacc[nt][0]);
      sacc[nt][1] = mfma_bf16(k1, qo, sacc[nt][1]);
    }
  }
  // An infinity in the other map's half of a key met the zeros of this map's row:
  // where a logit is NaN, every row once more over its own half alone. (Codes have
  // no infinities, and a NaN makes the maps' difference NaN through either.)
  if constexpr (KV::BITS == 16) {
    if (second) {
      bool odd = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 8; ++e) odd |= sacc[nt][e / 4][e % 4] != sacc[nt][e / 4][e % 4];
      if (__any(odd)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            f32x4 half[2];
#pragma unroll
            for (int s = 0; s < KS; ++s) {
              f32x4& h = half[s / (KS / 2)];
              if (s % (KS / 2) == 0) h = f32x4{0.f, 0.f, 0.f, 0.f};
              h = mfma_bf16(A.kop(kl, a, s, lane), q_at(nt, s), h);
            }
            const bool upper = nt * kRowsPerTile + (lane & 15) >= second;
#pragma unroll
            for (int j = 0; j < 4; ++j) sacc[nt][a][j] = upper ? half[1][j] : half[0][j];
          }
      }
    }
  }
  // The reference maximum only has to bound the logits within 2^kRescaleSlack:
  // it is raised (with a rescale) when some lane's logit exceeds the threshold.
  float x[NT][8], lmax[NT];  // x[nt][4a + j]: key 16a + 4G + j
  bool raise_any = false;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[nt][e] = sacc[nt][e / 4][e % 4];
    if (rem < kTileKeys + ntok - 1) {
      const int nv = __builtin_amdgcn_readfirstlane(rem) - (ntok - 1);
      const int lim = ntok == 1 ? nv : nv + (nt * kRowsPerTile + (lane & 15)) % ntok;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (16 * (e / 4) + 4 * G + e % 4 >= lim) x[nt][e] = kNegInf;
    }
    float m = x[nt][0];
#pragma unroll
    for (int e = 1; e < 8; ++e) m = fmaxf(m, x[nt][e]);
    lmax[nt] = m;
    raise_any |= m > st.thr[nt];
  }
  if (__any(raise_any)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float tmax = xor32_max(xor16_max(lmax[nt])) * scale_log2;
      const bool raise = tmax > st.mref[nt] + kRescaleSlack;
      const float alpha = raise ? exp2_fast(st.mref[nt] - tmax) : 1.f;
      st.l[nt] *= alpha;
#pragma unroll
      for (int t = 0; t < DV; ++t) st.acc[nt][t] *= alpha;
      st.mref[nt] = raise ? tmax : st.mref[nt];
      st.thr[nt] = (st.mref[nt] + kRescaleSlack) / scale_log2;
    }
  }
  u32x4 hi[NT], lo[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float nbase = st.mref[nt] == kNegInf ? 0.f : -st.mref[nt];
    float pr[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) pr[e] = exp2_fast(__builtin_fmaf(x[nt][e], scale_log2, nbase));
    float psum = pr[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) psum += pr[e];
    st.l[nt] += psum;
    uint32_t h[4], o[4];
    split_weights<4>(pr, h, o);
    hi[nt] = u32x4{h[0], h[1], h[2], h[3]};
    lo[nt] = u32x4{o[0], o[1], o[2], o[3]};
  }
  if (ntok > 1 && rem < kTileKeys + ntok - 1 && has_odd_values<D>(vl, lane))
    take_odd_values<D, NT>(st, vl, hi, lo, rem - (ntok - 1), ntok, lane);
#pragma unroll
  for (int t = 0; t < DV; ++t) {
    const u32x4 v = PageTile<D, KV>::vop(vl, t, lane);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      st.acc[nt][t] = mfma_bf16(v, hi[nt], st.acc[nt][t]);
      st.acc[nt][t] = mfma_bf16(v, lo[nt], st.acc[nt][t]);
    }
  }
}

// LDS of a streaming work-group: Q^T operands, then a K and a V tile per wave.
template <int D, typename KV> struct StreamLds {
  static constexpr int KT = KV::MX ? 0 : kTileKeys * PageRow<D>::KROW;
  static constexpr int VT = kTileKeys * PageRow<D>::VROW;
  static constexpr int TILE = KT + VT;
};
template <int D, int NT> constexpr int q_bytes() { return NT * (D / 32) * 64 * 16; }

// Q^T operand slot (nt, s) of a unit: row r = 16nt + n, 8 elements from qdim.
// ptr(r): the bf16 row of tile row r (any valid row for padding ones: the load
// is unconditional, so that a slot's loads issue together); on(r): not padding;
// map(r): its map. With maps = 2 a row's other half is zero.
template <int D, typename KV, typename Rows>
__device__ __forceinline__ u32x4 query_slot(const Rows& rows, int nt, int s, int maps, uint32_t sign, int lane) {
  const int r = nt * kRowsPerTile + (lane & 15), dim = PageTile<D, KV>::qdim(s, lane >> 4);
  const u32x4 q = load16(rows.ptr(r) + dim) ^ sign;
  const bool on = rows.on(r) && (maps == 1 || dim / (D / 2) == rows.map(r));
  u32x4 z;
#pragma unroll
  for (int w = 0; w < 4; ++w) z[w] = on ? q[w] : 0u;
  return z;
}

// Page ids of the halves of the 32-key tile at `key`: lane 0 the first's, lane
// 1 the second's. Rows from `end` (> 0) on have no entry of their own.
__device__ __forceinline__ int tile_ids(const int32_t* table, int key, int end, int shift, int lane) {
  return table[min(key + 16 * (lane & 1), end - 1) >> shift];
}

// One wave streams the tiles k0, k0 + stride, ... below k1 of one sequence;
// ids0, ids1 are the first two tiles' ids. DEPTH tiles are in flight: a bf16
// tile is 16 KB a wave, enough at one; of codes, four (two) times smaller, two
// (measured on 32 samples of an MHA layer over 8k, MXFP4). A tile's ids are
// requested an iteration before its rows, ahead of rows that are waited for
// anyway. kend: the end that the tokens' limits count from. Returns whether a
// page id was outside the pool (read as page 0).
template <int D, int NT, typename KV, int AUX = kAuxStream, typename QAt>
__device__ __forceinline__ bool stream_pages(PageState<D, NT>& st, const PagePool& P, int gam,
                                             const int32_t* table, QAt&& q_at, unsigned char* kl,
                                             unsigned char* vl, int ids0, int ids1, int k0, int k1, int kend,
                                             int stride, int ntok, int second, float scale_log2, int lane) {
  constexpr int DEPTH = KV::BITS == 16 ? 1 : 2;
  bool bad = false;
  if (k0 >= k1) return false;
  PageTile<D, KV> T[DEPTH];
  auto load = [&](PageTile<D, KV>& t, int ids, int key) {
    const bool wrong = (unsigned)ids >= (unsigned)P.num_pages;
    bad |= wrong && key + 16 * (lane & 1) < k1;
    ids = wrong ? 0 : ids;
    t.template load<AUX>(P, gam, __builtin_amdgcn_readlane(ids, 0), __builtin_amdgcn_readlane(ids, 1), min(key, k1), k1, lane);
  };
  auto ids_at = [&](int key) { return tile_ids(table, min(key, k1 - 1), k1, P.shift, lane); };
  load(T[0], ids0, k0);
  int next = ids1;  // ids of the next tile to load
  if constexpr (DEPTH == 2) {
    next = ids_at(k0 + 2 * stride);
    load(T[1], ids1, k0 + stride);
  }
  for (int key = k0; key < k1;) {
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) {
      T[u].stage(kl, vl, lane);
      PageTile<D, KV> cur;
      if constexpr (KV::MX) cur = T[u];  // K operands come from the registers
      const int ids = next;
      next = ids_at(key + (DEPTH + 1) * stride);
      load(T[u], ids, key + DEPTH * stride);
      page_update(st, KV::MX ? cur : T[u], kl, vl, q_at, kend - key, ntok, second, scale_log2, lane);
      key += stride;
      if (key >= k1) break;
    }
  }
  return bad;
}

// Row totals of the per-lane sums (the four lanes of a row share the row).
template <int D, int NT> __device__ __forceinline__ void total_sums(PageState<D, NT>& st) {
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) st.l[nt] = xor32_sum(xor16_sum(st.l[nt]));
}

__device__ __forceinline__ float group_scale_log2(const PagedAttnParams& P, int gam) {
  return P.pool.k_scale ? P.scale_log2 * P.pool.k_scale[gam] : P.scale_log2;
}

// Own rows: work-group (sample i, group gam, chunk s) of four waves, which take
// interleaved tiles and write a partial each of the unit's R rows. All waves
// of the work-group call it (`on`: whether this unit exists). The length, the
// first page ids and the queries are requested together: the ids within the
// row capacity, whose entries past the length are not used.
struct OwnRows {
  const uint16_t* base;
  int D, R, pn;
  __device__ __forceinline__ const uint16_t* ptr(int r) const {
    const int rr = min(r, R - 1);
    return base + (size_t)(rr < pn ? rr : rr - pn) * D;
  }
  __device__ __forceinline__ bool on(int r) const { return r < R; }
  __device__ __forceinline__ int map(int r) const { return r < pn ? 0 : 1; }
};
template <int D, int NT, typename KV>
__device__ __forceinline__ void own_block(const PagedAttnParams& P, int blk, bool on, int wave, int lane,
                                          unsigned char* qs, unsigned char* kl, unsigned char* vl) {
  constexpr int KS = D / 32;
  blk = on ? blk : 0;
  // All units' first chunks, then their second ones, ...: XCDs take work-groups
  // in turn, and chunk-minor order would put the later, emptier chunks of every
  // unit on the same ones (48 samples of up to 4k rows: 95 us, so 79).
  const int s = blk / (P.b * P.g), ig = blk - s * (P.b * P.g);
  const int gam = ig % P.g, i = ig / P.g;
  const int c0 = s * P.dec_keys, k0 = c0 + wave * kTileKeys, cap = min(P.m_d_max, c0 + P.dec_keys);
  constexpr int stride = kWaves * kTileKeys;
  const int32_t* table = P.tables + (size_t)i * P.table_pages;
  const int ids0 = tile_ids(table, min(k0, cap - 1), cap, P.pool.shift, lane);
  const int ids1 = tile_ids(table, min(k0 + stride, cap - 1), cap, P.pool.shift, lane);
  const int raw = P.lens[i];
  const OwnRows rows = {P.q + ((size_t)i * P.hn + (size_t)gam * P.pn) * D, D, P.R, P.pn};
  u32x4 qreg[NT == 1 ? KS : 1];
  if constexpr (NT == 1) {
#pragma unroll
    for (int k = 0; k < KS; ++k) qreg[k] = query_slot<D, KV>(rows, 0, k, P.maps, P.q_sign, lane);
  } else {
    for (int k = wave; k < NT * KS; k += kWaves)
      write128(qs + (k * 64 + lane) * 16, query_slot<D, KV>(rows, k / KS, k % KS, P.maps, P.q_sign, lane));
    __syncthreads();
  }
  if (!on) return;
  const int total = scalar(raw < 0 ? 0 : (raw > P.m_d_max ? P.m_d_max : raw));
  auto q_at = [&](int nt, int k) -> u32x4 {
    if constexpr (NT == 1) return qreg[k];
    return *(volatile const lds_u32x4*)(qs + ((nt * KS + k) * 64 + lane) * 16);
  };
  PageState<D, NT> st;
  st.init();
  const bool bad =
      stream_pages<D, NT, KV>(st, P.pool, gam, table, q_at, kl, vl, ids0, ids1, k0, min(total, c0 + P.dec_keys), total,
                              stride, P.ntok, P.maps == 2 ? P.pn : 0, group_scale_log2(P, gam), lane);
  if (__any(bad) && lane == 0) atomicOr(P.status, kStatusPage);
  total_sums(st);
  const size_t prow = (((size_t)ig * P.S_d + s) * kWaves + wave) * P.R;
  const int n = lane & 15, G = lane >> 4;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = nt * kRowsPerTile + n;
    if (row < P.R) {
      float* dst = P.dec_acc + (prow + row) * D + 4 * G;
#pragma unroll
      for (int t = 0; t < D / 16; ++t) *reinterpret_cast<f32x4*>(dst + 16 * t) = st.acc[nt][t];
      if (G == 0) P.dec_ml[prow + row] = float2{st.mref[nt], st.l[nt]};
    }
  }
}

template <int D, int NT> struct PageMerge {
  static constexpr int LD = D + 4;
  static constexpr int ROWS = NT * kRowsPerTile;
  static constexpr int bytes = (ROWS * LD + 2 * ROWS) * 4;
};

// Merge the four waves' states of the same rows in LDS, in wave order: row r is
// then merge[r*LD ..], its maximum and sum behind the rows.
template <int D, int NT>
__device__ __forceinline__ void merge_states(const PageState<D, NT>& st, float* merge, int wave, int lane) {
  constexpr int LD = PageMerge<D, NT>::LD, ROWS = PageMerge<D, NT>::ROWS;
  float* m_s = merge + ROWS * LD;
  float* l_s = m_s + ROWS;
  const int n = lane & 15, G = lane >> 4;
  __syncthreads();  // the merge buffer overlays the waves' tiles
  for (int turn = 0; turn < kWaves; ++turn) {
    if (wave == turn) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int row = nt * kRowsPerTile + n;
        const float mo = turn ? m_s[row] : kNegInf, lo = turn ? l_s[row] : 0.f;
        const float mn = fmaxf(mo, st.mref[nt]), base = mn == kNegInf ? 0.f : mn;
        const float fa = exp2_fast(mo - base), fb = exp2_fast(st.mref[nt] - base);
        float* dst = merge + row * LD + 4 * G;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) {
          const f32x4 old = turn ? *reinterpret_cast<f32x4*>(dst + 16 * t) : f32x4{0.f, 0.f, 0.f, 0.f};
          *reinterpret_cast<f32x4*>(dst + 16 * t) = old * fa + st.acc[nt][t] * fb;
        }
        if (G == 0) {
          m_s[row] = mn;
          l_s[row] = lo * fa + st.l[nt] * fb;
        }
      }
    }
    __syncthreads();
  }
}

struct GroupRows {  // row u*Mh + i*pn + jp of a group
  const uint16_t* base;
  int D, M, Mh, pn, hn;
  __device__ __forceinline__ const uint16_t* ptr(int r) const {
    const int rr = min(r, M - 1), rm = rr < Mh ? rr : rr - Mh, i = rm / pn;
    return base + ((size_t)i * hn + (rm - i * pn)) * D;
  }
  __device__ __forceinline__ bool on(int r) const { return r < M; }
  __device__ __forceinline__ int map(int r) const { return r < Mh ? 0 : 1; }
};
// Context, few rows per group: the 4 S_c waves of a group take its tiles round
// robin; the four waves' states merge in LDS, in wave order, into the split's
// partial.
template <int D, int NT, typename KV>
__device__ __forceinline__ void ctx_few_block(const PagedAttnParams& P, int blk, int wave, int lane,
                                              unsigned char* qs, unsigned char* kl, unsigned char* vl,
                                              float* merge) {
  constexpr int LD = PageMerge<D, NT>::LD, ROWS = PageMerge<D, NT>::ROWS;
  const int s = blk % P.S_c, gam = blk / P.S_c;
  constexpr int KS = D / 32;
  const int M = P.M;
  const int k0 = (s * kWaves + wave) * kTileKeys, stride = P.S_c * kWaves * kTileKeys;
  const int ids0 = tile_ids(P.ctx_table, min(k0, P.m_c - 1), P.m_c, P.pool.shift, lane);
  const int ids1 = tile_ids(P.ctx_table, min(k0 + stride, P.m_c - 1), P.m_c, P.pool.shift, lane);
  const GroupRows rows = {P.q + (size_t)gam * P.pn * D, D, M, P.Mh, P.pn, P.hn};
  for (int k = wave; k < NT * KS; k += kWaves)
    write128(qs + (k * 64 + lane) * 16, query_slot<D, KV>(rows, k / KS, k % KS, P.maps, P.q_sign, lane));
  __syncthreads();
  u32x4 qreg[NT == 1 ? KS : 1];
  if constexpr (NT == 1) {
#pragma unroll
    for (int k = 0; k < KS; ++k) qreg[k] = read128(qs + (k * 64 + lane) * 16);
  }
  auto q_at = [&](int nt, int k) -> u32x4 {
    if constexpr (NT == 1) return qreg[k];
    return *(volatile const lds_u32x4*)(qs + ((nt * KS + k) * 64 + lane) * 16);
  };
  PageState<D, NT> st;
  st.init();
  const bool bad = stream_pages<D, NT, KV>(st, P.pool, gam, P.ctx_table, q_at, kl, vl, ids0, ids1, k0, P.m_c, P.m_c, stride,
                                           1, P.maps == 2 ? P.Mh : 0, group_scale_log2(P, gam), lane);
  if (__any(bad) && lane == 0) atomicOr(P.status, kStatusPage);
  total_sums(st);
  merge_states(st, merge, wave, lane);
  const float* m_s = merge + ROWS * LD;
  const float* l_s = m_s + ROWS;
  const size_t prow = (size_t)blk * M;
  for (int idx = threadIdx.x; idx < M * (D / 4); idx += kThreads) {
    const int row = idx / (D / 4), c = idx % (D / 4);
    *reinterpret_cast<f32x4*>(P.ctx_acc + (prow + row) * D + 4 * c) =
        *reinterpret_cast<const f32x4*>(merge + row * LD + 4 * c);
  }
  for (int row = threadIdx.x; row < M; row += kThreads) P.ctx_ml[prow + row] = float2{m_s[row], l_s[row]};
}

// Grid: n_ctx_small_blocks context work-groups, then n_dec_blocks decode ones.
// Over bf16 bound by memory: 32 samples of a 32-head layer over 8k rows 66 us
// for 403 MB, 6.1 TB/s. Over MXFP4 (107 MB, 29 us) by the work and the latency of
// a tile: vector units 48%, matrix cores 22% of the cycles, a third of the waves'
// time waiting for memory; registers for three waves per SIMD instead of two hide
// more of it (31.5, so 29). More query tiles need the registers of two, or one.
template <int D, typename KV, int NTC, int NTD>
__device__ __forceinline__ void stream_body(const PagedAttnParams& P) {
  typedef StreamLds<D, KV> S;
  constexpr int QB = q_bytes<D, cmax(NTC, NTD)>();
  constexpr int MERGE = NTC ? PageMerge<D, cmax(NTC, 1)>::bytes : 0;
  __shared__ __attribute__((aligned(16))) unsigned char lds[QB + cmax(kWaves * S::TILE, MERGE)];
  const int lane = threadIdx.x & 63, wave = wave_id();
  unsigned char* kl = lds + QB + wave * S::TILE;
  unsigned char* vl = kl + S::KT;
  const int blk = blockIdx.x;
  if (blk < P.n_ctx_small_blocks) {
    if constexpr (NTC > 0)
      ctx_few_block<D, NTC, KV>(P, blk, wave, lane, lds, kl, vl, reinterpret_cast<float*>(lds + QB));
  } else {
    const int own = blk - P.n_ctx_small_blocks;
    own_block<D, NTD, KV>(P, own, own < P.n_dec_blocks, wave, lane, lds, kl, vl);
  }
}
template <int D, typename KV, int NTC, int NTD>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void stream_kernel_2w(PagedAttnParams P) {
  stream_body<D, KV, NTC, NTD>(P);
}
template <int D, typename KV, int NTC, int NTD>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3))) void stream_kernel_3w(PagedAttnParams P) {
  stream_body<D, KV, NTC, NTD>(P);
}
template <int D, typename KV, int NTC, int NTD>
__global__ __launch_bounds__(kThreads) void stream_kernel(PagedAttnParams P) {
  stream_body<D, KV, NTC, NTD>(P);
}

// ---------------------------------------------------------------------------
// Context, many rows per group, on v_mfma_f32_32x32x16_bf16: work-group (group,
// key split, row block) of NW waves with 32 query rows each. Stages of SK keys
// pass from memory through registers (widened) into one of two LDS buffers, a
// stage ahead of the products, their page ids two stages ahead; one barrier a
// stage. With maps = 2 a row block belongs to one map, whose half of the key
// rows alone enters its logits.
//
// Bound by what a block of 32 keys costs a CU: matrix cores, vector units and LDS
// take turns, each busy for 40 to 47% of the cycles of the CUs that have work (256
// samples of a grouped layer over 32k rows in MXFP4: 178 us a step, 790 TFLOP/s),
// and by the CUs of the own rows, which end early.
//
// Code caches take fp16 for the value product: one term of 11 bits for the weights
// (their error 2e-4 beside the output's 1.7e-3) where bf16 values need two. The
// reference lies 2^kUp below the largest weight, so that fp16's range lies where
// theirs does: raised once a weight exceeds the last one's largest by 2^5, they keep
// 11 bits down to 2^-24 of the row's largest among the work-group's keys; below, a
// fixed step of 2^-34 of it. A smaller slack reaches further and raises more often:
// grouped layer over 32k in MXFP4, multi-query one over 16k in fp8 and grouped
// differential one over 16k in MXFP4 in turn 180, 58 and 37.3 us with 8, 180.5, 58 and
// 37.4 with 5, 182, 60 and 38.0 with 4, 193, 66 and 43.6 with 2. E4M3 values are exact
// in fp16. MXFP4 values enter relative to the largest scale of the same 32 elements
// among the work-group's keys, read ahead (1/16 of the chunk's value bytes), which
// enters as 2^13 (the largest value is then 6 * 2^13 of fp16's 65504), and are exact
// down to 2^-36 of it.
template <int D, int NW, int SK, typename KV, int MAPS>
__device__ __forceinline__ void ctx_many_block(const PagedAttnParams& P, unsigned char* lds) {
  constexpr int KD = D / MAPS;             // dims of the logits
  constexpr int KSTEPS = KD / 16, DB = D / 32;
  constexpr int KROW = PageRow<D>::KROW, VROW = PageRow<D>::VROW;
  constexpr int STAGE = SK * (KROW + VROW);
  constexpr int RB = D * KV::BITS / 8, CPR = RB / 16, EB = D / kMxBlock;
  constexpr int LOADS = 2 * SK * CPR, PER = LOADS / (64 * NW);
  static_assert(LOADS % (64 * NW) == 0 && (SK * CPR) % 64 == 0, "whole loads, waves of K or V alone");
  const int blk = xcd_logical(blockIdx.x, P.g * P.S_c, P.ctx_row_blocks);
  const int rb = blk % P.ctx_row_blocks, sg = blk / P.ctx_row_blocks;
  const int s = sg % P.S_c, gam = sg / P.S_c;
  const int per_map = P.ctx_row_blocks / MAPS;
  const int map = MAPS == 1 ? 0 : rb / per_map;
  const int k0 = s * P.ctx_keys, nkeys = min(P.m_c, k0 + P.ctx_keys) - k0;
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int j = lane & 31, h = lane >> 5;
  const int row0 = (rb - map * per_map) * (32 * NW) + wave * 32;
  const float sl2 = group_scale_log2(P, gam);
  const PagePool& pool = P.pool;
  const int mask = (1 << pool.shift) - 1;
  bool bad = false;
  constexpr bool kHalf = KV::BITS < 16;  // values and weights in fp16, weights below 2^(kUp + kSlack)
  constexpr float kUp = kHalf ? 10.f : 0.f, kSlack = kHalf ? 5.f : kRescaleSlack;
  constexpr float kBound = kHalf ? 0x1p15f : kSumBound;  // 2^(kUp + kSlack)
  auto row_of = [&](int key, int id) {  // pool row of a context key, by its page id
    const bool wrong = (unsigned)id >= (unsigned)pool.num_pages;
    bad |= wrong;
    return ((size_t)((int64_t)(wrong ? 0 : id) * pool.g + gam) << pool.shift) + (key & mask);
  };

  // Load u of a thread: 16 bytes, chunk c of row `row` of K (first half of the
  // loads) or V. Rows past the range repeat its last one and are zeroed.
  int ids[PER];
  u32x4 reg[PER];
  uint32_t ex[KV::MX ? PER : 1];
  auto chunk = [&](int u, bool& is_v, int& row, int& c) {
    const int q = (int)threadIdx.x + 64 * NW * u;
    is_v = q >= SK * CPR;
    const int qq = is_v ? q - SK * CPR : q;
    row = qq / CPR;
    c = qq % CPR;
  };
  auto get_ids = [&](int key0) {
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      bool is_v;
      int row, c;
      chunk(u, is_v, row, c);
      ids[u] = P.ctx_table[(k0 + min(key0 + row, nkeys - 1)) >> pool.shift];
    }
  };
  auto stage_get = [&](int key0) {
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      bool is_v;
      int row, c;
      chunk(u, is_v, row, c);
      const size_t at = row_of(k0 + min(key0 + row, nkeys - 1), ids[u]);
      reg[u] = *reinterpret_cast<const u32x4*>((is_v ? pool.V : pool.K) + at * RB + 16 * c);
      if constexpr (KV::MX) ex[u] = ((is_v ? pool.V_exp : pool.K_exp) + at * EB)[c];
    }
  };
  int vref = 0;  // MXFP4: exponent that the scales of this thread's chunk column of values are relative to
  int vrefs[EB];  // of all columns
  auto stage_put = [&](int key0, int buf) {
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      bool is_v;
      int row, c;
      chunk(u, is_v, row, c);
      unsigned char* dst = lds + buf * STAGE + (is_v ? SK * KROW + row * VROW : row * KROW) + c * (256 / KV::BITS);
      u32x4 w = reg[u];
      if (key0 + SK > nkeys && key0 + row >= nkeys) w = u32x4{0, 0, 0, 0};
      if constexpr (KV::BITS == 16) {
        write128(dst, w);
      } else if constexpr (KV::BITS == 8) {
        write128(dst, is_v ? widen_fp8_f16(w[0], w[1]) : widen_fp8(w[0], w[1]));
        write128(dst + 16, is_v ? widen_fp8_f16(w[2], w[3]) : widen_fp8(w[2], w[3]));
      } else {
        uint32_t e = key0 + SK > nkeys && key0 + row >= nkeys ? 0u : ex[u];
        if (is_v) {  // wave-uniform
          e = e == 255u ? e : (uint32_t)max(0, (int)e - vref);
#pragma unroll
          for (int k = 0; k < 4; ++k) write128(dst + 16 * k, widen_mx4_f16(w[k], e));
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) write128(dst + 16 * k, widen_mx4(w[k], e));
        }
      }
    }
  };
  get_ids(0);
  stage_get(0);
  if (SK < nkeys) get_ids(SK);
  if constexpr (KV::MX) {
    // the largest scale byte of each column that is a number; values then reach 6 * 2^13
    static_assert(CPR == EB && (64 * NW) % EB == 0, "a chunk is a scale block, a thread's column stays");
    int top[EB];
#pragma unroll
    for (int c = 0; c < EB; ++c) top[c] = 0;
    for (int key = threadIdx.x; key < nkeys; key += 64 * NW) {
      const uint8_t* e = pool.V_exp + row_of(k0 + key, P.ctx_table[(k0 + key) >> pool.shift]) * EB;
#pragma unroll
      for (int c = 0; c < EB; ++c) top[c] = max(top[c], e[c] == 255 ? 0 : (int)e[c]);
    }
    int* tops = reinterpret_cast<int*>(lds);
#pragma unroll
    for (int c = 0; c < EB; ++c) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) top[c] = max(top[c], __shfl_xor(top[c], o));
      if (lane == 0) tops[wave * EB + c] = top[c];
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < EB; ++c) {
#pragma unroll
      for (int w = 0; w < NW; ++w) top[c] = max(top[c], tops[w * EB + c]);
      vrefs[c] = __builtin_amdgcn_readfirstlane(top[c]) - 127 - 13;
      vref = (int)threadIdx.x % EB == c ? vrefs[c] : vref;
    }
    __syncthreads();
  }

  const int Mh = P.Mh, pn = P.pn;
  const bool active = row0 < Mh;  // wave-uniform
  u32x4 qop[KSTEPS];
  {
    const int row = row0 + j;
    const bool valid = row < Mh;
    const int rr = valid ? row : Mh - 1;
    const int i = rr / pn;
    const uint16_t* qr = P.q + ((size_t)i * P.hn + (size_t)gam * pn + (rr - i * pn)) * D + map * KD;
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) qop[ks] = load16(qr + 16 * ks + 8 * h);
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
      for (int w = 0; w < 4; ++w) qop[ks][w] = valid ? qop[ks][w] ^ P.q_sign : 0u;
  }
  stage_put(0, 0);
  if (SK < nkeys) {
    stage_get(SK);
    if (2 * SK < nkeys) get_ids(2 * SK);
  }
  const int q4 = lane >> 4, ip = lane & 15;
  const int kbase = j * KROW + 2 * map * KD + h * 16;
  const int vbase = SK * KROW + (4 * (q4 >> 1) + (ip >> 2)) * VROW + (16 * (q4 & 1) + 4 * (ip & 3)) * 2;
  f32x16 acc[DB];
#pragma unroll
  for (int t = 0; t < DB; ++t)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[t][v] = 0.f;
  float mref = kNegInf, lsum = 0.f;

  const int nstages = (nkeys + SK - 1) / SK;
  for (int st = 0; st < nstages; ++st) {
    const int buf = st & 1;
    // hands stage st to all waves and frees the other buffer for stage st + 1
    __syncthreads();
    if (st + 1 < nstages) {
      stage_put((st + 1) * SK, buf ^ 1);
      if (st + 2 < nstages) {
        stage_get((st + 2) * SK);
        if (st + 3 < nstages) get_ids((st + 3) * SK);
      }
    }
    if (!active) continue;
    const unsigned char* kb = lds + buf * STAGE + kbase;
    const unsigned char* vb = lds + buf * STAGE + vbase;
    const int rem = nkeys - st * SK;
    // LDS reads ahead of their use: a block's V^T operands are read while its
    // weights are formed, the next block's K operands during the value products.
    u32x4 kw[KSTEPS];
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) kw[ks] = read128(kb + 32 * ks);
#pragma unroll
    for (int b = 0; b < SK / 32; ++b) {
      f32x16 sacc;
#pragma unroll
      for (int v = 0; v < 16; ++v) sacc[v] = 0.f;
      // The wave in its products goes first, so that the other one of the SIMD
      // does its softmax meanwhile (grouped layer over 32k in MXFP4 177.4 us, so
      // 175.7; multi-query one over 16k in fp8 56.9, so 56.5).
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) sacc = mfma32(kw[ks], qop[ks], sacc);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
      u32x4 vw[2][DB];
#pragma unroll
      for (int ss = 0; ss < 2; ++ss)
#pragma unroll
        for (int t = 0; t < DB; ++t) {
          const unsigned char* p = vb + (32 * b + 16 * ss) * VROW + 64 * t;
          const u32x2 v0 = read_tr(p), v1 = read_tr(p + 8 * VROW);
          vw[ss][t] = u32x4{v0[0], v0[1], v1[0], v1[1]};
        }
      __builtin_amdgcn_sched_barrier(0);
      float x[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) x[v] = sacc[v];
      if (rem < 32 * (b + 1)) {
        asm volatile("");  // a branch: 32 selects in every block otherwise
        const int nv = rem - 32 * b;
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (8 * (v / 4) + 4 * h + (v & 3) >= nv) x[v] = kNegInf;
      }
      // Weights against the current reference first; a raise needs a weight
      // above 2^(kUp + kSlack), which shows in their sum.
      float pr[16], ps;
      auto weights = [&]() {
        const float nbase = mref == kNegInf ? 0.f : -mref;
#pragma unroll
        for (int v = 0; v < 16; ++v) pr[v] = exp2_fast(__builtin_fmaf(x[v], sl2, nbase));
        ps = pr[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) ps += pr[v];
      };
      weights();
      if (__any(!(ps <= kBound) || mref == kNegInf)) {
        float lmax = x[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) lmax = fmaxf(lmax, x[v]);
        // by how much the largest logit exceeds the reference, in one rounding as
        // in the weights: those of huge logits stay in fp16's range too
        lmax = xor32_max(lmax);
        const float tmax = lmax * sl2;
        const bool raise = __builtin_fmaf(lmax, sl2, -mref) > kUp + kSlack;
        if (__any(raise)) {
          const float ref = tmax - kUp;  // whatever its rounding, the partial's own
          const float alpha = raise ? exp2_fast(mref - ref) : 1.f;
          lsum *= alpha;
#pragma unroll
          for (int t = 0; t < DB; ++t) acc[t] *= alpha;
          mref = raise ? ref : mref;
          weights();
        }
      }
      lsum += ps;
      // O^T += V^T P^T: k-step ss holds the lane's elements 8ss..8ss+7, keys
      // 16ss + 8(e/4) + 4h + e%4, the keys that the transposing reads deliver.
      u32x4 hi[2], lo[2];
#pragma unroll
      for (int ss = 0; ss < 2; ++ss) {
        uint32_t h4[4], l4[4] = {0, 0, 0, 0};
        if constexpr (kHalf) {
#pragma unroll
          for (int w = 0; w < 4; ++w) h4[w] = pack_f16(pr[8 * ss + 2 * w], pr[8 * ss + 2 * w + 1]);
        } else {
          split_weights<4>(pr + 8 * ss, h4, l4);
        }
        hi[ss] = u32x4{h4[0], h4[1], h4[2], h4[3]};
        lo[ss] = u32x4{l4[0], l4[1], l4[2], l4[3]};
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      if (b + 1 < SK / 32)
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) kw[ks] = read128(kb + 32 * (b + 1) * KROW + 32 * ks);
#pragma unroll
      for (int ss = 0; ss < 2; ++ss) {
#pragma unroll
        for (int t = 0; t < DB; ++t)
          acc[t] = kHalf ? mfma32_f16(vw[ss][t], hi[ss], acc[t]) : mfma32(vw[ss][t], hi[ss], acc[t]);
        if constexpr (!kHalf)
#pragma unroll
          for (int t = 0; t < DB; ++t) acc[t] = mfma32(vw[ss][t], lo[ss], acc[t]);
      }
    }
  }
  if (__any(bad) && lane == 0) atomicOr(P.status, kStatusPage);
  if (!active) return;
  const float ltot = xor32_sum(lsum);
  const int row = row0 + j;
  if (row < Mh) {
    const size_t prow = ((size_t)gam * P.S_c + s) * P.M + (size_t)map * Mh + row;
    float* dst = P.ctx_acc + prow * D;
    if constexpr (KV::MX) {
#pragma unroll
      for (int t = 0; t < DB; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[t][v] = ldexpf(acc[t][v], vrefs[t]);
    }
#pragma unroll
    for (int t = 0; t < DB; ++t)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<f32x4*>(dst + 32 * t + 8 * g4 + 4 * h) =
            f32x4{acc[t][4 * g4], acc[t][4 * g4 + 1], acc[t][4 * g4 + 2], acc[t][4 * g4 + 3]};
    if (h == 0) P.ctx_ml[prow] = float2{mref, ltot};
  }
}

// Grid: n_ctx_blocks context work-groups, then one work-group for every NW / 4
// of the n_dec_blocks decode ones.
template <int D, int NW, int SK, typename KV, int MAPS, int NTD>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2))) void many_kernel(PagedAttnParams P) {
  typedef StreamLds<D, KV> S;
  constexpr int QB = q_bytes<D, NTD>();
  constexpr int UNITS = NW / kWaves;
  constexpr int CTX = 2 * SK * (PageRow<D>::KROW + PageRow<D>::VROW);
  __shared__ __attribute__((aligned(16))) unsigned char lds[cmax(CTX, UNITS * QB + NW * S::TILE)];
  const int bid = blockIdx.x;
  if (bid < P.n_ctx_blocks) {
    ctx_many_block<D, NW, SK, KV, MAPS>(P, lds);
    return;
  }
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int unit = wave / kWaves, blk = (bid - P.n_ctx_blocks) * UNITS + unit;
  unsigned char* kl = lds + UNITS * QB + wave * S::TILE;
  own_block<D, NTD, KV>(P, blk, blk < P.n_dec_blocks, wave % kWaves, lane, lds + unit * QB, kl, kl + S::KT);
}

// The end of a row's work: the maps' difference, the head's norm and the one
// rounding. Row j of a sample (head x token), elements col .. col + 3 of each map in
// the d/4 lanes of the row; the packed elements of this lane.
template <int D, int MAPS>
__device__ __forceinline__ u32x2 finish_row(const PagedCombineParams& C, int j, const f32x4& y0, const f32x4& y1, int col) {
  f32x4 r = y0;
  if constexpr (MAPS == 2) {
    r -= C.lambda[j / C.ntok] * y1;
    if (C.weight) {
      auto mean_square = [&]() {
        float sq = r[0] * r[0] + r[1] * r[1] + r[2] * r[2] + r[3] * r[3];
        if constexpr (D == 128) sq = xor16_sum(sq);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) sq += __shfl_xor(sq, o);
        return sq * (1.f / D);
      };
      float mean = mean_square() + C.eps;
      // Squares at the ends of fp32's range, or past them: once more with the row
      // times a power of two, which the quotient does not see.
      const bool fits = mean > 0x1p-80f && mean < 0x1p120f;
      if (__any(!fits)) {
        const float by = fits ? 1.f : mean < 1.f ? 0x1p96f : 0x1p-70f;
        r *= by;
        mean = mean_square() + C.eps * by * by;  // 0: a row of zeros, which stays one
      }
      r *= *reinterpret_cast<const f32x4*>(C.weight + col) * (mean == 0.f ? 0.f : 1.f / sqrtf(mean));
    }
    r *= C.out_scale;
  }
  return u32x2{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
}

// ---------------------------------------------------------------------------
// Combine: a wave per output row (and map) merges the row's partials into
//   softmax @ V = vs sum_k 2^(m_k - M) acc_k / sum_k 2^(m_k - M) l_k
// (0 where no key was seen); the maps meet in LDS, and the first one's wave
// subtracts them, normalises the head and rounds the result to bf16 once. 16
// bytes of a value row per lane, so a load reads 256/D partials' rows; NL loads
// are issued ahead with the statistics. A chain of latencies for few rows (1024
// of 10 partials: 4.2 us), the partials' bytes for many (4096 of 16: 8.1 us for
// 35 MB, written by other XCDs).
template <int D, int NL, int MAPS>
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedCombineParams C) {
  constexpr int LPR = D / 4, PPL = 64 / LPR;
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int sub = lane / LPR, col = 4 * (lane % LPR);
  const int map = MAPS == 2 ? wave & 1 : 0;
  const int at = blockIdx.x * (4 / MAPS) + wave / MAPS, row = min(at, C.b * C.hn - 1);
  const int i = row / C.hn, j = row - i * C.hn;
  const int gam = j / C.pn, jp = j - gam * C.pn;
  if (j == 0 && lane == 0 && C.lens) {
    const int raw = C.lens[i];
    if (raw < 0 || raw > C.m_d_max) atomicOr(C.status, kStatusLens);
  }
  const float vs = C.v_scale ? C.v_scale[gam] : 1.f;
  if (i == 0 && jp == 0 && lane == 0) {
    const float ks = C.k_scale ? C.k_scale[gam] : 1.f;
    const bool ok = ks >= __FLT_MIN__ && ks <= __FLT_MAX__ && vs >= __FLT_MIN__ && vs <= __FLT_MAX__;
    if (!ok) atomicOr(C.status, kStatusScale);
  }
  const int np = C.S_c + C.S_d;
  auto merged = [&]() {
    const size_t cbase = (size_t)gam * C.S_c * C.M + (size_t)map * C.Mh + (size_t)i * C.pn + jp;  // + k*M
    const size_t dbase = ((size_t)(i * C.g + gam) * C.S_d) * C.R + map * C.pn + jp;               // + k*R
    const size_t coff = (size_t)sub * C.M * D + col, doff = (size_t)sub * C.R * D + col;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float L = 0.f, mx = kNegInf;
    for (int k0 = 0; k0 < np; k0 += 64) {
      const int k1 = min(k0 + 64, np);
      const int ce = min(k1, C.S_c), d0 = max(k0, C.S_c);
      const int nc = k0 < ce ? (ce - k0 + PPL - 1) / PPL : 0;
      const int nl = nc + (d0 < k1 ? (k1 - d0 + PPL - 1) / PPL : 0);
      f32x4 v[NL];
      auto load = [&](int l0) {
#pragma unroll
        for (int u = 0; u < NL; ++u) {
          const int l = l0 + u;
          if (l < nc) {
            const int k = k0 + l * PPL;
            const float* a = C.ctx_acc + (cbase + (size_t)k * C.M) * D;
            v[u] = *reinterpret_cast<const f32x4*>(a + (k + sub < ce ? coff : col));
          } else if (l < nl) {
            const int k = d0 + (l - nc) * PPL;
            const float* a = C.dec_acc + (dbase + (size_t)(k - C.S_c) * C.R) * D;
            v[u] = *reinterpret_cast<const f32x4*>(a + (k + sub < k1 ? doff : col));
          }
        }
      };
      load(0);
      const int k = k0 + lane;
      float2 ml = float2{kNegInf, 0.f};
      if (k < k1)
        ml = k < C.S_c ? C.ctx_ml[cbase + (size_t)k * C.M] : C.dec_ml[dbase + (size_t)(k - C.S_c) * C.R];
      const float mnew = fmaxf(mx, wave_max(ml.x));
      const float base = mnew == kNegInf ? 0.f : mnew;
      const float rescale = exp2_fast(mx - base);
      L *= rescale;
      acc *= rescale;
      mx = mnew;
      const float w = exp2_fast(ml.x - base);
      L += wave_sum(w * ml.y);
      for (int l0 = 0; l0 < nl; l0 += NL) {
        if (l0 > 0) load(l0);
#pragma unroll
        for (int u = 0; u < NL; ++u) {
          const int l = l0 + u;
          const int kf = l < nc ? k0 + l * PPL : d0 + (l - nc) * PPL;
          const int kend = l < nc ? ce : k1;
          const float wu = __shfl(w, min(kf + sub - k0, 63));
          if (l < nl) {
            const bool mine = kf + sub < kend;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += (mine ? v[u][e] : 0.f) * wu;
          }
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (PPL == 4) acc[e] = xor16_sum(acc[e]);
      acc[e] = xor32_sum(acc[e]);
    }
    const float inv = L == 0.f ? 0.f : vs / L;  // no key seen: 0
    return acc * inv;
  };
  const f32x4 y0 = merged();
  f32x4 y1 = y0;
  if constexpr (MAPS == 2) {
    __shared__ f32x4 second[2][LPR];
    if (map == 1 && sub == 0) second[wave / 2][lane] = y0;
    __syncthreads();
    y1 = second[wave / 2][lane % LPR];
  }
  const u32x2 o = finish_row<D, MAPS>(C, j, y0, y1, col);
  if (map == 0 && sub == 0 && at < C.b * C.hn) *reinterpret_cast<u32x2*>(C.out + (size_t)row * D + col) = o;
}

// ---------------------------------------------------------------------------
// Small steps: work-group (sample, group) streams the unit's context and own
// rows as one softmax and writes the output: one launch, no partials. The
// context is read once per sample, so this pays where launches and latency set
// the time (4 samples of 4 heads over 128 rows: 4.8 us on the GPU, 8.0 a call;
// in parts 8.7 a call at least).
template <int D, typename KV, int NT, int MAPS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void whole_kernel(PagedWholeParams W) {
  typedef StreamLds<D, KV> S;
  constexpr int KS = D / 32, QB = q_bytes<D, NT>(), LPR = D / 4, RPW = 64 / LPR;
  constexpr int LD = PageMerge<D, NT>::LD, ROWS = PageMerge<D, NT>::ROWS;
  __shared__ __attribute__((aligned(16))) unsigned char lds[QB + cmax(kWaves * S::TILE, PageMerge<D, NT>::bytes)];
  const PagedAttnParams& P = W.A;
  const PagedCombineParams& C = W.C;
  const int lane = threadIdx.x & 63, wave = wave_id();
  const int gam = blockIdx.x % P.g, i = blockIdx.x / P.g;
  unsigned char* kl = lds + QB + wave * S::TILE;
  unsigned char* vl = kl + S::KT;
  constexpr int stride = kWaves * kTileKeys;
  const int k0 = wave * kTileKeys;
  const int32_t* table = P.tables + (size_t)i * P.table_pages;
  int c0 = 0, c1 = 0, o0 = 0, o1 = 0, raw = 0;  // first page ids, all requested together
  if (P.m_c > 0) {
    c0 = tile_ids(P.ctx_table, min(k0, P.m_c - 1), P.m_c, P.pool.shift, lane);
    c1 = tile_ids(P.ctx_table, min(k0 + stride, P.m_c - 1), P.m_c, P.pool.shift, lane);
  }
  if (P.m_d_max > 0) {
    o0 = tile_ids(table, min(k0, P.m_d_max - 1), P.m_d_max, P.pool.shift, lane);
    o1 = tile_ids(table, min(k0 + stride, P.m_d_max - 1), P.m_d_max, P.pool.shift, lane);
    raw = P.lens[i];
  }
  const OwnRows rows = {P.q + ((size_t)i * P.hn + (size_t)gam * P.pn) * D, D, P.R, P.pn};
  u32x4 qreg[NT == 1 ? KS : 1];
  if constexpr (NT == 1) {
#pragma unroll
    for (int k = 0; k < KS; ++k) qreg[k] = query_slot<D, KV>(rows, 0, k, P.maps, P.q_sign, lane);
  } else {
    for (int k = wave; k < NT * KS; k += kWaves)
      write128(lds + (k * 64 + lane) * 16, query_slot<D, KV>(rows, k / KS, k % KS, P.maps, P.q_sign, lane));
    __syncthreads();
  }
  auto q_at = [&](int nt, int k) -> u32x4 {
    if constexpr (NT == 1) return qreg[k];
    return *(volatile const lds_u32x4*)(lds + ((nt * KS + k) * 64 + lane) * 16);
  };
  PageState<D, NT> st;
  st.init();
  const float sl2 = group_scale_log2(P, gam);
  // the context's rows are read by the group's other samples too: cached
  bool bad = stream_pages<D, NT, KV, 0>(st, P.pool, gam, P.ctx_table, q_at, kl, vl, c0, c1, k0, P.m_c, P.m_c, stride, 1,
                                        MAPS == 2 ? P.pn : 0, sl2, lane);
  const int total = scalar(raw < 0 ? 0 : (raw > P.m_d_max ? P.m_d_max : raw));
  bad |= stream_pages<D, NT, KV>(st, P.pool, gam, table, q_at, kl, vl, o0, o1, k0, total, total, stride, P.ntok,
                                     MAPS == 2 ? P.pn : 0, sl2, lane);
  if (__any(bad) && lane == 0) atomicOr(P.status, kStatusPage);
  total_sums(st);
  float* merge = reinterpret_cast<float*>(lds + QB);
  merge_states(st, merge, wave, lane);
  const float* l_s = merge + ROWS * LD + ROWS;
  const float vs = C.v_scale ? C.v_scale[gam] : 1.f;
  const int sub = lane / LPR, col = 4 * (lane % LPR);
  for (int r0 = wave * RPW; r0 < P.pn; r0 += kWaves * RPW) {
    const int jp = r0 + sub, row = min(jp, P.pn - 1), j = gam * P.pn + row;
    f32x4 y[MAPS];
#pragma unroll
    for (int u = 0; u < MAPS; ++u) {
      const int r = u * P.pn + row;
      const float L = l_s[r];
      y[u] = *reinterpret_cast<const f32x4*>(merge + r * LD + col) * (L == 0.f ? 0.f : vs / L);
    }
    const u32x2 o = finish_row<D, MAPS>(C, j, y[0], y[MAPS - 1], col);
    if (jp < P.pn) *reinterpret_cast<u32x2*>(C.out + ((size_t)i * P.hn + j) * D + col) = o;
  }
  if (threadIdx.x == 0) {
    int flags = gam == 0 && P.m_d_max > 0 && (raw < 0 || raw > P.m_d_max) ? kStatusLens : 0;
    if (i == 0) {
      const float ks = C.k_scale ? C.k_scale[gam] : 1.f;
      if (!(ks >= __FLT_MIN__ && ks <= __FLT_MAX__ && vs >= __FLT_MIN__ && vs <= __FLT_MAX__)) flags |= kStatusScale;
    }
    if (flags) atomicOr(P.status, flags);
  }
}

template <typename Prm>
hipError_t go(void (*kernel)(Prm), int grid, int block, hipStream_t stream, hipEvent_t stop, const Prm& p) {
  if (stop)
    hipExtLaunchKernelGGL(kernel, dim3(grid), dim3(block), 0, stream, nullptr, stop, 0, p);
  else
    kernel<<<grid, block, 0, stream>>>(p);
  return hipGetLastError();
}

template <int D, typename KV>
hipError_t stream_dk(const PagedAttnParams& P, int tc, int td, hipStream_t s) {
  const int grid = P.n_ctx_small_blocks + P.n_dec_blocks;
  if (grid == 0) return hipSuccess;
  if (td == 4)
    return tc == 0   ? go(stream_kernel<D, KV, 0, 4>, grid, kThreads, s, nullptr, P)
           : tc == 4 ? go(stream_kernel<D, KV, 4, 4>, grid, kThreads, s, nullptr, P)
                     : hipErrorInvalidValue;
  if (td == 2)
    return tc == 0   ? go(stream_kernel_2w<D, KV, 0, 2>, grid, kThreads, s, nullptr, P)
           : tc == 2 ? go(stream_kernel_2w<D, KV, 2, 2>, grid, kThreads, s, nullptr, P)
                     : hipErrorInvalidValue;
  if (td != 1) return hipErrorInvalidValue;
  if constexpr (KV::MX) {
    switch (tc) {
      case 0: return go(stream_kernel_3w<D, KV, 0, 1>, grid, kThreads, s, nullptr, P);
      case 1: return go(stream_kernel_3w<D, KV, 1, 1>, grid, kThreads, s, nullptr, P);
      case 2: return go(stream_kernel_3w<D, KV, 2, 1>, grid, kThreads, s, nullptr, P);
      default: return hipErrorInvalidValue;
    }
  } else switch (tc) {
    case 0: return go(stream_kernel_2w<D, KV, 0, 1>, grid, kThreads, s, nullptr, P);
    case 1: return go(stream_kernel_2w<D, KV, 1, 1>, grid, kThreads, s, nullptr, P);
    case 2: return go(stream_kernel_2w<D, KV, 2, 1>, grid, kThreads, s, nullptr, P);
    default: return hipErrorInvalidValue;
  }
}

template <int D, typename KV, int MAPS, int NTD>
hipError_t many_dkmn(const PagedAttnParams& P, hipStream_t s) {
  const int per = P.ctx_wide / kWaves;
  const int grid = P.n_ctx_blocks + (P.n_dec_blocks + per - 1) / per;
  if (P.ctx_wide == 8) return go(many_kernel<D, 8, 128, KV, MAPS, NTD>, grid, 512, s, nullptr, P);
  if (P.ctx_wide == 4) return go(many_kernel<D, 4, 64, KV, MAPS, NTD>, grid, 256, s, nullptr, P);
  return hipErrorInvalidValue;
}
template <int D, typename KV> hipError_t many_dk(const PagedAttnParams& P, int td, hipStream_t s) {
  if (P.ctx_wide != 4 && P.ctx_wide != 8) return hipErrorInvalidValue;
  if (P.n_dec_blocks > 0 && td > 2) return hipErrorInvalidValue;
  const bool two = P.n_dec_blocks > 0 && td == 2;
  if (P.maps == 2) return two ? many_dkmn<D, KV, 2, 2>(P, s) : many_dkmn<D, KV, 2, 1>(P, s);
  return two ? many_dkmn<D, KV, 1, 2>(P, s) : many_dkmn<D, KV, 1, 1>(P, s);
}

template <int D, int MAPS> hipError_t combine_dm(const PagedCombineParams& C, hipStream_t s, hipEvent_t stop) {
  const int rows = 4 / MAPS, grid = (C.b * C.hn + rows - 1) / rows, per = 256 / D;
  const int loads = (C.S_c + per - 1) / per + (C.S_d + per - 1) / per;
  // All of a row's loads at once need registers that leave three waves per SIMD:
  // only where that holds every row (4096 rows of 17 partials: 10.5 us, 7.1 in
  // two batches of 8).
  const bool one_round = grid <= 3 * 256;
  return loads <= 4   ? go(paged_combine_kernel<D, 4, MAPS>, grid, 256, s, stop, C)
         : loads <= 8 || !one_round ? go(paged_combine_kernel<D, 8, MAPS>, grid, 256, s, stop, C)
                      : go(paged_combine_kernel<D, 16, MAPS>, grid, 256, s, stop, C);
}

template <int D, typename KV, int MAPS>
hipError_t whole_dkm(const PagedWholeParams& W, int tiles, hipStream_t s, hipEvent_t stop) {
  const int grid = W.A.b * W.A.g;
  if (tiles == 1) return go(whole_kernel<D, KV, 1, MAPS>, grid, kThreads, s, stop, W);
  if (tiles == 2) return go(whole_kernel<D, KV, 2, MAPS>, grid, kThreads, s, stop, W);
  return hipErrorInvalidValue;
}
template <int D, typename KV>
hipError_t whole_dk(const PagedWholeParams& W, int tiles, hipStream_t s, hipEvent_t stop) {
  return W.A.maps == 2 ? whole_dkm<D, KV, 2>(W, tiles, s, stop) : whole_dkm<D, KV, 1>(W, tiles, s, stop);
}

}  // namespace

hipError_t launch_paged_whole(const PagedWholeParams& W, int d, int kv, int tiles, hipStream_t s, hipEvent_t stop) {
  if (d == 128) {
    if (kv == kPagedBf16) return whole_dk<128, PgBf16>(W, tiles, s, stop);
    if (kv == kPagedFp8) return whole_dk<128, PgFp8>(W, tiles, s, stop);
    if (kv == kPagedMxfp4) return whole_dk<128, PgMx4>(W, tiles, s, stop);
  } else if (d == 64) {
    if (kv == kPagedBf16) return whole_dk<64, PgBf16>(W, tiles, s, stop);
    if (kv == kPagedFp8) return whole_dk<64, PgFp8>(W, tiles, s, stop);
    if (kv == kPagedMxfp4) return whole_dk<64, PgMx4>(W, tiles, s, stop);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_paged_stream(const PagedAttnParams& P, int d, int kv, int tc, int td, hipStream_t s) {
  if (d == 128) {
    if (kv == kPagedBf16) return stream_dk<128, PgBf16>(P, tc, td, s);
    if (kv == kPagedFp8) return stream_dk<128, PgFp8>(P, tc, td, s);
    if (kv == kPagedMxfp4) return stream_dk<128, PgMx4>(P, tc, td, s);
  } else if (d == 64) {
    if (kv == kPagedBf16) return stream_dk<64, PgBf16>(P, tc, td, s);
    if (kv == kPagedFp8) return stream_dk<64, PgFp8>(P, tc, td, s);
    if (kv == kPagedMxfp4) return stream_dk<64, PgMx4>(P, tc, td, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_paged_wide(const PagedAttnParams& P, int d, int kv, int td, hipStream_t s) {
  if (d == 128) {
    if (kv == kPagedBf16) return many_dk<128, PgBf16>(P, td, s);
    if (kv == kPagedFp8) return many_dk<128, PgFp8>(P, td, s);
    if (kv == kPagedMxfp4) return many_dk<128, PgMx4>(P, td, s);
  } else if (d == 64) {
    if (kv == kPagedBf16) return many_dk<64, PgBf16>(P, td, s);
    if (kv == kPagedFp8) return many_dk<64, PgFp8>(P, td, s);
    if (kv == kPagedMxfp4) return many_dk<64, PgMx4>(P, td, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_paged_combine(const PagedCombineParams& C, int d, hipStream_t s, hipEvent_t stop) {
  if (d == 128) return C.maps == 2 ? combine_dm<128, 2>(C, s, stop) : combine_dm<128, 1>(C, s, stop);
  if (d == 64) return C.maps == 2 ? combine_dm<64, 2>(C, s, stop) : combine_dm<64, 1>(C, s, stop);
  return hipErrorInvalidValue;
}

}  // namespace bifattn
