// Products of matrices in 8-bit floats: what their kernels take, and the arithmetic behind the sums.
#pragma once

#include "fp8.h"

namespace qgtc {

struct ProductParams;
// Tiles of 256 x 256 (product_tile.hip), for results of 16 and 8 bits.
template <int MODE> qgtc_status launch_tiles(const ProductParams& p, hipStream_t stream);
// Tiles of 128 x 128 (product_mid.hip); wide: with fp32's sums.
template <int MODE> qgtc_status launch_mid(const ProductParams& p, bool wide, hipStream_t stream);

enum { kProduct = 0, kGated = 1, kGatedGrad = 2 };  // what is made of the sums

struct Fp8Operand {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t ld, ld_scales;
  int32_t rows;
};

struct ProductParams {
  Fp8Operand x, w, u;        // u: the second projection
  int32_t blocks;            // of K
  int32_t rows, cols;        // of the result
  int32_t type, act;
  void* out;                 // the product; h; dg
  int64_t ld_out;
  void* out2;                // du
  int64_t ld_out2;
  float* wide;               // h in fp32
  int64_t ld_wide;
  const void* dh;
  int64_t ld_dh;
  uint8_t* codes;            // h in 8-bit floats
  uint8_t* scales;
  int64_t ld_codes, ld_scales;
};

#if defined(__HIPCC__)

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

// A block of K, 16 rows of W by 16 rows of X, on the matrix cores.  Lane l has row l % 16 of each and 32 of its 128 codes, the same
// ones of both, and gets the sums of W's rows 4 (l / 16) + 0..3 with X's row l % 16.  B: the block's byte in the words of scales.
//
// For results of 16 or 8 bits one v_mfma_scale_f32_16x16x128_f8f6f4, which applies the scales as well.  It adds groups of 8
// products (consecutive codes), cutting each at 2^-13 of its group's largest, and the groups' sums in fp32: normal data come
// out 1.5e-5 of the result off (2-norms), a hundredth and less of what rounding to bf16 (2e-3) or fp16 (2.4e-4: a sixteenth) does.
// Where a group's large products cancel, what was cut off its small ones is more than that of what is left.
template <int B>
__device__ __forceinline__ v4f block_mfma(const v8i& w, const v8i& x, const v4f& acc, uint32_t sw, uint32_t sx) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc, 0, 0, B, (int)sw, B, (int)sx);
}
// For results of 32 bits operands go as bf16 to four v_mfma_f32_16x16x32_bf16, whose products are exact and whose sums fp32's: 7e-9 off
// on the same data, at half the rate.  bf16 holds a code exactly, and with its scale too if that does not leave fp32's range: values are
// lifted by 2^10, so that the smallest (2^-9 * 2^-127) are not subnormal, and the sums are put back by 2^-20.  What is too large for
// that (scales from 2^109 on, sums from 2^108 on) turns the sum into an infinity or a NaN.  A wave that ends with one makes its sums
// again, APART: codes alone, and both scales with the sum of each block, as one exponent, and takes those that were none from there (the
// others stay: a row's results do not depend on the rows beside it).  That way holds for every scale: 386 us
// for 8192 x 4096 x 4096 by it alone, 295 by the other.
constexpr int kLift = 10;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
struct WideCodes {
  bf16x8 v[4];
};
template <int B, bool APART>
__device__ __forceinline__ WideCodes widen(const v8i& codes, uint32_t scales) {
  const uint32_t e = scales >> (8 * B) & 255u;
  // (an infinity is e8m0's NaN to the conversion and makes every code NaN)
  const float two = APART ? (e == 255u ? __builtin_inff() : 1.0f) : __uint_as_float(min(e + kLift, 255u) << 23);
  WideCodes w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * i], two, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * i], two, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * i + 1], two, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * i + 1], two, true);
    w.v[i] = (bf16x8){a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
  }
  return w;
}
__device__ __forceinline__ v4f wide_mfma(const WideCodes& w, const WideCodes& x, v4f acc) {
#pragma unroll
  for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[i], x.v[i], acc, 0, 0, 0);
  return acc;
}
// The same for codes without their scales: rows are the words of scales of W's rows 4 (l / 16) + 0..3, of which the byte at `bit`
// counts, and sx X's scale.
__device__ __forceinline__ v4f apart_mfma(const WideCodes& w, const WideCodes& x, v4f acc, const v4i& rows, int bit, uint32_t sx) {
  const v4f sum = wide_mfma(w, x, (v4f){0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] += ldexpf(sum[i], (int)(((uint32_t)rows[i] >> bit & 255u) + sx) - 254);
  return acc;
}
__device__ __forceinline__ void take_apart(v4f& acc, const v4f& apart) {
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = abs_bits(acc[i]) >= 0x7f800000u ? apart[i] : acc[i];
}
// Puts lifted sums back; whether one of them is none.
__device__ __forceinline__ bool put_back(v4f& acc) {
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    top = max(top, abs_bits(acc[i]));
    acc[i] *= 0x1p-20f;
  }
  static_assert(kLift == 10, "both operands are lifted");
  return top >= 0x7f800000u;
}

// 32 codes of a lane's row: bytes 16 g and 64 + 16 g of the block on.
__device__ __forceinline__ v8i lane_codes(const uint8_t* p) {
  const v4i a = *reinterpret_cast<const v4i*>(p), b = *reinterpret_cast<const v4i*>(p + 64);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// exp(-a) for a >= 0 with one more step than the instruction alone: the product with log2(e) is rounded, and what the rounding left off
// is put back, so that the relative error stays near one unit for every a instead of growing with it.  0 where it is below 2^-126.
__device__ __forceinline__ float exp_minus(float a) {
  a = a > 150.0f ? 150.0f : a;                       // (an infinity times its rounding is NaN; NaN stays)
  const float hi = a * -1.44269504f, lo = fmaf(a, -1.44269504f, -hi) + a * -1.92596299e-8f;
  const float e = __builtin_amdgcn_exp2f(hi);
  return fmaf(e, lo * 0.693147181f, e);
}
// act(g) = g * s(z(g)), s the sigmoid, z = g (silu) or 2 sqrt(2/pi) (g + 0.044715 g^3) (gelu: (1 + tanh(z/2)) / 2 = s(z)).
// Its slope is s + g z' s (1 - s).  g z' grows as g^3 and beyond fp32's range, while s (1 - s) is 0 from |z| = 88 on, where g z' is below
// 3 * 88: held to 512 it changes no product that is not 0 anyway, and no infinity meets a 0.
struct Gate {
  float value, slope;
};
template <bool PRECISE>
__device__ __forceinline__ Gate gate(int act, float g) {
  float z = g, dz = 1.0f;
  if (act == QGTC_ACT_GELU) {
    const float k = 1.59576912f, g2 = g * g;
    z = k * fmaf(0.044715f * g2, g, g);
    dz = k * fmaf(0.134145f, g2, 1.0f);
  }
  const float t = __builtin_amdgcn_fmed3f(g * dz, -512.0f, 512.0f);   // (of NaN anything: s is NaN then)
  if constexpr (PRECISE) {
    const float e = exp_minus(fabsf(z)), r = __builtin_amdgcn_rcpf(1.0f + e), less = e * r;   // the sigmoids of |z| and -|z|
    const float s = z < 0.0f ? less : r;
    return {g * s, fmaf(t, less * r, s)};
  } else {
    // For results of 16 and 8 bits: off by |z| 2^-24 of the sigmoid, which is below 2^-16 where it is not below 2^-360 itself.
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
    return {g * s, s * fmaf(t, 1.0f - s, 1.0f)};
  }
}

// Scales of blocks of h beside a border: the 8-bit instruction's cuts move an entry of normal data by some 2^-17 of it, and now and then by
// 2^-12, which chose the other of two scales in 6 of 262144 blocks.  Where the block's largest entry lies within 2^-11 of a border the
// entries that near are computed again with fp32's sums, a wave an entry, in two blocks of a thousand, and choose.  5 % of the time of
// 4096 x 4096 x 8192 (238 us, and 225 without, on one device).  Where sums cancel, cuts can be larger than that window: the scale is
// then that of the sums that were cut, as the codes are.
constexpr uint32_t kNear = 1u << 12;               // in units of 2^-23
__device__ __forceinline__ bool near_border(uint32_t top) {
  return top < 0x7f800000u && top >= 0x01000000u && (top & 0x7fffffu) - (0x600000u - kNear) <= 2 * kNear;
}
// The bits from which on an entry may be the largest of such a block.
__device__ __forceinline__ uint32_t border_from(uint32_t top) { return ((top & 0x7f800000u) | 0x600000u) - kNear; }
// What such a block's scale is made from: the border itself or the next number above it, by the entry that was computed again, and nothing
// further away.  Where sums cancel that entry may be any number, but the codes are of the sums that were cut, with `top` among them.
__device__ __forceinline__ uint32_t border_side(uint32_t top, uint32_t exact) {
  const uint32_t border = (top & 0x7f800000u) | 0x600000u;
  return exact > border ? border + 1u : border;
}

// h of row m and column n (of all lanes alike), by all 64 lanes: 16 codes a lane at a time.
__device__ __forceinline__ float exact_h(const ProductParams& p, int64_t m, int64_t n) {
  const int lane = (int)(threadIdx.x & 63u);
  float sum[2] = {0.0f, 0.0f};
  auto one = [&](int c) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(p.x.codes + m * p.x.ld + (int64_t)c * 16);
    const int ex = p.x.scales[m * p.x.ld_scales + (c >> 3)];
    u32x4 w[2];
    int ew[2];
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const Fp8Operand& o = d ? p.u : p.w;
      w[d] = *reinterpret_cast<const u32x4*>(o.codes + n * o.ld + (int64_t)c * 16);
      ew[d] = o.scales[n * o.ld_scales + (c >> 3)];
    }
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      float part = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 xl = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[i], false), xh = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[i], true);
        const f32x2 wl = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[d][i], false), wh = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[d][i], true);
        part = fmaf(xl.x, wl.x, part);
        part = fmaf(xl.y, wl.y, part);
        part = fmaf(xh.x, wh.x, part);
        part = fmaf(xh.y, wh.y, part);
      }
      sum[d] += ldexpf(part, ex + ew[d] - 254);
    }
  };
  const int pieces = p.blocks * 8;
  int c = lane;
#pragma unroll 1
  for (; c + 192 < pieces; c += 256) {               // (four pieces on their way at once)
#pragma unroll
    for (int i = 0; i < 4; ++i) one(c + 64 * i);
  }
#pragma unroll 1
  for (; c < pieces; c += 64) one(c);
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) {
    sum[0] += __shfl_xor(sum[0], s);
    sum[1] += __shfl_xor(sum[1], s);
  }
  return gate<true>(p.act, sum[0]).value * sum[1];
}
// The largest of a lane's entries `want` (bit i: the one of row m and column n0 + i), computed again; the lanes' that share a row are
// the caller's to put together.
__device__ __forceinline__ uint32_t exact_top(const ProductParams& p, int m, int n0, uint32_t want) {
  uint32_t top = 0u;
#pragma unroll 1
  for (uint64_t lanes = __ballot(want != 0u); lanes; lanes = __ballot(want != 0u)) {
    const int from_lane = __ffsll((unsigned long long)lanes) - 1;
    const int mi = __builtin_amdgcn_readlane(m, from_lane), ni = __builtin_amdgcn_readlane(n0 + __ffs(want) - 1, from_lane);
    const uint32_t bits = abs_bits(exact_h(p, mi, ni));
    if ((int)(threadIdx.x & 63u) == from_lane) {
      top = max(top, bits);
      want &= want - 1u;
    }
  }
  return top;
}

// Four entries of a row from column c on.
template <int TYPE>
__device__ __forceinline__ void store4_of(void* base, int64_t at, int left, const float (&v)[4]) {
  typename Float<TYPE>::type* const to = (typename Float<TYPE>::type*)base + at;
  if (left >= 4) {
    Float<TYPE>::store4(to, v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) Float<TYPE>::store(to + i, v[i]);
  }
}
__device__ __forceinline__ void store4_as(int type, void* base, int64_t at, int left, const float (&v)[4]) {
  if (type == QGTC_F32) store4_of<QGTC_F32>(base, at, left, v);
  else if (type == QGTC_F16) store4_of<QGTC_F16>(base, at, left, v);
  else store4_of<QGTC_BF16>(base, at, left, v);
}
__device__ __forceinline__ float load_as(int type, const void* base, int64_t at) {
  if (type == QGTC_F32) return Float<QGTC_F32>::load((const float*)base + at);
  if (type == QGTC_F16) return Float<QGTC_F16>::load((const uint16_t*)base + at);
  return Float<QGTC_BF16>::load((const uint16_t*)base + at);
}
// Eight entries of row m from column n on.  WIDE: fp32, else one of the types of 16 bits.
template <bool WIDE>
__device__ __forceinline__ void store8_as(int type, void* base, int64_t ld, int m, int n, int cols, const float (&v)[8]) {
  if constexpr (WIDE) store8_of<QGTC_F32>((float*)base + (int64_t)m * ld, n, cols, v);
  else if (type == QGTC_F16) store8_of<QGTC_F16>((uint16_t*)base + (int64_t)m * ld, n, cols, v);
  else store8_of<QGTC_BF16>((uint16_t*)base + (int64_t)m * ld, n, cols, v);
}
template <bool WIDE>
__device__ __forceinline__ void load8_as(int type, const void* base, int64_t ld, int m, int n, int cols, float (&v)[8]) {
  if constexpr (WIDE) load8_of<QGTC_F32>((const float*)base + (int64_t)m * ld, n, cols, v);
  else if (type == QGTC_F16) load8_of<QGTC_F16>((const uint16_t*)base + (int64_t)m * ld, n, cols, v);
  else load8_of<QGTC_BF16>((const uint16_t*)base + (int64_t)m * ld, n, cols, v);
}

#endif  // __HIPCC__

}  // namespace qgtc
