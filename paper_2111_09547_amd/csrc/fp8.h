// 8-bit floats (e4m3 codes, one e8m0 scale per block of 128 entries of a row): checks and device helpers shared
// by the norm, the quantizer and the products.
#pragma once

#include "qgtc_internal.h"

namespace qgtc {

constexpr int kBlock = 128;                        // entries that share a scale
constexpr int kMostEntries = 1 << 29;              // rows, and columns, of one matrix
constexpr int64_t kMostThreads = (int64_t)1 << 31; // of a launch along an axis (their number has 32 bits): what is more takes several

inline int fp8_blocks(int cols) { return cdiv(cols, kBlock); }
qgtc_status check_fp8(const qgtc_fp8* m);          // quantize.hip
inline bool float_type(int type) { return type == QGTC_F32 || type == QGTC_F16 || type == QGTC_BF16; }
inline int float_bytes(int type) { return type == QGTC_F32 ? 4 : 2; }
// A row-major tensor of rows x cols with leading dimension ld.
qgtc_status check_matrix(const void* data, int type, int rows, int cols, int64_t ld);

// Whole matrices of `rows` x `cols` floats along rows into 8-bit floats (quantize.hip).
qgtc_status quantize_rows(const void* src, int type, int rows, int cols, int64_t ld, const qgtc_fp8& dst, hipStream_t stream);

#if defined(__HIPCC__)

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// The same at an address that is only known to be a multiple of an entry's size: the vector memory unit takes any.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

// Floats of one of the three types.  f16 and bf16 are rounded to the nearest, ties to even.
template <int TYPE> struct Float;
template <> struct Float<QGTC_F32> {
  typedef float type;
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ void store(float* p, float v) { *p = v; }
  static __device__ __forceinline__ float round(float v) { return v; }
  static __device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const u32x4 a = *reinterpret_cast<const u32x4_any*>(p), b = *reinterpret_cast<const u32x4_any*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(a[i]), v[4 + i] = __uint_as_float(b[i]);
  }
  static __device__ __forceinline__ void store4(float* p, const float (&v)[4]) {
    u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]);
    *reinterpret_cast<u32x4_any*>(p) = a;
  }
  static __device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    u32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]), b[i] = __float_as_uint(v[4 + i]);
    *reinterpret_cast<u32x4_any*>(p) = a;
    *reinterpret_cast<u32x4_any*>(p + 4) = b;
  }
};
template <int TYPE> struct Half;
template <> struct Half<QGTC_F16> {
  static __device__ __forceinline__ f32x2 wide(uint32_t v) { return __builtin_convertvector(__builtin_bit_cast(f16x2, v), f32x2); }
  static __device__ __forceinline__ uint32_t narrow(f32x2 v) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2)); }
};
template <> struct Half<QGTC_BF16> {
  static __device__ __forceinline__ f32x2 wide(uint32_t v) { return (f32x2){__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)}; }
  static __device__ __forceinline__ uint32_t narrow(f32x2 v) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2)); }
};
template <int TYPE> struct Float {
  typedef uint16_t type;
  typedef Half<TYPE> H;
  static __device__ __forceinline__ float load(const uint16_t* p) { return H::wide(*p).x; }
  static __device__ __forceinline__ void store(uint16_t* p, float v) { *p = (uint16_t)H::narrow((f32x2){v, 0.0f}); }
  static __device__ __forceinline__ float round(float v) { return H::wide(H::narrow((f32x2){v, 0.0f})).x; }
  static __device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
    const u32x4 a = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 w = H::wide(a[i]);
      v[2 * i] = w.x;
      v[2 * i + 1] = w.y;
    }
  }
  static __device__ __forceinline__ void store4(uint16_t* p, const float (&v)[4]) {
    *reinterpret_cast<u32x2_any*>(p) = (u32x2){H::narrow((f32x2){v[0], v[1]}), H::narrow((f32x2){v[2], v[3]})};
  }
  static __device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
    u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = H::narrow((f32x2){v[2 * i], v[2 * i + 1]});
    *reinterpret_cast<u32x4_any*>(p) = a;
  }
};

// Eight entries of a row from column c on, zeros past its end.
template <int TYPE>
__device__ __forceinline__ void load8_of(const typename Float<TYPE>::type* row, int c, int cols, float (&v)[8]) {
  if (c + 8 <= cols) {
    Float<TYPE>::load8(row + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? Float<TYPE>::load(row + c + i) : 0.0f;
  }
}
template <int TYPE>
__device__ __forceinline__ void store8_of(typename Float<TYPE>::type* row, int c, int cols, const float (&v)[8]) {
  if (c + 8 <= cols) {
    Float<TYPE>::store8(row + c, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) Float<TYPE>::store(row + c + i, v[i]);
  }
}

// The same, kept as they come from memory until they are wanted.
template <int TYPE> struct Raw8 {
  u32x4 v;
  __device__ __forceinline__ void load(const uint16_t* row, int c, int cols) {
    if (c + 8 <= cols) {
      v = *reinterpret_cast<const u32x4_any*>(row + c);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = c + 2 * i < cols ? row[c + 2 * i] : 0u, hi = c + 2 * i + 1 < cols ? row[c + 2 * i + 1] : 0u;
        v[i] = lo | hi << 16;
      }
    }
  }
  __device__ __forceinline__ void widen(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 w = Half<TYPE>::wide(v[i]);
      f[2 * i] = w.x;
      f[2 * i + 1] = w.y;
    }
  }
};
template <> struct Raw8<QGTC_F32> {
  float v[8];
  __device__ __forceinline__ void load(const float* row, int c, int cols) { load8_of<QGTC_F32>(row, c, cols, v); }
  __device__ __forceinline__ void widen(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = v[i];
  }
};

// The largest absolute value of a block goes as its bits: among floats without a sign these order as the values do,
// infinities and NaN above all others.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
template <int N>
__device__ __forceinline__ uint32_t abs_max(const float (&v)[N]) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < N; ++i) m = max(m, abs_bits(v[i]));
  return m;
}
// The scale's byte: 448 is 1.75 * 2^8, so 1.f * 2^(E - 127) wants E - 8, and one more where 1.f > 1.75.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  if (amax >= 0x7f800000u) return 255u;
  const int e = (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 0);
}
// 2^(e - 127).
__device__ __forceinline__ float scale_value(uint32_t e) { return __uint_as_float(e ? e << 23 : 0x00400000u); }
// Four codes of values over scale_value(e).  The instruction divides by the power of two and rounds to the nearest even; nothing is
// above 448 here.
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, uint32_t e) {
  const float two = scale_value(e);
  s16x2 w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, two, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, two, true);
  return e == 255u ? 0x7f7f7f7fu : __builtin_bit_cast(uint32_t, w);
}

// The maximum over 16 consecutive lanes, which hold a block of 8 entries each.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ uint32_t max_of_16_lanes(uint32_t v) {   // rotations within rows of 16 lanes
  v = dpp_max<0x128>(v);
  v = dpp_max<0x124>(v);
  v = dpp_max<0x122>(v);
  return dpp_max<0x121>(v);
}

// Codes of a lane's eight entries from column c on, of a block shared by 16 consecutive lanes, and the block's scale.
__device__ __forceinline__ void write_block8(uint8_t* codes, uint8_t* scales, int c, int cols, const float (&v)[8], uint32_t e) {
  if ((c & ~(kBlock - 1)) >= cols) return;
  u32x2 w = {encode4(v[0], v[1], v[2], v[3], e), encode4(v[4], v[5], v[6], v[7], e)};
  if (e == 255u && c + 8 > cols) {                 // (zeros past the end, whatever the block)
    uint64_t keep = c >= cols ? 0ull : ~0ull >> (8 * (c + 8 - cols));
    w.x &= (uint32_t)keep;
    w.y &= (uint32_t)(keep >> 32);
  }
  *reinterpret_cast<u32x2*>(codes + c) = w;
  if ((c & (kBlock - 1)) == 0) scales[c / kBlock] = (uint8_t)e;
}

__device__ __forceinline__ void write_block8(uint8_t* codes, uint8_t* scales, int c, int cols, const float (&v)[8]) {
  write_block8(codes, scales, c, cols, v, scale_byte(max_of_16_lanes(abs_max(v))));
}

#endif  // __HIPCC__

}  // namespace qgtc
