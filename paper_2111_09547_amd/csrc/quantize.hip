// 8-bit floats: descriptors, checks, and whole matrices into the form, along their rows or along their columns.
#include "fp8.h"

namespace qgtc {

qgtc_status check_fp8(const qgtc_fp8* m) {
  if (!m) return QGTC_ERR_NULL;
  if (m->rows < 0 || m->cols < 0 || m->rows > kMostEntries || m->cols > kMostEntries) return QGTC_ERR_SHAPE;
  if (m->rows > 0 && m->cols > 0 && (!m->codes || !m->scales)) return QGTC_ERR_NULL;
  if ((m->ld & (kBlock - 1)) != 0 || ((uintptr_t)m->codes & 15u) != 0) return QGTC_ERR_ALIGN;
  if ((m->ld_scales & 3) != 0 || ((uintptr_t)m->scales & 3u) != 0) return QGTC_ERR_ALIGN;
  if (m->ld < m->cols || m->ld_scales < fp8_blocks(m->cols)) return QGTC_ERR_SHAPE;
  return QGTC_OK;
}

qgtc_status check_matrix(const void* data, int type, int rows, int cols, int64_t ld) {
  if (!float_type(type)) return QGTC_ERR_UNSUPPORTED;
  if (!data) return QGTC_ERR_NULL;
  if (ld < cols) return QGTC_ERR_SHAPE;
  if (((uintptr_t)data & (unsigned)(float_bytes(type) - 1)) != 0) return QGTC_ERR_ALIGN;
  return QGTC_OK;
}

namespace {

struct QuantizeParams {
  const void* src;
  int64_t ld;                // elements
  int32_t rows, cols;        // of src
  uint8_t* codes;
  uint8_t* scales;
  int64_t ld_codes, ld_scales;
  uint32_t groups;           // along a row: of 512 columns
  int64_t first;             // of the launch's units
};

// Along rows: 16 lanes have a block, a wave 512 columns of a row, and ROWS of those at a time.
constexpr int kQuantRows = 4;
template <int TYPE>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const QuantizeParams p) {
  typedef typename Float<TYPE>::type T;
  const int64_t unit = p.first + blockIdx.x * 4u + (threadIdx.x >> 6), rg = unit / p.groups;
  const int c = (int)(unit - rg * p.groups) * 512 + (int)(threadIdx.x & 63u) * 8;
  const int64_t row0 = rg * kQuantRows;
  float v[kQuantRows][8];
#pragma unroll
  for (int i = 0; i < kQuantRows; ++i)
    if (row0 + i < p.rows) load8_of<TYPE>((const T*)p.src + (row0 + i) * p.ld, c, p.cols, v[i]);
#pragma unroll
  for (int i = 0; i < kQuantRows; ++i)
    if (row0 + i < p.rows) write_block8(p.codes + (row0 + i) * p.ld_codes, p.scales + (row0 + i) * p.ld_scales, c, p.cols, v[i]);
}

// Along columns: a workgroup takes 128 rows of src, a block of every column, by 64 columns, and turns them in LDS: [column]
// [row], so that a thread has 32 rows of one column and four neighbours a block.
template <int TYPE>
__global__ __launch_bounds__(256) void quantize_columns_kernel(const QuantizeParams p) {
  typedef typename Float<TYPE>::type T;
  constexpr int PITCH = kBlock + 8 / (int)sizeof(T);   // (8 bytes more: columns fall on different banks)
  __shared__ __align__(16) T tile[64 * PITCH];
  const int c0 = (int)blockIdx.x * 64, cl = (int)(threadIdx.x & 7u) * 8;
  const int64_t r0 = (int64_t)blockIdx.y * kBlock;
  const int rl = (int)(threadIdx.x >> 3) * 4;
  const T* const src = (const T*)p.src;
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    if (r0 + rl + i < p.rows) load8_of<TYPE>(src + (r0 + rl + i) * p.ld, c0 + cl, p.cols, v[i]);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float w[4] = {v[0][j], v[1][j], v[2][j], v[3][j]};
    Float<TYPE>::store4(tile + (cl + j) * PITCH + rl, w);
  }
  __syncthreads();
  const int c = (int)(threadIdx.x >> 2), k = (int)(threadIdx.x & 3u) * 32;
  float x[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) Float<TYPE>::load8(tile + c * PITCH + k + 8 * i, x[i]);
  uint32_t m = max(max(abs_max(x[0]), abs_max(x[1])), max(abs_max(x[2]), abs_max(x[3])));
  m = dpp_max<0xb1>(m);                                // quad_perm 1 0 3 2, then 2 3 0 1
  m = dpp_max<0x4e>(m);
  if (c0 + c >= p.cols) return;
  const uint32_t e = scale_byte(m);
  uint8_t* const to = p.codes + (int64_t)(c0 + c) * p.ld_codes + r0 + k;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float* const s = &x[2 * i + j / 2][4 * (j & 1)];
      w[j] = encode4(s[0], s[1], s[2], s[3], e);
      if (e == 255u) {                                 // (zeros past the end, whatever the block)
        const int64_t left = p.rows - (r0 + k + 16 * i + 4 * j);
        if (left < 4) w[j] &= left <= 0 ? 0u : 0xffffffffu >> (8 * (4 - (int)left));
      }
    }
    *reinterpret_cast<u32x4*>(to + 16 * i) = w;
  }
  if (k == 0) p.scales[(int64_t)(c0 + c) * p.ld_scales + (int64_t)blockIdx.y] = (uint8_t)e;
}

template <int TYPE>
qgtc_status launch_rows(QuantizeParams p, hipStream_t stream) {
  p.groups = (uint32_t)cdiv(p.cols, 512);
  const int64_t units = (int64_t)p.groups * cdiv(p.rows, kQuantRows);
  for (p.first = 0; p.first < units; p.first += kMostThreads / 64) {
    const int64_t here = units - p.first < kMostThreads / 64 ? units - p.first : kMostThreads / 64;
    hipLaunchKernelGGL(quantize_rows_kernel<TYPE>, dim3((unsigned)((here + 3) / 4)), dim3(256), 0, stream, p);
    const qgtc_status st = launch_status();
    if (st != QGTC_OK) return st;
  }
  return QGTC_OK;
}

template <int TYPE>
qgtc_status launch_columns(QuantizeParams p, hipStream_t stream) {
  // (a launch has at most 65535 workgroups along the second axis: rows beyond go in launches of their own)
  const int64_t most = (int64_t)65535 * kBlock;
  for (int64_t r0 = 0; r0 < p.rows; r0 += most) {
    QuantizeParams q = p;
    q.src = (const typename Float<TYPE>::type*)p.src + r0 * p.ld;
    q.rows = (int32_t)(p.rows - r0 < most ? p.rows - r0 : most);
    q.codes = p.codes + r0;
    q.scales = p.scales + r0 / kBlock;
    hipLaunchKernelGGL(quantize_columns_kernel<TYPE>, dim3((unsigned)cdiv(p.cols, 64), (unsigned)cdiv(q.rows, kBlock)), dim3(256), 0, stream, q);
    const qgtc_status st = launch_status();
    if (st != QGTC_OK) return st;
  }
  return QGTC_OK;
}

QuantizeParams params(const void* src, int rows, int cols, int64_t ld, const qgtc_fp8& dst) {
  QuantizeParams p{};
  p.src = src;
  p.ld = ld;
  p.rows = rows;
  p.cols = cols;
  p.codes = dst.codes;
  p.scales = dst.scales;
  p.ld_codes = dst.ld;
  p.ld_scales = dst.ld_scales;
  return p;
}

}  // namespace

qgtc_status quantize_rows(const void* src, int type, int rows, int cols, int64_t ld, const qgtc_fp8& dst, hipStream_t stream) {
  const QuantizeParams p = params(src, rows, cols, ld, dst);
  if (type == QGTC_F32) return launch_rows<QGTC_F32>(p, stream);
  return type == QGTC_F16 ? launch_rows<QGTC_F16>(p, stream) : launch_rows<QGTC_BF16>(p, stream);
}

}  // namespace qgtc

extern "C" qgtc_status qgtc_fp8_describe(qgtc_fp8* d, int32_t rows, int32_t cols) {
  if (!d) return QGTC_ERR_NULL;
  if (rows < 0 || cols < 0) return QGTC_ERR_SHAPE;
  d->rows = rows;
  d->cols = cols;
  d->ld = (int64_t)qgtc::fp8_blocks(cols) * qgtc::kBlock;
  d->ld_scales = ((int64_t)qgtc::fp8_blocks(cols) + 3) / 4 * 4;
  return QGTC_OK;
}

extern "C" qgtc_status qgtc_fp8_quantize(const void* src, int32_t type, int32_t rows, int32_t cols, int64_t ld_src,
                                         int32_t columns, const qgtc_fp8* dst, void* stream) {
  using namespace qgtc;
  if (rows < 0 || cols < 0) return QGTC_ERR_SHAPE;
  qgtc_status st = check_fp8(dst);
  if (st != QGTC_OK) return st;
  if (dst->rows != (columns ? cols : rows) || dst->cols != (columns ? rows : cols)) return QGTC_ERR_SHAPE;
  if (!float_type(type)) return QGTC_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return QGTC_OK;
  st = check_matrix(src, type, rows, cols, ld_src);
  if (st != QGTC_OK) return st;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  ProfScope prof(QGTC_KERNEL_PACK, s);
  if (!columns) return quantize_rows(src, type, rows, cols, ld_src, *dst, s);
  const QuantizeParams p = params(src, rows, cols, ld_src, *dst);
  if (type == QGTC_F32) return launch_columns<QGTC_F32>(p, s);
  return type == QGTC_F16 ? launch_columns<QGTC_F16>(p, s) : launch_columns<QGTC_BF16>(p, s);
}
