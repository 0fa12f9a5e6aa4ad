// Root-mean-square norm with the residual's addition and output in 8-bit floats, and its gradients.
//
// Both are bound by memory: forward, of a bf16 row with residual, 6 bytes read and written and one of codes per entry (8192 x 4096 43 us,
// 5.5 TB/s, a copy's rate).  A row's
// entries stay in registers from the load to the codes, so everything is read once: a lane has V pieces of 8 consecutive
// entries, 16 lanes a block of 128, and a row is shared by as many waves as it takes (one wave: no LDS, four rows a workgroup).
#include "fp8.h"

namespace qgtc {
namespace {

constexpr int kMostColumns = 32768;                // 16 waves of 4 pieces a lane
constexpr int kPiece = 512;                        // columns of a wave's piece

struct NormParams {
  const void *x, *residual, *weight;
  void *sum, *y;
  float* rstd;
  uint8_t *codes, *scales;
  int64_t ld_x, ld_residual, ld_sum, ld_y, ld_codes, ld_scales;
  int32_t weight_type, rows, cols;
  float eps;
};

__device__ __forceinline__ void load_weight8(const void* w, int type, int c, int cols, float (&v)[8]) {
  if (type == QGTC_F32) load8_of<QGTC_F32>((const float*)w, c, cols, v);
  else if (type == QGTC_F16) load8_of<QGTC_F16>((const uint16_t*)w, c, cols, v);
  else load8_of<QGTC_BF16>((const uint16_t*)w, c, cols, v);
}

// The same sum in every lane, whatever the order the waves come in.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
template <bool ONE>                                // one wave to a row
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = wave_sum(v);
  if constexpr (ONE) return v;
  const int waves = (int)(blockDim.x >> 6);
  if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.0f;
  for (int i = 0; i < waves; ++i) s += part[i];
  return s;
}

template <int TYPE, int V, bool ONE>
__global__ __launch_bounds__(ONE ? 256 : 1024) void norm_kernel(const NormParams p) {
  typedef typename Float<TYPE>::type T;
  __shared__ float part[16];
  const int wave = (int)(threadIdx.x >> 6), lane = (int)(threadIdx.x & 63u);
  const int64_t row = ONE ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  if (ONE && row >= p.rows) return;
  const int c0 = (ONE ? 0 : wave * V * kPiece) + lane * 8;
  const T* const x = (const T*)p.x + row * p.ld_x;
  float s[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) load8_of<TYPE>(x, c0 + i * kPiece, p.cols, s[i]);
  if (p.residual) {
    const T* const res = (const T*)p.residual + row * p.ld_residual;
    float r[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i) load8_of<TYPE>(res, c0 + i * kPiece, p.cols, r[i]);
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[i][j] = Float<TYPE>::round(s[i][j] + r[i][j]);
  }
  if (p.sum) {
#pragma unroll
    for (int i = 0; i < V; ++i) store8_of<TYPE>((T*)p.sum + row * p.ld_sum, c0 + i * kPiece, p.cols, s[i]);
  }
  float sq = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) sq = fmaf(s[i][j], s[i][j], sq);
  const float rstd = 1.0f / sqrtf(row_sum<ONE>(sq, part) / (float)p.cols + p.eps);
  if (p.rstd && lane == 0 && (ONE || wave == 0)) p.rstd[row] = rstd;
  if (!p.y && !p.codes) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = c0 + i * kPiece;
    float w[8];
    load_weight8(p.weight, p.weight_type, c, p.cols, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[i][j] = c + j < p.cols ? s[i][j] * rstd * w[j] : 0.0f;   // (a row of NaN ends in zeros too)
    if (p.y) store8_of<TYPE>((T*)p.y + row * p.ld_y, c, p.cols, s[i]);
    if (p.codes) write_block8(p.codes + row * p.ld_codes, p.scales + row * p.ld_scales, c, p.cols, s[i]);
  }
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
__host__ __device__ inline int64_t sum_pitch(int cols) { return ((int64_t)cols + 3) / 4 * 4; }   // of a group's share of dweight

struct GradParams {
  const void *dy, *sum, *weight, *dsum;
  const float* rstd;
  void* dx;
  float *partial, *dweight;
  int64_t ld_dy, ld_sum, ld_dsum, ld_dx;
  int32_t weight_type, rows, cols, groups;
};

// A workgroup takes every groups-th row (ONE: four times as many rows, a wave each) and keeps its share of dweight in
// registers; groups' shares are added up in order by the second kernel, so the result does not depend on timing.  Where a
// wave has a row to itself its next row is on the way meanwhile and the weight stays in registers; where waves share a row that loses
// to the other workgroups of the compute unit, which fewer registers leave room for (4095 x 5120 fp16: 46 us, and 37 without, 4.5 TB/s).
template <int TYPE, int V, bool ONE>
__global__ __launch_bounds__(ONE ? 256 : 1024) void norm_grad_kernel(const GradParams p) {
  typedef typename Float<TYPE>::type T;
  __shared__ float part[2][16];
  extern __shared__ float box[];                   // ONE: the shares of three waves
  const int wave = (int)(threadIdx.x >> 6), lane = (int)(threadIdx.x & 63u);
  const int c0 = (ONE ? 0 : wave * V * kPiece) + lane * 8;
  const int64_t step = (int64_t)p.groups * (ONE ? 4 : 1);
  float w[V][8], dw[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (ONE) load_weight8(p.weight, p.weight_type, c0 + i * kPiece, p.cols, w[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = 0.0f;
  }
  struct Row {
    Raw8<TYPE> dy[V], s[V], ds[V];
    float rstd;
  };
  auto load = [&](int64_t row, Row& to) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      to.dy[i].load((const T*)p.dy + row * p.ld_dy, c0 + i * kPiece, p.cols);
      to.s[i].load((const T*)p.sum + row * p.ld_sum, c0 + i * kPiece, p.cols);
      if (p.dsum) to.ds[i].load((const T*)p.dsum + row * p.ld_dsum, c0 + i * kPiece, p.cols);
    }
    to.rstd = p.rstd[row];
  };
  int64_t row = ONE ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  Row now, then;
  if (ONE && row < p.rows) load(row, now);
  int turn = 0;
  for (; row < p.rows; row += step) {
    if (!ONE) load(row, now);
    else if (row + step < p.rows) load(row + step, then);
    float dy[V][8], s[V][8];
    const float rstd = now.rstd;
    float along = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      now.dy[i].widen(dy[i]);
      now.s[i].widen(s[i]);
      if (!ONE) load_weight8(p.weight, p.weight_type, c0 + i * kPiece, p.cols, w[0]);
      const float(&wi)[8] = w[ONE ? i : 0];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s[i][j] = s[i][j] * rstd;                  // hat
        dw[i][j] = fmaf(dy[i][j], s[i][j], dw[i][j]);
        dy[i][j] = dy[i][j] * wi[j];               // g
        along = fmaf(dy[i][j], s[i][j], along);
      }
    }
    // (two boxes in turn: a wave that is a row ahead does not write where another still reads)
    const float mean = row_sum<ONE>(along, part[turn]) / (float)p.cols;
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float ds[8];
      if (p.dsum) now.ds[i].widen(ds);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = rstd * (dy[i][j] - s[i][j] * mean);
        dy[i][j] = p.dsum ? d + ds[j] : d;
      }
      store8_of<TYPE>((T*)p.dx + row * p.ld_dx, c0 + i * kPiece, p.cols, dy[i]);
    }
    if (ONE) now = then;
  }
  if (!p.partial) return;
  if constexpr (ONE) {
    if (wave > 0) {
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) box[((wave - 1) * V + i) * kPiece + j * 64 + lane] = dw[i][j];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] += box[(k * V + i) * kPiece + j * 64 + lane];
  }
#pragma unroll
  for (int i = 0; i < V; ++i) store8_of<QGTC_F32>(p.partial + (int64_t)blockIdx.x * sum_pitch(p.cols), c0 + i * kPiece, p.cols, dw[i]);
}

// 32 columns of the groups' shares: a thread adds up four columns of every 32nd share, and the threads' sums are added in order.
__global__ __launch_bounds__(256) void norm_grad_sum_kernel(const float* partial, float* dweight, int cols, int groups) {
  __shared__ float box[32][33];
  const int q = (int)(threadIdx.x & 7u) * 4, k = (int)(threadIdx.x >> 3), c = (int)blockIdx.x * 32 + q;
  const int64_t pitch = sum_pitch(cols);
  f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
  if (c < pitch) {
#pragma unroll 8
    for (int g = k; g < groups; g += 32) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(partial + (int64_t)g * pitch + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] += v[i];
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) box[k][q + i] = s[i];
  __syncthreads();
  const int col = (int)blockIdx.x * 32 + (int)threadIdx.x;
  if (threadIdx.x < 32 && col < cols) {
    float sum = box[0][threadIdx.x];
#pragma unroll
    for (int i = 1; i < 32; ++i) sum += box[i][threadIdx.x];
    dweight[col] = sum;
  }
}

// Pieces per lane: the fewest that leave a row to at most 16 waves.
int pieces(int cols) { return cols <= 8192 ? 1 : cols <= 16384 ? 2 : 4; }

template <int TYPE, int V, bool ONE>
qgtc_status launch_norm(const NormParams& p, hipStream_t stream) {
  typedef typename Float<TYPE>::type T;
  const int waves = ONE ? 4 : cdiv(p.cols, V * kPiece);
  const int64_t most = kMostThreads / (ONE ? 64 : 64 * waves) / 4 * 4;
  for (int64_t r0 = 0; r0 < p.rows; r0 += most) {
    NormParams q = p;
    q.rows = (int32_t)(p.rows - r0 < most ? p.rows - r0 : most);
    q.x = (const T*)p.x + r0 * p.ld_x;
    if (p.residual) q.residual = (const T*)p.residual + r0 * p.ld_residual;
    if (p.sum) q.sum = (T*)p.sum + r0 * p.ld_sum;
    if (p.y) q.y = (T*)p.y + r0 * p.ld_y;
    if (p.rstd) q.rstd = p.rstd + r0;
    if (p.codes) q.codes = p.codes + r0 * p.ld_codes, q.scales = p.scales + r0 * p.ld_scales;
    hipLaunchKernelGGL((norm_kernel<TYPE, V, ONE>), dim3((unsigned)(ONE ? cdiv(q.rows, 4) : q.rows)), dim3(64u * (unsigned)waves), 0, stream, q);
    const qgtc_status st = launch_status();
    if (st != QGTC_OK) return st;
  }
  return QGTC_OK;
}
template <int TYPE>
qgtc_status launch_norm(const NormParams& p, hipStream_t stream) {
  if (p.cols <= kPiece) return launch_norm<TYPE, 1, true>(p, stream);
  const int v = pieces(p.cols);
  if (v == 1) return launch_norm<TYPE, 1, false>(p, stream);
  return v == 2 ? launch_norm<TYPE, 2, false>(p, stream) : launch_norm<TYPE, 4, false>(p, stream);
}

// Up to 1024 columns a wave has a row to itself and no barriers (8192 x 1024 bf16: two waves a row 33.8 us, so 17.2; at 2048
// columns one wave loses to four, 24.6 and 19.5).  Two workgroups per compute unit: one 69 us, four 57 at 8192 x 4096, two 49.
constexpr int kOneWave = 1024;
int grad_groups(int rows, int cols) {
  const int64_t most = cdiv(rows, cols <= kOneWave ? 4 : 1), groups = 2 * device_compute_units();
  return (int)(most < groups ? most : groups);
}
template <int TYPE, int V, bool ONE>
qgtc_status launch_grad(const GradParams& p, hipStream_t stream) {
  const int waves = ONE ? 4 : cdiv(p.cols, V * kPiece);
  hipLaunchKernelGGL((norm_grad_kernel<TYPE, V, ONE>), dim3((unsigned)p.groups), dim3(64u * (unsigned)waves),
                     ONE && p.partial ? 3 * V * kPiece * 4 : 0, stream, p);
  return launch_status();
}
template <int TYPE>
qgtc_status launch_grad(const GradParams& p, hipStream_t stream) {
  if (p.cols <= kPiece) return launch_grad<TYPE, 1, true>(p, stream);
  if (p.cols <= kOneWave) return launch_grad<TYPE, 2, true>(p, stream);
  const int v = pieces(p.cols);
  if (v == 1) return launch_grad<TYPE, 1, false>(p, stream);
  return v == 2 ? launch_grad<TYPE, 2, false>(p, stream) : launch_grad<TYPE, 4, false>(p, stream);
}

}  // namespace
}  // namespace qgtc

extern "C" qgtc_status qgtc_rms_norm(const qgtc_norm* n, void* stream) {
  using namespace qgtc;
  if (!n) return QGTC_ERR_NULL;
  if (n->rows < 0 || n->cols < 0 || n->rows > kMostEntries) return QGTC_ERR_SHAPE;
  if (!float_type(n->type) || !float_type(n->weight_type) || n->cols > kMostColumns) return QGTC_ERR_UNSUPPORTED;
  qgtc_status st;
  if (n->out) {
    if ((st = check_fp8(n->out)) != QGTC_OK) return st;
    if (n->out->rows != n->rows || n->out->cols != n->cols) return QGTC_ERR_SHAPE;
  }
  if (n->rows == 0 || n->cols == 0) return QGTC_OK;
  if ((st = check_matrix(n->x, n->type, n->rows, n->cols, n->ld_x)) != QGTC_OK) return st;
  if (n->residual && (st = check_matrix(n->residual, n->type, n->rows, n->cols, n->ld_residual)) != QGTC_OK) return st;
  if (n->sum && (st = check_matrix(n->sum, n->type, n->rows, n->cols, n->ld_sum)) != QGTC_OK) return st;
  if (n->y && (st = check_matrix(n->y, n->type, n->rows, n->cols, n->ld_y)) != QGTC_OK) return st;
  if ((n->y || n->out) && (st = check_matrix(n->weight, n->weight_type, 1, n->cols, n->cols)) != QGTC_OK) return st;
  if (((uintptr_t)n->rstd & 3u) != 0) return QGTC_ERR_ALIGN;
  if (n->sum && ((n->sum == n->x && n->ld_sum != n->ld_x) || (n->sum == n->residual && n->ld_sum != n->ld_residual))) return QGTC_ERR_SHAPE;
  if (!n->sum && !n->y && !n->out && !n->rstd) return QGTC_OK;
  NormParams p{};
  p.x = n->x;
  p.residual = n->residual;
  p.weight = n->weight;
  p.sum = n->sum;
  p.y = n->y;
  p.rstd = n->rstd;
  p.codes = n->out ? n->out->codes : nullptr;
  p.scales = n->out ? n->out->scales : nullptr;
  p.ld_x = n->ld_x;
  p.ld_residual = n->ld_residual;
  p.ld_sum = n->ld_sum;
  p.ld_y = n->ld_y;
  p.ld_codes = n->out ? n->out->ld : 0;
  p.ld_scales = n->out ? n->out->ld_scales : 0;
  p.weight_type = n->weight_type;
  p.rows = n->rows;
  p.cols = n->cols;
  p.eps = n->eps;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  ProfScope prof(QGTC_KERNEL_NORM, s);
  if (n->type == QGTC_F32) return launch_norm<QGTC_F32>(p, s);
  return n->type == QGTC_F16 ? launch_norm<QGTC_F16>(p, s) : launch_norm<QGTC_BF16>(p, s);
}

extern "C" size_t qgtc_rms_norm_backward_workspace_bytes(int32_t rows, int32_t cols) {
  if (rows <= 0 || cols <= 0 || cols > qgtc::kMostColumns) return 0;
  return (size_t)qgtc::grad_groups(rows, cols) * (size_t)qgtc::sum_pitch(cols) * 4;
}

extern "C" qgtc_status qgtc_rms_norm_backward(const qgtc_norm_grad* n, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace qgtc;
  if (!n) return QGTC_ERR_NULL;
  if (n->rows < 0 || n->cols < 0 || n->rows > kMostEntries) return QGTC_ERR_SHAPE;
  if (!float_type(n->type) || !float_type(n->weight_type) || n->cols > kMostColumns) return QGTC_ERR_UNSUPPORTED;
  if (n->cols == 0) return QGTC_OK;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  qgtc_status st;
  if (((uintptr_t)n->dweight & 3u) != 0) return QGTC_ERR_ALIGN;
  GradParams p{};
  p.dweight = n->dweight;
  p.rows = n->rows;
  p.cols = n->cols;
  if (n->rows > 0) {
    if ((st = check_matrix(n->dy, n->type, n->rows, n->cols, n->ld_dy)) != QGTC_OK) return st;
    if ((st = check_matrix(n->sum, n->type, n->rows, n->cols, n->ld_sum)) != QGTC_OK) return st;
    if (n->dsum && (st = check_matrix(n->dsum, n->type, n->rows, n->cols, n->ld_dsum)) != QGTC_OK) return st;
    if ((st = check_matrix(n->dx, n->type, n->rows, n->cols, n->ld_dx)) != QGTC_OK) return st;
    if ((st = check_matrix(n->weight, n->weight_type, 1, n->cols, n->cols)) != QGTC_OK) return st;
    if (!n->rstd) return QGTC_ERR_NULL;
    if (((uintptr_t)n->rstd & 3u) != 0) return QGTC_ERR_ALIGN;
    if ((n->dx == n->dy && n->ld_dx != n->ld_dy) || (n->dx == n->dsum && n->ld_dx != n->ld_dsum)) return QGTC_ERR_SHAPE;
    if (n->dx == n->sum) return QGTC_ERR_UNSUPPORTED;
    if (n->dweight) {
      if (!workspace) return QGTC_ERR_NULL;
      if (((uintptr_t)workspace & 15u) != 0) return QGTC_ERR_ALIGN;
      if (workspace_bytes < qgtc_rms_norm_backward_workspace_bytes(n->rows, n->cols)) return QGTC_ERR_WORKSPACE;
      p.partial = reinterpret_cast<float*>(workspace);
    }
    p.dy = n->dy;
    p.sum = n->sum;
    p.weight = n->weight;
    p.dsum = n->dsum;
    p.rstd = n->rstd;
    p.dx = n->dx;
    p.ld_dy = n->ld_dy;
    p.ld_sum = n->ld_sum;
    p.ld_dsum = n->ld_dsum;
    p.ld_dx = n->ld_dx;
    p.weight_type = n->weight_type;
    p.groups = grad_groups(n->rows, n->cols);
  }
  if (n->rows == 0 && !n->dweight) return QGTC_OK;
  ProfScope prof(QGTC_KERNEL_NORM, s);
  if (n->rows > 0) {
    st = n->type == QGTC_F32 ? launch_grad<QGTC_F32>(p, s) : n->type == QGTC_F16 ? launch_grad<QGTC_F16>(p, s) : launch_grad<QGTC_BF16>(p, s);
    if (st != QGTC_OK || !n->dweight) return st;
  }
  hipLaunchKernelGGL(norm_grad_sum_kernel, dim3((unsigned)cdiv(n->cols, 32)), dim3(256), 0, s, p.partial, n->dweight, n->cols, p.groups);
  return launch_status();
}
