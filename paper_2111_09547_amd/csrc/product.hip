// Products of matrices in 8-bit floats: checks, the choice of a kernel, and the kernel for few rows.
#include "product.h"

#include <initializer_list>

namespace qgtc {
namespace {

// Few rows: what counts is reading W.  A workgroup has 16 rows of it and 16 MT rows of X; its waves share K in pieces of four
// blocks, straight from memory to registers, and add up through LDS.
template <int MODE, int MT, bool WIDE>
__global__ __launch_bounds__(512) void few_kernel(const ProductParams p) {
  constexpr int D = MODE == kProduct ? 1 : 2;
  extern __shared__ v4f box[];                       // [wave][D][MT][lane]
  const int wave = (int)(threadIdx.x >> 6), waves = (int)(blockDim.x >> 6), lane = (int)(threadIdx.x & 63u);
  const int r = lane & 15, g = lane >> 4;
  const int n0 = (int)blockIdx.x * 16, m0 = (int)blockIdx.y * (16 * MT);
  const uint8_t *wc[D], *ws[D], *xc[MT], *xs[MT];
  auto aim = [&](int r) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const Fp8Operand& w = d ? p.u : p.w;
      const int64_t n = min(n0 + r, p.cols - 1);
      wc[d] = w.codes + n * w.ld + 16 * g;
      ws[d] = w.scales + n * w.ld_scales;
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int64_t m = min(m0 + 16 * t + r, p.rows - 1);
      xc[t] = p.x.codes + m * p.x.ld + 16 * g;
      xs[t] = p.x.scales + m * p.x.ld_scales;
    }
  };
  aim(r);
  v4f acc[D][MT];
#pragma unroll
  for (int d = 0; d < D; ++d)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[d][t] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
  for (int b0 = wave * 4; b0 < p.blocks; b0 += waves * 4) {
    uint32_t sw[D], sx[MT];
#pragma unroll
    for (int d = 0; d < D; ++d) sw[d] = *reinterpret_cast<const uint32_t*>(ws[d] + b0);
#pragma unroll
    for (int t = 0; t < MT; ++t) sx[t] = *reinterpret_cast<const uint32_t*>(xs[t] + b0);
    auto one = [&](auto which) {
      constexpr int B = decltype(which)::value;
      const int64_t at = (int64_t)(b0 + B) * kBlock;
      v8i w[D], x[MT];
#pragma unroll
      for (int d = 0; d < D; ++d) w[d] = lane_codes(wc[d] + at);
#pragma unroll
      for (int t = 0; t < MT; ++t) x[t] = lane_codes(xc[t] + at);
      if constexpr (WIDE) {
        WideCodes wide[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) wide[t] = widen<B, false>(x[t], sx[t]);
#pragma unroll
        for (int d = 0; d < D; ++d) {
          const WideCodes v = widen<B, false>(w[d], sw[d]);
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[d][t] = wide_mfma(v, wide[t], acc[d][t]);
        }
      } else {
#pragma unroll
        for (int d = 0; d < D; ++d)
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[d][t] = block_mfma<B>(w[d], x[t], acc[d][t], sw[d], sx[t]);
      }
    };
    if (b0 + 4 <= p.blocks) {
      one(std::integral_constant<int, 0>());
      one(std::integral_constant<int, 1>());
      one(std::integral_constant<int, 2>());
      one(std::integral_constant<int, 3>());
    } else {
      one(std::integral_constant<int, 0>());
      if (b0 + 1 < p.blocks) one(std::integral_constant<int, 1>());
      if (b0 + 2 < p.blocks) one(std::integral_constant<int, 2>());
    }
  }
  if constexpr (WIDE) {
    bool none = false;
#pragma unroll
    for (int d = 0; d < D; ++d)
#pragma unroll
      for (int t = 0; t < MT; ++t) none |= put_back(acc[d][t]);
    if (__ballot(none)) {                              // this wave's blocks again, one at a time
      int again = r;
      asm volatile("" : "+v"(again));                  // (addresses that are kept for this cost the loop above its registers)
      aim(again);
      v4f other[D][MT];
#pragma unroll
      for (int d = 0; d < D; ++d)
#pragma unroll
        for (int t = 0; t < MT; ++t) other[d][t] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
      for (int b = wave * 4; b < p.blocks; b += (b & 3) == 3 ? waves * 4 - 3 : 1) {
        const int64_t at = (int64_t)b * kBlock;
        WideCodes x[MT];
        uint32_t sx[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          sx[t] = xs[t][b];
          x[t] = widen<0, true>(lane_codes(xc[t] + at), sx[t]);
        }
#pragma unroll
        for (int d = 0; d < D; ++d) {
          const uint32_t sw = ws[d][b];
          const WideCodes w = widen<0, true>(lane_codes(wc[d] + at), sw);
          v4i rows;
#pragma unroll
          for (int i = 0; i < 4; ++i) rows[i] = __shfl((int)sw, 4 * g + i);
#pragma unroll
          for (int t = 0; t < MT; ++t) other[d][t] = apart_mfma(w, x[t], other[d][t], rows, 0, sx[t]);
        }
      }
#pragma unroll
      for (int d = 0; d < D; ++d)
#pragma unroll
        for (int t = 0; t < MT; ++t) take_apart(acc[d][t], other[d][t]);
    }
  }
#pragma unroll
  for (int d = 0; d < D; ++d)
#pragma unroll
    for (int t = 0; t < MT; ++t) box[((wave * D + d) * MT + t) * 64 + lane] = acc[d][t];
  __syncthreads();
  for (int t = wave; t < MT; t += waves) {
    v4f sum[D];
#pragma unroll
    for (int d = 0; d < D; ++d) {
      sum[d] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
      for (int i = 0; i < waves; ++i) {
        const v4f v = box[((i * D + d) * MT + t) * 64 + lane];
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[d][k] += v[k];
      }
    }
    const int m = m0 + 16 * t + r, n = n0 + 4 * g, left = p.cols - n;
    if (m >= p.rows || left <= 0) continue;
    float a[4], b[4];
    if constexpr (MODE == kProduct) {
#pragma unroll
      for (int k = 0; k < 4; ++k) a[k] = sum[0][k];
      store4_as(p.type, p.out, (int64_t)m * p.ld_out + n, left, a);
    } else if constexpr (MODE == kGated) {
#pragma unroll
      for (int k = 0; k < 4; ++k) a[k] = gate<true>(p.act, sum[0][k]).value * sum[D - 1][k];
      if (p.out) store4_as(p.type, p.out, (int64_t)m * p.ld_out + n, left, a);
      if (p.wide) store4_of<QGTC_F32>(p.wide, (int64_t)m * p.ld_wide + n, left, a);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float dh = k < left ? load_as(p.type, p.dh, (int64_t)m * p.ld_dh + n + k) : 0.0f;
        const Gate v = gate<true>(p.act, sum[0][k]);
        a[k] = dh * sum[D - 1][k] * v.slope;
        b[k] = dh * v.value;
      }
      store4_as(p.type, p.out, (int64_t)m * p.ld_out + n, left, a);
      store4_as(p.type, p.out2, (int64_t)m * p.ld_out2 + n, left, b);
    }
  }
}

template <int MODE, int MT, bool WIDE>
qgtc_status launch_few(const ProductParams& p, hipStream_t stream) {
  constexpr int D = MODE == kProduct ? 1 : 2;
  const int waves = 8;
  const size_t lds = (size_t)waves * D * MT * 64 * 16;
  // (what is beyond a launch's size goes in launches of its own: 65535 workgroups along the second axis)
  const int most = 65535 * 16 * MT, most_cols = (int)(kMostThreads / (64 * waves) * 16);
  const int64_t b = float_bytes(p.type);
  for (int64_t m0 = 0; m0 < p.rows; m0 += most)
    for (int64_t n0 = 0; n0 < p.cols; n0 += most_cols) {
      ProductParams q = p;
      q.rows = (int32_t)(p.rows - m0 < most ? p.rows - m0 : most);
      q.cols = (int32_t)(p.cols - n0 < most_cols ? p.cols - n0 : most_cols);
      q.x.codes += m0 * p.x.ld;
      q.x.scales += m0 * p.x.ld_scales;
      q.w.codes += n0 * p.w.ld;
      q.w.scales += n0 * p.w.ld_scales;
      if (D == 2) q.u.codes += n0 * p.u.ld, q.u.scales += n0 * p.u.ld_scales;
      if (q.out) q.out = (char*)p.out + (m0 * p.ld_out + n0) * b;
      if (q.out2) q.out2 = (char*)p.out2 + (m0 * p.ld_out2 + n0) * b;
      if (q.dh) q.dh = (const char*)p.dh + (m0 * p.ld_dh + n0) * b;
      if (q.wide) q.wide += m0 * p.ld_wide + n0;
      hipLaunchKernelGGL((few_kernel<MODE, MT, WIDE>), dim3((unsigned)cdiv(q.cols, 16), (unsigned)cdiv(q.rows, 16 * MT)), dim3(64u * waves), lds, stream, q);
      const qgtc_status st = launch_status();
      if (st != QGTC_OK) return st;
    }
  return QGTC_OK;
}

template <int MODE, bool WIDE>
qgtc_status launch_few(const ProductParams& p, hipStream_t stream) {
  if (p.rows <= 16) return launch_few<MODE, 1, WIDE>(p, stream);
  if (p.rows <= 32) return launch_few<MODE, 2, WIDE>(p, stream);
  return launch_few<MODE, 4, WIDE>(p, stream);
}

// h from memory into 8-bit floats: 16 lanes have a block, a wave 512 columns of a row.
__global__ __launch_bounds__(256) void gated_rows_kernel(const ProductParams p, uint32_t groups, int64_t first) {
  const int64_t unit = first + blockIdx.x * 4u + (threadIdx.x >> 6);
  const int m = (int)(unit / groups), c = (int)(unit - (int64_t)m * groups) * 512 + (int)(threadIdx.x & 63u) * 8;
  if (m >= p.rows) return;
  float v[8];
  load8_of<QGTC_F32>(p.wide + (int64_t)m * p.ld_wide, c, p.cols, v);
  uint32_t top = max_of_16_lanes(abs_max(v));
  const bool near = near_border(top);
  if (__ballot(near)) {
    uint32_t want = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) want |= near && abs_bits(v[i]) >= border_from(top) ? 1u << i : 0u;
    const uint32_t block = max_of_16_lanes(exact_top(p, m, c, want));
    if (near) top = border_side(top, block);
  }
  write_block8(p.codes + (int64_t)m * p.ld_codes, p.scales + (int64_t)m * p.ld_scales, c, p.cols, v, scale_byte(top));
}

// Which kernel: the one that takes least by what each was measured to take, in us (bf16 results, M x N x K; few, mid, tiles):
//   product  32 x 4096 x 4096   9.1  17.8  43.5     gated  32 x 4096 x 4096  14.7  21.3  49.3
//           128 x 4096 x 4096  23.5  18.0  46.0           128 x 4096 x 4096  33.0  23.0  52.0
//           128 x 1024 x 1024   5.3   7.3  17.3          1024 x 1024 x 1024  24.2  13.9  23.4
//          1024 x 4096 x 4096   161  21.9  47.8          1024 x 4096 x 4096   216  47.5  54.6
//          4096 x 4096 x 4096         84.1  60.8          512 x 8192 x 2048   118  32.1  35.3
//          8192 x 2048 x 8192          160   109         4096 x 4096 x 4096   846   174   116
// few: its workgroups' reads, 16 rows of W and of X each, at 8 TB/s.  mid and tiles: rounds of tiles, a block of K at a time (a block
// takes longer where all compute units are busy and the clock falls), and what they start and end with.  Gated blocks that are not
// made by tiles pass their results through memory and another launch.
enum Path { kFew, kMid, kTiles };
Path path_of(int mode, int rows, int cols, int blocks, bool wide) {
  if (blocks == 0) return kFew;
  const bool two = mode != kProduct;
  const int cus = device_compute_units(), per_few = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  const double again = mode == kGated && !wide ? 3.5 + (double)rows * cols * 8 / 6e6 : 0.0;
  const double few = 2.5 + (double)cdiv(cols, 16) * cdiv(rows, per_few) * ((two ? 32 : 16) + per_few) * blocks * kBlock / 8.2e6 + again;
  const int64_t mids = (int64_t)cdiv(rows, 128) * cdiv(cols, two ? 64 : 128);
  const double mid = 4.0 + (double)cdiv(mids, cus) * blocks * (wide ? 1.05 : mids <= cus / 2 ? 0.45 : 0.6) + again;
  const Path less = few <= mid ? kFew : kMid;
  if (wide) return less;
  const int64_t tiles = (int64_t)cdiv(rows, 256) * cdiv(cols, two ? 128 : 256);
  const double tile = (two ? 14.0 : 8.0) + (double)cdiv(tiles, cus) * blocks * (tiles <= cus / 2 ? 1.2 : 1.6);
  return tile < (less == kFew ? few : mid) ? kTiles : less;
}

template <int MODE>
qgtc_status launch(const ProductParams& p, hipStream_t stream) {
  const bool wide = p.out && p.type == QGTC_F32;   // results in fp32 have sums that are worth it
  switch (path_of(MODE, p.rows, p.cols, p.blocks, wide)) {
    case kTiles: return launch_tiles<MODE>(p, stream);
    case kMid: return launch_mid<MODE>(p, wide, stream);
    default: return wide ? launch_few<MODE, true>(p, stream) : launch_few<MODE, false>(p, stream);
  }
}

constexpr int64_t kMostLd = 1 << 24;
Fp8Operand operand(const qgtc_fp8* m) { return {m->codes, m->scales, m->ld, m->ld_scales, m->rows}; }

// X, and the operands that it is multiplied with, of the same sizes.
qgtc_status check_operands(const qgtc_fp8* X, const qgtc_fp8* W, const qgtc_fp8* U) {
  qgtc_status st = check_fp8(X);
  if (st == QGTC_OK) st = check_fp8(W);
  if (st == QGTC_OK && U) st = check_fp8(U);
  if (st != QGTC_OK) return st;
  // (a tile's rows are addressed with 32 bits)
  for (const qgtc_fp8* m : {X, W, U})
    if (m && (m->ld > kMostLd || m->ld_scales > kMostLd || (int64_t)fp8_blocks(m->cols) * kBlock >= kMostLd)) return QGTC_ERR_UNSUPPORTED;
  if (X->cols != W->cols || (U && (U->cols != W->cols || U->rows != W->rows))) return QGTC_ERR_SHAPE;
  return QGTC_OK;
}

}  // namespace
}  // namespace qgtc

extern "C" qgtc_status qgtc_fp8_product(const qgtc_fp8* X, const qgtc_fp8* W, int32_t type, void* out, int64_t ld_out, void* stream) {
  using namespace qgtc;
  qgtc_status st = check_operands(X, W, nullptr);
  if (st != QGTC_OK) return st;
  if (!float_type(type)) return QGTC_ERR_UNSUPPORTED;
  if (X->rows == 0 || W->rows == 0) return QGTC_OK;
  if ((st = check_matrix(out, type, X->rows, W->rows, ld_out)) != QGTC_OK) return st;
  ProductParams p{};
  p.x = operand(X);
  p.w = operand(W);
  p.blocks = fp8_blocks(X->cols);
  p.rows = X->rows;
  p.cols = W->rows;
  p.type = type;
  p.out = out;
  p.ld_out = ld_out;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  ProfScope prof(QGTC_KERNEL_UPDATE, s);
  return launch<kProduct>(p, s);
}

extern "C" size_t qgtc_fp8_gated_workspace_bytes(int32_t rows, int32_t cols, int32_t inner) {
  if (rows <= 0 || cols <= 0 || inner < 0) return 0;
  return qgtc::path_of(qgtc::kGated, rows, cols, qgtc::fp8_blocks(inner), false) == qgtc::kTiles ? 0 : (size_t)rows * (size_t)cols * 4;
}

extern "C" qgtc_status qgtc_fp8_gated(const qgtc_fp8* X, const qgtc_fp8* G, const qgtc_fp8* U, int32_t act,
                                      const qgtc_fp8* out, int32_t type, void* h, int64_t ld_h,
                                      void* workspace, size_t workspace_bytes, void* stream) {
  using namespace qgtc;
  if (!U) return QGTC_ERR_NULL;
  qgtc_status st = check_operands(X, G, U);
  if (st != QGTC_OK) return st;
  if (act != QGTC_ACT_SILU && act != QGTC_ACT_GELU) return QGTC_ERR_UNSUPPORTED;
  if (out) {
    if ((st = check_fp8(out)) != QGTC_OK) return st;
    if (out->rows != X->rows || out->cols != G->rows) return QGTC_ERR_SHAPE;
  }
  if (X->rows == 0 || G->rows == 0) return QGTC_OK;
  if (!out && !h) return QGTC_ERR_NULL;
  if (h && (st = check_matrix(h, type, X->rows, G->rows, ld_h)) != QGTC_OK) return st;
  ProductParams p{};
  p.x = operand(X);
  p.w = operand(G);
  p.u = operand(U);
  p.blocks = fp8_blocks(X->cols);
  p.rows = X->rows;
  p.cols = G->rows;
  p.type = h ? type : QGTC_F32;
  p.act = act;
  p.out = h;
  p.ld_out = ld_h;
  const bool from_h = out && h && type == QGTC_F32;       // h is what is quantized
  if (out && !from_h) {
    const size_t need = qgtc_fp8_gated_workspace_bytes(X->rows, G->rows, X->cols);
    if (need) {
      if (!workspace) return QGTC_ERR_NULL;
      if (((uintptr_t)workspace & 15u) != 0) return QGTC_ERR_ALIGN;
      if (workspace_bytes < need) return QGTC_ERR_WORKSPACE;
      p.wide = reinterpret_cast<float*>(workspace);
      p.ld_wide = p.cols;
    }
    p.codes = out->codes;
    p.scales = out->scales;
    p.ld_codes = out->ld;
    p.ld_scales = out->ld_scales;
  }
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  ProfScope prof(QGTC_KERNEL_LAYER, s);
  st = launch<kGated>(p, s);
  if (st != QGTC_OK || !out) return st;
  if (from_h) return quantize_rows(h, QGTC_F32, p.rows, p.cols, ld_h, *out, s);
  if (!p.wide) return QGTC_OK;
  const uint32_t groups = (uint32_t)cdiv(p.cols, 512);
  const int64_t units = (int64_t)groups * p.rows;
  for (int64_t first = 0; first < units && st == QGTC_OK; first += kMostThreads / 64) {
    const int64_t here = units - first < kMostThreads / 64 ? units - first : kMostThreads / 64;
    hipLaunchKernelGGL(gated_rows_kernel, dim3((unsigned)((here + 3) / 4)), dim3(256), 0, s, p, groups, first);
    st = launch_status();
  }
  return st;
}

extern "C" qgtc_status qgtc_fp8_gated_backward(const qgtc_fp8* X, const qgtc_fp8* G, const qgtc_fp8* U, int32_t act,
                                               int32_t type, const void* dh, int64_t ld_dh, void* dg, int64_t ld_dg,
                                               void* du, int64_t ld_du, void* stream) {
  using namespace qgtc;
  if (!U) return QGTC_ERR_NULL;
  qgtc_status st = check_operands(X, G, U);
  if (st != QGTC_OK) return st;
  if (act != QGTC_ACT_SILU && act != QGTC_ACT_GELU) return QGTC_ERR_UNSUPPORTED;
  if (!float_type(type)) return QGTC_ERR_UNSUPPORTED;
  if (X->rows == 0 || G->rows == 0) return QGTC_OK;
  if ((st = check_matrix(dh, type, X->rows, G->rows, ld_dh)) != QGTC_OK) return st;
  if ((st = check_matrix(dg, type, X->rows, G->rows, ld_dg)) != QGTC_OK) return st;
  if ((st = check_matrix(du, type, X->rows, G->rows, ld_du)) != QGTC_OK) return st;
  ProductParams p{};
  p.x = operand(X);
  p.w = operand(G);
  p.u = operand(U);
  p.blocks = fp8_blocks(X->cols);
  p.rows = X->rows;
  p.cols = G->rows;
  p.type = type;
  p.act = act;
  p.out = dg;
  p.ld_out = ld_dg;
  p.out2 = du;
  p.ld_out2 = ld_du;
  p.dh = dh;
  p.ld_dh = ld_dh;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  ProfScope prof(QGTC_KERNEL_LAYER, s);
  return launch<kGatedGrad>(p, s);
}
