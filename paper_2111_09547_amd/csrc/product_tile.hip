// Products of matrices in 8-bit floats, many rows: tiles of 256 x 256 on the matrix cores.
//
// A workgroup of four waves, one per SIMD, has a tile of 256 rows of X by 256 rows of W, a wave 128 x 128 of it: 64
// v_mfma_scale_f32_16x16x128_f8f6f4 (2048 cycles) per block of K, whose sums fill half of the wave's 512 registers.  Operands of a
// block, 64 KiB, go to LDS without passing through registers, two buffers in turn; a wave reads 32 KiB of them back, which takes
// the LDS 1024 cycles for all four.  64 x 64 per wave would read twice that per product and be bound by the LDS.
//
// A step (a block of K) is four quarters of 16 instructions, of 64 x 64 products each: (w0, x0), (w1, x0), (w0, x1), (w1, x1).
// Beside each, one of the four halves of operands goes to registers: w1, x1, and then, behind the step's only barrier, the next
// step's x0 and w0, whose registers the quarters in front have left.  The buffer that is free from there on is loaded for the
// step after the next, which has a whole step's time to come.
//
// A row of a buffer is 128 bytes; its 16-byte piece c lies at c ^ (row % 8), so that 16 lanes reading a piece each of 16 rows meet
// every bank once.  W's rows are put into the buffer in another order: register i of lane group g of the t-th 16 of 64 belongs
// to row 16 g + 4 i + t of them, so that a lane ends up with 16 results that lie side by side.
#include "product.h"

namespace qgtc {
namespace {

constexpr int kTile = 256;
constexpr int kOperand = kTile * kBlock;           // bytes of an operand's block
constexpr int kBuffer = 2 * kOperand;              // X, then W
constexpr int kScales = 2 * kBuffer;               // words of four blocks' scales: [2][X, W][256]
constexpr int kTileLds = kScales + 2 * 2 * kTile * 4;

struct TileParams {
  ProductParams p;
  uint32_t tiles_m, tiles_n, per_group;            // per_group: tiles_m x tiles along n that are dealt together
  uint32_t per_xcd;
};

// Wave-wide loads straight to LDS address `to` (+ 16 or 4 bytes per lane); assembly because the compiler would make every later
// read of LDS wait for them.
__device__ __forceinline__ void load16_lds(const v4i& rsrc, uint32_t voff, uint32_t soff, uint32_t to) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" :: "v"(voff), "s"(rsrc), "s"(soff), "s"(to) : "m0");
}
__device__ __forceinline__ void load4_lds(const v4i& rsrc, uint32_t voff, uint32_t soff, uint32_t to) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dword %0, %1, %2 offen lds" :: "v"(voff), "s"(rsrc), "s"(soff), "s"(to) : "m0");
}
__device__ __forceinline__ uint32_t scalar(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ v4i buffer_of(const void* base, uint32_t bytes) {
  const uint64_t b = (uint64_t)base;
  return (v4i){(int)scalar((uint32_t)b), (int)scalar((uint32_t)(b >> 32)), (int)scalar(bytes), 0x00020000};
}

// Everything this wave has asked of memory and LDS has come; then every wave's.
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <int MODE>
__global__ __launch_bounds__(256, 1) void tile_kernel(const TileParams tp) {
  const ProductParams& p = tp.p;
  extern __shared__ __align__(128) uint8_t lds[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
  const int wave = (int)scalar(threadIdx.x >> 6), lane = (int)(threadIdx.x & 63u), r = lane & 15, g = lane >> 4;
  const int wm = wave & 1, wn = wave >> 1;

  // ---- which tile: an XCD's tiles are neighbours, in groups that are 8 tiles of rows high ----
  const uint32_t id = (blockIdx.x & 7u) * tp.per_xcd + (blockIdx.x >> 3);
  if (id >= tp.tiles_m * tp.tiles_n) return;
  const uint32_t group = id / tp.per_group, first_m = group * 8u, high = min(8u, tp.tiles_m - first_m);
  const uint32_t in = id - group * tp.per_group;
  const int m0 = (int)(first_m + in % high) * kTile, bn = (int)(in / high);
  constexpr int TN = MODE == kProduct ? kTile : kTile / 2;           // columns of the result
  const int n0 = bn * TN;
  const int rows_here = min(kTile, p.rows - m0), cols_here = min(TN, p.cols - n0);

  // ---- where this wave's loads come from: 64 rows of each operand, 8 rows a load ----
  const v4i rx = buffer_of(p.x.codes + (int64_t)m0 * p.x.ld, (uint32_t)((rows_here - 1) * p.x.ld) + (uint32_t)p.blocks * kBlock);
  const v4i rsx = buffer_of(p.x.scales + (int64_t)m0 * p.x.ld_scales, (uint32_t)((rows_here - 1) * p.x.ld_scales) + (uint32_t)((p.blocks + 3) & ~3));
  // (two projections: a wave's 128 rows are 64 of each)
  const Fp8Operand& ow = MODE != kProduct && (wave & 1) ? p.u : p.w;
  const v4i rw = buffer_of(ow.codes + (int64_t)n0 * ow.ld, (uint32_t)((cols_here - 1) * ow.ld) + (uint32_t)p.blocks * kBlock);
  const v4i rsw = buffer_of(ow.scales + (int64_t)n0 * ow.ld_scales, (uint32_t)((cols_here - 1) * ow.ld_scales) + (uint32_t)((p.blocks + 3) & ~3));
  const int w_first = MODE == kProduct ? 64 * wave : 64 * (wave >> 1);   // of the tile's rows of that operand
  const uint32_t piece = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16u;
  uint32_t xoff[8], woff[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    xoff[j] = (uint32_t)min(64 * wave + 8 * j + (lane >> 3), rows_here - 1) * (uint32_t)p.x.ld + piece;
    woff[j] = (uint32_t)min(w_first + 4 * (8 * (j & 1) + (lane >> 3)) + (j >> 1), cols_here - 1) * (uint32_t)ow.ld + piece;
  }
  const uint32_t sxoff = (uint32_t)min(64 * wave + lane, rows_here - 1) * (uint32_t)p.x.ld_scales;
  const uint32_t swoff = (uint32_t)min(w_first + 4 * r + g, cols_here - 1) * (uint32_t)ow.ld_scales;
  const uint32_t to_x = lds0 + (uint32_t)wave * (64 * kBlock), to_w = to_x + kOperand;
  auto load_pair = [&](uint32_t buffer, uint32_t from, int j) {   // an eighth of a wave's loads for a step
    load16_lds(rx, xoff[j], from, to_x + buffer + (uint32_t)j * 1024u);
    load16_lds(rw, woff[j], from, to_w + buffer + (uint32_t)j * 1024u);
  };
  auto load_scales = [&](int four) {
    const uint32_t at = lds0 + kScales + (uint32_t)(four & 1) * (2 * kTile * 4) + (uint32_t)wave * 256u;
    load4_lds(rsx, sxoff, (uint32_t)four * 4u, at);
    load4_lds(rsw, swoff, (uint32_t)four * 4u, at + kTile * 4);
  };

  // ---- operands from LDS ----
  const uint32_t lane_at = (uint32_t)r * kBlock + (uint32_t)((g ^ (r & 7)) * 16);
  auto read4 = [&](uint32_t buffer, int operand, int half, int t) -> v8i {
    const uint8_t* const at = lds + ((operand ? wn : wm) * (128 * kBlock) + operand * kOperand + (half * 64 + t * 16) * kBlock);
    const v4i a = *reinterpret_cast<const v4i*>(at + (buffer + lane_at)), b = *reinterpret_cast<const v4i*>(at + (buffer + (lane_at ^ 64u)));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto read_scale = [&](int k, int operand, int half, int t) -> uint32_t {
    return lds[kScales + (k & 4) * (kTile * 2) + (k & 3) + operand * (kTile * 4) + ((operand ? wn : wm) * 128 + half * 64 + t * 16) * 4 + r * 4];
  };

  v4f acc[2][2][4][4];                                 // [half of w][half of x][w][x]
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int d = 0; d < 4; ++d) acc[a][b][c][d] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
  v8i x[2][4], w[2][4];
  uint32_t sx[2][4], sw[2][4];

  // A quarter: 16 products, and beside them four operands (two reads each) and at most eight pairs of loads.
  auto quarter = [&](int hw, int hx, auto&& fetch, auto&& load) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      fetch(t);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        acc[hw][hx][t][u] = block_mfma<0>(w[hw][t], x[hx][u], acc[hw][hx][t][u], sw[hw][t], sx[hx][u]);
        if (u & 1) load(2 * t + (u >> 1));
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  load_scales(0);
#pragma unroll
  for (int j = 0; j < 8; ++j) load_pair(0, 0, j);
  const uint32_t last = (uint32_t)(p.blocks - 1) * kBlock;
#pragma unroll
  for (int j = 0; j < 8; ++j) load_pair(kBuffer, min((uint32_t)kBlock, last), j);
  meet();
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    x[0][t] = read4(0, 0, 0, t);
    w[0][t] = read4(0, 1, 0, t);
    sx[0][t] = read_scale(0, 0, 0, t);
    sw[0][t] = read_scale(0, 1, 0, t);
  }
  auto none = [](int) {};
#pragma unroll 1
  for (int k = 0; k < p.blocks; ++k) {
    const uint32_t cur = (uint32_t)(k & 1) * kBuffer, next = cur ^ kBuffer;
    quarter(0, 0, [&](int t) { w[1][t] = read4(cur, 1, 1, t); sw[1][t] = read_scale(k, 1, 1, t); }, none);
    quarter(1, 0, [&](int t) { x[1][t] = read4(cur, 0, 1, t); sx[1][t] = read_scale(k, 0, 1, t); }, none);
    meet();
    __builtin_amdgcn_sched_barrier(0);
    if ((k & 3) == 0 && k + 4 < p.blocks) load_scales((k >> 2) + 1);
    // (behind the last block: loads and reads of it that nobody uses)
    const uint32_t from = min((uint32_t)(k + 2) * kBlock, last);
    quarter(0, 1, [&](int t) { x[0][t] = read4(next, 0, 0, t); sx[0][t] = read_scale(k + 1, 0, 0, t); }, [&](int j) { load_pair(cur, from, j); });
    quarter(1, 1, [&](int t) { w[0][t] = read4(next, 1, 0, t); sw[0][t] = read_scale(k + 1, 1, 0, t); }, none);
  }
  meet();                                              // (nothing is on its way to LDS any more)

  // ---- what is made of the sums: lane (r, g) has row 16 t + r of each half of x and 16 columns from 16 g on of each half of w ----
  auto row_of = [&](int hx, int u) { return m0 + wm * 128 + hx * 64 + u * 16 + r; };
  if constexpr (MODE == kProduct) {
#pragma unroll
    for (int hx = 0; hx < 2; ++hx)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int m = row_of(hx, u);
        if (m >= p.rows) continue;
#pragma unroll
        for (int hw = 0; hw < 2; ++hw) {
          const int n = n0 + wn * 128 + hw * 64 + 16 * g, left = p.cols - n;
          float v[2][8];
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i >> 3][i & 7] = acc[hw][hx][i & 3][u][i >> 2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (p.type == QGTC_F16) store8_of<QGTC_F16>((uint16_t*)p.out + (int64_t)m * p.ld_out + n, 8 * k, left, v[k]);
            else store8_of<QGTC_BF16>((uint16_t*)p.out + (int64_t)m * p.ld_out + n, 8 * k, left, v[k]);
          }
        }
      }
  } else if constexpr (MODE == kGated) {
    const int n = n0 + wn * 64 + 16 * g, left = p.cols - n;
    uint32_t* const tops = reinterpret_cast<uint32_t*>(lds);          // [wn][256 rows]
#pragma unroll
    for (int hx = 0; hx < 2; ++hx)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint32_t top = 0u;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float h = gate<false>(p.act, acc[0][hx][i & 3][u][i >> 2]).value * acc[1][hx][i & 3][u][i >> 2];
          h = i < left ? h : 0.0f;
          acc[0][hx][i & 3][u][i >> 2] = h;
          top = max(top, abs_bits(h));
        }
        if (p.out) {
          const int m = row_of(hx, u);
          float v[2][8];
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i >> 3][i & 7] = acc[0][hx][i & 3][u][i >> 2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (m >= p.rows) continue;
            if (p.type == QGTC_F16) store8_of<QGTC_F16>((uint16_t*)p.out + (int64_t)m * p.ld_out + n, 8 * k, left, v[k]);
            else store8_of<QGTC_BF16>((uint16_t*)p.out + (int64_t)m * p.ld_out + n, 8 * k, left, v[k]);
          }
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        if (g == 0) tops[wn * kTile + wm * 128 + hx * 64 + u * 16 + r] = top;
      }
    if (!p.codes) return;
    meet();
#pragma unroll
    for (int hx = 0; hx < 2; ++hx)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int m = row_of(hx, u), lr = wm * 128 + hx * 64 + u * 16 + r;
        if (m >= p.rows) continue;
        const uint32_t e = scale_byte(max(tops[lr], tops[kTile + lr]));
        u32x4 c;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          c[k] = encode4(acc[0][hx][0][u][k], acc[0][hx][1][u][k], acc[0][hx][2][u][k], acc[0][hx][3][u][k], e);
          if (e == 255u && left < 4 * k + 4) c[k] &= left <= 4 * k ? 0u : 0xffffffffu >> (8 * (4 * k + 4 - left));   // (zeros past the end)
        }
        *reinterpret_cast<u32x4*>(p.codes + (int64_t)m * p.ld_codes + n) = c;
        if (g == 0 && wn == 0) p.scales[(int64_t)m * p.ld_scales + bn] = (uint8_t)e;
      }
  } else {
    const int n = n0 + wn * 64 + 16 * g, left = p.cols - n;
#pragma unroll
    for (int hx = 0; hx < 2; ++hx)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int m = row_of(hx, u);
        if (m >= p.rows || left <= 0) continue;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float dh[8], dg[8], du[8];
          if (p.type == QGTC_F16) load8_of<QGTC_F16>((const uint16_t*)p.dh + (int64_t)m * p.ld_dh + n, 8 * k, left, dh);
          else load8_of<QGTC_BF16>((const uint16_t*)p.dh + (int64_t)m * p.ld_dh + n, 8 * k, left, dh);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int i = 8 * k + j;
            const Gate v = gate<false>(p.act, acc[0][hx][i & 3][u][i >> 2]);
            dg[j] = dh[j] * acc[1][hx][i & 3][u][i >> 2] * v.slope;
            du[j] = dh[j] * v.value;
          }
          if (p.type == QGTC_F16) {
            store8_of<QGTC_F16>((uint16_t*)p.out + (int64_t)m * p.ld_out + n, 8 * k, left, dg);
            store8_of<QGTC_F16>((uint16_t*)p.out2 + (int64_t)m * p.ld_out2 + n, 8 * k, left, du);
          } else {
            store8_of<QGTC_BF16>((uint16_t*)p.out + (int64_t)m * p.ld_out + n, 8 * k, left, dg);
            store8_of<QGTC_BF16>((uint16_t*)p.out2 + (int64_t)m * p.ld_out2 + n, 8 * k, left, du);
          }
        }
      }
  }
}

}  // namespace

template <int MODE>
qgtc_status launch_tiles(const ProductParams& p, hipStream_t stream) {
  TileParams t{};
  t.p = p;
  t.tiles_m = (uint32_t)cdiv(p.rows, kTile);
  t.tiles_n = (uint32_t)cdiv(p.cols, MODE == kProduct ? kTile : kTile / 2);
  t.per_group = 8u * t.tiles_n;
  t.per_xcd = (uint32_t)cdiv((int64_t)t.tiles_m * t.tiles_n, 8);
  static OncePerDevice once;
  if (!allow_lds(once, reinterpret_cast<const void*>(&tile_kernel<MODE>), kTileLds)) return QGTC_ERR_HIP;
  hipLaunchKernelGGL(tile_kernel<MODE>, dim3(8u * t.per_xcd), dim3(256), kTileLds, stream, t);
  return launch_status();
}
template qgtc_status launch_tiles<kProduct>(const ProductParams& p, hipStream_t stream);
template qgtc_status launch_tiles<kGated>(const ProductParams& p, hipStream_t stream);
template qgtc_status launch_tiles<kGatedGrad>(const ProductParams& p, hipStream_t stream);

}  // namespace qgtc
