// Products of matrices in 8-bit floats, tiles of 128 x 128: for results that are too few for tiles of 256 x 256 to give every
// compute unit work, and for all larger ones in fp32.
//
// A workgroup of four waves has a tile, a wave 64 x 64 of it.  A block of K is 32 KiB of operands, in one of four buffers of LDS that
// loads fill without passing through registers, three blocks ahead; a wave reads the next block's 16 KiB into registers beside its
// 16 products of this one, so that a barrier per block is all it waits for.  The LDS bounds it: 96 KiB written and read per block,
// 768 cycles, beside 512 of products.  Columns' order in the buffer as in product_tile.hip: a lane has eight results side by side.
// Two projections: of a wave's 64 rows of W, 32 are one's and 32 the other's, so that a lane has the same columns of both.
#include "product_lds.h"

namespace qgtc {
namespace {

constexpr int kSide = 128;
constexpr int kOperand = kSide * kBlock, kBuffer = 2 * kOperand;
constexpr int kScales = 4 * kBuffer, kSlot = 2 * kSide * 4;      // words of four blocks' scales: [2 slots][X, W][128]
constexpr int kFlags = kScales + 2 * kSlot, kMidLds = kFlags + 16;    // a word for each wave

struct MidParams {
  ProductParams p;
  uint32_t tiles_m, tiles_n, per_group, per_xcd;
};

template <int MODE, bool WIDE>
__global__ __launch_bounds__(256, 1) void mid_kernel(const MidParams mp) {
  const ProductParams& p = mp.p;
  extern __shared__ __align__(128) uint8_t lds[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
  const int wave = (int)scalar(threadIdx.x >> 6), lane = (int)(threadIdx.x & 63u), r = lane & 15, g = lane >> 4, q = lane >> 3;
  const int wm = wave & 1, wn = wave >> 1;
  constexpr bool both = MODE != kProduct;
  constexpr int TN = both ? kSide / 2 : kSide;       // columns of the result

  const uint32_t id = (blockIdx.x & 7u) * mp.per_xcd + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= mp.per_xcd || id >= mp.tiles_m * mp.tiles_n) return;
  const uint32_t group = id / mp.per_group, first_m = group * 8u, high = min(8u, mp.tiles_m - first_m), in = id - group * mp.per_group;
  const int m0 = (int)scalar((first_m + in % high) * kSide), n0 = (int)scalar(in / high * TN);

  // ---- loads: of each block this wave's are 32 rows of each operand, 8 rows a load ----
  const uint32_t piece = (uint32_t)((lane & 7) ^ q) * 16u;
  const uint32_t row_bytes = (uint32_t)p.blocks * kBlock, row_words = (uint32_t)((p.blocks + 3) & ~3);
  const uint32_t most_x = (uint32_t)min(kSide, p.rows - m0) - 1u, most_w = (uint32_t)min(TN, p.cols - n0) - 1u;
  const int part = wave & 1;                         // two projections: even waves load one's rows, odd waves the other's
  const uint8_t* const w_codes = both && part ? p.u.codes : p.w.codes;
  const int64_t w_ld = both && part ? p.u.ld : p.w.ld;
  const v4i rx = buffer_of(p.x.codes + (int64_t)m0 * p.x.ld, most_x * (uint32_t)p.x.ld + row_bytes);
  const v4i rw = buffer_of(w_codes + (int64_t)n0 * w_ld, most_w * (uint32_t)w_ld + row_bytes);
  const v4i rsx = buffer_of(p.x.scales + (int64_t)m0 * p.x.ld_scales, most_x * (uint32_t)p.x.ld_scales + row_words);
  const v4i rsw = buffer_of(p.w.scales + (int64_t)n0 * p.w.ld_scales, most_w * (uint32_t)p.w.ld_scales + row_words);
  const v4i rsu = both ? buffer_of(p.u.scales + (int64_t)n0 * p.u.ld_scales, most_w * (uint32_t)p.u.ld_scales + row_words) : rsw;
  const uint32_t ldx = (uint32_t)p.x.ld, ldw = (uint32_t)w_ld;
  const uint32_t xoff = (uint32_t)(32 * wave + q) * ldx + piece;
  const uint32_t woff = (uint32_t)((both ? 32 * wn : 64 * wn + 32 * part) + 8 * (q >> 2) + (q & 3)) * ldw + piece;
  // words of scales: waves 0 and 1 load X's, 64 rows each, 2 and 3 W's; of two projections lanes 32.. are the second's
  const uint32_t sxoff = (uint32_t)(64 * part + lane) * (uint32_t)p.x.ld_scales;
  const uint32_t s_row = (uint32_t)(8 * (r >> 2) + 4 * (g & 1) + (r & 3) + (both ? 32 * part : 64 * part + 32 * (g >> 1)));
  const uint32_t swoff = s_row * (uint32_t)(both && g >= 2 ? p.u.ld_scales : p.w.ld_scales);
  const uint32_t last = (uint32_t)(p.blocks - 1) * kBlock;
  auto load = [&](int k, int j) {                    // a quarter of them.  (Behind the last block: that one again, for nobody.)
    const uint32_t from = scalar(min((uint32_t)k * kBlock, last)), to = lds0 + (uint32_t)(k & 3) * kBuffer + (uint32_t)(32 * wave) * kBlock;
    load16_lds(rx, xoff, from + (uint32_t)(8 * j) * ldx, to + (uint32_t)j * 1024u);
    load16_lds(rw, woff, from + (uint32_t)(16 * (j & 1) + 4 * (j >> 1)) * ldw, to + kOperand + (uint32_t)j * 1024u);
  };
  auto load_scales = [&](int k) {                    // of blocks k..k + 3, k a multiple of four
    if (k >= p.blocks) return;
    const uint32_t to = lds0 + kScales + (uint32_t)(k >> 2 & 1) * kSlot + (uint32_t)wave * 256u;
    if (wave < 2) {
      load4_lds(rsx, sxoff, (uint32_t)k, to);
    } else if (!both || lane < 32) {
      load4_lds(rsw, swoff, (uint32_t)k, to);
    } else {
      load4_lds(rsu, swoff, (uint32_t)k, to);
    }
  };

  // ---- a block's operands in registers ----
  struct Block {
    v8i x[4], w[4];
    uint32_t sx[4], sw[4];
  };
  const uint32_t lane_at = (uint32_t)r * kBlock + (uint32_t)((g ^ (r & 7)) * 16);
  const uint32_t sx_at = (uint32_t)(kScales + (wm * 64 + r) * 4), sw_at = (uint32_t)(kScales + (kSide + wn * 64 + r) * 4);
  auto read = [&](int k, Block& b, int t) {          // a quarter of them
    const uint32_t at = (uint32_t)(k & 3) * kBuffer, s_at = (uint32_t)(k >> 2 & 1) * kSlot + (uint32_t)(k & 3);
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      const uint8_t* const from = lds + o * kOperand + ((o ? wn : wm) * 64 + t * 16) * kBlock;
      const v4i lo = *reinterpret_cast<const v4i*>(from + (at + lane_at)), hi = *reinterpret_cast<const v4i*>(from + (at + (lane_at ^ 64u)));
      (o ? b.w : b.x)[t] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      (o ? b.sw : b.sx)[t] = lds[(o ? sw_at : sx_at) + s_at + (uint32_t)(t * 64)];
    }
  };
  auto sums = [&](auto way, v4f (&acc)[4][4]) {      // [w][x]
    constexpr bool APART = decltype(way)::value;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u) acc[t][u] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};

    Block b0, b1;
    load_scales(0);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) load(k, j);
    meet<24>();
#pragma unroll
    for (int t = 0; t < 4; ++t) read(0, b0, t);
    // 16 products of a block, a quarter of the next one's operands and of the loads in front of every four.  (All of them in front of the
    // products, products wait until the LDS has taken the reads: a block 0.59 us; in the compiler's order 0.74.)
    auto step = [&](int k, const Block& now, Block& then) {
      meet<16>();                                    // block k + 1 has come; everyone has read block k
      if ((k & 3) == 0) load_scales(k + 4);
      __builtin_amdgcn_sched_barrier(0);
      WideCodes x[4];
      if constexpr (WIDE) {
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = widen<0, APART>(now.x[u], now.sx[u]);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        read(k + 1, then, t);                        // (behind the last block: of what is there, not used)
        load(k + 4, t);
        if constexpr (WIDE) {
          const WideCodes w = widen<0, APART>(now.w[t], now.sw[t]);
          v4i rows;
          if constexpr (APART) rows = *reinterpret_cast<const v4i*>(lds + (kScales + (k >> 2 & 1) * kSlot + (kSide + wn * 64 + t * 16 + 4 * g) * 4));
#pragma unroll
          for (int u = 0; u < 4; ++u) acc[t][u] = APART ? apart_mfma(w, x[u], acc[t][u], rows, 8 * (k & 3), now.sx[u]) : wide_mfma(w, x[u], acc[t][u]);
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) acc[t][u] = block_mfma<0>(now.w[t], now.x[u], acc[t][u], now.sw[t], now.sx[u]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
#pragma unroll 1
    for (int k = 0; k + 1 < p.blocks; k += 2) {
      step(k, b0, b1);
      step(k + 1, b1, b0);
    }
    if (p.blocks & 1) step(p.blocks - 1, b0, b1);
    meet<0>();                                       // (nothing is on its way to LDS any more)
  };
  v4f acc[4][4];
  sums(std::false_type(), acc);
  if constexpr (WIDE) {                              // (waves share their loads, so all of them again or none)
    bool none = false;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u) none |= put_back(acc[t][u]);
    uint32_t* const flags = reinterpret_cast<uint32_t*>(lds + kFlags);
    const uint32_t mine = __ballot(none) != 0ull;
    if (lane == 0) flags[wave] = mine;
    meet_lds();
    if (scalar(flags[0] | flags[1] | flags[2] | flags[3])) {
      v4f other[4][4];
      sums(std::true_type(), other);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int u = 0; u < 4; ++u) take_apart(acc[t][u], other[t][u]);
    }
  }

  // ---- what is made of the sums ----
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int m = m0 + wm * 64 + u * 16 + r;
    if (m >= p.rows) continue;
    float v[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[k][j] = acc[2 * k + (j >> 2)][u][j & 3];
    if constexpr (MODE == kProduct) {
#pragma unroll
      for (int k = 0; k < 2; ++k) store8_as<WIDE>(p.type, p.out, p.ld_out, m, n0 + wn * 64 + 32 * k + 8 * g, p.cols, v[k]);
    } else if constexpr (MODE == kGated) {
      const int n = n0 + wn * 32 + 8 * g;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[0][j] = gate<WIDE>(p.act, v[0][j]).value * v[1][j];
      if (p.out) store8_as<WIDE>(p.type, p.out, p.ld_out, m, n, p.cols, v[0]);
      if (p.wide) store8_of<QGTC_F32>(p.wide + (int64_t)m * p.ld_wide, n, p.cols, v[0]);
    } else {
      const int n = n0 + wn * 32 + 8 * g;
      float dh[8], dg[8], du[8];
      load8_as<WIDE>(p.type, p.dh, p.ld_dh, m, n, p.cols, dh);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const Gate s = gate<WIDE>(p.act, v[0][j]);
        dg[j] = dh[j] * v[1][j] * s.slope;
        du[j] = dh[j] * s.value;
      }
      store8_as<WIDE>(p.type, p.out, p.ld_out, m, n, p.cols, dg);
      store8_as<WIDE>(p.type, p.out2, p.ld_out2, m, n, p.cols, du);
    }
  }
}

template <int MODE, bool WIDE>
qgtc_status launch(const MidParams& m, unsigned grid, hipStream_t stream) {
  static OncePerDevice once;
  if (!allow_lds(once, reinterpret_cast<const void*>(&mid_kernel<MODE, WIDE>), kMidLds)) return QGTC_ERR_HIP;
  hipLaunchKernelGGL((mid_kernel<MODE, WIDE>), dim3(grid), dim3(256), kMidLds, stream, m);
  return launch_status();
}

}  // namespace

template <int MODE>
qgtc_status launch_mid(const ProductParams& p, bool wide, hipStream_t stream) {
  MidParams m{};
  m.p = p;
  m.tiles_m = (uint32_t)cdiv(p.rows, kSide);
  m.tiles_n = (uint32_t)cdiv(p.cols, MODE == kProduct ? kSide : kSide / 2);
  m.per_group = 8u * m.tiles_n;
  m.per_xcd = (uint32_t)cdiv((int64_t)m.tiles_m * m.tiles_n, 8);
  return wide ? launch<MODE, true>(m, 8u * m.per_xcd, stream) : launch<MODE, false>(m, 8u * m.per_xcd, stream);
}
template qgtc_status launch_mid<kProduct>(const ProductParams& p, bool wide, hipStream_t stream);
template qgtc_status launch_mid<kGated>(const ProductParams& p, bool wide, hipStream_t stream);
template qgtc_status launch_mid<kGatedGrad>(const ProductParams& p, bool wide, hipStream_t stream);

}  // namespace qgtc
