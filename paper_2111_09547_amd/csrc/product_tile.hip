// Products of matrices in 8-bit floats, many rows: tiles of 256 x 256 on the matrix cores.
//
// A workgroup of four waves, one per SIMD, has a tile of 256 rows of X by 256 rows of W, a wave 128 x 128 of it: 64
// v_mfma_scale_f32_16x16x128_f8f6f4 (2048 cycles) per block of K, whose sums fill half of the wave's 512 registers.  Operands of a
// block, 64 KiB, go to LDS without passing through registers, two buffers in turn; a wave reads 32 KiB of them back, which takes
// the LDS 1024 cycles for all four.  64 x 64 per wave would read twice that per product and be bound by the LDS.
//
// A step (a block of K) is four quarters of 16 instructions, of 64 x 64 products each: (w0, x0), (w1, x0), (w0, x1), (w1, x1).
// Beside each, one of the four halves of operands goes to registers: w1, x1, then the next step's x0 and w0, whose registers
// the quarters in front have left.  There is a barrier in the middle of a step and at its end, behind which the halves that
// have just been read are loaded for the step after the next: each has one and a half steps to come (with one barrier, and so
// one step, waves waited a third of the time).  Nothing in the loop may use vector memory in the compiler's own way: its waits are
// for everything that is on its way (one word of scratch in the loop: a fifth more time for 8192 cubed).
//
// Workgroups stay and take several tiles: the loads run on to the next tile while one is finished (a workgroup per tile lost
// 19 us a tile with that, 7 % of 4096 x 16384 x 4096).
//
// A row of a buffer is 128 bytes; its 16-byte piece c lies at c ^ (row % 8), so that 16 lanes reading a piece each of 16 rows meet
// every bank once.  W's rows are put into the buffer in another order: register i of lane group g of the t-th 16 of 64 belongs
// to row 32 (t / 2) + 8 g + 4 (t % 2) + i of them, so that a lane ends up with twice eight results that lie side by side, and four
// lanes with 32, or, where results are bytes, to row 16 g + 4 t + i, and a lane has 16 side by side: 64 bytes of a row for a store
// either way (the other order for bytes: 3 % more for gated 4096 x 4096 x 8192).
#include "product_lds.h"

namespace qgtc {
namespace {

constexpr int kTile = 256;
constexpr int kOperand = kTile * kBlock;           // bytes of an operand's block
constexpr int kBuffer = 2 * kOperand;              // X, then W
constexpr int kScales = 2 * kBuffer;               // words of four blocks' scales: [4 slots][X, W][256]
constexpr int kSlot = 2 * kTile * 4;
constexpr int kTops = kScales + 4 * kSlot;         // largest values of rows: [2][256], and where they have been computed again
constexpr int kTileLds = kTops + 2 * 2 * kTile * 4;

struct TileParams {
  ProductParams p;
  uint32_t tiles_m, tiles_n, per_group;            // per_group: tiles of 8 rows of tiles, which are dealt together
  uint32_t per_xcd;
};

template <int MODE, int TYPE>
__global__ __launch_bounds__(256, 1) void tile_kernel(const TileParams tp) {
  const ProductParams& p = tp.p;
  extern __shared__ __align__(128) uint8_t lds[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
  const int wave = (int)scalar(threadIdx.x >> 6), lane = (int)(threadIdx.x & 63u), r = lane & 15, g = lane >> 4;
  const int wm = wave & 1, wn = wave >> 1;

  // ---- which tiles: an XCD's are neighbours, in groups that are 8 tiles of rows high; its workgroups take them in turn ----
  constexpr int TN = MODE == kProduct ? kTile : kTile / 2;           // columns of the result
  constexpr bool kBytes = MODE == kGated;
  const uint32_t first = (blockIdx.x & 7u) * tp.per_xcd, turn = gridDim.x >> 3;
  const uint32_t behind = min(first + tp.per_xcd, tp.tiles_m * tp.tiles_n);
  uint32_t id = first + (blockIdx.x >> 3);
  if (id >= behind) return;
  auto place = [&](uint32_t tile, int& m0, int& bn) {
    const uint32_t group = tile / tp.per_group, first_m = group * 8u, high = min(8u, tp.tiles_m - first_m), in = tile - group * tp.per_group;
    m0 = (int)scalar((first_m + in % high) * kTile);
    bn = (int)scalar(in / high);
  };

  // ---- loads: this wave's are 32 rows of each half of 128 rows of each operand, 8 rows a load, and 64 words of scales.  They
  // run two blocks ahead of the products, on to the next tile ----
  const bool both = MODE != kProduct;                    // two projections: the halves of a wave's 128 rows are one's and the other's
  const int part = wave & 1, pair = wave >> 1;
  const uint32_t piece = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16u;
  const uint8_t* const w_scales = both && part ? p.u.scales : p.w.scales;
  const int64_t w_ld_scales = both && part ? p.u.ld_scales : p.w.ld_scales;
  const uint32_t row_bytes = (uint32_t)p.blocks * kBlock, row_words = (uint32_t)((p.blocks + 3) & ~3);
  v4i rx, rsx, rw[2], rsw;
  auto aim = [&](uint32_t tile) {
    int m0, bn;
    place(tile, m0, bn);
    const int n0 = bn * TN;
    const uint32_t most_x = (uint32_t)min(kTile, p.rows - m0) - 1u, most_w = (uint32_t)min(TN, p.cols - n0) - 1u;
    rx = buffer_of(p.x.codes + (int64_t)m0 * p.x.ld, most_x * (uint32_t)p.x.ld + row_bytes);
    rsx = buffer_of(p.x.scales + (int64_t)m0 * p.x.ld_scales, most_x * (uint32_t)p.x.ld_scales + row_words);
    rw[0] = buffer_of(p.w.codes + (int64_t)n0 * p.w.ld, most_w * (uint32_t)p.w.ld + row_bytes);
    rw[1] = both ? buffer_of(p.u.codes + (int64_t)n0 * p.u.ld, most_w * (uint32_t)p.u.ld + row_bytes) : rw[0];
    rsw = buffer_of(w_scales + (int64_t)n0 * w_ld_scales, most_w * (uint32_t)w_ld_scales + row_words);
  };
  // rows 128 pair + 64 h + 32 part + 8 j + lane / 8 of X's buffer, which are X's; and of W's
  const uint32_t ldx = (uint32_t)p.x.ld, ldw[2] = {(uint32_t)p.w.ld, both ? (uint32_t)p.u.ld : (uint32_t)p.w.ld};
  const uint32_t xoff = (uint32_t)(128 * pair + 32 * part + (lane >> 3)) * ldx + piece;
  uint32_t woff[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) woff[h] = (uint32_t)((both ? 64 : 128) * pair + (kBytes ? 8 : 32) * part + (kBytes ? 16 : 8) * (lane >> 5) + (lane >> 3 & 3)) * ldw[h] + piece;
  const uint32_t sxoff = (uint32_t)(64 * wave + lane) * (uint32_t)p.x.ld_scales;
  const uint32_t swoff = (uint32_t)((both ? 64 * pair : 64 * wave) + (kBytes ? 4 * g + 16 * (r >> 2) : 32 * (g >> 1) + 8 * (r >> 2) + 4 * (g & 1)) + (r & 3)) * (uint32_t)w_ld_scales;
  const uint32_t to_x = lds0 + (uint32_t)(128 * pair + 32 * part) * kBlock, to_w = to_x + kOperand;
  uint32_t load_id = id;
  int load_step = 0, load_slot = 0;
  auto load_one = [&](uint32_t buffer, int h, int j) {   // an eighth of a wave's loads of a block's halves h
    const uint32_t at = buffer + (uint32_t)(64 * h) * kBlock + (uint32_t)(j & 3) * 1024u, from = (uint32_t)load_step * kBlock;
    if (j < 4) load16_lds(rx, xoff, from + (uint32_t)(64 * h + 8 * j) * ldx, to_x + at);
    else load16_lds(rw[h], woff[h], from + (uint32_t)((both ? 0 : 64 * h) + (kBytes ? 32 : 16) * (j & 1) + 4 * (j >> 1 & 1)) * ldw[h], to_w + at);
  };
  auto load_scales = [&] {                               // in front of every fourth block
    if ((load_step & 3) != 0) return;
    const uint32_t at = lds0 + kScales + (uint32_t)load_slot * kSlot + (uint32_t)wave * 256u;
    load4_lds(rsx, sxoff, (uint32_t)load_step, at);
    load4_lds(rsw, swoff, (uint32_t)load_step, at + kTile * 4);
    load_slot = (load_slot + 1) & 3;
  };
  auto load_next = [&] {
    if (++load_step < p.blocks) return;
    load_step = 0;                                       // (behind the last tile: that one again, for nobody)
    if (load_id + turn < behind) {
      load_id += turn;
      aim(load_id);
    }
  };

  // ---- operands from LDS ----
  const uint32_t lane_at = (uint32_t)r * kBlock + (uint32_t)((g ^ (r & 7)) * 16);
  auto read4 = [&](uint32_t buffer, int operand, int half, int t) -> v8i {
    const uint8_t* const at = lds + ((operand ? wn : wm) * (128 * kBlock) + operand * kOperand + (half * 64 + t * 16) * kBlock);
    const v4i a = *reinterpret_cast<const v4i*>(at + (buffer + lane_at)), b = *reinterpret_cast<const v4i*>(at + (buffer + (lane_at ^ 64u)));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  const uint32_t sx_at = (uint32_t)(kScales + (wm * 128 + r) * 4), sw_at = (uint32_t)(kScales + (kTile + wn * 128 + r) * 4);
  auto read_scale = [&](uint32_t at, int operand, int half, int t) -> uint32_t {   // at: slot and byte
    return lds[(operand ? sw_at : sx_at) + at + (uint32_t)((half * 64 + t * 16) * 4)];
  };

  v4f acc[2][2][4][4];                                 // [half of w][half of x][w][x]
  v8i x[2][4], w[2][4];
  uint32_t sx[2][4], sw[2][4];

  // A quarter: 16 products, and beside them four operands (two reads each) and four loads.
  auto quarter = [&](int hw, int hx, auto&& fetch, auto&& load) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      fetch(t);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        acc[hw][hx][t][u] = block_mfma<0>(w[hw][t], x[hx][u], acc[hw][hx][t][u], sw[hw][t], sx[hx][u]);
        if (u == 1) load(t);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // ---- what is made of the sums: lane (r, g) has row 16 u + r of each half of x, and of each half of w the columns 32 k + 8 g + j (bytes:
  // 8 k + 16 g + j), k = 0, 1 and j = 0..7, in register j % 4 of the sums 2 k + j / 4 ----
  typedef typename Float<TYPE>::type T;
  auto finish = [&](uint32_t tile) {
    // (Anew for every tile: what the compiler makes of these once for all tiles it keeps in scratch memory, and each load of it from
    // there waits for everything that is on its way: 8 % of gated 4096 x 4096 x 8192.)
    int own = lane;
    asm volatile("" : "+v"(own));
    const int r = own & 15, g = own >> 4;
    int m0, bn;
    place(tile, m0, bn);
    const bool whole = bn * TN + TN <= p.cols;           // (a branch for all lanes: the other way is long)
    auto row_of = [&](int hx, int u) { return m0 + wm * 128 + hx * 64 + u * 16 + r; };
    auto store8 = [&](void* base, int64_t ld, int m, int n, const float (&v)[8]) {
      T* const to = (T*)base + (int64_t)m * ld;
      if (whole) Float<TYPE>::store8(to + n, v);
      else store8_of<TYPE>(to, n, p.cols, v);
    };
    if constexpr (MODE == kProduct) {
#pragma unroll
      for (int hx = 0; hx < 2; ++hx)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int m = row_of(hx, u);
          if (m < p.rows) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float v[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) v[j] = acc[q >> 1][hx][2 * (q & 1) + (j >> 2)][u][j & 3];
              store8(p.out, p.ld_out, m, bn * TN + wn * 128 + 32 * q + 8 * g, v);
            }
          }
        }
    } else if constexpr (MODE == kGated) {
      const int n0 = bn * TN + wn * 64 + 16 * g;
      uint32_t* const tops = reinterpret_cast<uint32_t*>(lds + kTops);
      float h[8][16];                                    // (in the registers that operands of the products leave)
#pragma unroll
      for (int hx = 0; hx < 2; ++hx)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int m = row_of(hx, u);
          uint32_t top = 0u;
          // (columns past the end are products with the zeros that were loaded there)
          auto gates = [&](int act) {
#pragma unroll
            for (int j = 0; j < 16; ++j) h[hx * 4 + u][j] = gate<false>(act, acc[0][hx][j >> 2][u][j & 3]).value * acc[1][hx][j >> 2][u][j & 3];
          };
          if (p.act == QGTC_ACT_SILU) gates(QGTC_ACT_SILU);
          else gates(QGTC_ACT_GELU);
          top = abs_max(h[hx * 4 + u]);
          if (p.out && m < p.rows) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              float v[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) v[j] = h[hx * 4 + u][8 * k + j];
              store8(p.out, p.ld_out, m, n0 + 8 * k, v);
            }
          }
          top = max(top, (uint32_t)__shfl_xor((int)top, 16));
          top = max(top, (uint32_t)__shfl_xor((int)top, 32));
          if (g == 0) tops[wn * kTile + wm * 128 + hx * 64 + u * 16 + r] = top;
        }
      if (!p.codes) return;
      meet_lds();
      uint32_t* const again = tops + 2 * kTile;
      uint32_t near = 0u;                                // 16 rows in which the exact largest value is wanted
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int lr = wm * 128 + i * 16 + r;
        const uint32_t mine = tops[wn * kTile + lr];
        near |= __ballot(near_border(max(mine, tops[(wn ^ 1) * kTile + lr]))) ? 1u << i : 0u;
        if (g == 0) again[wn * kTile + lr] = mine;
      }
      if (near) {
        uint32_t want[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int lr = wm * 128 + i * 16 + r;
          const uint32_t top = max(tops[lr], tops[kTile + lr]), from = m0 + lr < p.rows && near_border(top) ? border_from(top) : 0xffffffffu;
          want[i] = 0u;
#pragma unroll
          for (int j = 0; j < 16; ++j) want[i] |= abs_bits(h[i][j]) >= from ? 1u << j : 0u;
        }
#pragma unroll 1
        for (; near; near &= near - 1u) {                // (once, not for every 16 rows: the loop of products has to stay in the cache)
          const int i = __ffs(near) - 1, lr = wm * 128 + i * 16 + r;
          uint32_t mine = 0u;
#pragma unroll
          for (int j = 0; j < 8; ++j) mine = j == i ? want[j] : mine;
          uint32_t exact = exact_top(p, m0 + lr, n0, mine);
          exact = max(exact, (uint32_t)__shfl_xor((int)exact, 16));
          exact = max(exact, (uint32_t)__shfl_xor((int)exact, 32));
          const uint32_t top = max(tops[lr], tops[kTile + lr]);
          if (g == 0 && near_border(top)) again[wn * kTile + lr] = border_side(top, exact);
        }
      }
      meet_lds();
#pragma unroll
      for (int hx = 0; hx < 2; ++hx)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int m = row_of(hx, u), lr = wm * 128 + hx * 64 + u * 16 + r;
          if (m < p.rows) {
            const uint32_t e = scale_byte(max(again[lr], again[kTile + lr]));
            u32x4 c;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const float* const v = &h[hx * 4 + u][4 * t];
              c[t] = encode4(v[0], v[1], v[2], v[3], e);
            }
            if (!whole && e == 255u) {                   // (zeros past the end, whatever the block)
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                const int left = p.cols - (n0 + 4 * t);
                if (left < 4) c[t] &= left <= 0 ? 0u : 0xffffffffu >> (8 * (4 - left));
              }
            }
            *reinterpret_cast<u32x4*>(p.codes + (int64_t)m * p.ld_codes + n0) = c;
            if (g == 0 && wn == 0) p.scales[(int64_t)m * p.ld_scales + bn] = (uint8_t)e;
          }
        }
      // (the next tile's largest values are written a barrier of its products later)
    } else {
      const int n0 = bn * TN + wn * 64 + 8 * g;
      // (all of dh at once: each load that is waited for waits for the next tile's operands as well)
      u32x4 dh_bits[8][2];
      if (whole) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int m = min(m0 + wm * 128 + (i >> 1) * 16 + r, p.rows - 1);
          dh_bits[i >> 1][i & 1] = *reinterpret_cast<const u32x4_any*>((const T*)p.dh + (int64_t)m * p.ld_dh + n0 + 32 * (i & 1));
        }
      }
#pragma unroll
      for (int hx = 0; hx < 2; ++hx)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int m = row_of(hx, u);
          if (m < p.rows) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int n = n0 + 32 * k;
              float dh[8], dg[8], du[8];
              if (whole) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const f32x2 v = Half<TYPE>::wide(dh_bits[hx * 4 + u][k][j]);
                  dh[2 * j] = v.x;
                  dh[2 * j + 1] = v.y;
                }
              } else {
                load8_of<TYPE>((const T*)p.dh + (int64_t)m * p.ld_dh, n, p.cols, dh);
              }
              auto gates = [&](int act) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  const int t = 2 * k + (j >> 2);
                  const Gate v = gate<false>(act, acc[0][hx][t][u][j & 3]);
                  dg[j] = dh[j] * acc[1][hx][t][u][j & 3] * v.slope;
                  du[j] = dh[j] * v.value;
                }
              };
              if (p.act == QGTC_ACT_SILU) gates(QGTC_ACT_SILU);
              else gates(QGTC_ACT_GELU);
              store8(p.out, p.ld_out, m, n, dg);
              store8(p.out2, p.ld_out2, m, n, du);
            }
          }
        }
    }
  };

  aim(id);
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    if (i) load_next();
    load_scales();
#pragma unroll
    for (int j = 0; j < 16; ++j) load_one((uint32_t)i * kBuffer, j >> 3, j & 7);
  }
  meet<16>();
  uint32_t cur = 0, slot = 0;
#pragma unroll 1
  for (; id < behind; id += turn) {
    // (once more behind a tile, whose last quarters have read these too: the registers are better used in between)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      x[0][t] = read4(cur, 0, 0, t);
      w[0][t] = read4(cur, 1, 0, t);
      sx[0][t] = read_scale(slot * kSlot, 0, 0, t);
      sw[0][t] = read_scale(slot * kSlot, 1, 0, t);
    }
    meet<16>();
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int d = 0; d < 4; ++d) acc[a][b][c][d] = (v4f){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int k = 0; k < p.blocks; ++k) {
      const uint32_t next = cur ^ kBuffer, at = slot * kSlot + (uint32_t)(k & 3);
      const int then = k + 1 < p.blocks ? k + 1 : 0;
      if ((then & 3) == 0) slot = (slot + 1) & 3;
      const uint32_t at_next = slot * kSlot + (uint32_t)(then & 3);
      load_next();
      load_scales();
      __builtin_amdgcn_sched_barrier(0);
      quarter(0, 0, [&](int t) { w[1][t] = read4(cur, 1, 1, t); sw[1][t] = read_scale(at, 1, 1, t); }, [&](int j) { load_one(cur, 0, j); });
      quarter(1, 0, [&](int t) { x[1][t] = read4(cur, 0, 1, t); sx[1][t] = read_scale(at, 0, 1, t); }, [&](int j) { load_one(cur, 0, 4 + j); });
      meet<16>();
      __builtin_amdgcn_sched_barrier(0);
      quarter(0, 1, [&](int t) { x[0][t] = read4(next, 0, 0, t); sx[0][t] = read_scale(at_next, 0, 0, t); }, [&](int j) { load_one(cur, 1, j); });
      quarter(1, 1, [&](int t) { w[0][t] = read4(next, 1, 0, t); sw[0][t] = read_scale(at_next, 1, 0, t); }, [&](int j) { load_one(cur, 1, 4 + j); });
      meet<16>();
      __builtin_amdgcn_sched_barrier(0);
      cur = next;
    }
    finish(id);
  }
  meet<0>();                                           // (nothing is on its way to LDS any more)
}

template <int MODE, int TYPE>
qgtc_status launch(const TileParams& t, unsigned workgroups, hipStream_t stream) {
  static OncePerDevice once;
  if (!allow_lds(once, reinterpret_cast<const void*>(&tile_kernel<MODE, TYPE>), kTileLds)) return QGTC_ERR_HIP;
  hipLaunchKernelGGL((tile_kernel<MODE, TYPE>), dim3(workgroups), dim3(256), kTileLds, stream, t);
  return launch_status();
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
  const uint32_t most = (uint32_t)(device_compute_units() / 8), workgroups = 8u * (t.per_xcd < most ? t.per_xcd : most);
  return p.type == QGTC_F16 ? launch<MODE, QGTC_F16>(t, workgroups, stream) : launch<MODE, QGTC_BF16>(t, workgroups, stream);
}
template qgtc_status launch_tiles<kProduct>(const ProductParams& p, hipStream_t stream);
template qgtc_status launch_tiles<kGated>(const ProductParams& p, hipStream_t stream);
template qgtc_status launch_tiles<kGatedGrad>(const ProductParams& p, hipStream_t stream);

}  // namespace qgtc
