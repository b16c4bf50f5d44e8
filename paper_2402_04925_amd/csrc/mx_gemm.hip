// Product of microscaled (MX) operands on gfx950, Y = X W^T: X in fp8 (E4M3) or
// fp4 (E2M1) rows, W in fp4 tiles (mx_internal.h), both with one E8M0 scale per 32
// elements of K. The scaled matrix instruction takes the codes and the scales as
// they are stored, so nothing is dequantized: an output is a sum of fp32 accumulators
// (of the waves, groups of waves or splits that share K, in their order), rounded once.
//
// The weights are the instruction's first operand and X its second, so that a
// lane's results are consecutive outputs of one row of X. A tile of 32 weight
// rows is two operands j = 0, 1 whose row r is weight row 8 (r / 4) + 4 j + r % 4:
// the lane (m, g) then holds outputs 8 g .. 8 g + 7 of row m in its two
// accumulators, one 16-byte store, and four lanes hold one block of 32 outputs,
// which is what quantizing them for the next product needs.
#include <algorithm>

#include "mx_common.h"

namespace tpdq {
namespace {

// Few rows of X: the weight stream bounds it. A workgroup owns TN operands of 16
// outputs (2: a whole tile; GATED: of the gate and the up projection) over the
// whole of K and MT tiles of 16 rows. Its waves take chunks of 512 elements of K in
// turn: the chunk's weights straight to registers (1 KB contiguous per load), its
// rows of X to a part of LDS of the wave's own, 8 rows of a 128-byte line per load
// and read back as the operand (a load of the operand itself would touch 16 rows
// of half a line). The waves add their accumulators in LDS at the end.
template <int DT, int FMT, int MT, int TN, bool GATED, bool QUANT, int NWMAX>
__global__ __launch_bounds__(NWMAX * 64) void k_mx_rows(MxArgs a) {
  static_assert(TN == 2 || (!GATED && !QUANT), "a block of outputs is a whole tile");
  constexpr int P = GATED ? 2 : 1;
  constexpr int NT = TN * P;                 // operands per workgroup
  constexpr int XW = FMT == kFp4 ? 1 : 2;    // 64-byte halves of a row's line per step
  constexpr int LINES = 2 * XW;              // 128-byte lines of a row per chunk
  constexpr int XWAVE = MT * LINES * 2048;   // LDS of a wave
  extern __shared__ __align__(16) unsigned char smem[];
  f4_t* red = (f4_t*)smem;  // [wave][MT * NT][64], after the loop
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nw = blockDim.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int steps = (a.K + kMxStep - 1) / kMxStep;
  const int chunks = (a.K + kMxChunk - 1) / kMxChunk;
  const int tiles = (a.N + kMxTile - 1) / kMxTile;
  const int wg = xcd_run(blockIdx.x, gridDim.x);
  const int T = TN == 2 ? wg : wg >> 1;      // the tile, and of half a tile the operand
  const int j0 = TN == 2 ? 0 : wg & 1;
  unsigned char* xl = smem + wave * XWAVE;

  // a tile past the last one and rows past M load zeros from the resource bounds
  const uint32_t wbytes = (uint32_t)(tiles - 1) * (uint32_t)a.ldwc + (uint32_t)steps * 2048u;
  const uint32_t sbytes = (uint32_t)(tiles - 1) * (uint32_t)a.ldws + (uint32_t)chunks * 512u;
  const uint32_t xbytes = (uint32_t)(a.M - 1) * (uint32_t)a.x.ld_c + (uint32_t)steps * (64u * XW);
  const uint32_t xsbytes = (uint32_t)(a.M - 1) * (uint32_t)a.x.ld_s + (uint32_t)chunks * 16u;
  const __amdgpu_buffer_rsrc_t rxs = buffer_rsrc(a.x.scales, xsbytes);
  uint32_t offx[2 * MT], offxs[MT];
#pragma unroll
  for (int t = 0; t < 2 * MT; ++t) {  // 8 rows each; lane: row lane / 8, chunk of 16 bytes swapped as in LDS
    const int m = 8 * t + (lane >> 3);
    offx[t] = m < a.M ? (uint32_t)m * (uint32_t)a.x.ld_c + 16u * (uint32_t)((lane & 7) ^ (lane >> 3))
                      : kOutOfRange;
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) offxs[t] = 16 * t + r < a.M ? (uint32_t)(16 * t + r) * (uint32_t)a.x.ld_s : kOutOfRange;
  const uint32_t offw = T < tiles ? (uint32_t)T * (uint32_t)a.ldwc + 1024u * j0 + 16u * lane : kOutOfRange;
  const uint32_t offs = T < tiles ? (uint32_t)T * (uint32_t)a.ldws + 8u * lane : kOutOfRange;
  // row r's chunk c of a line is at place c ^ (r % 8): 8 rows fill a 128-byte cycle
  const int xpos0 = r * 128 + ((g ^ (r & 7)) << 4), xpos1 = xpos0 ^ 64;

  f4_t acc[MT][NT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};

#pragma unroll 1
  for (int c = wave; c < chunks; c += nw) {
#pragma unroll
    for (int l = 0; l < LINES; ++l) {
      const bool in = 4 * c + 2 * l / XW < steps;
      const __amdgpu_buffer_rsrc_t rx = buffer_rsrc(a.x.codes, in ? xbytes : 0u);
#pragma unroll
      for (int t = 0; t < 2 * MT; ++t)
        if (8 * t < a.M)  // rows past M only reach outputs past M: their place may hold anything
          dma_lds<16>(rx, xl + ((t >> 1) * LINES + l) * 2048 + (t & 1) * 1024, offx[t],
                  in ? (uint32_t)(c * LINES + l) * 128u : 0u);
    }
    __builtin_amdgcn_sched_barrier(0);
    u4_t xs[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) xs[t] = buffer_load16(rxs, offxs[t] + 16u * c);
    u2_t ws[P];
    u4_t w[NT][4];
#pragma unroll
    for (int h = 0; h < P; ++h) {
      const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(h ? a.ws_up : a.ws, sbytes);
      ws[h] = __builtin_bit_cast(u2_t, __builtin_amdgcn_raw_buffer_load_b64(rs, offs + 512u * c, 0, 0));
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const bool in = 4 * c + s < steps;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const __amdgpu_buffer_rsrc_t rw = buffer_rsrc(GATED && i >= 2 ? a.wc_up : a.wc, in ? wbytes : 0u);
        w[i][s] = __builtin_bit_cast(u4_t, __builtin_amdgcn_raw_buffer_load_b128(
            rw, offw + 1024u * (i & 1), in ? (uint32_t)(4 * c + s) * 2048u : 0u, kNonTemporal));
      }
    }
    // X has landed, the loads issued after it may be in flight
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(MT + P + 4 * NT) : "memory");
    auto step = [&](auto sel) {
      constexpr int s = decltype(sel)::value;
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const unsigned char* xt = xl + (t * LINES + s * XW / 2) * 2048;
        const u4_t lo = *(const u4_t*)(xt + (XW == 1 && s % 2 ? xpos1 : xpos0));
        u4_t hi = {0u, 0u, 0u, 0u};
        if constexpr (XW == 2) hi = *(const u4_t*)(xt + xpos1);
        const i8_t x = {(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        const uint32_t xsc = xs[t][s] >> (8 * g);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const uint32_t wsc = TN == 2 ? ws[i >> 1][i & 1] : (j0 ? ws[0].y : ws[0].x);
          acc[t][i] = mfma_mx<FMT, s>(w[i][s], wsc, x, xsc, acc[t][i]);
        }
      }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
    // the next chunk's loads overwrite what was read here
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  __syncthreads();

  // operand i of row tile t -> red
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < NT; ++i) red[(wave * MT * NT + t * NT + i) * 64 + lane] = acc[t][i];
  __syncthreads();
  // sums over the waves, in the waves' order, into wave 0's part
  for (int i = threadIdx.x; i < MT * NT * 64; i += blockDim.x) {
    f4_t s = red[i];
    for (int w = 1; w < nw; ++w) s += red[w * MT * NT * 64 + i];
    red[i] = s;
  }
  __syncthreads();
  for (int t = wave; t < MT; t += nw) {
    const int m = 16 * t + r;
    if constexpr (TN == 1) {
      const f4_t y = red[t * 64 + lane];
      const int64_t n = (int64_t)T * kMxTile + 8 * g + 4 * j0;
      if (m < a.M && n < a.N) *(u2_t*)(a.Y + (int64_t)m * a.ldy + n) = u2_t{pack2<DT>(y[0], y[1]), pack2<DT>(y[2], y[3])};
    } else {
      float v[8];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f4_t y = red[(t * NT + j) * 64 + lane];
        f4_t u = y;
        if constexpr (GATED) u = red[(t * NT + 2 + j) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * j + e] = GATED ? silu_mul(y[e], u[e]) : y[e];
      }
      store_out8<DT, FMT, QUANT>(a, v, m, (int64_t)T * kMxTile + 8 * g);
    }
  }
}

template <int DT, int FMT, int MT, int TN, bool GATED, bool QUANT, int NWMAX>
hipError_t rows_launch(const MxArgs& a, hipStream_t s) {
  // quantized outputs: also the tiles of the padding to whole chunks (zeros)
  const int tiles = (int)(QUANT ? mx_chunks(a.N) * (kMxChunk / kMxTile) : (a.N + kMxTile - 1) / kMxTile);
  const int nw = (int)std::min<int64_t>(NWMAX, mx_chunks(a.K));
  constexpr int x = MT * (FMT == kFp4 ? 2 : 4) * 2048, red = MT * TN * (GATED ? 2 : 1) * 1024;
  constexpr int wave_lds = x > red ? x : red;
  static_assert((size_t)NWMAX * wave_lds <= kLdsMax, "");
  auto* k = k_mx_rows<DT, FMT, MT, TN, GATED, QUANT, NWMAX>;
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_lds((const void*)k, NWMAX * wave_lds, &done);
  if (e != hipSuccess) return e;
  k<<<dim3((unsigned)(TN == 2 ? tiles : 2 * tiles)), dim3((unsigned)nw * 64), nw * wave_lds, s>>>(a);
  return hipGetLastError();
}

template <int DT, int FMT, bool GATED, bool QUANT>
hipError_t rows_pick(const MxArgs& a, int kind, hipStream_t s) {
  constexpr int NW4 = FMT == kFp8 ? 5 : GATED ? 8 : 10;  // what LDS, or registers, hold of 64 rows
  if constexpr (!GATED && !QUANT) {
    if (kind == kMxRowsHalf) {
      if (a.M <= 16) return rows_launch<DT, FMT, 1, 1, GATED, QUANT, 16>(a, s);
      if (a.M <= 32) return rows_launch<DT, FMT, 2, 1, GATED, QUANT, 8>(a, s);
      return rows_launch<DT, FMT, 4, 1, GATED, QUANT, NW4>(a, s);
    }
  }
  if (a.M <= 16) return rows_launch<DT, FMT, 1, 2, GATED, QUANT, 16>(a, s);
  if (a.M <= 32) return rows_launch<DT, FMT, 2, 2, GATED, QUANT, 8>(a, s);
  return rows_launch<DT, FMT, 4, 2, GATED, QUANT, NW4>(a, s);
}

template <int FMT>
hipError_t rows_of(const MxArgs& a, int kind, int dt, hipStream_t s) {
  if (a.wc_up) return rows_pick<kF16, FMT, true, true>(a, kind, s);
  if (!a.Y) return rows_pick<kF16, FMT, false, true>(a, kind, s);
  return dt == TPDQ_BF16 ? rows_pick<kBF16, FMT, false, false>(a, kind, s) : rows_pick<kF16, FMT, false, false>(a, kind, s);
}

}  // namespace

// Microseconds of a product, fitted to 20,000 launches on 1,380 random sizes (1 to
// 2048 rows, 512 to 32768 outputs, 512 to 16384 of K; 7 to 14% rms, the few-row kernel
// up to 17%): the choice made by them is 1.1% slower than the best of all kernels,
// tiles and splits on average, 16% at the 99th percentile. A workgroup takes max(c1, c2 n)
// per step of K (of its groups' longest), n workgroups to a CU, e more for each beyond
// the first; parts are written and read once. What the choice is for: 8192 x 8192 at 64 rows fp8 takes
// 15.9 us in the few-row kernel, 16.4 in tiles of 64 x 128 over 4 splits and 22.9
// without (the first two are predicted alike, 14.2, and the splits taken); 28672 outputs
// there 55, 36 (2 splits) and 30; 8192 outputs of K 3584 at 1000 rows 28 in tiles of 64 x
// 512, 32 of 64 x 128, 41 of 128 x 512; 14336 of K 8192 at 2048 rows 204, 230 and 172.
// No term stands for memory: up to 128 rows of many outputs, where the weights' stream
// bounds every kernel, a prediction can lie under it (28672 outputs at 64 rows 18.4 us,
// the weights at a copy's rate 24) and the other terms choose.
// A row of 64 x 128 is of the plain product or, with two groups of waves over K, of the
// gated one, which no 64 x 64 serves.
enum Uses { kPlain = 1, kGated = 2, kBoth = 3 };
struct TileCost {
  int kind, uses, bm, bn, groups;
  double start, c1, c2, e, reduce, mb;
};
constexpr TileCost kTileFp8[] = {{kMxTiles128x512, kBoth, 128, 512, 1, 8.4, 0.71, 1.12, 1.0, 5.0, 6.7e6},
                                 {kMxTiles64x512, kBoth, 64, 512, 1, 5.0, 0.00, 0.674, 2.9, 3.4, 5.2e6},
                                 {kMxTiles64x256, kBoth, 64, 256, 1, 4.4, 0.18, 0.354, 1.5, 3.2, 4.8e6},
                                 {kMxTiles128x256, kBoth, 128, 256, 1, 6.9, 0.43, 0.61, 0.5, 4.8, 7.1e6},
                                 {kMxTiles64x128, kPlain, 64, 128, 1, 3.7, 0.05, 0.230, 0.9, 3.0, 4.4e6},
                                 {kMxTiles64x128, kGated, 64, 128, 2, 5.5, 0.235, 0.406, 4.3, 3.0, 4.4e6},
                                 {kMxTiles64x64, kPlain, 64, 64, 2, 4.9, 0.25, 0.314, 3.2, 3.0, 4.4e6}};
constexpr TileCost kTileFp4[] = {{kMxTiles128x512, kBoth, 128, 512, 1, 8.3, 0.00, 0.676, 8.6, 6.4, 8.5e6},
                                 {kMxTiles64x512, kBoth, 64, 512, 1, 4.5, 0.00, 0.546, 2.6, 3.8, 5.4e6},
                                 {kMxTiles64x256, kBoth, 64, 256, 1, 4.2, 0.01, 0.257, 2.0, 3.4, 5.2e6},
                                 {kMxTiles128x256, kBoth, 128, 256, 1, 6.2, 0.24, 0.400, 1.5, 5.0, 7.0e6},
                                 {kMxTiles64x128, kPlain, 64, 128, 1, 3.5, 0.10, 0.163, 1.0, 3.2, 4.6e6},
                                 {kMxTiles64x128, kGated, 64, 128, 2, 4.6, 0.235, 0.307, 1.4, 3.2, 4.6e6},
                                 {kMxTiles64x64, kPlain, 64, 64, 2, 4.3, 0.12, 0.217, 1.2, 3.2, 4.6e6}};
// The few-row kernel: start + n (workgroups to a CU) iter (chunks a wave takes) +
// wave (waves), by rows up to 16, 32, 64
struct RowsCost {
  int waves;
  double start, iter, wave;
};
constexpr RowsCost kRowsFp8[] = {{16, 2.5, 0.49, 0.26}, {8, 0.9, 2.67, 0.27}, {5, 0.9, 2.6, 0.59}};
constexpr RowsCost kRowsFp4[] = {{16, 2.1, 0.72, 0.25}, {8, 1.8, 1.37, 0.31}, {10, 1.4, 2.78, 0.34}};
constexpr int kCus = 256;
// split-K parts of a call take at most this much workspace
constexpr int64_t kMxPartBytes = (int64_t)64 << 20;

int up(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

MxPlan plan_mx(int M, int N, int K, int fmt, bool gated, bool quant) {
  const bool fp4 = fmt == TPDQ_MX_FP4;
  const int weights = gated ? 2 : 1;
  const int steps = (int)mx_steps(K), chunks = (int)mx_chunks(K), tiles = up(N, kMxTile);
  MxPlan best{kMxRows, 1};
  double least = 1e30;
  if (M <= 64) {
    const RowsCost& c = (fp4 ? kRowsFp4 : kRowsFp8)[M <= 16 ? 0 : M <= 32 ? 1 : 2];
    const int waves = std::min(c.waves, chunks);
    // gated: twice the weights on the same X (the MLP of 8192 / 3584 / 8192 at 32 rows
    // fp8 20.6 us so, 23.3 with tiles of 64 x 256 over 4 splits)
    least = c.start + up(tiles, kCus) * (gated ? 1.5 : 1.0) * c.iter * up(chunks, waves) + c.wave * waves;
    // Half tiles where they all find a CU of their own: 8192 x 3584 at 1 row 6.7 ->
    // 5.7 us, at 16 8.1 -> 7.1; past that they are slower (6144 x 6144 at 16 rows,
    // 192 tiles: 7.3 -> 9.8). A block of quantized outputs is a whole tile.
    if (!quant && 2 * tiles <= kCus) {
      best.kind = kMxRowsHalf;
      least *= M <= 16 ? 0.85 : 0.72;
    }
  }
  for (const TileCost& c : fp4 ? kTileFp4 : kTileFp8) {
    if (!(c.uses & (gated ? kGated : kPlain))) continue;
    if (c.bm > 64 && M <= 64) continue;  // half of the rows empty never pay
    const int64_t wgs = (int64_t)up(M, c.bm) * up((int64_t)N * weights, c.bn);
    const int block = !fp4 && c.bm == 128 ? 2 : 4, blocks = up(steps, block);
    for (int ks : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16}) {
      if (ks > blocks || (ks > 1 && (wgs * ks > 3 * kCus || (int64_t)ks * M * N * 4 * weights > kMxPartBytes))) break;
      const int n = up(wgs * ks, kCus);
      double t = c.start + (double)(up(blocks, ks * c.groups) * block) * std::max(c.c1, c.c2 * n) + c.e * (n - 1);
      if (ks > 1) t += c.reduce + (double)ks * M * N * weights * 8 / c.mb;
      // (3,000 gated launches: the choice 1.1% from the best so, 1.4 without; the first
      // product of 8192 / 3584 / 8192 at 1000 rows 53.5 us here, 49.3 in tiles of 64 x 512)
      if (gated && c.kind == kMxTiles128x256) t *= 1.06;
      if (t < least) {
        least = t;
        best = MxPlan{c.kind, ks};
      }
    }
  }
  return best;
}

size_t mx_part_bytes(const MxPlan& p, int M, int N, bool gated) {
  return p.ks > 1 ? align_up((size_t)p.ks * M * N * (gated ? 8 : 4)) : 0;
}

hipError_t allow_lds(const void* f, int bytes, std::atomic<uint64_t>* done) {
  if (bytes <= 64 * 1024) return hipSuccess;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = (uint64_t)1 << (dev & 63);
  if (dev < 64 && (done->load(std::memory_order_relaxed) & bit)) return hipSuccess;
  e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess && dev < 64) done->fetch_or(bit, std::memory_order_relaxed);
  return e;
}

hipError_t launch_mx_gemm(MxArgs a, int dt, int fmt, float* part, hipStream_t s) {
  const MxPlan p = plan_mx(a.M, a.N, a.K, fmt, a.wc_up != nullptr, a.Y == nullptr);
  a.ks = p.ks;
  a.part = part;
  if (p.kind != kMxRows && p.kind != kMxRowsHalf) return launch_mx_tiles(a, p.kind, dt, fmt, s);
  return fmt == TPDQ_MX_FP4 ? rows_of<kFp4>(a, p.kind, dt, s) : rows_of<kFp8>(a, p.kind, dt, s);
}

}  // namespace tpdq
