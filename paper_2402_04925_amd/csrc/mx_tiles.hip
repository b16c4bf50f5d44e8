// Product of microscaled (MX) operands with many rows of X on gfx950: the matrix
// pipe bounds it (mx_gemm.hip has the few-row kernel and the operands' layout).
//
// A workgroup of NW KG waves computes 16 RT rows x 32 NP NW outputs (GATED: NP = 2, a
// tile of the gate and one of the up projection per wave), a wave all of the rows,
// RT x 2 NP accumulators. Small tiles are worked by KG groups of NW waves, each over a
// part of K with LDS of its own and added there at the end, which gives a CU twice the
// loads in flight and needs no second kernel for the sum (gated, 1792 outputs of K 4096 at
// 400 rows fp8 13.5 us, in tiles of 64 x 256 17.2; 3584 of K 8192 at 100 rows fp4 15.3,
// in those over 4 splits 17.4). K advances a block of S instruction steps of 128 at a
// time:
//   * X's codes and scales of block b + 1 go from global memory straight to the
//     other of two LDS stages while block b is multiplied; one barrier per block. A
//     load takes 8 rows of a 128-byte line; loads laid out as the operand itself, 16
//     rows of half a line, cost 10 to 25% more time (256 x 8192 x 3584 fp8 13.5 against
//     11.3 us). In LDS the line's 16-byte chunks are swapped by row, so that neither
//     these writes nor the operand reads meet a bank twice;
//   * the weights, as they are tiled the operand itself, go straight to registers:
//     a step's records are loaded again, for the next block, as soon as its
//     instructions are issued. No two waves share a record (2 x 4 waves that shared
//     them and halved the rows took 196 us where 1 x 8 take 170).
// 8 waves (two per SIMD) with 128 x 512 outputs run 2048 x 14336 x 8192 in 163 to 178
// us fp8 (2.7 to 2.95 PFLOP/s, a loop of these instructions alone 4.4) and 106 to 114
// us fp4 (8.1): the matrix pipe is busy 66 and 57% of the clocks at 1.9 GHz. Of the rest an
// eighth of the machine is idle in the second round (448 tiles on 256 CUs), and most is
// the operands' loads: without X's, the weights' or both (timing only) fp8 took 161, 149
// and 138 us, without the block's barrier 163, as with it. A barrier in the middle of the
// block with three stages (171 and 113 us where this took 165 and 106) and operands
// read two or three row tiles ahead (no change) were not faster. Smaller tiles fill
// the CUs at fewer rows (plan_mx).
#include <algorithm>

#include "mx_common.h"

namespace tpdq {
namespace {

template <int DT, int FMT, int RT, int NP, int NW, int KG, int S, bool GATED, bool QUANT>
__global__ __launch_bounds__(NW * KG * 64) __attribute__((amdgpu_waves_per_eu(2))) void k_mx_tiles(MxArgs a) {
  static_assert(!GATED || NP == 2, "a tile of the gate and one of the up projection");
  constexpr int NT = 2 * NP;  // operands per wave
  constexpr int XW = FMT == kFp4 ? 1 : 2;      // 64-byte halves of a row's line per step
  constexpr int REC = S * XW;                  // code records (1 KB) of a row tile per block
  constexpr int BM = 16 * RT;
  static_assert(BM % 64 == 0 && (RT * REC) % NW == 0 && (S == 2 || S == 4), "whole records, evenly over the waves");
  constexpr int XREC = RT * REC / NW;     // ... per wave and block
  constexpr int SREC = BM / 16;                // scale records (256 B, a chunk's of 16 rows)
  constexpr int SPW = SREC > NW ? SREC / NW : 1;  // ... per wave (the same twice where there are more waves)
  constexpr int XBYTES = BM * REC * 64;
  constexpr int STAGE = XBYTES + SREC * 256;
  constexpr int ITEMS = XREC + SPW;              // loads to LDS per wave and block
  static_assert(RT % KG == 0, "a wave finishes whole row tiles");
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & 63;
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = KG > 1 ? wave_all / NW : 0;  // the wave's group, with LDS stages of its own
  const int wave = wave_all - kg * NW;
  unsigned char* const stages = smem + kg * 2 * STAGE;
  const int r16 = lane & 15, g = lane >> 4;
  const int nbm = (a.M + BM - 1) / BM;
  const int ks = a.ks;
  const int ntl = (int)(gridDim.x / ks);  // output tiles; neighbours take one split's X
  const int lt = xcd_run(blockIdx.x, gridDim.x);
  const int kidx = lt / ntl;
  const int tl = lt - kidx * ntl;
  // neighbours: 8 row tiles, then the next columns, so that an XCD's 32 workgroups
  // read 8 tiles of X and 4 of W (2048 x 14336 x 8192 fp8 168 -> 165 us)
  const int group = tl / (8 * (ntl / nbm)), in_group = tl - group * 8 * (ntl / nbm);
  const int group_rows = min(8, nbm - group * 8);
  const int bn = in_group / group_rows;
  const int row0 = (group * 8 + in_group - bn * group_rows) * BM;
  const int T0 = (GATED ? 1 : NP) * (NW * bn + wave);  // the wave's first 32-output tile
  const int steps = (a.K + kMxStep - 1) / kMxStep;
  const int chunks = (a.K + kMxChunk - 1) / kMxChunk;
  const int tiles = (a.N + kMxTile - 1) / kMxTile;
  const int nblk_all = (steps + S - 1) / S;
  const int wg0 = (int)((int64_t)nblk_all * kidx / ks);  // this workgroup's blocks
  const int wg1 = (int)((int64_t)nblk_all * (kidx + 1) / ks);
  // and the group's; all groups go through as many, the last one's past its end being zeros
  const int per_group = (wg1 - wg0 + KG - 1) / KG;
  const int kb0 = wg0 + kg * per_group, kb1 = kb0 + per_group;
  const int nblk = min(wg1, kb1);

  // Rows past M and tiles past the last one load zeros from the resource bounds
  // (an offset that stays out of range whatever block is added to it); steps past
  // the last one through an empty resource.
  const uint32_t xbytes = (uint32_t)(a.M - 1) * (uint32_t)a.x.ld_c + (uint32_t)steps * (64u * XW);
  const uint32_t xsbytes = (uint32_t)(a.M - 1) * (uint32_t)a.x.ld_s + (uint32_t)chunks * 16u;
  const uint32_t wbytes = (uint32_t)(tiles - 1) * (uint32_t)a.ldwc + (uint32_t)steps * 2048u;
  const uint32_t wsbytes = (uint32_t)(tiles - 1) * (uint32_t)a.ldws + (uint32_t)chunks * 512u;
  uint32_t offx[XREC], offw[NP], offws[NP];
#pragma unroll
  for (int k = 0; k < XREC; ++k) {
    // record = (row tile, 128-byte line, half of the rows): 8 rows of one line
    const int rec = XREC * wave + k, rt = rec / REC, line = rec % REC / 2, hr = rec & 1;
    const int m = row0 + 16 * rt + 8 * hr + (lane >> 3);
    const uint32_t chunk = (uint32_t)((lane & 7) ^ (lane >> 3));
    offx[k] = m < a.M ? (uint32_t)m * (uint32_t)a.x.ld_c + 128u * line + 16u * chunk : kOutOfRange;
  }
  // scale record in LDS: [word of the chunk][row], so that 16 rows' words are adjacent
  uint32_t offxs[SPW];
#pragma unroll
  for (int k = 0; k < SPW; ++k) {
    const int ms = row0 + 16 * ((wave + NW * k) % SREC) + r16;
    offxs[k] = ms < a.M ? (uint32_t)ms * (uint32_t)a.x.ld_s + 4u * g : kOutOfRange;
  }
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int T = GATED ? T0 : T0 + p;
    offw[p] = T < tiles ? (uint32_t)T * (uint32_t)a.ldwc + 16u * lane : kOutOfRange;
    offws[p] = T < tiles ? (uint32_t)T * (uint32_t)a.ldws + 8u * lane : kOutOfRange;
  }

  // All loads are unconditional and their conditions selects: a branch inside the
  // block would let the compiler move the matrix instructions past it.
  auto dma_item = [&](int b, int st, int k) {
    unsigned char* sb = stages + st * STAGE;
    if (k < XREC) {
      const int line = (XREC * wave + k) % REC / 2;
      const bool in = (b < nblk) & (S * b + 2 * line / XW < steps);
      const __amdgpu_buffer_rsrc_t r = buffer_rsrc(a.x.codes, in ? xbytes : 0u);
      dma_lds<16>(r, sb + (XREC * wave + k) * 1024, offx[k], in ? 64u * REC * (uint32_t)b : 0u);
    } else {
      const bool in = b < nblk;
      const __amdgpu_buffer_rsrc_t r = buffer_rsrc(a.x.scales, in ? xsbytes : 0u);
      dma_lds<4>(r, sb + XBYTES + ((wave + NW * (k - XREC)) % SREC) * 256, offxs[k - XREC], in ? ((uint32_t)(S * b) & ~3u) * 4u : 0u);
    }
  };
  auto load_w = [&](int b, int s, int i) {
    const bool in = (b < nblk) & (S * b + s < steps);
    const __amdgpu_buffer_rsrc_t r = buffer_rsrc(GATED && i >= 2 ? a.wc_up : a.wc, in ? wbytes : 0u);
    return __builtin_bit_cast(u4_t, __builtin_amdgcn_raw_buffer_load_b128(
        r, offw[i >> 1] + 1024u * (i & 1), in ? (uint32_t)(S * b + s) * 2048u : 0u, 0));
  };
  // scale words of both operands of tile p: a byte for each step of the block's chunk
  auto load_ws = [&](int b, int p) {
    const bool in = b < nblk;
    const __amdgpu_buffer_rsrc_t r = buffer_rsrc(GATED && p ? a.ws_up : a.ws, in ? wsbytes : 0u);
    return __builtin_bit_cast(u2_t, __builtin_amdgcn_raw_buffer_load_b64(
        r, offws[p], in ? ((uint32_t)(S * b) & ~3u) * 128u : 0u, 0));
  };

  // A 16-row tile's line in LDS: rows 128 bytes apart, the 16-byte chunk c of row r
  // at place c ^ (r % 8), so that 8 rows of one chunk fill a 128-byte cycle. Lane
  // (r, g) reads chunk g (first half of the line) or 4 + g.
  const int xpos0 = r16 * 128 + ((g ^ (r16 & 7)) << 4), xpos1 = xpos0 ^ 64;

  f4_t acc[RT][NT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[r][i] = f4_t{0.f, 0.f, 0.f, 0.f};
  u4_t w[S][NT];
  u2_t ws[NP], wsn[NP];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) dma_item(kb0, 0, k);
#pragma unroll
  for (int p = 0; p < NP; ++p) wsn[p] = load_ws(kb0, p);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      w[s][i] = load_w(kb0, s, i);
      __builtin_amdgcn_sched_barrier(0);
    }

  int st = 0;
#pragma unroll 1
  for (int b = kb0; b < kb1; ++b) {
    // this wave's LDS loads of block b (and its scale words) have landed, the
    // weight loads issued after them may be in flight; the barrier publishes
    // every wave's and frees the other stage
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::"n"(NT * S) : "memory");
    const unsigned char* xb = stages + st * STAGE;
    const unsigned char* sb = stages + st * STAGE + XBYTES + r16 * 4 + g + (S == 2 ? 128 * (b & 1) : 0);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      ws[p] = wsn[p];
      if (S == 2) ws[p] = ws[p] >> (16u * (b & 1));
    }
    static_assert(RT % 2 == 0, "the operand's two places alternate");
    // X's operand of row tile r and step s, read one row tile ahead of its use
    i8_t x[2];
    uint32_t xs[2];
    auto read_x = [&](int s, int r, int to) {
      const unsigned char* xl = xb + (r * (REC / 2) + s * XW / 2) * 2048;
      const u4_t lo = *(const u4_t*)(xl + (XW == 1 && s % 2 ? xpos1 : xpos0));
      u4_t hi = {0u, 0u, 0u, 0u};
      if constexpr (XW == 2) hi = *(const u4_t*)(xl + xpos1);
      x[to] = i8_t{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
      xs[to] = sb[r * 256 + s * 64];
    };
    read_x(0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    auto step = [&](auto sel) {
      constexpr int s = decltype(sel)::value;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        if (r + 1 < RT) read_x(s, r + 1, (r + 1) & 1);
        else if (s + 1 < S) read_x(s + 1, 0, 0);
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[r][i] = mfma_mx<FMT, s>(w[s][i], ws[i >> 1][i & 1], x[r & 1], xs[r & 1], acc[r][i]);
        if constexpr (s == 0) {  // the next block's loads to LDS, spread over the first step
#pragma unroll
          for (int k = r * ITEMS / RT; k < (r + 1) * ITEMS / RT; ++k) dma_item(b + 1, st ^ 1, k);
          if (r == RT - 1) {
#pragma unroll
            for (int p = 0; p < NP; ++p) wsn[p] = load_ws(b + 1, p);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        w[s][i] = load_w(b + 1, s, i);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    if constexpr (S >= 4) {
      step(std::integral_constant<int, 2>{});
      step(std::integral_constant<int, 3>{});
    }
    st ^= 1;
  }
  // the loads past the last block (zeros) still write LDS: let them land
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  // Groups: the sums of row tile r go through LDS, added in the groups' order by group r % KG
  f4_t* red = (f4_t*)smem;  // [group][wave][RT * NT][64]
  if constexpr (KG > 1) {
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < NT; ++i) red[((kg * NW + wave) * RT * NT + r * NT + i) * 64 + lane] = acc[r][i];
    __syncthreads();
  }
#pragma unroll
  for (int q = 0; q < RT / KG; ++q) {
    const int r = q * KG + kg;
    const int m = row0 + r * 16 + r16;
    f4_t y[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      if constexpr (KG == 1) {
        y[i] = acc[q][i];
      } else {
        const f4_t* p = red + (wave * RT * NT + r * NT + i) * 64 + lane;
        y[i] = p[0];
#pragma unroll
        for (int k = 1; k < KG; ++k) y[i] += p[k * NW * RT * NT * 64];
      }
    }
    if (ks > 1) {  // this split's part, [split][(gate, up)][M][N]
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int64_t n = (int64_t)(GATED ? T0 : T0 + p) * kMxTile + 8 * g;
        float* part = a.part + ((int64_t)(GATED ? 2 * kidx + p : kidx) * a.M + m) * a.N + n;
        if (m < a.M && n < a.N) {
          *(f4_t*)part = y[2 * p];
          *(f4_t*)(part + 4) = y[2 * p + 1];
        }
      }
      continue;
    }
#pragma unroll
    for (int p = 0; p < (GATED ? 1 : NP); ++p) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float o = y[2 * p + (e >> 2)][e & 3];
        v[e] = GATED ? silu_mul(o, y[2 + (e >> 2)][e & 3]) : o;
      }
      store_out8<DT, FMT, QUANT>(a, v, m, (int64_t)(T0 + p) * kMxTile + 8 * g);
    }
  }
}

// Adds the splits' parts in their order and finishes the outputs: 8 of a row per
// thread, a block of 32 in four lanes. QUANT: rows padded to whole chunks.
template <int DT, int FMT, bool GATED, bool QUANT>
__global__ __launch_bounds__(256) void k_mx_reduce(MxArgs a, int64_t octets, int per_row) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= octets) return;  // QUANT: whole waves
  const int64_t m = i / per_row;
  const int k8 = (int)(i - m * per_row);
  float v[GATED ? 2 : 1][8];
#pragma unroll
  for (int h = 0; h < (GATED ? 2 : 1); ++h) {
    f4_t lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
    if (8 * k8 < a.N) {
      const float* p = a.part + ((int64_t)h * a.M + m) * a.N + 8 * k8;
      const int64_t split = (int64_t)(GATED ? 2 : 1) * a.M * a.N;
      for (int k = 0; k < a.ks; ++k) {
        lo += *(const f4_t*)(p + k * split);
        hi += *(const f4_t*)(p + k * split + 4);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[h][e] = lo[e];
      v[h][4 + e] = hi[e];
    }
  }
  if constexpr (GATED) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[0][e] = silu_mul(v[0][e], v[1][e]);
  }
  if constexpr (QUANT)
    store_mx8<FMT>(v[0], k8, 16 * ((a.N + kMxStep - 1) / kMxStep), a.q.codes + m * a.q.ld_c, a.q.scales + m * a.q.ld_s);
  else
    *(u4_t*)(a.Y + m * a.ldy + 8 * k8) = pack8<DT>(v[0]);
}

template <int DT, int FMT, int RT, int NP, int NW, int KG, int S, bool GATED, bool QUANT>
hipError_t tiles_launch(const MxArgs& a, hipStream_t s) {
  constexpr int BM = 16 * RT;
  constexpr int stages = KG * 2 * BM * (S * (FMT == kFp4 ? 64 : 128) + 16), red = KG > 1 ? KG * NW * RT * 2 * NP * 1024 : 0;
  constexpr int lds = stages > red ? stages : red;
  static_assert((size_t)lds <= kLdsMax, "");
  auto* k = k_mx_tiles<DT, FMT, RT, NP, NW, KG, S, GATED, QUANT>;
  static std::atomic<uint64_t> done{0};
  hipError_t e = allow_lds((const void*)k, lds, &done);
  if (e != hipSuccess) return e;
  const int tiles = (int)(QUANT && a.ks == 1 ? mx_chunks(a.N) * (kMxChunk / kMxTile) : (a.N + kMxTile - 1) / kMxTile);
  const int per = (GATED ? 1 : NP) * NW;
  const int64_t grid = (int64_t)((a.M + BM - 1) / BM) * ((tiles + per - 1) / per) * a.ks;
  k<<<dim3((unsigned)grid), dim3(NW * KG * 64), lds, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess || a.ks == 1) return e;
  const int per_row = QUANT ? (int)(mx_chunks(a.N) * 64) : a.N / 8;
  const int64_t n = (int64_t)a.M * per_row;
  k_mx_reduce<DT, FMT, GATED, QUANT><<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s>>>(a, n, per_row);
  return hipGetLastError();
}

template <int DT, int FMT, bool GATED, bool QUANT>
hipError_t tiles_pick(const MxArgs& a, int kind, hipStream_t s) {
  constexpr int S2 = FMT == kFp4 ? 4 : 2;  // fp8, 128 rows: registers for two steps
  switch (kind) {
    case kMxTiles128x512: return tiles_launch<DT, FMT, 8, 2, 8, 1, S2, GATED, QUANT>(a, s);
    case kMxTiles64x512: return tiles_launch<DT, FMT, 4, 2, 8, 1, 4, GATED, QUANT>(a, s);
    case kMxTiles64x256: return tiles_launch<DT, FMT, 4, 2, 4, 1, 4, GATED, QUANT>(a, s);
    case kMxTiles128x256: return tiles_launch<DT, FMT, 8, 2, 4, 1, S2, GATED, QUANT>(a, s);
    // two groups of waves; of the gated product 64 outputs as well
    case GATED ? kMxTiles64x128 : kMxTiles64x64: return tiles_launch<DT, FMT, 4, GATED ? 2 : 1, 2, 2, 4, GATED, QUANT>(a, s);
  }
  if constexpr (!GATED)
    if (kind == kMxTiles64x128) return tiles_launch<DT, FMT, 4, 1, 4, 1, 4, GATED, QUANT>(a, s);
  return hipErrorInvalidValue;
}

// Outputs in 16 bits, or quantized (the gated product always is: the MLP's first
// half), which no element type enters.
template <int FMT>
hipError_t tiles_of(const MxArgs& a, int kind, int dt, hipStream_t s) {
  if (a.wc_up) return tiles_pick<kF16, FMT, true, true>(a, kind, s);
  if (!a.Y) return tiles_pick<kF16, FMT, false, true>(a, kind, s);
  return dt == TPDQ_BF16 ? tiles_pick<kBF16, FMT, false, false>(a, kind, s) : tiles_pick<kF16, FMT, false, false>(a, kind, s);
}

}  // namespace

hipError_t launch_mx_tiles(const MxArgs& a, int kind, int dt, int fmt, hipStream_t s) {
  return fmt == TPDQ_MX_FP4 ? tiles_of<kFp4>(a, kind, dt, s) : tiles_of<kFp8>(a, kind, dt, s);
}

}  // namespace tpdq
