// Product of microscaled (MX) operands with many rows of X on gfx950: the matrix
// pipe bounds it (mx_gemm.hip has the few-row kernel and the operands' layout).
//
// A workgroup of 8 waves (two per SIMD) computes 32 RT rows x 256 outputs (GATED:
// 128 of the gate and 128 of the up projection); a wave half of the rows and 64 of
// the outputs, RT x 4 accumulators. K advances a block of 256 bytes of X at a time
// (fp8 two instruction steps, fp4 four):
//   * X's codes and scales of block b + 1 go from global memory straight to the
//     other of two LDS stages, laid out as the instruction's operand, while block b
//     is multiplied; one barrier per block;
//   * the weights, as they are tiled the operand itself, go straight to registers:
//     a step's records are loaded again, for the next block, as soon as its
//     instructions are issued. Only two waves share a record, and through LDS it
//     would take a quarter of the LDS reads that bound the loop next.
#include <algorithm>

#include "mx_common.h"

namespace tpdq {
namespace {

// Consecutive tiles on one XCD (round-robin dispatch), whatever their number.
__device__ __forceinline__ int xcd_run(int b, int nb) {
  const int x = b & 7, q = nb >> 3, rem = nb & 7;
  return x * q + min(x, rem) + (b >> 3);
}

template <int BYTES>
__device__ __forceinline__ void dma_lds(__amdgpu_buffer_rsrc_t r, void* dst, uint32_t off, uint32_t soff) {
  if constexpr (BYTES == 16)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)dst, 16, off, soff, 0, 0);
  else
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)dst, 4, off, soff, 0, 0);
}

template <int DT, int FMT, int RT, bool GATED, bool QUANT>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void k_mx_tiles(MxArgs a) {
  constexpr int S = FMT == kFp4 ? 4 : 2;       // steps per block
  constexpr int XW = FMT == kFp4 ? 1 : 2;      // records of a row tile per step
  constexpr int BM = 32 * RT;
  constexpr int XREC = RT;                     // code records (1 KB) per wave and block
  constexpr int SREC = S * BM / 64;            // scale records (256 B) per block
  constexpr int SPW = (SREC + 7) / 8;          // ... per wave (some twice)
  constexpr int STAGE = BM * 256 + SREC * 256;
  constexpr int ITEMS = XREC + SPW;            // loads to LDS per wave and block
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const int r16 = lane & 15, g = lane >> 4;
  const int nbm = (a.M + BM - 1) / BM;
  const int tl = xcd_run(blockIdx.x, gridDim.x);
  const int bn = tl / nbm;
  const int row0 = (tl - bn * nbm) * BM;
  const int T0 = GATED ? 4 * bn + wn : 8 * bn + 2 * wn;  // the wave's first 32-output tile
  const int steps = (a.K + kMxStep - 1) / kMxStep;
  const int chunks = (a.K + kMxChunk - 1) / kMxChunk;
  const int tiles = (a.N + kMxTile - 1) / kMxTile;
  const int nblk = (steps + S - 1) / S;

  // Rows past M and tiles past the last one load zeros from the resource bounds
  // (an offset that stays out of range whatever block is added to it); steps past
  // the last one through an empty resource.
  const uint32_t xbytes = (uint32_t)(a.M - 1) * (uint32_t)a.x.ld_c + (uint32_t)steps * (64u * XW);
  const uint32_t xsbytes = (uint32_t)(a.M - 1) * (uint32_t)a.x.ld_s + (uint32_t)chunks * 16u;
  const uint32_t wbytes = (uint32_t)(tiles - 1) * (uint32_t)a.ldwc + (uint32_t)steps * 2048u;
  const uint32_t wsbytes = (uint32_t)(tiles - 1) * (uint32_t)a.ldws + (uint32_t)chunks * 512u;
  uint32_t offx[XREC], offxs[SPW], offw[2], offws[2];
#pragma unroll
  for (int k = 0; k < XREC; ++k) {
    // record = (row tile, step, half): lane (r, g) has 16 bytes of row r
    const int rec = XREC * wave + k, rt = rec >> 2, sh = rec & 3;
    const int m = row0 + 16 * rt + r16;
    offx[k] = m < a.M ? (uint32_t)m * (uint32_t)a.x.ld_c + 64u * sh + 16u * g : kOutOfRange;
  }
#pragma unroll
  for (int k = 0; k < SPW; ++k) {
    const int rec = (wave + 8 * k) % SREC, s = rec / (BM / 64), mb = rec % (BM / 64);
    const int m = row0 + 64 * mb + lane;
    offxs[k] = m < a.M ? (uint32_t)m * (uint32_t)a.x.ld_s + 4u * s : kOutOfRange;
  }
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int T = GATED ? T0 : T0 + p;
    offw[p] = T < tiles ? (uint32_t)T * (uint32_t)a.ldwc + 16u * lane : kOutOfRange;
    offws[p] = T < tiles ? (uint32_t)T * (uint32_t)a.ldws + 8u * lane : kOutOfRange;
  }

  auto dma_item = [&](int b, int st, int k) {
    unsigned char* sb = smem + st * STAGE;
    if (k < XREC) {
      const int sh = (XREC * wave + k) & 3;
      const bool in = b < nblk && S * b + sh / XW < steps;
      const __amdgpu_buffer_rsrc_t r = buffer_rsrc(a.x.codes, in ? xbytes : 0u);
      dma_lds<16>(r, sb + (XREC * wave + k) * 1024, offx[k], in ? 256u * (uint32_t)b : 0u);
    } else {
      const int rec = (wave + 8 * (k - XREC)) % SREC;
      const bool in = b < nblk;
      const __amdgpu_buffer_rsrc_t r = buffer_rsrc(a.x.scales, in ? xsbytes : 0u);
      dma_lds<4>(r, sb + BM * 256 + rec * 256, offxs[k - XREC], in ? (uint32_t)(4 * S) * (uint32_t)b : 0u);
    }
  };
  auto load_w = [&](int b, int s, int i) {
    const bool in = b < nblk && S * b + s < steps;
    const __amdgpu_buffer_rsrc_t r = buffer_rsrc(GATED && i >= 2 ? a.wc_up : a.wc, in ? wbytes : 0u);
    return __builtin_bit_cast(u4_t, __builtin_amdgcn_raw_buffer_load_b128(
        r, offw[i >> 1] + 1024u * (i & 1), in ? (uint32_t)(S * b + s) * 2048u : 0u, 0));
  };
  // scale words of both operands of tile p: bytes of the chunk's steps, the block's
  // steps lowest
  auto load_ws = [&](int b, int p) {
    const bool in = b < nblk;
    const __amdgpu_buffer_rsrc_t r = buffer_rsrc(GATED && p ? a.ws_up : a.ws, in ? wsbytes : 0u);
    return __builtin_bit_cast(u2_t, __builtin_amdgcn_raw_buffer_load_b64(
        r, offws[p], in ? (uint32_t)(S * b / 4) * 512u : 0u, 0));
  };

  f4_t acc[RT][4];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[r][i] = f4_t{0.f, 0.f, 0.f, 0.f};
  u4_t w[S][4];
  u2_t ws[2], wsn[2];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) dma_item(0, 0, k);
#pragma unroll
  for (int p = 0; p < 2; ++p) wsn[p] = load_ws(0, p);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[s][i] = load_w(0, s, i);
      __builtin_amdgcn_sched_barrier(0);
    }

  int st = 0;
#pragma unroll 1
  for (int b = 0; b < nblk; ++b) {
    // this wave's LDS loads of block b (and its scale words) have landed, the
    // weight loads issued after them may be in flight; the barrier publishes
    // every wave's and frees the other stage
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::"n"(4 * S) : "memory");
    const unsigned char* xb = smem + st * STAGE + (wm * RT) * 4096;
    const unsigned char* sb = smem + st * STAGE + BM * 256 + (wm * RT * 16 + r16) * 4 + g;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      ws[p] = wsn[p];
      if (S == 2 && (b & 1)) ws[p] = ws[p] >> 16;
    }
    auto step = [&](auto sel) {
      constexpr int s = decltype(sel)::value;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const u4_t lo = *(const u4_t*)(xb + (r * 4 + s * XW) * 1024 + lane * 16);
        u4_t hi = {0u, 0u, 0u, 0u};
        if constexpr (XW == 2) hi = *(const u4_t*)(xb + (r * 4 + s * XW + 1) * 1024 + lane * 16);
        const i8_t x = {(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        const uint32_t xs = sb[(s * BM + r * 16) * 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[r][i] = mfma_mx<FMT, s>(w[s][i], ws[i >> 1][i & 1], x, xs, acc[r][i]);
        if constexpr (s == 0) {  // the next block's loads to LDS, spread over the first step
#pragma unroll
          for (int k = r * ITEMS / RT; k < (r + 1) * ITEMS / RT; ++k) dma_item(b + 1, st ^ 1, k);
          if (r == RT - 1) {
            wsn[0] = load_ws(b + 1, 0);
            wsn[1] = load_ws(b + 1, 1);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[s][i] = load_w(b + 1, s, i);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    if constexpr (S == 4) {
      step(std::integral_constant<int, 2>{});
      step(std::integral_constant<int, 3>{});
    }
    st ^= 1;
  }
  // the loads past the last block (zeros) still write LDS: let them land
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int m = row0 + (wm * RT + r) * 16 + r16;
#pragma unroll
    for (int p = 0; p < (GATED ? 1 : 2); ++p) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = acc[r][2 * p + (e >> 2)][e & 3];
        v[e] = GATED ? silu_mul(y, acc[r][2 + (e >> 2)][e & 3]) : y;
      }
      store_out8<DT, FMT, QUANT>(a, v, m, (int64_t)(T0 + p) * kMxTile + 8 * g);
    }
  }
}

template <int DT, int FMT, int RT, bool GATED, bool QUANT>
hipError_t tiles_launch(const MxArgs& a, hipStream_t s) {
  constexpr int S = FMT == kFp4 ? 4 : 2, BM = 32 * RT;
  constexpr int lds = 2 * (BM * 256 + S * BM * 4);
  auto* k = k_mx_tiles<DT, FMT, RT, GATED, QUANT>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  const int tiles = (int)(QUANT ? mx_chunks(a.N) * (kMxChunk / kMxTile) : (a.N + kMxTile - 1) / kMxTile);
  const int per = GATED ? 4 : 8;
  const int64_t grid = (int64_t)((a.M + BM - 1) / BM) * ((tiles + per - 1) / per);
  k<<<dim3((unsigned)grid), dim3(512), lds, s>>>(a);
  return hipGetLastError();
}

template <int DT, int FMT, bool GATED, bool QUANT>
hipError_t tiles_pick(const MxArgs& a, hipStream_t s) {
  if (a.M > 128) return tiles_launch<DT, FMT, 8, GATED, QUANT>(a, s);
  return tiles_launch<DT, FMT, 4, GATED, QUANT>(a, s);
}

template <int DT, int FMT>
hipError_t tiles_of(const MxArgs& a, hipStream_t s) {
  const bool quant = a.Y == nullptr;
  if (a.wc_up) return quant ? tiles_pick<DT, FMT, true, true>(a, s) : tiles_pick<DT, FMT, true, false>(a, s);
  return quant ? tiles_pick<DT, FMT, false, true>(a, s) : tiles_pick<DT, FMT, false, false>(a, s);
}

}  // namespace

hipError_t launch_mx_tiles(const MxArgs& a, int dt, int fmt, hipStream_t s) {
  if (dt == TPDQ_BF16) return fmt == TPDQ_MX_FP4 ? tiles_of<kBF16, kFp4>(a, s) : tiles_of<kBF16, kFp8>(a, s);
  return fmt == TPDQ_MX_FP4 ? tiles_of<kF16, kFp4>(a, s) : tiles_of<kF16, kFp8>(a, s);
}

}  // namespace tpdq
