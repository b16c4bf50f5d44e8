// Product of microscaled (MX) operands on gfx950, Y = X W^T: X in fp8 (E4M3) or
// fp4 (E2M1) rows, W in fp4 tiles (mx_internal.h), both with one E8M0 scale per 32
// elements of K. The scaled matrix instruction takes the codes and the scales as
// they are stored, so nothing is dequantized: an output is one fp32 accumulator,
// rounded once.
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

// Few rows of X: the weight stream bounds it. A workgroup owns NP tiles of 32
// outputs (GATED: of the gate and the up projection) over the whole of K and MT
// tiles of 16 rows; its waves take chunks of 512 elements of K in turn, the
// weights of a chunk straight to registers (1 KB contiguous per load), and add
// their accumulators in LDS at the end.
template <int DT, int FMT, int MT, int NP, bool GATED, bool QUANT, int NWMAX>
__global__ __launch_bounds__(NWMAX * 64) void k_mx_rows(MxArgs a) {
  constexpr int P = GATED ? 2 : 1;
  constexpr int NT = NP * P * 2;  // operands (16 outputs) per workgroup
  constexpr int XW = FMT == kFp4 ? 1 : 2;  // 16-byte loads of X per step
  extern __shared__ __align__(16) unsigned char smem[];
  f4_t* red = (f4_t*)smem;  // [wave][MT * NT][64]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nw = blockDim.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int steps = (a.K + kMxStep - 1) / kMxStep;
  const int chunks = (a.K + kMxChunk - 1) / kMxChunk;
  const int tiles = (a.N + kMxTile - 1) / kMxTile;
  const int T0 = xcd_tile(blockIdx.x, gridDim.x) * NP;
  const int m0 = blockIdx.y * 16 * MT;

  // tiles past the last one and rows past M load zeros from the resource bounds
  const uint32_t wbytes = (uint32_t)(tiles - 1) * (uint32_t)a.ldwc + (uint32_t)steps * 2048u;
  const uint32_t sbytes = (uint32_t)(tiles - 1) * (uint32_t)a.ldws + (uint32_t)chunks * 512u;
  const uint32_t xbytes = (uint32_t)(a.M - 1) * (uint32_t)a.x.ld_c + (uint32_t)steps * (64u * XW);
  const uint32_t xsbytes = (uint32_t)(a.M - 1) * (uint32_t)a.x.ld_s + (uint32_t)chunks * 16u;
  const __amdgpu_buffer_rsrc_t rx = buffer_rsrc(a.x.codes, xbytes), rxs = buffer_rsrc(a.x.scales, xsbytes);
  uint32_t offx[MT], offxs[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = m0 + 16 * t + r;
    offx[t] = m < a.M ? (uint32_t)m * (uint32_t)a.x.ld_c + 16u * g : kOutOfRange;
    offxs[t] = m < a.M ? (uint32_t)m * (uint32_t)a.x.ld_s : kOutOfRange;
  }
  uint32_t offw[NP], offs[NP];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    offw[p] = T0 + p < tiles ? (uint32_t)(T0 + p) * (uint32_t)a.ldwc + 16u * lane : kOutOfRange;
    offs[p] = T0 + p < tiles ? (uint32_t)(T0 + p) * (uint32_t)a.ldws + 8u * lane : kOutOfRange;
  }

  f4_t acc[MT][NT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};

  for (int c = wave; c < chunks; c += nw) {
    u4_t w[NT][4];
    u2_t ws[NT / 2];
    u4_t xs[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) xs[t] = buffer_load16(rxs, offxs[t] + 16u * c);
#pragma unroll
    for (int h = 0; h < P; ++h) {
      const __amdgpu_buffer_rsrc_t rw = buffer_rsrc(h ? a.wc_up : a.wc, wbytes);
      const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(h ? a.ws_up : a.ws, sbytes);
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        ws[h * NP + p] = __builtin_bit_cast(u2_t, __builtin_amdgcn_raw_buffer_load_b64(rs, offs[p] + 512u * c, 0, 0));
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            w[(h * NP + p) * 2 + j][s] = buffer_load16<kNonTemporal>(
                rw, 4 * c + s < steps ? offw[p] + (uint32_t)(4 * c + s) * 2048u + 1024u * j : kOutOfRange);
      }
    }
    i8_t x[MT][4];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const bool in = 4 * c + s < steps;
        const uint32_t o = offx[t] + (uint32_t)(4 * c + s) * (64u * XW);
        const u4_t lo = buffer_load16(rx, in ? o : kOutOfRange);
        u4_t hi = {0u, 0u, 0u, 0u};
        if constexpr (XW == 2) hi = buffer_load16(rx, in ? o + 64u : kOutOfRange);
        x[t][s] = i8_t{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
      }
    auto step = [&](auto sel) {
      constexpr int s = decltype(sel)::value;
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const uint32_t xsc = xs[t][s] >> (8 * g);
#pragma unroll
        for (int i = 0; i < NT; ++i)
          acc[t][i] = mfma_mx<FMT, s>(w[i][s], ws[i >> 1][i & 1], x[t][s], xsc, acc[t][i]);
      }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
  }

  // acc of operand i of tile pair (h, p), j = i % 2, row tile t -> red
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
  for (int i = wave; i < MT * NP; i += nw) {
    const int t = i / NP, p = i - t * NP;
    float v[8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const f4_t y = red[(t * NT + 2 * p + j) * 64 + lane];
      f4_t u = y;
      if constexpr (GATED) u = red[(t * NT + 2 * (NP + p) + j) * 64 + lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * j + e] = GATED ? silu_mul(y[e], u[e]) : y[e];
    }
    store_out8<DT, FMT, QUANT>(a, v, m0 + 16 * t + r, (int64_t)(T0 + p) * kMxTile + 8 * g);
  }
}

template <int DT, int FMT, int MT, int NP, bool GATED, bool QUANT, int NWMAX>
hipError_t rows_launch(const MxArgs& a, hipStream_t s) {
  // quantized outputs: also the tiles of the padding to whole chunks (zeros)
  const int tiles = (int)(QUANT ? mx_chunks(a.N) * (kMxChunk / kMxTile) : (a.N + kMxTile - 1) / kMxTile);
  const int nw = (int)std::min<int64_t>(NWMAX, mx_chunks(a.K));
  const size_t lds = (size_t)nw * MT * NP * (GATED ? 4 : 2) * 1024;
  auto* k = k_mx_rows<DT, FMT, MT, NP, GATED, QUANT, NWMAX>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const int row_groups = (a.M + 16 * MT - 1) / (16 * MT);
  k<<<dim3((unsigned)((tiles + NP - 1) / NP), (unsigned)row_groups), dim3((unsigned)nw * 64), lds, s>>>(a);
  return hipGetLastError();
}

template <int DT, int FMT, bool GATED, bool QUANT>
hipError_t rows_pick(const MxArgs& a, hipStream_t s) {
  if (a.M <= 16) return rows_launch<DT, FMT, 1, 1, GATED, QUANT, 16>(a, s);
  if (a.M <= 32) return rows_launch<DT, FMT, 2, 1, GATED, QUANT, 8>(a, s);
  return rows_launch<DT, FMT, 4, 1, GATED, QUANT, 8>(a, s);
}

template <int FMT>
hipError_t rows_of(const MxArgs& a, int dt, hipStream_t s) {
  if (a.wc_up) return rows_pick<kF16, FMT, true, true>(a, s);
  if (!a.Y) return rows_pick<kF16, FMT, false, true>(a, s);
  return dt == TPDQ_BF16 ? rows_pick<kBF16, FMT, false, false>(a, s) : rows_pick<kF16, FMT, false, false>(a, s);
}

}  // namespace

MxPlan plan_mx(int M, int N, int K, int fmt, bool gated) {
  if (M <= 64) return MxPlan{0, 1};
  return MxPlan{M <= 128 ? 3 : 2, 1};
}

size_t mx_part_bytes(const MxPlan& p, int M, int N, bool gated) {
  return p.ks > 1 ? align_up((size_t)p.ks * M * N * (gated ? 8 : 4)) : 0;
}

hipError_t launch_mx_gemm(MxArgs a, int dt, int fmt, float* part, hipStream_t s) {
  const MxPlan p = plan_mx(a.M, a.N, a.K, fmt, a.wc_up != nullptr);
  a.ks = p.ks;
  a.part = part;
  if (p.bm) return launch_mx_tiles(a, p.bm, dt, fmt, s);
  return fmt == TPDQ_MX_FP4 ? rows_of<kFp4>(a, dt, s) : rows_of<kFp8>(a, dt, s);
}

}  // namespace tpdq
