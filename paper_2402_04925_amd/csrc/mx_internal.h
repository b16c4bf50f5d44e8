// Internal declarations of the microscaled (MX) operators: launch descriptions
// shared by mx_abi.hip (validation, dispatch), mx_rows.hip (row-wise kernels)
// and the product's kernels.
#pragma once

#include <atomic>

#include "tpdq_internal.h"

namespace tpdq {

// abi.hip: sets tpdq_last_error() and returns st
tpdq_status fail(tpdq_status st, const char* fmt, ...);
tpdq_status hip_fail(hipError_t e, const char* what);

// Elements per scale; elements of one matrix instruction's K step; of the run of
// steps whose scales one 32-bit word per lane holds.
constexpr int kMxBlock = 32;
constexpr int kMxStep = 128;
constexpr int kMxChunk = 512;
constexpr int kMxTile = 32;  // weight rows (outputs) of a tile: two 16-row operands

inline int64_t mx_steps(int64_t K) { return (K + kMxStep - 1) / kMxStep; }
inline int64_t mx_chunks(int64_t K) { return (K + kMxChunk - 1) / kMxChunk; }
// bytes of one row's codes and scales (TPDQ_MX_ROWS), padding included
inline int64_t mx_row_codes(int64_t K, int fmt) { return mx_steps(K) * (fmt == TPDQ_MX_FP4 ? 64 : 128); }
inline int64_t mx_row_scales(int64_t K) { return mx_chunks(K) * 16; }
// bytes of one 32-row tile's codes and scales (TPDQ_MX_TILED)
inline int64_t mx_tile_codes(int64_t K) { return mx_steps(K) * 2048; }
inline int64_t mx_tile_scales(int64_t K) { return mx_chunks(K) * 512; }

// Lets kernel f use `bytes` of LDS where that is more than the default: once for a
// kernel (each has its own `done`) and device. A launch of a few microseconds would
// feel it on every call.
hipError_t allow_lds(const void* f, int bytes, std::atomic<uint64_t>* done);

struct MxRows {  // a TPDQ_MX_ROWS tensor
  uint8_t* codes;
  int64_t ld_c;
  uint8_t* scales;
  int64_t ld_s;
};

hipError_t launch_mx_quantize(const uint16_t* X, int64_t ldx, int R, int K, int dt, int fmt, const MxRows& q,
                              hipStream_t s);
hipError_t launch_mx_dequantize(const MxRows& q, int R, int K, int dt, int fmt, uint16_t* X, int64_t ldx,
                                hipStream_t s);
hipError_t launch_mx_pack(const MxRows& q, int R, int K, uint8_t* codes, int64_t ld_c, uint8_t* scales,
                          int64_t ld_s, hipStream_t s);

// Columns of a row that k_rmsnorm holds in a workgroup's registers
constexpr int kNormMaxK = 65536;
// Threads of a row's workgroup: one octet each as far as 1024 reach, then up to eight
inline int norm_threads(int K, int fmt, int* octets_per_thread) {
  const int octets = fmt < 0 ? K / 8 : (int)(mx_chunks(K) * 64);
  const int waves = octets > 15 * 64 ? 16 : (octets + 63) / 64;
  *octets_per_thread = (octets + 64 * waves - 1) / (64 * waves);
  return 64 * waves;
}
struct NormArgs {
  const uint16_t* X;
  int64_t ldx;
  const uint16_t* res;  // or NULL
  int64_t ldr;
  const uint16_t* w;
  uint16_t* h;  // X + res in 16 bits, or NULL
  int64_t ldh;
  uint16_t* Y;  // 16-bit output, or NULL with q
  int64_t ldy;
  MxRows q;
  int M, K;
  float eps;
};
hipError_t launch_rmsnorm(const NormArgs& a, int dt, int fmt, hipStream_t s);  // fmt < 0: 16 bits

// One product Y = X W^T (device pointers).
struct MxArgs {
  MxRows x;            // [M][K], fp8 or fp4
  const uint8_t* wc;   // TPDQ_MX_TILED, fp4: [ceil(N/32)][ldwc]
  const uint8_t* ws;
  const uint8_t* wc_up;  // gated: the up projection, with the same leading dimensions
  const uint8_t* ws_up;
  int64_t ldwc, ldws;
  int M, N, K;
  uint16_t* Y;  // 16-bit output [M][ldy], or NULL with q
  int64_t ldy;
  MxRows q;     // output in X's format
  float* part;  // ks > 1: [ks][(gate, up)][M][N]
  int ks;       // K splits (tiles kernel)
};
// How a product runs: the few-row kernel over whole or half tiles of 32 outputs, or
// tiles of rows x weight rows (gated: half of them of each projection) with K split
// over ks workgroups (fp32 parts, added in the splits' order by a second kernel).
enum MxKind { kMxRows, kMxRowsHalf, kMxTiles128x512, kMxTiles64x512, kMxTiles64x256, kMxTiles128x256, kMxTiles64x128, kMxTiles64x64 };
struct MxPlan {
  int kind, ks;
};
MxPlan plan_mx(int M, int N, int K, int fmt, bool gated, bool quant);
size_t mx_part_bytes(const MxPlan& p, int M, int N, bool gated);
// part: mx_part_bytes of the plan
hipError_t launch_mx_gemm(MxArgs a, int dt, int fmt, float* part, hipStream_t s);
hipError_t launch_mx_tiles(const MxArgs& a, int kind, int dt, int fmt, hipStream_t s);  // mx_tiles.hip

}  // namespace tpdq
