// Row-wise kernels of the microscaled (MX) operators on gfx950: quantization to
// fp4 / fp8 with one scale per 32 elements, its inverse, the weights' storage
// order, and the root-mean-square norm that feeds a product.
//
// All of them are bound by memory: they read and write every element once (the
// norm keeps its row in registers between the sum and the output).
#include <algorithm>

#include "mx_common.h"

namespace tpdq {
namespace {

constexpr int kRowThreads = 256;

// A workgroup takes up to 256 octets of ROWS consecutive rows, an octet of each row
// per thread, all loads issued before the first is used; a block's four lanes share
// their maximum. Rows are padded to whole chunks of 512, so that a block's lanes are
// in one wave and the padding's codes and scales are written (zeros). seg: the
// row's workgroups.
template <int DT, int FMT, int ROWS>
__global__ __launch_bounds__(kRowThreads) void k_mx_quantize(const uint16_t* __restrict__ X, int64_t ldx, int R, int seg,
                                                             int per_row, int K, MxRows q) {
  const int rb = blockIdx.x / seg;
  const int k8 = (blockIdx.x - rb * seg) * blockDim.x + threadIdx.x;
  if (k8 >= per_row) return;  // whole waves
  const int64_t r0 = (int64_t)rb * ROWS;
  const int code_octets = 16 * ((K + kMxStep - 1) / kMxStep);
  u4_t x[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    x[i] = u4_t{0u, 0u, 0u, 0u};
    if (8 * k8 < K && r0 + i < R) x[i] = *(const u4_t*)(X + (r0 + i) * ldx + 8 * k8);
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    if (r0 + i >= R) break;
    float v[8];
    unpack8<DT>(x[i], v);
    store_mx8<FMT>(v, k8, code_octets, q.codes + (r0 + i) * q.ld_c, q.scales + (r0 + i) * q.ld_s);
  }
}

template <int FMT>
__device__ __forceinline__ void values8(u2_t w, uint32_t byte, float (&v)[8]) {
  // 2^(byte - 127); the smallest is subnormal
  const float s = byte == 255u ? __builtin_nanf("") : byte ? as_f32(byte << 23) : as_f32(0x00400000u);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float a;
    bool neg;
    if constexpr (FMT == kFp4) {
      const uint32_t c = (w.x >> (4 * e)) & 0xFu, m = c & 7u;
      // 0, 0.5, then (1 or 1.5) 2^(m / 2 - 1)
      a = m < 2u ? 0.5f * (float)m : as_f32(((126u + (m >> 1)) << 23) | ((m & 1u) << 22));
      neg = c & 8u;
    } else {
      const uint32_t c = (w[e >> 2] >> (8 * (e & 3))) & 0xFFu, m = c & 0x7Fu;
      // subnormal: m 2^-9; normal: the exponent's bias 7 against 127; NaN: 0x7F
      a = m < 8u ? (float)m * 0x1p-9f : as_f32((m << 20) + (120u << 23));
      if (m == 0x7Fu) a = __builtin_nanf("");
      neg = c & 0x80u;
    }
    v[e] = (neg ? -a : a) * s;
  }
}

template <int DT, int FMT, int ROWS>
__global__ __launch_bounds__(kRowThreads) void k_mx_dequantize(MxRows q, int R, int seg, int per_row,
                                                               uint16_t* __restrict__ X, int64_t ldx) {
  const int rb = blockIdx.x / seg;
  const int k8 = (blockIdx.x - rb * seg) * blockDim.x + threadIdx.x;
  if (k8 >= per_row) return;
  const int64_t r0 = (int64_t)rb * ROWS;
  u2_t w[ROWS];
  uint32_t byte[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    w[i] = u2_t{0u, 0u};
    byte[i] = 0u;
    if (r0 + i < R) {
      byte[i] = q.scales[(r0 + i) * q.ld_s + (k8 >> 2)];
      if constexpr (FMT == kFp4) w[i].x = *(const uint32_t*)(q.codes + (r0 + i) * q.ld_c + 4 * (int64_t)k8);
      else w[i] = *(const u2_t*)(q.codes + (r0 + i) * q.ld_c + 8 * (int64_t)k8);
    }
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    if (r0 + i >= R) break;
    float v[8];
    values8<FMT>(w[i], byte[i], v);
    *(u4_t*)(X + (r0 + i) * ldx + 8 * (int64_t)k8) = pack8<DT>(v);
  }
}

// Rows -> 32-row tiles. A thread moves one lane's 16 bytes: tile T, step s,
// operand j, lane l = 16 g + r is row 32 T + 8 (r / 4) + 4 j + r % 4 at elements
// 128 s + 32 g. Threads past the codes move the scales: tile T, chunk c, lane l,
// operand j: the word of steps 4 c .. 4 c + 3 of that row and g.
__device__ __forceinline__ int64_t tile_row(int64_t T, int j, int r) { return 32 * T + 8 * (r >> 2) + 4 * j + (r & 3); }

__global__ __launch_bounds__(kRowThreads) void k_mx_pack_codes(MxRows q, int R, int K, int64_t n, int steps,
                                                               uint8_t* __restrict__ codes, int64_t ld_c) {
  const int64_t i = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
  if (i >= n) return;
  const int64_t T = i / (steps * 128);
  const int o = (int)(i - T * (steps * 128));  // [s][j][lane]
  const int l = o & 63, j = (o >> 6) & 1, s = o >> 7;
  const int64_t row = tile_row(T, j, l & 15);
  const int k0 = 128 * s + 32 * (l >> 4);
  u4_t v = {0u, 0u, 0u, 0u};
  if (row < R && k0 < K) {
    v = *(const u4_t*)(q.codes + row * q.ld_c + k0 / 2);
    // codes past K, whatever the source's padding holds, are zero
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (k0 + 8 * e >= K) v[e] = 0u;
  }
  *(u4_t*)(codes + T * ld_c + (int64_t)o * 16) = v;
}

__global__ __launch_bounds__(kRowThreads) void k_mx_pack_scales(MxRows q, int R, int blocks, int64_t n, int chunks,
                                                                uint8_t* __restrict__ scales, int64_t ld_s) {
  const int64_t i = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
  if (i >= n) return;
  const int64_t T = i / (chunks * 128);
  const int o = (int)(i - T * (chunks * 128));  // [c][lane][j]
  const int j = o & 1, l = (o >> 1) & 63, c = o >> 7;
  const int64_t row = tile_row(T, j, l & 15);
  uint32_t w = 0u;
  if (row < R) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int b = 16 * c + 4 * t + (l >> 4);
      if (b < blocks) w |= (uint32_t)q.scales[row * q.ld_s + b] << (8 * t);
    }
  }
  *(uint32_t*)(scales + T * ld_s + (int64_t)o * 4) = w;
}

// h = x + residual (rounded to the element type, which is what later layers
// add to), y = h / sqrt(mean(h^2) + eps) * w. A workgroup per row; a thread holds
// its octets of the row in registers (fp32) between the sum of squares and the
// output: VPT octets, blockDim apart.
template <int DT, int FMT, int VPT>
__global__ __launch_bounds__(1024) void k_rmsnorm(NormArgs a) {
  __shared__ float sums[16];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, nt = blockDim.x;
  const int octets = a.K >> 3;
  float v[VPT][8];
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int k8 = tid + i * nt;
    u4_t x = {0u, 0u, 0u, 0u};
    if (k8 < octets) x = *(const u4_t*)(a.X + r * a.ldx + 8 * k8);
    unpack8<DT>(x, v[i]);
    if (a.res) {
      u4_t y = {0u, 0u, 0u, 0u};
      if (k8 < octets) y = *(const u4_t*)(a.res + r * a.ldr + 8 * k8);
      float t[8];
      unpack8<DT>(y, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] += v[i][e];
      y = pack8<DT>(t);
      if (k8 < octets) *(u4_t*)(a.h + r * a.ldh + 8 * k8) = y;
      unpack8<DT>(y, v[i]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(v[i][e], v[i][e], ss);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) ss += __shfl_xor(ss, o);
  if ((tid & 63) == 0) sums[tid >> 6] = ss;
  __syncthreads();
  ss = 0.f;
  for (int w = 0; w < nt >> 6; ++w) ss += sums[w];
  const float inv = rsqrtf(ss / (float)a.K + a.eps);
  const int code_octets = 16 * ((a.K + kMxStep - 1) / kMxStep);
  const int scale_octets = 64 * ((a.K + kMxChunk - 1) / kMxChunk);
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int k8 = tid + i * nt;
    u4_t w = {0u, 0u, 0u, 0u};
    if (k8 < octets) w = *(const u4_t*)(a.w + 8 * k8);
    float t[8];
    unpack8<DT>(w, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] *= v[i][e] * inv;
    if constexpr (FMT < 0) {
      if (k8 < octets) *(u4_t*)(a.Y + r * a.ldy + 8 * k8) = pack8<DT>(t);
    } else {
      // a row with a NaN or an infinity must not leave its padding's scales NaN
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (k8 >= octets) t[e] = 0.f;
      if (k8 < scale_octets) store_mx8<FMT>(t, k8, code_octets, a.q.codes + r * a.q.ld_c, a.q.scales + r * a.q.ld_s);
    }
  }
}

template <int DT, int FMT>
hipError_t norm_launch(const NormArgs& a, int threads, int vpt, hipStream_t s) {
  auto go = [&](auto* k) {
    k<<<dim3((unsigned)a.M), dim3((unsigned)threads), 0, s>>>(a);
    return hipGetLastError();
  };
  if (vpt <= 1) return go(k_rmsnorm<DT, FMT, 1>);
  if (vpt <= 2) return go(k_rmsnorm<DT, FMT, 2>);
  if (vpt <= 4) return go(k_rmsnorm<DT, FMT, 4>);
  return go(k_rmsnorm<DT, FMT, 8>);
}

unsigned blocks_of(int64_t n) { return (unsigned)((n + kRowThreads - 1) / kRowThreads); }

}  // namespace

namespace {

// Rows of a workgroup: four where that leaves every CU its eight workgroups
template <typename F1, typename F4>
hipError_t by_rows(int R, int per_row, F1 one, F4 four) {
  const int seg = (per_row + kRowThreads - 1) / kRowThreads;
  const int threads = std::min(kRowThreads, ((per_row + seg - 1) / seg + 63) / 64 * 64);
  if ((int64_t)R * seg >= 4 * 2048) four(dim3((unsigned)(((int64_t)R + 3) / 4 * seg)), dim3((unsigned)threads), seg);
  else one(dim3((unsigned)((int64_t)R * seg)), dim3((unsigned)threads), seg);
  return hipGetLastError();
}

template <int DT, int FMT>
hipError_t quantize(const uint16_t* X, int64_t ldx, int R, int K, const MxRows& q, hipStream_t s) {
  const int per_row = (int)(mx_chunks(K) * 64);
  return by_rows(
      R, per_row,
      [&](dim3 g, dim3 b, int seg) { k_mx_quantize<DT, FMT, 1><<<g, b, 0, s>>>(X, ldx, R, seg, per_row, K, q); },
      [&](dim3 g, dim3 b, int seg) { k_mx_quantize<DT, FMT, 4><<<g, b, 0, s>>>(X, ldx, R, seg, per_row, K, q); });
}

template <int DT, int FMT>
hipError_t dequantize(const MxRows& q, int R, int K, uint16_t* X, int64_t ldx, hipStream_t s) {
  const int per_row = K / 8;
  return by_rows(
      R, per_row,
      [&](dim3 g, dim3 b, int seg) { k_mx_dequantize<DT, FMT, 1><<<g, b, 0, s>>>(q, R, seg, per_row, X, ldx); },
      [&](dim3 g, dim3 b, int seg) { k_mx_dequantize<DT, FMT, 4><<<g, b, 0, s>>>(q, R, seg, per_row, X, ldx); });
}

}  // namespace

hipError_t launch_mx_quantize(const uint16_t* X, int64_t ldx, int R, int K, int dt, int fmt, const MxRows& q,
                              hipStream_t s) {
  if (dt == TPDQ_BF16)
    return fmt == kFp4 ? quantize<kBF16, kFp4>(X, ldx, R, K, q, s) : quantize<kBF16, kFp8>(X, ldx, R, K, q, s);
  return fmt == kFp4 ? quantize<kF16, kFp4>(X, ldx, R, K, q, s) : quantize<kF16, kFp8>(X, ldx, R, K, q, s);
}

hipError_t launch_mx_dequantize(const MxRows& q, int R, int K, int dt, int fmt, uint16_t* X, int64_t ldx,
                                hipStream_t s) {
  if (dt == TPDQ_BF16)
    return fmt == kFp4 ? dequantize<kBF16, kFp4>(q, R, K, X, ldx, s) : dequantize<kBF16, kFp8>(q, R, K, X, ldx, s);
  return fmt == kFp4 ? dequantize<kF16, kFp4>(q, R, K, X, ldx, s) : dequantize<kF16, kFp8>(q, R, K, X, ldx, s);
}

hipError_t launch_mx_pack(const MxRows& q, int R, int K, uint8_t* codes, int64_t ld_c, uint8_t* scales,
                          int64_t ld_s, hipStream_t s) {
  const int64_t tiles = (R + kMxTile - 1) / kMxTile;
  const int steps = (int)mx_steps(K), chunks = (int)mx_chunks(K);
  int64_t n = tiles * steps * 128;
  k_mx_pack_codes<<<dim3(blocks_of(n)), dim3(kRowThreads), 0, s>>>(q, R, K, n, steps, codes, ld_c);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  n = tiles * chunks * 128;
  k_mx_pack_scales<<<dim3(blocks_of(n)), dim3(kRowThreads), 0, s>>>(q, R, (K + kMxBlock - 1) / kMxBlock, n, chunks,
                                                                    scales, ld_s);
  return hipGetLastError();
}

hipError_t launch_rmsnorm(const NormArgs& a, int dt, int fmt, hipStream_t s) {
  int vpt = 0;
  const int threads = norm_threads(a.K, fmt, &vpt);
  if (dt == TPDQ_BF16) {
    if (fmt < 0) return norm_launch<kBF16, -1>(a, threads, vpt, s);
    return fmt == kFp4 ? norm_launch<kBF16, kFp4>(a, threads, vpt, s) : norm_launch<kBF16, kFp8>(a, threads, vpt, s);
  }
  if (fmt < 0) return norm_launch<kF16, -1>(a, threads, vpt, s);
  return fmt == kFp4 ? norm_launch<kF16, kFp4>(a, threads, vpt, s) : norm_launch<kF16, kFp8>(a, threads, vpt, s);
}

}  // namespace tpdq
