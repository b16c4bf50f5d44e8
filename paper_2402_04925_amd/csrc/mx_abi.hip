// extern "C" entry points of the microscaled (MX) operators: argument validation
// and dispatch. Every check is made on the host before anything is enqueued.
#include <algorithm>

#include "mx_internal.h"

using namespace tpdq;

namespace {

constexpr int64_t k2GiB = (int64_t)1 << 31;

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

tpdq_status check_dtype(tpdq_dtype dtype) {
  if (dtype != TPDQ_FP16 && dtype != TPDQ_BF16) return fail(TPDQ_ERR_SHAPE, "unknown dtype %d", (int)dtype);
  return TPDQ_OK;
}

// Shape, padding and alignment of an MX tensor in `layout`. addressed32: the
// products read it through 32-bit byte offsets.
tpdq_status check_mx(const tpdq_mx* q, const char* name, int layout, bool addressed32) {
  if (!q) return fail(TPDQ_ERR_NULL, "%s is NULL", name);
  if (!q->codes || !q->scales) return fail(TPDQ_ERR_NULL, "%s: codes and scales are required", name);
  if (q->format != TPDQ_MX_FP4 && q->format != TPDQ_MX_FP8)
    return fail(TPDQ_ERR_SHAPE, "%s: unknown format %d", name, q->format);
  if (q->layout != layout)
    return fail(TPDQ_ERR_SHAPE, "%s: layout %d, this call takes %s", name, q->layout,
                layout == TPDQ_MX_ROWS ? "TPDQ_MX_ROWS" : "TPDQ_MX_TILED");
  if (layout == TPDQ_MX_TILED && q->format != TPDQ_MX_FP4)
    return fail(TPDQ_ERR_UNSUPPORTED, "%s: tiled tensors are fp4", name);
  if (q->R <= 0 || q->K <= 0 || q->K % 8)
    return fail(TPDQ_ERR_SHAPE, "%s: R=%d and K=%d must be positive, K a multiple of 8", name, q->R, q->K);
  if (q->K > (1 << 30)) return fail(TPDQ_ERR_UNSUPPORTED, "%s: K=%d > 2^30", name, q->K);
  const int64_t c = layout == TPDQ_MX_ROWS ? mx_row_codes(q->K, q->format) : mx_tile_codes(q->K);
  const int64_t s = layout == TPDQ_MX_ROWS ? mx_row_scales(q->K) : mx_tile_scales(q->K);
  if (q->ld_c < c || q->ld_s < s)
    return fail(TPDQ_ERR_SHAPE, "%s: ld_c=%lld < %lld or ld_s=%lld < %lld (rows are padded)", name,
                (long long)q->ld_c, (long long)c, (long long)q->ld_s, (long long)s);
  if (!aligned(q->codes, 16) || !aligned(q->scales, 16) || q->ld_c % 16 || q->ld_s % 16)
    return fail(TPDQ_ERR_ALIGN, "%s: codes, scales and their leading dimensions need multiples of 16 bytes", name);
  const int64_t rows = layout == TPDQ_MX_ROWS ? q->R : (q->R + (int64_t)kMxTile - 1) / kMxTile;
  if (addressed32 && (q->ld_c >= k2GiB || q->ld_s >= k2GiB || rows * q->ld_c >= k2GiB || rows * q->ld_s >= k2GiB))
    return fail(TPDQ_ERR_UNSUPPORTED, "%s spans 2 GiB or more", name);
  return TPDQ_OK;
}

// 16-bit rows read and written with 16-byte accesses
tpdq_status check_rows16(const void* p, int64_t ld, int64_t K, const char* name) {
  if (!p) return fail(TPDQ_ERR_NULL, "%s is required", name);
  if (ld < K) return fail(TPDQ_ERR_SHAPE, "%s: leading dimension %lld < %lld", name, (long long)ld, (long long)K);
  if (!aligned(p, 16) || ld % 8)
    return fail(TPDQ_ERR_ALIGN, "%s needs 16-byte alignment and a leading dimension %% 8 == 0", name);
  return TPDQ_OK;
}

// `rows` rows of `bytes` bytes, `ld` bytes apart
struct Strip {
  const void* p;
  int64_t ld, bytes;
};

bool same(const Strip& a, const Strip& b, int64_t rows) { return a.p == b.p && (a.ld == b.ld || rows == 1); }

// Whether two strips share memory. With one leading dimension that is exact (columns of
// one buffer, side by side, do not meet); with two it is whether their extents meet.
bool meet(const Strip& a, const Strip& b, int64_t rows) {
  typedef __int128 wide;
  const wide pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
  if (pa + (wide)(rows - 1) * a.ld + a.bytes <= pb || pb + (wide)(rows - 1) * b.ld + b.bytes <= pa) return false;
  if (rows == 1 || a.ld != b.ld) return true;
  const wide d = ((pb - pa) % a.ld + a.ld) % a.ld;  // of b's rows behind a's
  return d < a.bytes || a.ld - d < b.bytes;
}

MxRows rows_of(const tpdq_mx* q) { return MxRows{(uint8_t*)q->codes, q->ld_c, (uint8_t*)q->scales, q->ld_s}; }

// A launch has fewer than 2^32 threads. Large calls take one for 32 elements: 16 for
// a chunk of a row, four rows (mx_pack: 32) together, and the chunks of a row in whole
// workgroups of at most four.
tpdq_status check_grid(int64_t R, int64_t K) {
  const int64_t chunks = mx_chunks(K), seg = (chunks + 3) / 4;
  if ((R + kMxTile) * (seg * ((chunks + seg - 1) / seg)) >= (int64_t)1 << 28)
    return fail(TPDQ_ERR_UNSUPPORTED, "%lld rows of %lld: more threads than a launch has, split the rows", (long long)R,
                (long long)K);
  return TPDQ_OK;
}

// What a product asks of X and w beyond their own shapes
tpdq_status check_product(const tpdq_mx* X, const tpdq_mx* w, const char* name) {
  tpdq_status st = check_mx(w, name, TPDQ_MX_TILED, true);
  if (st != TPDQ_OK) return st;
  if (w->R % 8) return fail(TPDQ_ERR_SHAPE, "%s: R=%d must be a multiple of 8", name, w->R);
  if (X && w->K != X->K) return fail(TPDQ_ERR_SHAPE, "%s: K=%d != X's K=%d", name, w->K, X->K);
  return TPDQ_OK;
}

MxArgs product(const MxRows& x, int M, const tpdq_mx* w, const tpdq_mx* up) {
  MxArgs a{};
  a.x = x;
  a.wc = (const uint8_t*)w->codes;
  a.ws = (const uint8_t*)w->scales;
  if (up) {
    a.wc_up = (const uint8_t*)up->codes;
    a.ws_up = (const uint8_t*)up->scales;
  }
  a.ldwc = w->ld_c;
  a.ldws = w->ld_s;
  a.M = M;
  a.N = w->R;
  a.K = w->K;
  return a;
}

// Y1 of the MLP in the workspace: codes (of fp8, the larger format), scales
size_t y1_codes_bytes(int64_t M, int64_t N) { return align_up((size_t)(M * mx_row_codes(N, TPDQ_MX_FP8))); }
size_t y1_bytes(int64_t M, int64_t N) { return y1_codes_bytes(M, N) + align_up((size_t)(M * mx_row_scales(N))); }

// split-K parts of one product, for the format of X that takes more
size_t part_bytes(int M, int N, int K, bool gated, bool quant) {
  size_t most = 0;
  for (int fmt : {(int)TPDQ_MX_FP4, (int)TPDQ_MX_FP8})
    most = std::max(most, mx_part_bytes(plan_mx(M, N, K, fmt, gated, quant), M, N, gated));
  return most;
}

bool valid_size(const tpdq_mx* w) { return w && w->R > 0 && w->K > 0 && w->K % 8 == 0 && w->R % 8 == 0; }

}  // namespace

extern "C" {

size_t tpdq_mx_workspace_bytes(int op, int32_t M, const tpdq_mx* a, const tpdq_mx* b) {
  if (M < 1 || !valid_size(a)) return 0;
  if (op == 0) return part_bytes(M, a->R, a->K, false, false);
  if (op != 1 || !valid_size(b) || b->K != a->R) return 0;
  // Y1, then the parts of the product at hand (the first may be gated or not)
  return y1_bytes(M, a->R) + std::max({part_bytes(M, a->R, a->K, true, true), part_bytes(M, a->R, a->K, false, true),
                                       part_bytes(M, b->R, b->K, false, false)});
}

tpdq_status tpdq_mx_quantize(const void* X, int64_t ldx, tpdq_dtype dtype, const tpdq_mx* q, void* stream) {
  tpdq_status st = check_dtype(dtype);
  if (st == TPDQ_OK) st = check_mx(q, "q", TPDQ_MX_ROWS, false);
  if (st == TPDQ_OK) st = check_rows16(X, ldx, q->K, "X");
  if (st == TPDQ_OK) st = check_grid(q->R, q->K);
  if (st != TPDQ_OK) return st;
  const hipError_t e = launch_mx_quantize((const uint16_t*)X, ldx, q->R, q->K, dtype, q->format, rows_of(q),
                                          (hipStream_t)stream);
  return e == hipSuccess ? TPDQ_OK : hip_fail(e, "quantize launch");
}

tpdq_status tpdq_mx_dequantize(const tpdq_mx* q, tpdq_dtype dtype, void* X, int64_t ldx, void* stream) {
  tpdq_status st = check_dtype(dtype);
  if (st == TPDQ_OK) st = check_mx(q, "q", TPDQ_MX_ROWS, false);
  if (st == TPDQ_OK) st = check_rows16(X, ldx, q->K, "X");
  if (st == TPDQ_OK) st = check_grid(q->R, q->K);
  if (st != TPDQ_OK) return st;
  const hipError_t e = launch_mx_dequantize(rows_of(q), q->R, q->K, dtype, q->format, (uint16_t*)X, ldx,
                                            (hipStream_t)stream);
  return e == hipSuccess ? TPDQ_OK : hip_fail(e, "dequantize launch");
}

tpdq_status tpdq_mx_pack(const tpdq_mx* src, const tpdq_mx* dst, void* stream) {
  tpdq_status st = check_mx(src, "src", TPDQ_MX_ROWS, false);
  if (st == TPDQ_OK && src->format != TPDQ_MX_FP4) st = fail(TPDQ_ERR_UNSUPPORTED, "src: tiled tensors are fp4");
  if (st == TPDQ_OK) st = check_mx(dst, "dst", TPDQ_MX_TILED, false);
  if (st == TPDQ_OK && (src->R != dst->R || src->K != dst->K))
    st = fail(TPDQ_ERR_SHAPE, "src is %d x %d, dst %d x %d", src->R, src->K, dst->R, dst->K);
  if (st == TPDQ_OK) st = check_grid(src->R, src->K);
  if (st != TPDQ_OK) return st;
  const hipError_t e = launch_mx_pack(rows_of(src), src->R, src->K, (uint8_t*)dst->codes, dst->ld_c,
                                      (uint8_t*)dst->scales, dst->ld_s, (hipStream_t)stream);
  return e == hipSuccess ? TPDQ_OK : hip_fail(e, "pack launch");
}

tpdq_status tpdq_rmsnorm(const void* X, int64_t ldx, const void* residual, int64_t ldr, const void* weight,
                         float eps, int32_t M, int32_t K, tpdq_dtype dtype, void* residual_out, int64_t ldh,
                         void* Y, int64_t ldy, const tpdq_mx* q, void* stream) {
  tpdq_status st = check_dtype(dtype);
  if (st != TPDQ_OK) return st;
  if (M < 1 || K < 1 || K % 8)
    return fail(TPDQ_ERR_SHAPE, "M=%d and K=%d must be positive, K a multiple of 8", M, K);
  if (K > kNormMaxK) return fail(TPDQ_ERR_UNSUPPORTED, "K=%d: rows of up to %d columns", K, kNormMaxK);
  if (!(eps >= 0.f)) return fail(TPDQ_ERR_SHAPE, "eps=%g must not be negative", (double)eps);
  st = check_rows16(X, ldx, K, "X");
  if (st == TPDQ_OK) st = check_rows16(weight, K, K, "weight");
  if (st != TPDQ_OK) return st;
  if ((residual == nullptr) != (residual_out == nullptr))
    return fail(TPDQ_ERR_NULL, "residual and residual_out are given together");
  if (residual) {
    st = check_rows16(residual, ldr, K, "residual");
    if (st == TPDQ_OK) st = check_rows16(residual_out, ldh, K, "residual_out");
    if (st != TPDQ_OK) return st;
  }
  if ((Y == nullptr) == (q == nullptr)) return fail(TPDQ_ERR_NULL, "one of Y and q is given");
  if (Y) {
    st = check_rows16(Y, ldy, K, "Y");
  } else {
    st = check_mx(q, "q", TPDQ_MX_ROWS, false);
    if (st == TPDQ_OK && (q->R != M || q->K != K))
      st = fail(TPDQ_ERR_SHAPE, "q is %d x %d, the call %d x %d", q->R, q->K, M, K);
  }
  if (st != TPDQ_OK) return st;
  int vpt = 0;
  if ((int64_t)M * norm_threads(K, q ? q->format : -1, &vpt) >= (int64_t)1 << 32)
    return fail(TPDQ_ERR_UNSUPPORTED, "%d rows: more threads than a launch has, split the rows", M);
  const Strip x{X, 2 * ldx, 2 * (int64_t)K}, res{residual, 2 * ldr, x.bytes}, h{residual_out, 2 * ldh, x.bytes},
      y{Y, 2 * ldy, x.bytes};
  if (residual) {
    const bool shared = Y ? meet(h, y, M)
                          : meet(h, Strip{q->codes, q->ld_c, mx_row_codes(K, q->format)}, M) ||
                                meet(h, Strip{q->scales, q->ld_s, mx_row_scales(K)}, M);
    if (shared) return fail(TPDQ_ERR_SHAPE, "the output and residual_out share memory");
  }
  // in place: the workgroup of a row reads it before it writes that row, and no other
  for (const Strip& out : {h, y})
    for (const Strip& in : {x, res})
      if (out.p && in.p && !same(out, in, M) && meet(out, in, M))
        return fail(TPDQ_ERR_SHAPE, "Y or residual_out shares memory with rows of X or residual other than its own");
  NormArgs a{};
  a.X = (const uint16_t*)X;
  a.ldx = ldx;
  a.res = (const uint16_t*)residual;
  a.ldr = ldr;
  a.w = (const uint16_t*)weight;
  a.h = (uint16_t*)residual_out;
  a.ldh = ldh;
  a.Y = (uint16_t*)Y;
  a.ldy = ldy;
  if (q) a.q = rows_of(q);
  a.M = M;
  a.K = K;
  a.eps = eps;
  const hipError_t e = launch_rmsnorm(a, dtype, q ? q->format : -1, (hipStream_t)stream);
  return e == hipSuccess ? TPDQ_OK : hip_fail(e, "rmsnorm launch");
}

tpdq_status tpdq_mx_gemm(const tpdq_mx* X, const tpdq_mx* w, tpdq_dtype dtype, void* Y, int64_t ldy,
                         void* workspace, size_t ws_bytes, void* stream) {
  tpdq_status st = check_dtype(dtype);
  if (st == TPDQ_OK) st = check_mx(X, "X", TPDQ_MX_ROWS, true);
  if (st == TPDQ_OK) st = check_product(X, w, "w");
  if (st == TPDQ_OK) st = check_rows16(Y, ldy, w->R, "Y");
  if (st != TPDQ_OK) return st;
  const size_t need = tpdq_mx_workspace_bytes(0, X->R, w, nullptr);
  if (need && (!workspace || ws_bytes < need))
    return fail(TPDQ_ERR_WORKSPACE, "product needs %zu workspace bytes, got %zu", need, ws_bytes);
  if (need && !aligned(workspace, 16)) return fail(TPDQ_ERR_ALIGN, "workspace needs 16-byte alignment");
  MxArgs a = product(rows_of(X), X->R, w, nullptr);
  a.Y = (uint16_t*)Y;
  a.ldy = ldy;
  const hipError_t e = launch_mx_gemm(a, dtype, X->format, (float*)workspace, (hipStream_t)stream);
  return e == hipSuccess ? TPDQ_OK : hip_fail(e, "product launch");
}

tpdq_status tpdq_mx_mlp_shard(const tpdq_mx* X, const tpdq_mx* w_gate, const tpdq_mx* w_up, const tpdq_mx* w_down,
                              tpdq_dtype dtype, void* Y2_partial, void* workspace, size_t ws_bytes, void* stream) {
  tpdq_status st = check_dtype(dtype);
  if (st == TPDQ_OK) st = check_mx(X, "X", TPDQ_MX_ROWS, true);
  if (st == TPDQ_OK) st = check_product(X, w_up, "w_up");
  if (st == TPDQ_OK && w_gate) st = check_product(X, w_gate, "w_gate");
  if (st == TPDQ_OK && w_gate && (w_gate->R != w_up->R || w_gate->ld_c != w_up->ld_c || w_gate->ld_s != w_up->ld_s))
    st = fail(TPDQ_ERR_SHAPE, "w_gate must match w_up in R, K and leading dimensions");
  if (st == TPDQ_OK) st = check_product(nullptr, w_down, "w_down");
  if (st == TPDQ_OK && w_down->K != w_up->R)
    st = fail(TPDQ_ERR_SHAPE, "w_down->K=%d != w_up->R=%d", w_down->K, w_up->R);
  if (st == TPDQ_OK) st = check_rows16(Y2_partial, w_down->R, w_down->R, "Y2_partial");
  if (st != TPDQ_OK) return st;
  const int M = X->R, N1 = w_up->R;
  if ((int64_t)M * mx_row_codes(N1, X->format) >= k2GiB) return fail(TPDQ_ERR_UNSUPPORTED, "Y1 spans 2 GiB or more");
  const size_t need = tpdq_mx_workspace_bytes(1, M, w_up, w_down);
  if (!workspace || ws_bytes < need)
    return fail(TPDQ_ERR_WORKSPACE, "MLP needs %zu workspace bytes, got %zu", need, ws_bytes);
  if (!aligned(workspace, 16)) return fail(TPDQ_ERR_ALIGN, "workspace needs 16-byte alignment");
  const MxRows y1{(uint8_t*)workspace, mx_row_codes(N1, X->format),
                  (uint8_t*)workspace + y1_codes_bytes(M, N1), mx_row_scales(N1)};
  const hipStream_t s = (hipStream_t)stream;
  // gated: the gate is the first weight, up the second
  MxArgs a = w_gate ? product(rows_of(X), M, w_gate, w_up) : product(rows_of(X), M, w_up, nullptr);
  a.q = y1;
  float* part = (float*)((char*)workspace + y1_bytes(M, N1));
  hipError_t e = launch_mx_gemm(a, dtype, X->format, part, s);
  if (e != hipSuccess) return hip_fail(e, "first product launch");
  MxArgs d = product(y1, M, w_down, nullptr);
  d.Y = (uint16_t*)Y2_partial;
  d.ldy = w_down->R;
  e = launch_mx_gemm(d, dtype, X->format, part, s);
  return e == hipSuccess ? TPDQ_OK : hip_fail(e, "second product launch");
}

}  // extern "C"
