// C ABI of the low-rank adapters and the activation checkpoints: argument validation on the host, then kernel launches on the caller's
// stream.  Nothing here allocates, frees or synchronises.
#include "adapter.h"

#include <cmath>

namespace sste {

static bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
static bool good_scale(float v) { return std::isfinite(v) && v > 0.0f; }
static bool is_8bit(int d) { return d == SSTE_F8E4M3 || d == SSTE_F8E5M2 || d == SSTE_F8BLOCK; }
static int hip_status(hipError_t e, const char* what) { return e == hipSuccess ? SSTE_OK : fail(SSTE_ERR_HIP, "%s: %s", what, hipGetErrorString(e)); }

// A rows x cols matrix with leading dimension ld in elements, whose rows start at multiples of 16 bytes (`step` elements)
static int check_matrix(const char* who, const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, int step) {
  if (ld < cols) return fail(SSTE_ERR_SHAPE, "%s: leading dimension of %s smaller than the row length", who, name);
  if (rows == 0 || cols == 0) return SSTE_OK;            // never addressed
  if (ld % step != 0 || !aligned(p, 16)) return fail(SSTE_ERR_ALIGN, "%s: %s must be 16-byte aligned with a leading dimension that is a multiple of %d", who, name, step);
  if (!p) return fail(SSTE_ERR_NULL, "%s: NULL %s", who, name);
  if (ld > kAdapterMaxWidth) return fail(SSTE_ERR_UNSUPPORTED, "%s: leading dimension of %s above 2^23", who, name);
  if (product_reaches(rows, ld, 1ll << 40)) return fail(SSTE_ERR_UNSUPPORTED, "%s: %s has more than 2^40 elements", who, name);
  return SSTE_OK;
}

static int check_segments(const char* who, int64_t T, const int32_t* row_start, int64_t segments, const int32_t* seg_adapter, int64_t adapters, int64_t R) {
  if (T < 0 || segments < 0 || adapters < 0) return fail(SSTE_ERR_SHAPE, "%s: negative number of rows, segments or adapters", who);
  if (R < 1) return fail(SSTE_ERR_SHAPE, "%s: rank %lld", who, (long long)R);
  if (R > kAdapterMaxRank || R % kAdapterRankStep != 0)
    return fail(SSTE_ERR_UNSUPPORTED, "%s: rank %lld is not a multiple of %d up to %d (pad A and B with rows of zeros)", who, (long long)R, kAdapterRankStep, kAdapterMaxRank);
  if (T >= kAdapterMaxRows || segments > kAdapterMaxSegments || adapters > kAdapterMaxAdapters)
    return fail(SSTE_ERR_UNSUPPORTED, "%s: 2^27 rows or more, more than 2^20 segments or more than 65535 adapters", who);
  if (segments > 0 && (!row_start || !seg_adapter)) return fail(SSTE_ERR_NULL, "%s: NULL row_start or seg_adapter", who);
  if (!aligned(row_start, 4) || !aligned(seg_adapter, 4)) return fail(SSTE_ERR_ALIGN, "%s: row_start and seg_adapter must be 4-byte aligned", who);
  return SSTE_OK;
}

static int check_width(const char* who, const char* name, int64_t n, int dtype) {
  const int step = is_8bit(dtype) ? 16 : 8;
  if (n < 0) return fail(SSTE_ERR_SHAPE, "%s: negative size", who);
  if (n % step != 0 || n > kAdapterMaxWidth) return fail(SSTE_ERR_UNSUPPORTED, "%s: %s=%lld must be a multiple of %d up to 2^23", who, name, (long long)n, step);
  return SSTE_OK;
}

#define TRY(expr)                              \
  do {                                         \
    const int st_ = (expr);                    \
    if (st_ != SSTE_OK) return st_;            \
  } while (0)

// D = scale_n x_scale X down_n^T and out = base + D up_n; K and C: widths of X and out, named as the caller knows them
static int apply(const char* who, const char* xname, const char* dname, const char* oname, const char* kname, const char* cname, const char* down_name, const char* up_name,
                 bool e5m2, void* ws, size_t ws_bytes, AdapterApply a, int64_t T, int64_t segments, int64_t adapters, int64_t R, int64_t K, int64_t C, hipStream_t s) {
  TRY(check_segments(who, T, a.seg.row_start, segments, a.seg.adapter, adapters, R));
  if (a.dtype != SSTE_BF16 && a.dtype != SSTE_F8E4M3 && !(e5m2 && a.dtype == SSTE_F8E5M2)) return fail(SSTE_ERR_DTYPE, "%s: dtype %d", who, a.dtype);
  if (!good_scale(a.x_scale) || (a.dtype == SSTE_BF16 && a.x_scale != 1.0f)) return fail(SSTE_ERR_VALUE, "%s: the scale of %s must be finite and > 0, and 1 for bf16", who, xname);
  TRY(check_width(who, kname, K, a.dtype));
  TRY(check_width(who, cname, C, SSTE_BF16));
  TRY(check_matrix(who, xname, a.X, T, K, a.ldx, is_8bit(a.dtype) ? 16 : 8));
  TRY(check_matrix(who, down_name, a.down, adapters * R, K, a.lddown, 8));
  TRY(check_matrix(who, up_name, a.up, adapters * R, C, a.ldup, 8));
  TRY(check_matrix(who, dname, a.D, T, R, a.ldd, 4));
  TRY(check_matrix(who, oname, a.out, T, C, a.ldout, 8));
  if (a.base) TRY(check_matrix(who, "base", a.base, T, C, a.ldbase, 8));
  if (a.base == a.out && a.base && T > 1 && a.ldbase != a.ldout) return fail(SSTE_ERR_VALUE, "%s: base may be %s itself only with the same leading dimension", who, oname);
  if (!aligned(a.scale, 4)) return fail(SSTE_ERR_ALIGN, "%s: scale must be 4-byte aligned", who);
  if (product_reaches(T / 32 + segments + 9, (C + 511) / 512, kAdapterMaxGrid)) return fail(SSTE_ERR_UNSUPPORTED, "%s: more than 2^24 tiles", who);
  // without the workspace (none, too small, misaligned) the contraction is not split: the same function, slower for few rows
  const size_t need = adapter_apply_workspace_bytes(T, (int)segments, (int)R, K, C);
  a.ws = ws && ws_bytes >= need && need > 0 && aligned(ws, 16) ? (float*)ws : nullptr;
  a.seg.segments = (int)segments;
  a.seg.adapters = (int)adapters;
  a.seg.T = (int)T;
  a.R = (int)R;
  a.K = (int)K;
  a.C = (int)C;
  return hip_status(launch_adapter_apply(a, s), who);
}

}  // namespace sste

using namespace sste;

extern "C" {

int sste_adapter_fwd(const void* X, int64_t T, int64_t I, int64_t ldx, int dtype, float x_scale,
                     const int32_t* row_start, int64_t segments, const int32_t* seg_adapter,
                     const void* A, int64_t lda, const void* B, int64_t ldb, const float* scale, int64_t adapters, int64_t R, int64_t O,
                     const void* base, int64_t ldbase, void* Z, int64_t ldz, float* S, int64_t lds, void* workspace, size_t workspace_bytes, void* hip_stream) {
  clear_error();
  AdapterApply a = {{row_start, seg_adapter, 0, 0, 0}, X, ldx, dtype, x_scale, A, lda, B, ldb, scale, 0, 0, 0, base, ldbase, Z, ldz, S, lds, nullptr};
  return apply("adapter_fwd", "X", "S", "Z", "I", "O", "A", "B", false, workspace, workspace_bytes, a, T, segments, adapters, R, I, O, (hipStream_t)hip_stream);
}

int sste_adapter_dgrad(const void* dZ, int64_t T, int64_t O, int64_t lddz, int dtype, float dz_scale,
                       const int32_t* row_start, int64_t segments, const int32_t* seg_adapter,
                       const void* A, int64_t lda, const void* B, int64_t ldb, const float* scale, int64_t adapters, int64_t R, int64_t I,
                       const void* base, int64_t ldbase, void* dX, int64_t lddx, float* dS, int64_t ldds, void* workspace, size_t workspace_bytes, void* hip_stream) {
  clear_error();
  AdapterApply a = {{row_start, seg_adapter, 0, 0, 0}, dZ, lddz, dtype, dz_scale, B, ldb, A, lda, scale, 0, 0, 0, base, ldbase, dX, lddx, dS, ldds, nullptr};
  return apply("adapter_dgrad", "dZ", "dS", "dX", "O", "I", "B", "A", true, workspace, workspace_bytes, a, T, segments, adapters, R, O, I, (hipStream_t)hip_stream);
}

static int check_sizes(const char* who, int64_t T, int64_t segments, int64_t R, int64_t I, int64_t O) {
  TRY(check_segments(who, T, nullptr, 0, nullptr, 0, R));
  if (segments < 0) return fail(SSTE_ERR_SHAPE, "%s: negative number of segments", who);
  if (segments > kAdapterMaxSegments) return fail(SSTE_ERR_UNSUPPORTED, "%s: more than 2^20 segments", who);
  TRY(check_width(who, "I", I, SSTE_BF16));
  TRY(check_width(who, "O", O, SSTE_BF16));
  return SSTE_OK;
}

size_t sste_adapter_workspace_bytes(int64_t T, int64_t segments, int64_t R, int64_t in, int64_t out) {
  clear_error();
  if (check_sizes("adapter_workspace_bytes", T, segments, R, in, out) != SSTE_OK) return 0;
  return adapter_apply_workspace_bytes(T, (int)segments, (int)R, in, out);
}

size_t sste_adapter_wgrad_workspace_bytes(int64_t T, int64_t segments, int64_t R, int64_t I, int64_t O) {
  clear_error();
  if (check_sizes("adapter_wgrad_workspace_bytes", T, segments, R, I, O) != SSTE_OK) return 0;
  return adapter_wgrad_workspace_bytes(T, (int)segments, (int)R, I, O);
}

// What a call needs whose number of adapters is known; never more than the same without that number
static size_t wgrad_workspace(int64_t T, int64_t segments, int64_t adapters, int64_t R, int64_t I, int64_t O) {
  switch (wgrad_way(T, segments, adapters, (int)R, I, O)) {
    case kWgradFew: return segments <= adapters ? adapter_wgrad_workspace_bytes(T, (int)segments, (int)R, I, O) : 0;
    case kWgradRows: return wgrad_rows_workspace_bytes(T, adapters, (int)R, I, O);
    default: return adapter_wgrad_workspace_bytes(T, (int)segments, (int)R, I, O);
  }
}

size_t sste_adapter_wgrad_workspace_bytes_ex(int64_t T, int64_t segments, int64_t adapters, int64_t R, int64_t I, int64_t O) {
  const char* who = "adapter_wgrad_workspace_bytes_ex";
  clear_error();
  if (check_sizes(who, T, segments, R, I, O) != SSTE_OK) return 0;
  if (adapters < 0 || adapters > kAdapterMaxAdapters) {
    fail(SSTE_ERR_SHAPE, "%s: %lld adapters", who, (long long)adapters);
    return 0;
  }
  return wgrad_workspace(T, segments, adapters, R, I, O);
}

int sste_adapter_wgrad(const void* dZ, int64_t T, int64_t O, int64_t lddz, int dtype, float dz_scale,
                       const void* X, int64_t I, int64_t ldx, int x_dtype, float x_scale, const void* x_blocks, int64_t ldxb,
                       const float* S, int64_t lds, const float* dS, int64_t ldds,
                       const int32_t* row_start, int64_t segments, const int32_t* seg_adapter, int64_t adapters, int64_t R,
                       float* dA, int64_t ldda, float* dB, int64_t lddb, int accumulate,
                       void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* who = "adapter_wgrad";
  clear_error();
  TRY(check_segments(who, T, row_start, segments, seg_adapter, adapters, R));
  if (dtype != SSTE_BF16 && dtype != SSTE_F8E4M3 && dtype != SSTE_F8E5M2) return fail(SSTE_ERR_DTYPE, "%s: dtype %d", who, dtype);
  if (x_dtype != SSTE_BF16 && x_dtype != SSTE_F8E4M3 && x_dtype != SSTE_F8BLOCK) return fail(SSTE_ERR_DTYPE, "%s: x_dtype %d", who, x_dtype);
  if (!good_scale(dz_scale) || (dtype == SSTE_BF16 && dz_scale != 1.0f)) return fail(SSTE_ERR_VALUE, "%s: dz_scale must be finite and > 0, and 1 for bf16", who);
  if (!good_scale(x_scale) || (x_dtype != SSTE_F8E4M3 && x_scale != 1.0f)) return fail(SSTE_ERR_VALUE, "%s: x_scale must be finite and > 0, and 1 but for e4m3", who);
  if (accumulate != 0 && accumulate != 1) return fail(SSTE_ERR_VALUE, "%s: accumulate must be 0 or 1", who);
  TRY(check_width(who, "O", O, dtype));
  TRY(check_width(who, "I", I, x_dtype));
  TRY(check_matrix(who, "dZ", dZ, T, O, lddz, is_8bit(dtype) ? 16 : 8));
  TRY(check_matrix(who, "X", X, T, I, ldx, is_8bit(x_dtype) ? 16 : 8));
  if (x_dtype == SSTE_F8BLOCK) {
    if (ldxb < (I + 31) / 32) return fail(SSTE_ERR_SHAPE, "%s: ldxb smaller than the blocks of a row", who);
    if (ldxb > kAdapterMaxWidth) return fail(SSTE_ERR_UNSUPPORTED, "%s: ldxb above 2^23", who);
    if (T > 0 && I > 0 && !x_blocks) return fail(SSTE_ERR_NULL, "%s: a checkpoint of X needs its scales", who);
  } else {
    x_blocks = nullptr;
    ldxb = 0;
  }
  TRY(check_matrix(who, "S", S, T, R, lds, 4));
  TRY(check_matrix(who, "dS", dS, T, R, ldds, 4));
  TRY(check_matrix(who, "dA", dA, adapters * R, I, ldda, 4));
  TRY(check_matrix(who, "dB", dB, adapters * R, O, lddb, 4));
  const size_t chunks = adapter_wgrad_workspace_bytes(T, (int)segments, (int)R, I, O), need = wgrad_workspace(T, segments, adapters, R, I, O);
  if (chunks > 0 && product_reaches((int64_t)(chunks / (4 * (size_t)R * (size_t)(I + O))), 2 * (I / 256 + O / 256 + 2), kAdapterMaxGrid))      // R x (I + O) floats for each
    return fail(SSTE_ERR_UNSUPPORTED, "%s: more than 2^24 tiles", who);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(SSTE_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", who, workspace ? workspace_bytes : (size_t)0, need);
  if (!aligned(workspace, 16)) return fail(SSTE_ERR_ALIGN, "%s: workspace must be 16-byte aligned", who);
  const AdapterSegments g = {row_start, seg_adapter, (int)segments, (int)adapters, (int)T};
  const AdapterOuter a = {dS, ldds, X, ldx, x_dtype, x_scale, (const uint8_t*)x_blocks, ldxb, (int)I, dA, ldda};
  const AdapterOuter b = {S, lds, dZ, lddz, dtype, dz_scale, nullptr, 0, (int)O, dB, lddb};
  return hip_status(launch_adapter_wgrad(g, (int)R, a, b, accumulate, workspace, (hipStream_t)hip_stream), who);
}

static int check_checkpoint(const char* who, int64_t R, int64_t C, const void* codes, int64_t ldc, const void* scales, int64_t lds) {
  if (R < 0 || C < 0) return fail(SSTE_ERR_SHAPE, "%s: negative size", who);
  if (C % 16 != 0 || C > kAdapterMaxWidth) return fail(SSTE_ERR_UNSUPPORTED, "%s: C=%lld must be a multiple of 16 up to 2^23", who, (long long)C);
  if (R >= 1ll << 31) return fail(SSTE_ERR_UNSUPPORTED, "%s: 2^31 rows or more", who);
  TRY(check_matrix(who, "codes", codes, R, C, ldc, 16));
  if (lds < (C + 31) / 32) return fail(SSTE_ERR_SHAPE, "%s: lds smaller than the blocks of a row", who);
  if (R > 0 && C > 0 && !scales) return fail(SSTE_ERR_NULL, "%s: NULL scales", who);
  if (product_reaches(R, lds, 1ll << 40)) return fail(SSTE_ERR_UNSUPPORTED, "%s: more than 2^40 scales", who);
  return SSTE_OK;
}

int sste_checkpoint_pack(const void* X, int64_t R, int64_t C, int64_t ldx, void* codes, int64_t ldc, void* scales, int64_t lds, void* hip_stream) {
  const char* who = "checkpoint_pack";
  clear_error();
  TRY(check_checkpoint(who, R, C, codes, ldc, scales, lds));
  TRY(check_matrix(who, "X", X, R, C, ldx, 8));
  return hip_status(launch_checkpoint_pack(X, R, C, ldx, codes, ldc, scales, lds, (hipStream_t)hip_stream), who);
}

int sste_checkpoint_backward(const void* codes, const void* scales, int64_t R, int64_t C, int64_t ldc, int64_t lds, int act,
                             void* A, int64_t lda, const void* dA, int64_t ldda, void* dH, int64_t lddh, void* hip_stream) {
  const char* who = "checkpoint_backward";
  clear_error();
  if (act != SSTE_ACT_NONE && act != SSTE_ACT_GELU_TANH) return fail(SSTE_ERR_VALUE, "%s: unknown activation %d", who, act);
  TRY(check_checkpoint(who, R, C, codes, ldc, scales, lds));
  const bool empty = R == 0 || C == 0;
  if (!empty && !A && !dH) return fail(SSTE_ERR_NULL, "%s: both A and dH are NULL", who);
  if (!empty && (dA != nullptr) != (dH != nullptr)) return fail(SSTE_ERR_NULL, "%s: dA and dH are given together", who);
  if (A) TRY(check_matrix(who, "A", A, R, C, lda, 8));
  if (dH) {
    TRY(check_matrix(who, "dA", dA, R, C, ldda, 8));
    TRY(check_matrix(who, "dH", dH, R, C, lddh, 8));
    if (dA == dH && R > 1 && ldda != lddh) return fail(SSTE_ERR_VALUE, "%s: dH may be dA itself only with the same leading dimension", who);
  }
  return hip_status(launch_checkpoint_backward(codes, scales, R, C, ldc, lds, act, A, lda, dA, ldda, dH, lddh, (hipStream_t)hip_stream), who);
}

}  // extern "C"
