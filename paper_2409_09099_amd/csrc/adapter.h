// Low-rank adapters beside a projection and 8-bit activation checkpoints: what the argument checks (adapter_api.hip) hand to the kernels.
#pragma once
#include "common.h"

namespace sste {

// 16 bytes at p, zeros where `ok` is false.  (As a conditional expression of two lvalues the choice falls on the address, and the load becomes a flat one.)
__device__ __forceinline__ uint4 load16(const void* p, bool ok) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (ok) v = *(const uint4*)p;
  return v;
}
// Rows of a batch by segments, as the caller's device arrays give them: segment s holds the rows row_start[s] .. row_start[s + 1] - 1 and
// uses adapter[s]; a number outside 0 .. adapters - 1 means none.
struct AdapterSegments {
  const int* row_start;
  const int* adapter;
  int segments, adapters, T;
};

// Widest low rank, and its granule; rows and segments whose tiles a grid can count (2^32 threads); widths whose tiles 32-bit offsets reach
constexpr int kAdapterMaxRank = 128, kAdapterRankStep = 8;
constexpr int64_t kAdapterMaxRows = 1ll << 27, kAdapterMaxSegments = 1ll << 20, kAdapterMaxAdapters = 65535, kAdapterMaxWidth = 1ll << 23, kAdapterMaxGrid = 1ll << 24;

// D = scale_n x_scale X down_n^T (T x R float32), out = base + D up_n (T x C bf16).  X is T x K of dtype; down_n is R x K, up_n is R x C, stacked.
struct AdapterApply {
  AdapterSegments seg;
  const void* X;
  int64_t ldx;
  int dtype;
  float x_scale;
  const void* down;
  int64_t lddown;
  const void* up;
  int64_t ldup;
  const float* scale;
  int R, K, C;
  const void* base;
  int64_t ldbase;
  void* out;
  int64_t ldout;
  float* D;
  int64_t ldd;
  float* ws;                // adapter_apply_workspace_bytes of it, or NULL
};
size_t adapter_apply_workspace_bytes(int64_t T, int segments, int R, int64_t K, int64_t C);
hipError_t launch_adapter_apply(const AdapterApply& a, hipStream_t s);

// One of the two weight gradients: G_n (R x C float32, stacked) (+)= m_scale sum over the rows of adapter n of L^T M, L T x R float32, M T x C.
struct AdapterOuter {
  const float* L;
  int64_t ldl;
  const void* M;
  int64_t ldm;
  int m_dtype;
  float m_scale;
  const uint8_t* blocks;    // SSTE_F8BLOCK: one scale byte per 32 features
  int64_t ldblocks;
  int C;
  float* G;
  int64_t ldg;
};
hipError_t launch_adapter_wgrad(const AdapterSegments& seg, int R, const AdapterOuter& a, const AdapterOuter& b, int accumulate, void* ws, hipStream_t s);
size_t adapter_wgrad_workspace_bytes(int64_t T, int segments, int R, int64_t I, int64_t O);

hipError_t launch_checkpoint_pack(const void* X, int64_t R, int64_t C, int64_t ldx, void* codes, int64_t ldc, void* scales, int64_t lds, hipStream_t s);
hipError_t launch_checkpoint_backward(const void* codes, const void* scales, int64_t R, int64_t C, int64_t ldc, int64_t lds, int act, void* A, int64_t lda,
                                      const void* dA, int64_t ldda, void* dH, int64_t lddh, hipStream_t s);

}  // namespace sste
