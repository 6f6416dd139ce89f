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
size_t adapter_wgrad_workspace_bytes(int64_t T, int segments, int R, int64_t I, int64_t O);      // of any number of adapters

// How the weight gradients are summed: the few rows of each adapter by one workgroup for each of its tiles, found by the segments' bounds; the same for every
// kFewRows rows, found by a table of every row's adapter; or by chunks of each segment's rows.
enum AdapterWgradWay { kWgradFew, kWgradRows, kWgradChunks };
constexpr int kFewRows = 2048, kFewSegments = 256;
inline int64_t wgrad_row_blocks(int64_t T) { return (T + kFewRows - 1) / kFewRows; }
// The table and, of several blocks, the number of rows that each adapter has in each and their sums
inline size_t wgrad_rows_workspace_bytes(int64_t T, int64_t adapters, int R, int64_t I, int64_t O) {
  const int64_t sums = T > kFewRows ? wgrad_row_blocks(T) * adapters : 0;
  return ((size_t)((T + sums + 3) / 4 * 4) + (size_t)sums * (size_t)R * (size_t)(I + O)) * 4;
}
// Few rows in one launch: its work grows with the adapters that have rows, and it reads M again for every 16 ranks.  Over 560 problems (64 to 2048 rows, 160 to
// 8192 features, ranks 16 to 128, 1 to 64 segments of as many adapters) the limit costs 0.8 % over the faster way in the mean, chunks everywhere 52 %.  64 rows
// of 1280 + 5120, rank 64, nine segments: 5 us against 20; 2048 rows, one segment: 23 against 20.
inline bool wgrad_few(int64_t T, int64_t segments, int64_t adapters, int R, int64_t I, int64_t O) {
  const int64_t n = segments < adapters ? segments : adapters;
  return T <= kFewRows && segments <= kFewSegments && T * R * (I + O) * (n > 8 ? n : 8) <= 6000000000ll;
}
// Chunks cost a sum of R x (I + O) floats for each segment, however few its rows; blocks of rows one for each adapter, and a table of the rows, but they read M again
// for every 16 ranks.  Over 3536 problems (200 to 100000 rows, 4 to 50000 segments, 1 to 64 adapters, ranks 8 to 128, 160 to 6400 features) this choice costs 2.8 %
// over the faster way in the mean and takes 3.0 times as long at most (100000 rows of 400 segments, 80 + 80, rank 16: 108 us, 36 in blocks), chunks everywhere
// 83 % and up to 446 times (50000 segments of one row).
inline AdapterWgradWay wgrad_way(int64_t T, int64_t segments, int64_t adapters, int R, int64_t I, int64_t O) {
  if (wgrad_few(T, segments, adapters, R, I, O)) return kWgradFew;
  const int64_t blocks = wgrad_row_blocks(T), tiles = ((I + 127) / 128 + (O + 127) / 128) * blocks;
  const bool short_segments = T > 0 && T <= 128 * segments && blocks * adapters <= segments;
  if (!short_segments || tiles >= 1 << 22 || I + O == 0) return kWgradChunks;
  // never more than chunks would need
  return wgrad_rows_workspace_bytes(T, adapters, R, I, O) <= (size_t)(segments + 2) * (size_t)R * (size_t)(I + O) * 4 ? kWgradRows : kWgradChunks;
}

hipError_t launch_checkpoint_pack(const void* X, int64_t R, int64_t C, int64_t ldx, void* codes, int64_t ldc, void* scales, int64_t lds, hipStream_t s);
hipError_t launch_checkpoint_backward(const void* codes, const void* scales, int64_t R, int64_t C, int64_t ldc, int64_t lds, int act, void* A, int64_t lda,
                                      const void* dA, int64_t ldda, void* dH, int64_t lddh, hipStream_t s);

}  // namespace sste
