// Low-rank adapters beside a shared projection: every row of a batch has its own adapter, or none.
//
//   down   D = scale_n X down_n^T               T x R, float32       S of the forward pass (down = A), dS of the input gradient (down = B)
//   up     out = base + D up_n                  T x C, bf16          Z (up = B), dX (up = A)
//   outer  G_n = sum over rows of n of L^T M    R x C, float32       dA (L = dS, M = X), dB (L = S, M = dZ)
//
// A and B are both kept rank-major (R x I, R x O), so the forward pass and the input gradient are the same two kernels with A and B
// exchanged, and the two weight gradients are one.  The rank is small: all three are bound by the bytes of X, base, out and M.
#include "adapter.h"

namespace sste {

namespace {

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

// ---- rows to tiles --------------------------------------------------------------------------------------------
// The grids are sized from T and the number of segments alone; the segments' bounds stay on the device.  With the rows before the first
// and behind the last segment as two more (without an adapter), bounds b_0 = 0 <= b_1 <= ... <= b_{S+2} = T, segment v's tiles of TR rows
// take the slots from floor(b_v / TR) + v on: floor(b_{v+1} / TR) - floor(b_v / TR) + 1 slots, never fewer than its tiles.
// Bounds are clamped to 0 .. T, so that no array of bounds leads outside the matrices.
struct Tile {
  int64_t row;    // first row
  int rows;       // <= 0: an empty slot
  int adapter;    // -1: none
};
__device__ __forceinline__ int segment_bound(const AdapterSegments& g, int v) {
  if (v <= 0) return 0;
  if (v >= g.segments + 2) return g.T;
  return min(max(g.row_start[v - 1], 0), g.T);
}
__device__ __forceinline__ int first_slot(const AdapterSegments& g, int v, int tr) { return (int)((uint32_t)segment_bound(g, v) / (uint32_t)tr) + v; }
__device__ __forceinline__ int segment_adapter(const AdapterSegments& g, int v) {
  if (v <= 0 || v > g.segments) return -1;
  const int n = g.adapter[v - 1];
  return n >= 0 && n < g.adapters ? n : -1;
}
// Every wave finds its tile by itself: 64 probes a round, so two rounds serve 4096 segments.
__device__ __forceinline__ Tile find_tile(const AdapterSegments& g, int slot, int tr) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = g.segments + 2;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int v = lo + lane * step;
    const bool before = lane * step < n && first_slot(g, v, tr) <= slot;
    const uint64_t mask = __ballot(before) | 1;
    const int hit = 63 - __clzll((long long)mask);
    n = min(step, n - hit * step);
    lo += hit * step;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  Tile t;
  t.row = segment_bound(g, lo) + (int64_t)(slot - first_slot(g, lo, tr)) * tr;
  t.rows = (int)min((int64_t)tr, segment_bound(g, lo + 1) - t.row);
  t.adapter = segment_adapter(g, lo);
  return t;
}
int64_t slots(const AdapterSegments& g, int tr) { return (int64_t)g.T / tr + g.segments + 2; }

// ---- operands -------------------------------------------------------------------------------------------------
// Eight consecutive elements as bf16.  8-bit formats convert exactly (e4m3 and e5m2 are subsets of bf16).
enum { M_BF16 = 0, M_E4M3 = 1, M_E5M2 = 2, M_BLOCK = 3 };
template <int DT>
__device__ __forceinline__ uint4 widen(uint2 c, float s) {
  uint4 r;
  bf16x2 v[4];
  if (DT == M_E5M2) {
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c.x, s, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c.x, s, true);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c.y, s, false);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c.y, s, true);
  } else {
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, s, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, s, true);
    v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, s, false);
    v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, s, true);
  }
  __builtin_memcpy(&r, v, 16);
  return r;
}
__device__ __forceinline__ bf16x8 frag(uint4 v) {
  bf16x8 r;
  __builtin_memcpy(&r, &v, 16);
  return r;
}
// A float as the sum of two bf16 to within 2^-17 of itself: hi the nearest, lo the nearest to what is left.  One bf16 alone would be off by up
// to 2^-8, a rounding of a 32-bit sum that nothing asks for; the second matrix instruction that lo takes is hidden under the memory traffic.
__device__ __forceinline__ void split8(const float (&x)[8], uint4& hi, uint4& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int p = 0; p < 4; p++) {
    h[p] = bf16_rne_pack(x[2 * p], x[2 * p + 1]);
    l[p] = bf16_rne_pack(x[2 * p] - bf16lo_f32(h[p]), x[2 * p + 1] - bf16hi_f32(h[p]));
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}
// The same in three parts, exact to the last bit of the float: what the weight gradients take, whose float32 results would show 2^-17.
__device__ __forceinline__ void split8(const float (&x)[8], uint4& hi, uint4& mid, uint4& lo) {
  uint32_t h[4], m[4], l[4];
#pragma unroll
  for (int p = 0; p < 4; p++) {
    h[p] = bf16_rne_pack(x[2 * p], x[2 * p + 1]);
    const float a = x[2 * p] - bf16lo_f32(h[p]), b = x[2 * p + 1] - bf16hi_f32(h[p]);
    m[p] = bf16_rne_pack(a, b);
    l[p] = bf16_rne_pack(a - bf16lo_f32(m[p]), b - bf16hi_f32(m[p]));
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  mid = make_uint4(m[0], m[1], m[2], m[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}
// Transposes an 8 x 8 block of 16-bit elements held by one lane: x[i] holds elements (i, 0..7); out[j] holds (0..7, j).
__device__ __forceinline__ void transpose8(const uint4 (&x)[8], uint4 (&out)[8]) {
  const uint32_t* s = (const uint32_t*)x;
  uint32_t* d = (uint32_t*)out;
#pragma unroll
  for (int j = 0; j < 8; j++)
#pragma unroll
    for (int p = 0; p < 4; p++)
      d[j * 4 + p] = __builtin_amdgcn_perm(s[(2 * p + 1) * 4 + (j >> 1)], s[2 * p * 4 + (j >> 1)], (j & 1) ? 0x07060302u : 0x05040100u);
}

// ---- down -----------------------------------------------------------------------------------------------------
// A workgroup takes 16 TT rows of one adapter, its waves the contraction in turn (64 elements a step: lane quarter q holds elements 16 q ..
// 16 q + 15, eight of them per matrix instruction, the same on both operands), so that every element of X and of the adapter is read once
// per workgroup; the waves' sums meet in LDS in a fixed order.
template <int DT, int RT, int TT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64)
k_adapter_down(AdapterSegments g, const uint8_t* __restrict__ X, int64_t ldx, int K, const uint16_t* __restrict__ W, int64_t ldw, int R,
               const float* __restrict__ scale, float x_scale, float* __restrict__ D, int64_t ldd) {
  constexpr int RP = RT * 16, TR = TT * 16, LD = RP + 4, EB = DT == M_BF16 ? 2 : 1;
  __shared__ float red[WAVES][TR][LD];
  const Tile t = find_tile(g, blockIdx.x, TR);
  if (t.rows <= 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (t.adapter < 0) {
    for (int i = tid; i < t.rows * (R / 4); i += WAVES * 64) {
      const int row = i / (R / 4), c = i - row * (R / 4);
      *(float4*)(D + (t.row + row) * ldd + c * 4) = make_float4(0, 0, 0, 0);
    }
    return;
  }
  const int m = lane & 15, q = lane >> 4;
  const uint8_t* xp[TT];
#pragma unroll
  for (int i = 0; i < TT; i++) xp[i] = X + ((t.row + min(i * 16 + m, t.rows - 1)) * ldx + 16 * q) * EB;
  const uint16_t* wp[RT];
#pragma unroll
  for (int i = 0; i < RT; i++) wp[i] = W + ((int64_t)t.adapter * R + min(i * 16 + m, R - 1)) * ldw + 16 * q;

  f32x4 acc[RT][TT];
#pragma unroll
  for (int i = 0; i < RT; i++)
#pragma unroll
    for (int j = 0; j < TT; j++) acc[i][j] = (f32x4){0, 0, 0, 0};

  for (int k = wave * 64; k < K; k += WAVES * 64) {
    // K is a multiple of 8 (16 in 8 bits): a lane's pieces of eight lie inside the row or behind it
    const bool in0 = k + 16 * q < K, in1 = k + 16 * q + 8 < K;
    uint4 x[TT][2], w[RT][2];
#pragma unroll
    for (int i = 0; i < TT; i++) {
      if (DT == M_BF16) {
        x[i][0] = load16(xp[i] + k * 2, in0);
        x[i][1] = load16(xp[i] + k * 2 + 16, in1);
      } else {
        const uint4 c = load16(xp[i] + k, in0);
        x[i][0] = widen<DT>(make_uint2(c.x, c.y), 1.0f);
        x[i][1] = widen<DT>(make_uint2(c.z, c.w), 1.0f);
      }
    }
#pragma unroll
    for (int i = 0; i < RT; i++) {
      w[i][0] = load16(wp[i] + k, in0);
      w[i][1] = load16(wp[i] + k + 8, in1);
    }
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int i = 0; i < RT; i++)
#pragma unroll
        for (int j = 0; j < TT; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(w[i][h]), frag(x[j][h]), acc[i][j], 0, 0, 0);
  }
  // lane (m, q) holds ranks 4 q .. 4 q + 3 of row m
#pragma unroll
  for (int i = 0; i < RT; i++)
#pragma unroll
    for (int j = 0; j < TT; j++) *(f32x4*)&red[wave][j * 16 + m][i * 16 + 4 * q] = acc[i][j];
  __syncthreads();
  const float s = (scale ? scale[t.adapter] : 1.0f) * x_scale;
  for (int i = tid; i < t.rows * (RP / 4); i += WAVES * 64) {
    const int row = i / (RP / 4), c = (i % (RP / 4)) * 4;
    if (c >= R) continue;
    f32x4 v = *(const f32x4*)&red[0][row][c];
#pragma unroll
    for (int u = 1; u < WAVES; u++) v += *(const f32x4*)&red[u][row][c];
    *(f32x4*)(D + (t.row + row) * ldd + c) = v * s;
  }
}

// ---- up -------------------------------------------------------------------------------------------------------
// A wave takes 128 features and walks the tile's rows 16 at a time.  Lane (n, q) holds eight neighbouring features of ranks 8 q .. 8 q + 7, in
// registers for all rows: eight loads of 16 bytes, transposed in registers, are the operands of eight matrix instructions, the j-th for features
// 8 n + j, so that the results of one row lie 8 in a lane and 128 in 16 lanes, 256 bytes in a row of base and out.
template <int RP, int TR>
__global__ void __launch_bounds__(256)
k_adapter_up(AdapterSegments g, const float* __restrict__ D, int64_t ldd, int R, const uint16_t* __restrict__ U, int64_t ldu, int C, int fblocks,
             const uint16_t* base, int64_t ldbase, uint16_t* out, int64_t ldout) {
  constexpr int SETS = RP <= 32 ? 1 : RP / 32;
  const int slot = blockIdx.x / fblocks, fb = blockIdx.x - slot * fblocks;
  const Tile t = find_tile(g, slot, TR);
  if (t.rows <= 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 15, q = lane >> 4, f = (fb * 4 + wave) * 128 + n * 8;
  const bool in = f < C;
  if (t.adapter < 0) {
    if (out == base || !in) return;
    for (int r = q; r < t.rows; r += 4)
      *(uint4*)(out + (t.row + r) * ldout + f) = load16(base + (t.row + r) * ldbase + f, base != nullptr);
    return;
  }
  uint4 b[SETS][8];
#pragma unroll
  for (int s = 0; s < SETS; s++) {
    uint4 x[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const int r = (RP == 16 ? (q & 1) * 8 : s * 32 + q * 8) + i;
      x[i] = load16(U + ((int64_t)t.adapter * R + r) * ldu + f, in && r < R);
    }
    transpose8(x, b[s]);
  }
  for (int r0 = 0; r0 < t.rows; r0 += 16) {
    uint4 old[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = r0 + 4 * q + i;
      old[i] = load16(base + (t.row + r) * ldbase + f, base && in && r < t.rows);
    }
    f32x4 acc[8];
#pragma unroll
    for (int j = 0; j < 8; j++) acc[j] = (f32x4){0, 0, 0, 0};
    const float* d = D + (t.row + min(r0 + n, t.rows - 1)) * ldd;
#pragma unroll
    for (int s = 0; s < SETS; s++) {
      const int r = RP == 16 ? (q & 1) * 8 : s * 32 + q * 8;
      float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (r < R) {
        const float4 u = *(const float4*)(d + r), v = *(const float4*)(d + r + 4);
        x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
      }
      uint4 hi, lo;
      split8(x, hi, lo);
      if (RP == 16) {                                  // hi and lo of 16 ranks fill one instruction's 32 places
        const uint4 a = q < 2 ? hi : lo;
#pragma unroll
        for (int j = 0; j < 8; j++) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(a), frag(b[s][j]), acc[j], 0, 0, 0);
      } else {
#pragma unroll
        for (int j = 0; j < 8; j++) {
          acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(hi), frag(b[s][j]), acc[j], 0, 0, 0);
          acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(lo), frag(b[s][j]), acc[j], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int r = r0 + 4 * q + i;
      if (!in || r >= t.rows) continue;
      uint4 v;
      v.x = bf16_rne_pack(bf16lo_f32(old[i].x) + acc[0][i], bf16hi_f32(old[i].x) + acc[1][i]);
      v.y = bf16_rne_pack(bf16lo_f32(old[i].y) + acc[2][i], bf16hi_f32(old[i].y) + acc[3][i]);
      v.z = bf16_rne_pack(bf16lo_f32(old[i].z) + acc[4][i], bf16hi_f32(old[i].z) + acc[5][i]);
      v.w = bf16_rne_pack(bf16lo_f32(old[i].w) + acc[6][i], bf16hi_f32(old[i].w) + acc[7][i]);
      *(uint4*)(out + (t.row + r) * ldout + f) = v;
    }
  }
}

// ---- outer ----------------------------------------------------------------------------------------------------
// A workgroup takes 128 features of a chunk of rows of one segment, its four waves 32 rows each in turn.  Lane (n, q) loads eight features of
// rows 8 q .. 8 q + 7 (256 bytes of a row in 16 lanes) and transposes them in registers into the operands of eight matrix instructions, as above.
// The waves' sums meet in LDS; the chunk's sum goes to the workspace, and k_adapter_outer_sum adds the chunks of each adapter in order.
template <int MT, int RT>
__global__ void __launch_bounds__(256)
k_adapter_outer(AdapterSegments g, const float* __restrict__ L, int64_t ldl, int R, const uint8_t* __restrict__ M, int64_t ldm, const uint8_t* __restrict__ blocks,
                int64_t ldblocks, int C, int fblocks, int chunk, float* __restrict__ part) {
  constexpr int EB = MT == M_BF16 ? 2 : 1;
  __shared__ float red[4][16][132];
  const int slot = blockIdx.x / fblocks, fb = blockIdx.x - slot * fblocks;
  const Tile t = find_tile(g, slot, chunk);
  if (t.rows <= 0 || t.adapter < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, q = lane >> 4, f = fb * 128 + n * 8;
  const bool in = f < C;
  f32x4 acc[RT][8];
#pragma unroll
  for (int i = 0; i < RT; i++)
#pragma unroll
    for (int j = 0; j < 8; j++) acc[i][j] = (f32x4){0, 0, 0, 0};
  for (int r0 = wave * 32; r0 < t.rows; r0 += 128) {
    uint4 x[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const int r = r0 + q * 8 + i;
      const bool ok = in && r < t.rows;
      const uint8_t* p = M + ((t.row + r) * ldm + f) * EB;
      if (MT == M_BF16) x[i] = load16(p, ok);
      else {
        const uint2 c = load8(p, ok);
        float s = 1.0f;
        if (MT == M_BLOCK && ok) s = u2f((uint32_t)blocks[(t.row + r) * ldblocks + (f >> 5)] << 23);
        x[i] = widen<MT>(c, s);
      }
    }
    uint4 b[8];
    transpose8(x, b);
#pragma unroll
    for (int i = 0; i < RT; i++) {
      float l[8];
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const int r = r0 + q * 8 + e;
        l[e] = r < t.rows && i * 16 + n < R ? L[(t.row + r) * ldl + i * 16 + n] : 0.0f;
      }
      uint4 hi, mid, lo;
      split8(l, hi, mid, lo);
#pragma unroll
      for (int j = 0; j < 8; j++) {
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(hi), frag(b[j]), acc[i][j], 0, 0, 0);
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(mid), frag(b[j]), acc[i][j], 0, 0, 0);
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(lo), frag(b[j]), acc[i][j], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < RT; i++) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; e++)
#pragma unroll
      for (int h = 0; h < 2; h++)
        *(f32x4*)&red[wave][4 * q + e][n * 8 + h * 4] = (f32x4){acc[i][h * 4][e], acc[i][h * 4 + 1][e], acc[i][h * 4 + 2][e], acc[i][h * 4 + 3][e]};
    __syncthreads();
    for (int u = tid; u < 512; u += 256) {
      const int r = u >> 5, c = (u & 31) * 4;
      if (i * 16 + r < R && fb * 128 + c < C) {
        f32x4 v = *(const f32x4*)&red[0][r][c];
        v += *(const f32x4*)&red[1][r][c];
        v += *(const f32x4*)&red[2][r][c];
        v += *(const f32x4*)&red[3][r][c];
        *(f32x4*)(part + ((int64_t)slot * R + i * 16 + r) * C + fb * 128 + c) = v;
      }
    }
  }
}

struct OuterSum {
  const float* part;
  float* G;
  int64_t ldg;
  float scale;
  int C;
};
// Adds the chunks of adapter n in the order of their rows.
__global__ void __launch_bounds__(256)
k_adapter_outer_sum(AdapterSegments g, int R, int chunk, OuterSum a, OuterSum b, int ablocks, int accumulate) {
  const bool second = (int)blockIdx.x >= ablocks;
  const OuterSum s = second ? b : a;
  const int f = ((int)(second ? blockIdx.x - ablocks : blockIdx.x) * 256 + (int)threadIdx.x) * 4, r = blockIdx.y, n = blockIdx.z;
  if (f >= s.C) return;
  f32x4 sum = {0, 0, 0, 0};
  for (int v = 1; v <= g.segments; v++) {
    if (g.adapter[v - 1] != n) continue;
    const int rows = segment_bound(g, v + 1) - segment_bound(g, v);
    if (rows <= 0) continue;
    const int first = first_slot(g, v, chunk), last = min(first + (rows - 1) / chunk + 1, first_slot(g, v + 1, chunk));
#pragma unroll 4
    for (int k = first; k < last; k++) sum += *(const f32x4*)(s.part + ((int64_t)k * R + r) * s.C + f);
  }
  float* p = s.G + ((int64_t)n * R + r) * s.ldg + f;
  sum *= s.scale;
  if (accumulate) sum += *(const f32x4*)p;
  *(f32x4*)p = sum;
}

int mode(int dtype) { return dtype == SSTE_F8E4M3 ? M_E4M3 : dtype == SSTE_F8E5M2 ? M_E5M2 : dtype == SSTE_F8BLOCK ? M_BLOCK : M_BF16; }
int padded_rank(int R) { return R <= 16 ? 16 : R <= 32 ? 32 : R <= 64 ? 64 : 128; }

template <int DT, int RP, int TT, int WAVES>
void down(const AdapterApply& a, hipStream_t s) {
  SSTE_LAUNCH(SSTE_K_ADAPTER, (k_adapter_down<DT, RP / 16, TT, WAVES>), dim3((unsigned)slots(a.seg, TT * 16)), dim3(WAVES * 64), s, a.seg, (const uint8_t*)a.X, a.ldx, a.K,
              (const uint16_t*)a.down, a.lddown, a.R, a.scale, a.x_scale, a.D, a.ldd);
}
template <int RP, int TR>
void up(const AdapterApply& a, hipStream_t s) {
  const int fblocks = (a.C + 511) / 512;
  SSTE_LAUNCH(SSTE_K_ADAPTER, (k_adapter_up<RP, TR>), dim3((unsigned)(slots(a.seg, TR) * fblocks)), dim3(256), s, a.seg, a.D, a.ldd, a.R, (const uint16_t*)a.up, a.ldup, a.C,
              fblocks, (const uint16_t*)a.base, a.ldbase, (uint16_t*)a.out, a.ldout);
}
template <int RP>
void apply(const AdapterApply& a, hipStream_t s) {
  const bool large = a.seg.T >= 8192;
  constexpr int TT = RP <= 64 ? 4 : 2, WL = 4, WS = 8;
  switch (mode(a.dtype)) {
    case M_BF16: large ? down<M_BF16, RP, TT, WL>(a, s) : down<M_BF16, RP, 1, WS>(a, s); break;
    case M_E4M3: large ? down<M_E4M3, RP, TT, WL>(a, s) : down<M_E4M3, RP, 1, WS>(a, s); break;
    default: large ? down<M_E5M2, RP, TT, WL>(a, s) : down<M_E5M2, RP, 1, WS>(a, s); break;
  }
  if (a.C > 0) large ? up<RP, 64>(a, s) : up<RP, 16>(a, s);
}

int outer_chunk(int64_t T, int64_t I, int64_t O) {
  // about 1024 workgroups of 128 features, whole rounds of 128 rows
  const int64_t blocks = (I + 127) / 128 + (O + 127) / 128;
  int64_t chunk = T * blocks / 1024 / 128 * 128;
  if (chunk < 128) chunk = 128;
  if (chunk > 1 << 20) chunk = 1 << 20;
  return (int)chunk;
}

template <int MT>
void outer(const AdapterSegments& g, int R, const AdapterOuter& a, int chunk, float* part, hipStream_t s) {
  const int fblocks = (a.C + 127) / 128;
  const dim3 grid((unsigned)(slots(g, chunk) * fblocks));
#define OUTER(RT) \
  SSTE_LAUNCH(SSTE_K_ADAPTER, (k_adapter_outer<MT, RT>), grid, dim3(256), s, g, a.L, a.ldl, R, (const uint8_t*)a.M, a.ldm, a.blocks, a.ldblocks, a.C, fblocks, chunk, part)
  switch (padded_rank(R)) {
    case 16: OUTER(1); break;
    case 32: OUTER(2); break;
    case 64: OUTER(4); break;
    default: OUTER(8); break;
  }
#undef OUTER
}

}  // namespace

hipError_t launch_adapter_apply(const AdapterApply& a, hipStream_t s) {
  if (a.seg.T == 0) return hipSuccess;
  switch (padded_rank(a.R)) {
    case 16: apply<16>(a, s); break;
    case 32: apply<32>(a, s); break;
    case 64: apply<64>(a, s); break;
    default: apply<128>(a, s); break;
  }
  return hipGetLastError();
}

size_t adapter_wgrad_workspace_bytes(int64_t T, int segments, int R, int64_t I, int64_t O) {
  if (T == 0) return 0;
  const AdapterSegments g = {nullptr, nullptr, segments, 0, (int)T};
  return (size_t)slots(g, outer_chunk(T, I, O)) * (size_t)R * (size_t)(I + O) * 4;
}

hipError_t launch_adapter_wgrad(const AdapterSegments& g, int R, const AdapterOuter& a, const AdapterOuter& b, int accumulate, void* ws, hipStream_t s) {
  const int chunk = outer_chunk(g.T, a.C, b.C);
  float* part[2] = {(float*)ws, (float*)ws + slots(g, chunk) * R * a.C};
  const AdapterOuter* both[2] = {&a, &b};
  if (g.T > 0)
    for (int k = 0; k < 2; k++) {
      if (both[k]->C == 0) continue;
      switch (mode(both[k]->m_dtype)) {
        case M_BF16: outer<M_BF16>(g, R, *both[k], chunk, part[k], s); break;
        case M_E4M3: outer<M_E4M3>(g, R, *both[k], chunk, part[k], s); break;
        case M_E5M2: outer<M_E5M2>(g, R, *both[k], chunk, part[k], s); break;
        default: outer<M_BLOCK>(g, R, *both[k], chunk, part[k], s); break;
      }
    }
  const int ablocks = (a.C + 1023) / 1024, bblocks = (b.C + 1023) / 1024;
  if (ablocks + bblocks > 0 && g.adapters > 0)
    SSTE_LAUNCH(SSTE_K_ADAPTER, k_adapter_outer_sum, dim3((unsigned)(ablocks + bblocks), (unsigned)R, (unsigned)g.adapters), dim3(256), s, g, R, chunk,
                (OuterSum{part[0], a.G, a.ldg, a.m_scale, a.C}), (OuterSum{part[1], b.G, b.ldg, b.m_scale, b.C}), ablocks, accumulate);
  return hipGetLastError();
}

}  // namespace sste
