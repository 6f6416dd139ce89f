// Low-rank adapters beside a shared projection: every row of a batch has its own adapter, or none.
//
//   down   D = scale_n X down_n^T               T x R, float32       S of the forward pass (down = A), dS of the input gradient (down = B)
//   up     out = base + D up_n                  T x C, bf16          Z (up = B), dX (up = A)
//   outer  G_n = sum over rows of n of L^T M    R x C, float32       dA (L = dS, M = X), dB (L = S, M = dZ)
//
// A and B are both kept rank-major (R x I, R x O), so the forward pass and the input gradient are the same two kernels with A and B
// exchanged, and the two weight gradients are one.  The rank is small: all three are bound by the bytes of X, base, out and M.  TB/s in these comments count
// what a kernel has to read and write, once each.
#include "adapter.h"

#include <cmath>

namespace sste {

namespace {

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// ---- rows to tiles --------------------------------------------------------------------------------------------
// The grids are sized from T and the number of segments alone; the segments' bounds stay on the device.  With the rows before the first
// and behind the last segment as two more (without an adapter), bounds b_0 = 0 <= b_1 <= ... <= b_{S+2} = T, segment v's tiles of TR rows
// take the slots from floor(b_v / TR) + v on: floor(b_{v+1} / TR) - floor(b_v / TR) + 1 slots, never fewer than its tiles.
// Bounds are clamped to 0 .. T, so that no array of bounds leads outside the matrices.
struct Tile {
  int64_t row;    // first row
  int rows;       // 0: an empty slot
  int adapter;    // -1: none
};
__device__ __forceinline__ int segment_bound(const AdapterSegments& g, int v) {
  if (v <= 0) return 0;
  if (v >= g.segments + 2 || g.segments == 0) return g.T;              // without segments there may be no arrays
  return min(max(g.row_start[v - 1], 0), g.T);
}
__device__ __forceinline__ int first_slot(const AdapterSegments& g, int v, int tr) { return (int)((uint32_t)segment_bound(g, v) / (uint32_t)tr) + v; }
__device__ __forceinline__ int segment_adapter(const AdapterSegments& g, int v) {
  if (v <= 0 || v > g.segments) return -1;
  const int n = g.adapter[v - 1];
  return n >= 0 && n < g.adapters ? n : -1;
}
// Every wave finds its tile by itself, 64 probes a round.  The last round (the only one up to 62 segments) has the adapters and the bounds that
// follow among its probes, so that a workgroup waits for one load before it knows its rows.
__device__ __forceinline__ Tile find_tile(const AdapterSegments& g, int slot, int tr) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = g.segments + 2;
  while (n > 63) {
    const int step = (n + 63) / 64;
    const int v = lo + lane * step;
    const bool before = lane * step < n && first_slot(g, v, tr) <= slot;
    const uint64_t mask = __ballot(before) | 1;
    const int hit = 63 - __clzll((long long)mask);
    n = min(step, n - hit * step);
    lo += hit * step;
  }
  const int v = lo + lane, bound = segment_bound(g, v), adapter = segment_adapter(g, v);
  const uint64_t mask = __ballot(lane < n && (int)((uint32_t)bound / (uint32_t)tr) + v <= slot) | 1;
  const int hit = __builtin_amdgcn_readfirstlane(63 - __clzll((long long)mask));       // at most 62: the next lane has the next bound
  const int b0 = __builtin_amdgcn_readlane(bound, hit), b1 = __builtin_amdgcn_readlane(bound, hit + 1);
  // (Divisions leave their results in vector registers; as scalars again, or every descriptor made from them costs a loop over the lanes.)
  Tile t;
  const int64_t row = b0 + (int64_t)(slot - (int)((uint32_t)b0 / (uint32_t)tr) - lo - hit) * tr;
  t.row = uniform((int)min(row, (int64_t)g.T));
  t.rows = uniform((int)max(min((int64_t)tr, b1 - row), (int64_t)0));
  t.adapter = __builtin_amdgcn_readlane(adapter, hit);
  return t;
}
// Workgroups go to the eight XCDs in turn: `grouped`, the `parts` of a slot are on one of them, whose L2 has what they share after the first (slots are
// rounded up to a multiple of eight, and the last may be empty).
struct Share {
  int parts;
  bool grouped;
  uint32_t magic;       // i / parts = i * magic >> shift for i < 2^25
  int shift;
};
Share share_of(int parts, bool grouped) {
  int bits = 0;
  while ((1 << bits) < parts) bits++;
  return {parts, grouped, (uint32_t)(((1ull << (25 + bits)) + parts - 1) / parts), 25 + bits};
}
struct Work {
  int slot, part;
};
// (All of it in scalar registers: a division would go through vector registers, and its results back.)
__device__ __forceinline__ Work work_of(Share s) {
  const int shift = s.grouped ? 3 : 0, i = (int)blockIdx.x >> shift, group = (int)((uint64_t)(uint32_t)i * s.magic >> s.shift);
  return {(group << shift) + ((int)blockIdx.x - (i << shift)), i - group * s.parts};
}
unsigned grid_of(int64_t slots, Share s) { return (unsigned)((s.grouped ? (slots + 7) / 8 * 8 : slots) * s.parts); }
int64_t slots(const AdapterSegments& g, int tr) { return (int64_t)g.T / tr + g.segments + 2; }

// ---- operands -------------------------------------------------------------------------------------------------
// Consecutive elements as bf16, times a power of two.  8-bit formats convert exactly (e4m3 and e5m2 are subsets of bf16).
enum { M_BF16 = 0, M_E4M3 = 1, M_E5M2 = 2, M_BLOCK = 3 };
template <int DT>
__device__ __forceinline__ void widen4(uint32_t& lo, uint32_t& hi, uint32_t c, float s) {
  bf16x2 v[2];
  if (DT == M_E5M2) {
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c, s, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c, s, true);
  } else {
    v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, false);
    v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, true);
  }
  __builtin_memcpy(&lo, &v[0], 4);
  __builtin_memcpy(&hi, &v[1], 4);
}
template <int DT>
__device__ __forceinline__ uint4 widen(uint2 c, float s) {
  uint4 r;
  widen4<DT>(r.x, r.y, c.x, s);
  widen4<DT>(r.z, r.w, c.y, s);
  return r;
}
__device__ __forceinline__ bf16x8 frag(uint4 v) {
  bf16x8 r;
  __builtin_memcpy(&r, &v, 16);
  return r;
}
// Two floats as sums of three bf16 each, which have all of their bits: S and dS are 32-bit sums, and neither the weight gradients nor the products with B and A
// are to see them rounded (where base and S B cancel, a bf16 result shows even two parts' 2^-17).  Each part is cut off, not rounded: 8 of 24 bits, 8 of the
// 16 that are left, and the last 8; rounded up, the first would be infinite from 2^128 (1 - 2^-9) on.
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  const auto cut = [&] {
    const uint32_t r = __builtin_amdgcn_perm(f2u(b), f2u(a), 0x07060302u);
    a -= bf16lo_f32(r), b -= bf16hi_f32(r);
    return r;
  };
  hi = cut();
  mid = cut();
  lo = cut();
}
__device__ __forceinline__ void split8(const float (&x)[8], uint4& hi, uint4& mid, uint4& lo) {
  uint32_t h[4], m[4], l[4];
#pragma unroll
  for (int p = 0; p < 4; p++) split2(x[2 * p], x[2 * p + 1], h[p], m[p], l[p]);
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  mid = make_uint4(m[0], m[1], m[2], m[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}
// Transposes a block of eight rows of eight 16-bit elements held by one lane: b[j] holds rows 0 .. 7 of element j.
__device__ __forceinline__ void transpose_rows(const uint32_t (&x)[8][4], uint4 (&b)[8]) {
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
    const int k = j >> 1;
    b[j] = make_uint4(__builtin_amdgcn_perm(x[1][k], x[0][k], sel), __builtin_amdgcn_perm(x[3][k], x[2][k], sel), __builtin_amdgcn_perm(x[5][k], x[4][k], sel),
                      __builtin_amdgcn_perm(x[7][k], x[6][k], sel));
  }
}

// ---- guarded memory -------------------------------------------------------------------------------------------
// Rows and elements that a tile does not have are left to the descriptor's range check: loads give zeros, stores nothing, without a branch around each
// (a branch a load costs more registers than it saves, since the loads can no longer be moved together).  A descriptor covers a tile's rows of one
// matrix, at most 2^31 bytes (leading dimensions are at most 2^23), so an offset of kNowhere lies behind every one.
constexpr uint32_t kNowhere = 0x80000000u;
template <class T>
__device__ __forceinline__ BufferRsrc rows_of(const T* base, int64_t first, int rows, int64_t ld, int width) {
  return make_rsrc(base + first * ld, rows > 0 && base ? ((uint32_t)(rows - 1) * (uint32_t)ld + (uint32_t)width) * (uint32_t)sizeof(T) : 0u);
}
__device__ __forceinline__ void buffer_store_b128(BufferRsrc r, uint32_t voffset, uint4 v) {
  i32x4 t;
  __builtin_memcpy(&t, &v, 16);
  __builtin_amdgcn_raw_buffer_store_b128(t, r, (int)voffset, 0, 0);
}

// ---- down and up ----------------------------------------------------------------------------------------------
// Down, for 16 TT rows of one adapter and the contraction's elements k0 .. k1 - 1, by a workgroup of eight waves: KC elements at a time go through LDS,
// of the rows and of the adapter, loaded in whole pieces of a row (the operands' own layout has a different row in every lane, at a quarter of the load
// rate) and kept two chunks ahead in registers.  A wave multiplies one step of 32 elements of each chunk; where a chunk has fewer steps than there are
// waves, the waves share the ranks out as well.  The sums of the steps' waves meet in LDS, in the order of the steps.
// Bound by HBM with few ranks (32768 e4m3 rows of 1280, rank 32: 17 us, 2.7 TB/s, the read of X and the write of D; 16384 bf16
// rows of 4096, rank 16: 30 us, 4.5 TB/s), by the adapter's way through L2 and LDS with many (5003 e5m2 rows of 3840, rank 128: 17 us).
// Elements of a chunk: as many as leave room for two or three workgroups a CU; for few rows, where the chunks' latency adds up, twice as many for rank 32 (one
// row of 1280 -> 3840: 5.7 us against 9.6) and 128 (one row of 1280 -> 1280: 10.5 against 12.1), not for 64 (64 rows of their own 16.1, against 20.8).
constexpr int down_chunk(int padded_rank, int rows) {
  return padded_rank == 16 ? 256 : padded_rank == 32 ? (rows == 16 ? 256 : 128) : padded_rank == 64 ? 128 : rows == 16 ? 128 : 64;
}
template <int DT, int RT, int TT>
struct Down {
  static constexpr int RP = RT * 16, TR = TT * 16, EB = DT == M_BF16 ? 2 : 1;
  static constexpr int KC = down_chunk(RP, TR), STEPS = KC / 32, GROUPS = 8 / STEPS;               // a chunk, its steps, the waves that share a step
  static constexpr int RW = RT / GROUPS;                                                          // by ranks; every wave has all rows: fewest operands a result
  static constexpr int LDK = KC + 8, LD = RP + 4;                                                  // LDS rows start four banks apart
  static constexpr int PC = KC / 8, XP = (TR * PC + 511) / 512, WP = RP * PC / 512;                // pieces of eight elements: of a row, a thread's
  static_assert(RP * PC % 512 == 0 && (TR * PC % 512 == 0 || 512 % (TR * PC) == 0), "whole rounds of pieces");
  static constexpr int STAGE = (TR + RP) * LDK * 2, RED = STEPS * TR * LD * 4, LDS = 2 * STAGE > RED ? 2 * STAGE : RED;
  template <bool BITS8> struct Raw { using T = uint4; };
  template <> struct Raw<true> { using T = uint2; };
  struct Chunk { typename Raw<DT != M_BF16>::T x[XP]; uint4 w[WP]; };

  // Leaves the steps' sums in lds as float [STEPS][TR][LD], behind a barrier.
  static __device__ __forceinline__ void run(uint8_t* lds, const Tile& t, const uint8_t* __restrict__ X, int64_t ldx, int K, int k0, int k1, const uint16_t* __restrict__ W, int64_t ldw, int R) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, q = lane >> 4;
    const int step = wave % STEPS, r0 = wave / STEPS * RW;
    f32x4 acc[RW][TT];
#pragma unroll
    for (int i = 0; i < RW; i++)
#pragma unroll
      for (int j = 0; j < TT; j++) acc[i][j] = (f32x4){0, 0, 0, 0};
    // Rows behind the tile's, ranks behind R and elements behind k1 are zeros; nothing is read for them.
    const BufferRsrc rx = make_rsrc(X + t.row * ldx * EB, ((uint32_t)(t.rows - 1) * (uint32_t)ldx + (uint32_t)K) * EB);
    const BufferRsrc rw = rows_of(W, (int64_t)t.adapter * R, R, ldw, K);
    auto load = [&](Chunk& c, int k) {
#pragma unroll
      for (int i = 0; i < XP; i++) {
        const int p = (i * 512 + tid) % (TR * PC), r = p / PC, e = k + p % PC * 8;      // of fewer pieces than threads some are loaded twice
        const uint32_t at = e < k1 ? ((uint32_t)r * (uint32_t)ldx + (uint32_t)e) * EB : kNowhere;
        if constexpr (DT == M_BF16) c.x[i] = buffer_load_b128(rx, at, 0);
        else c.x[i] = buffer_load_b64(rx, at, 0);
      }
#pragma unroll
      for (int i = 0; i < WP; i++) {
        const int p = i * 512 + tid, r = p / PC, e = k + p % PC * 8;
        c.w[i] = buffer_load_b128(rw, e < k1 ? ((uint32_t)r * (uint32_t)ldw + (uint32_t)e) * 2 : kNowhere, 0);
      }
    };
    auto put = [&](const Chunk& c, int buffer) {
      uint8_t* to = lds + buffer * STAGE;
#pragma unroll
      for (int i = 0; i < XP; i++) {
        const int p = (i * 512 + tid) % (TR * PC), r = p / PC;
        uint4* d = (uint4*)(to + (r * LDK + p % PC * 8) * 2);
        if constexpr (DT == M_BF16) *d = c.x[i];
        else *d = widen<DT>(c.x[i], 1.0f);
      }
#pragma unroll
      for (int i = 0; i < WP; i++) {
        const int p = i * 512 + tid, r = p / PC;
        *(uint4*)(to + ((TR + r) * LDK + p % PC * 8) * 2) = c.w[i];
      }
    };
    auto multiply = [&](int buffer) {
      const uint16_t* from = (const uint16_t*)(lds + buffer * STAGE) + step * 32 + q * 8;
      uint4 x[TT];
#pragma unroll
      for (int j = 0; j < TT; j++) x[j] = *(const uint4*)(from + (j * 16 + m) * LDK);
#pragma unroll
      for (int i = 0; i < RW; i++) {
        const uint4 w = *(const uint4*)(from + (TR + (r0 + i) * 16 + m) * LDK);
#pragma unroll
        for (int j = 0; j < TT; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(w), frag(x[j]), acc[i][j], 0, 0, 0);
      }
    };
    // (No branches in here: with one, the compiler waits for every load that is under way where it needs the oldest.)
    Chunk a, b;
    load(a, k0);
    load(b, k0 + KC);
    int k = k0;
    for (; k + KC < k1; k += 2 * KC) {
      put(a, 0);
      __syncthreads();
      load(a, k + 2 * KC);
      multiply(0);
      put(b, 1);                                       // the barrier before is behind the last reads of this buffer
      __syncthreads();
      load(b, k + 3 * KC);
      multiply(1);
    }
    if (k < k1) {
      put(a, 0);
      __syncthreads();
      multiply(0);
    }
    __syncthreads();
    // lane (m, q) holds ranks 4 q .. 4 q + 3 of row m
    float (*red)[TR][LD] = (float (*)[TR][LD])lds;
#pragma unroll
    for (int i = 0; i < RW; i++)
#pragma unroll
      for (int j = 0; j < TT; j++) *(f32x4*)&red[step][j * 16 + m][(r0 + i) * 16 + 4 * q] = acc[i][j];
    __syncthreads();
  }
  // Ranks c .. c + 3 of a row
  static __device__ __forceinline__ f32x4 sum(const uint8_t* lds, int row, int c) {
    const float (*red)[TR][LD] = (const float (*)[TR][LD])lds;
    f32x4 v = *(const f32x4*)&red[0][row][c];
#pragma unroll
    for (int u = 1; u < STEPS; u++) v += *(const f32x4*)&red[u][row][c];
    return v;
  }
};

constexpr int kMostSplits = 4;      // of the contraction of `down`

struct DownArgs {
  const uint8_t* X;
  int64_t ldx;
  int K;
  const uint16_t* W;
  int64_t ldw;
  int R;
  const float* scale;
  float x_scale;
  float* D;
  int64_t ldd;
};
struct UpArgs {
  const uint16_t* U;
  int64_t ldu;
  int C;
  const uint16_t* base;
  int64_t ldbase;
  uint16_t* out;
  int64_t ldout;
};

// A tile's rows of D as the sum of three bf16, and the features of a wave.
template <int RP, int TT>
struct Up {
  static constexpr int TR = TT * 16, LDP = RP + 8, SETS = RP <= 32 ? 1 : RP / 32;
  uint16_t parts[3][TR][LDP];

  // What a wave loads of its features before it needs the tile's D: the first 32 ranks of the adapter, and its rows of base.
  struct Ahead {
    uint32_t x[8][4];
    uint4 old[TT][4];
  };
  static __device__ __forceinline__ void load_ranks(uint32_t (&x)[8][4], int s, BufferRsrc ru, int64_t ldu, uint32_t at) {
    int q = ((int)threadIdx.x & 63) >> 4;
    asm("" : "+v"(q));                                  // offsets anew too (rank 64 in one launch, 200 rows of their own: 23.1 us, with spills 28.9)
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const uint32_t r = (RP == 16 ? (q & 1) * 8 : s * 32 + q * 8) + i;
      const uint4 v = buffer_load_b128(ru, at + r * (uint32_t)ldu * 2, 0);
      x[i][0] = v.x, x[i][1] = v.y, x[i][2] = v.z, x[i][3] = v.w;
    }
  }
  static __device__ __forceinline__ void load(Ahead& a, const Tile& t, int f0, const UpArgs& o, int R) {
    const int lane = threadIdx.x & 63, q = lane >> 4, f = f0 + (lane & 15) * 8;
    const uint32_t at = f < o.C ? (uint32_t)f * 2 : kNowhere;
    load_ranks(a.x, 0, rows_of(o.U, (int64_t)t.adapter * R, R, o.ldu, o.C), o.ldu, at);
    const BufferRsrc rb = rows_of(o.base, t.row, t.rows, o.ldbase, o.C);
#pragma unroll
    for (int j = 0; j < TT; j++)
#pragma unroll
      for (int i = 0; i < 4; i++) a.old[j][i] = buffer_load_b128(rb, at + (uint32_t)(j * 16 + 4 * q + i) * (uint32_t)o.ldbase * 2, 0);
  }
  __device__ __forceinline__ void put(int row, int c, f32x4 v) {
    uint2 hi, mid, lo;
    split2(v[0], v[1], hi.x, mid.x, lo.x);
    split2(v[2], v[3], hi.y, mid.y, lo.y);
    *(uint2*)&parts[0][row][c] = hi;
    *(uint2*)&parts[1][row][c] = mid;
    *(uint2*)&parts[2][row][c] = lo;
  }
  // Features f0 .. f0 + 127.  Lane (m, q) loads eight neighbouring features of ranks 8 q .. 8 q + 7 in eight pieces of 16 bytes and transposes them in
  // registers: the operands of eight matrix instructions, the j-th for features 8 m + j, so that the results of one row lie 8 in a lane and 128 in 16
  // lanes, 256 bytes in a row of base and out.
  __device__ __forceinline__ void run(Ahead& a, const Tile& t, int f0, const UpArgs& o, int R) const {
    const int lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4, f = f0 + m * 8;
    const uint32_t at = f < o.C ? (uint32_t)f * 2 : kNowhere;
    const BufferRsrc ru = rows_of(o.U, (int64_t)t.adapter * R, R, o.ldu, o.C), ro = rows_of((const uint16_t*)o.out, t.row, t.rows, o.ldout, o.C);
    f32x4 sum[SETS == 1 ? 1 : TT][8];                    // of one set of ranks the rows are finished 16 at a time
#pragma unroll
    for (int s = 0; s < SETS; s++) {
      uint4 u[8];
      transpose_rows(a.x, u);
      if (s + 1 < SETS) load_ranks(a.x, s + 1, ru, o.ldu, at);
#pragma unroll
      for (int k = 0; k < TT; k++) {
        f32x4 (&c)[8] = sum[SETS == 1 ? 0 : k];
        if (s == 0)
#pragma unroll
          for (int j = 0; j < 8; j++) c[j] = (f32x4){0, 0, 0, 0};
        // Of 16 ranks, hi and mid fill one instruction's 32 places, lo half of another's
        int row = k * 16 + m;
        asm("" : "+v"(row));                              // D from LDS for each 128 features anew: kept over them, it would take registers that the sums need
        const int at_rank = RP == 16 ? (q & 1) * 8 : s * 32 + q * 8;
        const uint4 hi = *(const uint4*)&parts[RP == 16 ? q >> 1 : 0][row][at_rank], mid = *(const uint4*)&parts[1][row][at_rank];
        uint4 lo = *(const uint4*)&parts[2][row][at_rank];
        if (RP == 16 && q >= 2) lo = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 8; j++) {
          c[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(hi), frag(u[j]), c[j], 0, 0, 0);
          if (RP > 16) c[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(mid), frag(u[j]), c[j], 0, 0, 0);
          c[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(lo), frag(u[j]), c[j], 0, 0, 0);
        }
        if (s + 1 < SETS) continue;
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const uint4 old = a.old[k][i];
          uint4 v;
          v.x = bf16_rne_pack(bf16lo_f32(old.x) + c[0][i], bf16hi_f32(old.x) + c[1][i]);
          v.y = bf16_rne_pack(bf16lo_f32(old.y) + c[2][i], bf16hi_f32(old.y) + c[3][i]);
          v.z = bf16_rne_pack(bf16lo_f32(old.z) + c[4][i], bf16hi_f32(old.z) + c[5][i]);
          v.w = bf16_rne_pack(bf16lo_f32(old.w) + c[6][i], bf16hi_f32(old.w) + c[7][i]);
          buffer_store_b128(ro, at + (uint32_t)(k * 16 + 4 * q + i) * (uint32_t)o.ldout * 2, v);
        }
      }
    }
  }
};

// Rows without an adapter: D is zero, out is base
__device__ __forceinline__ void bare_rows(const Tile& t, float* D, int64_t ldd, int R) {
  for (int i = threadIdx.x; i < t.rows * (R / 4); i += blockDim.x) {
    const int row = i / (R / 4), c = i - row * (R / 4);
    *(float4*)(D + (t.row + row) * ldd + c * 4) = make_float4(0, 0, 0, 0);
  }
}
__device__ __forceinline__ void bare_features(const Tile& t, int f0, int C, const uint16_t* base, int64_t ldbase, uint16_t* out, int64_t ldout) {
  const int lane = threadIdx.x & 63, f = f0 + (lane & 15) * 8;
  if (out == base || f >= C) return;
  for (int r = lane >> 4; r < t.rows; r += 4) *(uint4*)(out + (t.row + r) * ldout + f) = load16(base + (t.row + r) * ldbase + f, base != nullptr);
}

__device__ __forceinline__ float scale_of(const DownArgs& a, const Tile& t) { return (a.scale ? a.scale[t.adapter] : 1.0f) * a.x_scale; }

// Both products of 16 rows in one launch, for few rows, bound by the launch and four waits for memory in a row (the bounds, the first chunk, the features'
// ranks, the stores; one row of 1280 -> 3840, rank 16: 5.5 us; 96 rows of 64 adapters, 1280 -> 5120: 8.6 us, 1.8 TB/s, with a fifth wait for a second round of the search): `slices`
// workgroups share a tile's features, and each computes D for itself (five times here, 41 KB of the adapter through L2 each).
template <int DT, int RT>
__global__ void __launch_bounds__(512, RT <= 4 ? 4 : 2)      // two workgroups a CU up to rank 64 (200 rows of their own, 2560 -> 2560: 23.1 us against 29.4)
k_adapter_both(AdapterSegments g, DownArgs d, UpArgs o, Share share) {
  using D = Down<DT, RT, 1>;
  __shared__ __align__(16) uint8_t lds[D::LDS];
  __shared__ __align__(16) Up<RT * 16, 1> up;
  const Work w = work_of(share);
  const int slice = w.part, slices = share.parts;
  const Tile t = find_tile(g, w.slot, 16);
  if (t.rows <= 0) return;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  if (t.adapter < 0) {
    if (slice == 0) bare_rows(t, d.D, d.ldd, d.R);
    for (int f = (slice * 8 + wave) * 128; f < o.C; f += slices * 1024) bare_features(t, f, o.C, o.base, o.ldbase, o.out, o.ldout);
    return;
  }
  const float s = scale_of(d, t);
  D::run(lds, t, d.X, d.ldx, d.K, 0, d.K, d.W, d.ldw, d.R);
  for (int i = threadIdx.x; i < 16 * RT * 4; i += 512) {
    const int row = i / (RT * 4), c = i % (RT * 4) * 4;
    f32x4 v = D::sum(lds, row, c) * s;
    if (c >= d.R) v = (f32x4){0, 0, 0, 0};                                       // ranks of the padding, where s may be anything
    if (slice == 0 && row < t.rows && c < d.R) *(f32x4*)(d.D + (t.row + row) * d.ldd + c) = v;
    up.put(row, c, v);
  }
  __syncthreads();
  for (int f = (slice * 8 + wave) * 128; f < o.C; f += slices * 1024) {
    typename Up<RT * 16, 1>::Ahead a;
    up.load(a, t, f, o, d.R);
    up.run(a, t, f, o, d.R);
  }
}

// Down alone.  splits > 1: `splits` workgroups share a tile's contraction, `span` elements each, and leave their sums, unscaled, in part[split][row][rank].
template <int DT, int RT, int TT>
__global__ void __launch_bounds__(512)
k_adapter_down(AdapterSegments g, DownArgs d, int splits, int span, float* __restrict__ part) {
  using D = Down<DT, RT, TT>;
  __shared__ __align__(16) uint8_t lds[D::LDS];
  const int slot = uniform((int)blockIdx.x / splits), split = (int)blockIdx.x - slot * splits;
  const Tile t = find_tile(g, slot, TT * 16);
  if (t.rows <= 0) return;
  if (t.adapter < 0) {
    if (split == 0) bare_rows(t, d.D, d.ldd, d.R);
    return;
  }
  const float s = splits > 1 ? 1.0f : scale_of(d, t);
  D::run(lds, t, d.X, d.ldx, d.K, split * span, min(d.K, (split + 1) * span), d.W, d.ldw, d.R);
  float* to = splits > 1 ? part + ((int64_t)split * g.T + t.row) * d.R : d.D + t.row * d.ldd;
  const int64_t ld = splits > 1 ? d.R : d.ldd;
  for (int i = threadIdx.x; i < t.rows * (RT * 4); i += 512) {
    const int row = i / (RT * 4), c = i % (RT * 4) * 4;
    if (c < d.R) *(f32x4*)(to + row * ld + c) = D::sum(lds, row, c) * s;
  }
}

// Up alone, 512 features of a tile's rows in a workgroup of four waves.  Bound by HBM, base read and out written (32768 rows of 5120, rank 32: 118 us, 5.7 TB/s;
// 16384 rows of 1024, rank 16, with two partial sums: 16.8 us, 4.2 TB/s), with rank 128 by the adapter's way through L2 too (5003 rows of 1280: 12.9 us).  splits > 1:
// adds the splits' sums in order and scales them; the workgroups of the first features write D.
template <int RP, int TT>
__global__ void __launch_bounds__(256, RP <= 32 ? 3 : 2)
k_adapter_up(AdapterSegments g, DownArgs d, UpArgs o, Share share, int splits, const float* __restrict__ part) {
  __shared__ __align__(16) Up<RP, TT> up;
  const Work w = work_of(share);
  const int fb = w.part;
  const Tile t = find_tile(g, w.slot, TT * 16);
  if (t.rows <= 0) return;
  const int f = (fb * 4 + ((int)threadIdx.x >> 6)) * 128;
  if (t.adapter < 0) {
    bare_features(t, f, o.C, o.base, o.ldbase, o.out, o.ldout);
    return;
  }
  typename Up<RP, TT>::Ahead a;
  up.load(a, t, f, o, d.R);
  const float s = splits > 1 ? scale_of(d, t) : 1.0f;
  const float* from = splits > 1 ? part + t.row * d.R : d.D + t.row * d.ldd;
  const int64_t ld = splits > 1 ? d.R : d.ldd;
  for (int i = threadIdx.x; i < TT * RP * 4; i += 256) {
    const int row = i / (RP / 4), c = i % (RP / 4) * 4;
    f32x4 v = {0, 0, 0, 0};
    if (row < t.rows && c < d.R) {
      v = *(const f32x4*)(from + row * ld + c);
      if (splits > 1) {
        f32x4 more[kMostSplits - 1];                   // all under way at once
#pragma unroll
        for (int k = 1; k < kMostSplits; k++) {
          more[k - 1] = (f32x4){0, 0, 0, 0};
          if (k < splits) more[k - 1] = *(const f32x4*)(from + ((int64_t)k * g.T + row) * d.R + c);
        }
#pragma unroll
        for (int k = 1; k < kMostSplits; k++) v += more[k - 1];
        v *= s;
        if (fb == 0) *(f32x4*)(d.D + (t.row + row) * d.ldd + c) = v;
      }
    }
    up.put(row, c, v);
  }
  __syncthreads();
  if (f < o.C) up.run(a, t, f, o, d.R);
}

// ---- outer ----------------------------------------------------------------------------------------------------
// A workgroup of four waves takes 256 features of a chunk of rows of one segment and up to 64 ranks, 64 rows at a time: a wave 128 features and half the
// rows.  Lane (n, q) loads eight features of rows 8 q .. 8 q + 7 (256 bytes of a row in 16 lanes), one step ahead, and transposes them in registers into the
// operands of eight matrix instructions.  L is split into its three parts once per workgroup: each wave prepares its share of the operands and leaves them
// in LDS for the others; at the end the waves of the same features join their sums there.
// The chunk's sum goes to the workspace, and k_adapter_outer_sum adds the chunks of each adapter in order.  The sums' bytes are what costs with many ranks:
// with all four waves on the same rows (512 features, chunks of half the rows for as many workgroups) 7777 ragged rows of 1280 + 5120, rank 64, take 54 us
// against 47, 32768 rows 131 against 125; rank 16 is the same to 2 %.  Kept in registers, without LDS, L would have to be split by every wave.
// Bound by HBM with few ranks (16384 rows of 1024 + 4096, rank 16: 40 us, 4.2 TB/s, and 5.5 for the sums), by the sums' bytes and, from rank 64 on, the matrix
// instructions of three parts (16384 rows of 1280 + 5120, rank 128: 105 us, 80 GFLOP of them).
// Both weight gradients are one launch, the workgroups of X before those of dZ.  With more than 64 ranks two workgroups work on the same rows and features,
// eight apart in the grid, which is the same XCD: the second finds them in its L2.
struct OuterArgs {
  const float* L;
  int64_t ldl;
  const uint8_t* M;
  int64_t ldm;
  int type;
  const uint8_t* blocks;
  int64_t ldblocks;
  int C, fblocks;
  float* part;
};
// Raw elements of eight rows, eight features of each, and a checkpoint's scale bytes; and the same as operands.
template <bool BITS8>
struct OuterRows {
  static constexpr int WORDS = BITS8 ? 2 : 4;
  uint32_t x[8][WORDS];
  uint32_t e[BITS8 ? 8 : 1];

  static __device__ __forceinline__ void words(uint32_t (&to)[WORDS], BufferRsrc r, uint32_t at) {
    if constexpr (BITS8) {
      const uint2 v = buffer_load_b64(r, at, 0);
      to[0] = v.x, to[1] = v.y;
    } else {
      const uint4 v = buffer_load_b128(r, at, 0);
      to[0] = v.x, to[1] = v.y, to[2] = v.z, to[3] = v.w;
    }
  }
  // `f`: the lane's features, or kNowhere
  __device__ __forceinline__ void load(const OuterArgs& a, const Tile& t, int r0, uint32_t f) {
    uint32_t q8 = (((uint32_t)threadIdx.x & 63) >> 4) * 8;
    asm("" : "+v"(q8));                                // offsets anew in each step: kept, they would take registers that the sums need
    const int rows = min(t.rows - r0, 32);
    const BufferRsrc r = BITS8 ? rows_of(a.M, t.row + r0, rows, a.ldm, a.C) : rows_of((const uint16_t*)a.M, t.row + r0, rows, a.ldm, a.C);
#pragma unroll
    for (int i = 0; i < 8; i++) words(x[i], r, f == kNowhere ? f : ((q8 + i) * (uint32_t)a.ldm + f) * (BITS8 ? 1 : 2));
    if constexpr (BITS8) {
      const BufferRsrc rs = rows_of(a.type == M_BLOCK ? a.blocks : nullptr, t.row + r0, rows, a.ldblocks, (a.C + 31) / 32);
#pragma unroll
      for (int i = 0; i < 8; i++)
        e[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rs, (int)(f == kNowhere ? f : (q8 + i) * (uint32_t)a.ldblocks + (f >> 5)), 0, 0);
    }
  }
  // Rows of a list; `f` is a feature that there is
  __device__ __forceinline__ void load(const OuterArgs& a, const int* rows, int f) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const int64_t row = rows[i];
      if constexpr (BITS8) {
        const uint2 v = *(const uint2*)(a.M + row * a.ldm + f);
        x[i][0] = v.x, x[i][1] = v.y;
        e[i] = 127;
        if (a.type == M_BLOCK) e[i] = a.blocks[row * a.ldblocks + (f >> 5)];
      } else {
        const uint4 v = *(const uint4*)(a.M + (row * a.ldm + f) * 2);
        x[i][0] = v.x, x[i][1] = v.y, x[i][2] = v.z, x[i][3] = v.w;
      }
    }
  }
  // b[j]: rows 0 .. 7 of feature j
  __device__ __forceinline__ void operands(uint4 (&b)[8], int type) const {
    if constexpr (!BITS8) transpose_rows(x, b);
    else {
      uint32_t w[8][4];
      const bool e5m2 = type == M_E5M2, blocks = type == M_BLOCK;
      if (e5m2) {
#pragma unroll
        for (int i = 0; i < 8; i++)
#pragma unroll
          for (int k = 0; k < 2; k++) widen4<M_E5M2>(w[i][2 * k], w[i][2 * k + 1], x[i][k], 1.0f);
      } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
#pragma unroll
          for (int k = 0; k < 2; k++) widen4<M_E4M3>(w[i][2 * k], w[i][2 * k + 1], x[i][k], u2f(blocks ? e[i] << 23 : 0x3F800000u));
      }
      transpose_rows(w, b);
    }
  }
};
template <int RT>
struct Outer {
  static constexpr int OPS = 2 * RT, PW = (OPS + 3) / 4;                           // operands of L a step, and a wave's share
  static constexpr int STAGES = 2 * OPS * 3 * 64 * 16, JOIN = 4 * RT * 4 * 64 * 16, LDS = STAGES > JOIN ? STAGES : JOIN;

  template <bool BITS8>
  static __device__ __forceinline__ void run(uint8_t* lds, const OuterArgs& a, const Tile& t, int slot, int fb, int rank0, int R) {
    uint4 (*l)[OPS][3][64] = (uint4 (*)[OPS][3][64])lds;                           // [buffer][rows, ranks][part][lane]
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), fw = wave & 1, rw = wave >> 1;
    const int n = lane & 15, q = lane >> 4, f = (fb * 2 + fw) * 128 + n * 8;
    const bool in = f < a.C;
    const uint32_t at = in ? (uint32_t)f : kNowhere;
    f32x4 acc[RT][8];
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
      for (int j = 0; j < 8; j++) acc[i][j] = (f32x4){0, 0, 0, 0};

    float v[PW][8];
    auto load_l = [&](int r0) {
#pragma unroll
      for (int p = 0; p < PW; p++) {
        const int o = wave + 4 * p, first = r0 + o / RT * 32, rank = rank0 + o % RT * 16 + n;
        uint32_t q8 = (uint32_t)q * 8;
        asm("" : "+v"(q8));
        const BufferRsrc r = rows_of(a.L, t.row + first, min(t.rows - first, 32), a.ldl, R);
#pragma unroll
        for (int e = 0; e < 8; e++)
          v[p][e] = u2f((uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r, (int)(o < OPS && rank < R ? ((q8 + e) * (uint32_t)a.ldl + (uint32_t)rank) * 4 : kNowhere), 0, 0));
      }
    };
    OuterRows<BITS8> m;
    load_l(0);
    m.load(a, t, rw * 32, at);
    int buffer = 0;
    for (int r0 = 0; r0 < t.rows; r0 += 64, buffer ^= 1) {
#pragma unroll
      for (int p = 0; p < PW; p++) {
        const int o = wave + 4 * p;
        if (o < OPS) split8(v[p], l[buffer][o][0][lane], l[buffer][o][1][lane], l[buffer][o][2][lane]);
      }
      __syncthreads();                                 // nobody comes here before it has read the other buffer, which is written next
      uint4 b[8];
      m.operands(b, a.type);
      load_l(r0 + 64);
      m.load(a, t, r0 + 64 + rw * 32, at);
#pragma unroll
      for (int i = 0; i < RT; i++) {
        const int o = rw * RT + i;
        const uint4 hi = l[buffer][o][0][lane], mid = l[buffer][o][1][lane], lo = l[buffer][o][2][lane];
#pragma unroll
        for (int j = 0; j < 8; j++) {
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(hi), frag(b[j]), acc[i][j], 0, 0, 0);
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(mid), frag(b[j]), acc[i][j], 0, 0, 0);
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(lo), frag(b[j]), acc[i][j], 0, 0, 0);
        }
      }
    }
    // lane (n, q) holds ranks 4 q .. 4 q + 3 of features 8 n .. 8 n + 7; of two waves with the same features each takes half of them
    f32x4 (*join)[RT * 4][64] = (f32x4 (*)[RT * 4][64])lds;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
      for (int j = 0; j < 4; j++) join[wave][i * 4 + j][lane] = rw ? acc[i][j] : acc[i][j + 4];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const f32x4 other = join[wave ^ 2][i * 4 + j][lane];
        acc[i][j] = rw ? other + acc[i][j + 4] : acc[i][j] + other;
      }
    if (!in) return;
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int rank = rank0 + i * 16 + 4 * q + e;
        if (rank >= R) continue;
        *(f32x4*)(a.part + ((int64_t)slot * R + rank) * a.C + f + rw * 4) = (f32x4){acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]};
      }
  }
};
template <int RT>
__global__ void __launch_bounds__(256, RT == 1 ? 3 : 2)
k_adapter_outer(AdapterSegments g, OuterArgs x, OuterArgs z, int R, int chunk) {
  using O = Outer<RT>;
  __shared__ __align__(16) uint8_t lds[O::LDS];
  const bool pairs = R > 64;
  const int block = pairs ? (int)blockIdx.x / 16 * 8 + (int)blockIdx.x % 8 : (int)blockIdx.x, rank0 = pairs ? ((int)blockIdx.x / 8 & 1) * 64 : 0;
  const int fblocks = x.fblocks + z.fblocks, slot = uniform(block / fblocks);
  if (slot >= g.T / chunk + g.segments + 2) return;                                // the last pairs may be empty
  int fb = block - slot * fblocks;
  const bool second = fb >= x.fblocks;
  const OuterArgs a = second ? z : x;
  if (second) fb -= x.fblocks;
  const Tile t = find_tile(g, slot, chunk);
  if (t.rows <= 0 || t.adapter < 0) return;
  if (a.type == M_BF16) O::template run<false>(lds, a, t, slot, fb, rank0, R);
  else O::template run<true>(lds, a, t, slot, fb, rank0, R);
}

struct OuterSum {
  const float* part;
  float* G;
  int64_t ldg;
  float scale;
  int C;
};
// Adds the chunks of adapter n in a fixed order.  Bound by the reads, which mostly come from the last-level cache (34 MB in 9 us), and where there are few
// features, ranks and adapters by the waits for eight chunks after eight: then (`shares` 4, otherwise 1) a workgroup's waves take eight of them each in turn
// for the same 256 features, and meet in LDS.  Both kernels, 8192 rows of 80 + 80, rank 16: 9.8 us against 22.2; but 3000 rows of 1280 + 5120, rank 128,
// seven adapters 74 against 49.
__global__ void __launch_bounds__(256)
k_adapter_outer_sum(AdapterSegments g, int R, int chunk, OuterSum a, OuterSum b, int ablocks, int shares, int accumulate) {
  const bool second = (int)blockIdx.x >= ablocks;
  const OuterSum s = second ? b : a;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int block = second ? (int)blockIdx.x - ablocks : (int)blockIdx.x, f = ((shares > 1 ? block : block * 4 + wave) * 64 + lane) * 4, n = blockIdx.z;
  const bool in = f < s.C;                             // the lanes stay together for the segments
  __shared__ f32x4 join[3][64];
  for (int r = blockIdx.y; r < R; r += gridDim.y) {
    f32x4 sum = {0, 0, 0, 0};
    int turn = 0;
    bool rows_of_it = false;
    const float* from = s.part + (int64_t)r * s.C + f;
    const int64_t stride = (int64_t)R * s.C;
    // 64 segments at a time: each lane looks at one, and those of adapter n are worked through in order
    for (int v0 = 1; v0 <= g.segments; v0 += 64) {
      const int v = v0 + lane;
      const int rows = segment_bound(g, v + 1) - segment_bound(g, v), first = first_slot(g, v, chunk);
      const int last = min(first + (rows - 1) / chunk + 1, first_slot(g, v + 1, chunk));
      uint64_t todo = __ballot(v <= g.segments && rows > 0 && segment_adapter(g, v) == n);
      rows_of_it |= todo != 0;
      while (todo) {
        const int of = __builtin_ctzll(todo);
        todo &= todo - 1;
        const int end = __builtin_amdgcn_readlane(last, of);
        for (int k = __builtin_amdgcn_readlane(first, of); k < end; k += 8, turn++) {
          if (shares > 1 && (turn & 3) != wave) continue;
          f32x4 part[8];                                 // all under way at once
#pragma unroll
          for (int i = 0; i < 8; i++) {
            part[i] = (f32x4){0, 0, 0, 0};
            if (in && k + i < end) part[i] = *(const f32x4*)(from + (k + i) * stride);
          }
#pragma unroll
          for (int i = 0; i < 8; i++) sum += part[i];
        }
      }
    }
    if (!rows_of_it) {                                   // nothing to add, in any rank: zeros, or as it is
      if (!accumulate && in && (shares == 1 || wave == 0))
        for (; r < R; r += gridDim.y) *(f32x4*)(s.G + ((int64_t)n * R + r) * s.ldg + f) = (f32x4){0, 0, 0, 0};
      return;
    }
    if (shares > 1) {
      if (wave > 0) join[wave - 1][lane] = sum;
      __syncthreads();
      if (wave == 0)
#pragma unroll
        for (int w = 0; w < 3; w++) sum += join[w][lane];
      __syncthreads();
    }
    if (!in || (shares > 1 && wave > 0)) continue;
    float* p = s.G + ((int64_t)n * R + r) * s.ldg + f;
    sum *= s.scale;
    if (accumulate) sum += *(const f32x4*)p;
    *(f32x4*)p = sum;
  }
}

// Both weight gradients of few rows in one launch: a workgroup takes 128 features of one adapter, 16 ranks, and all rows that the adapter has, 32 in each of
// eight waves at a time.  The rows are listed in LDS first, in order, by a search of every row's segment, so that an adapter's short segments share a step; behind the
// last the list repeats it, with zeros of L.  The waves' sums meet in LDS, in the order of the rows.
// Bound by the launch and the waits in a row: the bounds, the rows of L and M, the stores (4 rows of 80 + 80, rank 16: 3.8 us; 256 rows of 1280 + 5120, rank
// 128, of one adapter 7.1, of seven 20).
struct RowList {
  int start[kFewSegments + 1], adapter[kFewSegments], counts[kFewRows / 64];
  int rows[kFewRows + 8];

  // Lists the rows of adapter n and returns their number.
  __device__ __forceinline__ int find(const AdapterSegments& g, int n) {
    const int tid = threadIdx.x;
    bool some = false;
    if (tid < g.segments) {
      const int v = g.adapter[tid];
      start[tid] = g.row_start[tid];
      adapter[tid] = v;
      some = v == n;
      if (tid == g.segments - 1) start[tid + 1] = g.row_start[tid + 1];
    }
    if (!__syncthreads_or(some)) return 0;
    uint64_t mine[kFewRows / 512];
#pragma unroll
    for (int j = 0; j < kFewRows / 512; j++) {
      mine[j] = 0;
      if (j * 512 < g.T) {
        const int row = j * 512 + tid;
        int lo = 0;                                    // segment lo - 1 is the last that starts at the row or before it, if lo > 0
        for (int step = 1 << (31 - __builtin_clz(g.segments)); step > 0; step >>= 1)
          if (lo + step <= g.segments && start[lo + step - 1] <= row) lo += step;
        mine[j] = __ballot(row < g.T && lo > 0 && row < start[lo] && adapter[max(lo - 1, 0)] == n);
      }
    }
    return list(mine, 0);
  }
  // The same for the kFewRows rows from row0 on, with a table of every row's adapter
  __device__ __forceinline__ int find(const int* ids, int row0, int T, int n) {
    uint64_t mine[kFewRows / 512];
#pragma unroll
    for (int j = 0; j < kFewRows / 512; j++) {
      const int row = row0 + j * 512 + (int)threadIdx.x;
      mine[j] = __ballot(row < T && ids[min(row, T - 1)] == n);
    }
    return list(mine, row0);
  }
  // `mine`: of 512 rows each, those of the wave's 64 that are listed
  __device__ __forceinline__ int list(const uint64_t (&mine)[kFewRows / 512], int row0) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (lane == 0)
#pragma unroll
      for (int j = 0; j < kFewRows / 512; j++) counts[j * 8 + wave] = __popcll(mine[j]);
    __syncthreads();
    int total = 0, at[kFewRows / 512];
#pragma unroll
    for (int k = 0; k < kFewRows / 64; k++) {
      if (k % 8 == wave) at[k / 8] = total;
      total += counts[k];
    }
#pragma unroll
    for (int j = 0; j < kFewRows / 512; j++)
      if (mine[j] >> lane & 1) {
        const int to = at[j] + __popcll(mine[j] & ((1ull << lane) - 1));
        rows[to] = row0 + j * 512 + tid;
        if (to == total - 1)
          for (int i = 1; i < 8; i++) rows[to + i] = row0 + j * 512 + tid;
      }
    __syncthreads();
    return uniform(total);
  }
};
struct OuterFew {
  RowList list;
  f32x4 join[8][8][64];

  template <bool BITS8>
  __device__ __forceinline__ void run(int count, const OuterArgs& a, const OuterSum& s, int n, int fb, int rank0, int R, int accumulate) {
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int m = lane & 15, q = lane >> 4, f = fb * 128 + m * 8, rank = min(rank0 + m, R - 1);
    f32x4 acc[8];
#pragma unroll
    for (int j = 0; j < 8; j++) acc[j] = (f32x4){0, 0, 0, 0};
    for (int at = wave * 32 + q * 8, r0 = wave * 32; r0 < count; r0 += 256, at += 256) {
      int rows[8];
      float v[8];
      uint4 b[8], hi, mid, lo;
      OuterRows<BITS8> x;
#pragma unroll
      for (int e = 0; e < 8; e++) rows[e] = list.rows[min(at, count - 1) + e];
      x.load(a, rows, f < a.C ? f : 0);
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] = a.L[rows[e] * a.ldl + rank];
#pragma unroll
      for (int e = 0; e < 8; e++) v[e] = at + e < count ? v[e] : 0.0f;
      x.operands(b, a.type);
      split8(v, hi, mid, lo);
#pragma unroll
      for (int j = 0; j < 8; j++) {
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(hi), frag(b[j]), acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(mid), frag(b[j]), acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(lo), frag(b[j]), acc[j], 0, 0, 0);
      }
    }
    if (wave * 32 < count)
#pragma unroll
      for (int j = 0; j < 8; j++) join[wave][j][lane] = acc[j];
    __syncthreads();
    // Wave w stores ranks w % 4 + 4 q, four of the lane's eight features
    const int e = wave & 3, h = wave >> 2 << 2, r = rank0 + 4 * q + e;
    if (f >= a.C || r >= R) return;
    float* p = s.G + ((int64_t)n * R + r) * s.ldg + f + h;
    f32x4 sum = {0, 0, 0, 0};
    for (int w = 0; w < 8 && w * 32 < count; w++)
#pragma unroll
      for (int j = 0; j < 4; j++) sum[j] += ((const float*)&join[w][h + j][lane])[e];
    sum *= s.scale;
    if (accumulate) sum += *(const f32x4*)p;
    *(f32x4*)p = sum;
  }
};
__global__ void __launch_bounds__(512, 4)
k_adapter_outer_few(AdapterSegments g, OuterArgs x, OuterArgs z, OuterSum gx, OuterSum gz, int R, int accumulate) {
  __shared__ __align__(16) OuterFew few;
  const bool second = (int)blockIdx.x >= x.fblocks;
  const OuterArgs a = second ? z : x;
  const OuterSum s = second ? gz : gx;
  const int fb = second ? (int)blockIdx.x - x.fblocks : (int)blockIdx.x, rank0 = blockIdx.y * 16, n = blockIdx.z;
  const int count = few.list.find(g, n);
  if (count == 0 && accumulate) return;
  if (a.type == M_BF16) few.run<false>(count, a, s, n, fb, rank0, R, accumulate);
  else few.run<true>(count, a, s, n, fb, rank0, R, accumulate);
}

// Many segments, for each of which chunks would take a sum: a table of every row's adapter first, then kFewRows rows at a time as above, and, of several such
// blocks, their sums in order.  Bound by the waits in a row of three launches and by the sums; M is read once for 16 ranks.  16384 rows of 4096 + 4096, rank 16,
// four adapters: 68 us in 1024 segments (4.0 TB/s; chunks 442), 74 in 16384 (chunks 6645), but 67 in eight, which chunks do in 60; 256 rows of 1280 + 5120,
// rank 128, one adapter in 256 segments: 11 us (chunks 491).
__global__ void __launch_bounds__(256)
k_adapter_row_ids(AdapterSegments g, int* __restrict__ ids) {
  const int row = (int)blockIdx.x * 256 + (int)threadIdx.x;
  if (row >= g.T) return;
  int lo = 0;                                            // as RowList::find
  for (int step = 1 << (31 - __builtin_clz(g.segments)); step > 0; step >>= 1)
    if (lo + step <= g.segments && g.row_start[lo + step - 1] <= row) lo += step;
  ids[row] = lo > 0 && row < g.row_start[lo] ? g.adapter[lo - 1] : -1;
}
// gx, gz: the gradients themselves of one block of rows, otherwise the blocks' sums, adapter n of block b at number b * adapters + n
__global__ void __launch_bounds__(512, 4)
k_adapter_outer_rows(AdapterSegments g, OuterArgs x, OuterArgs z, OuterSum gx, OuterSum gz, int R, int accumulate, const int* __restrict__ ids, int* __restrict__ counts) {
  __shared__ __align__(16) OuterFew few;
  const int fblocks = x.fblocks + z.fblocks, block = (int)blockIdx.x / fblocks, n = blockIdx.z, to = block * (int)gridDim.z + n;
  int fb = (int)blockIdx.x - block * fblocks;
  const bool second = fb >= x.fblocks;
  const OuterArgs a = second ? z : x;
  const OuterSum s = second ? gz : gx;
  const int count = uniform(few.list.find(ids, block * kFewRows, g.T, n));
  if (counts && fb == 0 && blockIdx.y == 0 && threadIdx.x == 0) counts[to] = count;
  if (second) fb -= x.fblocks;
  if (count == 0 && (counts || accumulate)) return;      // a block's sum that there is not is not read
  if (a.type == M_BF16) few.run<false>(count, a, s, to, fb, blockIdx.y * 16, R, accumulate);
  else few.run<true>(count, a, s, to, fb, blockIdx.y * 16, R, accumulate);
}
__global__ void __launch_bounds__(256)
k_adapter_outer_rows_sum(int R, int blocks, OuterSum a, OuterSum b, int ablocks, const int* __restrict__ counts, int accumulate) {
  const bool second = (int)blockIdx.x >= ablocks;
  const OuterSum s = second ? b : a;
  const int f = ((second ? (int)blockIdx.x - ablocks : (int)blockIdx.x) * 256 + (int)threadIdx.x) * 4, r = blockIdx.y, n = blockIdx.z, adapters = gridDim.z;
  if (f >= s.C) return;
  f32x4 sum = {0, 0, 0, 0};
  bool rows_of_it = false;
  for (int k = 0; k < blocks; k++) {
    const int64_t from = (int64_t)k * adapters + n;
    if (counts[from] == 0) continue;
    rows_of_it = true;
    sum += *(const f32x4*)(s.part + (from * R + r) * s.C + f);
  }
  float* p = s.G + ((int64_t)n * R + r) * s.ldg + f;
  if (accumulate && !rows_of_it) return;
  sum *= s.scale;
  if (accumulate) sum += *(const f32x4*)p;
  *(f32x4*)p = sum;
}

int mode(int dtype) { return dtype == SSTE_F8E4M3 ? M_E4M3 : dtype == SSTE_F8E5M2 ? M_E5M2 : dtype == SSTE_F8BLOCK ? M_BLOCK : M_BF16; }
int padded_rank(int R) { return R <= 16 ? 16 : R <= 32 ? 32 : R <= 64 ? 64 : 128; }

// How the two products of a call are shared out.  Times are of both kernels, or of the one, in us.
struct ApplyPlan {
  bool both;         // one launch
  Share share;       // of it or of the second: workgroups of a tile
  bool large;        // two launches: tiles of 64 rows for the first, otherwise of 32
  int splits, span;  // of its contraction
};
ApplyPlan plan_apply(const AdapterSegments& g, int R, int K, int C, bool workspace) {
  ApplyPlan p = {};
  const int64_t extra = (g.segments < g.T ? g.segments : g.T) + 1;     // tiles that segments, and the rows outside them, may add
  const int rank = padded_rank(R);
  int chunk = down_chunk(rank, 16), chunks = K > 0 ? (K + chunk - 1) / chunk : 1;
  // One launch does the first product in 16-row tiles, once for each of a tile's workgroups, and cannot share its contraction out.  Its time against that of
  // two, in us: the chunks' and the features' latencies by rounds of workgroups, and what does not come from the last-level cache, against rows and adapters by
  // bytes.  The factors are fitted to 2648 problems (ranks 16 to 128, 112 ... 5120 -> 136 ... 5120, 8 ... 32768 rows, up to a segment each): the choice costs
  // 0.75 % over the better in the mean and 70 % at most, where limits on rows and chunks cost 5 % and 87 %.  Rank 16, 1280 -> 3840: 1 row 5.6 against 8.6; rank 64,
  // 512 -> 208, 2500 rows 5.6 against 8.4; rank 64, 5120 -> 1280, 64 rows 16.6 against 10.7; rank 16, 1280 -> 5120, 1000 rows of their own 28.8 against 53.9,
  // 32768 rows of one segment 178 against 146 (rank 32).
  const bool single = 2 * (int64_t)g.segments >= g.T;                  // mostly one row a segment: a tile is as good as empty, whatever its size
  const int64_t passes = C > 0 ? (C + 1023) / 1024 : 1, tiles16 = g.T / 16 + extra, most = (1 << 22) / (slots(g, 16) + 8);
  int64_t slices = 520 / tiles16 < passes ? 520 / tiles16 : passes;
  if (slices > most) slices = most;                                    // what a grid can count, with a million empty segments
  if (slices < 1) slices = 1;
  const double r = rank / 64.0, few = extra - 1;
  const auto filled = [&](int rows) { return fmax(few, (double)g.T / rows + few * 0.5); };      // tiles with rows, more or less
  const double at_once = 200 * (single ? 1 + 8.0 / rank : 1) / (rank == 128 ? 1.5 : 1), mb = 1e-6 * g.T * (2.0 * K + 4.0 * C);
  const double one = 2 + (0.23 * chunks * (1 + r) + 0.8 * passes / slices * (1 + 1.8 * r)) * fmax(1, filled(16) * slices / at_once) + 0.1 * fmax(0, mb - 90);
  const double two = 7.8 + 1.1 * r + 0.14 * K / 1280.0 * (1 + r) + 0.085 * mb + 0.24e-6 * filled(32) * rank * ((double)K + C);
  p.both = one <= two && most > 0;
  const int64_t all = p.both ? tiles16 : g.T / 32 + extra;
  if (p.both) {
    // A tile's workgroups read the same rows and the same adapter: on one XCD (rank 16, 2560 -> 2560, 200 rows of 6 segments 6.0 us against 7.9; 96 of 96, 1280
    // -> 3840, 8.2 against 8.7, though -> 5120 9.9 against 9.2), unless some XCDs would have no tile (rank 128, 1280 -> 5120, 1 row: 13.1 against 10.7).
    p.share = share_of((int)slices, all >= 8);
    return p;
  }
  // Tiles of 32 or 64 rows, which read the adapter half as often (not of rank 16, whose adapters are small: 16384 rows of 4096 48.7 us against 57), and the
  // contraction shared out in up to four, in whole chunks and at least four of them: the least of what the first product loads, rows counted twice (they come
  // from memory, the adapter from L2), by rounds of a workgroup on every CU, the last as if half full, a workgroup as if 256 elements longer than it is; and,
  // with partial sums, of their writes and of each block of features reading them.  The factors are fitted to 446 problems (ranks 8 to 128, bf16 and e4m3,
  // 1280 ... 5120 wide, 700 ... 32768 rows): the choice costs 1.1 % over the best of the eight ways in the mean, 14 % at most, where limits on rows, ranks and
  // widths cost 4 % and 25 %.  Rank 128, 5003 ragged rows, 1280 -> 3840: 46.4 us in one part, 46.8 in two, 47.3 in four; 3840 -> 1280: 35.5, 33.3, 30.7, and
  // 28.5 in two of 64-row tiles.
  double best = 0;
  for (int rows = 32; rows <= (rank > 16 ? 64 : 32); rows += 32) {
    chunk = down_chunk(rank, rows), chunks = K > 0 ? (K + chunk - 1) / chunk : 1;
    const int64_t tiles = g.T / rows + extra;
    for (int want = 1; want <= (workspace ? kMostSplits : 1) && (want == 1 || want <= chunks / 4); want++) {
      const int each = (chunks + want - 1) / want, splits = (chunks + each - 1) / each;
      const double rounds = (double)(tiles * splits) / 256, whole = (double)((tiles * splits + 255) / 256), full = (rounds + whole) / 2;
      const double loads = (full < 1 ? 1 : full) * ((double)each * chunk + 256) * (2 * rows + rank);
      const double sums = splits > 1 ? 0.012 * splits * (double)g.T * R * (1 + (C + 511) / 512) : 0;
      if (best > 0 && loads + sums >= best) continue;
      best = loads + sums;
      p.large = rows == 64, p.splits = splits, p.span = each * chunk;
    }
  }
  // The workgroups of the second share a tile's D and its partial sums: on one XCD (rank 128, 1280 -> 3840, 1500 rows in three: 17.7 us against 21.6; rank 64,
  // 32768 rows in one 129 against 133) where these are many; with few the order of the rows in memory counts for more (rank 32, 1280 -> 5120, 32768 rows:
  // 135.5 against 132).
  p.share = share_of(C > 0 ? (C + 511) / 512 : 1, all >= 8 && rank * p.splits >= 64);      // without features D is still to be added up
  return p;
}

template <int DT, int RP>
void apply(const AdapterApply& a, hipStream_t s) {
  const ApplyPlan p = plan_apply(a.seg, a.R, a.K, a.C, a.ws != nullptr);
  const DownArgs d = {(const uint8_t*)a.X, a.ldx, a.K, (const uint16_t*)a.down, a.lddown, a.R, a.scale, a.x_scale, a.D, a.ldd};
  const UpArgs o = {(const uint16_t*)a.up, a.ldup, a.C, (const uint16_t*)a.base, a.ldbase, (uint16_t*)a.out, a.ldout};
  if (p.both) {
    SSTE_LAUNCH(SSTE_K_ADAPTER, (k_adapter_both<DT, RP / 16>), dim3(grid_of(slots(a.seg, 16), p.share)), dim3(512), s, a.seg, d, o, p.share);
    return;
  }
  const dim3 grid((unsigned)(slots(a.seg, p.large ? 64 : 32) * p.splits));
  if (RP > 16 && p.large) SSTE_LAUNCH(SSTE_K_ADAPTER, (k_adapter_down<DT, (RP > 16 ? RP / 16 : 2), 4>), grid, dim3(512), s, a.seg, d, p.splits, p.span, a.ws);
  else SSTE_LAUNCH(SSTE_K_ADAPTER, (k_adapter_down<DT, RP / 16, 2>), grid, dim3(512), s, a.seg, d, p.splits, p.span, a.ws);
  if (a.C > 0 || p.splits > 1)
    SSTE_LAUNCH(SSTE_K_ADAPTER, (k_adapter_up<RP, 2>), dim3(grid_of(slots(a.seg, 32), p.share)), dim3(256), s, a.seg, d, o, p.share, p.splits, a.ws);
}
template <int DT>
void apply(const AdapterApply& a, hipStream_t s) {
  switch (padded_rank(a.R)) {
    case 16: apply<DT, 16>(a, s); break;
    case 32: apply<DT, 32>(a, s); break;
    case 64: apply<DT, 64>(a, s); break;
    default: apply<DT, 128>(a, s); break;
  }
}

// Rows of a chunk of the weight gradients: about 384 workgroups of 256 features, one round of what fits the chip (16384 rows of 1024 + 4096, rank 16: 44.4 us;
// 256 workgroups 50.2, 512 46.7; 7777 ragged rows of 1280 + 5120, rank 64: 47.0, 52.1 and 54.2).  A chunk's sum has R / rows times four of its rows' bytes,
// written and read again: where 384 give fewer than 4 R rows (rank 64, 4096 rows of 1280 + 1280: 19.6 us, with half of them 23.2), 4 R unless that leaves
// fewer than 256 workgroups.  Narrow layers have few workgroups however short the chunks, and the waits for 64 rows in a chunk and for eight chunks in a sum
// balance at a chunk of 64 sqrt(T / 950) rows (over 576 problems of 3000 ... 16384 rows 1.2 % in the mean, 8192 rows of 80 + 80 up to 20 %).
int outer_chunk(int64_t T, int R, int64_t I, int64_t O) {
  const int64_t blocks = ((I + 255) / 256 + (O + 255) / 256) * (R > 64 ? 2 : 1), least = 4 * padded_rank(R), most = 1 << 20;
  const auto rows = [&](int64_t workgroups) { return (T * blocks / workgroups + 63) / 64 * 64; };
  const int64_t shortest = (int64_t)sqrt(T / 950.0) * 64;
  int64_t chunk = rows(384);
  if (chunk < least) chunk = rows(256) < least ? rows(256) : least;
  if (chunk < shortest) chunk = shortest;
  return (int)(chunk < 64 ? 64 : chunk > most ? most : chunk);
}

}  // namespace

hipError_t launch_adapter_apply(const AdapterApply& a, hipStream_t s) {
  if (a.seg.T == 0) return hipSuccess;
  switch (mode(a.dtype)) {
    case M_BF16: apply<M_BF16>(a, s); break;
    case M_E4M3: apply<M_E4M3>(a, s); break;
    default: apply<M_E5M2>(a, s); break;
  }
  return hipGetLastError();
}

size_t adapter_apply_workspace_bytes(int64_t T, int segments, int R, int64_t K, int64_t C) {
  const AdapterSegments g = {nullptr, nullptr, segments, 0, (int)T};
  if (T == 0) return 0;
  const ApplyPlan p = plan_apply(g, R, (int)K, (int)C, true);
  return p.both || p.splits == 1 ? 0 : (size_t)p.splits * (size_t)T * (size_t)R * 4;
}

size_t adapter_wgrad_workspace_bytes(int64_t T, int segments, int R, int64_t I, int64_t O) {
  if (T == 0 || wgrad_few(T, segments, segments, R, I, O)) return 0;
  const AdapterSegments g = {nullptr, nullptr, segments, 0, (int)T};
  return (size_t)slots(g, outer_chunk(T, R, I, O)) * (size_t)R * (size_t)(I + O) * 4;
}

hipError_t launch_adapter_wgrad(const AdapterSegments& g, int R, const AdapterOuter& a, const AdapterOuter& b, int accumulate, void* ws, hipStream_t s) {
  const AdapterWgradWay way = wgrad_way(g.T, g.segments, g.adapters, R, a.C, b.C);
  const int chunk = way == kWgradChunks ? outer_chunk(g.T, R, a.C, b.C) : 0, span = way == kWgradChunks ? 256 : 128;
  const auto args = [&](const AdapterOuter& o, float* part) {
    return OuterArgs{o.L, o.ldl, (const uint8_t*)o.M, o.ldm, mode(o.m_dtype), o.blocks, o.ldblocks, o.C, (o.C + span - 1) / span, part};
  };
  if (way == kWgradFew) {
    const OuterArgs x = args(a, nullptr), z = args(b, nullptr);
    const OuterSum gx = {nullptr, a.G, a.ldg, a.m_scale, a.C}, gz = {nullptr, b.G, b.ldg, b.m_scale, b.C};
    const dim3 grid((unsigned)(x.fblocks + z.fblocks), (unsigned)((R + 15) / 16), (unsigned)g.adapters);
    if (grid.x > 0 && grid.z > 0) SSTE_LAUNCH(SSTE_K_ADAPTER, k_adapter_outer_few, grid, dim3(512), s, g, x, z, gx, gz, R, accumulate);
    return hipGetLastError();
  }
  if (way == kWgradRows) {
    const int blocks = (int)wgrad_row_blocks(g.T);
    const int64_t sums = (int64_t)blocks * g.adapters;
    int *ids = (int*)ws, *counts = blocks > 1 ? ids + g.T : nullptr;
    float* part = (float*)ws + (g.T + sums + 3) / 4 * 4;      // of several blocks
    const OuterArgs x = args(a, nullptr), z = args(b, nullptr);
    const OuterSum gx = {part, a.G, a.ldg, a.m_scale, a.C}, gz = {part + sums * R * a.C, b.G, b.ldg, b.m_scale, b.C};
    const auto block_sum = [&](const OuterSum& o) { return blocks > 1 ? OuterSum{nullptr, (float*)o.part, o.C, 1.0f, o.C} : o; };
    if (g.adapters == 0) return hipSuccess;
    SSTE_LAUNCH(SSTE_K_ADAPTER, k_adapter_row_ids, dim3((unsigned)((g.T + 255) / 256)), dim3(256), s, g, ids);
    SSTE_LAUNCH(SSTE_K_ADAPTER, k_adapter_outer_rows, dim3((unsigned)((x.fblocks + z.fblocks) * blocks), (unsigned)((R + 15) / 16), (unsigned)g.adapters), dim3(512), s, g, x, z,
                block_sum(gx), block_sum(gz), R, blocks > 1 ? 0 : accumulate, ids, counts);
    const int ablocks = (a.C + 1023) / 1024, bblocks = (b.C + 1023) / 1024;
    if (blocks > 1)
      SSTE_LAUNCH(SSTE_K_ADAPTER, k_adapter_outer_rows_sum, dim3((unsigned)(ablocks + bblocks), (unsigned)R, (unsigned)g.adapters), dim3(256), s, R, blocks, gx, gz, ablocks, counts, accumulate);
    return hipGetLastError();
  }
  const OuterArgs x = args(a, (float*)ws), z = args(b, (float*)ws + slots(g, chunk) * R * a.C);
  if (g.T > 0 && x.fblocks + z.fblocks > 0) {
    const int64_t n = slots(g, chunk) * (x.fblocks + z.fblocks);
    const dim3 grid((unsigned)(R > 64 ? (n + 7) / 8 * 16 : n));
    switch (padded_rank(R)) {
      case 16: SSTE_LAUNCH(SSTE_K_ADAPTER, k_adapter_outer<1>, grid, dim3(256), s, g, x, z, R, chunk); break;
      case 32: SSTE_LAUNCH(SSTE_K_ADAPTER, k_adapter_outer<2>, grid, dim3(256), s, g, x, z, R, chunk); break;
      default: SSTE_LAUNCH(SSTE_K_ADAPTER, k_adapter_outer<4>, grid, dim3(256), s, g, x, z, R, chunk); break;
    }
  }
  // Chunks shared out among a workgroup's waves while that gives no more than 2048 workgroups, and where an adapter has more than eight in the mean
  const int64_t wide = (int64_t)((a.C + 1023) / 1024 + (b.C + 1023) / 1024) * R * g.adapters;
  const int shares = wide <= 512 && slots(g, chunk) > 8 * (int64_t)g.adapters ? 4 : 1, width = 1024 / shares, ablocks = (a.C + width - 1) / width, bblocks = (b.C + width - 1) / width;
  // Workgroups for several ranks each where there are many: of a thousand adapters most may have no rows
  const int64_t ranks = ablocks + bblocks > 0 && g.adapters > 0 ? 8192 / ((int64_t)(ablocks + bblocks) * g.adapters) : 1;
  if (ablocks + bblocks > 0 && g.adapters > 0)
    SSTE_LAUNCH(SSTE_K_ADAPTER, k_adapter_outer_sum, dim3((unsigned)(ablocks + bblocks), (unsigned)(ranks < 1 ? 1 : ranks < R ? ranks : R), (unsigned)g.adapters), dim3(256), s, g, R, chunk,
                (OuterSum{x.part, a.G, a.ldg, a.m_scale, a.C}), (OuterSum{z.part, b.G, b.ldg, b.m_scale, b.C}), ablocks, shares, accumulate);
  return hipGetLastError();
}

}  // namespace sste
