// Activations kept in 8 bits for the backward pass: e4m3 codes with one power of two for every 32 consecutive features of a row.
//
//   pack      e = the least exponent >= -117 with max |x| <= 448 * 2^e, code = RNE_e4m3(x * 2^-e), scale byte e + 127
//   backward  h = code * 2^e, A = act(h), dH = dA * act'(h)
//
// A power of two makes both directions exact but for the one rounding to e4m3, and a block of 32 keeps a feature with large values from
// taking the others' bits.  Both passes read every element once and write once: bound by memory traffic.  32768 x 5120: pack 92 us, 5.5 TB/s; 16384 x 5120:
// backward with GELU, its derivative and dA 113 us, 5.2 TB/s (a copy on the same card: 5.1).  333 x 1280 takes 3.2 us, a launch.
// A thread's two pieces a pass are loaded before either is converted.
#include "adapter.h"

namespace sste {

namespace {

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;

// A lane converts pieces of 16 consecutive elements, two neighbouring lanes share a block of 32.  A workgroup takes groups of whole rows, U pieces a
// thread; a row counts an even number of pieces, the last of them empty where the row ends in the middle of a block.
struct Rows {
  int64_t rows;
  int per_row;          // pieces of a row, even
  int columns;          // its elements, a multiple of 16
  int group;            // rows of a group
  uint32_t magic;       // i / per_row = mulhi(i, magic) for the piece numbers of a group; 0 where a group is one row
};
struct Piece {
  int64_t row;
  int at;               // piece of the row
  bool in;              // holds elements
};
__device__ __forceinline__ Piece piece(const Rows& g, int64_t first, int i) {
  const int r = (int)__umulhi((uint32_t)i, g.magic);
  Piece p;
  p.row = first + r;
  p.at = i - r * g.per_row;
  p.in = i < g.group * g.per_row && p.row < g.rows && p.at * 16 < g.columns;
  return p;
}

// Exponent byte of a block whose largest magnitude has these bf16 bits: 448 = 1.75 * 2^8, and a mantissa above 1.75 (96 of 128) takes one more.
// Infinities and NaN are not asked (they become NaN codes), so the byte is at most 247.
__device__ __forceinline__ int exponent_byte(uint32_t top) { return max((int)(top >> 7) - 8 + ((top & 127) > 96 ? 1 : 0), 10); }
// Largest finite magnitude of a pair of bf16, as bf16 bits
__device__ __forceinline__ uint32_t top_of(uint32_t w) {
  const uint32_t a = w & 0x7FFF, b = (w >> 16) & 0x7FFF;
  return max(a < 0x7F80 ? a : 0, b < 0x7F80 ? b : 0);
}
// x * s as a float for the conversion; an infinity becomes NaN, which e4m3 has and an infinity not
__device__ __forceinline__ float scaled(uint32_t bits, float s) { return (bits & 0x7FFFFFFF) < 0x7F800000u ? u2f(bits) * s : u2f(0x7FC00000u); }

// For GELU, whose products of zeros and infinities would be NaN: what pack rounded up to 2^128 is the largest float again, whose activation is itself (an infinity
// as bf16) or zero and whose slope 1 or 0.  NaN stays.
__device__ __forceinline__ float finite(float h) { return __builtin_fabsf(h) == __builtin_inff() ? __builtin_copysignf(0x1.fffffep127f, h) : h; }

template <int U>
__global__ void __launch_bounds__(256)
k_checkpoint_pack(Rows g, const uint8_t* __restrict__ X, int64_t ldx, uint8_t* __restrict__ codes, int64_t ldc, uint8_t* __restrict__ scales, int64_t lds) {
  for (int64_t row0 = (int64_t)blockIdx.x * g.group; row0 < g.rows; row0 += (int64_t)gridDim.x * g.group)
  for (int i0 = 0; i0 < g.group * g.per_row; i0 += 256 * U) {
    uint4 x[U][2];
    Piece p[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      p[u] = piece(g, row0, i0 + u * 256 + threadIdx.x);
      const uint4* s = (const uint4*)(X + (p[u].row * ldx + p[u].at * 16) * 2);
      x[u][0] = load16(s, p[u].in);
      x[u][1] = load16(s + 1, p[u].in);
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const uint32_t w[8] = {x[u][0].x, x[u][0].y, x[u][0].z, x[u][0].w, x[u][1].x, x[u][1].y, x[u][1].z, x[u][1].w};
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < 8; k++) top = max(top, top_of(w[k]));
      top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true));     // the neighbour's, lanes 1 0 3 2
      const int byte = exponent_byte(top);
      const float s = u2f((uint32_t)(254 - byte) << 23);
      uint32_t c[4];
#pragma unroll
      for (int k = 0; k < 4; k++)
        c[k] = e4m3_rne_pack(scaled(w[2 * k] << 16, s), scaled(w[2 * k] & 0xFFFF0000u, s)) |
               e4m3_rne_pack(scaled(w[2 * k + 1] << 16, s), scaled(w[2 * k + 1] & 0xFFFF0000u, s)) << 16;
      if (!p[u].in) continue;
      *(uint4*)(codes + p[u].row * ldc + p[u].at * 16) = make_uint4(c[0], c[1], c[2], c[3]);
      if ((p[u].at & 1) == 0) scales[p[u].row * lds + (p[u].at >> 1)] = (uint8_t)byte;
    }
  }
}

// GELU: the activation and its derivative, otherwise both of the identity.  A and dH each may be missing; dH may be dA.
template <bool GELU, bool ACT, bool GRAD, int U>
__global__ void __launch_bounds__(256)
k_checkpoint_backward(Rows g, const uint8_t* __restrict__ codes, int64_t ldc, const uint8_t* __restrict__ scales, int64_t lds, uint8_t* A, int64_t lda,
                      const uint8_t* dA, int64_t ldda, uint8_t* dH, int64_t lddh) {
  for (int64_t row0 = (int64_t)blockIdx.x * g.group; row0 < g.rows; row0 += (int64_t)gridDim.x * g.group)
  for (int i0 = 0; i0 < g.group * g.per_row; i0 += 256 * U) {
    uint4 c[U], d[U][2];
    float s[U];
    Piece p[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      p[u] = piece(g, row0, i0 + u * 256 + threadIdx.x);
      c[u] = load16(codes + p[u].row * ldc + p[u].at * 16, p[u].in);
      s[u] = 1.0f;
      if (p[u].in) s[u] = u2f((uint32_t)scales[p[u].row * lds + (p[u].at >> 1)] << 23);
      if (GRAD) {
        const uint4* y = (const uint4*)(dA + (p[u].row * ldda + p[u].at * 16) * 2);
        d[u][0] = load16(y, p[u].in);
        d[u][1] = load16(y + 1, p[u].in);
      }
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      if (!p[u].in) continue;
      const uint32_t w[4] = {c[u].x, c[u].y, c[u].z, c[u].w};
      const uint32_t y[8] = {d[u][0].x, d[u][0].y, d[u][0].z, d[u][0].w, d[u][1].x, d[u][1].y, d[u][1].z, d[u][1].w};
      uint32_t a[8], h[8];
#pragma unroll
      for (int k = 0; k < 8; k++) {
        f32x2 v = (k & 1) ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[k >> 1], s[u], true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[k >> 1], s[u], false);
        if (GELU) v[0] = finite(v[0]), v[1] = finite(v[1]);
        if (ACT) a[k] = GELU ? bf16_rne_pack(gelu_tanh(v[0]), gelu_tanh(v[1])) : bf16_rne_pack(v[0], v[1]);
        if (GRAD) h[k] = GELU ? bf16_rne_pack(bf16lo_f32(y[k]) * gelu_tanh_grad(v[0]), bf16hi_f32(y[k]) * gelu_tanh_grad(v[1])) : y[k];
      }
      if (ACT) {
        uint4* o = (uint4*)(A + (p[u].row * lda + p[u].at * 16) * 2);
        o[0] = make_uint4(a[0], a[1], a[2], a[3]);
        o[1] = make_uint4(a[4], a[5], a[6], a[7]);
      }
      if (GRAD) {
        uint4* o = (uint4*)(dH + (p[u].row * lddh + p[u].at * 16) * 2);
        o[0] = make_uint4(h[0], h[1], h[2], h[3]);
        o[1] = make_uint4(h[4], h[5], h[6], h[7]);
      }
    }
  }
}

Rows rows_of(int64_t R, int64_t C, int pieces) {
  Rows g;
  g.rows = R;
  g.columns = (int)C;
  g.per_row = (int)((C + 31) / 32 * 2);
  g.group = g.per_row < pieces ? pieces / g.per_row : 1;
  // mulhi(i, m) with m = ceil(2^32 / d) is i / d while i * d < 2^32: i < pieces here, d < pieces
  g.magic = g.group == 1 ? 0 : (uint32_t)(((1ull << 32) + g.per_row - 1) / g.per_row);
  return g;
}
// A workgroup a group of rows, as far as a grid can count
unsigned workgroups(const Rows& g) {
  const int64_t n = (g.rows + g.group - 1) / g.group;
  return (unsigned)(n < (1 << 22) ? n : 1 << 22);
}

}  // namespace

hipError_t launch_checkpoint_pack(const void* X, int64_t R, int64_t C, int64_t ldx, void* codes, int64_t ldc, void* scales, int64_t lds, hipStream_t s) {
  if (R == 0 || C == 0) return hipSuccess;
  const Rows g = rows_of(R, C, 512);
  SSTE_LAUNCH(SSTE_K_CHECKPOINT, k_checkpoint_pack<2>, dim3(workgroups(g)), dim3(256), s, g, (const uint8_t*)X, ldx, (uint8_t*)codes, ldc, (uint8_t*)scales, lds);
  return hipGetLastError();
}

hipError_t launch_checkpoint_backward(const void* codes, const void* scales, int64_t R, int64_t C, int64_t ldc, int64_t lds, int act, void* A, int64_t lda,
                                      const void* dA, int64_t ldda, void* dH, int64_t lddh, hipStream_t s) {
  if (R == 0 || C == 0) return hipSuccess;
  const Rows g = rows_of(R, C, 512);
#define BACKWARD(GELU, ACT, GRAD)                                                                                                                        \
  SSTE_LAUNCH(SSTE_K_CHECKPOINT, (k_checkpoint_backward<GELU, ACT, GRAD, 2>), dim3(workgroups(g)), dim3(256), s, g, (const uint8_t*)codes, ldc,             \
              (const uint8_t*)scales, lds, (uint8_t*)A, lda, (const uint8_t*)dA, ldda, (uint8_t*)dH, lddh)
  const bool gelu = act == SSTE_ACT_GELU_TANH;
  if (A && dH) { if (gelu) BACKWARD(true, true, true); else BACKWARD(false, true, true); }
  else if (A) { if (gelu) BACKWARD(true, true, false); else BACKWARD(false, true, false); }
  else { if (gelu) BACKWARD(true, false, true); else BACKWARD(false, false, true); }
#undef BACKWARD
  return hipGetLastError();
}

}  // namespace sste
