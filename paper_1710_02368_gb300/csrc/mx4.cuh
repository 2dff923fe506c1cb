// Microscaled 4-bit matrices (mx4.cu, mx4_linear.cu; layout in include/agn.h).
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace agn {

constexpr int kMxBlock = 32;          // elements that share a scale
constexpr int kMxTileRows = 128;      // a scale tile: 128 rows x 4 blocks, 512 bytes
constexpr int kMxTileBytes = 512;

constexpr int64_t mx_blocks(int64_t cols) { return ceil_div(cols, kMxBlock); }
constexpr int64_t mx_row_bytes(int64_t cols) { return mx_blocks(cols) * (kMxBlock / 2); }
constexpr int64_t mx_tiles_k(int64_t cols) { return ceil_div(mx_blocks(cols), 4); }
constexpr int64_t mx_code_bytes(int64_t rows, int64_t cols) { return rows * mx_row_bytes(cols); }
constexpr int64_t mx_scale_bytes(int64_t rows, int64_t cols) {
  return ceil_div(rows, kMxTileRows) * mx_tiles_k(cols) * kMxTileBytes;
}
// Byte of the scales that holds block kb of row r (tiles_k = mx_tiles_k(cols)); the four
// blocks of a tile are one 32-bit word.
__host__ __device__ __forceinline__ int64_t mx_scale_at(int64_t r, int64_t kb, int64_t tiles_k) {
  return ((r >> 7) * tiles_k + (kb >> 2)) * kMxTileBytes + (r & 31) * 16 + ((r >> 5) & 3) * 4 +
         (kb & 3);
}

// The scale code of a block whose largest magnitude has the bits `amax` (of a
// non-negative float): 2^(floor(log2 amax) - 2), so that amax lands in [4, 8),
// where E2M1's largest binade [4, 6] is; at least 2^-127 (code 0, which a block of
// zeros or of subnormal numbers gets too).  Infinity or NaN: 255, E8M0's NaN.
__device__ __forceinline__ uint32_t mx_scale_code(uint32_t amax) {
  const uint32_t e = amax >> 23;   // biased exponent, 0 for subnormal
  return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}
// 1 / scale, exact: 2^(127 - code), code <= 252.
__device__ __forceinline__ float mx_inverse(uint32_t code) {
  return __uint_as_float((254u - min(code, 252u)) << 23);
}
// The value of a scale code: 2^(code - 127); 255 is NaN.
__device__ __forceinline__ float mx_scale_value(uint32_t code) {
  return __uint_as_float(code == 255 ? 0x7fc00000u : code == 0 ? 0x00400000u : code << 23);
}
// Eight floats to E2M1 codes, round to nearest even, saturating at 6: v[0] in the low nibble.
__device__ __forceinline__ uint32_t mx_pack8(const float (&v)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// The values of eight codes.
__device__ __forceinline__ void mx_unpack8(uint32_t q, float (&v)[8]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(q));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

// y = act(x w^T + b) on quantised operands (mx4_linear.cu).
struct Mx4LinearArgs {
  const void *x_codes, *x_scales, *w_codes, *w_scales;
  const float* bias;      // [out] or null
  int64_t rows, in, out;
  int relu;
  void* y;                // [rows][ldy] of dtype; AGN_PREC_MX4: codes
  int dtype;
  int64_t ldy;
  void* y_scales;         // AGN_PREC_MX4
  int* err;               // set to 1 when a bounded wait gives up (null: none)
  // Test hook (agn_debug_waits, agn_debug_linear_waits): wait_ns > 0 is the limit of the waits
  // for each other instead of 2 s; withhold = r + 1: CTA r along K, or of each pair, leaves the last
  // stage of its first tile and all after it out (0 = none).
  uint64_t wait_ns;
  int withhold;
};
// The launches alone (the entry points check their arguments first).
Status mx4_linear(const Mx4LinearArgs& a, cudaStream_t st);
Status mx4_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx,
                    void* codes, void* scales, cudaStream_t st);

}  // namespace agn
