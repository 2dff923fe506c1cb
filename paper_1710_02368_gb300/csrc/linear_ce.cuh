// The output layer's softmax cross-entropy over many classes without keeping the
// logits (linear_ce.cu: entry points and small kernels; linear_ce_gemm.cu, linear_ce_raw.cu: the products;
// linear_ce_few.cu: a few rows).
#pragma once

#include <cuda.h>

#include <cmath>

#include "common.cuh"

namespace agn {
namespace ce {

__device__ __forceinline__ bool has_label(int label, int classes) { return (uint32_t)label < (uint32_t)classes; }

// (maximum, sum of exponentials) of two sets of values.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  constexpr float kLog2e = 1.44269504088896340736f;
  const float most = fmaxf(a.x, b.x), from = most == -INFINITY ? 0.f : most;
  return make_float2(most, a.y * exp2f((a.x - from) * kLog2e) + b.y * exp2f((b.x - from) * kLog2e));
}

enum Epilogue {
  kLse = 0,    // each row's maximum and sum of exponentials over a tile's columns
  kGrad = 1,   // p, the gradient with respect to the logits, and its column sums
  kOut = 2,    // the product itself
};

// Pieces of p, the gradient with respect to the logits, as the products read it: of bf16 operands two (one would
// round it, the factor 1 / rows of a mean loss among it, to 2^-8 of it: 777 x 1000 to 10007, dx off by 2.5e-3 of its
// norm where rounding it alone is 1.7e-3; two hold 2^-17).  Each is a product: dw and dx take twice the MMAs.
constexpr int p_pieces(int planes) { return planes == 3 ? 3 : 2; }

// One product of [M][K] and [N][K] operands.  Coordinates are elements; rows of x are
// those with a label, in order (`live` of them, `idx` their places).
struct GemmArgs {
  int M, N, K;              // M (live_is 0), K (1) or N (2) is a bound where live is given
  const int* live;          // device, null: as they are
  int live_is;
  int rows;                 // rows of x in all: live < rows means that x was gathered
  int alt;                  // 1 (2): A (B) comes from tmAlt where x was gathered
  int bn;                   // columns of a tile
  int a_mn, b_mn;           // operand stored [K][M] ([K][N]) instead
  int planes;               // 1, or 3 bf16 pieces of fp32 operands: six products
  int twice;                // planes 1: 1 (2): A (B) is p in two bf16 pieces, by steps of 64 k in turn
  int a_box;                // rows of A's boxes (128, fewer where M is less; its box is 64 along M with a_mn)
  int splits;               // ranges along K, each with sums of its own (kOut)
  int* err;
  uint32_t wait_ns;
  int withhold;             // test hook: CTA withhold - 1 of a tile leaves out its last stage and all after
  const int* idx;           // [live] places of the rows, null: their own
  // kLse, kGrad
  const float* bias;        // [classes] or null
  const int* labels;        // [rows]
  int class0, classes;      // first class of this product, classes in all
  float2* ms;               // kLse: [rows_pad][ld_ms], from column ms0 on 2 N / bn (maximum, sum)
  int64_t ld_ms;
  int ms0;
  float* zlab;              // kLse: [rows_pad] the label's logit
  const float *lse, *dloss, *dlse;   // kGrad, by place
  float scale;
  int p_plane;              // kGrad: rows from piece to piece of p (p_pieces of them)
  float* db;                // kGrad: [rows_pad / 32][ld_db] column sums of 32 rows, or null
  int64_t ld_db;
  // kOut
  int transposed;           // the output is [N][M] (whose rows `out`, `scatter` and `part_rows` speak of)
  void* out;                // [M][ldo] of dtype, rows at idx[m] where live < rows and scatter
  int dtype;
  int64_t ldo;
  int scatter;
  int tma_out;              // tmC is valid for `out`
  int part;                 // 0: to out; 1, 2: tmC is fp32 sums [splits][part_rows], stored, added
  int part_rows;
};

struct GemmMaps {
  CUtensorMap a, b, alt, c;
};

// A launch: one product, or (kOut) two with the same bn, planes and a_box, whose tiles one grid shares.
struct GemmLaunch {
  GemmMaps maps[2];
  GemmArgs args[2];
  int n;
};

// ctas: 1 or 2 (pairs); max_units: tiles times ranges along K, at most.  On the current device.
Status gemm(int ctas, int epilogue, const GemmLaunch& g, int64_t max_units, cudaStream_t st);

// A product with w read as it is (linear_ce_raw.cu): out [splits][part_rows][M] = B A^T, fp32, for up to 128 rows of
// B, three bf16 pieces each.
struct RawArgs {
  const float* w;           // (m, k) at w + m ld + k, mn: w + k ld + m
  int64_t ld;
  int M, K, mn;
  int vec;                  // rows of w are 16-byte aligned
  int groups;               // of 64 rows of B
  int splits;               // ranges along K, none without a step of 64
  int part_rows;
  int* err;
  uint32_t wait_ns;
  int withhold;             // as above
};
struct RawLaunch {
  CUtensorMap b, c;         // boxes of 64 k x 64 rows; of 32 x 32 outputs
  RawArgs args;
};
Status raw(const RawLaunch& launch, cudaStream_t st);

// A few rows (linear_ce_few.cu): up to 8 of fp32, 16 where w is small (linear_ce.cu's raw()); of bf16 up to 4,
// backward (us for 8 rows of fp32, 4096 to 32000 classes, 90 and 276, 9 rows as the products above 136 and 394, here
// 167 and 473; bf16, 4096 to 32000: gradients of 4 rows 151 for the tensor cores' 203, of 8 242 for 186).
struct FewArgs {
  const void *x, *w;
  const float* bias;
  const int* labels;
  int rows, inner, classes;
  float2* ms;               // forward: [rows][few_blocks] (maximum, sum)
  float* zlab;              // [rows]
  const float *lse, *dloss, *dlse;   // backward
  float scale;
  float* p;                 // [classes][few_rows]
  void *dx, *dw;
  float* dbias;
  float* dx_parts;          // [parts][rows][ld_parts], null: no dx
  int64_t ld_parts;
};
constexpr int kFewSms = 152;   // what grids are made for
constexpr int few_rows(int64_t rows) { return rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : rows <= 8 ? 8 : 16; }
constexpr bool few(int64_t rows, int dtype, bool backward) {
  return rows <= (dtype == AGN_PREC_FP32 ? 16 : backward ? 4 : 0);
}
// Blocks of the dot products: a warp, or several, takes four classes at a time.
constexpr int64_t few_blocks(int64_t classes) { return std::min<int64_t>(kFewSms, (classes + 3) / 4); }
// Blocks of the outer products: `along` threads along the columns of 16 bytes, ranges of classes.
struct FewCut {
  int along, parts;
  int64_t blocks_k, blocks_c;
};
inline FewCut few_cut(int64_t inner, int64_t classes, int es) {
  const int64_t columns = (inner * es + 15) / 16;
  FewCut c;
  c.along = (int)std::min<int64_t>(256, (columns + 31) / 32 * 32);
  c.blocks_k = (columns + c.along - 1) / c.along;
  const int64_t at_once = 256 / c.along;
  c.blocks_c = std::max<int64_t>(1, std::min<int64_t>(kFewSms * 2 / c.blocks_k, (classes + 16 * at_once - 1) / (16 * at_once)));
  c.parts = (int)(c.blocks_c * at_once);
  return c;
}
Status few(const FewArgs& a, int dtype, bool backward, cudaStream_t st);

}  // namespace ce
}  // namespace agn
