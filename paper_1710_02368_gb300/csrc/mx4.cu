// Quantisation of rows to microscaled 4-bit floating point and back (OCP
// Microscaling Formats 1.0, MXFP4: E2M1 elements, one E8M0 scale for 32
// consecutive elements of a row).
//   e = floor(log2 max |x|) - 2 (at least -127),  q = E2M1(x 2^-e)
// with q rounded to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to the even
// code) and saturating at 6; 2^-e is exact, so the one rounding is the element's.
// A block with an infinity or a NaN has no scale that could say so for one
// element: its scale is NaN, and so is every value of it.
//
// One pass: four lanes hold a block (8 elements each, 16 or 32 bytes a lane), its
// largest magnitude by two shuffles; sixteen lanes write four blocks' codes (64
// bytes) and the four scales as one word of a scale tile.  Bound by memory.
#include "mx4.cuh"
#include "ops.cuh"

namespace agn {

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;
constexpr int kLane = 8;        // elements of a lane
constexpr int kWordLanes = 16;  // lanes of a scale word: 128 elements

struct MxArgs {
  const void* x;
  void* y;
  uint8_t* codes;
  uint8_t* scales;
  int64_t rows, cols, ld;
  int64_t row_bytes, tiles_k;
  int64_t rows_per_block;
  int vec;              // rows of x (y) start 16-byte aligned
  int tx_shift;         // log2 of the lanes along a row (>= 4)
};

struct Eight {
  float v[kLane];
};

template <typename T>
struct Raw {
  uint4 q[sizeof(T) * kLane / 16];
};

template <typename T>
__device__ __forceinline__ Raw<T> load8(const T* p, bool full, int n) {
  Raw<T> r;
  constexpr int Q = sizeof(T) * kLane / 16;
  if (full) {
#pragma unroll
    for (int i = 0; i < Q; ++i) r.q[i] = AGN_LD(reinterpret_cast<const uint4*>(p) + i);
  } else {
    T* e = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int i = 0; i < Q; ++i) r.q[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < kLane; ++i)
      if (i < n) e[i] = AGN_LD(p + i);
  }
  return r;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx4_quantize_kernel(const MxArgs a) {
  pdl_begin();
  const int tx = threadIdx.x & ((1 << a.tx_shift) - 1), ty = threadIdx.x >> a.tx_shift;
  const int nty = kThreads >> a.tx_shift;
  const int64_t unit = ((int64_t)blockIdx.x << a.tx_shift) + tx;   // 8 columns
  const int64_t c = unit * kLane, kq = unit / kWordLanes;          // and its scale word
  const int64_t r0 = blockIdx.y * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  const int n = c < a.cols ? (int)min((int64_t)kLane, a.cols - c) : 0;
  const bool full = a.vec && n == kLane;
  const T* x = static_cast<const T*>(a.x);
  // a whole warp has the same rows or not: the shuffles below stay within groups of 16
  // lanes, whose lanes share a row
  const uint32_t group = 0xffffu << (threadIdx.x & 16);
  for (int64_t r = r0 + ty; r < r1; r += (int64_t)kUnroll * nty) {
    Raw<T> raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t ru = r + (int64_t)u * nty;
      if (ru < r1) raw[u] = load8(x + ru * a.ld + c, full, n);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t ru = r + (int64_t)u * nty;
      if (ru >= r1) break;
      const T* e = reinterpret_cast<const T*>(&raw[u]);
      float v[kLane];
      uint32_t amax = 0;
#pragma unroll
      for (int i = 0; i < kLane; ++i) {
        v[i] = static_cast<float>(e[i]);
        amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);   // (NaN is above infinity)
      }
      amax = max(amax, __shfl_xor_sync(group, amax, 1));
      amax = max(amax, __shfl_xor_sync(group, amax, 2));
      const uint32_t code = mx_scale_code(amax);
      const float inv = mx_inverse(code);
      uint32_t q = 0;
      if (code != 255) {
#pragma unroll
        for (int i = 0; i < kLane / 2; ++i)
          q |= mx_pair(__fmul_rn(v[2 * i], inv), __fmul_rn(v[2 * i + 1], inv)) << (8 * i);
      }
      if (unit * 4 < a.row_bytes)
        AGN_ST(reinterpret_cast<uint32_t*>(a.codes + ru * a.row_bytes) + unit, q);
      uint32_t word = code << (8 * ((tx >> 2) & 3));   // (blocks past the row: code 0)
      word |= __shfl_xor_sync(group, word, 4);
      word |= __shfl_xor_sync(group, word, 8);
      if ((tx & 15) == 0 && kq < a.tiles_k)
        AGN_ST(reinterpret_cast<uint32_t*>(a.scales + mx_scale_at(ru, 4 * kq, a.tiles_k)), word);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx4_dequantize_kernel(const MxArgs a) {
  pdl_begin();
  const int tx = threadIdx.x & ((1 << a.tx_shift) - 1), ty = threadIdx.x >> a.tx_shift;
  const int nty = kThreads >> a.tx_shift;
  const int64_t unit = ((int64_t)blockIdx.x << a.tx_shift) + tx;
  const int64_t c = unit * kLane;
  const int64_t r0 = blockIdx.y * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  const int n = c < a.cols ? (int)min((int64_t)kLane, a.cols - c) : 0;
  if (n == 0) return;
  const bool full = a.vec && n == kLane;
  T* y = static_cast<T*>(a.y);
  for (int64_t r = r0 + ty; r < r1; r += (int64_t)kUnroll * nty) {
    uint32_t q[kUnroll], s[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t ru = r + (int64_t)u * nty;
      if (ru >= r1) break;
      q[u] = AGN_LD(reinterpret_cast<const uint32_t*>(a.codes + ru * a.row_bytes) + unit);
      s[u] = AGN_LD(a.scales + mx_scale_at(ru, unit >> 2, a.tiles_k));
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t ru = r + (int64_t)u * nty;
      if (ru >= r1) break;
      const float scale = mx_scale_value(s[u]);
      Raw<T> out;
      T* e = reinterpret_cast<T*>(&out);
#pragma unroll
      for (int i = 0; i < kLane; ++i)
        e[i] = static_cast<T>(__fmul_rn(mx_element((q[u] >> (4 * i)) & 15u), scale));
      T* p = y + ru * a.ld + c;
      if (full) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) * kLane / 16); ++i)
          AGN_ST(reinterpret_cast<uint4*>(p) + i, out.q[i]);
      } else {
#pragma unroll
        for (int i = 0; i < kLane; ++i)
          if (i < n) AGN_ST(p + i, e[i]);
      }
    }
  }
}

// Blocks of 2^tx_shift lanes along a row (16 to 256, what leaves the fewest idle) by
// rows_per_block rows, one wave of resident blocks.
dim3 geometry(MxArgs* a) {
  const int64_t units = a->tiles_k * kWordLanes;
  int best = 4;
  int64_t pad = INT64_MAX;
  for (int s = 8; s >= 4; --s) {
    const int64_t p = round_up(units, (int64_t)1 << s);
    if (p < pad) {
      best = s;
      pad = p;
    }
  }
  a->tx_shift = best;
  const int64_t tiles = ceil_div(units, (int64_t)1 << best), nty = kThreads >> best;
  const int64_t most = std::max<int64_t>(1, (int64_t)current_sms() * 6 / tiles);
  int64_t blocks = std::min<int64_t>(std::min<int64_t>(most, 65535), ceil_div(a->rows, nty));
  a->rows_per_block = ceil_div(a->rows, blocks);
  blocks = ceil_div(a->rows, a->rows_per_block);
  return dim3((unsigned)tiles, (unsigned)blocks);
}

bool rows_aligned(const void* p, int64_t ld, size_t es) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (size_t)ld * es % 16 == 0;
}

// Quantise (y null) or dequantise (x null).
Status launch_mx(const void* x, void* y, void* codes, void* scales, int dtype, int64_t rows,
                 int64_t cols, int64_t ld, cudaStream_t st) {
  MxArgs a{};
  a.x = x; a.y = y;
  a.codes = static_cast<uint8_t*>(codes);
  a.scales = static_cast<uint8_t*>(scales);
  a.rows = rows; a.cols = cols; a.ld = ld;
  a.row_bytes = mx_row_bytes(cols);
  a.tiles_k = mx_tiles_k(cols);
  const bool f32 = dtype == AGN_PREC_FP32;
  a.vec = rows_aligned(x ? x : y, ld, f32 ? 4 : 2);
  const dim3 grid = geometry(&a);
  auto k = x ? (f32 ? mx4_quantize_kernel<float> : mx4_quantize_kernel<bf16>)
             : (f32 ? mx4_dequantize_kernel<float> : mx4_dequantize_kernel<bf16>);
  AGN_TRY_CUDA(launch_pdl(k, grid, kThreads, 0, st, a));
  AGN_TRY_CUDA(cudaGetLastError());
  return Status::Ok();
}

Status mx_call(const char* name, const void* x, void* y, const void* codes, const void* scales,
               int dtype, int64_t rows, int64_t cols, int64_t ld, bool quantize, cudaStream_t st) {
  const size_t es = dtype_size(dtype);
  if (!es) return Status::Err(AGN_E_INVALID, "unknown dtype");
  AGN_TRY(check_matrix(name, rows, cols, ld));
  if (rows == 0 || cols == 0) return Status::Ok();
  const void* m = quantize ? x : y;
  if (!m || !codes || !scales) return Status::Err(AGN_E_INVALID, "null pointer");
  const CallBuffer bm{name, m, matrix_bytes(rows, cols, ld, es), es},
      bc{"codes", codes, (size_t)mx_code_bytes(rows, cols), 16},
      bs{"scales", scales, (size_t)mx_scale_bytes(rows, cols), 16};
  AGN_TRY(check_apart(bm, {bc, bs}));
  AGN_TRY(check_apart(bc, {bs}));
  AGN_TRY(check_buffers({bm, bc, bs}));
  KnownBuffers known({bm, bc, bs});
  AGN_TRY(bounds_upload(st));
  AGN_TRY(launch_mx(x, y, const_cast<void*>(codes), const_cast<void*>(scales), dtype, rows, cols,
                    ld, st));
  return bounds_collect(st);
}

}  // namespace

Status mx4_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx,
                    void* codes, void* scales, cudaStream_t st) {
  return launch_mx(x, nullptr, codes, scales, dtype, rows, cols, ldx, st);
}

AGN_BOUNDS_UNIT(mx4)

}  // namespace agn

extern "C" int agn_mx4_bytes(int64_t rows, int64_t cols, int64_t* codes, int64_t* scales) {
  return agn::guarded([&] {
    AGN_TRY(agn::check_matrix("matrix", rows, cols, cols));
    if (codes) *codes = agn::mx_code_bytes(rows, cols);
    if (scales) *scales = agn::mx_scale_bytes(rows, cols);
    return agn::Status::Ok();
  });
}

extern "C" int agn_mx4_quantize(const void* x, int32_t dtype, int64_t rows, int64_t cols,
                                int64_t ldx, void* codes, void* scales, void* stream) {
  return agn::guarded([&] {
    return agn::mx_call("x", x, nullptr, codes, scales, dtype, rows, cols, ldx, true,
                        static_cast<cudaStream_t>(stream));
  });
}

extern "C" int agn_mx4_dequantize(const void* codes, const void* scales, int64_t rows,
                                  int64_t cols, void* y, int32_t dtype, int64_t ldy,
                                  void* stream) {
  return agn::guarded([&] {
    return agn::mx_call("y", nullptr, y, codes, scales, dtype, rows, cols, ldy, false,
                        static_cast<cudaStream_t>(stream));
  });
}
