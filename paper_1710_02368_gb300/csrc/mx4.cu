// Quantisation of rows to microscaled 4-bit floating point and back (OCP
// Microscaling Formats 1.0, MXFP4: E2M1 elements, one E8M0 scale for 32
// consecutive elements of a row).
//   e = floor(log2 max |x|) - 2 (at least -127),  q = E2M1(x 2^-e)
// with q rounded to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to the even
// code) and saturating at 6; 2^-e is exact, so the one rounding is the element's.
// A block with an infinity or a NaN has no scale that could say so for one
// element: its scale is NaN, and so is every value of it.
//
// One pass.  A lane holds 32 bytes of a row (16 bf16 or 8 fp32 elements), two or four
// lanes a block, whose largest magnitude goes between them by shuffles; the lanes
// of four blocks write their codes (64 bytes) and the four scales as one word of a
// scale tile.  Bound by memory in fp32, by the conversions as much in bf16.
#include "mx4.cuh"
#include "ops.cuh"

namespace agn {

namespace {

constexpr int kThreads = 256;
// Rows of a thread whose loads are in flight together, quantising, back, and back into rows that
// are not aligned, and blocks of a launch for each SM.  Quantising: as many as are resident with
// the kernel's registers.  Back: more rows in flight are better in the largest matrices only.  us, new
// inputs each time, 10000 x 784 fp32, 4096 x 4096 bf16, 16384 x 4096 bf16 and fp32: quantising
// 8.0, 9.4, 29.2, 48.3 (eight blocks: 8.7, 9.7, 29.4, 49.7; three: 10.4, 10.6, 34.5, 60.3); back 7.2,
// 7.9, 28.9, 51.9 (eight rows: 8.4, 8.9, 27.8, 49.6; four blocks: 7.2, 8.4, 31.0, 53.1).  Not
// aligned, two, four, eight rows, 65536 x 100 bf16: 11.0, 11.2, 14.1.
constexpr int kQuantRows = 2, kBackRows = 4, kShiftRows = 2;
constexpr int quant_blocks(bool f32) { return f32 ? 5 : 4; }
constexpr int kBackBlocks = 8;

// Elements of a lane, its lanes of a block and of four blocks (a scale word).
template <typename T>
struct Lanes {
  static constexpr int kElems = 32 / (int)sizeof(T);
  static constexpr int kBlock = kMxBlock / kElems;
  static constexpr int kWord = 4 * kBlock;
};

struct MxArgs {
  const void* x;
  void* y;
  uint8_t* codes;
  uint8_t* scales;
  int64_t rows, cols, ld;
  int64_t row_bytes, tiles_k;
  int64_t rows_per_block;
  int vec;              // rows of x (y) start 16-byte aligned (1), 32-byte (2), neither (0)
  const void* x_end;    // past x's last element
  int tx_shift;         // log2 of the lanes along a row (>= those of a word)
};

// 32 bytes of a row as they are: one load (vec 2: 32-byte aligned), two (vec 1), the 48 aligned
// bytes that hold them (vec 0, 48 bytes within the matrix begin .. end), or the n valid elements.
template <typename T>
struct __align__(32) Raw {
  uint4 q[2];
};
template <typename T, bool kShift>
__device__ __forceinline__ Raw<T> load32(const T* p, int vec, int n, const void* begin,
                                         const void* end) {
  Raw<T> r;
  const uint32_t past = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15;
  const char* from = reinterpret_cast<const char*>(p) - past;
  const bool whole = n == Lanes<T>::kElems;
  if (kShift && whole && from >= begin && from + 48 <= end) {
    uint32_t w[12];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const uint4 q = AGN_LD(reinterpret_cast<const uint4*>(from) + i);
      w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
    }
#pragma unroll
    for (int i = 0; i < 10; ++i) w[i] = past & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 9; ++i) w[i] = past & 4 ? w[i + 1] : w[i];
    if (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 8 * (past & 2));
    }
    r.q[0] = make_uint4(w[0], w[1], w[2], w[3]);
    r.q[1] = make_uint4(w[4], w[5], w[6], w[7]);
  } else if (!kShift && whole && vec == 2) {
    if (AGN_BOUNDS_OK(p, 32)) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(r.q[0].x), "=r"(r.q[0].y), "=r"(r.q[0].z), "=r"(r.q[0].w), "=r"(r.q[1].x),
                     "=r"(r.q[1].y), "=r"(r.q[1].z), "=r"(r.q[1].w)
                   : "l"(p));
    } else {
      AGN_BOUNDS_FAIL(p);
      r.q[0] = r.q[1] = make_uint4(0, 0, 0, 0);
    }
  } else if (!kShift && whole && vec == 1) {
    r.q[0] = AGN_LD(reinterpret_cast<const uint4*>(p));
    r.q[1] = AGN_LD(reinterpret_cast<const uint4*>(p) + 1);
  } else {
    r.q[0] = r.q[1] = make_uint4(0, 0, 0, 0);
    T* e = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int i = 0; i < Lanes<T>::kElems; ++i)
      if (i < n) e[i] = AGN_LD(p + i);
  }
  return r;
}

template <typename T>
__device__ __forceinline__ void store32(T* p, int vec, const Raw<T>& r) {
  if (vec == 2) {
    if (AGN_BOUNDS_OK(p, 32))
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r.q[0].x),
                   "r"(r.q[0].y), "r"(r.q[0].z), "r"(r.q[0].w), "r"(r.q[1].x), "r"(r.q[1].y),
                   "r"(r.q[1].z), "r"(r.q[1].w)
                   : "memory");
    else
      AGN_BOUNDS_FAIL(p);
  } else {
    AGN_ST(reinterpret_cast<uint4*>(p), r.q[0]);
    AGN_ST(reinterpret_cast<uint4*>(p) + 1, r.q[1]);
  }
}

// The bits of the largest magnitude as a float (a NaN is above infinity).
__device__ __forceinline__ uint32_t largest(const Raw<float>& r) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7fffffffu);
  return m;
}
__device__ __forceinline__ uint32_t largest(const Raw<bf16>& r) {   // two halves at a time
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
  return max(m & 0xffff0000u, m << 16);
}

// kShift: rows that are not 16-byte aligned (16384 x 4095 bf16 44 us, with single elements 70).
template <typename T, bool kShift>
__global__ void __launch_bounds__(kThreads) mx4_quantize_kernel(const MxArgs a) {
  using L = Lanes<T>;
  constexpr int kUnroll = kQuantRows;
  pdl_begin();
  const int tx = threadIdx.x & ((1 << a.tx_shift) - 1), ty = threadIdx.x >> a.tx_shift;
  const int nty = kThreads >> a.tx_shift;
  const int64_t unit = ((int64_t)blockIdx.x << a.tx_shift) + tx;   // a lane's 32 bytes
  const int64_t c = unit * L::kElems, kq = unit / L::kWord;        // and its scale word
  const int64_t r0 = blockIdx.y * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  const int n = c < a.cols ? (int)min((int64_t)L::kElems, a.cols - c) : 0;
  const bool in_row = c / 2 < a.row_bytes, leads = tx % L::kWord == 0 && kq < a.tiles_k;
  const T* x = static_cast<const T*>(a.x) + (r0 + ty) * a.ld + c;
  uint8_t* codes = a.codes + (r0 + ty) * a.row_bytes + c / 2;
  // the shuffles stay within the lanes of a scale word, which share a row
  const uint32_t group = ((1u << L::kWord) - 1) << (threadIdx.x & 31 & ~(L::kWord - 1));
  for (int64_t r = r0 + ty; r < r1; r += (int64_t)kUnroll * nty) {
    Raw<T> raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (r + (int64_t)u * nty < r1) raw[u] = load32<T, kShift>(x + (int64_t)u * nty * a.ld, a.vec, n, a.x, a.x_end);
    x += (int64_t)kUnroll * nty * a.ld;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u, codes += nty * a.row_bytes) {
      const int64_t ru = r + (int64_t)u * nty;
      if (ru >= r1) break;
      uint32_t amax = largest(raw[u]);
#pragma unroll
      for (int o = 1; o < L::kBlock; o <<= 1) amax = max(amax, __shfl_xor_sync(group, amax, o));
      const uint32_t code = mx_scale_code(amax);
      const float inv = mx_inverse(code);
      const T* e = reinterpret_cast<const T*>(&raw[u]);
      uint32_t q[L::kElems / 8];
#pragma unroll
      for (int i = 0; i < L::kElems / 8; ++i) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(static_cast<float>(e[8 * i + j]), inv);
        q[i] = code == 255 ? 0u : mx_pack8(v);
      }
      if (in_row) {
        if constexpr (L::kElems == 16) AGN_ST(reinterpret_cast<uint2*>(codes), make_uint2(q[0], q[1]));
        else AGN_ST(reinterpret_cast<uint32_t*>(codes), q[0]);
      }
      uint32_t word = code << (8 * (tx / L::kBlock % 4));   // (blocks past the row: code 0)
      word |= __shfl_xor_sync(group, word, L::kBlock);
      word |= __shfl_xor_sync(group, word, 2 * L::kBlock);
      if (leads)
        AGN_ST(reinterpret_cast<uint32_t*>(a.scales + mx_scale_at(ru, 4 * kq, a.tiles_k)), word);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx4_dequantize_kernel(const MxArgs a) {
  using L = Lanes<T>;
  constexpr int kUnroll = kBackRows;
  pdl_begin();
  const int tx = threadIdx.x & ((1 << a.tx_shift) - 1), ty = threadIdx.x >> a.tx_shift;
  const int nty = kThreads >> a.tx_shift;
  const int64_t unit = ((int64_t)blockIdx.x << a.tx_shift) + tx;
  const int64_t c = unit * L::kElems;
  const int64_t r0 = blockIdx.y * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  const bool in_row = c / 2 < a.row_bytes;
  const bool full = c + L::kElems <= a.cols;
  T* y = static_cast<T*>(a.y) + (r0 + ty) * a.ld;
  for (int64_t r = r0 + ty; r < r1; r += (int64_t)kUnroll * nty) {
    uint32_t q[kUnroll][L::kElems / 8], s[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t ru = r + (int64_t)u * nty;
      s[u] = 0;
#pragma unroll
      for (int i = 0; i < L::kElems / 8; ++i) q[u][i] = 0;
      if (ru >= r1 || !in_row) continue;
      const uint8_t* p = a.codes + ru * a.row_bytes + c / 2;
      if constexpr (L::kElems == 16) {
        const uint2 v = AGN_LD(reinterpret_cast<const uint2*>(p));
        q[u][0] = v.x;
        q[u][1] = v.y;
      } else {
        q[u][0] = AGN_LD(reinterpret_cast<const uint32_t*>(p));
      }
      s[u] = AGN_LD(a.scales + mx_scale_at(ru, c / kMxBlock, a.tiles_k));
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u, y += nty * a.ld) {
      if (r + (int64_t)u * nty >= r1) break;
      const float scale = mx_scale_value(s[u]);
      Raw<T> out;
      T* e = reinterpret_cast<T*>(&out);
#pragma unroll
      for (int i = 0; i < L::kElems / 8; ++i) {
        float v[8];
        mx_unpack8(q[u][i], v);
#pragma unroll
        for (int j = 0; j < 8; ++j) e[8 * i + j] = static_cast<T>(__fmul_rn(v[j], scale));
      }
      if (full) {
        store32(y + c, a.vec, out);
      } else {
#pragma unroll
        for (int i = 0; i < L::kElems; ++i)
          if (c + i < a.cols) AGN_ST(y + c + i, e[i]);
      }
    }
  }
}

// Into rows that are not 16-byte aligned: a lane has the eight elements c .. c + 7 of a row
// that lie in aligned 16 (fp32: 32) bytes, c up to 7 before a multiple of 8; its codes are a
// piece of two words, its scales those of one block or two.  (us, with a lane's consecutive
// codes passed on by shuffles and stores of single elements, and so: 16384 x 4095 bf16 198, 66;
// 65536 x 100 bf16 27, 11; 2865 x 3183 fp32 13.7, 10.4.)
template <typename T>
__global__ void __launch_bounds__(kThreads) mx4_dequantize_shift_kernel(const MxArgs a) {
  constexpr int V = 8, kUnroll = kShiftRows;
  pdl_begin();
  const int tx = threadIdx.x & ((1 << a.tx_shift) - 1), ty = threadIdx.x >> a.tx_shift;
  const int nty = kThreads >> a.tx_shift;
  const int64_t c0 = (((int64_t)blockIdx.x << a.tx_shift) + tx) * V;
  const int64_t r0 = blockIdx.y * a.rows_per_block, r1 = min(a.rows, r0 + a.rows_per_block);
  const int64_t last = a.row_bytes / 4 - 1;   // a row's last word of codes
  T* y = static_cast<T*>(a.y);
  for (int64_t r = r0 + ty; r < r1; r += (int64_t)kUnroll * nty) {
    uint32_t lo[kUnroll], hi[kUnroll], s0[kUnroll], s1[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t ru = r + (int64_t)u * nty;
      lo[u] = hi[u] = s0[u] = s1[u] = 0;
      const int past = (int)(reinterpret_cast<uintptr_t>(y + ru * a.ld) / sizeof(T)) & (V - 1);
      const int64_t c = c0 - past;
      if (ru >= r1 || c >= a.cols) continue;
      const uint32_t* p = reinterpret_cast<const uint32_t*>(a.codes + ru * a.row_bytes);
      const int64_t w = c >> 3;   // (-1: the elements before the row)
      if (w >= 0) lo[u] = AGN_LD(p + w);
      if (w < last) hi[u] = AGN_LD(p + w + 1);
      const int64_t k0 = max(c, (int64_t)0) / kMxBlock, k1 = min(c + V - 1, a.cols - 1) / kMxBlock;
      s0[u] = AGN_LD(a.scales + mx_scale_at(ru, k0, a.tiles_k));
      s1[u] = k1 == k0 ? s0[u] : AGN_LD(a.scales + mx_scale_at(ru, k1, a.tiles_k));
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t ru = r + (int64_t)u * nty;
      if (ru >= r1) break;
      const int past = (int)(reinterpret_cast<uintptr_t>(y + ru * a.ld) / sizeof(T)) & (V - 1);
      const int64_t c = c0 - past;
      if (c >= a.cols) continue;
      float v[8];
      mx_unpack8(__funnelshift_r(lo[u], hi[u], 4 * (uint32_t)(c & 7)), v);
      const float by0 = mx_scale_value(s0[u]), by1 = mx_scale_value(s1[u]);
      const int first = kMxBlock - (int)(c & (kMxBlock - 1));   // elements of the first block
      alignas(16) T e[V];
#pragma unroll
      for (int i = 0; i < V; ++i)
        e[i] = static_cast<T>(__fmul_rn(v[i], i < first || c < 0 ? by0 : by1));
      T* to = y + ru * a.ld + c;
      if (c >= 0 && c + V <= a.cols) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
          AGN_ST(reinterpret_cast<uint4*>(to) + i, reinterpret_cast<const uint4*>(e)[i]);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (c + i >= 0 && c + i < a.cols) AGN_ST(to + i, e[i]);
      }
    }
  }
}

// Blocks of 2^tx_shift lanes along a row of `units` (2^word_shift to 256, what leaves the fewest
// idle) by rows_per_block rows, one wave of resident blocks.
dim3 geometry(MxArgs* a, int64_t units, int word_shift, int64_t resident) {
  int best = word_shift;
  int64_t pad = INT64_MAX;
  for (int s = 8; s >= word_shift; --s) {
    const int64_t p = round_up(units, (int64_t)1 << s);
    if (p < pad) {
      best = s;
      pad = p;
    }
  }
  a->tx_shift = best;
  const int64_t tiles = ceil_div(units, (int64_t)1 << best), nty = kThreads >> best;
  const int64_t most = std::max<int64_t>(1, resident / tiles);
  int64_t blocks = std::min<int64_t>(std::min<int64_t>(most, 65535), ceil_div(a->rows, nty));
  a->rows_per_block = ceil_div(a->rows, blocks);
  blocks = ceil_div(a->rows, a->rows_per_block);
  return dim3((unsigned)tiles, (unsigned)blocks);
}

int row_alignment(const void* p, int64_t ld, size_t es) {
  const uint64_t at = reinterpret_cast<uintptr_t>(p) | (uint64_t)ld * es;
  return at % 32 == 0 ? 2 : at % 16 == 0 ? 1 : 0;
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
  a.vec = row_alignment(x ? x : y, ld, f32 ? 4 : 2);
  const int es = f32 ? 4 : 2, word_shift = f32 ? 4 : 3;
  if (x) a.x_end = static_cast<const char*>(x) + matrix_bytes(rows, cols, ld, es);
  const bool shift = a.vec == 0;
  int dev = 0, sms = 0;
  AGN_TRY(current_device(&dev));
  AGN_TRY(device_sms(dev, &sms));
  const int64_t resident = (int64_t)sms * (x ? quant_blocks(f32) : kBackBlocks);
  const dim3 grid = !x && shift ? geometry(&a, ceil_div(cols, 8) + 1, 3, resident)
                                : geometry(&a, a.tiles_k << word_shift, word_shift, resident);
  auto k = x ? (shift ? (f32 ? mx4_quantize_kernel<float, true> : mx4_quantize_kernel<bf16, true>)
                      : (f32 ? mx4_quantize_kernel<float, false> : mx4_quantize_kernel<bf16, false>))
             : (shift ? (f32 ? mx4_dequantize_shift_kernel<float> : mx4_dequantize_shift_kernel<bf16>)
                      : (f32 ? mx4_dequantize_kernel<float> : mx4_dequantize_kernel<bf16>));
  AGN_TRY_CUDA(launch_pdl(k, grid, kThreads, 0, st, a));
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
