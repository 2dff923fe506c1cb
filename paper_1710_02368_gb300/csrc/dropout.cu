// Dropout of a layer's activations from a counter-based generator, with the
// layer's bias and ReLU (and a residual) in the same pass, and its gradient.
//
// Element (r, c) of a [rows][cols] matrix takes 16 bits of one splitmix64
// number (generator.cuh): number offset + r ceil(cols / 4) + floor(c / 4) of
// the stream key(seed, kDropout), bits 16 (c mod 4) and up, as u in [0, 65536).
// With T = round(65536 p) the element is kept iff u >= T, and kept values are
// scaled by 65536 / (65536 - T), so that the mean is exact for the probability
// that 16 bits can express (p is off by at most 2^-17).  The mask is a function
// of (seed, offset, r, c) alone: the backward pass computes it again, whatever
// its own layout, and nothing is stored.
//   forward : y = (keep ? act(x + b) scale : 0) + residual
//   backward: dx = keep and not (ReLU and x + b <= 0) ? dy scale : 0,
//             db[c] = sum_r dx[r][c] of the values before they are rounded
// One draw (two 64-bit multiplications, three shifts) serves four elements:
// 16 bits rather than 32 because the generator would otherwise take as many
// issue slots (about 14 an element) as a bf16 pass has at the memory's rate (22).
#include "generator.cuh"
#include "mlp.cuh"
#include "ops.cuh"

#include <cmath>

namespace agn {

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;      // rows of a thread whose loads are in flight together
constexpr int kBlocksPerSm = 4;
constexpr int kSumTxShift = 3;  // with sums: tiles of at most 8 units (128 bytes of a row)

struct DropArgs {
  const void* x;          // forward: input; backward: the layer's input (ReLU), or null
  const float* bias;      // [cols] or null
  const void* extra;      // forward: residual or null; backward: dy
  void* y;                // forward: output; backward: dx
  float* dbias;           // backward: [cols] or null
  int64_t rows, cols, ldx, lde, ldy;
  int64_t rows_per_block;
  uint64_t key, offset;
  uint32_t t16;           // T << 16
  float scale;
  int relu, vec;          // vec: every row of every matrix starts 16-byte aligned
  int tx_shift;           // log2 of the threads along a row
  // hidden layers of a training run (kHidden): matrices [slots][rows][cols]
  const int* slot_worker;
  const long long* slot_t0;
  int step, layers, layer;
  bf16* pieces;           // also the three exact bf16 pieces, planes `plane` apart; null = no
  int64_t plane;
};

// 16 bytes of a row, as they are: from aligned memory in one load, else the n
// valid elements one by one.
template <typename T>
__device__ __forceinline__ uint4 load16(const T* p, bool full, int n) {
  if (full) return AGN_LD(reinterpret_cast<const uint4*>(p));
  uint4 q = make_uint4(0, 0, 0, 0);
  T* e = reinterpret_cast<T*>(&q);
#pragma unroll
  for (int i = 0; i < (int)(16 / sizeof(T)); ++i)
    if (i < n) e[i] = AGN_LD(p + i);
  return q;
}
template <typename T>
__device__ __forceinline__ float element(const uint4& q, int i) {
  return static_cast<float>(reinterpret_cast<const T*>(&q)[i]);
}
template <typename T>
__device__ __forceinline__ void store16(T* p, bool full, int n, const float (&v)[16 / sizeof(T)]) {
  uint4 q;
  T* e = reinterpret_cast<T*>(&q);
#pragma unroll
  for (int i = 0; i < (int)(16 / sizeof(T)); ++i) e[i] = static_cast<T>(v[i]);
  if (full) {
    AGN_ST(reinterpret_cast<uint4*>(p), q);
  } else {
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i)
      if (i < n) AGN_ST(p + i, e[i]);
  }
}

// The keep mask of V consecutive elements from the draws of their groups of
// four: number i0 of the stream, and i0 + 1 for V = 8.  The upper half of a word
// compares as it is (u >= T iff word >= T << 16), the lower half shifted up.
template <int V>
__device__ __forceinline__ uint32_t keep_mask(uint64_t key, uint64_t i0, uint32_t t16) {
  uint32_t m = 0;
#pragma unroll
  for (int g = 0; g < V / 4; ++g) {
    const uint64_t d = gen::draw(key, i0 + g);
    const uint32_t w[2] = {(uint32_t)d, (uint32_t)(d >> 32)};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      m |= (w[h] << 16) >= t16 ? 1u << (4 * g + 2 * h) : 0u;
      m |= w[h] >= t16 ? 2u << (4 * g + 2 * h) : 0u;
    }
  }
  return m;
}

// A block: tiles of 2^tx_shift units of 16 bytes along the row (blockIdx.x) by
// rows_per_block rows (blockIdx.y); a thread keeps its columns (the bias stays
// in registers) and steps down the rows.
template <typename T, bool kBackward, bool kHidden>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) dropout_kernel(const DropArgs a) {
  constexpr int V = 16 / sizeof(T);
  pdl_begin();
  const int tx = threadIdx.x & ((1 << a.tx_shift) - 1), ty = threadIdx.x >> a.tx_shift;
  const int nty = kThreads >> a.tx_shift;
  const int64_t c = (((int64_t)blockIdx.x << a.tx_shift) + tx) * V;
  const int n = c < a.cols ? (int)min((int64_t)V, a.cols - c) : 0;   // elements of this thread
  const bool full = a.vec && n == V;
  const int64_t r0 = blockIdx.y * a.rows_per_block;
  const int64_t r1 = min(a.rows, r0 + a.rows_per_block);
  const uint64_t groups = (uint64_t)((a.cols + 3) / 4);
  const T* x = static_cast<const T*>(a.x);
  const T* extra = static_cast<const T*>(a.extra);
  T* y = static_cast<T*>(a.y);
  uint64_t key = a.key, first = a.offset;
  int64_t piece0 = 0;
  if (kHidden) {
    // the hidden layer of this slot's worker at its step counter (never reset):
    // agn_dropout with the worker's seed for the layer, offset t rows groups
    const int z = blockIdx.z, w = AGN_LD(a.slot_worker + z);
    const uint64_t t = (uint64_t)(AGN_LD(a.slot_t0 + z) + a.step);
    key = gen::key(gen::draw(a.key, (uint64_t)w * a.layers + a.layer), gen::kDropout);
    first = t * (uint64_t)a.rows * groups;
    x += z * a.rows * a.ldx;
    y += z * a.rows * a.ldy;
    piece0 = z * a.rows * a.ldy;
  }
  first += (uint64_t)c / 4;
  float b[V], sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    b[e] = a.bias && e < n ? AGN_LD(a.bias + c + e) : 0.f;
    sum[e] = 0.f;
  }
  if (n > 0) {
    for (int64_t r = r0 + ty; r < r1; r += (int64_t)kUnroll * nty) {
      uint4 v[kUnroll], q[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int64_t ru = r + (int64_t)u * nty;
        if (ru >= r1) break;
        if (!kBackward || a.relu) v[u] = load16(x + ru * a.ldx + c, full, n);
        if (kBackward || extra) q[u] = load16(extra + ru * a.lde + c, full, n);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int64_t ru = r + (int64_t)u * nty;
        if (ru >= r1) break;
        const uint32_t keep = keep_mask<V>(key, first + (uint64_t)ru * groups, a.t16);
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          bool k = (keep >> e) & 1;
          if (kBackward) {
            // (a value that is not a number passes, forward and backward)
            if (a.relu) k = k && !(__fadd_rn(element<T>(v[u], e), b[e]) <= 0.f);
            o[e] = k ? __fmul_rn(element<T>(q[u], e), a.scale) : 0.f;
            sum[e] += o[e];
          } else {
            float t = a.bias ? __fadd_rn(element<T>(v[u], e), b[e]) : element<T>(v[u], e);
            if (a.relu && t <= 0.f) t = 0.f;
            o[e] = k ? __fmul_rn(t, a.scale) : 0.f;
            if (extra) o[e] = __fadd_rn(o[e], element<T>(q[u], e));
          }
        }
        store16(y + ru * a.ldy + c, full, n, o);
        if (kHidden && a.pieces) {
          bf16* pp = a.pieces + piece0 + ru * a.ldy + c;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            if (e >= n) break;
            bf16 q0, q1, q2;
            split3(o[e], q0, q1, q2);
            AGN_ST(pp + e, q0);
            AGN_ST(pp + a.plane + e, q1);
            AGN_ST(pp + 2 * a.plane + e, q2);
          }
        }
      }
    }
  }
  if (kBackward && a.dbias) {
    // db of the block's columns: the threads of a column in order, then the
    // cluster's blocks (all the rows of these columns) in rank order through
    // distributed shared memory: no workspace, no atomics, the same bits each time
    __shared__ float part[kThreads * V];
    __shared__ float col[V << kSumTxShift];
    const int width = V << a.tx_shift;
#pragma unroll
    for (int e = 0; e < V; ++e) part[ty * width + tx * V + e] = sum[e];
    __syncthreads();
    for (int j = threadIdx.x; j < width; j += kThreads) {
      float s = 0.f;
      for (int t = 0; t < nty; ++t) s += part[t * width + j];
      col[j] = s;
    }
    cluster_sync();
    const int ranks = gridDim.y;
    for (int j = threadIdx.x; j < width; j += kThreads) {
      const int64_t cj = ((int64_t)blockIdx.x << a.tx_shift) * V + j;
      if (j % ranks != (int)blockIdx.y || cj >= a.cols) continue;
      float s = 0.f;
      for (int k = 0; k < ranks; ++k) s += ld_cluster(col + j, k);
      AGN_ST(a.dbias + cj, s);
    }
    cluster_sync();   // the other blocks' reads, before this one's memory goes
  }
}

// Threads along a row: a power of two up to `most`, the largest that wastes at
// most a sixteenth of the threads on columns past the end, else the least wasteful.
int pick_tx_shift(int64_t units, int most) {
  int best = 0;
  int64_t best_pad = units;
  for (int s = most; s >= 0; --s) {
    const int64_t pad = round_up(units, (int64_t)1 << s);
    if (pad * 16 <= units * 17) return s;
    if (s == most || pad < best_pad) {
      best = s;
      best_pad = pad;
    }
  }
  return best;
}

constexpr int kMaxCluster = 8;

template <typename T>
Status launch_dropout(DropArgs a, bool backward, int slots, cudaStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const int sms = current_sms();
  const int64_t units = ceil_div(a.cols, V);
  const bool sums = backward && a.dbias;
  a.tx_shift = pick_tx_shift(units, sums ? kSumTxShift : 5);
  const int64_t tiles = ceil_div(units, (int64_t)1 << a.tx_shift);
  const int nty = kThreads >> a.tx_shift;
  // one wave of resident blocks; with sums, all the rows of a column tile in a cluster
  const int64_t most = sums ? kMaxCluster
                            : std::max<int64_t>(1, (int64_t)sms * kBlocksPerSm / (tiles * slots));
  int64_t blocks = std::min<int64_t>(std::min<int64_t>(most, 65535),
                                     std::max<int64_t>(1, ceil_div(a.rows, nty)));
  a.rows_per_block = std::max<int64_t>(1, ceil_div(a.rows, blocks));
  if (!sums) blocks = std::max<int64_t>(1, ceil_div(a.rows, a.rows_per_block));
  const dim3 grid((unsigned)tiles, (unsigned)blocks, (unsigned)slots);
  if (a.slot_worker) {
    auto k = dropout_kernel<T, false, true>;
    AGN_TRY_CUDA(launch_pdl(k, grid, kThreads, 0, st, a));
  } else if (!backward) {
    auto k = dropout_kernel<T, false, false>;
    AGN_TRY_CUDA(launch_pdl(k, grid, kThreads, 0, st, a));
  } else if (!sums) {
    auto k = dropout_kernel<T, true, false>;
    AGN_TRY_CUDA(launch_pdl(k, grid, kThreads, 0, st, a));
  } else {
    auto k = dropout_kernel<T, true, false>;
    AGN_TRY_CUDA(launch_pdl_cluster(k, grid, kThreads, 0, dim3(1, grid.y, 1), st, a));
  }
  AGN_TRY_CUDA(cudaGetLastError());
  return Status::Ok();
}

Status run_dropout(DropArgs a, bool backward, int dtype, int slots, cudaStream_t st) {
  return dtype == AGN_PREC_FP32 ? launch_dropout<float>(a, backward, slots, st)
                                : launch_dropout<bf16>(a, backward, slots, st);
}

Status set_probability(double p, DropArgs* a) {
  uint32_t t;
  if (!dropout_threshold(p, &t, &a->scale))
    return Status::Err(AGN_E_INVALID, "the dropout probability must be in [0, 1)");
  a->t16 = t << 16;
  return Status::Ok();
}

bool rows_aligned(const void* p, int64_t ld, size_t es) {
  return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && (size_t)ld * es % 16 == 0);
}

Status forward(const void* x, const float* bias, const void* residual, void* y, int dtype,
               int relu, int64_t rows, int64_t cols, int64_t ldx, int64_t ldr, int64_t ldy,
               double p, uint64_t seed, uint64_t offset, cudaStream_t st) {
  const size_t es = dtype_size(dtype);
  if (!es) return Status::Err(AGN_E_INVALID, "unknown dtype");
  AGN_TRY(check_matrix("x", rows, cols, ldx));
  AGN_TRY(check_matrix("y", rows, cols, ldy));
  if (residual) AGN_TRY(check_matrix("residual", rows, cols, ldr));
  DropArgs a{};
  AGN_TRY(set_probability(p, &a));
  if (rows == 0 || cols == 0) return Status::Ok();
  if (!x || !y) return Status::Err(AGN_E_INVALID, "null pointer");
  const CallBuffer bx{"x", x, matrix_bytes(rows, cols, ldx, es), es},
      bb{"bias", bias, bias ? (size_t)cols * 4 : 0, 4},
      br{"residual", residual, residual ? matrix_bytes(rows, cols, ldr, es) : 0, es},
      by{"y", y, matrix_bytes(rows, cols, ldy, es), es};
  AGN_TRY(check_apart(by, {bb}));
  // in place: exactly x's (or the residual's) elements
  if (!(y == x && ldy == ldx)) AGN_TRY(check_apart(by, {bx}));
  if (!(y == residual && ldy == ldr)) AGN_TRY(check_apart(by, {br}));
  AGN_TRY(check_buffers({bx, bb, br, by}));
  a.x = x; a.bias = bias; a.extra = residual; a.y = y;
  a.rows = rows; a.cols = cols; a.ldx = ldx; a.lde = ldr; a.ldy = ldy;
  a.key = gen::key(seed, gen::kDropout);
  a.offset = offset;
  a.relu = relu != 0;
  a.vec = rows_aligned(x, ldx, es) && rows_aligned(y, ldy, es) && rows_aligned(residual, ldr, es);
  KnownBuffers known({bx, bb, br, by});
  AGN_TRY(bounds_upload(st));
  AGN_TRY(run_dropout(a, false, dtype, 1, st));
  return bounds_collect(st);
}

Status backward(const void* dy, const void* x, const float* bias, void* dx, float* dbias,
                int dtype, int relu, int64_t rows, int64_t cols, int64_t lddy, int64_t ldx,
                int64_t lddx, double p, uint64_t seed, uint64_t offset, cudaStream_t st) {
  const size_t es = dtype_size(dtype);
  if (!es) return Status::Err(AGN_E_INVALID, "unknown dtype");
  AGN_TRY(check_matrix("dy", rows, cols, lddy));
  AGN_TRY(check_matrix("dx", rows, cols, lddx));
  if (relu) AGN_TRY(check_matrix("x", rows, cols, ldx));
  DropArgs a{};
  AGN_TRY(set_probability(p, &a));
  if (cols == 0 || (rows == 0 && !dbias)) return Status::Ok();
  if (rows > 0 && (!dy || !dx || (relu && !x)))
    return Status::Err(AGN_E_INVALID, "null pointer (with relu the layer's input x is needed)");
  if (!relu) x = nullptr, bias = nullptr;   // not read
  const CallBuffer bg{"dy", dy, matrix_bytes(rows, cols, lddy, es), es},
      bx{"x", x, x ? matrix_bytes(rows, cols, ldx, es) : 0, es},
      bb{"bias", bias, bias ? (size_t)cols * 4 : 0, 4},
      bo{"dx", dx, matrix_bytes(rows, cols, lddx, es), es},
      bs{"dbias", dbias, dbias ? (size_t)cols * 4 : 0, 4};
  AGN_TRY(check_apart(bs, {bg, bx, bb, bo}));
  AGN_TRY(check_apart(bo, {bb}));
  if (!(dx == dy && lddx == lddy)) AGN_TRY(check_apart(bo, {bg}));
  if (!(dx == x && lddx == ldx)) AGN_TRY(check_apart(bo, {bx}));
  AGN_TRY(check_buffers({bg, bx, bb, bo, bs}));
  a.x = x; a.bias = bias; a.extra = dy; a.y = dx; a.dbias = dbias;
  a.rows = rows; a.cols = cols; a.ldx = ldx; a.lde = lddy; a.ldy = lddx;
  a.key = gen::key(seed, gen::kDropout);
  a.offset = offset;
  a.relu = relu != 0;
  a.vec = rows_aligned(x, ldx, es) && rows_aligned(dx, lddx, es) && rows_aligned(dy, lddy, es);
  KnownBuffers known({bg, bx, bb, bo, bs});
  AGN_TRY(bounds_upload(st));
  AGN_TRY(run_dropout(a, true, dtype, 1, st));
  return bounds_collect(st);
}

}  // namespace

bool dropout_threshold(double p, uint32_t* t, float* scale) {
  if (!(p >= 0.0 && p < 1.0)) return false;
  *t = (uint32_t)std::min(65535.0, std::nearbyint(p * 65536.0));
  *scale = (float)(65536.0 / (65536.0 - *t));
  return true;
}

template <typename T>
Status dropout_hidden(const HiddenDropArgs& h, int slots, cudaStream_t st) {
  if (slots <= 0) return Status::Ok();
  DropArgs a{};
  AGN_TRY(set_probability(h.p, &a));
  a.x = h.H; a.y = h.H;
  a.rows = h.m; a.cols = h.d; a.ldx = h.d; a.ldy = h.d;
  a.key = gen::key(h.seed, gen::kDropout);
  a.vec = rows_aligned(h.H, h.d, sizeof(T));
  a.slot_worker = h.slot_worker; a.slot_t0 = h.slot_t0;
  a.step = h.step; a.layers = h.layers; a.layer = h.layer;
  a.pieces = h.pieces; a.plane = h.plane;
  return launch_dropout<T>(a, false, slots, st);
}
template Status dropout_hidden<float>(const HiddenDropArgs&, int, cudaStream_t);
template Status dropout_hidden<bf16>(const HiddenDropArgs&, int, cudaStream_t);

AGN_BOUNDS_UNIT(dropout)

}  // namespace agn

extern "C" int agn_dropout(const void* x, const float* bias, const void* residual, void* y,
                           int32_t dtype, int32_t relu, int64_t rows, int64_t cols, int64_t ldx,
                           int64_t ldr, int64_t ldy, double p, uint64_t seed, uint64_t offset,
                           void* stream) {
  return agn::guarded([&] {
    return agn::forward(x, bias, residual, y, dtype, relu, rows, cols, ldx, ldr, ldy, p, seed,
                        offset, static_cast<cudaStream_t>(stream));
  });
}

extern "C" int agn_dropout_backward(const void* dy, const void* x, const float* bias, void* dx,
                                    float* dbias, int32_t dtype, int32_t relu, int64_t rows,
                                    int64_t cols, int64_t lddy, int64_t ldx, int64_t lddx,
                                    double p, uint64_t seed, uint64_t offset, void* stream) {
  return agn::guarded([&] {
    return agn::backward(dy, x, bias, dx, dbias, dtype, relu, rows, cols, lddy, ldx, lddx, p,
                         seed, offset, static_cast<cudaStream_t>(stream));
  });
}
