// Softmax cross-entropy of a linear layer over many classes, and its gradients, without
// the logits in memory (formulas in include/agn.h).
//
// Forward: one product x w^T whose epilogue keeps (maximum, sum of exponentials) of each row and
// half a tile of columns, 16 bytes for 256 logits; a small kernel joins them.  (Where tiles are few, or w is read as
// it is, the logits are in scratch for once: products by ranges of K.)  Backward, from the rows'
// lse alone: the product again, its epilogue turns logits into p, the gradient with respect
// to them (two bf16 pieces, of fp32 operands three), for a piece of the classes at a time; then dw = p^T x
// and dx += p w of the piece.  Pieces keep p's buffer at 128 MB, w's pieces of fp32 at 96 (384 for few rows); the
// products that read w as it is have one piece of all classes (up to 2^18, 201 MB of p).
// Rows without a label cost nothing and may hold anything: the rows with one are counted and, where
// some are missing, gathered on the device; all sizes that depend on it are read there.
// Small problems (w in a few 10 KB) take plain kernels instead: a block a row.
#include "linear_ce.cuh"

#include <cfloat>
#include <cmath>

#include "mlp_tc.cuh"
#include "ops.cuh"

namespace agn {
namespace ce {

namespace {

constexpr int kSms = 152;                       // what splits along K are made for
constexpr int64_t kPieceBytes = 128ll << 20;    // of p's pieces
constexpr int64_t kPackBytes = 96ll << 20;      // of w's pieces (they stay in the L2)
constexpr int64_t kPartBytes = 64ll << 20;      // of a product's sums by ranges along K
constexpr float kLog2e = 1.44269504088896340736f;

struct Sizes {
  int64_t rows, inner, classes;
  int prec;
};

// How one or two products of a launch are cut.
struct Cut {
  int ctas, bn;
  int64_t tiles[2];
  int splits[2];
  double time;   // estimated clocks
};
struct Extents {
  int64_t M, N, K;
  bool b_mn;
};

// The estimates below, in clocks and us of one GB300, decide between widths, cuts and kinds of kernels that are all right
// for a size: where their constants do not suit it, that costs time alone.
//
// Clocks of a tile's 64 k: the MMAs at 4096 multiply-adds a clock and SM, its operands at 64 bytes a clock
// from the L2, or shared memory at 128: what arrives, and what the MMAs read (B stored along N twice).
// fp32: six products of three pieces each.
double step_clocks(int ctas, int bn, int planes, int64_t a_box, bool b_mn) {
  const int products = planes == 3 ? 6 : 1;
  const double mma = bn * 2.0 * products, in = (a_box * 128 + bn / ctas * 128) * planes;
  const double read = (128 * 128 + bn / ctas * 128 * (b_mn ? 2 : 1)) * products;
  // (fp32 as measured: 128 columns wait for their operands, with B along either side, 256 for sums to be read)
  if (planes == 3 && bn < 256) return 1.3 * std::max(mma, (in + (128 * 128 + bn / ctas * 128) * products) / 128.0);
  return std::max({mma, in / 64.0, (in + read) / 128.0}) * (planes == 3 ? 1.1 : 1.0);
}

// Time of the CTA that ends last, in steps: `n` units of each of two kinds on `at_once` CTAs, the longer ones first
// and in turn, the others where there is least to do.
double makespan(int64_t at_once, const int64_t (&n)[2], const double (&cost)[2]) {
  const int longer = cost[1] > cost[0] ? 1 : 0;
  const int64_t q = n[longer] / at_once, rest = n[longer] % at_once, others = n[1 - longer];
  const double low = q * cost[longer], high = low + (rest ? cost[longer] : 0), each = cost[1 - longer];
  // By `high` the CTAs that have no longer unit more have done `ahead` of the shorter ones each, and `part` of another.
  const double apart = rest ? cost[longer] / each : 0;
  const int64_t ahead = (int64_t)(apart + 1e-9), left = others - (at_once - rest) * ahead;
  if (left <= 0) return high;
  // Then all do `late` each; what is still left takes those a part of one first.
  const double part = std::max(0.0, apart - (double)ahead);
  const int64_t late = left / at_once, over = left % at_once;
  return high + ((double)late + (over == 0 ? 0.0 : over <= at_once - rest ? 1.0 - part : 1.0)) * each;
}

// Tile width by the estimated time: rounds of tiles over the SMs, or B's bytes from memory (24 a clock and
// SM) if that is more.  Of products cut along K also the ranges: as many as even out the work, where
// that saves more than the pass over their sums costs.  A tile takes its epilogue's time at least, 14 clocks
// a column (fp32's 256, whose sums are read in between, 28).
Cut cut(int ctas, int planes, int a_box, const Extents* e, int n, bool ranges, double pass_clocks = 8000) {
  Cut best{};
  const int64_t at_once = kSms / ctas;
  int least = 64;   // (a box is 64 columns of an operand stored along N)
  for (int i = 0; i < n; ++i)
    if (e[i].b_mn && ctas == 2) least = 128;
  for (int bn = planes > 1 && ctas == 1 ? 128 : 256; bn >= least; bn /= 2) {
    Cut c{};
    c.ctas = ctas;
    c.bn = bn;
    const double finish = bn * (planes == 3 && bn == 256 ? 28 : 14);
    double step = 0;
    for (int i = 0; i < n; ++i) step = std::max(step, step_clocks(ctas, bn, planes, a_box, e[i].b_mn));
    double steps = 0, bytes = 0;
    int64_t tiles = 0, kt[2], most[2];
    for (int i = 0; i < n; ++i) {
      c.tiles[i] = ceil_div(e[i].M, 128 * ctas) * ceil_div(e[i].N, bn);
      c.splits[i] = 1;
      kt[i] = ceil_div(e[i].K, 64);
      most[i] = ranges ? std::min({kPartBytes / (round_up(e[i].M, 256) * round_up(e[i].N, 256) * 4), (int64_t)64,
                                   ceil_div((int64_t)std::ceil(kt[i] * step), 4000)})
                       : 1;
      tiles += c.tiles[i];
      steps += c.tiles[i] * std::max((double)kt[i], finish / step);
      bytes += (double)ceil_div(e[i].N, bn) * bn * kt[i] * 128 * planes;
    }
    double rounds = 0, more = 0;   // steps one after the other, clocks of passes over sums
    // writing and reading the sums of k ranges
    auto pass = [&](int i, int64_t k) { return pass_clocks + 250 * k + 2.0 * k * e[i].M * e[i].N * 4 / (24.0 * kSms); };
    if (n == 1) {
      auto after = [&](int64_t k) {
        return ceil_div(tiles * k, at_once) * std::max((double)ceil_div(kt[0], k), finish / step);
      };
      rounds = after(1);
      for (int64_t k = 2; k <= most[0]; ++k) {
        const double r = after(k);
        if (r * step + pass(0, k) < rounds * step + more) rounds = r, more = pass(0, k), c.splits[0] = (int)k;
      }
    } else {
      const double share = std::max(1.0, steps / at_once), beside = 0.5;
      double least_time = 0;
      for (int j = 0; j < 9; ++j) {   // each uncut, by its share of the work, or twice as often
        int64_t k[2], units[2];
        double cost[2], passes = 0;
        for (int i = 0; i < 2; ++i) {
          const int often = i ? j / 3 : j % 3;
          k[i] = often ? std::max<int64_t>(1, std::min<int64_t>(most[i], (int64_t)std::ceil(kt[i] / share) * often)) : 1;
          units[i] = c.tiles[i] * k[i];
          cost[i] = std::max((double)ceil_div(kt[i], k[i]), finish / step) + beside;
          if (k[i] > 1) passes += pass(i, k[i]);
        }
        const double r = makespan(at_once, units, cost);
        if (j == 0 || r * step + passes < least_time) {
          least_time = r * step + passes;
          rounds = r;
          more = passes;
          for (int i = 0; i < 2; ++i) c.splits[i] = (int)k[i];
        }
      }
    }
    c.time = std::max(rounds * step, bytes / (24.0 * kSms)) + more + 500.0 * tiles / at_once;
    if (best.bn == 0 || c.time < best.time) best = c;
  }
  return best;
}

// Plain kernels for small problems, where their estimated time (us: every row reads all of w from the L2, short
// rows a class a thread: 0.65 multiply-adds a picosecond forward and 0.17 backward, longer rows 1.9 and 0.36) is less
// than that of the products, whose launches (8 and 16) and k steps (1.2 fp32, 0.35 bf16) are one after the other.
bool small(const Sizes& s, bool backward) {
  if (s.rows > 1024 || s.classes > 4096 || s.inner * s.classes > 32768) return false;
  const double products = (double)s.rows * s.inner * s.classes;
  const double step = s.prec == AGN_PREC_FP32 ? 1.2 : 0.35, k = (double)ceil_div(s.inner, 64);
  if (!backward) return 3 + products / (s.inner <= 64 ? 0.65e6 : 1.9e6) < 8 + step * std::min(k, 12.0);
  return 5 + products / (s.inner <= 64 ? 0.17e6 : 0.36e6) < 16 + step * std::min(k + (double)(std::max(s.rows, s.classes) / 64), 24.0);
}

// Products that read fp32 w as it is, where it is not small (us forward and backward, w packed first in brackets: 56
// rows of 2392 to 55366 classes 138 and 467 (496 and -), 128 of 4096 to 32000 189 and 550 (502 and 976), 128 of
// 2048 to 8192 38 and 115 (68 and 126); 128 of 8192 to 300 26 and 58 (24 and 45): its launches are more).  Its logits lie in
// scratch, 134 MB for 128 rows and 2^18 classes, and 201 of p backward: more classes take the products of packed pieces,
// whose scratch does not grow with them.
bool raw(const Sizes& s) {
  return s.prec == AGN_PREC_FP32 && s.rows <= 128 && s.classes <= 1 << 18 && s.inner * s.classes >= 3 << 20;
}

// Ranges along K of such a product of M along w's side: by the time of the CTA that ends last and that of a pass
// over the ranges' sums; each has a step.
int raw_ranges(int64_t M, int64_t K, int64_t rows) {
  const int64_t tiles = ceil_div(M, 128), steps = ceil_div(K, 64);
  const double step = rows <= 64 ? 1800 : 2800;
  auto time = [&](int64_t k) {
    return (double)ceil_div(tiles * k, kSms) * ((double)ceil_div(steps, k) * step + 3000) + 250.0 * k +
           2.0 * (double)k * rows * M * 4 / (24.0 * kSms);
  };
  int64_t best = 1;
  for (int64_t k = 2; k <= std::min<int64_t>({steps, 64, kPartBytes / (round_up(rows, 64) * round_up(M, 64) * 4)}); ++k)
    if (ceil_div(steps, ceil_div(steps, k)) == k && time(k) < time(best)) best = k;
  return (int)best;
}

struct Layout {
  int planes, pieces_p;    // of x and w, of p
  int64_t kp;              // x's and w's row stride where they are packed (whole 128 bytes)
  bool direct;             // bf16 rows that the copy engine reads as they are
  int64_t rows_pad, piece; // classes of a piece (a multiple of 256, but for one piece of all)
  int64_t pieces, ldp;     // p's row stride
  Cut z;
  int z_splits;            // more than 1: the logits by ranges of K, in scratch (few tiles with a long K)
  int64_t ldz;
  int a_box;               // rows of x in a box of the logits' product
  bool both;               // dw and dx are one launch
  Cut grads[2];            // dw, dx (both: the first alone, with two products)
  int dw_splits, dx_splits;
  bool dx_part;
  bool x_t;                // dw reads x laid out along its rows
  bool small, few;
  bool raw;                // w is read as it is by its products (linear_ce_raw.cu), the logits are in scratch
  int64_t halves;          // forward: partial (maximum, sum) of a row
  size_t idx, live, x, xt, w, zs, ms, zlab, p, db, dxs, dws, bytes;
};

Layout layout(const Sizes& s, bool backward) {
  Layout l{};
  l.planes = s.prec == AGN_PREC_FP32 ? 3 : 1;
  l.pieces_p = p_pieces(l.planes);
  l.kp = round_up(s.inner, 64);
  l.direct = l.planes == 1 && s.inner % 8 == 0;
  l.rows_pad = round_up(s.rows, 256);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (size_t)round_up((int64_t)bytes, 1024);
    return here;
  };
  if (small(s, backward)) {
    l.small = true;
    if (backward) l.p = take((size_t)s.rows * s.classes * 4);
    l.bytes = std::max<size_t>(at, 1024);
    return l;
  }
  if (few(s.rows, s.prec, backward) && !(s.rows > 8 && raw(s))) {
    l.few = true;
    l.halves = few_blocks(s.classes);
    if (!backward) {
      l.ms = take((size_t)s.rows * l.halves * 8);
      l.zlab = take((size_t)s.rows * 4);
    } else {
      l.p = take((size_t)s.classes * few_rows(s.rows) * 4);
      l.dxs = take((size_t)few_cut(s.inner, s.classes, s.prec == AGN_PREC_FP32 ? 4 : 2).parts * s.rows * l.kp * 4);
    }
    l.bytes = at;
    return l;
  }
  l.raw = raw(s);
  if (l.raw) l.rows_pad = round_up(s.rows, 64);
  int64_t most = s.classes;
  auto limit = [&](int64_t bytes, int64_t each) { most = std::min(most, std::max<int64_t>(1024, bytes / each / 256 * 256)); };
  if (backward && !l.raw) limit(kPieceBytes, l.rows_pad * 2 * l.pieces_p);
  if (!l.direct && !l.raw) {   // (so many that tiles of few rows still occupy all SMs)
    const int64_t tm = ceil_div(s.rows, s.rows > 128 ? 256 : 128);
    const int64_t full = (s.rows > 128 ? kSms / 2 * 128 : kSms * 64) / tm;
    limit(std::max(kPackBytes, std::min(full * l.kp * 2 * l.planes, 4 * kPackBytes)), l.kp * 2 * l.planes);
  }
  limit((int64_t)1 << 29, std::max<int64_t>(1, l.rows_pad / 16384));   // tiles of a launch
  l.pieces = ceil_div(s.classes, most);
  l.a_box = (int)std::min<int64_t>(128, round_up(s.rows, 8));
  auto logits = [&](int64_t n) {
    const Extents e{s.rows, n, s.inner, false};
    return cut(s.rows > 128 ? 2 : 1, l.planes, l.a_box, &e, 1, false);
  };
  l.piece = most;
  if (l.pieces > 1) {   // pieces alike, or as large as they may be and one of the rest
    const int64_t alike = std::min(most, round_up(ceil_div(s.classes, l.pieces), 256));
    auto time = [&](int64_t n) {
      return (double)(s.classes / n) * logits(n).time + (s.classes % n ? logits(s.classes % n).time : 0);
    };
    if (time(alike) < time(most)) l.piece = alike;
  }
  l.pieces = ceil_div(s.classes, l.piece);
  l.ldp = round_up(l.piece, 64);
  l.z = logits(l.piece);
  l.z_splits = 1;
  if (l.raw) {
    l.z_splits = raw_ranges(s.classes, s.inner, s.rows);
  } else if (l.pieces == 1) {
    const Extents e{s.rows, s.classes, s.inner, false};
    const Cut c = cut(s.rows > 128 ? 2 : 1, l.planes, l.a_box, &e, 1, true, 2000);
    if (c.splits[0] > 1 && c.time < l.z.time) l.z = c, l.z_splits = c.splits[0];
  }
  l.live = take(4);
  l.idx = take((size_t)l.rows_pad * 4);
  l.x = take((size_t)l.planes * l.rows_pad * l.kp * 2);
  if (!l.direct && !l.raw) l.w = take((size_t)l.planes * l.piece * l.kp * 2);
  if (l.z_splits > 1 || l.raw) {
    l.ldz = round_up(s.classes, 64);
    l.zs = take((size_t)l.z_splits * l.rows_pad * l.ldz * 4);
  }
  if (!backward) {
    l.halves = 2 * (ceil_div(l.piece, l.z.bn) * (l.pieces - 1) +
                    ceil_div(s.classes - (l.pieces - 1) * l.piece, l.z.bn));
    l.ms = take((size_t)l.halves * l.rows_pad * 8);
    l.zlab = take((size_t)l.rows_pad * 4);
  } else {
    l.p = take((size_t)l.pieces_p * l.rows_pad * l.ldp * 2);
    l.db = take((size_t)(l.rows_pad / 32) * l.ldp * 4);
    // x along its rows, for dw, where the products' gain (us, a fifth of their time) is more than a pass over x
    const double elements = (double)s.rows * s.inner;
    l.x_t = elements * s.classes * (l.planes == 3 ? 14e-10 : 4.6e-10) > elements * (l.planes == 3 ? 1.5e-6 : 0.6e-6) + 2.5;
    if (l.x_t) l.xt = take((size_t)l.planes * round_up(s.inner, 64) * l.rows_pad * 2);
    const int64_t twice = l.planes == 1 ? 2 : 1;   // (steps along K for p's two pieces)
    const Extents e[2] = {{l.piece, s.inner, twice * round_up(s.rows, 64), !l.x_t},     // dw
                          {s.inner, s.rows, twice * round_up(l.piece, 64), false}};     // dx (transposed)
    const int dw_ctas = l.piece > 128 ? 2 : 1, dx_ctas = s.inner > 128 ? 2 : 1;
    for (int i = 0; i < 2; ++i) l.grads[i] = cut(i ? dx_ctas : dw_ctas, l.planes, 128, e + i, 1, true);
    if (dw_ctas == dx_ctas && !l.raw) {   // one launch, where one width suits both
      const Cut c = cut(dw_ctas, l.planes, 128, e, 2, true);
      l.both = c.time < l.grads[0].time + l.grads[1].time + 8000;
      if (l.both) l.grads[0] = c;
    }
    l.dw_splits = l.grads[0].splits[0];
    l.dx_splits = l.raw ? raw_ranges(s.inner, s.classes, s.rows) : l.both ? l.grads[0].splits[1] : l.grads[1].splits[0];
    l.dx_part = l.pieces > 1 || l.dx_splits > 1 || l.raw;
    if (l.dx_part) l.dxs = take((size_t)l.dx_splits * l.rows_pad * round_up(s.inner, 64) * 4);
    if (l.dw_splits > 1)
      l.dws = take((size_t)l.dw_splits * round_up(l.piece, 256) * round_up(s.inner, 64) * 4);
  }
  l.bytes = at;
  return l;
}

// ------------------------------------------------------------------ kernels

constexpr int kThreads = 256;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float* p, float v) { AGN_ST(p, v); }
__device__ __forceinline__ void from_float(bf16* p, float v) { AGN_ST(p, __float2bfloat16_rn(v)); }

// The places of the rows with a label, in order, and their number: one block, 8 rows a thread at a time.
__global__ void __launch_bounds__(1024) rows_kernel(const int* labels, int rows, int classes, int* idx, int* live) {
  pdl_begin();
  __shared__ int sums[33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int base = 0;
  for (int r0 = 0; r0 < rows; r0 += 8192) {
    const int first = r0 + 8 * threadIdx.x;
    uint32_t mask = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (first + i < rows && has_label(AGN_LD(labels + first + i), classes)) mask |= 1u << i;
    const int n = __popc(mask);
    int before = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += v;
    }
    if (lane == 31) sums[warp] = before;
    __syncthreads();
    if (warp == 0) {
      int v = sums[lane], all = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int w = __shfl_up_sync(0xffffffffu, all, o);
        if (lane >= o) all += w;
      }
      sums[lane] = all - v;
      if (lane == 31) sums[32] = all;
    }
    __syncthreads();
    int to = base + sums[warp] + before - n;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (mask >> i & 1) AGN_ST(idx + to++, first + i);
    base += sums[32];
    __syncthreads();
  }
  if (threadIdx.x == 0) AGN_ST(live, base);
}

// Eight columns from c on of a row of `inner` elements (null: zeros) to dst, as bf16 or three pieces.
template <typename T>
__device__ __forceinline__ void pack8(const T* row, int inner, int c, bf16* dst, int64_t plane) {
  float v[8];
  if (row && inner % 8 == 0 && c < inner) {   // (rows are 16-byte aligned then)
    constexpr int n = 16 / (int)sizeof(T);
#pragma unroll
    for (int j = 0; j < 8 / n; ++j) {
      const uint4 q = AGN_LD(reinterpret_cast<const uint4*>(row + c) + j);
      const T* e = reinterpret_cast<const T*>(&q);
#pragma unroll
      for (int k = 0; k < n; ++k) v[j * n + k] = to_float(e[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = row && c + k < inner ? to_float(AGN_LD(row + c + k)) : 0.f;
  }
  bf16 q[3][8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (sizeof(T) == 4) split3(v[k], q[0][k], q[1][k], q[2][k]);
    else q[0][k] = __float2bfloat16_rn(v[k]);
  }
#pragma unroll
  for (int j = 0; j < (sizeof(T) == 4 ? 3 : 1); ++j)
    AGN_ST(reinterpret_cast<uint4*>(dst + j * plane + c), *reinterpret_cast<const uint4*>(q[j]));
}

// A matrix to be packed: rows with zeros up to the stride.
template <typename T>
struct Pack {
  const T* src;
  int64_t rows;
  int inner;
  bf16* dst;
  int64_t ld, plane;
};

template <typename T>
__device__ __forceinline__ void pack_rows(const Pack<T>& p, int64_t first, int64_t step) {
  const int groups = (int)(p.ld / 8);
  for (int64_t i = first; i < p.rows * groups; i += step) {
    const int64_t r = i / groups;
    pack8(p.src + r * p.inner, p.inner, (int)(i - r * groups) * 8, p.dst + r * p.ld, p.plane);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) pack_kernel(const Pack<T> p) {
  pdl_begin();
  pack_rows(p, (int64_t)blockIdx.x * blockDim.x + threadIdx.x, (int64_t)gridDim.x * blockDim.x);
}

// x's rows with a label to consecutive rows (and zeros up to a multiple of 64 rows); nothing where the copy
// engine reads x itself (direct) and no row is missing.  dx: its rows without a label are zeroed.
template <typename T>
__global__ void __launch_bounds__(kThreads)
gather_kernel(const Pack<T> x, bool direct, const int* idx, const int* live_p, const int* labels, int classes, T* dx) {
  pdl_begin();
  const int64_t first = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
  const int groups = (int)(x.ld / 8);
  const int64_t live = AGN_LD(live_p), out_rows = (live + 63) / 64 * 64;
  if (live < x.rows && dx) {
    for (int64_t i = first; i < x.rows * x.inner; i += step)
      if (!has_label(AGN_LD(labels + i / x.inner), classes)) from_float(dx + i, 0.f);
  }
  if (direct && live == x.rows) return;
  for (int64_t i = first; i < out_rows * groups; i += step) {
    const int64_t r = i / groups;
    pack8(r < live ? x.src + (int64_t)AGN_LD(idx + r) * x.inner : nullptr, x.inner, (int)(i - r * groups) * 8,
          x.dst + r * x.ld, x.plane);
  }
}

// rows_kernel, gather_kernel and w's packing in one launch for up to kMostRows rows: a block has a range of
// rows, and each counts all labels, so that none waits for another (16384 labels: 1 us).
constexpr int kMostRows = 32768, kRangeRows = 256;
template <typename T>
__global__ void __launch_bounds__(1024)
prepare_kernel(const Pack<T> x, const Pack<T> w, bool direct, int range, const int* labels, int classes, int* idx,
               int* live_p, T* dx) {
  pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rows = (int)x.rows, r0 = min(rows, (int)blockIdx.x * range), r1 = min(rows, r0 + range);
  __shared__ int counts[2][32];
  __shared__ int list[kRangeRows], first_of[kRangeRows / 32];
  __shared__ bool known[kRangeRows];
  int all = 0, before = 0;
#pragma unroll 8
  for (int i = threadIdx.x; i < rows; i += 1024) {
    const int n = has_label(AGN_LD(labels + i), classes);
    all += n;
    before += i < r0 ? n : 0;
  }
  all = __reduce_add_sync(0xffffffffu, all);
  before = __reduce_add_sync(0xffffffffu, before);
  if (lane == 0) counts[0][warp] = all, counts[1][warp] = before;
  const int mine = r0 + (int)threadIdx.x;
  bool has = false;
  uint32_t ballot = 0;
  if (warp < kRangeRows / 32) {
    has = mine < r1 && has_label(AGN_LD(labels + mine), classes);
    ballot = __ballot_sync(0xffffffffu, has);
    if (lane == 0) first_of[warp] = __popc(ballot);
    known[threadIdx.x] = has;
  }
  __syncthreads();
  all = __reduce_add_sync(0xffffffffu, counts[0][lane]);
  before = __reduce_add_sync(0xffffffffu, counts[1][lane]);
  int n = 0;   // of this range
#pragma unroll
  for (int k = 0; k < kRangeRows / 32; ++k) {
    if (k == warp && has) {
      const int at = n + __popc(ballot & ((1u << lane) - 1));
      list[at] = mine;
      AGN_ST(idx + before + at, mine);
    }
    n += first_of[k];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) AGN_ST(live_p, all);
  __syncthreads();
  const int groups = (int)(x.ld / 8);
  if (!direct || all < rows) {
    for (int i = threadIdx.x; i < n * groups; i += 1024) {
      const int r = i / groups;
      pack8(x.src + (int64_t)list[r] * x.inner, x.inner, (i - r * groups) * 8, x.dst + (int64_t)(before + r) * x.ld,
            x.plane);
    }
    for (int r = all + blockIdx.x; r < (all + 63) / 64 * 64; r += gridDim.x)
      for (int i = threadIdx.x; i < groups; i += 1024) pack8((const T*)nullptr, x.inner, i * 8, x.dst + (int64_t)r * x.ld, x.plane);
  }
  if (dx && all < rows) {
    for (int i = threadIdx.x; i < (r1 - r0) * x.inner; i += 1024)
      if (!known[i / x.inner]) from_float(dx + (int64_t)r0 * x.inner + i, 0.f);
  }
  if (w.src) pack_rows(w, (int64_t)blockIdx.x * 1024 + threadIdx.x, (int64_t)gridDim.x * 1024);
}

// dst [inner][ld] = x's rows with a label along their columns (zeros up to a multiple of 64 rows), tiles of
// 64 x 64 elements through shared memory.
template <typename T>
__global__ void __launch_bounds__(kThreads)
transpose_kernel(const T* x, int inner, const int* idx, const int* live_p, bf16* dst, int64_t ld, int64_t plane) {
  pdl_begin();
  constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
  __shared__ bf16 tile[kPlanes][64][66];   // [column][row]
  const int live = AGN_LD(live_p), tiles_r = (live + 63) / 64, tiles_c = (inner + 63) / 64;
  constexpr int kVec = 16 / (int)sizeof(T), kPieces = 64 / kVec;   // 16 bytes of a row a thread
  const bool vec = inner % kVec == 0;
  for (int64_t t = blockIdx.x; t < (int64_t)tiles_r * tiles_c; t += gridDim.x) {
    const int r0 = (int)(t / tiles_c) * 64, c0 = (int)(t % tiles_c) * 64;
    __syncthreads();
    uint4 raw[kPieces / 4];
#pragma unroll
    for (int j = 0; j < kPieces / 4; ++j) {
      const int i = j * kThreads + threadIdx.x, r = i / kPieces, c = i % kPieces * kVec;
      alignas(16) T e[kVec] = {};
      if (r0 + r < live && c0 + c < inner) {
        const T* p = x + (int64_t)AGN_LD(idx + r0 + r) * inner + c0 + c;
        if (vec) {
          *reinterpret_cast<uint4*>(e) = AGN_LD(reinterpret_cast<const uint4*>(p));
        } else {
          for (int k = 0; k < kVec; ++k)
            if (c0 + c + k < inner) e[k] = AGN_LD(p + k);
        }
      }
      raw[j] = *reinterpret_cast<const uint4*>(e);
    }
#pragma unroll
    for (int j = 0; j < kPieces / 4; ++j) {
      const int i = j * kThreads + threadIdx.x, r = i / kPieces, c = i % kPieces * kVec;
      const T* e = reinterpret_cast<const T*>(&raw[j]);
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        const float v = to_float(e[k]);
        bf16 q[3];
        if (kPlanes == 3) split3(v, q[0], q[1], q[2]);
        else q[0] = __float2bfloat16_rn(v);
#pragma unroll
        for (int p = 0; p < kPlanes; ++p) tile[p][c + k][r] = q[p];
      }
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < kPlanes; ++p)
#pragma unroll 2
      for (int i = threadIdx.x; i < 64 * 8; i += kThreads) {   // 8 rows a thread
        const int c = i >> 3, r = (i & 7) * 8;
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const uint32_t*>(&tile[p][c][r + 2 * k]);
        if (c0 + c < inner)
          AGN_ST(reinterpret_cast<uint4*>(dst + p * plane + (int64_t)(c0 + c) * ld + r0 + r),
                 make_uint4(w[0], w[1], w[2], w[3]));
      }
  }
}

// lse and loss from the partial maxima and sums: a warp a row, or where there are few rows a block.  idx
// null: no row was moved.
__global__ void __launch_bounds__(kThreads)
join_kernel(const float2* ms, int halves, int64_t ld, int rows_a_block, const float* zlab, const int* labels,
            int classes, int rows, const int* idx, const int* live_p, float* loss, float* lse) {
  pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int live = idx ? AGN_LD(live_p) : rows;
  const int shared_by = kThreads / 32 / rows_a_block;   // warps of a row
  const int row = blockIdx.x * rows_a_block + warp / shared_by, part = warp % shared_by;
  float2 v = make_float2(-INFINITY, 0.f);
  if (row < live) {
    const float2* p = ms + (int64_t)row * ld;
    for (int j = part * 32 + lane; j < halves; j += 4 * 32 * shared_by) {
      float2 q[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int at = j + k * 32 * shared_by;
        q[k] = at < halves ? AGN_LD(p + at) : make_float2(-INFINITY, 0.f);
      }
      v = join(v, join(join(q[0], q[1]), join(q[2], q[3])));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    v = join(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
  if (shared_by > 1) {   // (the same for all: a block a row)
    __shared__ float2 parts[kThreads / 32];
    if (lane == 0) parts[warp] = v;
    __syncthreads();
    if (part != 0) return;
    for (int j = 1; j < shared_by; ++j) v = join(v, parts[warp + j]);
  }
  if (lane != 0) return;
  if (row < live && (idx || has_label(AGN_LD(labels + row), classes))) {
    const int at = idx ? AGN_LD(idx + row) : row;
    const float total = v.x == -INFINITY && v.y == 0.f ? -INFINITY : v.x + logf(v.y);
    AGN_ST(lse + at, total);
    AGN_ST(loss + at, total == -INFINITY ? INFINITY : total - AGN_LD(zlab + row));
  }
  if (row < rows && !has_label(AGN_LD(labels + row), classes)) {
    AGN_ST(lse + row, 0.f);
    AGN_ST(loss + row, 0.f);
  }
}

// ---- logits that lie in scratch as sums of ranges along K

struct Logits {
  const float* z;           // [splits][rows_pad][ld]
  int splits;
  int64_t plane, ld;
  const float* bias;
  const int* labels;
  int classes, rows;
  const int *idx, *live;    // null: rows are where they were
};

// Four logits from class c on of row r (past the last class: minus infinity).
__device__ __forceinline__ void logits4(const Logits& a, int64_t r, int c, float (&v)[4]) {
  const float* p = a.z + r * a.ld + c;
  float4 s = AGN_LD(reinterpret_cast<const float4*>(p));
#pragma unroll 4
  for (int k = 1; k < a.splits; ++k) {
    const float4 q = AGN_LD(reinterpret_cast<const float4*>(p + k * a.plane));
    s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
  }
  v[0] = s.x; v[1] = s.y; v[2] = s.z; v[3] = s.w;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    v[j] = c + j < a.classes ? v[j] + (a.bias ? AGN_LD(a.bias + c + j) : 0.f) : -INFINITY;
}

// lse and loss, a block a row (of many threads where rows are few).
__global__ void __launch_bounds__(1024) logits_loss_kernel(const Logits a, float* loss, float* lse) {
  pdl_begin();
  __shared__ float2 parts[32];
  __shared__ float picked;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x;
  const bool own = has_label(AGN_LD(a.labels + row), a.classes);
  if (threadIdx.x == 0 && !own) {
    AGN_ST(lse + row, 0.f);
    AGN_ST(loss + row, 0.f);
  }
  if (a.idx ? row >= AGN_LD(a.live) : !own) return;   // (the same for the block)
  const int at = a.idx ? AGN_LD(a.idx + row) : row, label = AGN_LD(a.labels + at);
  float2 v = make_float2(-INFINITY, 0.f);
  for (int c = threadIdx.x * 4; c < a.classes; c += blockDim.x * 4) {
    float z[4];
    logits4(a, row, c, z);
    float most = v.x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      most = fmaxf(most, z[j]);
      if (c + j == label) picked = z[j];
    }
    const float from = most == -INFINITY ? 0.f : most;
    v.y *= exp2f((v.x - from) * kLog2e);
#pragma unroll
    for (int j = 0; j < 4; ++j) v.y += exp2f((z[j] - from) * kLog2e);
    v.x = most;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    v = join(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
  if (lane == 0) parts[warp] = v;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int j = 1; j < (int)blockDim.x / 32; ++j) v = join(v, parts[j]);
  const float total = v.x == -INFINITY && v.y == 0.f ? -INFINITY : v.x + logf(v.y);
  AGN_ST(lse + at, total);
  AGN_ST(loss + at, total == -INFINITY ? INFINITY : total - picked);
}

// p and its sums over 32 rows: 32 rows x 64 columns a block, eight columns a thread.
template <int kPieces>
__global__ void __launch_bounds__(kThreads)
logits_grad_kernel(const Logits a, const float* lse, const float* dloss, const float* dlse, float scale, bf16* p,
                   int64_t ldp, int64_t plane, float* db) {
  pdl_begin();
  __shared__ float sums[32][65];
  const int live = AGN_LD(a.live);
  const int row0 = blockIdx.y * 32, row = row0 + (threadIdx.x >> 3), c0 = blockIdx.x * 64, c = c0 + (threadIdx.x & 7) * 8;
  if (row0 >= (live + 63) / 64 * 64) return;   // (rows up to a multiple of 64 are zeros)
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.f;
  if (row < live && c < a.classes) {
    const int at = AGN_LD(a.idx + row), label = AGN_LD(a.labels + at);
    const float total = AGN_LD(lse + at), dl = dloss ? AGN_LD(dloss + at) : 1.f, fb = scale * dl;
    const float fa = dlse ? scale * (dl + AGN_LD(dlse + at)) : fb;
    if (total != -INFINITY) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float z[4];
        logits4(a, row, c + 4 * h, z);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[4 * h + j] = fa * exp2f((z[j] - total) * kLog2e);
          if (c + 4 * h + j == label) v[4 * h + j] -= fb;
        }
      }
    }
  }
  bf16 q[3][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    split3(v[i], q[0][i], q[1][i], q[2][i]);
    sums[threadIdx.x >> 3][(threadIdx.x & 7) * 8 + i] = v[i];
  }
#pragma unroll
  for (int k = 0; k < kPieces; ++k)
    AGN_ST(reinterpret_cast<uint4*>(p + k * plane + row * ldp + c), *reinterpret_cast<const uint4*>(q[k]));
  if (!db) return;
  __syncthreads();
  if (threadIdx.x < 64 && c0 + (int)threadIdx.x < a.classes && row0 < live) {
    float s = 0.f;
#pragma unroll 8
    for (int r = 0; r < 32; ++r) s += sums[r][threadIdx.x];
    AGN_ST(db + (int64_t)blockIdx.y * ldp + c0 + threadIdx.x, s);
  }
}

// What a piece leaves to be added up, a launch for all of it.
// Threads of a block: many where the sums of a column are (16384 rows have 512 of 32 rows: 8 warps took 3 us more).
constexpr int kSumThreads = 1024;
int sum_threads(int64_t rows, bool dbias) { return dbias && rows > 2048 ? kSumThreads : 256; }
template <typename T>
struct Ranges {   // out[idx[m]][n] = the sum of the ranges' sums, in order (idx null: row m)
  const float* part;
  int splits;
  int64_t plane, ld, rows;
  int cols;
  const int* idx;
  T* out;
  bool vec;
  int blocks;     // of the launch
};
struct Columns {  // out[c] = the sums of 32 rows each, in order
  const float* db;
  int64_t ld;
  int cols;
  float* out;
  int blocks;
};

template <typename T>
__device__ __forceinline__ void sum_ranges(const Ranges<T>& a, int block, int live) {
  const int64_t rows = a.idx ? live : a.rows;
  const int groups = (a.cols + 3) / 4;
  const int64_t step = (int64_t)a.blocks * blockDim.x;
  for (int64_t i = (int64_t)block * blockDim.x + threadIdx.x; i < rows * groups; i += step) {
    const int64_t r = i / groups;
    const int c = (int)(i - r * groups) * 4;
    const float* p = a.part + r * a.ld + c;
    float4 s = AGN_LD(reinterpret_cast<const float4*>(p));
#pragma unroll 8
    for (int k = 1; k < a.splits; ++k) {
      const float4 v = AGN_LD(reinterpret_cast<const float4*>(p + k * a.plane));
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const int64_t to = (a.idx ? (int64_t)AGN_LD(a.idx + r) : r) * a.cols + c;
    const float v[4] = {s.x, s.y, s.z, s.w};
    if (a.vec && c + 4 <= a.cols) {
      if (sizeof(T) == 4) {
        AGN_ST(reinterpret_cast<float4*>(a.out + to), s);
      } else {
        const __nv_bfloat162 o[2] = {__floats2bfloat162_rn(v[0], v[1]), __floats2bfloat162_rn(v[2], v[3])};
        AGN_ST(reinterpret_cast<uint2*>(a.out + to), *reinterpret_cast<const uint2*>(o));
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < a.cols) from_float(a.out + to + k, v[k]);
    }
  }
}

// 32 columns a block, whose warps share the blocks of rows; a warp's sum carries what rounding leaves (2^28 rows are
// 2^18 additions for it; Knuth's two-sum).
__device__ __forceinline__ void sum_columns(const Columns& a, int block, int live) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int blocks = (live + 31) / 32, c = block * 32 + lane;
  __shared__ float part[kSumThreads / 32][33];
  float s = 0.f, rest = 0.f;
  if (c < a.cols) {
#pragma unroll 4
    for (int b = warp; b < blocks; b += warps) {
      const float v = AGN_LD(a.db + b * a.ld + c), both = __fadd_rn(s, v), back = __fsub_rn(both, s);
      rest = __fadd_rn(rest, __fadd_rn(__fsub_rn(s, __fsub_rn(both, back)), __fsub_rn(v, back)));
      s = both;
    }
    if (fabsf(s) <= FLT_MAX) s += rest;   // (an infinite sum's remainder is NaN)
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= a.cols) return;
  for (int j = 1; j < warps; ++j) s += part[j][lane];
  AGN_ST(a.out + c, s);
}

template <typename T>
__global__ void __launch_bounds__(kSumThreads)
sums_kernel(const Columns db, const Ranges<T> dw, const Ranges<T> dx, const int* live_p) {
  pdl_begin();
  const int live = AGN_LD(live_p);
  int block = blockIdx.x;
  if (block < db.blocks) return sum_columns(db, block, live);
  block -= db.blocks;
  if (block < dw.blocks) return sum_ranges(dw, block, live);
  sum_ranges(dx, block - dw.blocks, live);
}

// ---- small problems: a block a row, fp32 arithmetic

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// A row's logits into shared memory z [classes]: short rows a class a thread, with x [64] in shared memory
// too, others four classes a warp, 16 bytes a lane where rows are aligned.
template <typename T>
__device__ __forceinline__ void logits(const T* x, const T* w, const float* bias, int inner, int classes, float* xs,
                                       float* z) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (inner <= 64) {
    if ((int)threadIdx.x < inner) xs[threadIdx.x] = to_float(AGN_LD(x + threadIdx.x));
    __syncthreads();
    for (int c = threadIdx.x; c < classes; c += kThreads) {
      const T* p = w + c * inner;
      float s = 0.f;
#pragma unroll 8
      for (int k = 0; k < inner; ++k) s = fmaf(xs[k], to_float(AGN_LD(p + k)), s);
      z[c] = s + (bias ? AGN_LD(bias + c) : 0.f);
    }
  } else {
    constexpr int n = 16 / (int)sizeof(T);
    for (int c = 4 * warp; c < classes; c += 4 * (kThreads / 32)) {
      float s[4] = {0.f, 0.f, 0.f, 0.f};
      const T* rows[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) rows[j] = w + min(c + j, classes - 1) * inner;
      if (inner % n == 0) {
#pragma unroll 2
        for (int k = lane * n; k < inner; k += 32 * n) {
          const uint4 xq = AGN_LD(reinterpret_cast<const uint4*>(x + k));
          const T* xe = reinterpret_cast<const T*>(&xq);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint4 wq = AGN_LD(reinterpret_cast<const uint4*>(rows[j] + k));
            const T* we = reinterpret_cast<const T*>(&wq);
#pragma unroll
            for (int e = 0; e < n; ++e) s[j] = fmaf(to_float(xe[e]), to_float(we[e]), s[j]);
          }
        }
      } else {
#pragma unroll 4
        for (int k = lane; k < inner; k += 32) {
          const float xv = to_float(AGN_LD(x + k));
#pragma unroll
          for (int j = 0; j < 4; ++j) s[j] = fmaf(xv, to_float(AGN_LD(rows[j] + k)), s[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j] = warp_sum(s[j]);
        if (lane == 0 && c + j < classes) z[c + j] = s[j] + (bias ? AGN_LD(bias + c + j) : 0.f);
      }
    }
  }
  __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
small_loss_kernel(const T* x, const T* w, const float* bias, const int* labels, int inner, int classes, float* loss,
                  float* lse) {
  pdl_begin();
  extern __shared__ float z[];
  __shared__ float xs[64], warps[kThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x;
  const int label = AGN_LD(labels + row);
  if (!has_label(label, classes)) {   // (the same for the block)
    if (threadIdx.x == 0) {
      AGN_ST(lse + row, 0.f);
      AGN_ST(loss + row, 0.f);
    }
    return;
  }
  logits(x + (int64_t)row * inner, w, bias, inner, classes, xs, z);
  float most = -INFINITY;
  for (int c = threadIdx.x; c < classes; c += kThreads) most = fmaxf(most, z[c]);
  most = warp_max(most);
  if (lane == 0) warps[warp] = most;
  __syncthreads();
  for (int j = 0; j < kThreads / 32; ++j) most = fmaxf(most, warps[j]);
  const float from = most == -INFINITY ? 0.f : most;
  float s = 0.f;
  for (int c = threadIdx.x; c < classes; c += kThreads) s += exp2f((z[c] - from) * kLog2e);
  s = warp_sum(s);
  __syncthreads();
  if (lane == 0) warps[warp] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int j = 1; j < kThreads / 32; ++j) s += warps[j];
    const float total = most == -INFINITY && s == 0.f ? -INFINITY : most + logf(s);
    AGN_ST(lse + row, total);
    AGN_ST(loss + row, total == -INFINITY ? INFINITY : total - z[label]);
  }
}

// p [rows][classes] (fp32) and dx.
template <typename T>
__global__ void __launch_bounds__(kThreads)
small_rows_kernel(const T* x, const T* w, const float* bias, const int* labels, const float* lse, const float* dloss,
                  const float* dlse, float scale, int inner, int classes, float* p, T* dx) {
  pdl_begin();
  extern __shared__ float z[];
  __shared__ float xs[64], part[kThreads / 32][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x;
  const int label = AGN_LD(labels + row);
  const bool known = has_label(label, classes);   // (the same for the block)
  const float total = known ? AGN_LD(lse + row) : 0.f;
  const bool live = known && total != -INFINITY;
  float fa = 0.f, fb = 0.f;
  if (live) {
    const float dl = dloss ? AGN_LD(dloss + row) : 1.f;
    fb = scale * dl;
    fa = dlse ? scale * (dl + AGN_LD(dlse + row)) : fb;
    logits(x + (int64_t)row * inner, w, bias, inner, classes, xs, z);
  }
  for (int c = threadIdx.x; c < classes; c += kThreads) {
    float v = 0.f;
    if (live) {
      v = fa * exp2f((z[c] - total) * kLog2e);
      if (c == label) v -= fb;
    }
    z[c] = v;
    AGN_ST(p + (int64_t)row * classes + c, v);
  }
  __syncthreads();
  if (!dx) return;
  T* out = dx + (int64_t)row * inner;
  if (classes <= 64 || inner >= kThreads) {   // a column a thread
    for (int k = threadIdx.x; k < inner; k += kThreads) {
      float s = 0.f;
      if (live) {
#pragma unroll 8
        for (int c = 0; c < classes; ++c) s = fmaf(z[c], to_float(AGN_LD(w + c * inner + k)), s);
      }
      from_float(out + k, s);
    }
  } else {   // 32 columns at a time, whose classes the warps share
    for (int k0 = 0; k0 < inner; k0 += 32) {
      const int k = min(k0 + lane, inner - 1);
      float s = 0.f;
      if (live) {
#pragma unroll 8
        for (int c = warp; c < classes; c += kThreads / 32) s = fmaf(z[c], to_float(AGN_LD(w + c * inner + k)), s);
      }
      part[warp][lane] = s;
      __syncthreads();
      if (warp == 0 && k0 + lane < inner) {
        for (int j = 1; j < kThreads / 32; ++j) s += part[j][lane];
        from_float(out + k, s);
      }
      __syncthreads();
    }
  }
}

// dw and dbias: 32 columns of a class a block, its warps share the rows.  (Column `inner`: the bias.)
template <typename T>
__global__ void __launch_bounds__(1024)
small_columns_kernel(const float* p, const T* x, const int* labels, int rows, int inner, int classes, T* dw,
                     float* dbias) {
  pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int c = blockIdx.x, k = blockIdx.y * 32 + lane;
  __shared__ float part[32][33];
  float s = 0.f;
  const int at = min(k, inner - 1);
#pragma unroll 4
  for (int r = warp; r < rows; r += warps) {
    const bool known = has_label(AGN_LD(labels + r), classes);
    const float v = AGN_LD(p + (int64_t)r * classes + c), xv = to_float(AGN_LD(x + (int64_t)r * inner + at));
    s = fmaf(v, !known ? 0.f : k < inner ? xv : 1.f, s);
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || k > inner) return;
  for (int j = 1; j < warps; ++j) s += part[j][lane];
  if (k < inner) {
    if (dw) from_float(dw + (int64_t)c * inner + k, s);
  } else if (dbias) {
    AGN_ST(dbias + c, s);
  }
}

// ------------------------------------------------------------------ calls

struct Call {
  const void *x, *w;
  const float* bias;
  const int* labels;
  Sizes s;
  float *loss, *lse_out;                       // forward
  const float *lse, *dloss, *dlse;             // backward
  float scale;
  void *dx, *dw;
  float* dbias;
  uint8_t* work;
  int64_t work_bytes;
  int* err;
  uint64_t wait_ns;
  int withhold;
};

template <typename... A>
Status run(void (*kern)(A...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args) {
  AGN_TRY_CUDA(launch_pdl(kern, grid, dim3((unsigned)threads), smem, st, args...));
  return Status::Ok();
}

unsigned grid_for(int64_t items, int per) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(ceil_div(items, per), 8 * kSms)); }

template <typename T>
Status small_forward(const Call& c, cudaStream_t st) {
  return run(small_loss_kernel<T>, dim3((unsigned)c.s.rows), kThreads, (size_t)c.s.classes * 4, st,
             static_cast<const T*>(c.x), static_cast<const T*>(c.w), c.bias, c.labels, (int)c.s.inner,
             (int)c.s.classes, c.loss, c.lse_out);
}

template <typename T>
Status small_backward(const Call& c, const Layout& l, cudaStream_t st) {
  float* p = reinterpret_cast<float*>(c.work + l.p);
  const int rows = (int)c.s.rows, inner = (int)c.s.inner, classes = (int)c.s.classes;
  AGN_TRY(run(small_rows_kernel<T>, dim3((unsigned)rows), kThreads, (size_t)classes * 4, st,
              static_cast<const T*>(c.x), static_cast<const T*>(c.w), c.bias, c.labels, c.lse, c.dloss, c.dlse,
              c.scale, inner, classes, p, static_cast<T*>(c.dx)));
  if (!c.dw && !c.dbias) return Status::Ok();
  return run(small_columns_kernel<T>, dim3((unsigned)classes, (unsigned)ceil_div(inner + 1, 32)),
             rows > 128 ? 1024 : 256, 0, st,
             (const float*)p, static_cast<const T*>(c.x), c.labels, rows, inner, classes, static_cast<T*>(c.dw),
             c.dbias);
}

template <typename T>
Pack<T> w_pack(const Call& c, const Layout& l, int64_t c0, int64_t n) {
  return Pack<T>{static_cast<const T*>(c.w) + c0 * c.s.inner, n, (int)c.s.inner,
                 reinterpret_cast<bf16*>(c.work + l.w), l.kp, l.piece * l.kp};
}

// Rows c0 .. c0 + n - 1 of w as bf16 rows or pieces, where they are not read as they are.
template <typename T>
Status prepare_w(const Call& c, const Layout& l, int64_t c0, int64_t n, cudaStream_t st) {
  if (l.direct || l.raw) return Status::Ok();
  return run(pack_kernel<T>, dim3(grid_for(n * (l.kp / 8), kThreads)), kThreads, 0, st, w_pack<T>(c, l, c0, n));
}

// Rows of x that have a label: counted, and packed (or gathered where some are missing); the first piece
// of w.
template <typename T>
Status prepare(const Call& c, const Layout& l, cudaStream_t st) {
  int* idx = reinterpret_cast<int*>(c.work + l.idx);
  int* live = reinterpret_cast<int*>(c.work + l.live);
  const Pack<T> x{static_cast<const T*>(c.x), c.s.rows, (int)c.s.inner, reinterpret_cast<bf16*>(c.work + l.x), l.kp,
                  l.rows_pad * l.kp};
  const int64_t n = std::min(l.piece, c.s.classes);
  if (c.s.rows <= kMostRows) {
    const bool as_is = l.direct || l.raw;
    const Pack<T> w = as_is ? Pack<T>{} : w_pack<T>(c, l, 0, n);
    const int64_t items = (as_is ? 0 : n * l.kp / 8192) + ceil_div(c.s.rows, 4);
    const int64_t grid = std::max(std::min<int64_t>(kSms, items), ceil_div(c.s.rows, kRangeRows));
    return run(prepare_kernel<T>, dim3((unsigned)grid), 1024, 0, st, x, w, l.direct, (int)ceil_div(c.s.rows, grid),
               c.labels, (int)c.s.classes, idx, live, static_cast<T*>(c.dx));
  }
  AGN_TRY(run(rows_kernel, dim3(1), 1024, 0, st, c.labels, (int)c.s.rows, (int)c.s.classes, idx, live));
  AGN_TRY(run(gather_kernel<T>, dim3(grid_for(l.rows_pad * (l.kp / 8), kThreads)), kThreads, 0, st, x, l.direct,
              (const int*)idx, (const int*)live, c.labels, (int)c.s.classes, static_cast<T*>(c.dx)));
  return prepare_w<T>(c, l, 0, n, st);
}

// x as an operand: as it is and gathered, or packed alone.
Status x_maps(const Call& c, const Layout& l, uint32_t box_inner, uint32_t box_rows, CUtensorMap* own, CUtensorMap* alt) {
  const void* packed = c.work + l.x;
  AGN_TRY(make_tmap_bf16_3d(alt, packed, l.kp, l.rows_pad, l.planes, l.kp, l.rows_pad * l.kp, box_inner, box_rows));
  if (!l.direct) {
    *own = *alt;
    return Status::Ok();
  }
  return make_tmap_bf16_3d(own, c.x, c.s.inner, c.s.rows, 1, c.s.inner, c.s.rows * c.s.inner, box_inner, box_rows);
}

// Rows c0 .. c0 + n - 1 of w as an operand.
Status w_map(const Call& c, const Layout& l, int64_t c0, int64_t n, uint32_t box_inner, uint32_t box_rows,
             CUtensorMap* m) {
  if (l.direct)
    return make_tmap_bf16_3d(m, static_cast<const bf16*>(c.w) + c0 * c.s.inner, c.s.inner, n, 1, c.s.inner,
                             n * c.s.inner, box_inner, box_rows);
  return make_tmap_bf16_3d(m, c.work + l.w, l.kp, n, l.planes, l.kp, l.piece * l.kp, box_inner, box_rows);
}

GemmArgs common_args(const Call& c, const Layout& l) {
  GemmArgs a{};
  a.live = reinterpret_cast<const int*>(c.work + l.live);
  a.idx = reinterpret_cast<const int*>(c.work + l.idx);
  a.rows = (int)c.s.rows;
  a.planes = l.planes;
  a.a_box = 128;
  a.splits = 1;
  a.err = c.err;
  a.wait_ns = (uint32_t)c.wait_ns;
  a.withhold = c.withhold;
  return a;
}

// The product of the logits of classes c0 .. c0 + n - 1.
GemmArgs logit_args(const Call& c, const Layout& l, int64_t c0, int64_t n) {
  GemmArgs a = common_args(c, l);
  a.M = (int)c.s.rows; a.N = (int)n; a.K = (int)c.s.inner;
  a.alt = l.direct ? 1 : 0;
  a.bn = l.z.bn;
  a.a_box = l.a_box;
  a.bias = c.bias;
  a.labels = c.labels;
  a.class0 = (int)c0; a.classes = (int)c.s.classes;
  return a;
}

int64_t logit_units(const Call& c, const Layout& l, int64_t n) {
  return ceil_div(c.s.rows, 128 * l.z.ctas) * ceil_div(n, l.z.bn);
}

Status join_rows(const Call& c, const float2* ms, int64_t halves, const float* zlab, const int* idx, const int* live,
                 cudaStream_t st) {
  const int rows_a_block = c.s.rows >= 4 * kSms || halves <= 64 ? 8 : 1;
  return run(join_kernel, dim3((unsigned)ceil_div(c.s.rows, rows_a_block)), kThreads, 0, st, ms, (int)halves, halves,
             rows_a_block, zlab, c.labels, (int)c.s.classes, (int)c.s.rows, idx, live, c.loss, c.lse_out);
}

Status run_few(const Call& c, const Layout& l, bool backward_call, cudaStream_t st) {
  FewArgs a{};
  a.x = c.x; a.w = c.w; a.bias = c.bias; a.labels = c.labels;
  a.rows = (int)c.s.rows; a.inner = (int)c.s.inner; a.classes = (int)c.s.classes;
  a.ms = reinterpret_cast<float2*>(c.work + l.ms);
  a.zlab = reinterpret_cast<float*>(c.work + l.zlab);
  a.lse = c.lse; a.dloss = c.dloss; a.dlse = c.dlse;
  a.scale = c.scale;
  a.p = reinterpret_cast<float*>(c.work + l.p);
  a.dx = c.dx; a.dw = c.dw; a.dbias = c.dbias;
  a.dx_parts = c.dx ? reinterpret_cast<float*>(c.work + l.dxs) : nullptr;
  a.ld_parts = l.kp;
  AGN_TRY(few(a, c.s.prec, backward_call, st));
  if (backward_call) return Status::Ok();
  return join_rows(c, a.ms, l.halves, a.zlab, nullptr, nullptr, st);
}

// out [splits][rows_pad][ld] = x w^T (mn: p w), w read as it is.
Status raw_product(const Call& c, const Layout& l, bool mn, float* out, int64_t ld, int splits, cudaStream_t st) {
  RawLaunch r{};
  if (mn) AGN_TRY(make_tmap_bf16_3d(&r.b, c.work + l.p, l.ldp, l.rows_pad, 3, l.ldp, l.rows_pad * l.ldp, 64, 64));
  else AGN_TRY(make_tmap_bf16_3d(&r.b, c.work + l.x, l.kp, l.rows_pad, 3, l.kp, l.rows_pad * l.kp, 64, 64));
  AGN_TRY(make_tmap_store_2d(&r.c, out, 4, ld, splits * l.rows_pad, ld, 32, 32));
  RawArgs& a = r.args;
  a.w = static_cast<const float*>(c.w);
  a.ld = c.s.inner;
  a.M = (int)(mn ? c.s.inner : c.s.classes);
  a.K = (int)(mn ? c.s.classes : c.s.inner);
  a.mn = mn;
  a.vec = c.s.inner % 4 == 0;
  a.groups = (int)(l.rows_pad / 64);
  a.splits = splits;
  a.part_rows = (int)l.rows_pad;
  a.err = c.err;
  a.wait_ns = (uint32_t)c.wait_ns;
  a.withhold = c.withhold;
  return raw(r, st);
}

// The logits into scratch: their product by ranges of K, or with w as it is.
Status logit_ranges(const Call& c, const Layout& l, GemmLaunch& g, bool as_is, cudaStream_t st, Logits* out) {
  float* zs = reinterpret_cast<float*>(c.work + l.zs);
  *out = Logits{zs, l.z_splits, l.rows_pad * l.ldz, l.ldz, c.bias, c.labels, (int)c.s.classes, (int)c.s.rows,
                as_is ? nullptr : reinterpret_cast<const int*>(c.work + l.idx),
                as_is ? nullptr : reinterpret_cast<const int*>(c.work + l.live)};
  if (l.raw) return raw_product(c, l, false, zs, l.ldz, l.z_splits, st);
  AGN_TRY(w_map(c, l, 0, c.s.classes, 64, l.z.bn / l.z.ctas, &g.maps[0].b));
  AGN_TRY(make_tmap_store_2d(&g.maps[0].c, zs, 4, l.ldz, l.z_splits * l.rows_pad, l.ldz, 32, 32));
  GemmArgs& a = g.args[0];
  a = logit_args(c, l, 0, c.s.classes);
  a.splits = l.z_splits;
  a.part = 1;
  a.part_rows = (int)l.rows_pad;
  if (as_is) a.live = nullptr;
  return gemm(l.z.ctas, kOut, g, logit_units(c, l, c.s.classes) * l.z_splits, st);
}

template <typename T>
Status forward(const Call& c, const Layout& l, cudaStream_t st) {
  // One tile of rows is read as it is: rows without a label cost nothing more and are their own alone (3 us).
  const bool as_is = l.direct && c.s.rows <= 128;
  if (!as_is) AGN_TRY(prepare<T>(c, l, st));
  float2* ms = reinterpret_cast<float2*>(c.work + l.ms);
  float* zlab = reinterpret_cast<float*>(c.work + l.zlab);
  GemmLaunch g{};
  g.n = 1;
  GemmMaps& maps = g.maps[0];
  AGN_TRY(x_maps(c, l, 64, l.a_box, &maps.a, &maps.alt));
  if (l.z_splits > 1 || l.raw) {
    Logits z;
    AGN_TRY(logit_ranges(c, l, g, as_is, st, &z));
    return run(logits_loss_kernel, dim3((unsigned)c.s.rows), c.s.rows <= kSms && c.s.classes > 4096 ? 1024 : kThreads, 0, st, z, c.loss, c.lse_out);
  }
  int64_t half = 0;
  for (int64_t c0 = 0; c0 < c.s.classes; c0 += l.piece) {
    const int64_t n = std::min(l.piece, c.s.classes - c0);
    if (c0 > 0) AGN_TRY(prepare_w<T>(c, l, c0, n, st));
    AGN_TRY(w_map(c, l, c0, n, 64, l.z.bn / l.z.ctas, &maps.b));
    g.args[0] = logit_args(c, l, c0, n);
    g.args[0].ms = ms;
    g.args[0].ld_ms = l.halves;
    g.args[0].ms0 = (int)half;
    g.args[0].zlab = zlab;
    if (as_is) {
      g.args[0].live = nullptr;
      g.args[0].idx = nullptr;
    }
    AGN_TRY(gemm(l.z.ctas, kLse, g, logit_units(c, l, n), st));
    half += 2 * ceil_div(n, l.z.bn);
  }
  return join_rows(c, ms, half, zlab, as_is ? nullptr : reinterpret_cast<const int*>(c.work + l.idx),
                   reinterpret_cast<const int*>(c.work + l.live), st);
}

template <typename T>
Ranges<T> ranges(const void* part, int splits, int64_t plane, int64_t ld, int64_t rows, int64_t cols, const int* idx, T* out, int threads) {
  const bool vec = cols % 4 == 0 && reinterpret_cast<uintptr_t>(out) % (4 * sizeof(T)) == 0;
  return {static_cast<const float*>(part), splits, plane, ld, rows, (int)cols, idx, out, vec,
          (int)grid_for(rows * ceil_div(cols, 4), threads)};
}

template <typename T>
Status backward(const Call& c, const Layout& l, cudaStream_t st) {
  constexpr int es = (int)sizeof(T);
  const int64_t rows = c.s.rows, inner = c.s.inner;
  const int* idx = reinterpret_cast<const int*>(c.work + l.idx);
  const int* live = reinterpret_cast<const int*>(c.work + l.live);
  AGN_TRY(prepare<T>(c, l, st));
  bf16* p = reinterpret_cast<bf16*>(c.work + l.p);
  float* db = reinterpret_cast<float*>(c.work + l.db);
  const int64_t p_plane = l.rows_pad * l.ldp, ldn = round_up(inner, 64), dw_rows = round_up(l.piece, 256);
  GemmLaunch z{}, dw{}, dx{};
  z.n = dw.n = dx.n = 1;
  AGN_TRY(x_maps(c, l, 64, l.a_box, &z.maps[0].a, &z.maps[0].alt));
  AGN_TRY(make_tmap_store_2d(&z.maps[0].c, p, 2, l.ldp, l.pieces_p * l.rows_pad, l.ldp, 32, 32));
  AGN_TRY(make_tmap_bf16_3d(&dw.maps[0].a, p, l.ldp, l.rows_pad, l.pieces_p, l.ldp, p_plane, 64, 64));
  const Cut &cw = l.grads[0], &cx = l.both ? l.grads[0] : l.grads[1];
  if (!l.x_t) {
    AGN_TRY(x_maps(c, l, 64, 64, &dw.maps[0].b, &dw.maps[0].alt));
  } else if (c.dw) {
    bf16* xt = reinterpret_cast<bf16*>(c.work + l.xt);
    const int64_t plane = round_up(inner, 64) * l.rows_pad;
    AGN_TRY(run(transpose_kernel<T>, dim3(grid_for(l.rows_pad / 64 * ceil_div(inner, 64), 1)), kThreads, 0, st,
                static_cast<const T*>(c.x), (int)inner, idx, live, xt, l.rows_pad, plane));
    AGN_TRY(make_tmap_bf16_3d(&dw.maps[0].b, xt, l.rows_pad, inner, l.planes, l.rows_pad, plane, 64, cw.bn / cw.ctas));
  }
  AGN_TRY(make_tmap_bf16_3d(&dx.maps[0].b, p, l.ldp, l.rows_pad, l.pieces_p, l.ldp, p_plane, 64, cx.bn / cx.ctas));
  const bool rows16 = inner * es % 16 == 0;
  for (int64_t c0 = 0; c0 < c.s.classes; c0 += l.piece) {
    const int64_t n = std::min(l.piece, c.s.classes - c0);
    if (c0 > 0) AGN_TRY(prepare_w<T>(c, l, c0, n, st));
    if (l.z_splits > 1 || l.raw) {
      Logits a;
      AGN_TRY(logit_ranges(c, l, z, false, st, &a));
      AGN_TRY(run(logits_grad_kernel<sizeof(T) == 4 ? 3 : 2>, dim3((unsigned)(l.ldp / 64), (unsigned)(l.rows_pad / 32)),
                  kThreads, 0, st, a, c.lse, c.dloss, c.dlse, c.scale, p, l.ldp, p_plane, c.dbias ? db : nullptr));
    } else {
      AGN_TRY(w_map(c, l, c0, n, 64, l.z.bn / l.z.ctas, &z.maps[0].b));
      GemmArgs& a = z.args[0];
      a = logit_args(c, l, c0, n);
      a.lse = c.lse; a.dloss = c.dloss; a.dlse = c.dlse; a.scale = c.scale;
      a.p_plane = (int)l.rows_pad;
      a.db = c.dbias ? db : nullptr;
      a.ld_db = l.ldp;
      AGN_TRY(gemm(l.z.ctas, kGrad, z, logit_units(c, l, n), st));
    }
    T* dw_out = static_cast<T*>(c.dw) + c0 * inner;
    int64_t dw_units = 0, dx_units = 0;
    if (c.dw) {   // [n][inner] = p^T x
      GemmArgs& d = dw.args[0];
      d = common_args(c, l);
      d.M = (int)n; d.N = (int)inner; d.K = (int)rows;
      d.live_is = 1;
      d.twice = l.planes == 1 ? 1 : 0;
      d.alt = l.direct && !l.x_t ? 2 : 0;
      d.bn = cw.bn;
      d.a_mn = 1;
      d.b_mn = !l.x_t;
      d.splits = l.dw_splits;
      d.out = dw_out; d.ldo = inner; d.dtype = c.s.prec;
      if (l.dw_splits > 1) {
        d.part = 1;
        d.part_rows = (int)dw_rows;
        AGN_TRY(make_tmap_store_2d(&dw.maps[0].c, c.work + l.dws, 4, ldn, l.dw_splits * dw_rows, ldn, 32, 32));
      } else if (rows16) {
        d.tma_out = 1;
        AGN_TRY(make_tmap_store_2d(&dw.maps[0].c, dw_out, es, inner, n, inner, 32, 32));
      }
      dw_units = ceil_div(n, 128 * cw.ctas) * ceil_div(inner, cw.bn) * d.splits;
    }
    if (c.dx && !l.raw) {   // [rows][inner] += p w, as w^T p^T
      GemmArgs& d = dx.args[0];
      d = common_args(c, l);
      d.M = (int)inner; d.N = (int)rows; d.K = (int)n;
      d.live_is = 2;
      d.twice = l.planes == 1 ? 2 : 0;
      d.transposed = 1;
      d.bn = cx.bn;
      d.a_mn = 1;
      d.splits = l.dx_splits;
      d.out = c.dx; d.ldo = inner; d.dtype = c.s.prec;
      d.scatter = 1;
      AGN_TRY(w_map(c, l, c0, n, 64, 64, &dx.maps[0].a));
      if (l.dx_part) {
        d.part = c0 == 0 ? 1 : 2;
        d.part_rows = (int)l.rows_pad;
        AGN_TRY(make_tmap_store_2d(&dx.maps[0].c, c.work + l.dxs, 4, ldn, l.dx_splits * l.rows_pad, ldn, 32, 32));
      } else if (rows16) {
        d.tma_out = 1;
        AGN_TRY(make_tmap_store_2d(&dx.maps[0].c, c.dx, es, inner, rows, inner, 32, 32));
      }
      dx_units = ceil_div(inner, 128 * cx.ctas) * ceil_div(rows, cx.bn) * d.splits;
    }
    if (c.dw && c.dx && l.both) {
      dw.n = 2;
      dw.maps[1] = dx.maps[0];
      dw.args[1] = dx.args[0];
      AGN_TRY(gemm(cw.ctas, kOut, dw, dw_units + dx_units, st));
    } else {
      if (c.dw) AGN_TRY(gemm(cw.ctas, kOut, dw, dw_units, st));
      if (c.dx && l.raw)
        AGN_TRY(raw_product(c, l, true, reinterpret_cast<float*>(c.work + l.dxs), ldn, l.dx_splits, st));
      else if (c.dx) AGN_TRY(gemm(cx.ctas, kOut, dx, dx_units, st));
    }
    const int threads = sum_threads(rows, c.dbias);
    Columns columns{};
    Ranges<T> rw{}, rx{};
    if (c.dbias) columns = {db, l.ldp, (int)n, c.dbias + c0, (int)ceil_div(n, 32)};
    if (c.dw && l.dw_splits > 1)
      rw = ranges<T>(c.work + l.dws, l.dw_splits, dw_rows * ldn, ldn, n, inner, nullptr, dw_out,
                     threads);
    if (c.dx && l.dx_part && c0 + n == c.s.classes)
      rx = ranges<T>(c.work + l.dxs, l.dx_splits, l.rows_pad * ldn, ldn, rows, inner, idx, static_cast<T*>(c.dx),
                     threads);
    const int blocks = columns.blocks + rw.blocks + rx.blocks;
    if (blocks > 0) AGN_TRY(run(sums_kernel<T>, dim3((unsigned)blocks), threads, 0, st, columns, rw, rx, live));
  }
  return Status::Ok();
}

Status check_sizes(const Sizes& s) {
  if (!dtype_size(s.prec)) return Status::Err(AGN_E_INVALID, "unknown dtype");
  if (s.rows < 0 || s.rows > 1 << 28 || s.inner < 1 || s.inner > 1 << 20 || s.classes < 1 || s.classes > 1 << 28)
    return Status::Err(AGN_E_INVALID, "need 0 <= rows <= 2^28, 1 <= inner <= 2^20, 1 <= classes <= 2^28");
  return Status::Ok();
}

Status call(Call& c, bool backward_call, cudaStream_t st) {
  AGN_TRY(check_sizes(c.s));
  const size_t es = dtype_size(c.s.prec);
  const int64_t rows = c.s.rows, inner = c.s.inner, classes = c.s.classes;
  const size_t xb = (size_t)rows * inner * es, wb = (size_t)classes * inner * es, rb = (size_t)rows * 4,
               cb = (size_t)classes * 4;
  const Layout l = layout(c.s, backward_call);
  if (rows > 0) {
    if (!c.x || !c.w || !c.labels || (backward_call ? !c.lse : !c.loss || !c.lse_out))
      return Status::Err(AGN_E_INVALID, "null pointer");
    if (!c.work || c.work_bytes < (int64_t)l.bytes)
      return Status::Err(AGN_E_INVALID, "work needs " + std::to_string(l.bytes) + " bytes");
  }
  const CallBuffer x{"x", c.x, xb, 16}, w{"w", c.w, wb, 16}, bias{"bias", c.bias, c.bias ? cb : 0, 4},
      labels{"labels", c.labels, rb, 4}, lse{"lse", backward_call ? c.lse : c.lse_out, rb, 4},
      loss{"loss", c.loss, c.loss ? rb : 0, 4}, dloss{"dloss", c.dloss, c.dloss ? rb : 0, 4},
      dlse{"dlse", c.dlse, c.dlse ? rb : 0, 4}, dx{"dx", c.dx, c.dx ? xb : 0, 16}, dw{"dw", c.dw, c.dw ? wb : 0, 16},
      dbias{"dbias", c.dbias, c.dbias ? cb : 0, 4}, work{"work", rows > 0 ? c.work : nullptr, l.bytes, 256},
      err{"err", c.err, c.err ? 4u : 0u, 4};
  AGN_TRY(check_apart(work, {x, w, bias, labels, lse, loss, dloss, dlse, dx, dw, dbias, err}));
  if (backward_call) {
    AGN_TRY(check_apart(dx, {x, w, bias, labels, lse, dloss, dlse, dw, dbias, err}));
    AGN_TRY(check_apart(dw, {x, w, bias, labels, lse, dloss, dlse, dbias, err}));
    AGN_TRY(check_apart(dbias, {x, w, bias, labels, lse, dloss, dlse, err}));
    AGN_TRY(check_apart(err, {x, w, bias, labels, lse, dloss, dlse}));
  } else {
    AGN_TRY(check_apart(loss, {x, w, bias, labels, lse, err}));
    AGN_TRY(check_apart(lse, {x, w, bias, labels, err}));
    AGN_TRY(check_apart(err, {x, w, bias, labels}));
  }
  if (rows == 0) {   // no rows: the sums over them are zero
    if (!c.dw && !c.dbias) return Status::Ok();
    AGN_TRY(check_buffers({dw, dbias}));
    if (c.dw) AGN_TRY_CUDA(cudaMemsetAsync(c.dw, 0, wb, st));
    if (c.dbias) AGN_TRY_CUDA(cudaMemsetAsync(c.dbias, 0, cb, st));
    return Status::Ok();
  }
  AGN_TRY(check_buffers({x, w, bias, labels, lse, loss, dloss, dlse, dx, dw, dbias, work, err}));
  KnownBuffers known({x, w, bias, labels, lse, loss, dloss, dlse});
  KnownBuffers known2({dx, dw, dbias, work, err});
  AGN_TRY(bounds_upload(st));
  const bool fp32 = c.s.prec == AGN_PREC_FP32;
  if (!backward_call) {
    if (l.small) AGN_TRY(fp32 ? small_forward<float>(c, st) : small_forward<bf16>(c, st));
    else if (l.few) AGN_TRY(run_few(c, l, false, st));
    else AGN_TRY(fp32 ? forward<float>(c, l, st) : forward<bf16>(c, l, st));
  } else if (c.dx || c.dw || c.dbias) {
    if (l.small) AGN_TRY(fp32 ? small_backward<float>(c, l, st) : small_backward<bf16>(c, l, st));
    else if (l.few) AGN_TRY(run_few(c, l, true, st));
    else AGN_TRY(fp32 ? backward<float>(c, l, st) : backward<bf16>(c, l, st));
  }
  return bounds_collect(st);
}

// agn_debug_linear_ce_waits: of the calling thread's calls
thread_local uint64_t t_wait_ns = 0;
thread_local int t_withhold = 0;

}  // namespace
}  // namespace ce

AGN_BOUNDS_UNIT(linear_ce)

}  // namespace agn

extern "C" int agn_linear_ce_bytes(int64_t rows, int64_t inner, int64_t classes, int32_t dtype, int32_t backward,
                                   int64_t* bytes) {
  return agn::guarded([&] {
    const agn::ce::Sizes s{rows, inner, classes, dtype};
    if (!bytes) return agn::Status::Err(AGN_E_INVALID, "null pointer");
    AGN_TRY(agn::ce::check_sizes(s));
    *bytes = (int64_t)agn::ce::layout(s, backward != 0).bytes;
    return agn::Status::Ok();
  });
}

extern "C" int agn_linear_ce(const void* x, const void* w, const float* bias, const int32_t* labels, int32_t dtype,
                             int64_t rows, int64_t inner, int64_t classes, float* loss, float* lse, void* work,
                             int64_t work_bytes, int32_t* err, void* stream) {
  return agn::guarded([&] {
    agn::ce::Call c{};
    c.x = x; c.w = w; c.bias = bias; c.labels = labels;
    c.s = {rows, inner, classes, dtype};
    c.loss = loss; c.lse_out = lse;
    c.work = static_cast<uint8_t*>(work); c.work_bytes = work_bytes;
    c.err = err;
    c.wait_ns = agn::ce::t_wait_ns; c.withhold = agn::ce::t_withhold;
    return agn::ce::call(c, false, static_cast<cudaStream_t>(stream));
  });
}

extern "C" int agn_linear_ce_backward(const void* x, const void* w, const float* bias, const int32_t* labels,
                                      const float* lse, const float* dloss, const float* dlse, double scale,
                                      int32_t dtype, int64_t rows, int64_t inner, int64_t classes, void* dx, void* dw,
                                      float* dbias, void* work, int64_t work_bytes, int32_t* err, void* stream) {
  return agn::guarded([&] {
    agn::ce::Call c{};
    c.x = x; c.w = w; c.bias = bias; c.labels = labels;
    c.s = {rows, inner, classes, dtype};
    c.lse = lse; c.dloss = dloss; c.dlse = dlse;
    c.scale = (float)scale;
    c.dx = dx; c.dw = dw; c.dbias = dbias;
    c.work = static_cast<uint8_t*>(work); c.work_bytes = work_bytes;
    c.err = err;
    c.wait_ns = agn::ce::t_wait_ns; c.withhold = agn::ce::t_withhold;
    return agn::ce::call(c, true, static_cast<cudaStream_t>(stream));
  });
}

extern "C" int agn_debug_linear_ce_waits(int64_t wait_ns, int32_t withhold_rank) {
  return agn::guarded([&] {
    if (wait_ns < 0 || wait_ns > 2000000000ll || withhold_rank < -1 || withhold_rank > 1)
      return agn::Status::Err(AGN_E_INVALID, "wait_ns must be in [0, 2e9], withhold_rank -1, 0 or 1");
    agn::ce::t_wait_ns = (uint64_t)wait_ns;
    agn::ce::t_withhold = withhold_rank + 1;
    return agn::Status::Ok();
  });
}
