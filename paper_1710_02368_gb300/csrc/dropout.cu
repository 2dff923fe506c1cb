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
// Resident blocks of an SM and rows of a thread whose loads are in flight together, for one
// input matrix or two and without or with column sums (more rows spill).  16384 x 4096 bf16,
// us: two matrices 65 with (4, 2), 67 with (3, 3); with sums 82 and 74.
constexpr int blocks_per_sm(bool two, bool sums) { return two && sums ? 3 : 4; }
constexpr int unroll(bool two, bool sums) { return two ? (sums ? 3 : 2) : 4; }
constexpr int kMaxUnits = 32;   // 16-byte units of a row in a block's tile

// How the rows of the call's matrices lie to 16-byte boundaries.
enum Rows { kOther, kAligned, kAlike };

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
  int relu;
  // Rows::kAligned, kAlike (every matrix's row r starts `start` + r ldy elements past a 16-byte
  // boundary, modulo 16 bytes), kOther
  int layout, start;
  int tile_units;         // units of 16 bytes of a row in a block's tile: a thread each
  // hidden layers of a training run (kHidden): matrices [slots][rows][cols]
  const int* slot_worker;
  const long long* slot_t0;
  int step, layers, layer;
  bf16* pieces;           // also the three exact bf16 pieces, planes `plane` apart; null = no
  int64_t plane;
};

// 16 bytes of a row, as they are: from aligned memory in one load, else the
// valid elements lo .. n - 1 one by one.
template <typename T>
__device__ __forceinline__ uint4 load16(const T* p, bool full, int lo, int n) {
  if (full) return AGN_LD(reinterpret_cast<const uint4*>(p));
  uint4 q = make_uint4(0, 0, 0, 0);
  T* e = reinterpret_cast<T*>(&q);
#pragma unroll
  for (int i = 0; i < (int)(16 / sizeof(T)); ++i)
    if (i >= lo && i < n) e[i] = AGN_LD(p + i);
  return q;
}
template <typename T>
__device__ __forceinline__ float2 element2(const uint4& q, int i) {   // elements i and i + 1
  const T* e = reinterpret_cast<const T*>(&q);
  return make_float2(static_cast<float>(e[i]), static_cast<float>(e[i + 1]));
}
// Two fp32 operations of one instruction, each rounded to nearest.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "add.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "mul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
template <typename T>
__device__ __forceinline__ void store16(T* p, bool full, int lo, int n,
                                        const float (&v)[16 / sizeof(T)]) {
  uint4 q;
  T* e = reinterpret_cast<T*>(&q);
#pragma unroll
  for (int i = 0; i < (int)(16 / sizeof(T)); ++i) e[i] = static_cast<T>(v[i]);
  if (full) {
    AGN_ST(reinterpret_cast<uint4*>(p), q);
  } else {
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i)
      if (i >= lo && i < n) AGN_ST(p + i, e[i]);
  }
}

// Whether element e of a draw's four is kept.  The upper half of a word compares as
// it is (u >= T iff word >= T << 16), the lower half shifted up.
__device__ __forceinline__ bool kept(uint64_t d, int e, uint32_t t16) {
  const uint32_t w = (uint32_t)(e & 2 ? d >> 32 : d);
  return (e & 1 ? w : w << 16) >= t16;
}

// A block: tiles of tile_units units of 16 bytes along the row (blockIdx.x) by
// rows_per_block rows (blockIdx.y); a thread keeps its columns (the bias stays
// in registers) and steps down the rows.
// kTwo: two input matrices (forward: x and the residual; backward: dy and the ReLU's x).
// kSums: backward with the bias's gradient.
// kShift: rows that are not aligned, but all alike (Rows::kAlike).  A thread's 16 bytes
// are aligned ones, so its columns start up to 16 bytes before the tile's; its rows are a
// multiple of 8 apart and start at the same place, so they are the same columns all the way down.
// With column sums a tile has a unit less than its threads: the last reads the unit that
// the next tile's first reads and stores, and each sums the columns of its own tile (so the output
// is no input here).  Against elements one by one, us: 19620 x 287 bf16 8.3 for 27.5, with ReLU and
// sums 22 for 72; 16384 x 4095 bf16 73 for 160 (aligned 4096: 51, two draws for this one's three),
// with ReLU and sums 97 for 247 (73); 2865 x 3183 fp32 12.4 for 12.0, with sums 14.5 for 21.0.
template <typename T, bool kBackward, bool kTwo, bool kSums, bool kShift, bool kHidden = false>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(kTwo, kSums)) dropout_kernel(const DropArgs a) {
  constexpr int V = 16 / sizeof(T), kUnroll = kHidden ? 2 : unroll(kTwo, kSums);
  constexpr bool kReadX = !kBackward || kTwo, kReadExtra = kBackward || kTwo;
  pdl_begin();
  const int w = a.tile_units, ty = threadIdx.x / w, tx = threadIdx.x % w;
  const int nty = kThreads / w;   // (threads past w nty have no rows)
  constexpr bool kShared = kShift && kSums;   // the last unit is the next tile's too
  const int own = (kShared ? w - 1 : w) * V;  // columns of a tile
  const int64_t r0 = blockIdx.y * a.rows_per_block;
  const int64_t r1 = min(a.rows, r0 + a.rows_per_block);
  const int64_t tile0 = (int64_t)blockIdx.x * own;
  // row t of the block starts so many elements past a boundary
  auto past = [&](int t) { return (int)((a.start + (uint32_t)(r0 + t) * (uint32_t)a.ldy) & (V - 1)); };
  const int m = kShift ? past(ty) : 0;
  const int64_t c = tile0 + tx * V - m;
  // this thread's elements: lo .. n - 1
  const int lo = kShift && c < 0 ? m : 0;
  const bool last = kShared && tx == w - 1 && blockIdx.x + 1 < gridDim.x;
  const int n = ty < nty && c + lo < a.cols && !(last && m == 0) ? (int)min((int64_t)V, a.cols - c) : 0;
  const bool full = (kShift || a.layout == kAligned) && lo == 0 && n == V;
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
  first += (uint64_t)(c >> 2);
  const int skip = (int)(c & 3);   // (kShift: elements of the first draw before this thread's)
  float b[V], sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    b[e] = a.bias && e >= lo && e < n ? AGN_LD(a.bias + c + e) : 0.f;
    sum[e] = 0.f;
  }
  if (n > 0) {
    uint64_t z = key + (first + (uint64_t)(r0 + ty) * groups + 1) * gen::kG;
    const uint64_t z_step = (uint64_t)nty * groups * gen::kG;
    for (int64_t r = r0 + ty; r < r1; r += (int64_t)kUnroll * nty) {
      uint4 v[kUnroll], q[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int64_t ru = r + (int64_t)u * nty;
        if (ru >= r1) break;
        // (kShift: a unit at a row's end is read whole where it lies in the matrix; single
        // elements made the blocks at the ends the last by far: 16384 x 4095 bf16 with ReLU and sums 203 us, so 97)
        auto whole = [&](int64_t ld) {
          const int64_t at = ru * ld + c;
          return full || (kShift && at >= 0 && at + V <= (a.rows - 1) * ld + a.cols);
        };
        if (kReadX) v[u] = load16(x + ru * a.ldx + c, whole(a.ldx), lo, n);
        if (kReadExtra) q[u] = load16(extra + ru * a.lde + c, whole(a.lde), lo, n);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int64_t ru = r + (int64_t)u * nty;
        if (ru >= r1) break;
        uint64_t d[V / 4];   // draw(key, i) = mix(key + (i + 1) G), from z by addition
#pragma unroll
        for (int g = 0; g < V / 4; ++g) d[g] = gen::mix(z + (uint64_t)g * gen::kG);
        if (kShift) {   // 16 skip bits off the front, the rest from one more draw
          const uint64_t more = gen::mix(z + (uint64_t)(V / 4) * gen::kG);
          uint32_t s[V / 2 + 2];
#pragma unroll
          for (int g = 0; g <= V / 4; ++g) {
            const uint64_t f = g < V / 4 ? d[g < V / 4 ? g : 0] : more;
            s[2 * g] = (uint32_t)f;
            s[2 * g + 1] = (uint32_t)(f >> 32);
          }
#pragma unroll
          for (int i = 0; i <= V / 2; ++i) s[i] = skip & 2 ? s[i + 1] : s[i];
#pragma unroll
          for (int g = 0; g < V / 4; ++g) {
            const uint32_t l = __funnelshift_r(s[2 * g], s[2 * g + 1], 16 * (skip & 1));
            const uint32_t h = __funnelshift_r(s[2 * g + 1], s[2 * g + 2], 16 * (skip & 1));
            d[g] = (uint64_t)h << 32 | l;
          }
        }
        z += z_step;
        float o[V];
#pragma unroll
        for (int e = 0; e < V; e += 2) {   // two at a time: packed products and sums
          const float2 xv = kReadX ? element2<T>(v[u], e) : make_float2(0.f, 0.f);
          const float2 ev = kReadExtra ? element2<T>(q[u], e) : make_float2(0.f, 0.f);
          const float2 be = make_float2(b[e], b[e + 1]);
          const bool k0 = kept(d[e / 4], e & 3, a.t16), k1 = kept(d[e / 4], (e & 3) + 1, a.t16);
          float2 t;
          if (kBackward) {
            t = mul2(ev, make_float2(a.scale, a.scale));
            // (a value that is not a number passes, forward and backward)
            const float2 p = kTwo ? add2(xv, be) : make_float2(1.f, 1.f);
            t.x = k0 && !(p.x <= 0.f) ? t.x : 0.f;
            t.y = k1 && !(p.y <= 0.f) ? t.y : 0.f;
            if (kSums) {
              const float2 sv = add2(make_float2(sum[e], sum[e + 1]), t);
              sum[e] = sv.x;
              sum[e + 1] = sv.y;
            }
          } else {
            t = a.bias ? add2(xv, be) : xv;
            if (a.relu) t = make_float2(t.x <= 0.f ? 0.f : t.x, t.y <= 0.f ? 0.f : t.y);
            t = mul2(t, make_float2(a.scale, a.scale));
            t.x = k0 ? t.x : 0.f;
            t.y = k1 ? t.y : 0.f;
            if (kTwo) t = add2(t, ev);
          }
          o[e] = t.x;
          o[e + 1] = t.y;
        }
        if (!last) store16(y + ru * a.ldy + c, full, lo, n, o);
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
  if constexpr (kSums) {
    // db of the block's columns: the threads of a column in order, then the
    // cluster's blocks (all the rows of these columns) in rank order through
    // distributed shared memory: no workspace, no atomics, the same bits each time
    __shared__ float part[kThreads * V];
    __shared__ float col[V * kMaxUnits];
    const int width = V * w;
    if (ty < nty) {
#pragma unroll
      for (int e = 0; e < V; ++e) part[ty * width + tx * V + e] = sum[e];
    }
    __syncthreads();
    for (int j = threadIdx.x; j < own; j += kThreads) {
      float s = 0.f;
      for (int t = 0; t < nty; ++t) s += part[t * width + j + (kShift ? past(t) : 0)];
      col[j] = s;
    }
    cluster_sync();
    const int ranks = gridDim.y;
    for (int j = threadIdx.x; j < own; j += kThreads) {
      const int64_t cj = tile0 + j;
      if (j % ranks != (int)blockIdx.y || cj >= a.cols) continue;
      float s = 0.f;
      for (int k = 0; k < ranks; ++k) s += ld_cluster(col + j, k);
      AGN_ST(a.dbias + cj, s);
    }
    cluster_sync();   // the other blocks' reads, before this one's memory goes
  }
}

// Blocks of a cluster: the portable eight, and more where a thread has so many rows (see
// launch_kernel).
constexpr int kMaxCluster = 8, kWideCluster = 16, kWideRows = 16;

// The launch of one instantiation: tiles, rows and clusters.
template <typename T, bool kBackward, bool kTwo, bool kSums, bool kShift, bool kHidden = false>
Status launch_kernel(DropArgs a, int slots, cudaStream_t st) {
  constexpr int V = 16 / sizeof(T);
  auto kern = dropout_kernel<T, kBackward, kTwo, kSums, kShift, kHidden>;
  int dev = 0, sms = 0;
  AGN_TRY(current_device(&dev));
  AGN_TRY(device_sms(dev, &sms));
  const int64_t units = ceil_div(a.cols, V) + (kShift && !kSums ? 1 : 0);   // (a part at each end)
  const int64_t fit =   // resident blocks
      std::max<int64_t>(1, (int64_t)sms * blocks_per_sm(kTwo, kSums) / slots);
  int64_t tiles = 0, blocks = 0;
  if (!kSums) {
    // wide tiles, and as many blocks down the rows as are resident
    int best = 1;
    for (int w = 2; w <= kMaxUnits; w *= 2)
      if (round_up(units, w) * 16 <= round_up(units, best) * 17) best = w;
    a.tile_units = best;
    tiles = ceil_div(units, best);
    blocks = std::min<int64_t>(std::max<int64_t>(1, fit / tiles), ceil_div(a.rows, kThreads / best));
    a.rows_per_block = ceil_div(a.rows, blocks);
    blocks = ceil_div(a.rows, a.rows_per_block);
  } else {
    // A cluster has all the rows of its tile.  The kernel is as much bound by instructions
    // as by memory, so what counts is how many of the resident blocks have work, over the
    // rounds: the width (whole 32-byte sectors but for a row of one unit; shifted rows: powers of
    // two) and the cluster with the most, the widest of about equals (16384 x 4096 bf16 with ReLU,
    // three blocks an SM: 86 tiles of 6 units, clusters of 5, 430 of 456 blocks, 73 us; 64 of 8, clusters
    // of 6, 384 blocks 79, clusters of 7, 448 blocks but two rounds (59 clusters are resident) 103;
    // 128 of 4, clusters of 3 77; 7197 x 6736 fp32: 842 tiles of 2 units in two rounds 86, 106 of
    // 16 and clusters of 5 66).  Where that leaves a quarter idle,
    // clusters of up to 16, if threads have kWideRows rows or more of eight blocks (us, 8 and 16:
    // 65536 x 64 bf16 28 and 16, 16384 x 32 fp32 7.5 and 5.3; 2048 x 1000 fp32, 8 rows, 6.1 and
    // 6.5; 16384 x 4096 bf16 without ReLU, 512 blocks with 8, 52.5 and 54.1).
    double most = 0.0;
    const int narrowest = kShift || units > 1 ? 2 : 1;
    for (int widest : {kMaxCluster, kWideCluster}) {
      if (4 * most > 3 * (double)fit) break;
      for (int w = 16; w >= narrowest; w = kShift || w == 2 ? w / 2 : w - 2) {
        const int64_t t = ceil_div(units, kShift ? w - 1 : w), nty = kThreads / w;
        if (widest == kWideCluster && a.rows < kMaxCluster * kWideRows * nty) continue;
        int64_t c = std::min<int64_t>(widest, std::max<int64_t>(1, ceil_div(a.rows, nty)));
        struct Tag {};
        for (; c > 1; --c) {
          int resident = 0;
          AGN_TRY(max_clusters<Tag>(kern, kThreads, 0, (int)c, dev, &resident));
          if (resident >= t) break;
        }
        const double used = (double)(t * c) / ceil_div(t * c, fit) * units / (double)(t * w);
        if (used > most * 1.02) {
          most = used;
          a.tile_units = w;
          tiles = t;
          blocks = c;
        }
      }
    }
    a.rows_per_block = std::max<int64_t>(1, ceil_div(a.rows, blocks));
  }
  const dim3 grid((unsigned)tiles, (unsigned)blocks, (unsigned)slots);
  if (kSums)
    AGN_TRY_CUDA(launch_pdl_cluster(kern, grid, kThreads, 0, dim3(1, grid.y, 1), st, a));
  else
    AGN_TRY_CUDA(launch_pdl(kern, grid, kThreads, 0, st, a));
  return Status::Ok();
}

template <typename T, bool kBackward, bool kTwo, bool kSums>
Status launch_rows(const DropArgs& a, cudaStream_t st) {
  return a.layout == kAlike ? launch_kernel<T, kBackward, kTwo, kSums, true>(a, 1, st)
                            : launch_kernel<T, kBackward, kTwo, kSums, false>(a, 1, st);
}

template <typename T>
Status launch_dropout(const DropArgs& a, bool backward, cudaStream_t st) {
  if (!backward)
    return a.extra ? launch_rows<T, false, true, false>(a, st) : launch_rows<T, false, false, false>(a, st);
  if (a.dbias)
    return a.x ? launch_rows<T, true, true, true>(a, st) : launch_rows<T, true, false, true>(a, st);
  return a.x ? launch_rows<T, true, true, false>(a, st) : launch_rows<T, true, false, false>(a, st);
}

Status run_dropout(const DropArgs& a, bool backward, int dtype, cudaStream_t st) {
  return dtype == AGN_PREC_FP32 ? launch_dropout<float>(a, backward, st)
                                : launch_dropout<bf16>(a, backward, st);
}

Status set_probability(double p, DropArgs* a) {
  uint32_t t;
  if (!dropout_threshold(p, &t, &a->scale))
    return Status::Err(AGN_E_INVALID, "the dropout probability must be in [0, 1)");
  a->t16 = t << 16;
  return Status::Ok();
}

// The layout of up to three matrices (null: none); the last is the output.
void set_layout(DropArgs* a, const void* p0, int64_t ld0, const void* p1, int64_t ld1, const void* y,
                int64_t ldy, size_t es) {
  auto at = [&](const void* p) { return (int)(reinterpret_cast<uintptr_t>(p) % 16 / es); };
  auto step = [&](int64_t ld) { return (int)((uint64_t)ld * es % 16 / es); };
  const bool alike = (!p0 || (at(p0) == at(y) && step(ld0) == step(ldy))) &&
                     (!p1 || (at(p1) == at(y) && step(ld1) == step(ldy)));
  a->start = at(y);
  a->layout = !alike ? kOther : at(y) == 0 && step(ldy) == 0 ? kAligned : kAlike;
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
  set_layout(&a, x, ldx, residual, ldr, y, ldy, es);
  KnownBuffers known({bx, bb, br, by});
  AGN_TRY(bounds_upload(st));
  AGN_TRY(run_dropout(a, false, dtype, st));
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
  set_layout(&a, x, ldx, dy, lddy, dx, lddx, es);
  if (a.layout == kAlike && dbias && (dx == dy || dx == x)) a.layout = kOther;   // (kShift)
  KnownBuffers known({bg, bx, bb, bo, bs});
  AGN_TRY(bounds_upload(st));
  AGN_TRY(run_dropout(a, true, dtype, st));
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
  set_layout(&a, nullptr, 0, nullptr, 0, h.H, h.d, sizeof(T));
  if (a.layout == kAlike) a.layout = kOther;   // (small: one by one)
  a.slot_worker = h.slot_worker; a.slot_t0 = h.slot_t0;
  a.step = h.step; a.layers = h.layers; a.layer = h.layer;
  a.pieces = h.pieces; a.plane = h.plane;
  return launch_kernel<T, false, false, false, false, true>(a, slots, st);
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
