// The three products of the output layer's loss on the tensor cores (tcgen05 kind::f16, f32
// sums in TMEM), with what follows each in its epilogue:
//   logits z = x w^T (K along both operands' rows): kLse leaves (max, sum of exponentials) of
//     each row and half a tile, kGrad writes p = a softmax - b [label] in bf16 pieces and sums its columns;
//   dw = p^T x and dx = p w (kOut): the MMA takes operands stored along M or N (MN-major) too, but
//     B's so stored cost it: 256 x 256 tiles of 8192 x 8192 x 4096 1.25 times the clocks, A's none (B's reads
//     of shared memory, it seems, twice as many).  So dx is made as w^T p^T, p in B's place as it lies,
//     and leaves transposed, and x is laid out along its rows for dw where that pays.
// fp32 operands are three exact bf16 pieces (planes): six products of pieces, the first in one
// accumulator and the five smaller ones in another.  The tensor cores cut what they add to an
// accumulator off below its last bit, always towards zero, so sums are taken over a part of K at
// a time (sum_steps) and added in registers, rounded (fp32, one accumulator over K = 50000: 1.5e-5 of dx off).
// Many fp32 tiles are 256 x 256 as bf16's are, both accumulators then fill TMEM: their sums (512 k) are
// read between the MMAs, the larger one's first, so that its next products run while the other is read.
// One CTA a tile of 128 rows, or a pair (cta_group::2) a tile of 256, each CTA loading its 128 rows
// of A and half of B's: 64 bytes a clock of MMA time instead of 96 with 256 columns.  Persistent:
// a CTA (pair) walks over tiles in bands of eight along M, so that what runs at a time shares operands
// in the L2.  Roles by warp: 0 loads (TMA, 128-byte swizzle), 1 issues the MMAs, 4-11 finish, two
// accumulators in turn, so that a tile's epilogue runs beside the next one's MMAs.
// Every wait is bounded (2 s); whoever gives up says so to all roles, what could not be computed
// is NaN, *err is 1, and stages in flight are waited for before the CTA ends.
#include "linear_ce.cuh"
#include "ops.cuh"
#include "tc_ptx.cuh"

namespace agn {
namespace ce {

namespace {

constexpr int kThreads = 384;
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr int kBK = 64;                   // k of a stage: 128-byte rows
constexpr int kBox = 64 * 128;            // an operand stored along M or N: boxes of 64 x 64 k
constexpr int kRing = 176 * 1024;
constexpr int kMaxStages = 16;
// Stages of a sum in TMEM, where there are more of them the rest is added in registers: fp32 256 k, wide tiles 512; bf16's
// logits by one CTA 512, by pairs 1024 (by 512 the tensor cores wait for it: 8192 x 4096 to 32768 1252 us, by 1024 1168,
// one sum 1121); bf16's gradients 8192 k of p's pieces (2e-5 of them, their rounding 2e-3).
constexpr int sum_steps(int ctas, int epilogue, int planes, bool wide) {
  return planes == 3 ? (wide ? 8 : 4) : epilogue == kOut ? 128 : ctas == 2 ? 16 : 8;
}
constexpr int kStaged = 4096;             // a finishing warp's tile of outputs
constexpr size_t kSmem = 1024 + kRing + 8 * (kStaged + 512) + 512;
constexpr float kLog2e = 1.44269504088896340736f;

struct Geometry {
  int M, N, K, tiles_n, tiles, units, kt_per, KT;
  bool gathered;
};

template <int kCtas>
__device__ __forceinline__ Geometry geometry(const GemmArgs& a) {
  Geometry g;
  g.M = a.M; g.N = a.N; g.K = a.K;
  g.gathered = false;
  if (a.live) {
    const int live = min(AGN_LD(a.live), a.rows);
    g.gathered = live < a.rows;
    if (a.live_is == 0) g.M = live;
    else if (a.live_is == 1) g.K = live;
    else g.N = live;
  }
  g.tiles_n = (g.N + a.bn - 1) / a.bn;
  g.tiles = (g.M + 128 * kCtas - 1) / (128 * kCtas) * g.tiles_n;
  g.units = g.tiles * a.splits;
  g.KT = (g.K + kBK - 1) / kBK * (a.twice ? 2 : 1);
  g.kt_per = (g.KT + a.splits - 1) / a.splits;
  return g;
}

// Tile (in units of a tile) and range along K of unit u: bands of eight tiles along M.
struct Unit {
  int m, n, split, kt0, kt;
  __device__ __forceinline__ Unit(const Geometry& g, int splits, int u) {
    split = u % splits;
    const int t = u / splits, tiles_m = g.tiles / g.tiles_n;
    const int band = t / (8 * g.tiles_n), m0 = band * 8, gm = min(8, tiles_m - m0);
    const int r = t - m0 * g.tiles_n;
    m = m0 + r % gm;
    n = r / gm;
    kt0 = min(g.KT, split * g.kt_per);
    kt = min(g.KT, kt0 + g.kt_per) - kt0;
  }
};

// 16-byte piece c of row `row` of a staged tile of rows of kRow bytes, swizzled as its tensor map says.
template <int kRow>
__device__ __forceinline__ uint8_t* staged_at(uint8_t* tile, int row, int c) {
  const int sw = kRow == 128 ? row & 7 : (row >> 1) & 3;
  return tile + row * kRow + ((c ^ sw) << 4);
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// 2^x to 2^-22 of it, as exp2f; below 2^-126 it is 0 (beside a sum of such that is at least 1, or a probability's gradient)
__device__ __forceinline__ float exp2_or_0(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Lane l gets the sum over the warp's lanes of v[l]: halves are exchanged and added.
__device__ __forceinline__ float column_sums(float (&v)[32], int lane) {
#pragma unroll
  for (int h = 16; h > 0; h >>= 1) {
#pragma unroll
    for (int j = 0; j < h; ++j) {
      const float send = lane & h ? v[j] : v[j + h], keep = lane & h ? v[j + h] : v[j];
      v[j] = keep + __shfl_xor_sync(0xffffffffu, send, h);
    }
  }
  return v[0];
}

// A finishing warp's 32 rows x 32 columns to memory from its staged tile: by bulk stores where a
// tensor map allows it, else row by row.
struct Writer {
  const CUtensorMap* map;
  uint8_t* tile;
  int lane;
  uint32_t slot;   // 2 KB halves of the tile in turn
  bool whole = false;   // the last bulk store reads all of the tile

  // Before a half of the tile is overwritten, or all of it: the stores that may still read it have.  (Of halves in
  // turn all but the last.)
  __device__ __forceinline__ void wait_half() {
    if (lane == 0) {
      if (whole) tc::bulk_wait_read();
      else tc::bulk_wait_read_1();
    }
    whole = false;
    __syncwarp();
  }
  __device__ __forceinline__ void wait_whole() {
    if (lane == 0) tc::bulk_wait_read();
    whole = true;
    __syncwarp();
  }
  __device__ __forceinline__ void send(uint8_t* src, int x, int y, bool add) {
    tc::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      if (add) tc::tma_add_2d(map, src, x, y);
      else tc::tma_store_2d(map, src, x, y);
      tc::bulk_commit();
    }
  }
  // 16 words of 2 bf16 a lane
  __device__ __forceinline__ void stage_bf16(uint8_t* to, const uint32_t (&w)[16]) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uint4*>(staged_at<64>(to, lane, j)) =
          make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
  }
  // the tile's rows are the 32 columns, its columns the lanes
  template <typename T>
  __device__ __forceinline__ void stage_transposed(uint8_t* to, const float (&v)[32]) {
    constexpr int kRow = 32 * (int)sizeof(T), kVec = 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      uint8_t* p = staged_at<kRow>(to, i, lane / kVec) + lane % kVec * sizeof(T);
      if (sizeof(T) == 4) *reinterpret_cast<float*>(p) = v[i];
      else *reinterpret_cast<bf16*>(p) = __float2bfloat16_rn(v[i]);
    }
  }
  template <typename T>
  __device__ __forceinline__ void put_transposed(const float (&v)[32], int x, int y, bool add) {
    if (sizeof(T) == 4) wait_whole();
    else wait_half();
    uint8_t* to = sizeof(T) == 4 ? tile : tile + 2048 * slot;
    slot ^= 1;
    stage_transposed<T>(to, v);
    send(to, x, y, add);
  }
  __device__ __forceinline__ void put_bf16(const uint32_t (&w)[16], int x, int y) {
    wait_half();
    uint8_t* to = tile + 2048 * slot;
    slot ^= 1;
    stage_bf16(to, w);
    send(to, x, y, false);
  }
  __device__ __forceinline__ void stage_fp32(const float (&v)[32]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      *reinterpret_cast<float4*>(staged_at<128>(tile, lane, j)) =
          make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
  }
  __device__ __forceinline__ void put_fp32(const float (&v)[32], int x, int y, bool add) {
    wait_whole();
    stage_fp32(v);
    send(tile, x, y, add);
  }
  // rows 0 .. n - 1 to out + at[row] * ldo: columns 0 .. cols - 1; `at` of row l is lane l's
  template <typename T>
  __device__ __forceinline__ void put_rows(const float (&v)[32], T* out, int64_t at, int n, int cols,
                                           bool transposed) {
    constexpr int kRow = 32 * (int)sizeof(T), kVec = 16 / (int)sizeof(T), kLanes = 32 / kVec;
    wait_whole();   // (bulk stores of a joint launch's other product)
    if (transposed) {
      stage_transposed<T>(tile, v);
    } else if (sizeof(T) == 4) {
      stage_fp32(v);
    } else {
      uint32_t w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1]);
      stage_bf16(tile, w);
    }
    __syncwarp();
    // (the same for the warp: its rows' places differ by whole rows)
    const bool vec = cols == 32 && __all_sync(0xffffffffu, (reinterpret_cast<uintptr_t>(out + at) & 15) == 0);
    if (vec) {
      const int piece = lane % kLanes;
#pragma unroll 1
      for (int r0 = 0; r0 < 32; r0 += kVec) {
        const int row = r0 + lane / kLanes;
        const int64_t to = __shfl_sync(0xffffffffu, at, row);
        if (row < n)
          AGN_ST(reinterpret_cast<uint4*>(out + to + piece * kVec),
                 *reinterpret_cast<const uint4*>(staged_at<kRow>(tile, row, piece)));
      }
    } else {
#pragma unroll 1
      for (int r0 = 0; r0 < n; r0 += 8) {   // eight under way
        int64_t to[8];
        T value[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int row = min(r0 + j, n - 1);
          to[j] = __shfl_sync(0xffffffffu, at, row);
          value[j] = *reinterpret_cast<const T*>(staged_at<kRow>(tile, row, lane / kVec) + lane % kVec * sizeof(T));
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (r0 + j < n && lane < cols) AGN_ST(out + to[j] + lane, value[j]);
      }
    }
  }
};

// After a role gave up and all have ended: wait for the copies of the last stages, where what will not
// come any more (the loads of the CTA that armed fewer stages) is made up for.
template <int kCtas>
__device__ __forceinline__ void land(uint64_t* full, const int* loaded, int stages, uint32_t bytes) {
  const int n0 = *loaded, n1 = kCtas == 2 ? tc::ld_cluster_int(loaded, 1) : n0, n = max(n0, n1);
#pragma unroll 1
  for (int i = max(0, n - stages); i < n; ++i) {
    uint64_t* bar = &full[i % stages];
    if (i >= n0) tc::mbar_arrive_expect_tx(bar, bytes);   // (the second CTA's copies alone)
    else if (i >= n1) tc::mbar_complete_tx(bar, bytes);
    tc::mbar_wait_bounded(bar, (uint32_t)(i / stages) & 1, kWaitNs);
  }
}

// kWide: the finishing warps hold 128 sums a thread: fp32 tiles of 256 columns; bf16 with more k than a sum takes
// (one row, K = 4096: the loss is off by 2e-7 of it, by 1.7e-6 with one sum; K = 65536, sums that only grow: 2e-4).
template <int kCtas, int kEpi, int kPlanes, bool kWide>
__global__ void __launch_bounds__(kThreads, 1) ce_gemm_kernel(const __grid_constant__ GemmLaunch launch) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staged = ring + kRing;                                          // [finishing warp][4 KB]
  float* biases = reinterpret_cast<float*>(staged + 8 * kStaged);          // [finishing warp][128]
  uint64_t* full = reinterpret_cast<uint64_t*>(biases + 8 * 128);          // (first CTA's: both CTAs' operands)
  uint64_t* empty = full + kMaxStages;
  uint64_t* acc_full = empty + kMaxStages;
  uint64_t* acc_empty = acc_full + 2;                                      // (first CTA's)
  uint64_t* drained = acc_empty + 2;
  int* loaded_out = reinterpret_cast<int*>(drained + 1);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(loaded_out + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = kCtas == 2 ? (int)cluster_rank() : 0;
  const int group = blockIdx.x / kCtas, groups = gridDim.x / kCtas;
  const int bn = launch.args[0].bn, nb = bn / kCtas;
  // (A's rows past its box are whatever follows in shared memory: rows of sums that nobody reads)
  const uint32_t a_bytes = launch.args[0].a_box * 128, stage = a_bytes + nb * 128;
  const int stages = min(kMaxStages, (int)(kRing / stage));
  const uint32_t wait_ns = launch.args[0].wait_ns;

  auto stop_all = [&] {
    if (kCtas == 2) tc::give_up(abort_flag);
    else *abort_flag = 1;
  };
  auto commit = [&](uint64_t* bar) {
    if (kCtas == 2) tc::mma_commit_pair(bar);
    else tc::mma_commit(bar);
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < kMaxStages; ++s) {
      tc::mbar_init(&full[s], 1);
      tc::mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      tc::mbar_init(&acc_full[b], 1);
      tc::mbar_init(&acc_empty[b], 8 * kCtas);
    }
    tc::mbar_init(drained, 1);
    *loaded_out = 0;
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 2) {
    if (kCtas == 2) {
      tc::tmem_alloc_pair(tmem_holder, 512);
      tc::tmem_relinquish_pair();
    } else {
      tc::tmem_alloc(tmem_holder, 512);
      tc::tmem_relinquish();
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  if (kCtas == 2) cluster_sync();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  pdl_begin();

  __shared__ Geometry geo[2];
  if (threadIdx.x < 2 && (int)threadIdx.x < launch.n) geo[threadIdx.x] = geometry<kCtas>(launch.args[threadIdx.x]);
  __syncthreads();
  constexpr uint32_t kSets = kPlanes == 3 ? 2 : 1;   // accumulators of a sum
  const uint32_t acc_cols = kSets * bn;
  constexpr bool kOne = kWide && kPlanes == 3;   // one set of sums in TMEM, not two in turn
  constexpr int kSumK = sum_steps(kCtas, kEpi, kPlanes, kWide);
  // Unit i of this CTA (pair): of product p, number u.  One product: in turn.  Two: the longer units first, in
  // turn; the CTAs that then have one less begin with as many of the shorter as take that one's time, and are
  // the first when the rest is given out in turn.
  const bool two = kEpi == kOut && launch.n == 2;
  const int longer = two && geo[1].kt_per > geo[0].kt_per ? 1 : 0;
  const int n_long = geo[longer].units, n_short = two ? geo[1 - longer].units : 0;
  const int more = n_long % groups;   // CTAs with one more long unit
  constexpr int kBeside = kPlanes == 3 ? 3 : 6;   // a unit's time beside its stages, in stages
  const int ahead = two && more ? (geo[longer].kt_per + kBeside) / (geo[1 - longer].kt_per + kBeside) : 0;
  const int mine = n_long / groups + (group < more ? 1 : 0);
  const int rank = group >= more ? group - more : group - more + groups;
  struct Place {
    int p, u;   // u < 0: no more
  };
  auto place = [&](int i) {
    if (i < mine) return Place{longer, i * groups + group};
    int j = i - mine, u = -1;
    if (group >= more) {
      if (j < ahead) u = j * (groups - more) + rank;
      else j -= ahead;
    }
    if (u < 0) u = ahead * (groups - more) + j * groups + rank;
    return Place{1 - longer, u < n_short ? u : -1};
  };
  auto unit_of = [&](Place at) { return Unit(geo[at.p], launch.args[at.p].splits, at.u); };

  // (kWide: 128 x 72 + 256 x 216 registers are the launch's 384 x 168)
  if (warp < 4) {
    if (kWide) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0 && lane == 0) {
      const uint32_t full0 = kCtas == 2 ? tc::map_cluster(full, 0) : 0;
      int s = 0, loaded = 0, stop = INT32_MAX;
      uint32_t phase = 1;   // (the first round finds every stage free)
      bool ok = true;
      for (int i = 0; ok; ++i) {
        const Place at = place(i);
        if (at.u < 0) break;
        const int p = at.p;
        const GemmArgs& a = launch.args[p];
        const bool gathered = geo[p].gathered;
        const CUtensorMap* pa = gathered && a.alt == 1 ? &launch.maps[p].alt : &launch.maps[p].a;
        const CUtensorMap* pb = gathered && a.alt == 2 ? &launch.maps[p].alt : &launch.maps[p].b;
        const Unit t = unit_of(at);
        const int m = (t.m * kCtas + cta) * 128, n = t.n * bn + cta * nb;
        const bool a_mn = a.a_mn, b_mn = a.b_mn;
        const int twice = a.twice;
        if (a.withhold == cta + 1) stop = max(0, t.kt * kPlanes - 1);
        for (int kt = t.kt0; ok && kt < t.kt0 + t.kt; ++kt) {
#pragma unroll 1
          for (int z = 0; z < kPlanes; ++z) {
            if (loaded >= stop) {
              ok = false;
              break;
            }
            if (!tc::wait_mbar<false>(&empty[s], phase, abort_flag, wait_ns)) {
              stop_all();
              ok = false;
              break;
            }
            uint8_t* st = ring + s * stage;
            auto load = [&](uint8_t* dst, const CUtensorMap* map, int x, int y, int piece) {
              if (kCtas == 2) tc::tma_load_3d_pair(dst, map, full0 + 8u * (uint32_t)s, x, y, piece);
              else tc::tma_load_3d(dst, map, &full[s], x, y, piece);
            };
            if (cta == 0) tc::mbar_arrive_expect_tx(&full[s], kCtas * stage);
            const int k = (twice ? kt >> 1 : kt) * kBK;
            const int za = twice == 1 ? kt & 1 : z, zb = twice == 2 ? kt & 1 : z;
            if (a_mn) {
              load(st, pa, m, k, za);
              load(st + kBox, pa, m + 64, k, za);
            } else {
              load(st, pa, k, m, za);
            }
            if (b_mn) {
              for (int j = 0; j < nb; j += 64) load(st + a_bytes + j * 128, pb, n + j, k, zb);
            } else {
              load(st + a_bytes, pb, k, n, zb);
            }
            ++loaded;
            if (++s == stages) s = 0, phase ^= 1;
          }
        }
      }
      *loaded_out = loaded;
    } else if (warp == 1 && lane == 0 && cta == 0) {
      const uint32_t r0 = tc::smem_u32(ring);
      const uint32_t step = stage >> 4;
      int s = 0, done = 0;   // (done: sums, from the launch's first)
      uint32_t phase = 0;
      bool ok = true;
      for (int i = 0; ok; ++i) {
        const Place at = place(i);
        if (at.u < 0) break;
        const int p = at.p;
        const GemmArgs& a = launch.args[p];
        const Unit t = unit_of(at);
        const bool a_mn = a.a_mn, b_mn = a.b_mn;
        const uint32_t idesc = tc::idesc_bf16_f32(128 * kCtas, bn, a_mn, b_mn);
        const uint64_t da0 = tc::smem_desc_sw128(r0, a_mn ? kBox : 16, 1024);
        const uint64_t db0 = tc::smem_desc_sw128(r0 + a_bytes, b_mn ? kBox : 16, 1024);
        const uint64_t ka = (a_mn ? 2048 : 32) >> 4, kb = (b_mn ? 2048 : 32) >> 4;   // 16 k
        // 64 k of A in slot i times B in slot j
        auto product = [&](uint32_t d, int i, int j, bool first) {
          const uint64_t da = da0 + (uint64_t)(i * step), db = db0 + (uint64_t)(j * step);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            if (kCtas == 2) tc::mma_bf16_pair(d, da + kk * ka, db + kk * kb, idesc, kk > 0 || !first);
            else tc::mma_bf16(d, da + kk * ka, db + kk * kb, idesc, kk > 0 || !first);
          }
        };
        auto arrived = [&](int i, uint32_t ph) {
          ok = ok && tc::wait_mbar<false>(&full[i], ph, abort_flag, wait_ns);
          tc::tc_fence_after();
          return ok;
        };
        auto next = [&] {
          if (++s == stages) s = 0, phase ^= 1;
        };
        int kt = 0;
        do {   // a sum (of nothing: announced as it is)
          const int buf = kOne ? 0 : done & 1;
          // (kOne: the larger products' sums have been read; the others' further down)
          if (kOne ? done >= 1 : done >= 2)
            ok = tc::wait_mbar<true>(&acc_empty[buf], kOne ? (done - 1) & 1 : ((done >> 1) - 1) & 1, abort_flag,
                                     wait_ns);
          if (!ok) break;
          tc::tc_fence_after();
          const uint32_t d = tmem + buf * acc_cols;
          const int end = kPlanes == 3 || kWide ? min(t.kt, kt + kSumK) : t.kt;
          for (bool first = true; kt < end; ++kt, first = false) {
            if (kPlanes == 1) {
              if (!arrived(s, phase)) break;
              product(d, s, s, first);
              commit(&empty[s]);
              next();
            } else {   // pieces 0, 1, 2 as they come; a slot is free with the last product that reads it
              const int s0 = s;
              if (!arrived(s0, phase)) break;
              product(d, s0, s0, first);
              next();
              const int s1 = s;
              if (!arrived(s1, phase)) break;
              if (kOne && first && done >= 1) {
                ok = tc::wait_mbar<true>(&acc_empty[1], (done - 1) & 1, abort_flag, wait_ns);
                if (!ok) break;
                tc::tc_fence_after();
              }
              product(d + bn, s0, s1, first);
              product(d + bn, s1, s0, false);
              product(d + bn, s1, s1, false);
              commit(&empty[s1]);
              next();
              const int s2 = s;
              if (!arrived(s2, phase)) break;
              product(d + bn, s0, s2, false);
              product(d + bn, s2, s0, false);
              commit(&empty[s0]);
              commit(&empty[s2]);
              next();
            }
          }
          if (!ok || *abort_flag) {
            ok = false;   // no sums: the finishing warps give up
            break;
          }
          commit(&acc_full[buf]);
          ++done;
        } while (kt < t.kt);
      }
      if (!ok) stop_all();
    }
  } else {
    if (kWide) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int e = warp - 4, quad = warp & 3, half = e >> 2, chunks = bn / 64;   // of 32 columns
    float* bias = biases + 128 * e;
    const uint32_t empty0 = kCtas == 2 ? tc::map_cluster(acc_empty, 0) : tc::smem_u32(acc_empty);
    Writer out{nullptr, staged + e * kStaged, lane, 0};
    bool ok = true;
    int done = 0;
    for (int i = 0;; ++i) {
      const Place at = place(i);
      if (at.u < 0) break;
      const int p = at.p;
      const GemmArgs& a = launch.args[p];
      const Geometry& g = geo[p];
      const Unit t = unit_of(at);
      out.map = &launch.maps[p].c;
      const int row0 = (t.m * kCtas + cta) * 128 + 32 * quad, row = row0 + lane;
      const int col0 = t.n * bn + half * 32 * chunks;
      const bool live = row < g.M;
      // what the row needs, on its way while the sums are
      int label = -1;
      float lse = 0.f, fa = 0.f, fb = 0.f;
      if (kEpi != kOut) {
        if (live) {
          const int at = a.idx ? AGN_LD(a.idx + row) : row;
          label = AGN_LD(a.labels + at) - a.class0 - col0;
          if (kEpi == kGrad) {
            lse = AGN_LD(a.lse + at);
            const float dl = a.dloss ? AGN_LD(a.dloss + at) : 1.f;
            fb = a.scale * dl;
            fa = a.dlse ? a.scale * (dl + AGN_LD(a.dlse + at)) : fb;
          }
        }
        __syncwarp();
        for (int i = lane; i < 32 * chunks; i += 32) {
          const int c = a.class0 + col0 + i;
          bias[i] = col0 + i >= g.N ? -INFINITY : a.bias ? AGN_LD(a.bias + c) : 0.f;
        }
        __syncwarp();
      }
      float top = -INFINITY, sum = 0.f;

      // The sums in buffer `buf` are there (or will not come).
      auto wait_sums = [&](int buf) {
        ok = ok && tc::wait_mbar<true>(&acc_full[buf], kOne ? done & 1 : (done >> 1) & 1, abort_flag, wait_ns) &&
             !*abort_flag;
        ok = __all_sync(0xffffffffu, ok);
        tc::tc_fence_after();
        if (!ok && lane == 0) {
          stop_all();
          if (a.err) atomicExch(a.err, 1);
        }
      };
      auto free_sums = [&](int buf) {
        if (!ok) return;
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive_relaxed(empty0 + 8u * (uint32_t)buf);
      };
      const uint32_t at0 = tmem + ((uint32_t)(32 * quad) << 16) + half * 32 * chunks;

      // 32 columns of sums of this row
      auto finish = [&](int ch, float (&v)[32]) {
        const int col = col0 + 32 * ch;   // (of this product)
        if (kEpi != kOut) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 b = *reinterpret_cast<const float4*>(bias + 32 * ch + i);
            v[i] += b.x; v[i + 1] += b.y; v[i + 2] += b.z; v[i + 3] += b.w;
          }
        }
        const uint32_t hit = (uint32_t)(label - 32 * ch);   // < 32: the label's column is here
        if (kEpi == kLse) {
          if (hit < 32) {
            float z = v[0];
#pragma unroll
            for (int i = 1; i < 32; ++i) z = hit == i ? v[i] : z;
            AGN_ST(a.zlab + row, z);
          }
          float m[4] = {top, v[1], v[2], v[3]}, s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 32; ++i) m[i & 3] = fmaxf(m[i & 3], v[i]);
          const float most = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
          const float from = most == -INFINITY ? 0.f : most;
          sum *= exp2_or_0((top - from) * kLog2e);
#pragma unroll
          for (int i = 0; i < 32; ++i) s[i & 3] += exp2_or_0((v[i] - from) * kLog2e);
          sum += (s[0] + s[1]) + (s[2] + s[3]);
          top = most;
        } else if (kEpi == kGrad) {
          const bool dead = !live || lse == -INFINITY;   // (no class that is not masked: no gradient)
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = fa * exp2_or_0((v[i] - lse) * kLog2e);
          if (hit < 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = hit == i ? v[i] - fb : v[i];
          }
          if (dead) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
          }
#pragma unroll
          for (int z = 0; z < p_pieces(kPlanes); ++z) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              if (z == 0) {
                w[i] = pack2(v[2 * i], v[2 * i + 1]);
              } else {   // what the pieces before left
                float x[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  bf16 p0, p1, p2;
                  split3(v[2 * i + k], p0, p1, p2);
                  x[k] = __bfloat162float(z == 1 ? p1 : p2);
                }
                w[i] = pack2(x[0], x[1]);
              }
            }
            out.put_bf16(w, col, z * a.p_plane + row0);
          }
          if (a.db && row0 < g.M) {
            const float s = column_sums(v, lane);
            if (col + lane < g.N) AGN_ST(a.db + (int64_t)(row0 >> 5) * a.ld_db + col + lane, s);
          }
        } else {
          if (row0 >= g.M || col >= g.N) return;   // (warp-uniform)
          const bool flip = a.transposed;
          const int x0 = flip ? row0 : col, y0 = flip ? col : row0;   // the output's column and row
          if (a.part) {
            if (flip) out.put_transposed<float>(v, x0, t.split * a.part_rows + y0, a.part == 2);
            else out.put_fp32(v, x0, t.split * a.part_rows + y0, a.part == 2);
          } else if (a.tma_out && !(a.scatter && g.gathered)) {
            if (a.dtype == AGN_PREC_BF16) {
              if (flip) {
                out.put_transposed<bf16>(v, x0, y0, false);
              } else {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1]);
                out.put_bf16(w, x0, y0);
              }
            } else if (flip) {
              out.put_transposed<float>(v, x0, y0, false);
            } else {
              out.put_fp32(v, x0, y0, false);
            }
          } else {
            const int n = min(32, (flip ? g.N : g.M) - y0), cols = min(32, (flip ? g.M : g.N) - x0);
            const int y = y0 + min(lane, n - 1);
            const int64_t to = (int64_t)(a.scatter ? AGN_LD(a.idx + y) : y) * a.ldo + x0;
            if (a.dtype == AGN_PREC_BF16) out.put_rows(v, static_cast<bf16*>(a.out), to, n, cols, flip);
            else out.put_rows(v, static_cast<float*>(a.out), to, n, cols, flip);
          }
        }
      };

      const uint32_t none = 0x7fc00000u;   // what could not be computed
      if (kPlanes == 1 && !kWide) {
        const int buf = done & 1;
        wait_sums(buf);
#pragma unroll 1
        for (int ch = 0; ch < chunks; ++ch) {
          uint32_t r[32];
          float v[32];
          if (ok) {
            tc::tmem_ld_32x32b_x32(at0 + buf * acc_cols + 32 * ch, r);
            tc::tmem_ld_wait();
          }
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(!ok ? none : t.kt == 0 ? 0u : r[i]);
          if (ch + 1 == chunks) free_sums(buf);
          finish(ch, v);
        }
        ++done;
      } else {
        constexpr int kMost = kWide ? 4 : 2;   // chunks
        float v[kMost][32];
#pragma unroll
        for (int i = 0; i < 32 * kMost; ++i) v[i / 32][i % 32] = -0.f;   // (one sum stays as it is)
        // adds one accumulator's columns of a chunk, 16 at a time
        auto add = [&](uint32_t at, float (&sum)[32]) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[16];
            if (ok) {
              tc::tmem_ld_32x32b_x16(at + 16 * h, r);
              tc::tmem_ld_wait();
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[16 * h + i] += __uint_as_float(!ok ? none : t.kt == 0 ? 0u : r[i]);
          }
        };
        int kt = 0;
        do {
          const int buf = kOne ? 0 : done & 1;
          wait_sums(buf);
          const uint32_t at = at0 + buf * acc_cols;
          if (kOne) {
#pragma unroll
            for (int ch = 0; ch < kMost; ++ch) add(at + 32 * ch, v[ch]);
            free_sums(0);
#pragma unroll
            for (int ch = 0; ch < kMost; ++ch) add(at + bn + 32 * ch, v[ch]);
            free_sums(1);
          } else {
#pragma unroll
            for (int ch = 0; ch < kMost; ++ch) {
              if (ch >= chunks) break;
              add(at + 32 * ch, v[ch]);
              if (kPlanes == 3) add(at + bn + 32 * ch, v[ch]);
            }
            free_sums(buf);
          }
          ++done;
          kt += kSumK;
        } while (kt < t.kt);
#pragma unroll
        for (int ch = 0; ch < kMost; ++ch)
          if (ch < chunks) finish(ch, v[ch]);
      }
      if (kEpi == kLse && live)
        AGN_ST(a.ms + (int64_t)row * a.ld_ms + a.ms0 + 2 * t.n + half, make_float2(top, sum));
    }
    if (kEpi != kLse && lane == 0) tc::bulk_wait();   // the last stores are done before the kernel is
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  if (kCtas == 2) cluster_sync();   // no CTA leaves while the other reads its memory or signals its barriers
  if (__builtin_expect(*abort_flag, 0)) {   // (the same in both CTAs: nobody is left who could set it)
    if (warp == 1 && lane == 0) {
      if (cta == 0) {
        commit(drained);   // (the thread that issued the MMAs)
        tc::mbar_wait_bounded(drained, 0, kWaitNs);
        land<kCtas>(full, loaded_out, stages, stage);
      } else {
        tc::mbar_wait_bounded(drained, 0, kWaitNs);
      }
    }
    __syncthreads();
    if (kCtas == 2) cluster_sync();
  }
  if (warp == 2) {
    if (kCtas == 2) tc::tmem_dealloc_pair(tmem, 512);
    else tc::tmem_dealloc(tmem, 512);
  }
}

template <int kCtas, int kEpi, int kPlanes, bool kWide>
Status queue(const GemmLaunch& g, int64_t max_units, cudaStream_t st) {
  struct Tag {};
  auto kern = ce_gemm_kernel<kCtas, kEpi, kPlanes, kWide>;
  int dev = 0, sms = 0;
  AGN_TRY(current_device(&dev));
  AGN_TRY(device_sms(dev, &sms));
  AGN_TRY_CUDA(allow_smem<Tag>(kern, kSmem, dev));
  const unsigned groups = (unsigned)std::max<int64_t>(1, std::min<int64_t>(max_units, sms / kCtas));
  if (kCtas == 2)
    AGN_TRY_CUDA(launch_pdl_cluster(kern, dim3(2 * groups), dim3(kThreads), kSmem, dim3(2, 1, 1), st, g));
  else
    AGN_TRY_CUDA(launch_pdl(kern, dim3(groups), dim3(kThreads), kSmem, st, g));
  return Status::Ok();
}

template <int kCtas, int kPlanes, bool kWide = false>
Status queue_for(int epilogue, const GemmLaunch& g, int64_t max_units, cudaStream_t st) {
  if (epilogue == kLse) return queue<kCtas, kLse, kPlanes, kWide>(g, max_units, st);
  if (epilogue == kGrad) return queue<kCtas, kGrad, kPlanes, kWide>(g, max_units, st);
  return queue<kCtas, kOut, kPlanes, kWide>(g, max_units, st);
}

}  // namespace

Status gemm(int ctas, int epilogue, const GemmLaunch& launch, int64_t max_units, cudaStream_t st) {
  GemmLaunch g = launch;
  for (GemmArgs& a : g.args)
    if (!a.wait_ns) a.wait_ns = (uint32_t)kWaitNs;
  bool wide = false;   // bf16: more than a sum
  for (int i = 0; i < g.n; ++i) {
    const int64_t steps = ceil_div(g.args[i].K, kBK) * (g.args[i].twice ? 2 : 1);
    wide = wide || ceil_div(steps, g.args[i].splits) > std::max(16, sum_steps(ctas, epilogue, 1, true));
  }
  if (g.args[0].planes == 3 && g.args[0].bn == 256) return queue_for<2, 3, true>(epilogue, g, max_units, st);
  if (g.args[0].planes == 3)
    return ctas == 2 ? queue_for<2, 3>(epilogue, g, max_units, st) : queue_for<1, 3>(epilogue, g, max_units, st);
  if (wide)
    return ctas == 2 ? queue_for<2, 1, true>(epilogue, g, max_units, st) : queue_for<1, 1, true>(epilogue, g, max_units, st);
  return ctas == 2 ? queue_for<2, 1>(epilogue, g, max_units, st) : queue_for<1, 1>(epilogue, g, max_units, st);
}

}  // namespace ce

AGN_BOUNDS_UNIT(linear_ce_gemm)

}  // namespace agn
