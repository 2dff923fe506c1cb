// Product of microscaled 4-bit matrices on the tensor cores: rows of x and rows
// of w (both along K) quantised as in mx4.cu,
//   y[r][f] = act(sum_k x[r][k] w[f][k] + b[f]),
// tcgen05.mma kind::mxf4 (products of E2M1 values scaled by both blocks'
// powers of two, f32 sums in TMEM), output fp32, bf16 or 4-bit codes again.
//
// Few rows, one CTA a tile: the features are the MMA's M (128 TMEM lanes), the rows
// of x its N (BN columns), so that narrow tiles read each weight once and a lane's
// features are contiguous in every output row.  (Many rows: see the pairs of CTAs
// below.)  A stage is 256 k: 128-byte rows
// of codes (TMA, 128-byte swizzle) and two scale tiles of 512 bytes (bulk copies;
// the scales are stored as the tensor core wants them), copied to TMEM by the
// thread that issues the MMAs.  K past the last element costs nothing: codes and
// scales are zero there.  Few output tiles split K over a cluster: every CTA
// leaves its sums in its shared memory, and each finishes a share of the columns,
// adding the others' in rank order through distributed shared memory (no
// workspace, no atomics, the same bits each time).
// Every wait on an mbarrier is bounded (2 s): a tile that gives up is stored as
// NaN and sets *err.  Whoever gives up, each stage that was armed is waited for (with a
// limit of its own) before its memory is used again or its CTA ends.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <type_traits>

#include "mlp.cuh"
#include "mlp_tc.cuh"
#include "mx4.cuh"
#include "ops.cuh"
#include "tc_ptx.cuh"

namespace agn {

namespace {

constexpr int kThreads = 256;
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr int kABytes = 128 * 128;
constexpr int kSfBytes = 2 * kMxTileBytes; // a stage's scales of 128 rows

// Shared memory that keeps every other kernel with TMEM off the SM (the library's take
// 47 KB and more): CTAs of one launch wait for each other, and one that holds TMEM
// while it waits for a CTA that another launch's CTA keeps from allocating, and the other
// way round, would wait for ever.
constexpr size_t kAlone = 184 * 1024;

template <int BN>
struct Tile {
  static constexpr int kBBytes = BN * 128;
  static constexpr int kStageBytes = kABytes + kBBytes + 2 * kSfBytes;
  static constexpr int kStages = BN <= 32 ? 8 : BN == 64 ? 7 : 6;
  static constexpr uint32_t kSfCol = BN < 32 ? 32 : BN;   // first TMEM column of the scales
  static constexpr uint32_t kCols = kSfCol + 16;
  static constexpr uint32_t kTmemCols = kCols <= 64 ? 64 : kCols <= 128 ? 128 : 256;
  static constexpr size_t kNeeded = (size_t)kStages * kStageBytes + 1024 + 256;
  static constexpr size_t kSmem = kNeeded < kAlone ? kAlone : kNeeded;
  static_assert(kStageBytes % 1024 == 0, "tiles of the 128-byte swizzle");
  static_assert(kSmem <= 232448, "shared memory");
  static_assert(BN * 128 * 4 <= kStages * kStageBytes, "the sums fit into the ring");
};

// Bounded waits that give up when another role of the CTA has: kTmem for barriers
// that order TMEM accesses alone (relaxed, with a tcgen05 fence after it).
template <bool kTmem>
__device__ __forceinline__ bool wait_mbar(uint64_t* bar, uint32_t parity, volatile int* abort_flag,
                                          uint64_t limit_ns) {
  uint64_t t0 = 0;
  for (uint32_t it = 1;; ++it) {
    uint32_t got;
    if (kTmem)
      asm volatile(
          "{\n\t.reg .pred p;\n\t"
          "mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(got) : "r"(tc::smem_u32(bar)), "r"(parity) : "memory");
    else
      got = tc::mbar_try_wait(bar, parity);
    if (got) return true;
    if ((it & 63) == 0) {
      const uint64_t now = tc::globaltimer_ns();
      if (t0 == 0) t0 = now;
      if (*abort_flag || now - t0 > limit_ns) return false;
    }
  }
}

struct LinearArgs {
  const uint8_t *w_scales, *x_scales;
  int64_t rows, out;
  int64_t tiles_k;          // scale tiles along K
  int64_t row_tiles;        // 128-row scale tiles of x
  int k_steps;              // ceil(in / 64)
  uint16_t split;           // CTAs of a cluster, along K
  uint16_t withhold;        // test hook: rank r = withhold - 1 leaves out a stage (0: none)
  const float* bias;
  int relu, dtype;
  int vec;                  // rows of y start 16-byte aligned
  uint32_t wait_ns;         // limit of the roles' waits
  int64_t bulk_out;         // features that bulk stores may write: whole 16-byte pieces of
                            // aligned rows (4-bit output: all)
  void* y;
  int64_t ldy;
  uint8_t* y_scales;
  int64_t y_tiles_k;
  int* err;
};
// (With 144 bytes the one-CTA kernel was compiled to 40 registers, not 48, and took longer: 128 rows
// of 4096 to 4096 9.3 us for 8.3, 37 of 784 to 1000 4.7 for 4.2.)
static_assert(sizeof(LinearArgs) == 128, "kernel arguments");

__device__ __forceinline__ float4 ld_cluster4(const float* p, uint32_t rank) {
  const uint32_t own = tc::smem_u32(p);
  uint32_t at;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(own), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}

// Four features f .. f + 3 (n of them exist) of row r: bias, ReLU, store.  A warp
// calls it for one row, lane by lane along 128 features: in the 4-bit form
// eight lanes are a block and the warp's four scales one word.
__device__ __forceinline__ void finish(const LinearArgs& a, int64_t r, int64_t f, int n,
                                       const float (&b)[4], float4 s) {
  float v[4] = {s.x + b[0], s.y + b[1], s.z + b[2], s.w + b[3]};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (a.relu && v[e] <= 0.f) v[e] = 0.f;
  if (a.dtype == AGN_PREC_MX4) {
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (e >= n) v[e] = 0.f;
      amax = max(amax, __float_as_uint(v[e]) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    const uint32_t code = mx_scale_code(amax);
    const float inv = mx_inverse(code);
    const float u[8] = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv, 0.f, 0.f, 0.f, 0.f};
    const uint32_t q = code == 255 ? 0u : mx_pack8(u) & 0xffffu;
    const uint32_t hi = __shfl_down_sync(0xffffffffu, q, 1);
    const int lane = threadIdx.x & 31;
    const int64_t row_bytes = mx_row_bytes(a.out);
    if ((lane & 1) == 0 && f / 2 < row_bytes)
      AGN_ST(reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.y) + r * row_bytes + f / 2),
             q | hi << 16);
    uint32_t word = code << (8 * (lane >> 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
    word |= __shfl_xor_sync(0xffffffffu, word, 16);
    if (lane == 0)
      AGN_ST(reinterpret_cast<uint32_t*>(a.y_scales + mx_scale_at(r, f / kMxBlock, a.y_tiles_k)),
             word);
  } else if (a.dtype == AGN_PREC_BF16) {
    bf16* p = static_cast<bf16*>(a.y) + r * a.ldy + f;
    if (a.vec && n == 4) {
      const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
      AGN_ST(reinterpret_cast<uint2*>(p), make_uint2(*reinterpret_cast<const uint32_t*>(&lo),
                                                     *reinterpret_cast<const uint32_t*>(&hi)));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < n) AGN_ST(p + e, __float2bfloat16_rn(v[e]));
    }
  } else {
    float* p = static_cast<float*>(a.y) + r * a.ldy + f;
    if (a.vec && n == 4) {
      AGN_ST(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < n) AGN_ST(p + e, v[e]);
    }
  }
}

// One bulk copy (or, in the bounds-checked build, its bytes alone).
__device__ __forceinline__ void load_scales(void* dst, const uint8_t* src, uint32_t bytes,
                                            uint64_t* bar) {
  if (AGN_BOUNDS_OK(src, bytes)) {
    tc::bulk_load(dst, src, bytes, bar);
  } else {
    AGN_BOUNDS_FAIL(src);
    tc::mbar_complete_tx(bar, bytes);
  }
}

template <int BN>
__global__ void __launch_bounds__(kThreads)
mx4_linear_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX,
                  const LinearArgs a) {
  using Cfg = Tile<BN>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  constexpr int stages = Cfg::kStages;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + stages * Cfg::kStageBytes);
  uint64_t* empty = full + stages;
  uint64_t* done = empty + stages;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t f0 = (int64_t)blockIdx.x * 128, n0 = (int64_t)blockIdx.y * BN;
  const int rank = blockIdx.z;
  const int KT_all = (a.k_steps + 3) / 4, kt_per = (KT_all + a.split - 1) / a.split;
  const int kt0 = rank * kt_per, KT = min(KT_all, kt0 + kt_per) - kt0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      tc::mbar_init(&full[s], 1);
      tc::mbar_init(&empty[s], 1);
    }
    tc::mbar_init(done, 1);
    *abort_flag = 0;
    tc::fence_mbar_init();
    tc::tma_prefetch_desc(&tmW);
    tc::tma_prefetch_desc(&tmX);
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_holder, Cfg::kTmemCols);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  pdl_begin();

  if (warp == 0 && lane == 0) {
    const int64_t xt = n0 >> 7;   // 128-row scale tile of x
    int s = 0, armed = 0;
    uint32_t phase = 1;   // (the first round finds every stage free)
    const int kt1 = kt0 + KT - (a.withhold == rank + 1 ? 1 : 0);
    for (int kg = kt0; kg < kt1; ++kg) {   // stages along the whole K
      if (!wait_mbar<false>(&empty[s], phase, abort_flag, a.wait_ns)) {
        *abort_flag = 1;
        break;
      }
      uint8_t* st = smem + s * Cfg::kStageBytes;
      uint8_t* sf = st + kABytes + Cfg::kBBytes;
      const uint32_t sfb = (uint32_t)min((int64_t)2, a.tiles_k - 2 * kg) * kMxTileBytes;
      tc::mbar_arrive_expect_tx(&full[s], kABytes + Cfg::kBBytes + 2 * sfb);
      tc::tma_load_2d(st, &tmW, &full[s], kg * 128, (int)f0);
      tc::tma_load_2d(st + kABytes, &tmX, &full[s], kg * 128, (int)n0);
      load_scales(sf, a.w_scales + ((int64_t)blockIdx.x * a.tiles_k + 2 * kg) * kMxTileBytes, sfb,
                  &full[s]);
      load_scales(sf + kSfBytes, a.x_scales + (xt * a.tiles_k + 2 * kg) * kMxTileBytes, sfb, &full[s]);
      armed = min(armed + 1, stages);
      if (++s == stages) s = 0, phase ^= 1;
    }
    // Nobody passes the barrier below while copies are in flight: the stages armed last are waited for,
    // for as long as the others' waits can last and 2 s more.
    for (; armed > 0; --armed) {
      if (--s < 0) s = stages - 1, phase ^= 1;
      tc::mbar_wait_bounded(&full[s], phase ^ 1, 2 * kWaitNs);
    }
  } else if (warp == 1 && lane == 0) {
    // (short between the MMAs: see the pairs' kernel)
    const uint32_t sfa = tmem + Cfg::kSfCol, sfb = sfa + 8;
    const uint32_t s0 = tc::smem_u32(smem);
    const uint64_t da0 = tc::smem_desc_sw128(s0, 16, 1024);
    const uint64_t ds0 = tc::smem_desc_rows16(s0 + kABytes + Cfg::kBBytes, 128);
    constexpr uint64_t kToB = kABytes >> 4, kTile = kMxTileBytes >> 4, kToX = kSfBytes >> 4;
    const uint32_t sfx = sfb + (uint32_t)(n0 & 127) / 32;   // this tile's rows of the 128 (BN = 64)
    uint64_t da = da0, ds = ds0;
    int s = 0;
    uint32_t phase = 0;
    bool ready = false;
    for (int left = min(a.k_steps - 4 * kt0, 4 * KT), first = 1; left > 0; left -= 4, first = 0) {
      if (!ready && !wait_mbar<false>(&full[s], phase, abort_flag, a.wait_ns)) {
        *abort_flag = 1;
        break;
      }
      tc::tc_fence_after();
      // scale words: blocks 0-3 of the stage, then 4-7
      tc::cp_32x128b_warpx4(sfa, ds);
      tc::cp_32x128b_warpx4(sfb, ds + kToX);
      if (left > 2) {
        tc::cp_32x128b_warpx4(sfa + 4, ds + kTile);
        tc::cp_32x128b_warpx4(sfb + 4, ds + kToX + kTile);
      }
      tc::mma_mxf4(tmem, da, da + kToB, tc::idesc_mxf4(128, BN, 0), sfa, sfx, !first);
      if (left > 1)
        tc::mma_mxf4(tmem, da + 2, da + kToB + 2, tc::idesc_mxf4(128, BN, 2), sfa, sfx, 1);
      uint64_t* const mine = &empty[s];
      const uint64_t d = da + 4;
      da += Cfg::kStageBytes >> 4;
      ds += Cfg::kStageBytes >> 4;
      if (++s == stages) s = 0, phase ^= 1, da = da0, ds = ds0;
      ready = tc::mbar_test_wait(&full[s], phase);
      if (left > 2)
        tc::mma_mxf4(tmem, d, d + kToB, tc::idesc_mxf4(128, BN, 0), sfa + 4, sfx + 4, 1);
      if (left > 3)
        tc::mma_mxf4(tmem, d + 2, d + kToB + 2, tc::idesc_mxf4(128, BN, 2), sfa + 4, sfx + 4, 1);
      tc::mma_commit(mine);
    }
    tc::mma_commit(done);
    tc::mbar_wait_bounded(done, 0, kWaitNs);   // (nor while MMAs are)
  }
  __syncwarp();
  const bool ok =
      __syncthreads_and(wait_mbar<false>(done, 0, abort_flag, a.wait_ns) && !*abort_flag) != 0;
  tc::tc_fence_after();
  if (!ok && threadIdx.x == 0 && a.err) atomicExch(a.err, 1);

  // the sums to shared memory (the ring is free): [column][128 features]
  float* sums = reinterpret_cast<float*>(smem);
  {
    constexpr int kPer = BN == 16 ? 16 : BN / 2;   // columns of this warp
    const int g = warp & 3, c0 = (warp >> 2) * kPer;
    if (c0 < BN) {
#pragma unroll 1
      for (int c = c0; c < c0 + kPer; c += 16) {
        uint32_t r[16];
        tc::tmem_ld_32x32b_x16(tmem + ((uint32_t)(32 * g) << 16) + (uint32_t)c, r);
        tc::tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; ++i)
          sums[(c + i) * 128 + 32 * g + lane] = ok ? __uint_as_float(r[i]) : NAN;
      }
    }
  }
  tc::tc_fence_before();
  if (a.split > 1) cluster_sync();
  else __syncthreads();
  if (warp == 1) tc::tmem_dealloc(tmem, Cfg::kTmemCols);

  // finish this CTA's columns: a warp a row of y, a lane four features
  {
    const int64_t f = f0 + 4 * lane;
    const int n = (int)max((int64_t)0, min((int64_t)4, a.out - f));
    float b[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = a.bias && e < n ? AGN_LD(a.bias + f + e) : 0.f;
    const int own1 = BN * (rank + 1) / a.split;
    for (int j = BN * rank / a.split + warp; j < own1; j += kThreads / 32) {
      if (n0 + j >= a.rows) break;   // (warp-uniform)
      const float* p = sums + j * 128 + 4 * lane;
      float4 s;
      if (a.split == 1) {
        s = *reinterpret_cast<const float4*>(p);
      } else {
        s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < a.split; ++k) {
          const float4 t = ld_cluster4(p, k);
          s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
        }
      }
      finish(a, n0 + j, f, n, b, s);
    }
  }
  if (a.split > 1) cluster_sync();   // the others' reads, before this CTA's memory goes
}

template <int BN>
Status launch_linear(const Mx4LinearArgs& m, LinearArgs a, int dev, cudaStream_t st) {
  using Cfg = Tile<BN>;
  const dim3 grid0((unsigned)ceil_div(m.out, 128), (unsigned)ceil_div(m.rows, BN));
  // CTAs along K: the most whose clusters are all resident (us, clusters of 8, 4, 2: one row of
  // 4096 to 1000, 8 tiles, 4.9, 5.6, 7.4; 64 rows of 2048 to 2048, 16 tiles, two rounds of
  // clusters of 8, 10.3, 5.7, 7.0)
  auto kern = mx4_linear_kernel<BN>;
  constexpr size_t smem = Cfg::kSmem;
  AGN_TRY_CUDA(allow_smem<Cfg>(kern, smem, dev));
  const int64_t tiles = (int64_t)grid0.x * grid0.y;
  const int kt = (a.k_steps + 3) / 4;
  a.split = std::min(8, kt);
  for (; a.split > 1; --a.split) {
    int resident = 0;
    AGN_TRY(max_clusters<Cfg>(kern, kThreads, smem, a.split, dev, &resident));
    if (resident >= tiles) break;
  }
  a.split = (int)ceil_div(kt, ceil_div(kt, a.split));   // no empty rank
  CUtensorMap tw, tx;
  AGN_TRY(make_tmap_u8_2d(&tw, m.w_codes, mx_row_bytes(m.in), m.out, mx_row_bytes(m.in), 128));
  AGN_TRY(make_tmap_u8_2d(&tx, m.x_codes, mx_row_bytes(m.in), m.rows, mx_row_bytes(m.in), BN));
  const dim3 grid(grid0.x, grid0.y, (unsigned)a.split);
  if (a.split > 1)
    AGN_TRY_CUDA(launch_pdl_cluster(kern, grid, kThreads, smem, dim3(1, 1, (unsigned)a.split), st, tw,
                                    tx, a));
  else
    AGN_TRY_CUDA(launch_pdl(kern, grid, kThreads, smem, st, tw, tx, a));
  return Status::Ok();
}

// ---------------------------------------------------------------------------
// Many rows: pairs of CTAs
// ---------------------------------------------------------------------------

// Two SMs share a tile of 256 rows x 256 features (tcgen05 cta_group::2): each
// loads its 128 rows and half of the features, 64 bytes a clock of MMA time where a CTA
// alone would load 96.  Here the rows are the MMA's M: a lane holds a row's
// consecutive features, whole blocks of a 4-bit output.  One pair for every two SMs walks over the tiles; roles by warp:
//   4     loads: codes complete on the first CTA's barriers, each CTA's scales on its own
//   0-3   bring a stage's scales from shared memory into TMEM (tcgen05.st, each warp
//         its lane quadrant): tcgen05.cp takes 97 clocks for 512 bytes, six of them a stage,
//         and little of it beside the MMAs (four MMAs 513 clocks, with six copies 860)
//   5     issues the MMAs (first CTA)
//   8-15  finish: their 128 columns into registers at once, bias, ReLU, rounding, bulk
//         stores from shared memory
// A second accumulator of 256 columns would leave no TMEM columns for the scales: the next
// tile's MMAs start once the sums are in registers.
// What bounds it, in clocks of a pair with most units (clock64 and globaltimer in a copy of the
// kernel; the SMs run at 1.87 to 1.91 GHz under it, whatever the samples of 2.07 say):
//   16384 x 4096 x 4096 to bf16, 176 thousand, 93 us (5.9 PFLOP/s): 3.5 to the first stage, 143 for 13
//   units of 16 stages and a half one, 10.7 waiting for loads, 14.5 for the sums to leave TMEM (1100
//   a unit, 940 of them a finishing warp's reads of its 128 columns), 2.3 to finish the last
//   unit, 2.4 until its stores are done.  The pairs end within 6 us of each other.
//   A stage of four MMAs takes 660 clocks there and 620 where a unit has 32 stages (8192^3, 160 us,
//   6.9 PFLOP/s); 513 are the MMAs' own, the rest the issuing thread's work between them (the scale
//   warps' reads cost nothing).  Four stages and two tiles of outputs a finishing warp: 102 us.
//   10000 x 1000 x 1000 to fp32, 24 thousand, 13 us: 3.1 to the first stage; 60 pairs of two units end at 19,
//   16 with a half one more at 23; 2.5 of each until the last stores are done.  The outputs leave at
//   3.1 TB/s over the kernel.
constexpr int kPairThreads = 512;
constexpr int kPairStages = 5;
constexpr int kPairStaged = 4096;                          // a finishing warp's tile of outputs
constexpr int kPairHalf = 128 * 128;                       // codes of 128 rows or features
constexpr int kPairStage = 2 * kPairHalf + 3 * kSfBytes;   // x, w, scales of 128 rows and 256 features
constexpr size_t kPairSmem = (size_t)kPairStages * kPairStage + 8 * (kPairStaged + 512) + 1024 + 512;
static_assert(kPairStage % 1024 == 0 && kPairSmem <= 232448 && kPairSmem >= kAlone, "shared memory");
constexpr uint32_t kPairSf = 256, kPairSfCols = 24;        // a stage's scales in TMEM: x's 8, w's 16
static_assert(kPairSf + kPairStages * kPairSfCols <= 512, "TMEM");

__device__ __forceinline__ float relu_nan(float x) {   // max(x, 0), NaN stays
  float r;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(x));
  return r;
}

// Bias (32 values in shared memory, or null) and ReLU on a row's 32 consecutive sums.
__device__ __forceinline__ void activate(const LinearArgs& a, const float* bias, uint32_t (&s)[32],
                                         float (&v)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(s[i]);
  if (bias) {
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      const float4 b = *reinterpret_cast<const float4*>(bias + i);
      v[i] += b.x; v[i + 1] += b.y; v[i + 2] += b.z; v[i + 3] += b.w;
    }
  }
  if (a.relu) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = relu_nan(v[i]);
  }
}

// 16-byte piece c of a lane's row in a staged tile of rows of kRow bytes, swizzled as
// the output's tensor map says (128: by row mod 8, 64: by row / 2 mod 4): eight lanes
// write eight different bank groups.
template <int kRow>
__device__ __forceinline__ uint4* staged_at(uint8_t* tile, int lane, int c) {
  const int sw = kRow == 128 ? lane & 7 : (lane >> 1) & 3;
  return reinterpret_cast<uint4*>(tile + lane * kRow + ((c ^ sw) << 4));
}

// A warp's 32 rows x 128 (32 chunks) features of one tile to y by bulk stores from its staged tile
// (4 KB): a store instruction of 32 rows takes the load/store unit about 64 clocks
// whatever its width, a bulk store none.  Where y's rows are not 16-byte aligned, and
// where the last features of a row are no whole 16 bytes (the bulk store's pieces), the
// warp stores the tile row by row.  kOut: AGN_PREC_*.
template <int kOut>
__device__ __forceinline__ void store_rows(const LinearArgs& a, const CUtensorMap* tmY, uint8_t* tile,
                                           const float* bias, int64_t r0, int64_t f0, int chunks,
                                           int lane, uint32_t (&s)[4][32]) {
  auto reuse = [&] {   // the bulk stores have read the tile
    if (lane == 0) tc::bulk_wait_read();
    __syncwarp();
  };
  auto send = [&](int x) {
    tc::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      tc::tma_store_2d(tmY, tile, x, (int)r0);
      tc::bulk_commit();
    }
  };
  // a tile of kW features from f on, by a bulk store or row by row
  using T = typename std::conditional<kOut == AGN_PREC_BF16, bf16, float>::type;
  constexpr int kW = 128 / (int)sizeof(T);
  auto put = [&](int64_t f) {
    if (a.bulk_out == a.out || f + kW <= a.bulk_out) return send((int)f);
    __syncwarp();
    const int n = (int)min((int64_t)32, a.rows - r0);
#pragma unroll
    for (int e = 0; e < kW; e += 32) {
      const int i = e + lane;   // this lane's feature
      if (f + i >= a.out) break;
      T* p = static_cast<T*>(a.y) + r0 * a.ldy + f + i;
      for (int row = 0; row < n; ++row, p += a.ldy)
        AGN_ST(p, *reinterpret_cast<const T*>(tile + row * 128 + (((i * (int)sizeof(T) >> 4) ^ (row & 7)) << 4) +
                                              (i * (int)sizeof(T) & 15)));
    }
  };
  if (kOut == AGN_PREC_MX4) {
    uint32_t word = 0;
    reuse();
#pragma unroll
    for (int c = 0; c < 4; ++c) {   // a block each
      float v[32];
      activate(a, bias ? bias + 32 * c : nullptr, s[c], v);
      uint32_t amax = 0;
      const int n = (int)max((int64_t)0, min((int64_t)32, a.out - f0 - 32 * c));   // (warp-uniform)
      if (n < 32) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (i >= n) v[i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);
      const uint32_t code = mx_scale_code(amax);
      const float inv = mx_inverse(code);
      uint32_t q[4] = {0, 0, 0, 0};
      if (code != 255) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float u[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) u[j] = v[8 * i + j] * inv;
          q[i] = mx_pack8(u);
        }
      }
      word |= code << (8 * c);
      *staged_at<64>(tile, lane, c) = make_uint4(q[0], q[1], q[2], q[3]);
    }
    send((int)(f0 / 2));
    if (r0 + lane < a.rows)
      AGN_ST(reinterpret_cast<uint32_t*>(a.y_scales + mx_scale_at(r0 + lane, f0 / kMxBlock, a.y_tiles_k)),
             word);
  } else if (kOut == AGN_PREC_BF16) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {   // 64 features: 128 bytes of a row
      if (2 * p >= chunks || f0 + 64 * p >= a.out) break;
      reuse();
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float v[32];
        activate(a, bias ? bias + 64 * p + 32 * c : nullptr, s[2 * p + c], v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float* u = v + 8 * j;
          const __nv_bfloat162 o[4] = {__floats2bfloat162_rn(u[0], u[1]), __floats2bfloat162_rn(u[2], u[3]),
                                       __floats2bfloat162_rn(u[4], u[5]), __floats2bfloat162_rn(u[6], u[7])};
          *staged_at<128>(tile, lane, 4 * c + j) = *reinterpret_cast<const uint4*>(o);
        }
      }
      put(f0 + 64 * p);
    }
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c) {   // 32 features
      if (c >= chunks || f0 + 32 * c >= a.out) break;
      float v[32];
      activate(a, bias ? bias + 32 * c : nullptr, s[c], v);
      reuse();
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *staged_at<128>(tile, lane, j) =
            make_uint4(__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]),
                       __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3]));
      put(f0 + 32 * c);
    }
  }
}

// Unit u of the work: a tile, or (from tile n_whole on) half of one, 128 of its features, so
// that a last round of few tiles occupies twice the pairs for half the time.
struct PairUnit {
  int f, n;      // first feature, first row
  bool narrow;   // 128 features
  __device__ __forceinline__ PairUnit(int u, int tiles_f, int n_whole) {
    narrow = u >= n_whole;
    const int t = narrow ? n_whole + (u - n_whole) / 2 : u;
    f = (t % tiles_f) * 256 + (narrow ? ((u - n_whole) & 1) * 128 : 0);
    n = (t / tiles_f) * 256;
  }
};

// A role that gives up says so in both CTAs: whatever it leaves out, the other's would wait for.
__device__ __forceinline__ void give_up(volatile int* abort_flag) {
#pragma unroll
  for (uint32_t r = 0; r < 2; ++r)
    asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(
                     tc::map_cluster(const_cast<int*>(abort_flag), r)), "r"(1)
                 : "memory");
}

// Stages, from the launch's first, that a CTA's loading thread armed and whose scales each of its
// scale warps brought to TMEM (far from 2^31: operands that fill the memory make 10^8).
struct PairStages {
  int loaded, scaled[4];
};
__device__ __forceinline__ int ld_cluster_int(const int* p, uint32_t rank) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(tc::map_cluster(p, rank)) : "memory");
  return v;
}

// After a role gave up and all have ended (one thread of each CTA): wait for the copies of the last
// stages, each CTA's scales on its own barriers and both CTAs' codes on the first's, where what
// will not come any more (the loads of the CTA that armed fewer stages, the arrivals of scale warps)
// is made up for: a stage's phase then ends when its copies have landed.
__device__ __forceinline__ void land(uint64_t* full, uint64_t* scales_in, const PairStages* done, int cta) {
  const int n0 = done->loaded, n1 = cta == 0 ? ld_cluster_int(&done->loaded, 1) : 0, n = max(n0, n1);
#pragma unroll 1
  for (int i = max(0, n - kPairStages); i < n; ++i) {
    const uint32_t s = (uint32_t)i % kPairStages, parity = (uint32_t)i / kPairStages & 1;
    if (i < n0) tc::mbar_wait_bounded(&scales_in[s], parity, kWaitNs);
    if (cta != 0) continue;
    if (i >= n0) tc::mbar_arrive_expect_tx(&full[s], 2 * kPairHalf);   // (the second CTA's codes alone)
    else if (i >= n1) tc::mbar_complete_tx(&full[s], 2 * kPairHalf);
#pragma unroll 1
    for (uint32_t w = 0; w < 8; ++w)
      if (i >= ld_cluster_int(&done->scaled[w & 3], w >> 2)) tc::mbar_arrive(&full[s]);
    tc::mbar_wait_bounded(&full[s], parity, kWaitNs);
  }
}

template <int kOut>
__global__ void __launch_bounds__(kPairThreads, 1)
mx4_linear_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX,
                       const __grid_constant__ CUtensorMap tmWs,
                       const __grid_constant__ CUtensorMap tmXs,
                       const __grid_constant__ CUtensorMap tmY, const LinearArgs a, int tiles_f,
                       int n_whole, int units) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  uint8_t* staged = smem + kPairStages * kPairStage;                           // [finishing warp][4 KB]
  float* biases = reinterpret_cast<float*>(staged + 8 * kPairStaged);          // [finishing warp][128]
  // first CTA's: both CTAs' codes in shared memory and scales in TMEM
  uint64_t* full = reinterpret_cast<uint64_t*>(biases + 8 * 128);
  uint64_t* empty = full + kPairStages;
  uint64_t* scales_in = empty + kPairStages;        // this CTA's scales in shared memory
  uint64_t* sums_full = scales_in + kPairStages;
  uint64_t* sums_empty = sums_full + 1;             // (first CTA's)
  uint64_t* drained = sums_empty + 1;
  PairStages* stages_done = reinterpret_cast<PairStages*>(drained + 1);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(stages_done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = (int)cluster_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int KT = (a.k_steps + 3) / 4;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kPairStages; ++s) {
      tc::mbar_init(&full[s], 1 + 8);    // the loads, and four scale warps of each CTA
      tc::mbar_init(&empty[s], 1);
      tc::mbar_init(&scales_in[s], 1);
    }
    tc::mbar_init(sums_full, 1);
    tc::mbar_init(sums_empty, 16);       // the finishing warps of both CTAs
    tc::mbar_init(drained, 1);
    *abort_flag = 0;
    tc::fence_mbar_init();
    tc::tma_prefetch_desc(&tmW);
    tc::tma_prefetch_desc(&tmX);
    tc::tma_prefetch_desc(&tmWs);
    tc::tma_prefetch_desc(&tmXs);
  }
  if (warp == 5) {
    tc::tmem_alloc_pair(tmem_holder, 512);
    tc::tmem_relinquish_pair();
  }
  tc::tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  pdl_begin();

  // The finishing warps hold 128 sums a thread: 2 x 128 threads x (48 + 208) registers
  // are the launch's 512 x 128.
  if (warp >= 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int q = warp & 3, half = (warp - 8) >> 2;
    const uint32_t empty_at = tc::map_cluster(sums_empty, 0);
    float* bias = biases + 128 * (warp - 8);
    uint8_t* tile = staged + (warp - 8) * kPairStaged;
    bool ok = true;
    int done = 0;
    for (int t = pair; t < units; t += pairs, ++done) {
      const PairUnit unit(t, tiles_f, n_whole);
      const int chunks = unit.narrow ? 2 : 4;   // of 32 features
      const int64_t f0 = unit.f + 32 * chunks * half;
      const int64_t r0 = (int64_t)unit.n + 128 * cta + 32 * q;
      if (a.bias) {   // (on its way while the sums are)
        float b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          b[i] = f0 + lane + 32 * i < a.out ? AGN_LD(a.bias + f0 + lane + 32 * i) : 0.f;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[lane + 32 * i] = b[i];
        __syncwarp();
      }
      ok = ok && wait_mbar<true>(sums_full, done & 1, abort_flag, a.wait_ns) && !*abort_flag;
      ok = __all_sync(0xffffffffu, ok);
      tc::tc_fence_after();
      if (!ok && lane == 0) {
        give_up(abort_flag);
        if (a.err) atomicExch(a.err, 1);
      }
      uint32_t v[4][32];
      if (ok) {
        const uint32_t col = tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)(32 * chunks * half);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (c < chunks) tc::tmem_ld_32x32b_x32(col + 32 * c, v[c]);
        tc::tmem_ld_wait();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive_relaxed(empty_at);
      } else {
#pragma unroll
        for (int i = 0; i < 128; ++i) v[i / 32][i % 32] = 0x7fc00000u;
      }
      if (f0 < a.out && r0 < a.rows) {   // (warp-uniform)
        const float* b = a.bias ? bias : nullptr;
        store_rows<kOut>(a, &tmY, tile, b, r0, f0, chunks, lane, v);
      }
    }
    if (lane == 0) tc::bulk_wait();   // the last stores are done before the kernel is
  } else if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    // a stage's scales: lane l holds words j (rows 32 j + l) of every tile; the
    // stage was loaded again only after the MMAs that read its TMEM columns
    const uint32_t quadrant = (uint32_t)(32 * warp) << 16;
    const uint32_t full0 = tc::map_cluster(full, 0);
    int s = 0;
    uint32_t phase = 0;
    bool ok = true;
    int t = pair, kt = 0;
    for (; t < units; t += pairs) {
      for (kt = 0; kt < KT; ++kt) {
        ok = __all_sync(0xffffffffu, wait_mbar<false>(&scales_in[s], phase, abort_flag, a.wait_ns));
        if (!ok) break;
        const uint4* src = reinterpret_cast<const uint4*>(smem + s * kPairStage + 2 * kPairHalf) + lane;
        uint32_t x[8], w[16];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const uint4 v = src[32 * q];
          x[4 * q] = v.x; x[4 * q + 1] = v.y; x[4 * q + 2] = v.z; x[4 * q + 3] = v.w;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 u = src[64 * (1 + h) + 32 * q];
            w[8 * q + 4 * h] = u.x; w[8 * q + 4 * h + 1] = u.y;
            w[8 * q + 4 * h + 2] = u.z; w[8 * q + 4 * h + 3] = u.w;
          }
        }
        const uint32_t col = tmem + quadrant + kPairSf + (uint32_t)s * kPairSfCols;
        tc::tmem_st_32x32b_x8(col, x);
        tc::tmem_st_32x32b_x16(col + 8, w);
        tc::tmem_st_wait();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive_relaxed(full0 + 8u * (uint32_t)s);
        if (++s == kPairStages) s = 0, phase ^= 1;
      }
      if (!ok) break;
    }
    if (lane == 0) {
      stages_done->scaled[warp] = (t - pair) / pairs * KT + (ok ? 0 : kt);
      if (!ok) give_up(abort_flag);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 4 && lane == 0) {
      const uint32_t full0 = tc::map_cluster(full, 0);
      int s = 0;
      int loaded = 0;
      const int stop = a.withhold == cta + 1 ? KT - 1 : INT32_MAX;
      uint32_t phase = 1;   // (the first round finds every stage free)
      for (int t = pair; t < units && loaded < stop && !*abort_flag; t += pairs) {
        const PairUnit unit(t, tiles_f, n_whole);
        const int f = unit.f, n = unit.n + 128 * cta, fb = f + (unit.narrow ? 64 : 128) * cta;
        for (int kt = 0; kt < KT && loaded < stop; ++kt) {
          if (!wait_mbar<false>(&empty[s], phase, abort_flag, a.wait_ns)) {
            give_up(abort_flag);
            break;
          }
          uint8_t* st = smem + s * kPairStage;
          const uint32_t bar = full0 + 8u * (uint32_t)s;
          tc::mbar_arrive_expect_tx(&scales_in[s], 3 * kSfBytes);
          tc::tma_load_3d(st + 2 * kPairHalf, &tmXs, &scales_in[s], 0, 2 * kt, n >> 7);
          tc::tma_load_3d(st + 2 * kPairHalf + kSfBytes, &tmWs, &scales_in[s], 0, 2 * kt, f >> 7);
          if (cta == 0) tc::mbar_arrive_expect_tx(&full[s], 4 * kPairHalf);
          tc::tma_load_2d_pair(st, &tmX, bar, kt * 128, n);
          tc::tma_load_2d_pair(st + kPairHalf, &tmW, bar, kt * 128, fb);
          ++loaded;
          if (++s == kPairStages) s = 0, phase ^= 1;
        }
      }
      stages_done->loaded = loaded;
    } else if (warp == 5 && lane == 0 && cta == 0) {
      // An MMA is issued in about the time that it takes, and few wait in line: what this
      // thread does between them is tensor time lost unless it is short.  So: one barrier
      // a stage, asked for the next stage between this stage's MMAs, descriptors by addition
      // or constant, whole stages without a test (clocks a stage: 836 with two barriers
      // waited on in turn and the descriptors made anew, 646 with tests of the last stage's
      // length, now 588-603 from stage to stage; 513 for the MMAs alone; by the whole warp, one lane issuing, 650).
      const uint64_t da0 = tc::smem_desc_sw128(tc::smem_u32(smem), 16, 1024);
      constexpr uint64_t kToB = kPairHalf >> 4;
      uint64_t da = da0;
      uint32_t sf = tmem + kPairSf;
      int s = 0, done = 0;
      uint32_t phase = 0;
      bool ready = false;
      for (int t = pair; t < units; t += pairs, ++done) {
        if (done > 0 && !wait_mbar<true>(sums_empty, (done - 1) & 1, abort_flag, a.wait_ns)) {
          give_up(abort_flag);   // (the sums of the tile before may still be read)
          break;
        }
        // (N a constant: the instruction descriptor is then one too)
        auto mainloop = [&](auto columns) {
          constexpr uint32_t id0 = tc::idesc_mxf4(256, decltype(columns)::value, 0);
          constexpr uint32_t id2 = tc::idesc_mxf4(256, decltype(columns)::value, 2);
          uint32_t acc = 0;   // the tile's first MMA overwrites
          auto next = [&] {
            da += kPairStage >> 4;
            sf += kPairSfCols;
            if (++s == kPairStages) s = 0, phase ^= 1, da = da0, sf = tmem + kPairSf;
            ready = tc::mbar_test_wait(&full[s], phase);
            acc = 1;
          };
          int left = a.k_steps;
          for (; left >= 4; left -= 4) {   // whole stages
            if (!ready && !wait_mbar<false>(&full[s], phase, abort_flag, a.wait_ns)) {
              give_up(abort_flag);
              return;
            }
            tc::tc_fence_after();
            tc::mma_mxf4_pair(tmem, da, da + kToB, id0, sf, sf + 8, acc);
            tc::mma_mxf4_pair(tmem, da + 2, da + kToB + 2, id2, sf, sf + 8, 1);
            tc::mma_mxf4_pair(tmem, da + 4, da + kToB + 4, id0, sf + 4, sf + 16, 1);
            uint64_t* const mine = &empty[s];
            const uint64_t d = da + 6;
            const uint32_t f = sf;
            next();
            tc::mma_mxf4_pair(tmem, d, d + kToB, id2, f + 4, f + 16, 1);
            tc::mma_commit_pair(mine);
          }
          if (left > 0) {
            if (!ready && !wait_mbar<false>(&full[s], phase, abort_flag, a.wait_ns)) {
              give_up(abort_flag);
              return;
            }
            tc::tc_fence_after();
            tc::mma_mxf4_pair(tmem, da, da + kToB, id0, sf, sf + 8, acc);
            if (left > 1) tc::mma_mxf4_pair(tmem, da + 2, da + kToB + 2, id2, sf, sf + 8, 1);
            if (left > 2) tc::mma_mxf4_pair(tmem, da + 4, da + kToB + 4, id0, sf + 4, sf + 16, 1);
            tc::mma_commit_pair(&empty[s]);
            next();
          }
        };
        if (t >= n_whole) mainloop(std::integral_constant<int, 128>());
        else mainloop(std::integral_constant<int, 256>());
        if (*abort_flag) break;   // no sums: the finishing warps of both CTAs give up
        tc::mma_commit_pair(sums_full);
      }
    }
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  cluster_sync();   // no CTA leaves while the other reads its memory or signals its barriers
  if (__builtin_expect(*abort_flag, 0)) {   // (the same in both CTAs: nobody is left who could set it)
    if (warp == 5 && lane == 0) {
      if (cta == 0) tc::mma_commit_pair(drained);   // (the thread that issued the MMAs)
      tc::mbar_wait_bounded(drained, 0, kWaitNs);
      land(full, scales_in, stages_done, cta);
    }
    cluster_sync();
  }
  if (warp == 5) tc::tmem_dealloc_pair(tmem, 512);
}

template <int kOut>
Status launch_pair(const Mx4LinearArgs& m, const LinearArgs& a, int dev, cudaStream_t st) {
  CUtensorMap tw, tx, tws, txs, ty{};
  const int64_t rb = mx_row_bytes(m.in);
  AGN_TRY(make_tmap_u8_2d(&tw, m.w_codes, rb, m.out, rb, 128));
  AGN_TRY(make_tmap_u8_2d(&tx, m.x_codes, rb, m.rows, rb, 128));
  // the scales: words of a tile, tiles along K, tiles of rows
  AGN_TRY(make_tmap_u32_3d(&tws, m.w_scales, kMxTileBytes / 4, a.tiles_k,
                           ceil_div(m.out, kMxTileRows), 2, 2));
  AGN_TRY(make_tmap_u32_3d(&txs, m.x_scales, kMxTileBytes / 4, a.tiles_k, a.row_tiles, 2, 1));
  if (kOut == AGN_PREC_MX4)
    AGN_TRY(make_tmap_store_2d(&ty, m.y, 1, mx_row_bytes(m.out), m.rows, mx_row_bytes(m.out), 64, 32));
  else if (a.bulk_out > 0)
    AGN_TRY(make_tmap_store_2d(&ty, m.y, (int)dtype_size(kOut), a.bulk_out, m.rows, m.ldy,
                               128 / (int)dtype_size(kOut), 32));
  auto kern = mx4_linear_pair_kernel<kOut>;
  AGN_TRY_CUDA((allow_smem<std::integral_constant<int, kOut>>(kern, kPairSmem, dev)));
  const int64_t tiles_f = ceil_div(m.out, 256), tiles = tiles_f * ceil_div(m.rows, 256);
  // the last round in halves where they fit (4-bit outputs: a warp's scales are whole words)
  int sms = 0;
  AGN_TRY(device_sms(dev, &sms));
  const int64_t most = std::max(1, sms / 2), rest = tiles % most;
  const int64_t halves = kOut != AGN_PREC_MX4 && 2 * rest <= most ? rest : 0;
  const int64_t units = tiles + halves, pairs = std::min(units, most);
  AGN_TRY_CUDA(launch_pdl_cluster(kern, dim3((unsigned)(2 * pairs)), kPairThreads, kPairSmem,
                                  dim3(2, 1, 1), st, tw, tx, tws, txs, ty, a, (int)tiles_f,
                                  (int)(tiles - halves), (int)units));
  return Status::Ok();
}

}  // namespace

Status mx4_linear(const Mx4LinearArgs& m, cudaStream_t st) {
  LinearArgs a{};
  a.w_scales = static_cast<const uint8_t*>(m.w_scales);
  a.x_scales = static_cast<const uint8_t*>(m.x_scales);
  a.rows = m.rows; a.out = m.out;
  a.tiles_k = mx_tiles_k(m.in);
  a.row_tiles = ceil_div(m.rows, kMxTileRows);
  a.k_steps = (int)ceil_div(m.in, 64);
  a.bias = m.bias;
  a.relu = m.relu != 0; a.dtype = m.dtype;
  a.y = m.y; a.ldy = m.ldy;
  a.y_scales = static_cast<uint8_t*>(m.y_scales);
  a.y_tiles_k = mx_tiles_k(m.out);
  a.err = m.err;
  a.wait_ns = m.wait_ns ? m.wait_ns : kWaitNs;
  a.withhold = m.withhold;
  const uint64_t rows_at = reinterpret_cast<uintptr_t>(m.y) | (uint64_t)m.ldy * dtype_size(m.dtype);
  a.vec = m.dtype != AGN_PREC_MX4 && rows_at % 16 == 0;
  a.bulk_out = m.dtype == AGN_PREC_MX4 ? m.out
               : a.vec                 ? m.out / (16 / (int64_t)dtype_size(m.dtype)) * (16 / (int64_t)dtype_size(m.dtype))
                                       : 0;
  int dev = 0, fours = 0;
  AGN_TRY(current_device(&dev));
  // One tile of rows while it holds them all.  More: tiles of 64 rows while K can be split
  // over four CTAs for each, pairs of CTAs from 257 rows, or from 129 with 64 tiles of 128 x
  // 128, else tiles of 128.  us with 64, 128, pairs: 200 rows of 1000 to 1000 5.3, 6.1, 6.4; 1024
  // of 784 to 128 5.2, 6.4, 6.5; 128 of 4096 to 4096 8.9, 8.0, 9.8; 200 of 4096 to 4096 10.9, 10.5,
  // 9.8; 300 of 4096 to 4096 20.1, 12.3, 10.2.
  if (m.rows <= 16) return launch_linear<16>(m, a, dev, st);
  if (m.rows <= 32) return launch_linear<32>(m, a, dev, st);
  const int64_t tiles_f = ceil_div(m.out, 128);
  if (m.rows <= 64) return launch_linear<64>(m, a, dev, st);
  AGN_TRY(max_clusters<Tile<64>>(mx4_linear_kernel<64>, kThreads, Tile<64>::kSmem, 4, dev, &fours));
  if (tiles_f * ceil_div(m.rows, 64) <= fours) return launch_linear<64>(m, a, dev, st);
  if (m.rows <= 128 || (m.rows <= 256 && 2 * tiles_f < 64)) return launch_linear<128>(m, a, dev, st);
  return m.dtype == AGN_PREC_FP32   ? launch_pair<AGN_PREC_FP32>(m, a, dev, st)
         : m.dtype == AGN_PREC_BF16 ? launch_pair<AGN_PREC_BF16>(m, a, dev, st)
                                    : launch_pair<AGN_PREC_MX4>(m, a, dev, st);
}

namespace {

// agn_debug_linear_waits: of the calling thread's calls
thread_local uint64_t t_wait_ns = 0;
thread_local int t_withhold = 0;

Status linear_call(const Mx4LinearArgs& m, cudaStream_t st) {
  const bool mx = m.dtype == AGN_PREC_MX4;
  const size_t es = mx ? 1 : dtype_size(m.dtype);
  constexpr int64_t kMost = INT32_MAX - 256;
  if (!es) return Status::Err(AGN_E_INVALID, "unknown dtype");
  // (a tile's sums take about 0.5 us for 256 k: far from the waits' limit at 2^28)
  if (m.rows < 0 || m.in < 1 || m.out < 1 || m.rows > kMost || m.in > 1 << 28 || m.out > kMost)
    return Status::Err(AGN_E_INVALID,
                       "need rows >= 0 and out >= 1, below 2^31 - 256, and 1 <= in <= 2^28");
  if (!mx) AGN_TRY(check_matrix("y", m.rows, m.out, m.ldy));
  if (m.rows == 0) return Status::Ok();
  if (!m.x_codes || !m.x_scales || !m.w_codes || !m.w_scales || !m.y || (mx && !m.y_scales))
    return Status::Err(AGN_E_INVALID, "null pointer");
  const CallBuffer xc{"x codes", m.x_codes, (size_t)mx_code_bytes(m.rows, m.in), 16},
      xs{"x scales", m.x_scales, (size_t)mx_scale_bytes(m.rows, m.in), 16},
      wc{"w codes", m.w_codes, (size_t)mx_code_bytes(m.out, m.in), 16},
      ws{"w scales", m.w_scales, (size_t)mx_scale_bytes(m.out, m.in), 16},
      bb{"bias", m.bias, m.bias ? (size_t)m.out * 4 : 0, 4},
      y{"y", m.y, mx ? (size_t)mx_code_bytes(m.rows, m.out) : matrix_bytes(m.rows, m.out, m.ldy, es),
        mx ? 16 : es},
      ys{"y scales", mx ? m.y_scales : nullptr, mx ? (size_t)mx_scale_bytes(m.rows, m.out) : 0, 16},
      er{"err", m.err, m.err ? sizeof(int) : 0, 4};
  AGN_TRY(check_apart(y, {xc, xs, wc, ws, bb, ys, er}));
  AGN_TRY(check_apart(ys, {xc, xs, wc, ws, bb, er}));
  AGN_TRY(check_apart(er, {xc, xs, wc, ws, bb}));
  AGN_TRY(check_buffers({xc, xs, wc, ws, bb, y, ys, er}));
  KnownBuffers known({xc, xs, wc, ws, bb, y, ys, er});
  AGN_TRY(bounds_upload(st));
  AGN_TRY(mx4_linear(m, st));
  return bounds_collect(st);
}

}  // namespace

AGN_BOUNDS_UNIT(mx4_linear)

}  // namespace agn

extern "C" int agn_mx4_linear(const void* x_codes, const void* x_scales, const void* w_codes,
                              const void* w_scales, const float* bias, int64_t rows, int64_t in,
                              int64_t out, int32_t relu, void* y, int32_t dtype, int64_t ldy,
                              void* y_scales, int32_t* err, void* stream) {
  return agn::guarded([&] {
    agn::Mx4LinearArgs m{};
    m.x_codes = x_codes; m.x_scales = x_scales;
    m.w_codes = w_codes; m.w_scales = w_scales;
    m.bias = bias;
    m.rows = rows; m.in = in; m.out = out;
    m.relu = relu;
    m.y = y; m.dtype = dtype; m.ldy = ldy; m.y_scales = y_scales;
    m.err = err;
    m.wait_ns = agn::t_wait_ns;
    m.withhold = agn::t_withhold;
    return agn::linear_call(m, static_cast<cudaStream_t>(stream));
  });
}

extern "C" int agn_debug_linear_waits(int64_t wait_ns, int32_t withhold_rank) {
  return agn::guarded([&] {
    if (wait_ns < 0 || wait_ns > 2000000000ll || withhold_rank < -1 || withhold_rank > 65534)
      return agn::Status::Err(AGN_E_INVALID, "wait_ns must be in [0, 2e9], withhold_rank >= -1");
    agn::t_wait_ns = (uint64_t)wait_ns;
    agn::t_withhold = withhold_rank + 1;
    return agn::Status::Ok();
  });
}
