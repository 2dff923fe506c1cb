// Products of the output layer's loss for fp32 and up to 128 rows that read w once, as it is:
//   z^T = w x^T (w's rows along M) and dx^T = w^T p^T (w's columns along M: MN-major), fp32 sums of ranges along K
// to [split][row][column of w's side], which leave transposed.  With one tile of rows a tile of w is of use once, so
// making its three bf16 pieces in memory first (2.5 times its bytes) would be most of the work.  Here
// eight warps load a tile of 128 x 64 elements, one or two steps ahead in registers, and write its pieces to
// shared memory as the MMAs read them; four take the sums out of TMEM.  x's (p's) pieces come by TMA, those of
// 64 rows under one another, so that one MMA multiplies a piece of w by all three of them (N = 192): w0 by
// (x0 x1 x2), w1 by (x0 x1), w2 by x0, three reads of w's pieces where six products would make six.  Three
// accumulators, largest products first; sums over 256 or 512 k are added in registers (linear_ce_gemm.cu).
// Bound by w's bytes and shared memory together: a step's 32 KB come in 1370 clocks of an SM's share of the memory,
// shared memory moves 168 KB for it (264 KB with more than 64 rows).  56 rows, 2392 to 55366: 117 us, w at 4.5 TB/s; 128
// rows, 4096 to 32000: 164 us, 3.2 TB/s.  Loads a step further ahead gained nothing; with eight warps
// that both made pieces and took sums it was 160 and 194.
// Every wait is bounded as in linear_ce_gemm.cu.
#include "linear_ce.cuh"
#include "ops.cuh"
#include "tc_ptx.cuh"

namespace agn {
namespace ce {

namespace {

constexpr int kThreads = 512;
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr int kStages = 2;
constexpr uint32_t kPlane = 128 * 128;       // a piece of a tile of w
constexpr uint32_t kBox = 64 * 128;          // 64 rows of 64 elements
constexpr int kStaged = 4096;                // a finishing warp's 32 x 32 outputs

template <int kGroups>
struct Shape {   // kGroups: of 64 rows of x
  static constexpr uint32_t stage = 3 * kPlane + kGroups * 3 * kBox;
  static constexpr size_t smem = 1024 + kStages * stage + 4 * kStaged + 256;
  static constexpr int sets = kGroups == 1 ? 2 : 1;      // sums in TMEM: 192 columns a group
  static constexpr int sum_k = kGroups == 1 ? 4 : 8;     // steps of a sum
  static constexpr int depth = kGroups == 1 ? 2 : 1;     // steps that loads are ahead
};

__device__ __forceinline__ uint32_t bits(__nv_bfloat162 v) { return *reinterpret_cast<const uint32_t*>(&v); }

// Two values' pieces, one word each (split3 of both).
__device__ __forceinline__ void pieces2(float x, float y, uint32_t (&w)[3]) {
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    w[k] = bits(__floats2bfloat162_rn(x, y));
    x = __fsub_rn(x, __uint_as_float(w[k] << 16));
    y = __fsub_rn(y, __uint_as_float(w[k] & 0xffff0000u));
  }
}

template <bool kMn, int kGroups>
__global__ void __launch_bounds__(kThreads, 1) ce_raw_kernel(const __grid_constant__ RawLaunch launch) {
  using S = Shape<kGroups>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* staged = ring + kStages * S::stage;
  uint64_t* full = reinterpret_cast<uint64_t*>(staged + 4 * kStaged);   // x's pieces
  uint64_t* made = full + kStages;                                      // w's pieces
  uint64_t* empty = made + kStages;
  uint64_t* acc_full = empty + kStages;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* drained = acc_empty + 2;
  int* loaded_out = reinterpret_cast<int*>(drained + 1);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(loaded_out + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  const RawArgs& a = launch.args;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t wait_ns = a.wait_ns;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(&full[s], 1);
      tc::mbar_init(&made[s], 8);
      tc::mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      tc::mbar_init(&acc_full[b], 1);
      tc::mbar_init(&acc_empty[b], 4);
    }
    tc::mbar_init(drained, 1);
    *loaded_out = 0;
    *abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (warp == 2) {
    tc::tmem_alloc(tmem_holder, 512);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  pdl_begin();

  const int KT = (a.K + 63) / 64, per = (KT + a.splits - 1) / a.splits;
  const int units = (a.M + 127) / 128 * a.splits;
  // Unit u: a tile and a range of steps (never none).
  struct Unit {
    int m, split, kt0, kt;
  };
  auto unit_of = [&](int u) {
    Unit t;
    t.split = u % a.splits;
    t.m = u / a.splits * 128;
    t.kt0 = t.split * per;
    t.kt = min(KT, t.kt0 + per) - t.kt0;
    return t;
  };

  // (128 threads of each kind: the registers are the launch's 512 x 128)
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0 && lane == 0) {
      int s = 0, loaded = 0, stop = INT32_MAX;
      uint32_t phase = 1;   // (the first round finds every stage free)
      bool ok = true;
      for (int u = blockIdx.x; ok && u < units; u += gridDim.x) {
        const Unit t = unit_of(u);
        if (a.withhold == 1) stop = t.kt - 1;
        for (int kt = t.kt0; ok && kt < t.kt0 + t.kt; ++kt) {
          ok = loaded < stop;
          if (!ok) break;
          ok = tc::wait_mbar<false>(&empty[s], phase, abort_flag, wait_ns);
          if (!ok) {
            *abort_flag = 1;
            break;
          }
          uint8_t* to = ring + s * S::stage + 3 * kPlane;
          tc::mbar_arrive_expect_tx(&full[s], kGroups * 3 * kBox);
#pragma unroll
          for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int z = 0; z < 3; ++z)
              tc::tma_load_3d(to + (3 * g + z) * kBox, &launch.b, &full[s], kt * 64, 64 * g, z);
          ++loaded;
          if (++s == kStages) s = 0, phase ^= 1;
        }
      }
      *loaded_out = loaded;
    } else if (warp == 1 && lane == 0) {
      const uint32_t r0 = tc::smem_u32(ring);
      const uint64_t da0 = tc::smem_desc_sw128(r0, kMn ? kBox : 16, 1024);
      const uint64_t db0 = tc::smem_desc_sw128(r0 + 3 * kPlane, 16, 1024);
      constexpr uint64_t ka = (kMn ? 2048 : 32) >> 4, kb = 32 >> 4;   // 16 k
      int s = 0, done = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int u = blockIdx.x; ok && u < units; u += gridDim.x) {
        const int steps = unit_of(u).kt;
        for (int kt = 0; ok && kt < steps;) {   // a sum
          const int buf = done % S::sets, round = done / S::sets;
          if (round > 0) ok = tc::wait_mbar<true>(&acc_empty[buf], (round - 1) & 1, abort_flag, wait_ns);
          tc::tc_fence_after();
          const int end = min(steps, kt + S::sum_k);
          for (bool first = true; ok && kt < end; ++kt, first = false) {
            ok = tc::wait_mbar<false>(&full[s], phase, abort_flag, wait_ns) &&
                 tc::wait_mbar<false>(&made[s], phase, abort_flag, wait_ns);
            if (!ok) break;
            tc::tc_fence_after();
            const uint64_t da = da0 + (uint64_t)(s * (S::stage >> 4)), db = db0 + (uint64_t)(s * (S::stage >> 4));
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
              for (int g = 0; g < kGroups; ++g) {
                const uint32_t d = tmem + buf * 256 + g * 192;
                const uint64_t b = db + g * (3 * kBox >> 4) + kk * kb;
#pragma unroll
                for (int p = 0; p < 3; ++p)
                  tc::mma_bf16(d + 64 * p, da + p * (kPlane >> 4) + kk * ka, b,
                               tc::idesc_bf16_f32(128, 64 * (3 - p), kMn, false), p > 0 || kk > 0 || !first);
              }
            tc::mma_commit(&empty[s]);
            if (++s == kStages) s = 0, phase ^= 1;
          }
          if (!ok) break;
          tc::mma_commit(&acc_full[buf]);
          ++done;
        }
      }
      if (!ok) *abort_flag = 1;
    }
  } else if (warp < 12) {
    if (kGroups == 1) asm volatile("setmaxnreg.inc.sync.aligned.u32 152;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    const int tid = threadIdx.x - 128;
    bool ok = true;
    // Elements of a step: 16 lanes a row of 64 (K-major), 32 a row of 128 (a box of 64 columns by 16 lanes).
    const int row = kMn ? tid >> 5 : tid >> 4, col = (kMn ? tid & 31 : tid & 15) * 4;
    constexpr int kRows = kMn ? 8 : 16;   // from one of a thread's eight rows to the next
    const uint32_t at0 = (col / 64) * kBox + row * 128 + (((col % 64 / 8) ^ (row & 7)) << 4) + (col / 4 % 2) * 8;
    const int rows_all = kMn ? a.K : a.M, cols_all = kMn ? a.M : a.K;
    const bool vec = a.vec;
    // The next step to load: its first row of this thread's and column, steps left of its unit
    const int64_t apart = (int64_t)kRows * a.ld;
    int load_u = blockIdx.x, load_left = 0, r0 = 0, c0 = 0;
    const float* src = nullptr;
    auto begin = [&] {
      if (load_u >= units) return;
      const Unit t = unit_of(load_u);
      load_left = t.kt;
      r0 = (kMn ? t.kt0 * 64 : t.m) + row;
      c0 = (kMn ? t.m : t.kt0 * 64) + col;
      src = a.w + (int64_t)r0 * a.ld + c0;
    };
    auto load = [&](float4 (&q)[8]) {
      if (load_left == 0) return;
      if (vec && c0 < cols_all && r0 + 7 * kRows < rows_all) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = AGN_LD(reinterpret_cast<const float4*>(src + i * apart));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            v[j] = r0 + i * kRows < rows_all && c0 + j < cols_all ? AGN_LD(src + i * apart + j) : 0.f;
          q[i] = make_float4(v[0], v[1], v[2], v[3]);
        }
      }
      (kMn ? r0 : c0) += 64;
      src += kMn ? 64 * a.ld : 64;
      if (--load_left == 0) {
        load_u += gridDim.x;
        begin();
      }
    };

    float4 q[S::depth][8];
    begin();
#pragma unroll
    for (int d = 0; d < S::depth; ++d) load(q[d]);
    int s = 0;
    uint32_t phase = 1;
    int left = 0;   // steps of this CTA
    for (int u = blockIdx.x; u < units; u += gridDim.x) left += unit_of(u).kt;
    while (left > 0) {
#pragma unroll
      for (int d = 0; d < S::depth; ++d) {
        if (left-- <= 0) break;
        ok = ok && tc::wait_mbar<false>(&empty[s], phase, abort_flag, wait_ns);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) {
          if (lane == 0) *abort_flag = 1;
          left = 0;
          break;
        }
        uint8_t* to = ring + s * S::stage + at0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t lo[3], hi[3];
          pieces2(q[d][i].x, q[d][i].y, lo);
          pieces2(q[d][i].z, q[d][i].w, hi);
#pragma unroll
          for (int p = 0; p < 3; ++p)
            *reinterpret_cast<uint2*>(to + p * kPlane + i * kRows * 128) = make_uint2(lo[p], hi[p]);
        }
        load(q[d]);
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&made[s]);
        if (++s == kStages) s = 0, phase ^= 1;
      }
    }
  } else {
    if (kGroups == 1) asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int quad = warp & 3;
    uint8_t* tile = staged + quad * kStaged;
    bool ok = true;
    int done = 0;
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
      const Unit t = unit_of(u);
      float sums[kGroups][64];
#pragma unroll
      for (int i = 0; i < 64 * kGroups; ++i) sums[i / 64][i % 64] = 0.f;
#pragma unroll 1
      for (int kt = 0; kt < t.kt; kt += S::sum_k) {
        const int buf = done % S::sets;
        ok = ok && tc::wait_mbar<true>(&acc_full[buf], (done / S::sets) & 1, abort_flag, wait_ns) && !*abort_flag;
        ok = __all_sync(0xffffffffu, ok);
        tc::tc_fence_after();
        if (!ok && lane == 0) {
          *abort_flag = 1;
          if (a.err) atomicExch(a.err, 1);
        }
        const uint32_t at = tmem + ((uint32_t)(32 * quad) << 16) + buf * 256;
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            // (the smaller products' sums first)
            float v[16];
#pragma unroll
            for (int p = 2; p >= 0; --p) {
              uint32_t r[16];
              if (ok) {
                tc::tmem_ld_32x32b_x16(at + g * 192 + 64 * p + 16 * h, r);
                tc::tmem_ld_wait();
              }
#pragma unroll
              for (int i = 0; i < 16; ++i)
                v[i] = !ok ? __uint_as_float(0x7fc00000u)   // (what could not be computed)
                           : p == 2 ? __uint_as_float(r[i]) : v[i] + __uint_as_float(r[i]);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) sums[g][16 * h + i] += v[i];
          }
        if (ok) {
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive_relaxed(tc::smem_u32(&acc_empty[buf]));
        }
        ++done;
      }
      if (t.m + 32 * quad >= a.M) continue;
#pragma unroll
      for (int j = 0; j < 2 * kGroups; ++j) {   // 32 of x's rows x 32 columns
        if (lane == 0) tc::bulk_wait_read();
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 32; ++i)
          *reinterpret_cast<float*>(tile + i * 128 + (((lane >> 2) ^ (i & 7)) << 4) + (lane & 3) * 4) =
              sums[j / 2][j % 2 * 32 + i];
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          tc::tma_store_2d(&launch.c, tile, t.m + 32 * quad, t.split * a.part_rows + 32 * j);
          tc::bulk_commit();
        }
      }
    }
    if (lane == 0) tc::bulk_wait();   // the last stores are done before the kernel is
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  if (__builtin_expect(*abort_flag, 0)) {   // copies in flight land before the CTA ends
    if (warp == 1 && lane == 0) {
      tc::mma_commit(drained);   // (the thread that issued the MMAs)
      tc::mbar_wait_bounded(drained, 0, kWaitNs);
      const int n = *loaded_out;
      for (int i = max(0, n - kStages); i < n; ++i)
        tc::mbar_wait_bounded(&full[i % kStages], (uint32_t)(i / kStages) & 1, kWaitNs);
    }
    __syncthreads();
  }
  if (warp == 2) tc::tmem_dealloc(tmem, 512);
}

template <bool kMn, int kGroups>
Status queue(const RawLaunch& l, cudaStream_t st) {
  struct Tag {};
  auto kern = ce_raw_kernel<kMn, kGroups>;
  int dev = 0, sms = 0;
  AGN_TRY(current_device(&dev));
  AGN_TRY(device_sms(dev, &sms));
  AGN_TRY_CUDA(allow_smem<Tag>(kern, Shape<kGroups>::smem, dev));
  const int64_t units = ceil_div(l.args.M, 128) * l.args.splits;
  AGN_TRY_CUDA(launch_pdl(kern, dim3((unsigned)std::min<int64_t>(units, sms)), dim3(kThreads), Shape<kGroups>::smem, st,
                          l));
  return Status::Ok();
}

}  // namespace

Status raw(const RawLaunch& launch, cudaStream_t st) {
  RawLaunch l = launch;
  if (!l.args.wait_ns) l.args.wait_ns = (uint32_t)kWaitNs;
  if (l.args.mn) return l.args.groups == 1 ? queue<true, 1>(l, st) : queue<true, 2>(l, st);
  return l.args.groups == 1 ? queue<false, 1>(l, st) : queue<false, 2>(l, st);
}

}  // namespace ce

AGN_BOUNDS_UNIT(linear_ce_raw)

}  // namespace agn
