// The output layer's loss for a few rows: bound by w's bytes, so w is read as it
// is, by plain loads, and the products are fp32 multiply-adds.
//   dots: a warp takes four classes at a time, every lane 16 bytes of each class's row in turn, by
//     asynchronous copies into a ring of its own (a lane reads back what it copied itself: no barriers);
//     x's rows lie in shared memory as fp32 and are read once for the four classes (16 rows: 20 loads of 16 bytes
//     a lane for four of w, 26 bytes of w a clock and SM; 23 come from memory).  The 4 R sums of
//     32 lanes are exchanged in halves, so that each lane ends with one or two; forward: a lane keeps
//     (maximum, sum) of what it gets; backward: p [classes][R].
//   outer: a thread owns 16 bytes of columns, x's and dx's R values of them in registers, and
//     walks over classes, four loads ahead: dw = p^T x goes out, dx += p w stays; ranges of classes are
//     added afterwards.
// w is read twice backward, three passes of w's bytes with dw's (the single pass would need dx's sums of a
// whole row beside w's in every SM).
#include <cfloat>

#include "linear_ce.cuh"
#include "ops.cuh"

namespace agn {
namespace ce {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kClasses = 4;                 // of a warp at a time
constexpr int kXFloats = 32 * 1024;         // of x in shared memory
// Threads of a block of dots (16 rows' sums need 255 registers), and the ring of a warp's copies: 16 bytes a
// lane of four classes each.
template <int R>
struct Dots {
  static constexpr int threads = R == 16 ? 256 : 512, warps = threads / 32, ring = R == 16 ? 6 : 3;
  static constexpr size_t ring_bytes = (size_t)warps * ring * kClasses * 512;
};
constexpr int kPFloats = 8192;              // of p in shared memory
constexpr float kLog2e = 1.44269504088896340736f;

template <typename T>
struct Vec {
  static constexpr int n = 16 / (int)sizeof(T);   // elements of 16 bytes
};

// The elements of 16 bytes.
template <typename T, int n>
__device__ __forceinline__ void unpack(uint4 q, float (&v)[n]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < n; ++i)
    v[i] = __uint_as_float(sizeof(T) == 4 ? w[i % 4] : i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
}

// 16 bytes at p: aligned and all there (wide), or element by element with zeros past `left` of them.
template <typename T>
__device__ __forceinline__ uint4 load16(const T* p, int64_t left, bool wide) {
  if (wide) return left > 0 ? AGN_LD(reinterpret_cast<const uint4*>(p)) : make_uint4(0, 0, 0, 0);
  alignas(16) T v[16 / sizeof(T)];
#pragma unroll
  for (int i = 0; i < 16 / (int)sizeof(T); ++i) v[i] = i < left ? AGN_LD(p + i) : T(0.f);
  return *reinterpret_cast<const uint4*>(v);
}

// The same into shared memory, asynchronously where wide.
template <typename T>
__device__ __forceinline__ void copy16(void* to, const T* p, int64_t left, bool wide) {
  if (wide && AGN_BOUNDS_OK(p, 16)) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                     static_cast<uint32_t>(__cvta_generic_to_shared(to))),
                 "l"(p)
                 : "memory");
  } else {
    *static_cast<uint4*>(to) = load16(p, left, wide);
  }
}

// Sums over the warp of V values: lane l gets those from V l / 32 on (fewer than 32: value l V / 32).
template <int V>
__device__ __forceinline__ void exchange(float (&a)[V], int lane) {
  int n = V;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    if (n > 1) {
      n /= 2;
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        if (j >= n) break;
        const float send = lane & o ? a[j] : a[j + n], keep = lane & o ? a[j + n] : a[j];
        a[j] = keep + __shfl_xor_sync(0xffffffffu, send, o);
      }
    } else {
      a[0] += __shfl_xor_sync(0xffffffffu, a[0], o);
    }
  }
}

// R: rows, rounded up to a power of two.
template <typename T, int R, bool kBackward>
__global__ void __launch_bounds__(Dots<R>::threads, 1)
dots_kernel(const FewArgs a, int chunk, int share, bool wide) {
  pdl_begin();
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int n = Vec<T>::n, V = kClasses * R, kOwn = V >= 32 ? V / 32 : 1;
  constexpr int kDotThreads = Dots<R>::threads, kDotWarps = Dots<R>::warps, kRing = Dots<R>::ring;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ __align__(16) float shared_sums[kDotWarps][R < 16 ? 32 : 64];   // (and the rows' (maximum, sum) at the end)
  uint4* ring = reinterpret_cast<uint4*>(smem) + warp * (kRing * kClasses * 32) + lane;
  // [R][chunk]; bf16: of eight consecutive columns the first four in a row's first half, the others in its
  // second, so that lanes read consecutive 16 bytes
  float* xs = reinterpret_cast<float*>(smem + Dots<R>::ring_bytes);
  const T* x = static_cast<const T*>(a.x);
  const T* w = static_cast<const T*>(a.w);
  uint32_t known = 0;   // rows with a label (the others are zeros)
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r < a.rows && has_label(AGN_LD(a.labels + r), a.classes)) known |= 1u << r;
  auto load_x = [&](int k0) {
    for (int j = threadIdx.x * n; j < chunk; j += kDotThreads * n) {
      const int at = n == 4 ? j : j / 2;
      uint4 q[R];
#pragma unroll
      for (int r = 0; r < R; ++r)
        q[r] = load16(x + (int64_t)min(r, a.rows - 1) * a.inner + k0 + j, known >> r & 1 ? (int64_t)a.inner - k0 - j : 0,
                      wide);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float v[n];
        unpack<T, n>(q[r], v);
#pragma unroll
        for (int i = 0; i < n; i += 4)
          *reinterpret_cast<float4*>(xs + r * chunk + at + (i ? chunk / 2 : 0)) =
              make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
      }
    }
  };
  const bool whole = chunk >= a.inner;
  if (whole) {
    load_x(0);
    __syncthreads();
  }
  // this lane's values: (class of the four, row)
  const int v0 = V >= 32 ? lane * kOwn : lane * V / 32;
  const bool owner = V >= 32 || lane % (32 / (V < 32 ? V : 32)) == 0;
  float2 ms[kOwn];
  float lse[kOwn], fa[kOwn], fb[kOwn];
  int label[kOwn];
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    const int r = (v0 + j) % R;
    ms[j] = make_float2(-INFINITY, 0.f);
    label[j] = r < a.rows ? AGN_LD(a.labels + r) : -1;
    lse[j] = fa[j] = fb[j] = 0.f;
    if (kBackward && has_label(label[j], a.classes)) {
      lse[j] = AGN_LD(a.lse + r);
      const float dl = a.dloss ? AGN_LD(a.dloss + r) : 1.f;
      fb[j] = a.scale * dl;
      fa[j] = a.dlse ? a.scale * (dl + AGN_LD(a.dlse + r)) : fb[j];
    }
  }
  // `share` warps of a block take a group of four classes together, a range of its steps each.  Groups go to
  // the blocks in turn.
  const int groups = (a.classes + kClasses - 1) / kClasses, teams = kDotWarps / share;
  const int team = warp / share, mine = warp % share, all = gridDim.x * teams;
  const int rounds = (groups + all - 1) / all;   // (the same for all warps: barriers below)
  auto group_of = [&](int round) { return (round * teams + team) * gridDim.x + blockIdx.x; };
  // A warp's work is a sequence of (round, columns) steps of 32 lanes x 16 bytes; copies run kRing - 1 ahead,
  // from one group into the next where x lies whole in shared memory, else within a chunk of columns.
  const int all_steps = (a.inner + 32 * n - 1) / (32 * n), each = (all_steps + share - 1) / share;
  int ahead_round = 0, ahead_step = mine * each;   // of the next copy
  uint32_t put = 0, take = 0;                      // slots of the ring
  auto fetch_at = [&](int c0, int k) {
    if (k < a.inner) {
#pragma unroll
      for (int c = 0; c < kClasses; ++c)
        copy16(ring + (put * kClasses + c) * 32, w + (int64_t)min(c0 + c, a.classes - 1) * a.inner + k, a.inner - k,
               wide);
    }
    if (++put == kRing) put = 0;
  };
  auto fetch_next = [&] {   // (whole)
    const int end = min(all_steps, (mine + 1) * each);
    if (ahead_step < end && ahead_round < rounds) {
      const int group = group_of(ahead_round);
      if (group < groups) fetch_at(group * kClasses, (ahead_step * 32 + lane) * n);
      if (++ahead_step == end) ahead_step = mine * each, ++ahead_round;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (whole)
    for (int i = 0; i < kRing - 1; ++i) fetch_next();
  for (int round = 0; round < rounds; ++round) {
    const int group = group_of(round);
    const int c0 = group * kClasses;
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    // one step: 16 bytes of four classes from the ring, and x's rows
    auto step_at = [&](int k, int k0) {
      float wv[kClasses][n];
#pragma unroll
      for (int c = 0; c < kClasses; ++c) unpack<T, n>(ring[(take * kClasses + c) * 32], wv[c]);
      if (++take == kRing) take = 0;
      if (k >= a.inner) return;
      const float* xk = xs + (n == 4 ? k - k0 : (k - k0) / 2);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float xv[n];
#pragma unroll
        for (int i = 0; i < n; i += 4) {
          const float4 q = *reinterpret_cast<const float4*>(xk + r * chunk + (i ? chunk / 2 : 0));
          xv[i] = q.x; xv[i + 1] = q.y; xv[i + 2] = q.z; xv[i + 3] = q.w;
        }
#pragma unroll
        for (int c = 0; c < kClasses; ++c)
#pragma unroll
          for (int i = 0; i < n; ++i) acc[c * R + r] = fmaf(wv[c][i], xv[i], acc[c * R + r]);
      }
    };
    if (whole) {
      if (group < groups) {
        for (int step = mine * each; step < min(all_steps, (mine + 1) * each); ++step) {
          fetch_next();
          asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
          step_at((step * 32 + lane) * n, 0);
        }
      }
    } else {
      for (int k0 = 0; k0 < a.inner; k0 += chunk) {   // (share is 1)
        __syncthreads();
        load_x(k0);
        __syncthreads();
        if (group >= groups) continue;
        const int steps = (min(chunk, a.inner - k0) + 32 * n - 1) / (32 * n);
        auto fetch = [&](int step) {
          if (step < steps) fetch_at(c0, k0 + (step * 32 + lane) * n);
          asm volatile("cp.async.commit_group;" ::: "memory");
        };
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i) fetch(i);
        for (int step = 0; step < steps; ++step) {
          fetch(step + kRing - 1);
          asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
          step_at(k0 + (step * 32 + lane) * n, k0);
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
    }
    __syncwarp();
    exchange<V>(acc, lane);
    if (share > 1) {   // (all warps: rounds are the same)
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kOwn; ++j) shared_sums[warp][32 * j + lane] = acc[j];
      __syncthreads();
      if (mine == 0)
        for (int k = 1; k < share; ++k)
#pragma unroll
          for (int j = 0; j < kOwn; ++j) acc[j] += shared_sums[warp + k][32 * j + lane];
    }
    if (group >= groups || mine != 0) continue;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int c = c0 + (v0 + j) / R, r = (v0 + j) % R;
      const bool in = c < a.classes;
      const float z = in ? acc[j] + (a.bias ? AGN_LD(a.bias + c) : 0.f) : -INFINITY;
      if (!kBackward) {
        ms[j] = join(ms[j], make_float2(z, z == -INFINITY ? 0.f : 1.f));
        if (owner && in && c == label[j]) AGN_ST(a.zlab + r, z);
      } else {
        float p = 0.f;
        if (has_label(label[j], a.classes) && lse[j] != -INFINITY) {
          p = fa[j] * exp2f((z - lse[j]) * kLog2e);
          if (c == label[j]) p -= fb[j];
        }
        if (owner && in) AGN_ST(a.p + (int64_t)c * R + r, p);
        acc[j] = p;
      }
    }
    if (kBackward && a.dbias) {   // a class's R values lie in eight neighbouring lanes
      float s = kOwn == 2 ? acc[0] + acc[kOwn - 1] : acc[0];
#pragma unroll
      for (int o = 32 / kClasses / 2; o > 0; o >>= 1)
        if (V >= 32 || o >= 32 / V) s += __shfl_xor_sync(0xffffffffu, s, o);   // (not lanes with the same value)
      constexpr int lanes = 32 / kClasses;
      if (lane % lanes == 0 && c0 + lane / lanes < a.classes) AGN_ST(a.dbias + c0 + lane / lanes, s);
    }
  }
  if constexpr (!kBackward) {
    // rows' (maximum, sum) of this block: over the lanes of a row, then the warps
    __syncthreads();
    float2(*parts)[R] = reinterpret_cast<float2(*)[R]>(shared_sums);
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      float2 v = ms[j];
#pragma unroll
      for (int o = 32 / kClasses; o < 32; o <<= 1)
        v = join(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
      if (owner && lane < 32 / kClasses) parts[warp][(v0 + j) % R] = v;
    }
    __syncthreads();
    if (threadIdx.x < R && (int)threadIdx.x < a.rows) {
      float2 v = parts[0][threadIdx.x];
      for (int k = 1; k < kDotWarps; ++k) v = join(v, parts[k][threadIdx.x]);
      AGN_ST(a.ms + (int64_t)threadIdx.x * gridDim.x + blockIdx.x, v);
    }
  }
}

// Classes whose loads are under way (a block an SM where the registers leave no room for two).
template <int kHeld>
struct Ahead {
  static constexpr int n = kHeld >= 64 ? 16 : 8;
  static constexpr size_t smem = (size_t)n * kThreads * 16 + kPFloats * 4;
};

// Threads: `along` columns of 16 bytes times kThreads / along ranges of classes.
template <typename T, int R>
__global__ void __launch_bounds__(kThreads) outer_kernel(const FewArgs a, int along, bool wide) {
  pdl_begin();
  constexpr int n = Vec<T>::n, kAhead = Ahead<R * n>::n;
  extern __shared__ __align__(16) uint8_t smem[];
  uint4* ring = reinterpret_cast<uint4*>(smem) + threadIdx.x;   // [kAhead][threads]
  float* ps = reinterpret_cast<float*>(smem + kAhead * kThreads * 16);
  const int tys = kThreads / along, ty = threadIdx.x / along, tx = threadIdx.x - ty * along;
  const int64_t k = ((int64_t)blockIdx.x * along + tx) * n, left = a.inner - k;
  const int part = blockIdx.y * tys + ty, parts = gridDim.y * tys;
  const bool in = ty < tys && left > 0, whole = wide && left >= n;
  const T* x = static_cast<const T*>(a.x);
  const T* w = static_cast<const T*>(a.w) + k;
  T* dw = a.dw ? static_cast<T*>(a.dw) + k : nullptr;
  float xv[R][n], dx[R][n];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool known = in && r < a.rows && has_label(AGN_LD(a.labels + min(r, a.rows - 1)), a.classes);
    unpack<T, n>(known ? load16(x + (int64_t)r * a.inner + k, left, whole) : make_uint4(0, 0, 0, 0), xv[r]);
#pragma unroll
    for (int i = 0; i < n; ++i) dx[r][i] = 0.f;
  }
  // this range's classes, `most` at a time: their p in shared memory
  const int each = (int)(((int64_t)a.classes + parts - 1) / parts), most = kPFloats / (R * tys);
  const int lo = (int)min((int64_t)a.classes, (int64_t)part * each), hi = (int)min((int64_t)a.classes, (int64_t)lo + each);
  const float* mine = ps + ty * most * R;
  for (int done = 0; done < each; done += most) {
    __syncthreads();
    for (int i = threadIdx.x; i < tys * most * R; i += kThreads) {
      const int y = i / (most * R), j = i - y * most * R;
      const int64_t first = (int64_t)(blockIdx.y * tys + y) * each + done;   // (class)
      const int64_t c = first + j / R;
      ps[i] = done + j / R < each && c < a.classes ? AGN_LD(a.p + first * R + j) : 0.f;
    }
    __syncthreads();
    const int c0 = lo + done, c1 = min(hi, c0 + most);
    if (!in || c0 >= c1) continue;
    auto fetch = [&](int c) {
      if (c < c1) copy16(ring + (c - c0) % kAhead * kThreads, w + (int64_t)c * a.inner, left, whole);
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (a.dx_parts) {
#pragma unroll
      for (int j = 0; j < kAhead - 1; ++j) fetch(c0 + j);
    }
#pragma unroll 2
    for (int c = c0; c < c1; ++c) {
      float out[n], wv[n], p[R];
      if (a.dx_parts) {
        fetch(c + kAhead - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
        unpack<T, n>(ring[(c - c0) % kAhead * kThreads], wv);
      }
      const float* pc = mine + (c - c0) * R;
#pragma unroll
      for (int r = 0; r < R; r += R < 4 ? 1 : 4) {
        if (R < 4) {
          p[r] = pc[r];
        } else {
          const float4 q = *reinterpret_cast<const float4*>(pc + r);
          p[r] = q.x; p[(r + 1) % R] = q.y; p[(r + 2) % R] = q.z; p[(r + 3) % R] = q.w;
        }
      }
#pragma unroll
      for (int i = 0; i < n; ++i) out[i] = 0.f;
#pragma unroll
      for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
          out[i] = fmaf(p[r], xv[r][i], out[i]);
          if (a.dx_parts) dx[r][i] = fmaf(p[r], wv[i], dx[r][i]);
        }
      }
      if (!dw) continue;
      T* to = dw + (int64_t)c * a.inner;
      if (whole) {
        if (sizeof(T) == 4) {
          AGN_STCS(reinterpret_cast<float4*>(to), make_float4(out[0], out[1], out[2], out[3]));
        } else {
          uint32_t q[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 o = __floats2bfloat162_rn(out[(2 * i) % n], out[(2 * i + 1) % n]);
            q[i] = *reinterpret_cast<const uint32_t*>(&o);
          }
          AGN_STCS(reinterpret_cast<uint4*>(to), make_uint4(q[0], q[1], q[2], q[3]));
        }
      } else {
#pragma unroll
        for (int i = 0; i < n; ++i)
          if (i < left) {
            if (sizeof(T) == 4) AGN_ST(reinterpret_cast<float*>(to) + i, out[i]);
            else AGN_ST(reinterpret_cast<bf16*>(to) + i, __float2bfloat16_rn(out[i]));
          }
      }
    }
  }
  if (!a.dx_parts || !in) return;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r >= a.rows) break;
    float* to = a.dx_parts + ((int64_t)part * a.rows + r) * a.ld_parts + k;   // (16-byte aligned, padded)
#pragma unroll
    for (int i = 0; i < n; i += 4)
      AGN_ST(reinterpret_cast<float4*>(to + i), make_float4(dx[r][i], dx[r][i + 1], dx[r][i + 2], dx[r][i + 3]));
  }
}

// dx: the ranges' sums in order: 32 columns a block, its warps share the ranges.
template <typename T>
__global__ void __launch_bounds__(kThreads) parts_kernel(const FewArgs a, int parts, T* dx) {
  pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = blockIdx.y, k = blockIdx.x * 32 + lane;
  __shared__ float sums[kWarps][32];
  float s = 0.f;
  if (k < a.inner) {
#pragma unroll 4
    for (int q = warp; q < parts; q += kWarps) s += AGN_LD(a.dx_parts + ((int64_t)q * a.rows + r) * a.ld_parts + k);
  }
  sums[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || k >= a.inner) return;
  for (int j = 1; j < kWarps; ++j) s += sums[j][lane];
  if (!has_label(AGN_LD(a.labels + r), a.classes)) s = 0.f;
  if (sizeof(T) == 4) AGN_ST(reinterpret_cast<float*>(dx) + (int64_t)r * a.inner + k, s);
  else AGN_ST(reinterpret_cast<bf16*>(dx) + (int64_t)r * a.inner + k, __float2bfloat16_rn(s));
}

template <typename T, int R, bool kBackward>
Status dots(const FewArgs& a, cudaStream_t st) {
  struct Tag {};
  auto kern = dots_kernel<T, R, kBackward>;
  int dev = 0;
  AGN_TRY(current_device(&dev));
  const int chunk = (int)std::min<int64_t>(round_up(a.inner, 32 * Vec<T>::n), kXFloats / R / 256 * 256);
  constexpr int kDotWarps = Dots<R>::warps;
  constexpr size_t most = Dots<R>::ring_bytes + kXFloats * sizeof(float);
  AGN_TRY_CUDA(allow_smem<Tag>(kern, most, dev));
  // warps of a group: so many that all have work, a step each at least
  const int64_t groups = ceil_div(a.classes, kClasses), steps = ceil_div(a.inner, 32 * Vec<T>::n);
  int share = 1;
  while (chunk >= a.inner && share < kDotWarps && 2 * share <= steps && groups * share < (int64_t)kFewSms * kDotWarps)
    share *= 2;
  AGN_TRY_CUDA(launch_pdl(kern, dim3((unsigned)few_blocks(a.classes)), dim3(Dots<R>::threads),
                          Dots<R>::ring_bytes + (size_t)R * chunk * 4, st, a, chunk, share, a.inner % Vec<T>::n == 0));
  return Status::Ok();
}

template <typename T, int R>
Status outer(const FewArgs& a, cudaStream_t st) {
  struct Tag {};
  const FewCut c = few_cut(a.inner, a.classes, (int)sizeof(T));
  constexpr size_t smem = Ahead<R * Vec<T>::n>::smem;
  auto kern = outer_kernel<T, R>;
  int dev = 0;
  AGN_TRY(current_device(&dev));
  AGN_TRY_CUDA(allow_smem<Tag>(kern, smem, dev));
  AGN_TRY_CUDA(launch_pdl(kern, dim3((unsigned)c.blocks_k, (unsigned)c.blocks_c), dim3(kThreads), smem, st, a, c.along,
                          a.inner % Vec<T>::n == 0));
  if (!a.dx_parts) return Status::Ok();
  AGN_TRY_CUDA(launch_pdl(parts_kernel<T>, dim3((unsigned)ceil_div(a.inner, 32), (unsigned)a.rows), dim3(kThreads), 0,
                          st, a, c.parts, static_cast<T*>(a.dx)));
  return Status::Ok();
}

template <typename T, int R>
Status run_few_backward(const FewArgs& a, cudaStream_t st) {
  AGN_TRY((dots<T, R, true>(a, st)));
  if (!a.dw && !a.dx_parts) return Status::Ok();
  return outer<T, R>(a, st);
}

template <int R>
Status run_few(const FewArgs& a, bool backward, cudaStream_t st) {
  return backward ? run_few_backward<float, R>(a, st) : dots<float, R, false>(a, st);
}

}  // namespace

Status few(const FewArgs& a, int dtype, bool backward, cudaStream_t st) {
  const int R = few_rows(a.rows);
  if (dtype == AGN_PREC_FP32) {
    switch (R) {
      case 1: return run_few<1>(a, backward, st);
      case 2: return run_few<2>(a, backward, st);
      case 4: return run_few<4>(a, backward, st);
      case 8: return run_few<8>(a, backward, st);
      default: return run_few<16>(a, backward, st);
    }
  }
  switch (R) {   // (backward alone)
    case 1: return run_few_backward<bf16, 1>(a, st);
    case 2: return run_few_backward<bf16, 2>(a, st);
    default: return run_few_backward<bf16, 4>(a, st);
  }
}

}  // namespace ce

AGN_BOUNDS_UNIT(linear_ce_few)

}  // namespace agn
