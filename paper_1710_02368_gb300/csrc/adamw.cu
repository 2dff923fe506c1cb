// AdamW over many tensors in one launch (decoupled weight decay), with 32-bit states or
// with 8-bit ones, and the norm of all gradients with the factor that clips it (formulas and
// the 8-bit form in include/agn.h).
//
// Every pass is bound by its bytes: an element with 32-bit states moves 28 (fp32 gradient) or
// 26 bytes (bf16), with 8-bit states 16 or 14 and 1/8 for the scales, 2 more with the copy.  The
// tensors are cut into pieces of 2048 elements, a list of which lies on the device, so that many
// small tensors and a few large ones are the same launch; a block of 256 threads takes pieces in turn,
// a thread eight consecutive elements: 32 bytes a load or store of fp32.  Four lanes are a
// block of 32 elements with one scale: its largest value is two shuffles.
// Each operation of a state is rounded to fp32 by itself (no fused multiply-add), so that
// the codes of the 8-bit form do not depend on how a compiler contracts.
#include <cfloat>
#include <cmath>
#include <memory>
#include <type_traits>
#include <vector>

#include "common.cuh"
#include "generator.cuh"
#include "ops.cuh"

namespace agn {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                       // elements of a thread
constexpr int kPiece = kThreads * kPer;
constexpr int kBlock = 32;                    // elements that share a scale
constexpr int kMantM = 3, kMantR = 4;         // mantissa bits of the codes of m and sqrt(v)
constexpr int kMostGrid = 4096;               // blocks of the norm's first pass

// A tensor as the kernels see it.
struct Tensor {
  float* param;
  const void* grad;
  void *m, *v;
  uint8_t *ms, *vs;
  bf16* copy;
  int64_t n;
  uint64_t first;    // draws of the tensors before it
  double decay;
  int32_t bf16_grad;
  int32_t wide;      // every buffer takes its widest loads and stores
};
struct Piece {
  int32_t tensor, index;
};

struct StepArgs {
  const Tensor* tensors;
  const Piece* pieces;
  int n_pieces, group;
  float b1, ob1, b2, ob2, eps, rc2, size;   // rc2 = 1 / sqrt(1 - beta2^t), size = lr / (1 - beta1^t)
  double lr;
  const float* scale;
  uint64_t key, offset;
};

// Eight elements at p: in one piece (wide: aligned, and all there), or the first n one by one.
__device__ __forceinline__ void load8(const float* p, int n, bool wide, float (&x)[8]) {
  if (wide) {
    if (AGN_BOUNDS_OK(p, 32)) {
      asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]),
                     "=f"(x[7])
                   : "l"(p));
    } else {
      AGN_BOUNDS_FAIL(p);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? AGN_LD(p + i) : 0.f;
  }
}
__device__ __forceinline__ void store8(float* p, int n, bool wide, const float (&x)[8]) {
  if (wide) {
    if (AGN_BOUNDS_OK(p, 32)) {
      asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(x[0]),
                   "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                   : "memory");
    } else {
      AGN_BOUNDS_FAIL(p);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) AGN_ST(p + i, x[i]);
  }
}
__device__ __forceinline__ void store8(bf16* p, int n, bool wide, const float (&x)[8]) {
  if (wide) {
    const __nv_bfloat162 o[4] = {__floats2bfloat162_rn(x[0], x[1]), __floats2bfloat162_rn(x[2], x[3]),
                                 __floats2bfloat162_rn(x[4], x[5]), __floats2bfloat162_rn(x[6], x[7])};
    AGN_ST(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(o));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) AGN_ST(p + i, __float2bfloat16_rn(x[i]));
  }
}
// Eight gradients as they lie, and their values: apart, so that what is loaded beside them is under way before
// anything waits for them.
template <typename T>
struct Raw {
  uint32_t w[sizeof(T) == 4 ? 8 : 4];
};
__device__ __forceinline__ void load8(const float* p, int n, bool wide, Raw<float>& r) {
  float x[8];
  load8(p, n, wide, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) r.w[i] = __float_as_uint(x[i]);
}
__device__ __forceinline__ void load8(const bf16* p, int n, bool wide, Raw<bf16>& r) {
  if (wide) {
    const uint4 q = AGN_LD(reinterpret_cast<const uint4*>(p));
    r.w[0] = q.x; r.w[1] = q.y; r.w[2] = q.z; r.w[3] = q.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = 2 * i < n ? AGN_LD(reinterpret_cast<const uint16_t*>(p) + 2 * i) : 0;
      const uint32_t hi = 2 * i + 1 < n ? AGN_LD(reinterpret_cast<const uint16_t*>(p) + 2 * i + 1) : 0;
      r.w[i] = hi << 16 | lo;
    }
  }
}
template <typename T>
__device__ __forceinline__ void unpack8(const Raw<T>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    x[i] = __uint_as_float(sizeof(T) == 4 ? r.w[i % (sizeof(r.w) / 4)] : i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
}
__device__ __forceinline__ uint2 load8_codes(const uint8_t* p, int n, bool wide) {
  if (wide) return AGN_LD(reinterpret_cast<const uint2*>(p));
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) w[i >> 2] |= (uint32_t)AGN_LD(p + i) << (8 * (i & 3));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store8_codes(uint8_t* p, int n, bool wide, const uint32_t (&c)[8]) {
  if (wide) {
    auto four = [&](int i) {   // their low bytes
      return __byte_perm(__byte_perm(c[i], c[i + 1], 0x0040), __byte_perm(c[i + 2], c[i + 3], 0x0040), 0x5410);
    };
    AGN_ST(reinterpret_cast<uint2*>(p), make_uint2(four(0), four(4)));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) AGN_ST(p + i, (uint8_t)c[i]);
  }
}
// Code i of eight, in the upper byte (the lower ones are 0).
__device__ __forceinline__ uint32_t code_at(uint2 q, int i) {
  return __byte_perm(i < 4 ? q.x : q.y, 0, (i & 3) << 12 | 0x444);
}

// The magnitude of a code (in the upper byte): its exponent and mantissa lie where a float's do, 112
// exponents lower (so a code with exponent 0 is a subnormal float, its product with 2^112 exact).  kOnce:
// `scale` has the factor 2^112 in it, which fits scales up to 2^15.
template <int kMant, bool kOnce>
__device__ __forceinline__ float decode(uint32_t code, float scale) {
  const float u = __uint_as_float(code >> (kMant + 1));
  return kOnce ? __fmul_rn(u, scale) : __fmul_rn(__fmul_rn(u, 0x1p112f), scale);
}
__device__ __forceinline__ float scale_value(uint32_t e) { return __uint_as_float(e << 23); }
constexpr uint32_t kOnceMost = 141;   // scale bytes whose factors with 2^112 and 2^-112 are floats

// The scale of a block whose largest magnitude has the bits `top`: the power of two that brings it
// into [1, 2 - 2^-kMant], the largest code's value.
template <int kMant>
__device__ __forceinline__ uint32_t scale_code(uint32_t top) {
  return min(max((top + ((1u << (23 - kMant)) - 1)) >> 23, 1u), 253u);
}
// The code of x >= 0: up to the next one where the fraction left and (bits + 1/2) / 65536 reach one.  kOnce:
// `inverse` has the factor 2^-112 in it, and no value is above the largest code's.
// `bits`: the 16 bits and a 1 behind them, where they are added.
template <int kMant, bool kOnce>
__device__ __forceinline__ uint32_t encode(float x, float inverse, uint32_t bits) {
  const float u = kOnce ? __fmul_rn(x, inverse) : __fmul_rn(__fmul_rn(x, inverse), 0x1p-112f);
  constexpr int shift = 23 - kMant;
  const uint32_t code = (__float_as_uint(u) + bits) >> shift;
  return kOnce ? code : min(code, (16u << kMant) - 1);
}

// m, sqrt(v) and the parameter after the step; v is given and left as sqrt(v)'s square (8 bits) or itself.
__device__ __forceinline__ void step_one(const StepArgs& a, float g, float keep, float& p, float& m, float& v, float& r) {
  m = __fadd_rn(__fmul_rn(m, a.b1), __fmul_rn(g, a.ob1));
  v = __fadd_rn(__fmul_rn(v, a.b2), __fmul_rn(__fmul_rn(g, g), a.ob2));
  r = __fsqrt_rn(v);
  // (by an approximate reciprocal, two units off: 32 bits the same, 8 bits 431 us for 447, 100 M elements)
  const float q = __fdiv_rn(m, __fadd_rn(__fmul_rn(r, a.rc2), a.eps));
  p = __fsub_rn(__fmul_rn(p, keep), __fmul_rn(q, a.size));
}

// Eight elements of a tensor as they are loaded.
template <typename G>
struct Held {
  Raw<G> g;
  float p[8], m[8], v[8];   // (m, v: 32 bits)
  uint2 qm, qv;             // (8 bits: codes and scale bytes)
  uint32_t em, er;
};

// One step on elements e to e + n - 1 (n may be 0: the warp shares scales).
template <int kBits, typename G>
__device__ __forceinline__ void step_eight(const StepArgs& a, const Tensor& t, float s, int64_t e, int n, bool wide,
                                           Held<G>& h) {
  float (&p)[8] = h.p, (&m)[8] = h.m, (&v)[8] = h.v;
  uint32_t em = h.em, er = h.er;
  const uint2 qm = h.qm, qv = h.qv;
  float g[8];
  unpack8(h.g, g);
  const float keep = (float)__dsub_rn(1.0, __dmul_rn(a.lr, t.decay));   // (after the loads: an SM does few of these)
  if (a.scale) {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = __fmul_rn(g[i], s);
  }
  float r[8];
  if (kBits == 8) {
    auto values = [&](auto once) {
      constexpr bool kOnce = decltype(once)::value;
      const float sm = scale_value(kOnce && em ? em + 112 : em), sr = scale_value(kOnce && er ? er + 112 : er);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t cm = code_at(qm, i);
        m[i] = __uint_as_float(__float_as_uint(decode<kMantM, kOnce>(cm & 0x7f000000u, sm)) | (cm & 0x80000000u));
        const float root = decode<kMantR, kOnce>(code_at(qv, i), sr);
        v[i] = __fmul_rn(root, root);
      }
    };
    if (__any_sync(0xffffffffu, max(em, er) > kOnceMost)) values(std::false_type());
    else values(std::true_type());
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) step_one(a, g[i], keep, p[i], m[i], v[i], r[i]);
  if (kBits == 8) {
    auto scales = [&](auto finite) {   // finite: of the values that are
      uint32_t top_m = 0, top_r = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        top_m = max(top_m, __float_as_uint(m[i]) & 0x7fffffffu);
        if (!decltype(finite)::value || r[i] <= FLT_MAX) top_r = max(top_r, __float_as_uint(r[i]));
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        top_m = max(top_m, __shfl_xor_sync(0xffffffffu, top_m, o));
        top_r = max(top_r, __shfl_xor_sync(0xffffffffu, top_r, o));
      }
      em = scale_code<kMantM>(top_m), er = scale_code<kMantR>(top_r);
    };
    scales(std::false_type());
    const uint64_t d0 = a.key + (a.offset + t.first + (uint64_t)(e / 2) + 1) * gen::kG;
    uint32_t cm[8], cr[8];
    auto codes = [&](auto once) {
      constexpr bool kOnce = decltype(once)::value;
      const float im = scale_value((kOnce ? 142u : 254u) - em), ir = scale_value((kOnce ? 142u : 254u) - er);
#pragma unroll
      for (int d2 = 0; d2 < 4; ++d2) {   // a draw for two elements: 16 bits for m, 16 for sqrt(v)
        const uint64_t d = gen::mix(d0 + (uint64_t)d2 * gen::kG);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int i = 2 * d2 + k;
          const uint32_t w = (uint32_t)(d >> (32 * k));
          constexpr uint32_t kM = 23 - kMantM - 16, kR = 23 - kMantR - 16;
          cm[i] = encode<kMantM, kOnce>(fabsf(m[i]), im, (w << kM & 0xffffu << kM) | 1u << (kM - 1)) |
                  (__float_as_uint(m[i]) >> 24 & 0x80u);
          cr[i] = encode<kMantR, kOnce>(r[i], ir, (w >> (16 - kR) & 0xffffu << kR) | 1u << (kR - 1));
          if (r[i] > 0.f) cr[i] = max(cr[i], 1u);   // m / eps would follow
        }
      }
    };
    if (__any_sync(0xffffffffu, max(em, er) > kOnceMost)) {
      // An element whose v is not finite stays out of its block's scales, which would be the largest and leave the
      // others nothing: its m becomes 0 and its sqrt(v) the largest code.
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (!(r[i] <= FLT_MAX)) m[i] = 0.f;
      scales(std::true_type());
      codes(std::false_type());
    } else {
      codes(std::true_type());
    }
    if (n > 0) {
      store8_codes(static_cast<uint8_t*>(t.m) + e, n, wide, cm);
      store8_codes(static_cast<uint8_t*>(t.v) + e, n, wide, cr);
      if ((threadIdx.x & 3) == 0) {
        AGN_ST(t.ms + e / kBlock, (uint8_t)em);
        AGN_ST(t.vs + e / kBlock, (uint8_t)er);
      }
    }
  } else if (n > 0) {
    store8(static_cast<float*>(t.m) + e, n, wide, m);
    store8(static_cast<float*>(t.v) + e, n, wide, v);
  }
  if (n > 0) {
    store8(t.param + e, n, wide, p);
    if (t.copy) store8(t.copy + e, n, wide, p);
  }
}

// 16 or 8 bytes into shared memory, asynchronously.
template <int kBytes>
__device__ __forceinline__ void copy_async(void* to, const void* p) {
  if (AGN_BOUNDS_OK(p, kBytes)) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(
                     static_cast<uint32_t>(__cvta_generic_to_shared(to))),
                 "l"(p), "n"(kBytes)
                 : "memory");
  } else {
    AGN_BOUNDS_FAIL(p);
    for (int i = 0; i < kBytes / 4; ++i) static_cast<uint32_t*>(to)[i] = 0;
  }
}

// A piece of a tensor with 8-bit states in shared memory, a thread's own part of it: what the next piece needs
// comes while this one's arithmetic runs (99 instructions an element; with an approximate quotient, 100 M elements took 328 us
// without it).
struct Slot {
  uint4 p[2][kThreads], g[2][kThreads];
  uint2 m[kThreads], v[kThreads];
};

template <typename G>
__device__ __forceinline__ void fetch(const Tensor& t, int64_t e, Slot& to) {
  const int i = threadIdx.x;
#pragma unroll
  for (int k = 0; k < 2; ++k) copy_async<16>(&to.p[k][i], t.param + e + 4 * k);
#pragma unroll
  for (int k = 0; k < (int)sizeof(G) / 2; ++k)
    copy_async<16>(&to.g[k][i], static_cast<const G*>(t.grad) + e + 16 / (int)sizeof(G) * k);
  copy_async<8>(&to.m[i], static_cast<const uint8_t*>(t.m) + e);
  copy_async<8>(&to.v[i], static_cast<const uint8_t*>(t.v) + e);
  asm volatile("cp.async.commit_group;" ::: "memory");
}

// Pieces `index` to `end` - 1 of a tensor.
template <int kBits, typename G>
__device__ __forceinline__ void step_pieces(const StepArgs& a, const Tensor& t, float s, int64_t index, int64_t end,
                                            Slot* slots) {
  if (kBits == 8) {   // whole pieces, one ahead
    const int64_t whole = t.wide ? min(end, t.n / kPiece) : 0;
    const int i = threadIdx.x;
    uint32_t em = 0, er = 0;
    auto scales = [&](int64_t e) {
      em = AGN_LD(t.ms + e / kBlock);
      er = AGN_LD(t.vs + e / kBlock);
    };
    int64_t e = index * kPiece + i * kPer;
    if (index < whole) {
      fetch<G>(t, e, slots[0]);
      scales(e);
    }
    for (int slot = 0; index < whole; ++index, slot ^= 1, e += kPiece) {
      Held<G> h;
      h.em = em;
      h.er = er;
      if (index + 1 < whole) {
        fetch<G>(t, e + kPiece, slots[slot ^ 1]);
        scales(e + kPiece);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      const Slot& from = slots[slot];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 q = from.p[k][i];
        h.p[4 * k] = __uint_as_float(q.x); h.p[4 * k + 1] = __uint_as_float(q.y);
        h.p[4 * k + 2] = __uint_as_float(q.z); h.p[4 * k + 3] = __uint_as_float(q.w);
      }
#pragma unroll
      for (int k = 0; k < (int)sizeof(G) / 2; ++k) {
        const uint4 q = from.g[k][i];
        h.g.w[4 * k] = q.x; h.g.w[4 * k + 1] = q.y; h.g.w[4 * k + 2] = q.z; h.g.w[4 * k + 3] = q.w;
      }
      h.qm = from.m[i];
      h.qv = from.v[i];
      step_eight<kBits>(a, t, s, e, kPer, true, h);
    }
  }
  for (; index < end; ++index) {
    const int64_t e = index * kPiece + threadIdx.x * kPer;
    const int n = (int)max((int64_t)0, min((int64_t)kPer, t.n - e));
    const bool wide = t.wide && n == kPer;
    // (what is not there is loaded as zeros, whose states and codes are zeros)
    Held<G> h;
    if (kBits == 32 && t.bf16_grad) {   // (G is float; us for 20 M elements 87, with all loads at once 92)
      Raw<bf16> raw;
      float g[8];
      load8(static_cast<const bf16*>(t.grad) + e, n, wide, raw);
      unpack8(raw, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) h.g.w[i] = __float_as_uint(g[i]);
    } else {
      load8(static_cast<const G*>(t.grad) + e, n, wide, h.g);
    }
    load8(t.param + e, n, wide, h.p);
    if (kBits == 8) {
      h.qm = load8_codes(static_cast<const uint8_t*>(t.m) + e, n, wide);
      h.qv = load8_codes(static_cast<const uint8_t*>(t.v) + e, n, wide);
      h.em = h.er = 0;
      if (n > 0) {
        h.em = AGN_LD(t.ms + e / kBlock);
        h.er = AGN_LD(t.vs + e / kBlock);
      }
    } else {
      load8(static_cast<const float*>(t.m) + e, n, wide, h.m);
      load8(static_cast<const float*>(t.v) + e, n, wide, h.v);
    }
    step_eight<kBits>(a, t, s, e, n, wide, h);
  }
}

template <int kBits>
__global__ void __launch_bounds__(kThreads, 4) adamw_kernel(const StepArgs a) {
  pdl_begin();
  float s = 1.f;
  if (a.scale) {
    s = AGN_LD(a.scale);
    if (!(fabsf(s) <= FLT_MAX)) return;
  }
  extern __shared__ __align__(16) uint8_t smem[];   // [2] slots, 8 bits
  Slot* slots = reinterpret_cast<Slot*>(smem);
  // A block takes `group` consecutive pieces in turn; a tensor's among them are a run that needs no look at
  // the list.
  for (int c0 = blockIdx.x * a.group; c0 < a.n_pieces; c0 += gridDim.x * a.group) {
    const int last = min(a.n_pieces, c0 + a.group);
    for (int c = c0; c < last;) {
      const Piece piece = AGN_LD(a.pieces + c);
      const Tensor t = AGN_LD(a.tensors + piece.tensor);
      const int64_t end = min((int64_t)piece.index + last - c, (t.n + kPiece - 1) / kPiece);
      if (kBits == 8 && t.bf16_grad) step_pieces<kBits, bf16>(a, t, s, piece.index, end, slots);
      else step_pieces<kBits, float>(a, t, s, piece.index, end, slots);
      c += (int)(end - piece.index);
    }
  }
}

// Squares and sums of up to 32 of them in fp32, a thread's sum of these with the rounding's remainder carried along,
// a warp's 32 in fp32, the rest in 64 bits (an SM adds few of those: sums of threads took most of the time).  Gradients of
// 1e18 and more can take that out of fp32's range, though the norm is a number: such a warp reads its gradients once more.
constexpr int kNormPieces = 4;   // in flight
__global__ void __launch_bounds__(kThreads)
norm_kernel(const Tensor* tensors, const Piece* pieces, int n_pieces, double* partials) {
  pdl_begin();
  float sum = 0.f, rest = 0.f;
  auto add = [&](float part) {   // (Knuth's two-sum)
    const float both = __fadd_rn(sum, part), back = __fsub_rn(both, sum);
    rest = __fadd_rn(rest, __fadd_rn(__fsub_rn(sum, __fsub_rn(both, back)), __fsub_rn(part, back)));
    sum = both;
  };
  auto squares = [&](auto kind, const Tensor& t, int64_t index, int64_t end) {
    using G = decltype(kind);
    const G* grad = static_cast<const G*>(t.grad);
    // whole pieces, four in flight; then one by one
    const int64_t whole = t.wide ? min(end, t.n / kPiece) : 0;
    for (; index + kNormPieces <= whole; index += kNormPieces) {
      const int64_t e = index * kPiece + threadIdx.x * kPer;
      Raw<G> raw[kNormPieces];
#pragma unroll
      for (int k = 0; k < kNormPieces; ++k) load8(grad + e + k * kPiece, kPer, true, raw[k]);
      float part = 0.f;
#pragma unroll
      for (int k = 0; k < kNormPieces; ++k) {
        float g[8];
        unpack8(raw[k], g);
#pragma unroll
        for (int i = 0; i < 8; ++i) part = fmaf(g[i], g[i], part);
      }
      add(part);
    }
    for (; index < end; ++index) {
      const int64_t e = index * kPiece + threadIdx.x * kPer;
      const int n = (int)max((int64_t)0, min((int64_t)kPer, t.n - e));
      if (n <= 0) continue;
      Raw<G> raw;
      load8(grad + e, n, t.wide && n == kPer, raw);
      float g[8], part = 0.f;
      unpack8(raw, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) part = fmaf(g[i], g[i], part);
      add(part);
    }
  };
  const int last = (int)((int64_t)n_pieces * (blockIdx.x + 1) / gridDim.x);
  auto each_run = [&](auto&& f) {
    for (int c = (int)((int64_t)n_pieces * blockIdx.x / gridDim.x); c < last;) {
      const Piece piece = AGN_LD(pieces + c);
      const Tensor t = AGN_LD(tensors + piece.tensor);
      const int64_t end = min((int64_t)piece.index + last - c, (t.n + kPiece - 1) / kPiece);
      if (t.bf16_grad) f(bf16(), t, piece.index, end);
      else f(float(), t, piece.index, end);
      c += (int)(end - piece.index);
    }
  };
  each_run(squares);
  if (fabsf(sum) <= FLT_MAX) sum += rest;   // (an infinite sum's remainder is NaN)
  __shared__ double warps[kThreads / 32];
  if (__any_sync(0xffffffffu, !(sum < 0x1p122f))) {   // a warp whose sum may leave fp32's range: anew in 64 bits
    double all = 0.0;
    each_run([&](auto kind, const Tensor& t, int64_t index, int64_t end) {
      using G = decltype(kind);
      for (; index < end; ++index) {
        const int64_t e = index * kPiece + threadIdx.x * kPer;
        const int n = (int)max((int64_t)0, min((int64_t)kPer, t.n - e));
        if (n <= 0) continue;
        Raw<G> raw;
        load8(static_cast<const G*>(t.grad) + e, n, t.wide && n == kPer, raw);
        float g[8];
        unpack8(raw, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) all = fma((double)g[i], (double)g[i], all);
      }
    });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = all;
  } else {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = (double)sum;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double all = warps[0];
    for (int w = 1; w < kThreads / 32; ++w) all += warps[w];
    AGN_ST(partials + blockIdx.x, all);
  }
}

__global__ void __launch_bounds__(32)
norm_finish_kernel(const double* partials, int n, double max_norm, float* norm, float* scale) {
  pdl_begin();
  double sum = 0.0;
  for (int i = threadIdx.x; i < n; i += 32) sum += AGN_LD(partials + i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (threadIdx.x == 0) {
    const float total = (float)sqrt(sum), most = (float)max_norm;
    if (norm) AGN_ST(norm, total);
    if (scale)
      AGN_ST(scale, !(total <= FLT_MAX) ? __uint_as_float(0x7fc00000u) : total > most ? __fdiv_rn(most, total) : 1.f);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(const uint8_t* m, const uint8_t* ms, const uint8_t* v, const uint8_t* vs, int64_t n,
                  T* m_out, T* r_out, bool wide) {
  pdl_begin();
  const int64_t step = (int64_t)gridDim.x * kPiece;
  for (int64_t e = (int64_t)blockIdx.x * kPiece + threadIdx.x * kPer; e < n; e += step) {
    const int k = (int)min((int64_t)kPer, n - e);
    const bool whole = wide && k == kPer;
    float x[8];
    if (m_out) {
      const uint2 q = load8_codes(m + e, k, whole);
      const float s = scale_value(AGN_LD(ms + e / kBlock));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t c = code_at(q, i);
        x[i] = __uint_as_float(__float_as_uint(decode<kMantM, false>(c & 0x7f000000u, s)) | (c & 0x80000000u));
      }
      store8(m_out + e, k, whole, x);
    }
    if (r_out) {
      const uint2 q = load8_codes(v + e, k, whole);
      const float s = scale_value(AGN_LD(vs + e / kBlock));
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = decode<kMantR, false>(code_at(q, i), s);
      store8(r_out + e, k, whole, x);
    }
  }
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace

AGN_BOUNDS_UNIT(adamw)

}  // namespace agn

struct agn_optim {
  int device = 0, bits = 32;
  bool has_param = false;
  int64_t tensors = 0;
  int pieces = 0, norm_grid = 0;
  agn::Tensor* d_tensors = nullptr;
  agn::Piece* d_pieces = nullptr;
  double* d_partials = nullptr;
  std::vector<agn::CallBuffer> buffers;   // every buffer of the tensors (the bounds-checked build's)
  // the bytes of all buffers and of those that a step writes: intervals apart and in order
  std::vector<std::pair<uintptr_t, uintptr_t>> all, written;
  ~agn_optim() {
    cudaFree(d_tensors);
    cudaFree(d_pieces);
    cudaFree(d_partials);
  }
};

namespace agn {
namespace {

// Bounds-checked build: a plan's buffers and tables are known while a call lasts.
struct KnownPlan {
  std::vector<const void*> p;
  explicit KnownPlan(const agn_optim& o) {
#ifdef AGN_BOUNDS_CHECK
    auto add = [&](const void* q, size_t bytes) {
      if (!q || !bytes) return;
      bounds_add(q, bytes);
      p.push_back(q);
    };
    for (const CallBuffer& b : o.buffers) add(b.p, b.bytes);
    // (tables are not a caller's: the bounds check's self-test does not shorten them)
    add(o.d_tensors, (size_t)o.tensors * sizeof(Tensor) + 256);
    add(o.d_pieces, (size_t)o.pieces * sizeof(Piece) + 256);
    add(o.d_partials, (size_t)o.norm_grid * sizeof(double) + 256);
#else
    (void)o;
#endif
  }
  ~KnownPlan() {
    for (const void* q : p) bounds_remove(q);
  }
};

Status optim_create(const agn_optim_tensor* ts, int32_t n_tensors, int32_t bits, agn_optim** out) {
  if (!out) return Status::Err(AGN_E_INVALID, "null pointer");
  *out = nullptr;
  if (bits != 32 && bits != 8) return Status::Err(AGN_E_INVALID, "state_bits must be 32 or 8");
  if (n_tensors < 0 || (n_tensors > 0 && !ts)) return Status::Err(AGN_E_INVALID, "bad tensor list");
  std::unique_ptr<agn_optim> o(new agn_optim);
  o->bits = bits;
  bool any = false;   // (an empty tensor's addresses may be null)
  std::vector<Tensor> host;
  std::vector<Piece> pieces;
  struct Range {
    uintptr_t lo, hi;
    bool written;
    int tensor;
  };
  std::vector<Range> ranges;
  uint64_t first = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const agn_optim_tensor& t = ts[i];
    const std::string name = "tensor " + std::to_string(i);
    const size_t gs = dtype_size(t.grad_dtype);
    if (!gs) return Status::Err(AGN_E_INVALID, name + ": unknown grad_dtype");
    if (t.n < 0 || t.n > (int64_t)1 << 40) return Status::Err(AGN_E_INVALID, name + ": n must be in [0, 2^40]");
    if (!(t.weight_decay >= 0.0 && t.weight_decay <= 1e30))
      return Status::Err(AGN_E_INVALID, name + ": weight_decay must be finite and >= 0");
    if (t.n > 0) {
      if (!any) o->has_param = t.param != nullptr;
      any = true;
      if ((t.param != nullptr) != o->has_param)
        return Status::Err(AGN_E_INVALID, name + ": all tensors have a param or none has");
      if (!t.grad) return Status::Err(AGN_E_INVALID, name + ": null grad");
      if (t.param && (!t.m || !t.v || (bits == 8 && (!t.m_scale || !t.v_scale))))
        return Status::Err(AGN_E_INVALID, name + ": null state");
    }
    const size_t n = (size_t)t.n, nb = (n + kBlock - 1) / kBlock, ss = bits == 8 ? 1 : 4;
    const bool p = t.param != nullptr;
    const CallBuffer bufs[7] = {{"grad", t.grad, n * gs, gs},
                                {"param", t.param, n * 4, 4},
                                {"m", p ? t.m : nullptr, n * ss, ss},
                                {"v", p ? t.v : nullptr, n * ss, ss},
                                {"m_scale", p && bits == 8 ? t.m_scale : nullptr, nb, 1},
                                {"v_scale", p && bits == 8 ? t.v_scale : nullptr, nb, 1},
                                {"copy", p ? t.copy : nullptr, n * 2, 2}};
    Tensor d{};
    d.param = t.param; d.grad = t.grad; d.m = t.m; d.v = t.v;
    d.ms = t.m_scale; d.vs = t.v_scale;
    d.copy = p ? static_cast<bf16*>(t.copy) : nullptr;
    d.n = t.n;
    d.first = first;
    d.decay = t.weight_decay;
    d.bf16_grad = t.grad_dtype == AGN_PREC_BF16;
    d.wide = aligned(t.grad, 8 * gs) && (!p || (aligned(t.param, 32) && aligned(t.m, 8 * ss) &&
                                                aligned(t.v, 8 * ss) && aligned(t.copy, 16)));
    for (int k = 0; k < 7; ++k) {
      if (!bufs[k].p || !bufs[k].bytes) continue;
      if (reinterpret_cast<uintptr_t>(bufs[k].p) % bufs[k].align != 0)
        return Status::Err(AGN_E_INVALID, name + ": " + bufs[k].name + " is not aligned");
      const uintptr_t lo = reinterpret_cast<uintptr_t>(bufs[k].p);
      ranges.push_back({lo, lo + bufs[k].bytes, k > 0, i});
      o->buffers.push_back(bufs[k]);
    }
    first += (uint64_t)(t.n + 1) / 2;
    const int64_t count = ceil_div(t.n, kPiece);
    if ((int64_t)pieces.size() + count > INT32_MAX / 2)
      return Status::Err(AGN_E_INVALID, "too many elements for one plan");
    for (int64_t k = 0; k < count; ++k) pieces.push_back({i, (int32_t)k});
    host.push_back(d);
  }
  // What is written overlaps nothing (gradients may be the same memory).
  std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
  uintptr_t end = 0, end_written = 0;
  auto join = [](std::vector<std::pair<uintptr_t, uintptr_t>>& to, const Range& r) {
    if (!to.empty() && r.lo <= to.back().second) to.back().second = std::max(to.back().second, r.hi);
    else to.push_back({r.lo, r.hi});
  };
  for (const Range& r : ranges) {
    if ((r.written && r.lo < end) || r.lo < end_written)
      return Status::Err(AGN_E_INVALID, "tensor " + std::to_string(r.tensor) + ": a buffer overlaps another one");
    join(o->all, r);
    if (r.written) join(o->written, r);
    end = std::max(end, r.hi);
    if (r.written) end_written = std::max(end_written, r.hi);
  }
  AGN_TRY(current_device(&o->device));
  for (const CallBuffer& b : o->buffers) AGN_TRY(check_buffers({b}));
  int sms = 0;
  AGN_TRY(device_sms(o->device, &sms));
  o->tensors = (int64_t)host.size();
  o->pieces = (int)pieces.size();
  o->norm_grid = std::max(1, std::min({(int)ceil_div(o->pieces, kNormPieces), kMostGrid, 4 * sms}));
  AGN_TRY_CUDA(cudaMalloc(&o->d_tensors, host.size() * sizeof(Tensor) + 256));
  AGN_TRY_CUDA(cudaMalloc(&o->d_pieces, pieces.size() * sizeof(Piece) + 256));
  AGN_TRY_CUDA(cudaMalloc(&o->d_partials, (size_t)o->norm_grid * sizeof(double) + 256));
  if (!host.empty())
    AGN_TRY_CUDA(cudaMemcpy(o->d_tensors, host.data(), host.size() * sizeof(Tensor), cudaMemcpyHostToDevice));
  if (!pieces.empty())
    AGN_TRY_CUDA(cudaMemcpy(o->d_pieces, pieces.data(), pieces.size() * sizeof(Piece), cudaMemcpyHostToDevice));
  // (a copy from pageable memory may still be under way when it returns; later work of streams that
  // do not wait for the default one must find it done)
  AGN_TRY_CUDA(cudaStreamSynchronize(nullptr));
  *out = o.release();
  return Status::Ok();
}

// A call's own buffer shares no bytes with the plan's.
Status check_apart(const CallBuffer& b, const std::vector<std::pair<uintptr_t, uintptr_t>>& of) {
  if (!b.p || !b.bytes) return Status::Ok();
  const uintptr_t lo = reinterpret_cast<uintptr_t>(b.p);
  const auto next = std::upper_bound(of.begin(), of.end(), std::make_pair(lo, UINTPTR_MAX));
  if ((next != of.end() && next->first < lo + b.bytes) || (next != of.begin() && std::prev(next)->second > lo))
    return Status::Err(AGN_E_INVALID, std::string(b.name) + " overlaps a tensor's buffer");
  return Status::Ok();
}

Status plan_device(const agn_optim* o) {
  if (!o) return Status::Err(AGN_E_INVALID, "null plan");
  int dev = 0;
  AGN_TRY(current_device(&dev));
  if (dev != o->device) return Status::Err(AGN_E_INVALID, "the plan belongs to another device than the current one");
  return Status::Ok();
}

Status optim_norm(agn_optim* o, double max_norm, float* norm, float* scale, cudaStream_t st) {
  if (!(max_norm > 0.0)) return Status::Err(AGN_E_INVALID, "max_norm must be > 0");
  if (!norm && !scale) return Status::Err(AGN_E_INVALID, "null pointer");
  const CallBuffer nb{"norm", norm, norm ? sizeof(float) : 0, 4}, sb{"scale", scale, scale ? sizeof(float) : 0, 4};
  AGN_TRY(check_apart(nb, {sb}));
  AGN_TRY(plan_device(o));
  AGN_TRY(check_apart(nb, o->all));
  AGN_TRY(check_apart(sb, o->all));
  AGN_TRY(check_buffers({nb, sb}));
  KnownPlan plan(*o);
  KnownBuffers known({nb, sb});
  AGN_TRY(bounds_upload(st));
  AGN_TRY_CUDA(launch_pdl(norm_kernel, dim3((unsigned)o->norm_grid), dim3(kThreads), 0, st,
                          (const Tensor*)o->d_tensors, (const Piece*)o->d_pieces, o->pieces, o->d_partials));
  AGN_TRY_CUDA(launch_pdl(norm_finish_kernel, dim3(1), dim3(32), 0, st, (const double*)o->d_partials,
                          o->norm_grid, max_norm, norm, scale));
  return bounds_collect(st);
}

Status optim_step(agn_optim* o, double lr, int64_t step, double beta1, double beta2, double eps,
                  const float* scale, uint64_t seed, uint64_t offset, cudaStream_t st) {
  auto below_one = [](double b) { return b >= 0.0 && b < 1.0; };
  if (!(std::fabs(lr) <= 1e30) || step < 1 || !below_one(beta1) || !below_one(beta2) ||
      !(eps == 0.0 || (eps >= FLT_MIN && eps <= 1e30)))   // (smaller ones would keep few of their bits)
    return Status::Err(AGN_E_INVALID,
                       "need a finite lr, step >= 1, beta1 and beta2 in [0, 1), eps 0 or a normal fp32 number >= 0");
  const CallBuffer sb{"scale", scale, scale ? sizeof(float) : 0, 4};
  AGN_TRY(plan_device(o));
  if (!o->has_param && o->pieces > 0) return Status::Err(AGN_E_INVALID, "the plan has gradients alone");
  AGN_TRY(check_apart(sb, o->written));
  AGN_TRY(check_buffers({sb}));
  if (o->pieces == 0) return Status::Ok();
  StepArgs a{};
  a.tensors = o->d_tensors;
  a.pieces = o->d_pieces;
  a.n_pieces = o->pieces;
  a.b1 = (float)beta1; a.ob1 = (float)(1.0 - beta1);
  a.b2 = (float)beta2; a.ob2 = (float)(1.0 - beta2);
  a.eps = (float)eps;
  a.rc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
  a.size = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
  a.lr = lr;
  a.scale = scale;
  a.key = gen::key(seed, gen::kOptimState);
  a.offset = offset;
  int sms = 0;
  AGN_TRY(device_sms(o->device, &sms));
  KnownPlan plan(*o);
  KnownBuffers known({sb});
  AGN_TRY(bounds_upload(st));
  // (a round of resident blocks; 32 bits two: 40 M elements 188 us for 196)
  const dim3 grid((unsigned)std::min(o->pieces, (o->bits == 8 ? 4 : 8) * sms));
  // (8 bits: two, unless that takes a block longer; us for 100 M elements with one, two, four, eight at a time
  // 367, 335, 348, 375: pieces far apart cost the memory, single ones the loads ahead)
  auto longest = [&](int64_t group) { return ceil_div(o->pieces, grid.x * group) * group; };
  a.group = o->bits == 8 && longest(2) <= longest(1) + longest(1) / 16 ? 2 : 1;
  struct Tag {};
  if (o->bits == 8) {
    AGN_TRY_CUDA(allow_smem<Tag>(adamw_kernel<8>, 2 * sizeof(Slot), o->device));
    AGN_TRY_CUDA(launch_pdl(adamw_kernel<8>, grid, dim3(kThreads), 2 * sizeof(Slot), st, a));
  } else AGN_TRY_CUDA(launch_pdl(adamw_kernel<32>, grid, dim3(kThreads), 0, st, a));
  return bounds_collect(st);
}

Status dequantize(const uint8_t* m, const uint8_t* ms, const uint8_t* v, const uint8_t* vs, int64_t n,
                  void* m_out, void* r_out, int32_t dtype, cudaStream_t st) {
  const size_t es = dtype_size(dtype);
  if (!es) return Status::Err(AGN_E_INVALID, "unknown dtype");
  if (n < 0 || n > (int64_t)1 << 48) return Status::Err(AGN_E_INVALID, "n must be in [0, 2^48]");
  if (n == 0 || (!m_out && !r_out)) return Status::Ok();
  if ((m_out && (!m || !ms)) || (r_out && (!v || !vs))) return Status::Err(AGN_E_INVALID, "null pointer");
  const size_t nb = (size_t)ceil_div(n, kBlock);
  const CallBuffer cm{"m", m_out ? m : nullptr, (size_t)n, 1}, sm{"m_scale", m_out ? ms : nullptr, nb, 1},
      cv{"v", r_out ? v : nullptr, (size_t)n, 1}, sv{"v_scale", r_out ? vs : nullptr, nb, 1},
      om{"m_out", m_out, m_out ? (size_t)n * es : 0, es}, orr{"r_out", r_out, r_out ? (size_t)n * es : 0, es};
  AGN_TRY(check_apart(om, {cm, sm, cv, sv, orr}));
  AGN_TRY(check_apart(orr, {cm, sm, cv, sv}));
  AGN_TRY(check_buffers({cm, sm, cv, sv, om, orr}));
  KnownBuffers known({cm, sm, cv, sv, om, orr});
  AGN_TRY(bounds_upload(st));
  int dev = 0, sms = 0;
  AGN_TRY(current_device(&dev));
  AGN_TRY(device_sms(dev, &sms));
  const bool wide = aligned(m, 8) && aligned(v, 8) && aligned(m_out, 8 * es) && aligned(r_out, 8 * es);
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(n, kPiece), 16 * (int64_t)sms));
  if (dtype == AGN_PREC_FP32)
    AGN_TRY_CUDA(launch_pdl(dequantize_kernel<float>, grid, dim3(kThreads), 0, st, m, ms, v, vs, n,
                            static_cast<float*>(m_out), static_cast<float*>(r_out), wide));
  else
    AGN_TRY_CUDA(launch_pdl(dequantize_kernel<bf16>, grid, dim3(kThreads), 0, st, m, ms, v, vs, n,
                            static_cast<bf16*>(m_out), static_cast<bf16*>(r_out), wide));
  return bounds_collect(st);
}

}  // namespace
}  // namespace agn

extern "C" int agn_optim_create(const agn_optim_tensor* tensors, int32_t n_tensors, int32_t state_bits,
                                agn_optim** out) {
  return agn::guarded([&] { return agn::optim_create(tensors, n_tensors, state_bits, out); });
}

extern "C" int agn_optim_grad_norm(agn_optim* plan, double max_norm, float* norm, float* scale, void* stream) {
  return agn::guarded(
      [&] { return agn::optim_norm(plan, max_norm, norm, scale, static_cast<cudaStream_t>(stream)); });
}

extern "C" int agn_optim_adamw(agn_optim* plan, double lr, int64_t step, double beta1, double beta2,
                               double eps, const float* scale, uint64_t seed, uint64_t offset, void* stream) {
  return agn::guarded([&] {
    return agn::optim_step(plan, lr, step, beta1, beta2, eps, scale, seed, offset,
                           static_cast<cudaStream_t>(stream));
  });
}

extern "C" void agn_optim_destroy(agn_optim* plan) { delete plan; }

extern "C" int agn_adamw_dequantize(const uint8_t* m, const uint8_t* m_scale, const uint8_t* v,
                                    const uint8_t* v_scale, int64_t n, void* m_out, void* r_out,
                                    int32_t dtype, void* stream) {
  return agn::guarded([&] {
    return agn::dequantize(m, m_scale, v, v_scale, n, m_out, r_out, dtype, static_cast<cudaStream_t>(stream));
  });
}
