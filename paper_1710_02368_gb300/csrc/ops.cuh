// What the entry points on the caller's device buffers share (dropout.cu,
// mx4.cu, mx4_linear.cu): checks of the arguments, the bounds-checked build's
// buffers of a call, launches with a cluster.
#pragma once

#include <initializer_list>
#include <new>
#include <string>

#include "common.cuh"

namespace agn {

void set_global_error(const std::string& msg);   // agn_api.cu: agn_last_error(NULL)

// A caller's buffer of a call: `bytes` from p on (p null: not given).
struct CallBuffer {
  const char* name;
  const void* p;
  size_t bytes;
  size_t align;
};

// Element size of a dtype argument (AGN_PREC_FP32, AGN_PREC_BF16), 0 for any other.
inline size_t dtype_size(int dtype) {
  return dtype == AGN_PREC_FP32 ? 4 : dtype == AGN_PREC_BF16 ? 2 : 0;
}

// Bytes of [rows][cols] elements with row stride ld (0 for an empty matrix).
inline size_t matrix_bytes(int64_t rows, int64_t cols, int64_t ld, size_t es) {
  return rows > 0 && cols > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * es : 0;
}

// Sizes whose byte offsets stay well inside 63 bits.
inline Status check_matrix(const char* name, int64_t rows, int64_t cols, int64_t ld) {
  if (rows < 0 || cols < 0 || cols > INT32_MAX)
    return Status::Err(AGN_E_INVALID, std::string(name) + ": rows and columns must be >= 0, columns < 2^31");
  if (ld < cols) return Status::Err(AGN_E_INVALID, std::string(name) + ": row stride shorter than a row");
  if (rows > 0 && ld > 0 && rows > ((int64_t)1 << 58) / ld)
    return Status::Err(AGN_E_INVALID, std::string(name) + ": too large");
  return Status::Ok();
}

inline bool overlaps(const void* a, size_t an, const void* b, size_t bn) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && an && bn && x < y + bn && y < x + an;
}

// Every buffer is aligned and lies in memory of the current device (a host
// pointer, or memory of another device, would fault in the kernel).
inline Status check_buffers(std::initializer_list<CallBuffer> bufs) {
  for (const CallBuffer& b : bufs)
    if (b.p && reinterpret_cast<uintptr_t>(b.p) % b.align != 0)
      return Status::Err(AGN_E_INVALID, std::string(b.name) + " must be " + std::to_string(b.align) +
                                            "-byte aligned");
  int dev = -1;
  AGN_TRY_CUDA(cudaGetDevice(&dev));
  for (const CallBuffer& b : bufs) {
    if (!b.p || !b.bytes) continue;
    cudaPointerAttributes at{};
    AGN_TRY_CUDA(cudaPointerGetAttributes(&at, b.p));
    if (at.type != cudaMemoryTypeManaged && (at.type != cudaMemoryTypeDevice || at.device != dev))
      return Status::Err(AGN_E_INVALID,
                         std::string(b.name) + " is not memory of the current device");
  }
  return Status::Ok();
}

// No output shares bytes with another buffer.  `same`: outputs may be exactly
// the first buffer of `ins` (in place).
inline Status check_apart(const CallBuffer& out, std::initializer_list<CallBuffer> others) {
  for (const CallBuffer& b : others)
    if (overlaps(out.p, out.bytes, b.p, b.bytes))
      return Status::Err(AGN_E_INVALID, std::string(out.name) + " overlaps " + b.name);
  return Status::Ok();
}

// Bounds-checked build: a call's buffers are known while it lasts.
struct KnownBuffers {
  const void* p[8] = {};
  int k = 0;
  explicit KnownBuffers(std::initializer_list<CallBuffer> bufs) {
    for (const CallBuffer& b : bufs)
      if (b.p && b.bytes && k < 8) {
        bounds_add(b.p, b.bytes);
        p[k++] = b.p;
      }
  }
  KnownBuffers(const KnownBuffers&) = delete;
  KnownBuffers& operator=(const KnownBuffers&) = delete;
  ~KnownBuffers() {
    for (int i = 0; i < k; ++i) bounds_remove(p[i]);
  }
};

// What is asked of a device is asked once and kept by its ordinal (the current device's in these
// calls), but for an answer that is an error: the call returns it and the next one asks again.
// (A stand-in would decide clusters, and with them the order of sums, for every later call.)
constexpr int kMaxDevices = 64;   // ordinals from here on are asked every time

inline bool kept_device(int dev) { return dev >= 0 && dev < kMaxDevices; }

inline Status current_device(int* dev) {
  AGN_TRY_CUDA(cudaGetDevice(dev));
  return Status::Ok();
}

inline Status device_sms(int dev, int* sms) {
  static std::atomic<int> known[kMaxDevices];
  if (kept_device(dev) && (*sms = known[dev].load(std::memory_order_relaxed)) > 0) return Status::Ok();
  AGN_TRY_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
  if (*sms < 1) return Status::Err(AGN_E_CUDA, "the device reports no multiprocessors");
  if (kept_device(dev)) known[dev].store(*sms, std::memory_order_relaxed);
  return Status::Ok();
}

// Lets a kernel have `smem` bytes of dynamic shared memory (a Tag for each kernel).
template <typename Tag, typename... KArgs>
cudaError_t allow_smem(void (*kern)(KArgs...), size_t smem, int dev) {
  static std::atomic<int> done[kMaxDevices];
  if (kept_device(dev) && done[dev].load(std::memory_order_relaxed)) return cudaSuccess;
  const cudaError_t e =
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess && kept_device(dev)) done[dev].store(1, std::memory_order_relaxed);
  return e;
}

// *n: clusters of c blocks, 2 to 16 (along y; more than the portable 8 are allowed for the kernel
// first), of this kernel that are resident at once on the current device: fewer blocks than single
// ones, since a cluster stays within a GPC (a block to an SM: 152 single ones, 36 clusters of four,
// 15 of eight); 0 where they cannot be.  Kept for each Tag and device.
template <typename Tag, typename... KArgs>
Status max_clusters(void (*kern)(KArgs...), int threads, size_t smem, int c, int dev, int* n) {
  static std::atomic<int> known[kMaxDevices][17];   // + 1
  if (c < 2 || c > 16) return Status::Err(AGN_E_INVALID, "clusters have 2 to 16 blocks");
  if (kept_device(dev) && (*n = known[dev][c].load(std::memory_order_relaxed) - 1) >= 0) return Status::Ok();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1, (unsigned)c, 1);
  cfg.blockDim = threads;
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1;
  attr[0].val.clusterDim.y = (unsigned)c;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (smem > 0)
    AGN_TRY_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  if (c > 8) AGN_TRY_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  AGN_TRY_CUDA(cudaOccupancyMaxActiveClusters(n, kern, &cfg));
  if (kept_device(dev)) known[dev][c].store(*n + 1, std::memory_order_relaxed);
  return Status::Ok();
}

// launch_pdl with clusters of `cluster` blocks.
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl_cluster(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem,
                               dim3 cluster, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster.x;
  attr[0].val.clusterDim.y = cluster.y;
  attr[0].val.clusterDim.z = cluster.z;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = g_pdl_off.load(std::memory_order_relaxed) > 0 ? 1 : 2;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<Args>(args)...);
}

// Runs an entry point's body: its status as the C code, the message kept (and
// the runtime's last error cleared, which a later launch check of the caller's
// would take for its own).
template <typename F>
int guarded(F&& body) {
  Status s;
  try {
    s = body();
    if (s.code == AGN_E_CUDA || s.code == AGN_E_OOM) cudaGetLastError();
    if (!s.ok()) set_global_error(s.msg);
  } catch (const std::exception&) {
    s.code = AGN_E_OOM;
    try {
      set_global_error("host allocation failed");
    } catch (...) {
    }
  }
  return s.code;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// Every thread of every CTA of the cluster.  The barrier's aligned form asks for a converged warp,
// which loops that lanes leave on different trips do not give.
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;"
               ::: "memory");
}
// A float of CTA `rank`'s shared memory, at this CTA's own address p.
__device__ __forceinline__ float ld_cluster(const float* p, uint32_t rank) {
  const uint32_t own = static_cast<uint32_t>(__cvta_generic_to_shared(p));
  uint32_t at;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(own), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

}  // namespace agn
