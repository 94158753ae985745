// Shared by the language-model operators (internal): element types, checks of arguments.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>
#include <mutex>

#include "../../include/gem_lm.h"
#include "pdl.h"

namespace gem {
namespace lm {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

// Rounds to nearest even; fp16 overflows to infinity.
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// V floats; for V = 2 sums and products are one packed instruction on the pair.
template <int V>
struct Vec {
  float v[V];
};

__device__ __forceinline__ uint64_t bits(const Vec<2>& a) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.v[0]), "f"(a.v[1]));
  return r;
}
__device__ __forceinline__ Vec<2> pair(uint64_t r) {
  Vec<2> a;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a.v[0]), "=f"(a.v[1]) : "l"(r));
  return a;
}

template <int V>
__device__ __forceinline__ Vec<V> splat(float x) {
  Vec<V> r;
#pragma unroll
  for (int k = 0; k < V; ++k) r.v[k] = x;
  return r;
}

template <int V>
__device__ __forceinline__ Vec<V> fma(const Vec<V>& a, const Vec<V>& b, const Vec<V>& c) {
  if constexpr (V == 2) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
    return pair(r);
  } else {
    return {fmaf(a.v[0], b.v[0], c.v[0])};
  }
}
template <int V>
__device__ __forceinline__ Vec<V> operator*(const Vec<V>& a, const Vec<V>& b) {
  if constexpr (V == 2) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
    return pair(r);
  } else {
    return {a.v[0] * b.v[0]};
  }
}
template <int V>
__device__ __forceinline__ Vec<V> operator+(const Vec<V>& a, const Vec<V>& b) {
  if constexpr (V == 2) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
    return pair(r);
  } else {
    return {a.v[0] + b.v[0]};
  }
}
template <int V>
__device__ __forceinline__ Vec<V> operator-(const Vec<V>& a, const Vec<V>& b) {
  return fma<V>(b, splat<V>(-1.0f), a);
}

inline int dtype_size(int dtype) { return dtype == GEM_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == GEM_F32 || dtype == GEM_BF16 || dtype == GEM_F16; }

inline bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// A required / an optional array of 4-byte values.
inline bool array_ok(const void* p) { return p && aligned_to(p, 4); }
inline bool optional_ok(const void* p) { return aligned_to(p, 4); }

// Sizes and strides that 64-bit offsets hold with room to spare.
constexpr int64_t kMaxExtent = int64_t(1) << 31;
constexpr int64_t kMaxStride = int64_t(1) << 46;

inline bool extent_ok(int64_t n) { return n >= 0 && n < kMaxExtent; }

// Channels of which 32-bit indices hold those of a whole block past the last.
inline bool channels_ok(int64_t D) { return D >= 0 && D <= int64_t(1) << 30; }

// An input: any strides (0: one step or sequence for all).
inline bool input_ok(const gem_seq_t* s, int dtype, int64_t B, int64_t T, int64_t D) {
  if (!s) return false;
  if (B == 0 || T == 0 || D == 0) return true;
  if (!s->data || !aligned_to(s->data, size_t(dtype_size(dtype)))) return false;
  if (B > 1 && (s->stride_b < 0 || s->stride_b > kMaxStride / B)) return false;
  if (T > 1 && (s->stride_t < 0 || s->stride_t > kMaxStride / T)) return false;
  return true;
}

// An output: its elements also have places of their own.
inline bool output_ok(const gem_seq_t* s, int dtype, int64_t B, int64_t T, int64_t D) {
  if (!input_ok(s, dtype, B, T, D)) return false;
  if (B == 0 || T == 0 || D == 0) return true;
  const int64_t sb = s->stride_b, st = s->stride_t;
  if (T == 1) return B == 1 || sb >= D;
  if (B == 1) return st >= D;
  return (st >= D && sb >= (T - 1) * st + D) || (sb >= D && st >= (B - 1) * sb + D);
}

// Most dynamic shared memory of a block of these kernels: 227 KB less their static shared memory (up to
// 8.3 KB).
constexpr size_t kMaxShared = 216 << 10;

// Lets a kernel be launched with up to MOST of dynamic shared memory (LARGE: and in clusters of
// more than 8 blocks).  Asked of the runtime once for each kernel and device.
template <auto KERNEL, bool LARGE = false, size_t MOST = kMaxShared>
cudaError_t allow_shared(size_t bytes) {
  if (bytes > MOST) return cudaErrorInvalidValue;
  if (!LARGE && MOST == kMaxShared && bytes <= 32 << 10) return cudaSuccess;   // within the 48 KB that need no permission
  static std::atomic<uint64_t> allowed{0};
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const uint64_t bit = uint64_t(1) << (device & 63);
  if (device < 64 && (allowed.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, int(MOST));
  if (LARGE && e == cudaSuccess) e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess && device < 64) allowed.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// launch_pdl for a grid of clusters of `cluster` blocks.
template <typename... KArgs, typename... Args>
cudaError_t launch_cluster_pdl(void (*kernel)(KArgs...), unsigned blocks, unsigned threads, unsigned cluster, size_t smem,
                               cudaStream_t stream, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

// Clusters of a kernel that the GPU holds at once (asked of the runtime once for each shape).
inline cudaError_t resident_clusters(const void* kernel, int cluster, int threads, size_t shared, int* clusters) {
  struct Known {
    const void* kernel;
    int device, cluster, threads, clusters;
    size_t shared;
  };
  static std::mutex mutex;
  static Known known[64];
  static int count = 0;
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  std::lock_guard<std::mutex> lock(mutex);
  for (const Known& k : known)
    if (k.kernel == kernel && k.device == device && k.cluster == cluster && k.threads == threads && k.shared == shared) {
      *clusters = k.clusters;
      return cudaSuccess;
    }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(cluster));
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = shared;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = unsigned(cluster);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaOccupancyMaxActiveClusters(clusters, kernel, &cfg);
  if (e != cudaSuccess) return e;
  known[count++ % 64] = {kernel, device, cluster, threads, *clusters, shared};
  return cudaSuccess;
}

// Ends a call: a launch that failed is reported, and its error is not left for the caller's
// next check.
inline int launch_status(cudaError_t e) {
  if (e == cudaSuccess) return GEM_OK;
  cudaGetLastError();
  return GEM_ECUDA;
}

// Calls F<E>(...) for the element type `dtype`.
#define BY_TYPE(F, ...) \
  (dtype == GEM_F32 ? F<float>(__VA_ARGS__) : dtype == GEM_BF16 ? F<__nv_bfloat16>(__VA_ARGS__) : F<__half>(__VA_ARGS__))

}  // namespace lm
}  // namespace gem
