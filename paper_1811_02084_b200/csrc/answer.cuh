// What the kernels of answering share: waits for copies into shared memory, and other blocks' shared memory.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "per_device.h"

namespace mtf {

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Waits are bounded: behind one that was given up a kernel records a code for mtf_device_status, gives the copies under way a little more time and ends; what it writes is unspecified.
constexpr long long kWaitCycles = 4000000000LL;      // about two seconds
constexpr long long kLandCycles = 200000000LL;       // 0.1 s, for copies in flight
__device__ __forceinline__ void landing_init(const uint64_t* bar) { asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_at(bar)) : "memory"); }
__device__ __forceinline__ void landing_ready() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool has_landed(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
static __device__ __noinline__ bool landed_late(uint32_t bar, uint32_t parity, long long limit) {
  const long long t0 = clock64();
  while (!has_landed(bar, parity))
    if (clock64() - t0 > limit) return false;
  return true;
}
// A whole warp's wait; the same for all lanes.
__device__ __forceinline__ bool landed(uint32_t bar, uint32_t parity, const long long& limit) {
  const bool ok = has_landed(bar, parity);
  if (__all_sync(0xffffffffu, ok)) return true;
  return __all_sync(0xffffffffu, landed_late(bar, parity, limit));
}

// Another block's shared memory, and the barrier of all threads of the cluster.
__device__ __forceinline__ uint32_t in_block(uint32_t at, int rank) {
  uint32_t x;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(x) : "r"(at), "r"(rank));
  return x;
}
__device__ __forceinline__ float far(uint32_t at) {
  float x;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ float2 far2(uint32_t at) {
  float2 x;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The shared memory that a kernel may have, always the same number: set once a device, as `known` has it.
template <typename K>
cudaError_t shared_memory_limit(KnownPerDevice& known, K* kernel, int bytes) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  known.get(dev, [&] {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e == cudaSuccess ? 1 : 0;
  });
  return e;
}

// A launch that may be set up while the one before it drains, as clusters of so many blocks.
template <typename... P, typename... A>
void launch_clusters(void (*kernel)(P...), dim3 grid, unsigned block, size_t smem, int cluster, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace mtf
