// What the kernels of decayed linear attention and of draft verification share: their launch, and a request's token range.
#pragma once
#include <cuda_bf16.h>

#include "dasc_internal.h"
#include "launch.cuh"

// launch_in_order (see launch.cuh) with a cluster of `cluster` thread blocks along x.
template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kernel)(P...), dim3 grid, dim3 block, unsigned cluster, size_t smem, void *stream, const A &...args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}
template <typename... P, typename... A>
cudaError_t launch_blocks(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, void *stream, const A &...args) {
  return launch_in_order(kernel, grid, block, smem, stream, args...);
}

// Request r's first token in the streams of a layer, and how many of its tokens are run.
struct DecayRange {
  int64_t begin;
  int32_t n;
};
__device__ __forceinline__ DecayRange decay_range(const DascDecayArgs &a, int r) {
  if (!a.cu_seqlens) return {r, 1};
  const int32_t b = a.cu_seqlens[r];
  int32_t n = max(a.cu_seqlens[r + 1] - b, 0);
  if (a.seq_used) n = min(n, max(a.seq_used[r], 0));
  return {b, n};
}

// `bytes` bytes (a multiple of 16) into L2 only.
__device__ __forceinline__ void bulk_prefetch(const void *src, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}

// packed pairs of fp32 (one instruction per pair)
__device__ __forceinline__ uint64_t dpack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 dunpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t dsub2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t dmul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t dfma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
