// Running sums over a block of 1024 threads, and the block that is the last of a launch.
#pragma once
#include <cuda_runtime.h>

namespace hs {
namespace {

// Exclusive running sums over the block's threads of a pair of counts below 2^31, packed in 64 bits; `total` is the same in every thread.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long* warp_sums, unsigned long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long x = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += x;
  }
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  unsigned long long w = warp_sums[lane];               // (32 warps)
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long x = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += x;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  const unsigned long long before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
  return (warp > 0 ? before : 0ull) + inc - v;
}

__device__ __forceinline__ bool last_block(int* done) {
  __shared__ int last;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(done, 1) == int(gridDim.x) - 1;
    if (last) *done = 0;                                 // ready for the next call
    __threadfence();
  }
  __syncthreads();
  return last != 0;
}

}  // namespace
}  // namespace hs
