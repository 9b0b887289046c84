// Running sums over the one workgroup that plans a call.
#pragma once
#include "common.h"

namespace scout {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int x, int lane) {
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const int y = __shfl_up(x, s);
    if (lane >= s) x += y;
  }
  return x;
}

// Exclusive sum over the threads of the planning workgroup, and the total; `lds`: kPlanWaves words.
__device__ __forceinline__ int plan_scan(int x, int* lds, int* total) {
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int inc = wave_scan(x, lane);
  __syncthreads();  // the words may still be read from the call before
  if (lane == kWave - 1) lds[wave] = inc;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const int t = lds[w];
    before += w < wave ? t : 0;
    all += t;
  }
  *total = all;
  return before + inc - x;
}

}  // namespace scout
