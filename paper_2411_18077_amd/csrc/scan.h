// Prefix sums over the threads of a workgroup of the kernels that build block tables.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace minikv {

constexpr int kScanThreads = 1024;

// Sums saturate: lengths come from the device and may be anything, what is indexed with them may not.  (a, b <= cap < 2^31;
// min(a + b, cap) is associative, so a scan in any order gives the same.)
__device__ inline uint32_t sat_add(uint32_t a, uint32_t b, uint32_t cap) { return min(a + b, cap); }
template <int CTRL, int ROWS> __device__ inline uint32_t sat_step(uint32_t v, uint32_t cap)
{
    return sat_add(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false), cap);
}
__device__ inline uint32_t wave_scan(uint32_t v, uint32_t cap)         // inclusive
{
    v = sat_step<0x111, 0xf>(v, cap), v = sat_step<0x112, 0xf>(v, cap);              // row_shr 1, 2, 4, 8
    v = sat_step<0x114, 0xf>(v, cap), v = sat_step<0x118, 0xf>(v, cap);
    return sat_step<0x143, 0xc>(sat_step<0x142, 0xa>(v, cap), cap);                    // row_bcast 15, 31
}

// exclusive scans over the workgroup's threads of N values at once; `total` receives the whole sums
template <int N>
__device__ inline void block_scan(uint32_t (&v)[N], const uint32_t (&cap)[N], uint32_t (*part)[kScanThreads / 64], uint32_t (&total)[N])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t in[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        in[i] = wave_scan(v[i], cap[i]);
        if (lane == 63) part[i][wave] = in[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {                      // (the sixteen sums are one more scan, in every wave)
        const uint32_t sums = wave_scan(lane < kScanThreads / 64 ? part[i][lane] : 0, cap[i]);
        total[i] = __builtin_amdgcn_readlane(sums, kScanThreads / 64 - 1);
        const uint32_t before = wave ? (uint32_t)__shfl((int)sums, wave - 1, 64) : 0;
        const uint32_t ex = __builtin_amdgcn_update_dpp(0, in[i], 0x138, 0xf, 0xf, false);     // wave_shr 1
        v[i] = sat_add(before, lane ? ex : 0, cap[i]);
    }
}

}  // namespace minikv
