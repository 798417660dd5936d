// What the kernels of attention over many query rows share: the 32x32x16 product, and tiles of 64 rows of 128 16-bit values in local memory.
#pragma once

#include "common.h"

namespace minikv {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr int kPfD = 128;            // head dimension
constexpr int kPfN = 64;             // keys (forward) / queries (column sums) per LDS tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// 16-bit operands are kept as halves whatever they are; BF16 instances differ in the product and in the two roundings (a product's operands
// are of one type, and bf16 values leave fp16's range, so the weights have bf16's 8 bits there).
typedef __bf16 bfloat8 __attribute__((ext_vector_type(8)));

template <bool BF16 = false>
__device__ __forceinline__ float16v mfma32(half8 a, half8 b, float16v c)
{
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bfloat8, a), __builtin_bit_cast(bfloat8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
template <bool BF16>
__device__ __forceinline__ _Float16 to16(float v)
{
    if constexpr (BF16) return __builtin_bit_cast(_Float16, (__bf16)v);
    else return (_Float16)v;
}

// Row of accumulator element i (0..15) inside a 32x32 result tile, for a lane of half-wave g.
__device__ __forceinline__ int acc_row(int i, int g) { return (i >> 2) * 8 + g * 4 + (i & 3); }

// Tiles in local memory have unpadded rows of 256 bytes; chunk k (16 bytes) of row r sits at place k ^ (r & 15), so
// that the fragment reads of 32 consecutive rows use all banks evenly.
__device__ __forceinline__ int tile_place(int row, int chunk) { return row * kPfD + ((chunk ^ (row & 15)) << 3); }

constexpr int kPfTile = kPfN * kPfD;                    // halves of one unpadded tile in LDS

// Place (in halves) of 16-byte chunk k of row `key` in a V tile: the rows 4j .. 4j+3 that one transposing read takes
// fall on different banks.
__device__ __forceinline__ int v_swizzle(int key) { return 4 * (key & 3) + 2 * ((key >> 1) & 1); }

typedef __fp16 fp16x4 __attribute__((__vector_size__(8)));
__device__ __forceinline__ half4 read_transposed(const _Float16 *p)
{
    return (half4)__builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) fp16x4 *)p);
}

// Local memory that one wave writes and reads: its operations are done in order, the compiler is told to keep them so.
__device__ __forceinline__ void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

}  // namespace minikv
