// Norms of queries and keys for each head with the position rotation in the same pass (minikv_norm_rope).
//
//   y = x * rsqrt(mean(x^2) + eps) * w        (w NULL: y = x)
//   the first rot channels in pairs (u, v), pair i turned by a = pos * inv_freq[i]:  u cos a - v sin a,  v cos a + u sin a
//
// Sixteen lanes hold a row, eight channels each, four rows a load.  The sum of squares crosses the sixteen lanes by DPP; where the pairs are
// channels i and rot/2 + i, the other half of a pair comes from another lane as the two bytes it was loaded as (the row's norm is
// the same there, the weight is a register).  All in binary32, rounded once at the end.
//
// Angles.  A far position times a frequency has more bits than binary32: pos * inv_freq / (2 pi) is formed in binary64 and whole turns are dropped
// there.  For angles up to 2^31 the product's rounding and that of 1 / (2 pi) leave 2^-21.3 of a radian, and what is left of a turn goes on in binary32,
// rounded to 2^-26 of a turn.  Sine and cosine of the eighth of a turn around the nearest
// quarter are their Taylor sums up to x^9 and x^8 (the next terms are below 2^-28 and 2^-25 at pi/4); quarters swap and negate them.  A token's
// angles are formed once per wave, which takes several heads.
//
// What bounds it: memory (32768 tokens of 40 heads 122 us, 5.5 TB/s), for few tokens two dependent round trips (64 of 40 heads 3.7 us).
#include "decode_common.h"

namespace minikv {

typedef uint32_t u4n __attribute__((ext_vector_type(4)));

// Loads of four rows that a wave has under way at once: 32768 tokens of 40 heads 122 us with three, 124 with five, 126 with ten; 4096 18.7, 18.0, 17.8.
constexpr int kNrQuads = 3;

struct NormArgs {
    const uint16_t *X[2];                              // Q and K rows
    uint16_t *Y[2];
    int64_t x_stride[2], y_stride[2];
    const uint16_t *w[2];
    const float *inv_freq;
    const int32_t *pos;
    int T, Hq, rows, rot, quads;                       // rows = Hq + Hkv; quads: of a wave
    float eps;
    uint32_t split, split_magic, split_shift;          // waves of a token
};

template <bool BF16> __device__ inline float nr_from(uint32_t bits)
{
    if (BF16) return __uint_as_float(bits << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
template <bool BF16> __device__ inline uint32_t nr_to(float lo, float hi)
{
    if constexpr (BF16) {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, bf2{(__bf16)lo, (__bf16)hi});
    } else {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, h2{(_Float16)lo, (_Float16)hi});
    }
}
template <int CTRL> __device__ inline float add_ror(float v)
{
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, false));
}

__device__ inline void turn(int pos, float freq, float &c, float &s)
{
    constexpr double kTurn = 0.15915494309189533577;
    const double angle = (double)pos * (double)freq;
    const float part = (float)__builtin_fma(angle, kTurn, -__builtin_rint(angle * kTurn));              // [-1/2, 1/2]
    const float quarter = __builtin_rintf(4.0f * part), x = __builtin_fmaf(-0.25f, quarter, part) * 6.28318530717958647692f, z = x * x;
    const float sn = x * __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), 1.0f);
    const float cs = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.0f / 40320, -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
    const int q = (int)quarter & 3;
    const float a = q & 1 ? sn : cs, b = q & 1 ? cs : sn;
    c = q == 1 || q == 2 ? -a : a;
    s = q & 2 ? -b : b;
}

// A wave takes `quads` times four heads (Q's first, K's behind them) of one token.
template <bool BF16, bool ADJACENT>
__global__ __launch_bounds__(256) void norm_rope_kernel(NormArgs a)
{
    const int lane = threadIdx.x & 63, chunk = lane & 15, sub = lane >> 4;
    const uint32_t item = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t token = fast_div(item, a.split_magic, a.split_shift);
    if (token >= (uint32_t)a.T) return;
    const int t = (int)token, first = (int)(item - token * a.split) * a.quads * 4, end = min(first + a.quads * 4, a.rows);

    const uint16_t *in[2];
    uint16_t *out[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) in[k] = a.X[k] + t * a.x_stride[k] + chunk * 8, out[k] = a.Y[k] + t * a.y_stride[k] + chunk * 8;
    u4n x[kNrQuads];
    auto load = [&](int base) {
#pragma unroll
        for (int i = 0; i < kNrQuads; ++i)
            if (base + 4 * i < end) {
                const int row = min(base + 4 * i + sub, end - 1);
                x[i] = *(const u4n *)(row < a.Hq ? in[0] + row * kD : in[1] + (row - a.Hq) * kD);
            }
    };
    load(first);
    const int pos = a.pos[t];
    if (pos < 0) return;

    // the lane's part in the rotation: partner lane (itself behind the rotated channels), and cosines and sines by channel or by pair
    const int half = a.rot >> 4;                       // of the rotated chunks
    const bool turned = chunk < 2 * half;
    const int other = ADJACENT || !turned ? chunk : chunk < half ? chunk + half : chunk - half;
    constexpr int kAngles = ADJACENT ? 4 : 8;
    float c[kAngles], s[kAngles];
#pragma unroll
    for (int j = 0; j < kAngles; ++j) c[j] = 1.0f, s[j] = 0.0f;
    if (turned) {
        const float *freq = a.inv_freq + (ADJACENT ? chunk * 4 : (chunk < half ? chunk : chunk - half) * 8);
#pragma unroll
        for (int j = 0; j < kAngles; ++j) turn(pos, freq[j], c[j], s[j]);
        if (!ADJACENT && chunk < half)
#pragma unroll
            for (int j = 0; j < kAngles; ++j) s[j] = -s[j];
    }
    u4n w[2], w_other[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (a.w[k]) {
            w[k] = *(const u4n *)(a.w[k] + chunk * 8);
            if (!ADJACENT) w_other[k] = *(const u4n *)(a.w[k] + other * 8);
        }
    const int from = ((lane & 48) + other) << 2;

    for (int base = first; base < end; base += 4 * kNrQuads) {
        if (base > first) load(base);
#pragma unroll
        for (int i = 0; i < kNrQuads; ++i) {
            if (base + 4 * i >= end) break;
            const int row = base + 4 * i + sub;
            const bool is_k = row >= a.Hq;
            float v[8], u[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[2 * j] = nr_from<BF16>(x[i][j] & 0xffff), v[2 * j + 1] = nr_from<BF16>(x[i][j] >> 16);
            if (!ADJACENT) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t p = __builtin_amdgcn_ds_bpermute(from, x[i][j]);
                    u[2 * j] = nr_from<BF16>(p & 0xffff), u[2 * j + 1] = nr_from<BF16>(p >> 16);
                }
            }
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(v[j], v[j], sum);
            sum = add_ror<0x121>(add_ror<0x122>(add_ror<0x124>(add_ror<0x128>(sum))));       // row_ror 8, 4, 2, 1
            if (is_k ? a.w[1] != nullptr : a.w[0] != nullptr) {
                const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, 1.0f / kD, a.eps));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t g = is_k ? w[1][j] : w[0][j];
                    v[2 * j] *= r * nr_from<BF16>(g & 0xffff), v[2 * j + 1] *= r * nr_from<BF16>(g >> 16);
                    if (!ADJACENT) {
                        const uint32_t h = is_k ? w_other[1][j] : w_other[0][j];
                        u[2 * j] *= r * nr_from<BF16>(h & 0xffff), u[2 * j + 1] *= r * nr_from<BF16>(h >> 16);
                    }
                }
            }
            u4n y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = v[2 * j], q = v[2 * j + 1];
                if (ADJACENT)
                    y[j] = nr_to<BF16>(p * c[j] - q * s[j], q * c[j] + p * s[j]);
                else
                    y[j] = nr_to<BF16>(p * c[2 * j] + u[2 * j] * s[2 * j], q * c[2 * j + 1] + u[2 * j + 1] * s[2 * j + 1]);
            }
            if (row < end) *(u4n *)(is_k ? out[1] + (row - a.Hq) * kD : out[0] + row * kD) = y;
        }
    }
}

int launch_norm_rope(int32_t Hq, int32_t Hkv, int32_t T, int32_t dtype, const void *Q, int64_t q_stride, const void *K, int64_t k_stride,
                     const void *w_q, const void *w_k, float eps, const float *inv_freq, int32_t rot, int32_t adjacent, const int32_t *pos,
                     void *Q_out, int64_t q_out_stride, void *K_out, int64_t k_out_stride, hipStream_t st)
{
    NormArgs a;
    a.X[0] = (const uint16_t *)Q, a.X[1] = (const uint16_t *)K, a.Y[0] = (uint16_t *)Q_out, a.Y[1] = (uint16_t *)K_out;
    a.x_stride[0] = q_stride, a.x_stride[1] = k_stride, a.y_stride[0] = q_out_stride, a.y_stride[1] = k_out_stride;
    a.w[0] = (const uint16_t *)w_q, a.w[1] = (const uint16_t *)w_k, a.inv_freq = inv_freq, a.pos = pos;
    a.T = T, a.Hq = Hq, a.rows = Hq + Hkv, a.rot = rot, a.eps = eps;
    // One quad of rows a wave while that makes no more than eight waves a compute unit, then more.  Us with 4, 8, 16, 64 waves, 40 heads: 777 tokens
    // 7.6, 6.5, 7.8, 7.7, 2048 11.5, 11.4, 11.2, 15.9; 777 of 16 heads 4.4, 4.8, 4.8, 4.8.
    const int64_t all = (a.rows + 3) / 4, share = T * all / (kComputeUnits * 8);
    a.quads = (int)(share < 1 ? 1 : share < all ? share : all);
    a.split = (uint32_t)((all + a.quads - 1) / a.quads);
    fast_div_setup(a.split, a.split_magic, a.split_shift);
    const dim3 grid((unsigned)(((int64_t)T * a.split + 3) / 4));
    const bool bf16 = dtype == MINIKV_BF16;
    if (bf16 && adjacent) hipLaunchKernelGGL((norm_rope_kernel<true, true>), grid, dim3(256), 0, st, a);
    else if (bf16) hipLaunchKernelGGL((norm_rope_kernel<true, false>), grid, dim3(256), 0, st, a);
    else if (adjacent) hipLaunchKernelGGL((norm_rope_kernel<false, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((norm_rope_kernel<false, false>), grid, dim3(256), 0, st, a);
    return hipGetLastError() == hipSuccess ? MINIKV_OK : MINIKV_ELAUNCH;
}

}  // namespace minikv
