// Attention of one query token per request over the paged 8-bit cache (minikv_decode_attn_blk).
//
// The products have 1 to 8 query heads on one side (the heads of a KV head), which the 16x16x32 matrix instruction takes
// with the keys: S^T = K Q^T and O^T = V^T P^T, the tokens and then the channels as its rows, the heads as its columns.
// The 16 columns hold the heads twice, and the two copies stand for two halves of a tile's tokens:
//   scores   A = 16 tokens x 32 channels of K (a lane's two 16-byte loads of one token row, codes to 16 bits by one
//            conversion per pair, exact), B = the queries.  A lane (n, g) receives tokens 4g .. 4g+3 of each 16 for head
//            n % 8; lanes n < 8 go on with tokens 0..31 of the tile, the others with 32..63: eight weights a lane.
//   output   B = those eight weights as they are, no exchange between lanes.  A must then hold, for the row of lane
//            (n, g), the same eight tokens: a lane loads 16 channels of eight tokens, a row of V per eight lanes, and
//            transposes 4x4 bytes with byte permutes; rows n < 8 belong to the first half of the tokens, the others to
//            the second.  Of the 16 x 16 results the two quadrants whose row and column belong to one half count.
// So every lane of the instruction works, loads are whole rows and neither K, V nor the weights pass through local memory.
//
// Weights are rounded to fp16 for the second product (relative 2^-11, to nearest, the sum of weights is kept in fp32 from
// the unrounded ones), scaled by the block's V scale over the largest one seen so far: at most 1, whatever the scales.
#include "common.h"

#include <type_traits>

namespace minikv {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float f4v __attribute__((ext_vector_type(4)));

constexpr int kBkThreads = 256;
constexpr int kBkRow = kD + 4;                         // floats of a head's state in local memory: m, l, 2 pad, o
constexpr float kBkNone = -3.0e38f;                    // running maximum before the first token: finite, so that no difference is NaN

struct BlkArgs {
    const uint16_t *q;
    int64_t q_stride;
    const uint8_t *K, *V;
    const float *Ks, *Vs;
    const int32_t *table, *q_len;
    uint16_t *out;
    int *tickets;                                      // [kBlkGroups]
    float *partials;                                   // [2 * kBlkGroups][kBlkPartial]: m and l [8] each, o [8][128]
    float c;                                           // sm_scale * log2(e)
    int R, Hq, Hkv, rep, n_blocks, width;
};

__device__ inline uint64_t ld8(const float *p)         // device scope: other dies wrote it in this launch
{
    return __hip_atomic_load((const uint64_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline void st8(float *p, float a, float b)
{
    const uint64_t v = (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a);
    __hip_atomic_store((uint64_t *)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline float lo8(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ inline float hi8(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }

template <bool BF16> struct Frag;
template <> struct Frag<false> {
    typedef half8v type;
    static __device__ type codes(uint32_t w0, uint32_t w1)
    {
        const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.0f, true);
        const half2v c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.0f, true);
        return type{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ f4v mul(type a, type b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Frag<true> {
    typedef bf8v type;
    static __device__ type codes(uint32_t w0, uint32_t w1)
    {
        const bf2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, true);
        const bf2v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, true);
        return type{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ f4v mul(type a, type b, f4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// maximum / sum over the four lanes n, n + 16, n + 32, n + 48
__device__ inline float max_over_g(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ inline float sum_over_g(float v)
{
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Work: the tiles of 64 tokens of all (request, KV head) units laid end to end and cut into equal ranges, one per
// workgroup, so that lengths of any kind fill the card; every workgroup reads all lengths and finds its range by
// itself.  Its four waves take quarters of a unit's part and meet in local memory; a unit that lies in several workgroups
// is merged by the one that finishes last (a ticket per unit, counted at the unit's first workgroup).
template <int BS, bool BF16>
__global__ __launch_bounds__(kBkThreads, 2) void decode_blk_kernel(BlkArgs a)
{
    constexpr int kIds = BS < kBlkTile ? kBlkTile / BS : 1;             // blocks of a tile
    extern __shared__ float lds[];
    float *parts = lds;                                // [4 waves][2 halves][8 heads][kBkRow]
    int *before = (int *)(lds + 64 * kBkRow);          // [R+1] tiles of the requests before r (of one KV head)
    __shared__ int wave_sum[4], ticket;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int n = lane & 15, g = lane >> 4, half = n >> 3, head = n & 7;
    const int wg = blockIdx.x;
    const int64_t most = (int64_t)a.width * BS;

    {                                                  // prefix sums of the requests' tiles
        auto tiles = [&](int r) { return (int)((min((int64_t)max(a.q_len[r], 0), most) + kBlkTile - 1) / kBlkTile); };
        const int per = (a.R + kBkThreads - 1) / kBkThreads, r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
        int sum = 0;
        for (int r = r0; r < r1; ++r) sum += tiles(r);
        int in = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(in, d, 64);
            if (lane >= d) in += o;
        }
        if (lane == 63) wave_sum[wave] = in;
        __syncthreads();
        int at = in - sum;
        for (int w = 0; w < wave; ++w) at += wave_sum[w];
        for (int r = r0; r < r1; ++r) before[r] = at, at += tiles(r);
        if (tid == kBkThreads - 1) before[a.R] = at;
        __syncthreads();
    }
    const int all = uniform(before[a.R] * a.Hkv);
    const int span = max((all + (int)gridDim.x - 1) / (int)gridDim.x, 4);
    int x = (int)min((int64_t)wg * span, (int64_t)all);
    const int end = (int)min((int64_t)x + span, (int64_t)all);

    for (int r = wg; r < a.R; r += gridDim.x)          // requests without tokens
        if (before[r + 1] == before[r])
            for (int i = tid; i < a.Hq * kD / 8; i += kBkThreads)
                ((uint4 *)(a.out + (int64_t)r * a.Hq * kD))[i] = uint4{0, 0, 0, 0};

    while (x < end) {
        // the unit that tile x belongs to, and the part [t0, t1) of its tiles that lies in this workgroup
        int r = 0;
        {
            const int y = x / a.Hkv;
            for (int step = a.R > 1 ? 1 << (31 - __builtin_clz(a.R - 1)) : 0; step; step >>= 1)
                if (r + step < a.R && before[r + step] <= y) r += step;
            r = uniform(r);
        }
        const int line = uniform(before[r] * a.Hkv), nt = uniform(before[r + 1] - before[r]);
        const int h = (x - line) / nt, t0 = x - line - h * nt, t1 = min(nt, t0 + (end - x));
        const int len = uniform((int)min((int64_t)max(a.q_len[r], 0), most));
        const int32_t *row = a.table + (int64_t)r * a.width;
        const int used = (len + BS - 1) / BS;          // table entries of the request

        typename Frag<BF16>::type qf[4];
        {
            const uint16_t *q = a.q + (int64_t)r * a.q_stride + (h * a.rep + min(head, a.rep - 1)) * kD + g * 16;
#pragma unroll
            for (int k = 0; k < 4; ++k) qf[k] = *(const typename Frag<BF16>::type *)(q + (k >> 1) * 64 + (k & 1) * 8);
        }
        f4v o[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) o[j] = f4v{0.0f, 0.0f, 0.0f, 0.0f};
        float m = kBkNone, l = 0.0f, vref = 0.0f, ivref = 0.0f;

        const int begin = t0 + (int)((int64_t)(t1 - t0) * wave / 4), stop = t0 + (int)((int64_t)(t1 - t0) * (wave + 1) / 4);
        int batch = 0, id = -1;                        // table entries batch + lane: block, K factor, V scale
        float kf = 0.0f, vs = 0.0f;
        auto fetch = [&](int entry) {
            batch = entry;
            id = batch + lane < used ? row[batch + lane] : -1;
            if ((uint32_t)id >= (uint32_t)a.n_blocks) id = -1;
            const int64_t at = (int64_t)max(id, 0) * a.Hkv + h;
            kf = a.Ks[at] * a.c, vs = id < 0 ? 0.0f : a.Vs[at];
        };
        auto entry_of = [&](int t) { return BS < kBlkTile ? t * kIds : t / (BS / kBlkTile); };
        auto lane_value = [&](int v, int i) { return __builtin_amdgcn_readlane(v, i); };
        auto lane_float = [&](float v, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), i)); };
        uint4 kx[4][2], vx[8];
        auto block_base = [&](const uint8_t *p, int t, int i) {         // block i of tile t, its first row of the tile
            const int64_t b = max(lane_value(id, entry_of(t) - batch + i), 0);
            return p + ((b * a.Hkv + h) * BS + (BS > kBlkTile ? (t % (BS / kBlkTile)) * kBlkTile : 0)) * kD;
        };
        auto load_k = [&](int t) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint8_t *p = block_base(a.K, t, j * kIds / 4) + (j * 16) % (BS < kBlkTile ? BS : kBlkTile) * kD;
#pragma unroll
                for (int k = 0; k < 2; ++k) kx[j][k] = *(const uint4 *)(p + n * kD + g * 16 + k * 64);
            }
        };
        auto load_v = [&](int t) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {              // token quad 4g of the 16 tokens 2 half + k
                int b = lane_value(id, entry_of(t) - batch + k * kIds / 4);
                if (kIds > 1) b = half ? lane_value(id, entry_of(t) - batch + (2 + k) * kIds / 4) : b;
                const int first = (BS > kBlkTile ? (t % (BS / kBlkTile)) * kBlkTile : 0) + ((2 * half + k) * 16) % (BS < kBlkTile ? BS : kBlkTile);
                const uint8_t *p = a.V + (((int64_t)max(b, 0) * a.Hkv + h) * BS + first + g * 4) * kD + head * 16;
#pragma unroll
                for (int i = 0; i < 4; ++i) vx[4 * k + i] = *(const uint4 *)(p + i * kD);
            }
        };
        if (begin < stop) {
            fetch(entry_of(begin));
            load_k(begin), load_v(begin);
        }
        for (int t = begin; t < stop; ++t) {
            const int e0 = entry_of(t) - batch;
            bool whole = (t + 1) * kBlkTile <= len;
            float vmax = 0.0f, f[2], vf[2];            // largest V scale; this lane's K factors and V scales (of 16 tokens each)
#pragma unroll
            for (int i = 0; i < kIds; ++i) whole &= lane_value(id, e0 + i) >= 0, vmax = fmaxf(vmax, lane_float(vs, e0 + i));
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int lo = e0 + k * kIds / 4, hi = e0 + (2 + k) * kIds / 4;
                const float k0 = lane_float(kf, lo), k1 = lane_float(kf, hi), v0 = lane_float(vs, lo), v1 = lane_float(vs, hi);
                f[k] = half ? k1 : k0, vf[k] = half ? v1 : v0;
            }
            bool absent[2] = {false, false};           // (as the tile's last block may be fetched over before they are used)
            if (!whole) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int lo = lane_value(id, e0 + k * kIds / 4), hi = lane_value(id, e0 + (2 + k) * kIds / 4);
                    absent[k] = (half ? hi : lo) < 0;
                }
            }
            const bool more = t + 1 < stop;
            f4v s[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[j] = f4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint4 w = kx[j][k >> 1];
                    s[j] = Frag<BF16>::mul(k & 1 ? Frag<BF16>::codes(w.z, w.w) : Frag<BF16>::codes(w.x, w.y), qf[k], s[j]);
                }
            }
            if (more) {
                if (entry_of(t + 1) + kIds > batch + 64) fetch(entry_of(t + 1));
                load_k(t + 1);
            }
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = (half ? s[2 + (i >> 2)][i & 3] : s[i >> 2][i & 3]) * f[i >> 2];
            if (!whole) {                              // the last tile of a request, or a block that is not there
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int token = t * kBlkTile + 16 * (2 * half + (i >> 2)) + 4 * g + (i & 3);
                    if (token >= len || absent[i >> 2]) {              // (the codes may be NaN: the weight 0 alone would not do)
                        w[i] = -INFINITY;
                        vx[i] = uint4{0, 0, 0, 0};
                    }
                }
            }
            float mx = w[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) mx = fmaxf(mx, w[i]);
            mx = max_over_g(mx);
            if (__any(mx > m) || vmax > vref) {
                const float top = fmaxf(mx, m), alpha = __builtin_amdgcn_exp2f(m - top);
                m = top, l *= alpha;
                float both = alpha;
                if (vmax > vref) both *= vref / vmax, vref = vmax, ivref = 1.0f / vmax;
#pragma unroll
                for (int j = 0; j < 16; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[j][i] *= both;
            }
            half8v p;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e = __builtin_amdgcn_exp2f(w[i] - m);
                l += e;
                p[i] = (_Float16)(e * (vf[i >> 2] * ivref));
            }
#pragma unroll
            for (int d = 0; d < 4; ++d) {              // channels 16 head + 4 d .. + 3
                uint32_t col[2][4];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t r0 = (&vx[4 * k].x)[d], r1 = (&vx[4 * k + 1].x)[d], r2 = (&vx[4 * k + 2].x)[d], r3 = (&vx[4 * k + 3].x)[d];
                    const uint32_t a0 = __builtin_amdgcn_perm(r1, r0, 0x05010400), a1 = __builtin_amdgcn_perm(r1, r0, 0x07030602);
                    const uint32_t b0 = __builtin_amdgcn_perm(r3, r2, 0x05010400), b1 = __builtin_amdgcn_perm(r3, r2, 0x07030602);
                    col[k][0] = __builtin_amdgcn_perm(b0, a0, 0x05040100), col[k][1] = __builtin_amdgcn_perm(b0, a0, 0x07060302);
                    col[k][2] = __builtin_amdgcn_perm(b1, a1, 0x05040100), col[k][3] = __builtin_amdgcn_perm(b1, a1, 0x07060302);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    o[4 * d + i] = Frag<false>::mul(Frag<false>::codes(col[0][i], col[1][i]), p, o[4 * d + i]);
            }
            if (more) load_v(t + 1);
        }

        // the waves' states meet in local memory: 8 parts (wave, half), of each its quadrant
        {
            float *part = parts + (wave * 2 + half) * 8 * kBkRow + head * kBkRow;
            l = sum_over_g(l);
            if (g == 0) part[0] = m, part[1] = l;
            if ((g >> 1) == half) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 16; j += 4)
                        *(float4 *)(part + 4 + (4 * (g & 1) + i) * 16 + j) =
                            float4{o[j][i] * vref, o[j + 1][i] * vref, o[j + 2][i] * vref, o[j + 3][i] * vref};
            }
        }
        __syncthreads();
        const int hh = tid >> 5, ch = (tid & 31) * 4;  // this thread's head and channels
        float M = kBkNone, L = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < 8; ++k) M = fmaxf(M, parts[(k * 8 + hh) * kBkRow]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float *part = parts + (k * 8 + hh) * kBkRow;
            const float f = __builtin_amdgcn_exp2f(part[0] - M);
            const float4 v = *(const float4 *)(part + 4 + ch);
            L += part[1] * f;
            acc[0] += v.x * f, acc[1] += v.y * f, acc[2] += v.z * f, acc[3] += v.w * f;
        }
        auto write_out = [&]() {
            const float inv = L > 0.0f ? 1.0f / L : 0.0f;
            uint16_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = BF16 ? __builtin_bit_cast(uint16_t, (__bf16)(acc[i] * inv)) : __builtin_bit_cast(uint16_t, (_Float16)(acc[i] * inv));
            *(uint2 *)(a.out + ((int64_t)r * a.Hq + h * a.rep + hh) * kD + ch) =
                uint2{(uint32_t)v[1] << 16 | v[0], (uint32_t)v[3] << 16 | v[2]};
        };
        if (t0 == 0 && t1 == nt) {
            if (hh < a.rep) write_out();
        } else {
            // (device scope throughout: the unit's workgroups run on different dies)
            const int ustart = line + h * nt, first = ustart / span, count = (ustart + nt - 1) / span - first + 1;
            float *slot = a.partials + (int64_t)(2 * wg + (t0 == 0)) * kBlkPartial;
            if (hh < a.rep) {
                if (ch == 0) st8(slot + 2 * hh, M, L);
                st8(slot + 16 + hh * kD + ch, acc[0], acc[1]);
                st8(slot + 16 + hh * kD + ch + 2, acc[2], acc[3]);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // this wave's stores are acknowledged ...
            __syncthreads();                                           // ... and every wave's
            if (tid == 0) ticket = __hip_atomic_fetch_add(a.tickets + first, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            if (ticket == count - 1) {
                if (tid == 0) __hip_atomic_store(a.tickets + first, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                M = kBkNone, L = 0.0f, acc[0] = acc[1] = acc[2] = acc[3] = 0.0f;
                if (hh < a.rep) {
                    constexpr int kAtOnce = 8;
                    for (int k0 = 0; k0 < count; k0 += kAtOnce) {
                        uint64_t ml[kAtOnce], v0[kAtOnce], v1[kAtOnce];
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k) {
                            const int kk = min(k0 + k, count - 1);
                            const float *src = a.partials + (int64_t)(kk == 0 ? 2 * first + 1 : 2 * (first + kk)) * kBlkPartial;
                            ml[k] = ld8(src + 2 * hh), v0[k] = ld8(src + 16 + hh * kD + ch), v1[k] = ld8(src + 16 + hh * kD + ch + 2);
                        }
                        float top = M;
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, lo8(ml[k]));
                        float f = __builtin_amdgcn_exp2f(M - top);
                        M = top, L *= f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[i] *= f;
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k) {
                            f = k0 + k < count ? __builtin_amdgcn_exp2f(lo8(ml[k]) - top) : 0.0f;
                            L += hi8(ml[k]) * f;
                            acc[0] += lo8(v0[k]) * f, acc[1] += hi8(v0[k]) * f, acc[2] += lo8(v1[k]) * f, acc[3] += hi8(v1[k]) * f;
                        }
                    }
                    write_out();
                }
            }
        }
        __syncthreads();                               // the parts are read: the next unit's may come
        x += t1 - t0;
    }
}

int launch_decode_blk(const minikv_blk_shape &s, const void *q, int64_t q_stride, const minikv_blk_cache &c, const int32_t *table,
                      const int32_t *q_len, float sm_scale, void *out, void *workspace, hipStream_t st)
{
    BlkArgs a;
    a.q = (const uint16_t *)q, a.q_stride = q_stride, a.K = c.K, a.V = c.V, a.Ks = c.Ks, a.Vs = c.Vs;
    a.table = table, a.q_len = q_len, a.out = (uint16_t *)out;
    a.tickets = (int *)workspace, a.partials = (float *)((char *)workspace + kBlkGroups * sizeof(int));
    a.c = sm_scale * 1.4426950408889634f;
    a.R = s.R, a.Hq = s.Hq, a.Hkv = s.Hkv, a.rep = s.Hq / s.Hkv, a.n_blocks = s.n_blocks, a.width = s.max_blocks;
    const int64_t tiles = ((int64_t)s.max_blocks * s.block + kBlkTile - 1) / kBlkTile * s.R * s.Hkv;
    const dim3 grid((unsigned)(tiles < kBlkGroups ? tiles : kBlkGroups));
    const size_t lds = (64 * kBkRow + s.R + 1) * sizeof(float);
    auto launch = [&](auto bs) {
        constexpr int BS = decltype(bs)::value;
        if (s.dtype == MINIKV_BF16) hipLaunchKernelGGL((decode_blk_kernel<BS, true>), grid, dim3(kBkThreads), lds, st, a);
        else hipLaunchKernelGGL((decode_blk_kernel<BS, false>), grid, dim3(kBkThreads), lds, st, a);
    };
    if (s.block == 16) launch(std::integral_constant<int, 16>{});
    else if (s.block == 32) launch(std::integral_constant<int, 32>{});
    else if (s.block == 64) launch(std::integral_constant<int, 64>{});
    else launch(std::integral_constant<int, 128>{});
    return hipGetLastError() == hipSuccess ? MINIKV_OK : MINIKV_ELAUNCH;
}

}  // namespace minikv
