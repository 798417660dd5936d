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
// Weights are rounded to fp16 for the second product (relative 2^-11, to nearest; the sum of weights is kept in fp32 from
// the unrounded ones), each with its block's V scale, over a reference that no such product so far exceeds, times 2^15: at most 2^15, and with
// all 11 bits down to 2^-29 of the reference.  The reference is the largest V scale that the wave has seen of the unit while its scales lie
// within 2^12 of each other (some token of weight 1 then has a product of 2^-12 or more of it), which costs nothing per tile.
// From the first tile where they do not on, it is per column the largest product itself, so that neither a large scale without weight nor a large
// weight without a scale takes the bits of the others: what is lost of a product is at most 2^-28 of the largest one either way.
#include "decode_common.h"

#include <type_traits>

namespace minikv {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float f4v __attribute__((ext_vector_type(4)));

constexpr int kBkWaves = 8;                            // of a workgroup: two per SIMD, the registers of a compute unit
constexpr int kBkThreads = 64 * kBkWaves;
constexpr int kBkRow = kD + 4;                         // floats of a head's state in local memory: m, l, 2 pad, o
constexpr int kBkEntry = kMaxRep * kBkRow;             // of a part of a unit
constexpr float kBkNone = -3.0e38f;                    // running maximum before the first token: finite, so that no difference is NaN
constexpr float kBkHeadroom = 32768.0f;                // fp16 weights run to 65504
constexpr int kBkFar = 12 << 23;                       // V scales whose bits (of positive floats) differ by more lie more than 2^12 apart
constexpr float kBkLeast = 0x1p-110f, kBkRange = 0x1p-100f;            // the reference: at least this, and this times the largest V scale (no quotient overflows)
// What a unit costs a wave besides its tiles (table, scales, queries, output), in tiles on the line of work.  Us with 0 / 1 / 2, 8 KV heads: 1000
// requests of 1 to 300 tokens 53.0 / 52.0 / 56.1, 48 of 1 to 16000 57.4 / 48.7 / 48.4, 200 of 120 16.6 each, 100 of 1 to 2000 25.7 / 27.2 / 26.7;
// 400 of 700, one KV head, 32.1 / 24.3 / 28.4.
constexpr int kBkUnitCost = 1;
// Workgroups of their own for every unit beat the line of work (where there are enough of them) while their waves have at most so
// many tiles more than the line's.  Us with 1 / 3 / 6 / 12, 8 KV heads: 32 requests of 1 to 2000 tokens 22.8 / 14.3 / 14.3 / 14.3, of 1 to 4000 23.1 /
// 23.1 / 22.2 / 22.2, of 1 to 8000 23.5 / 23.5 / 23.5 / 36.0; 16 of 1 to 5000 21.6 / 21.6 / 25.6 / 25.5; 24 of 1 to 8000 23.8 / 23.8 / 23.8 / 41.0.
constexpr int kBkUnitTiles = 3;

struct BlkArgs {
    const uint16_t *q;
    int64_t q_stride;
    const uint8_t *K, *V;
    const float *Ks, *Vs;
    const int32_t *table, *q_len;
    uint16_t *out;
    int *tickets;                                      // [kBlkGroups] of the line's units, then [kBlkGroups / 2][kMaxRep] of shared units
    float *partials;                                   // [2 * kBlkGroups][kBlkPartial]: (m, l) of 8 heads, o [8][128]
    float c;                                           // sm_scale * log2(e)
    int R, Hq, Hkv, rep, n_blocks, width;
    uint32_t hkv_magic, hkv_shift, units_magic, units_shift;            // division by Hkv and by R Hkv
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

// Codes are read once a call, and a program's other layers have caches of their own before this one's turn comes again: loaded
// with the streaming hint (without -> with: 16 requests of 32768 tokens 185 -> 166 us, one of 131072 56.0 -> 50.9, 48 of 1 to 16000 51.2 -> 48.7, 1000
// of 1 to 300 50.6 -> 51.8).  Where requests share their blocks, which a call cannot tell, it costs: 64 requests of 100 tokens behind one
// prefix of 8192 104 -> 151, behind one of 2048 40 -> 55, 32 of 4096 behind one of 4096 59 -> 67.
__device__ inline uint4 load_codes(const uint8_t *p)
{
    typedef uint32_t u4v __attribute__((ext_vector_type(4)));
    const u4v v = __builtin_nontemporal_load((const u4v *)p);
    return uint4{v[0], v[1], v[2], v[3]};
}

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
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_over_g(float v)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline float other_half(float v)            // of lane n ^ 8
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x128, 0xf, 0xf, false));
}

__device__ inline int wave_max(int v)                  // of values >= 0, the same in every lane
{
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));       // row_shr 1, 2, 4, 8
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));       // row_bcast 15, 31
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ inline int wave_sum_of(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
    return __builtin_amdgcn_readlane(v, 63);
}
// local memory that one wave writes and reads: its operations are done in order, the compiler is told to keep them so
__device__ inline void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <bool BF16> __device__ inline uint32_t pack2(float a, float b)
{
    if constexpr (BF16) return __builtin_bit_cast(uint32_t, bf2v{(__bf16)a, (__bf16)b});
    else return __builtin_bit_cast(uint32_t, half2v{(_Float16)a, (_Float16)b});
}

// Work.  A unit is a (request, KV head), its tiles are 64 tokens.  Every workgroup reads all lengths and finds what it does.
//   The line: tiles of all units laid end to end, each unit behind kBkUnitCost empty ones, cut into equal ranges, one per WAVE, so that
//   lengths of any kind fill the card.  A unit inside a wave's range is that wave's alone, from queries to output.  Of the
//   units that its ends cut, a wave leaves its part in local memory (two at most, "A" of a unit that began before, "B" of one that goes
//   on); behind one barrier the wave with the unit's first part in the workgroup merges the parts, and writes the output or, where
//   other workgroups have parts too, publishes the result and takes a ticket; the last one's workgroup merges them.
//   A workgroup per unit, or several, if there are enough of them and no wave gets many more tiles than on the line: one up to eight tiles, else a
//   power of two of them with about four tiles each, so that every SIMD has one.  (A wave's tile is 2800 cycles of one SIMD, most of them
//   conversions, and merging between workgroups 4000.)
// What bounds it: memory, where there is much to read (16 requests of 32768 tokens, 8 KV heads, 1.07 GB: 166 us, 6.5 TB/s, a plain
// streaming read reaches 6.0; one of 131072 tokens 50.3 us, 5.3 TB/s; 48 of 1 to 16000 tokens 48.6 us, 4.2 TB/s); round trips and the
// first pass through the code where there is little (8 heads of 1024 tokens 7.6 us); the conversions and what a unit costs besides
// its tiles where there are many short ones (1000 requests of 1 to 300 tokens 52 us).  Earlier forms: a workgroup of four waves on one
// unit at a time, with a barrier for each, 130 us for the 48 and 9.1 for the 1024 tokens; the line alone 178 for the 16, 11.4 for the 1024 tokens.
template <int BS, bool BF16>
__global__ __launch_bounds__(kBkThreads, 2) void decode_blk_kernel(BlkArgs a)
{
    constexpr int kIds = BS < kBlkTile ? kBlkTile / BS : 1, kTiles = BS > kBlkTile ? BS / kBlkTile : 1;     // blocks of a tile, tiles of a block
    constexpr int kRun = BS < kBlkTile ? BS : kBlkTile;                 // tokens of a tile that lie together
    extern __shared__ float lds[];
    float *parts = lds;                                // [2 * kBkWaves][8 heads][kBkRow]
    int *before = (int *)(lds + 2 * kBkWaves * kBkEntry);              // [R+1] line of the requests before r (of one KV head)
    int *lens = before + a.R + 1;                      // [R]
    __shared__ int wave_sum[kBkWaves], last[2][4]; // units whose last part came from here: r, h, first workgroup, count
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int n = lane & 15, g = lane >> 4, half = n >> 3, head = n & 7;
    const int wg = blockIdx.x;

    f4v o[16];                                         // this lane's sums, see the top of the file
    float m, l, ref;                                   // maximum and sum of weights, reference of the products: o is in units of ref / kBkHeadroom
    auto entry_of = [&](int t) { return t * kIds / kTiles; };
    // What is loaded for: the unit, its table entries batch + lane (block, K factor, V scale), its queries, one tile of codes.
    int ld_h = 0, ld_len = 0, batch = 0, id = -1;
    const int32_t *ld_row = nullptr;
    float kf = 0.0f, vs = 0.0f;
    typename Frag<BF16>::type qf[4];
    uint4 kx[4][2], vx[8];
    // found: in lane i, table entry `entry` + i (anything where the request has none)
    auto take = [&](int entry, int found) {
        batch = entry;
        id = (batch + lane) * BS < ld_len && (uint32_t)found < (uint32_t)a.n_blocks ? found : -1;
        const int64_t at = (int64_t)max(id, 0) * a.Hkv + ld_h;
        kf = a.Ks[at] * a.c, vs = id < 0 ? 0.0f : a.Vs[at];
    };
    auto turn_to = [&](int r, int h, int len, int t, int found) {      // tiles from t on of unit (r, h) are loaded next
        ld_h = h, ld_len = len, ld_row = a.table + (int64_t)r * a.width;
        const uint16_t *q = a.q + (int64_t)r * a.q_stride + (h * a.rep + min(head, a.rep - 1)) * kD + g * 16;
#pragma unroll
        for (int k = 0; k < 4; ++k) qf[k] = *(const typename Frag<BF16>::type *)(q + (k >> 1) * 64 + (k & 1) * 8);
        take(entry_of(t), found);
    };
    auto lane_value = [&](int v, int i) { return __builtin_amdgcn_readlane(v, i); };
    auto lane_float = [&](float v, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), i)); };
    // Rows behind the request's last token are not loaded: their lanes repeat a row that is (for V, four rows that begin before it).
    auto load_k = [&](int t) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {                  // tokens 16 j .. of the tile
            const int64_t b = max(lane_value(id, entry_of(t) - batch + j * kIds / 4), 0);
            const int first = t % kTiles * kBlkTile + j * 16 % kRun, there = min(max(ld_len - t * kBlkTile - j * 16, 1), 16);
            const uint8_t *p = a.K + ((b * a.Hkv + ld_h) * BS + first) * kD;
            const int at = min(n, there - 1) * kD + g * 16;
#pragma unroll
            for (int k = 0; k < 2; ++k) kx[j][k] = load_codes(p + at + k * 64);
        }
    };
    auto load_v = [&](int t) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {                  // token quad 4g of the 16 tokens 2 half + k
            int b = lane_value(id, entry_of(t) - batch + k * kIds / 4);
            if (kIds > 1) b = half ? lane_value(id, entry_of(t) - batch + (2 + k) * kIds / 4) : b;
            const int left = ld_len - t * kBlkTile - (2 * half + k) * 16, quad = min(g, max(left - 1, 0) >> 2);
            const int first = t % kTiles * kBlkTile + (2 * half + k) * 16 % kRun;
            const uint8_t *p = a.V + (((int64_t)max(b, 0) * a.Hkv + ld_h) * BS + first + quad * 4) * kD + head * 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) vx[4 * k + i] = load_codes(p + i * kD);
        }
    };
    // Tiles [t0, t1) of the unit of `len` tokens that is being loaded, its first tile already.  more: another unit's first tile is to be loaded
    // behind the last one, next() turns to it.
    auto attend = [&](int len, int t0, int t1, bool more, auto next) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 16; ++j) o[j] = f4v{0.0f, 0.0f, 0.0f, 0.0f};
        m = kBkNone, l = 0.0f, ref = kBkLeast;
        float iref = kBkHeadroom / kBkLeast;
        int vmin = 0x7f800000, vmax = 0;               // bits of the V scales seen, smallest and largest
        for (int t = t0; t < t1; ++t) {
            const int e0 = entry_of(t) - batch;
            bool whole = (t + 1) * kBlkTile <= len;
            float f[2], vf[2];                         // this lane's K factors and V scales (of 16 tokens each)
#pragma unroll
            for (int i = 0; i < kIds; ++i) {
                const int bits = lane_value(__float_as_int(vs), e0 + i);
                const bool there = lane_value(id, e0 + i) >= 0;
                whole &= there, vmax = max(vmax, bits), vmin = there ? min(vmin, bits) : vmin;
            }
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
            int ahead = t + 1;                         // the tile loaded next: of this unit, or the next unit's first
            if (ahead < t1) {
                const int entry = entry_of(ahead);
                if (entry + kIds > batch + 64) take(entry, ld_row[min(entry + lane, a.width - 1)]);
            } else if (more) {
                ahead = 0, next();
            }
            if (ahead < t1 || more) load_k(ahead);
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
            const float mx0 = fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3])), mx1 = fmaxf(fmaxf(w[4], w[5]), fmaxf(w[6], w[7]));
            const float mx = max_over_g(fmaxf(mx0, mx1)), largest = __int_as_float(vmax);
            const bool far = vmax - vmin > kBkFar;
            if (__any(mx > m || largest > ref) || far) {
                const float top = fmaxf(mx, m), alpha = __builtin_amdgcn_exp2f(m - top);
                m = top, l *= alpha;
                float both = alpha;
                if (far) {                             // (o stands for sums relative to the maximum: where that grows, the reference shrinks instead)
                    const float here = fmaxf(__builtin_amdgcn_exp2f(mx0 - m) * vf[0], __builtin_amdgcn_exp2f(mx1 - m) * vf[1]);
                    const float old = ref * alpha;
                    ref = fmaxf(fmaxf(old, max_over_g(here)), fmaxf(largest * kBkRange, kBkLeast)), iref = kBkHeadroom / ref;
                    both = old / ref;
                } else if (largest > ref) {
                    both *= ref / largest, ref = largest, iref = kBkHeadroom / ref;
                }
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
                p[i] = (_Float16)(e * (vf[i >> 2] * iref));
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
            if (ahead < t1 || more) load_v(ahead);
        }
    };
    // The wave's sums of a unit to local memory.  o[j][i] belongs to channel 16 (4 (g & 1) + i) + j, in the lanes whose row and
    // column belong to one half of the tokens.
    auto leave_halves = [&](int slot) __attribute__((always_inline)) {      // each half to a slot of its own
        l = sum_over_g(l);
        const float f = ref / kBkHeadroom;
        float *p = parts + (slot + half) * kBkEntry + head * kBkRow;
        if (g == 0) p[0] = m, p[1] = l;
        p += 4 + (g & 1) * 64;
        if ((g >> 1) == half) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 16; j += 4)
                    *(float4 *)(p + i * 16 + j) = float4{o[j][i] * f, o[j + 1][i] * f, o[j + 2][i] * f, o[j + 3][i] * f};
        }
    };
    // both to one slot: the second half's lanes put theirs down, the first half's add theirs
    auto leave_part = [&](int slot) __attribute__((always_inline)) {
        const float both = fmaxf(m, other_half(m)), mine = __builtin_amdgcn_exp2f(m - both);
        l = sum_over_g(l) * mine;
        l += other_half(l);
        float *p = parts + slot * kBkEntry + head * kBkRow;
        if (lane < 8) p[0] = both, p[1] = l;
        const float f = mine * (ref / kBkHeadroom);
        p += 4 + (g & 1) * 64;
        if (half && g >= 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 16; j += 4)
                    *(float4 *)(p + i * 16 + j) = float4{o[j][i] * f, o[j + 1][i] * f, o[j + 2][i] * f, o[j + 3][i] * f};
        }
        wave_order();
        if (!half && g < 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    const float4 v = *(const float4 *)(p + i * 16 + j);
                    *(float4 *)(p + i * 16 + j) = float4{v.x + o[j][i] * f, v.y + o[j + 1][i] * f, v.z + o[j + 2][i] * f, v.w + o[j + 3][i] * f};
                }
        }
        wave_order();
    };

    // parts in slots 0, step, 2 step ... (below end), of head `wave`: a lane takes two channels
    float M, L, x0, x1;
    auto merge_slots = [&](int step, int end) __attribute__((always_inline)) {
        const float *p = parts + wave * kBkRow;
        M = kBkNone, L = x0 = x1 = 0.0f;
        for (int w = 0; w < end; w += step) M = fmaxf(M, p[w * kBkEntry]);
        for (int w = 0; w < end; w += step) {
            const float *q = p + w * kBkEntry;
            const float f = __builtin_amdgcn_exp2f(q[0] - M);
            const float2 v = *(const float2 *)(q + 4 + 2 * lane);
            L += q[1] * f, x0 += v.x * f, x1 += v.y * f;
        }
    };
    // partials of head hd of the workgroups place(k), k = from, from + step ... < count, sixteen at once
    auto merge_partials = [&](int hd, int from, int step, int count, auto place) __attribute__((always_inline)) {
        constexpr int kAtOnce = 16;
        M = kBkNone, L = x0 = x1 = 0.0f;
        for (int k0 = from; k0 < count; k0 += kAtOnce * step) {
            uint64_t ml[kAtOnce], v[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const float *src = a.partials + (int64_t)place(min(k0 + k * step, count - 1)) * kBlkPartial;
                ml[k] = ld8(src + 2 * hd), v[k] = ld8(src + 2 * kMaxRep + hd * kD + 2 * lane);
            }
            float top = M;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, lo8(ml[k]));
            float f = __builtin_amdgcn_exp2f(M - top);
            M = top, L *= f, x0 *= f, x1 *= f;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                f = k0 + k * step < count ? __builtin_amdgcn_exp2f(lo8(ml[k]) - top) : 0.0f;
                L += hi8(ml[k]) * f, x0 += lo8(v[k]) * f, x1 += hi8(v[k]) * f;
            }
        }
    };
    auto write_out = [&](int r, int h, int hd) __attribute__((always_inline)) {
        const float inv = L > 0.0f ? 1.0f / L : 0.0f;
        *(uint32_t *)(a.out + ((int64_t)r * a.Hq + h * a.rep + hd) * kD + 2 * lane) = pack2<BF16>(x0 * inv, x1 * inv);
    };

    const int units = a.R * a.Hkv;
    const int share = (int)fast_div((uint32_t)wg, a.units_magic, a.units_shift), unit = wg - share * units;      // a unit's workgroups are `units` apart
    int r = (int)fast_div((uint32_t)unit, a.hkv_magic, a.hkv_shift), h = unit - r * a.Hkv, log_shares = 0;
    bool by_unit = units <= (int)gridDim.x;
    int unit_len = 0, unit_t0 = 0, unit_t1 = 0, unit_first = 0;
    if (by_unit) {                                     // (lengths and the table are requested together, as few units wait for)
        const int64_t most = (int64_t)a.width * BS;
        auto len_of = [&](int i) { return (int)min((int64_t)max(a.q_len[i], 0), most); };
        const int32_t *row = a.table + (int64_t)r * a.width;
        unit_len = uniform(len_of(r));
        const int e0 = row[min(lane, a.width - 1)];
        int top = 0, sum = 0;                          // (as many requests as workgroups, at most)
        for (int i = lane; i < a.R; i += 64) {
            const int tiles = (len_of(i) + kBlkTile - 1) / kBlkTile;
            top = max(top, tiles), sum += tiles;
        }
        top = wave_max(top), sum = wave_sum_of(sum) * a.Hkv;
        if (top > kBkWaves)
            while ((4 << log_shares) < top && (2 * units << log_shares) <= (int)gridDim.x) ++log_shares;
        by_unit = (top + (kBkWaves << log_shares) - 1) / (kBkWaves << log_shares) <= sum / ((int)gridDim.x * kBkWaves) + kBkUnitTiles;
        if (by_unit) {
            if (share >= 1 << log_shares) return;      // (the whole workgroup)
            const int64_t nt = (unit_len + kBlkTile - 1) / kBlkTile;
            const int from = (int)(nt * share >> log_shares), n = (int)(nt * (share + 1) >> log_shares) - from;
            const int each = n / kBkWaves, more = n % kBkWaves;        // (waves 0 .. 3 are on SIMDs of their own)
            unit_t0 = from + wave * each + min(wave, more), unit_t1 = unit_t0 + each + (wave < more);
            const int entry = entry_of(unit_t0);
            unit_first = __shfl(e0, (entry + lane) & 63, 64);
            if (entry_of(unit_t1) + kIds > 64) unit_first = row[min(entry + lane, a.width - 1)];
        }
    }
    int total = 0;
    if (__builtin_expect(!by_unit, 0)) {
        {
            auto cost = [&](int len) { return len ? (len + kBlkTile - 1) / kBlkTile + kBkUnitCost : 0; };
            const int64_t most = (int64_t)a.width * BS;
            const int per = (a.R + kBkThreads - 1) / kBkThreads, r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
            int sum = 0;
            for (int r = r0; r < r1; ++r) {
                const int len = (int)min((int64_t)max(a.q_len[r], 0), most);
                lens[r] = len, sum += cost(len);
            }
            int in = sum;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(in, d, 64);
                if (lane >= d) in += o;
            }
            if (lane == 63) wave_sum[wave] = in;
            if (tid < 2) last[tid][3] = 0;
            __syncthreads();
            int at = in - sum;
#pragma unroll
            for (int w = 0; w < kBkWaves; ++w)
                if (w < wave) at += wave_sum[w];
            for (int r = r0; r < r1; ++r) before[r] = at, at += cost(lens[r]);
            if (tid == kBkThreads - 1) before[a.R] = at;
            __syncthreads();
        }
        for (int r = wg; r < a.R; r += gridDim.x)          // requests without tokens
            if (lens[r] == 0)
                for (int i = tid; i < a.Hq * kD / 8; i += kBkThreads)
                    ((uint4 *)(a.out + (int64_t)r * a.Hq * kD))[i] = uint4{0, 0, 0, 0};
        total = uniform(before[a.R] * a.Hkv);
        if (total == 0) return;
    }
    // The line: tile t of a unit that begins at `start` on it stands at start + kBkUnitCost + t.
    // (total is below 2^31, the sum below 2^32)
    const int span = by_unit ? 1 : max((int)(((uint32_t)total + gridDim.x * kBkWaves - 1) / (gridDim.x * kBkWaves)), kBkUnitCost + 1);
    const int64_t from = (int64_t)(wg * kBkWaves + wave) * span;
    int x = (int)min(from, (int64_t)total);
    const int end = (int)min(from + span, (int64_t)total);
    // the units of this wave's parts A and B: which, and their first and last wave with tiles
    int a_r = -1, a_h = 0, a_first = 0, a_stop = 0, b_r = -1, b_h = 0, b_first = 0, b_stop = 0;
    int len = unit_len, t0 = unit_t0, t1 = unit_t1, first = unit_first, start = 0, c = 0;
    // where unit (r, h) lies on the line and which of its tiles are this wave's
    auto locate = [&](int r, int h, int &len, int &t0, int &t1, int &start, int &c) {
        len = uniform(lens[r]), c = uniform(before[r + 1] - before[r]), start = uniform(before[r] * a.Hkv) + h * c;
        t0 = max(x - start - kBkUnitCost, 0), t1 = min(end - start, c) - kBkUnitCost;
    };
    auto request_at = [&](int x) {                     // the request that place x of the line belongs to (the last one that begins there)
        const int y = (int)fast_div((uint32_t)x, a.hkv_magic, a.hkv_shift);
        int r = 0;
        for (int step = a.R > 1 ? 1 << (31 - __builtin_clz(a.R - 1)) : 0; step; step >>= 1)
            if (r + step < a.R && before[r + step] <= y) r += step;
        return uniform(r);
    };
    if (!by_unit && x < end) {
        r = request_at(x);
        h = uniform((x - before[r] * a.Hkv) / (before[r + 1] - before[r]));
        locate(r, h, len, t0, t1, start, c);
        if (t0 < t1) first = a.table[(int64_t)r * a.width + min(entry_of(t0) + lane, a.width - 1)];
    }
    if (t0 < t1) {
        turn_to(r, h, len, t0, first);
        load_k(t0), load_v(t0);
    }
    while (by_unit || t0 < t1) {                       // (a range that has none of a unit's tiles ends before them)
        int r2 = r, h2 = h + 1, len2 = 0, from2 = 0, to2 = 0, start2 = 0, c2 = 0, first2 = 0;
        if (!by_unit) {                                // the next unit, and its table while this one's tiles are worked on
            x = start + c;
            if (x < end) {
                if (h2 == a.Hkv) {
                    h2 = 0, ++r2;
                    if (uniform(before[r2 + 1] - before[r2]) == 0) r2 = request_at(x);          // (requests without tokens between)
                }
                locate(r2, h2, len2, from2, to2, start2, c2);
                if (from2 < to2) first2 = a.table[(int64_t)r2 * a.width + min(lane, a.width - 1)];
            }
        }
        attend(len, t0, t1, from2 < to2, [&]() { turn_to(r2, h2, len2, 0, first2); });
        const bool goes_on = !by_unit && t0 == 0, alone = goes_on && t1 == c - kBkUnitCost;
        const int slot = 2 * wave + goes_on;           // (a part B is a wave's last: until then its slot is free)
        if (by_unit) {
            leave_halves(slot);
            break;
        }
        leave_part(slot);
        if (alone) {
            for (int hd = 0; hd < a.rep; ++hd) {
                const float *p = parts + slot * kBkEntry + hd * kBkRow;
                const float2 v = *(const float2 *)(p + 4 + 2 * lane);
                const float inv = p[1] > 0.0f ? 1.0f / p[1] : 0.0f;
                *(uint32_t *)(a.out + ((int64_t)r * a.Hq + h * a.rep + hd) * kD + 2 * lane) = pack2<BF16>(v.x * inv, v.y * inv);
            }
        } else {
            const int lead = (start + kBkUnitCost) / span, stop = (start + c - 1) / span;
            if (goes_on) b_r = r, b_h = h, b_first = lead, b_stop = stop;
            else a_r = r, a_h = h, a_first = lead, a_stop = stop;
        }
        r = r2, h = h2, len = len2, t0 = from2, t1 = to2, start = start2, c = c2;
    }
    __syncthreads();
    if (by_unit) {
        if (wave >= a.rep) return;                     // a wave per head from here on
        merge_slots(1, 2 * kBkWaves);
        if (log_shares) {
            float *out = a.partials + (int64_t)2 * wg * kBlkPartial;
            if (lane == 0) st8(out + 2 * wave, M, L);
            st8(out + 2 * kMaxRep + wave * kD + 2 * lane, x0, x1);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // the stores are acknowledged before the ticket is taken
            int *counter = a.tickets + kBlkGroups + unit * kMaxRep + wave, ticket = 0;
            if (lane == 0) ticket = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (uniform(ticket) != (1 << log_shares) - 1) return;
            if (lane == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            merge_partials(wave, 0, 1, 1 << log_shares, [&](int k) { return 2 * (unit + k * units); });
        }
        write_out(r, h, wave);
        return;
    }
    // the parts of a unit in this workgroup: slot `first`, then the A parts of the next waves; lanes take two channels each
    auto merge_parts = [&](int cut_r, int cut_h, int cut_first, int cut_stop, int b) __attribute__((always_inline)) {
        const int lead = b == 0 ? 0 : wave, stop = min(cut_stop - wg * kBkWaves, kBkWaves - 1);
        const int first_wg = cut_first / kBkWaves, count = cut_stop / kBkWaves - first_wg + 1;
        float *out = a.partials + (int64_t)(2 * wg + b) * kBlkPartial;
        for (int hd = 0; hd < a.rep; ++hd) {
            const float *p0 = parts + (2 * lead + b) * kBkEntry + hd * kBkRow;
            float M = p0[0];
            for (int w = lead + 1; w <= stop; ++w) M = fmaxf(M, parts[2 * w * kBkEntry + hd * kBkRow]);
            float f = __builtin_amdgcn_exp2f(p0[0] - M);
            float2 v = *(const float2 *)(p0 + 4 + 2 * lane);
            float L = p0[1] * f, x0 = v.x * f, x1 = v.y * f;
            for (int w = lead + 1; w <= stop; ++w) {
                const float *p = parts + 2 * w * kBkEntry + hd * kBkRow;
                f = __builtin_amdgcn_exp2f(p[0] - M);
                v = *(const float2 *)(p + 4 + 2 * lane);
                L += p[1] * f, x0 += v.x * f, x1 += v.y * f;
            }
            if (count == 1) {
                const float inv = L > 0.0f ? 1.0f / L : 0.0f;
                *(uint32_t *)(a.out + ((int64_t)cut_r * a.Hq + cut_h * a.rep + hd) * kD + 2 * lane) = pack2<BF16>(x0 * inv, x1 * inv);
            } else {                                   // (device scope throughout: the unit's workgroups run on different dies)
                if (lane == 0) st8(out + 2 * hd, M, L);
                st8(out + 2 * kMaxRep + hd * kD + 2 * lane, x0, x1);
            }
        }
        if (count > 1) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // the stores are acknowledged before the ticket is taken
            if (lane == 0) {
                const int ticket = __hip_atomic_fetch_add(a.tickets + first_wg, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (ticket == count - 1) {
                    __hip_atomic_store(a.tickets + first_wg, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    last[b][0] = cut_r, last[b][1] = cut_h, last[b][2] = first_wg, last[b][3] = count;
                }
            }
        }
    };
    if (a_r >= 0 && wave == 0) merge_parts(a_r, a_h, a_first, a_stop, 0);               // (behind another wave's part, that one merges it)
    if (b_r >= 0) merge_parts(b_r, b_h, b_first, b_stop, 1);
    __syncthreads();
    for (int b = 0; b < 2; ++b) {
        r = uniform(last[b][0]), h = uniform(last[b][1]);
        const int first_wg = uniform(last[b][2]), count = uniform(last[b][3]);
        if (count == 0) continue;
        // the workgroups' partials of a head and of every sets-th workgroup to a wave, sixteen at once; then a wave per head
        const int sets = kBkWaves / a.rep, set = wave / a.rep, hd = wave - set * a.rep;
        if (set < sets) {
            merge_partials(hd, set, sets, count, [&](int k) { return k == 0 ? 2 * first_wg + 1 : 2 * (first_wg + k); });
            float *p = parts + 2 * set * kBkEntry + hd * kBkRow;
            if (lane == 0) p[0] = M, p[1] = L;
            *(float2 *)(p + 4 + 2 * lane) = float2{x0, x1};
        }
        __syncthreads();
        if (wave < a.rep) {
            merge_slots(2, 2 * sets);
            write_out(r, h, wave);
        }
        __syncthreads();
    }
}

int launch_decode_blk(const minikv_blk_shape &s, const void *q, int64_t q_stride, const minikv_blk_cache &c, const int32_t *table,
                      const int32_t *q_len, float sm_scale, void *out, void *workspace, hipStream_t st)
{
    BlkArgs a;
    a.q = (const uint16_t *)q, a.q_stride = q_stride, a.K = c.K, a.V = c.V, a.Ks = c.Ks, a.Vs = c.Vs;
    a.table = table, a.q_len = q_len, a.out = (uint16_t *)out;
    a.tickets = (int *)workspace, a.partials = (float *)((char *)workspace + kBlkTickets * sizeof(int));
    a.c = sm_scale * 1.4426950408889634f;
    a.R = s.R, a.Hq = s.Hq, a.Hkv = s.Hkv, a.rep = s.Hq / s.Hkv, a.n_blocks = s.n_blocks, a.width = s.max_blocks;
    fast_div_setup((uint32_t)s.Hkv, a.hkv_magic, a.hkv_shift);
    fast_div_setup((uint32_t)(s.R * s.Hkv), a.units_magic, a.units_shift);
    const int64_t tiles = ((int64_t)s.max_blocks * s.block + kBlkTile - 1) / kBlkTile * s.R * s.Hkv;
    // (a workgroup per unit where that is chosen, else eight waves of at least two places on the line each)
    const dim3 grid((unsigned)(tiles < kBlkGroups ? tiles : kBlkGroups));
    const size_t lds = (2 * kBkWaves * kBkEntry + 2 * s.R + 1) * sizeof(float);
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
