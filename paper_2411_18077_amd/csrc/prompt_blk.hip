// Attention of several new tokens of each request over its tokens in the paged 8-bit cache (minikv_prompt_attn_blk).
//
// The rows of one KV head of a request are its new tokens times the query heads of that head: row i * rep + h.  Scores are computed
// transposed, S^T = K Q^T on the 32x32x16 instruction, so that a lane holds one row: maximum and sum of the softmax are the lane's own, and its
// weights are the B operand of O^T = V^T P^T as they are.  A workgroup of four waves takes
//   wide    128 rows, 32 a wave, and walks the tokens in tiles of 64: a tile's codes go from memory through registers to local memory as 16-bit
//           operands, every code once per workgroup (keys in the queries' type, values in fp16: e4m3 is exact in both);
//   narrow  the last up to 64 rows of a request, 32 of them: all waves hold the same rows and take every fourth 32 tokens each, keys from memory to
//           registers, values through a wave's own local memory, and no barrier; their results meet at the end.
//
// The scales of a block are factors of whole keys and values: that of K is part of the factor that takes a score to a power of two, that
// of V becomes part of the weight, as its logarithm in the exponent: w = 2^(s c Ks + log2 Vs - m'), m' the largest such exponent of the row so far.  So
// the second product takes codes as they are, and no weight loses bits to a large scale without weight.  w, times 2^15, is rounded to fp16:
// 11 bits down to 2^-29 of the row's largest.  The sum of the weights without Vs is kept over a reference of its own, the largest score.
//
// Long walks are made in parts, by as many workgroups as the card holds (see find_item); the parts of a block's rows are joined by the last
// workgroup of each eight to arrive, the results of eight of those by the last of them, and so on, always summed in the parts' order.
#include "decode_common.h"
#include "attn_tile.h"

#include <type_traits>

namespace minikv {

constexpr int kPbNarrow = 32;                          // rows of a narrow block
constexpr int kPbRows = 128;                           // rows of a wide one
constexpr int kPbTail = 64;                            // most rows behind the last wide block that narrow ones take
constexpr int kPbThreads = 256;
constexpr float kPbNone = -3.0e38f;                    // references before the first token: finite, so that no difference is NaN
constexpr float kPbHead = 15.0f;                       // log2 of the largest weight
constexpr float kPbRange = 60.0f;                      // V scales, as powers of two, further below the largest one: weights with them do not give those without
constexpr float kPbNothing = -1024.0f;                 // log2 of a V scale of 0: its products are below all that binary32 holds
constexpr int kPbWideCost = 2;                         // of a tile of 64 tokens for a wide block, 1 for a narrow one
constexpr int kPbLeastWide = 6, kPbLeastNarrow = 2;    // least tiles of a part of a walk
constexpr int kPbWholeNarrow = 6;                      // narrow walks of fewer tiles are not made in parts
constexpr int kPbSlots = 2 * kComputeUnits;            // workgroups at once
constexpr int kPbFine = kPbSlots;                      // most narrow blocks that are taken instead of wide ones
constexpr int kPbStream = 16384;                       // cost of all blocks, in tiles of 16 KB, from which on caches do not hold them (256 MB beside the memory)
constexpr int kPbJoin = 8;                             // parts joined at once
constexpr int kPbMost = 512;                           // parts of a walk: three rounds of joins
constexpr int kPbGroups = 4;                           // of items, by the length of their walks
constexpr uint32_t kPbCut = 1 << 22;                   // most items of a thread in a group; 2^8 threads and four groups: sums below 2^32

struct PromptBlkArgs {
    const uint16_t *q;
    int64_t q_stride;
    const uint8_t *K, *V;
    const float *Ks, *Vs;
    const int32_t *table, *q_len, *cu;
    uint16_t *out;
    float *lse;
    int *tickets;                                      // [3][2 * kPbSlots], of the first part of each eight, 64, 512
    float *ml, *o;                                     // [part][row] (m, l) and [part][row][128]
    int part_rows;
    float c;                                           // sm_scale * log2(e)
    int R, T, Hq, Hkv, rep, n_blocks, width, shift;
    uint32_t hkv_magic, hkv_shift, rep_magic, rep_shift;
};

// What a workgroup works on.
struct PromptItem {
    int r, at, n, L;                                   // request, its first row of q, new tokens, tokens held
    int row0, narrow;                                  // first row of the block, and its kind
    int part, parts, slot;                             // which part of the walk, of how many; part 0's place in the workspace, for parts > 1
    int chunk;                                         // tiles of a part
    int stream;                                        // the call reads more than caches hold
};

__device__ inline uint64_t pb_load(const float *p)     // device scope: other dies wrote it in this launch
{
    return __hip_atomic_load((const uint64_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline void pb_store(float *p, float a, float b)
{
    __hip_atomic_store((uint64_t *)p, (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline float2 pb_pair(uint64_t v) { return float2{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))}; }

// The requests' rows in blocks, each block's walk in cost / share parts, share = ceil(all blocks' cost / slots) (of workgroups at once): rounded up
// if the items of more than half a share are then not more than slots, so that they run at once and the others fill what is left, else
// down.  (Always up, 16 x 8 tokens behind 16384 have 568 parts for 512 slots: 123 us instead of 100; always down, a step of 24 uneven
// requests 59 us instead of 49.)  Blocks in two or more parts, slots of these at most (rounded down, a part has at least a share; rounded up, more than half
// of one, and those were counted), come first, then those in one, long ones first;
// of a request the narrow blocks, then the wide ones from the last on, whose walks are the longest.  Every workgroup counts all that for itself.
template <int CTRL, int ROWS> __device__ inline uint64_t add_dpp64(uint64_t v)
{
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)v, CTRL, ROWS, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
    return v + ((uint64_t)hi << 32 | lo);
}
__device__ inline uint64_t wave_sum64(uint64_t v)
{
    v = add_dpp64<0x111, 0xf>(v), v = add_dpp64<0x112, 0xf>(v), v = add_dpp64<0x114, 0xf>(v), v = add_dpp64<0x118, 0xf>(v);       // row_shr 1, 2, 4, 8
    v = add_dpp64<0x142, 0xa>(v), v = add_dpp64<0x143, 0xc>(v);                       // row_bcast 15, 31
    return (uint64_t)__builtin_amdgcn_readlane((uint32_t)(v >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)v, 63);
}

template <int CTRL, int ROWS> __device__ inline uint32_t add_dpp(uint32_t v)
{
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
// Sum of the lanes up to this one.  (Not saturating, as that of scan.h: counts of a thread are cut to kPbCut, and the launch refuses calls that have more.)
__device__ inline uint32_t wave_prefix(uint32_t v)
{
    v = add_dpp<0x111, 0xf>(v), v = add_dpp<0x112, 0xf>(v), v = add_dpp<0x114, 0xf>(v), v = add_dpp<0x118, 0xf>(v);
    return add_dpp<0x143, 0xc>(add_dpp<0x142, 0xa>(v));
}

// WAVE: up to 64 requests, one a lane, and every wave finds for itself; else every thread has some in a row, and the workgroup meets between the steps.
template <bool WAVE>
__device__ inline bool find_item_in(const PromptBlkArgs &a, uint32_t idx, PromptItem &it)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = WAVE ? 1 : (a.R + kPbThreads - 1) / kPbThreads, r0 = min(WAVE ? lane : tid * per, a.R), r1 = min(r0 + per, a.R);
    struct Request {
        int at, n, L;
        uint32_t rows, wide, narrow, tiles;
    };
    bool fine = false;                                 // all blocks narrow
    auto cut = [&](Request &q) {
        const uint32_t rest = q.rows % kPbRows;
        q.wide = fine ? 0 : q.rows / kPbRows + (rest > kPbTail);
        q.narrow = fine ? (q.rows + kPbNarrow - 1) / kPbNarrow : rest > kPbTail ? 0 : (rest + kPbNarrow - 1) / kPbNarrow;
    };
    auto read = [&](int r) {
        Request q;
        q.at = a.cu[r];
        const int end = a.cu[r + 1];
        q.n = q.at >= 0 && end > q.at && end <= a.T ? end - q.at : 0;
        q.L = (int)min((int64_t)max(a.q_len[r], 0), (int64_t)a.width << a.shift);
        q.rows = (uint32_t)q.n * a.rep;
        q.tiles = (uint32_t)max((q.L + 63) >> 6, 1);
        cut(q);
        return q;
    };
    Request mine{0, 0, 0, 0, 0, 0, 1};
    if (r0 < r1) mine = read(r0);
    auto each = [&](auto take) {                       // until one takes the item
        if constexpr (WAVE)
            take(mine, r0);
        else
            for (int r = r0; r < r1; ++r)
                if (take(r == r0 ? mine : read(r), r)) break;
    };
    __shared__ uint64_t costs[2][kPbThreads / 64];     // of the waves
    __shared__ uint32_t counts[2 + kPbGroups][kPbThreads / 64];
    __shared__ PromptItem found;
    // the workgroup's sum of the counts whose prefix v is, behind a barrier
    auto total = [&](int k, uint32_t v) {
        return WAVE ? (uint32_t)__builtin_amdgcn_readlane(v, 63) : counts[k][0] + counts[k][1] + counts[k][2] + counts[k][3];
    };
    auto meet = [&](int k, uint32_t v) {
        if (!WAVE && lane == 63) counts[k][wave] = v;
    };

    uint64_t all = 0, all_fine = 0;                    // the blocks' cost, with wide ones and without
    uint32_t count = 0;                                // of the narrow ones without
    each([&](const Request &q, int) {
        const uint32_t n = (q.rows + kPbNarrow - 1) / kPbNarrow;
        all += (uint64_t)(q.wide * kPbWideCost + q.narrow) * q.tiles, all_fine += (uint64_t)n * q.tiles, count += n;
        return false;
    });
    all = wave_sum64(all), all_fine = wave_sum64(all_fine), count = wave_prefix(min(count, kPbCut));
    meet(0, count);
    if constexpr (!WAVE) {
        if (lane == 63) costs[0][wave] = all, costs[1][wave] = all_fine;
        if (tid == 0) found.r = -1;
        __syncthreads();
        all = costs[0][0] + costs[0][1] + costs[0][2] + costs[0][3], all_fine = costs[1][0] + costs[1][1] + costs[1][2] + costs[1][3];
    }
    fine = (uint64_t)total(0, count) * a.Hkv <= kPbFine;
    if (fine) cut(mine), all = all_fine;
    all *= a.Hkv;
    const uint32_t share = (uint32_t)min((all + kPbSlots - 1) / kPbSlots, (uint64_t)1 << 26);          // (at most above any cost)
    const uint32_t chunk[2] = {max(share, (uint32_t)kPbLeastNarrow), max(share, (uint32_t)kPbLeastWide * kPbWideCost)};
    const float by[2] = {__builtin_amdgcn_rcpf((float)chunk[0]), __builtin_amdgcn_rcpf((float)chunk[1])};
    // cost / chunk, rounded up or down, 1 to kPbMost.  (cost < 2^26; a quotient that is off by more than the one that is put right is beyond kPbMost)
    auto parts_for = [&](const Request &q, int wide, bool up) {
        const uint32_t cost = wide ? q.tiles * kPbWideCost : q.tiles, c = chunk[wide];
        uint32_t p = (uint32_t)fminf((float)cost * by[wide], (float)kPbMost);
        if (p * c > cost) --p;
        if ((p + 1) * c <= cost) ++p;
        if (up && p * c < cost) ++p;
        if (!wide && q.tiles < (uint32_t)kPbWholeNarrow) p = 1;
        return min(max(p, 1u), (uint32_t)kPbMost);
    };
    uint32_t large = 0;                                // items of more than half a share, rounded up
    each([&](const Request &q, int) {
        const uint32_t w = parts_for(q, 1, true), n = parts_for(q, 0, true);
        if (q.tiles * kPbWideCost * 2 > chunk[1] * w) large += q.wide * w;
        if (q.tiles * 2 > chunk[0] * n) large += q.narrow * n;
        return false;
    });
    large = wave_prefix(min(large, kPbCut));
    meet(1, large);
    if constexpr (!WAVE) __syncthreads();
    const bool up = (uint64_t)total(1, large) * a.Hkv <= kPbSlots;
    // Groups: of walks in two or more parts, and in one of more than half a share, a quarter, less.  (25 requests of 226 new tokens behind up to 482, 16
    // heads, two groups: 54 us instead of 44.)
    auto group_of = [&](uint32_t cost, uint32_t p) { return p > 1 ? 0 : cost * 2 > share ? 1 : cost * 4 > share ? 2 : 3; };
    uint32_t items[kPbGroups] = {}, v[kPbGroups];
    each([&](const Request &q, int) {
        const uint32_t w = parts_for(q, 1, up), n = parts_for(q, 0, up);
        const int gw = group_of(q.tiles * kPbWideCost, w), gn = group_of(q.tiles, n);
#pragma unroll
        for (int k = 0; k < kPbGroups; ++k) items[k] += (gw == k ? q.wide * w : 0) + (gn == k ? q.narrow * n : 0);
        return false;
    });
#pragma unroll
    for (int k = 0; k < kPbGroups; ++k) items[k] = min(items[k], kPbCut), v[k] = wave_prefix(items[k]), meet(2 + k, v[k]);
    if constexpr (!WAVE) __syncthreads();
    if ((uint64_t)total(2, v[0]) * a.Hkv > gridDim.x) return false;    // (cu that falls and rises: not all parts of a walk would come to their join)
    int group = 0;                                     // what is looked for, and where the thread's own begin
    uint32_t start = 0, own = items[0], before = v[0] - items[0];
#pragma unroll
    for (int k = 1; k < kPbGroups; ++k) {
        const uint32_t next = start + total(1 + k, v[k - 1]);
        if (group == k - 1 && idx >= next) start = next, group = k, own = items[k], before = v[k] - items[k];
    }
    uint32_t first = start + before;
    if (!WAVE)
        for (int w = 0; w < wave; ++w) first += counts[2 + group][w];
    PromptItem got;
    got.r = -1;
    if (idx >= first && idx - first < own)
        each([&](const Request &q, int r) {
            const uint32_t w = parts_for(q, 1, up), n = parts_for(q, 0, up), at = idx - first;
            const uint32_t narrow = group_of(q.tiles, n) == group ? q.narrow * n : 0, wide = group_of(q.tiles * kPbWideCost, w) == group ? q.wide * w : 0;
            first += narrow + wide;
            if (at >= narrow + wide) return false;
            const bool is_narrow = at < narrow;
            const uint32_t p = is_narrow ? n : w, i = is_narrow ? at : at - narrow, k = i / p;
            got.at = q.at, got.n = q.n, got.L = q.L, got.r = r;
            got.narrow = is_narrow;
            got.row0 = (int)(is_narrow ? q.wide * kPbRows + k * kPbNarrow : (q.wide - 1 - k) * kPbRows);
            got.part = (int)(i - k * p), got.parts = (int)p, got.chunk = (int)((q.tiles + p - 1) / p);
            got.slot = (int)(idx - got.part);
            got.stream = all >= (uint64_t)kPbStream;
            return true;
        });
    int src = 0;                                       // the lane that has it
    if constexpr (WAVE) {
        const uint64_t who = __ballot(got.r >= 0);
        if (!who) return false;
        it = got, src = __builtin_ctzll(who);
    } else {
        if (got.r >= 0) found = got;
        __syncthreads();
        it = found;
    }
    int *p = (int *)&it;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(it) / sizeof(int)); ++i) p[i] = __builtin_amdgcn_readlane(p[i], src);
    return it.r >= 0;
}
__device__ inline bool find_item(const PromptBlkArgs &a, uint32_t idx, PromptItem &it)
{
    return a.R <= 64 ? find_item_in<true>(a, idx, it) : find_item_in<false>(a, idx, it);
}

typedef _Float16 half2p __attribute__((ext_vector_type(2)));
typedef __bf16 bf2p __attribute__((ext_vector_type(2)));
typedef uint32_t u4b __attribute__((ext_vector_type(4)));

// 16 codes as 16-bit values
template <bool BF16>
__device__ __forceinline__ void widen(const u4b &codes, u4b (&out)[2])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (BF16) {
            out[j >> 1][(j & 1) * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[j], 1.0f, false));
            out[j >> 1][(j & 1) * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[j], 1.0f, true));
        } else {
            out[j >> 1][(j & 1) * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[j], 1.0f, false));
            out[j >> 1][(j & 1) * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[j], 1.0f, true));
        }
    }
}

// log2 of a positive scale, exact for a power of two
__device__ __forceinline__ float log2_scale(float s)
{
    const uint32_t b = __float_as_uint(s);
    return (float)((int)(b >> 23) - 127) + __builtin_amdgcn_logf(__uint_as_float((b & 0x7fffff) | 0x3f800000));
}

// Where a lane reads the transposed fragments of a tile of values: rows 4 g + 0..3 and 8 more, channels 32 db + r
__device__ __forceinline__ void value_places(int (&v_place)[4])
{
    const int lane = threadIdx.x & 63, i = lane & 15, row = 4 * (lane >> 5) + (i >> 2), c0 = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
#pragma unroll
    for (int db = 0; db < 4; ++db) v_place[db] = row * kPfD + (((4 * db + c0) ^ v_swizzle(row)) << 3) + (i & 1) * 4;
}

// Blocks' scales as the softmax takes them: ck takes a score to a power of two, lv = log2 Vs, add what is added (lv, or -inf where the block is
// absent), add_m = add - lv, sum what takes a sum of weights with Vs to one without (-inf for a block whose Vs is 0 or far below the largest, where
// a weight with it may be 0 and the one without all there is: there these are summed by themselves).
struct BlockScale {
    float ck, add, add_m, sum;
};
// Scales of NG blocks, block lane % NG in each lane (negative: absent).  none: a bit for each block that is absent; most: the largest lv so far.
// Returns whether a block's weights have to be summed by themselves.
template <int NG>
__device__ __forceinline__ bool block_scales(float ks, float vs, float c, float &most, BlockScale (&b)[NG], uint32_t &none)
{
    const float l = vs > 0.0f ? log2_scale(vs) : kPbNone;
    float top = l;
    if (NG >= 2) top = fmaxf(top, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(top), 0xb1, 0xf, 0xf, false)));        // quad_perm 1, 0, 3, 2
    if (NG == 4) top = fmaxf(top, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(top), 0x4e, 0xf, 0xf, false)));        // quad_perm 2, 3, 0, 1
    most = fmaxf(most, top);
    none = (uint32_t)__ballot(vs < 0.0f) & ((1u << NG) - 1);
    const bool apart = vs >= 0.0f && !(l >= most - kPbRange);
    const float lv = vs > 0.0f ? l : vs == 0.0f ? kPbNothing : most > -1.0e29f ? most : 0.0f, add = vs < 0.0f ? -INFINITY : lv;
    const float add_m = vs < 0.0f ? -INFINITY : 0.0f, sum = apart ? -INFINITY : -lv - kPbHead;
    const float ck = fmaxf(vs < 0.0f ? 0.0f : ks * c, 0x1p-149f);      // (not 0: a masked score is -inf; the least there is, as raw products may be large)
    auto of = [](float v, int k) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), k)); };
#pragma unroll
    for (int k = 0; k < NG; ++k) b[k].ck = of(ck, k), b[k].add = of(add, k), b[k].add_m = of(add_m, k), b[k].sum = of(sum, k);
    return __any(apart);
}

// Per lane: a row's references of the weights with and without Vs, the sum of those without (of this half's keys), and O^T:
// o[db][i] = out[row][32 db + acc_row(i, g)].
struct RowState {
    float mv, m, l;
    float16v o[4];
    __device__ void clear()
    {
        mv = m = kPbNone, l = 0.0f;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] = 0.0f;
    }
    // o * by().x * by().y is o to the weights over m: two factors, as one may be below the numbers that the instruction makes (mv - m is a scale's logarithm)
    __device__ float2 by() const
    {
        const float half = __builtin_amdgcn_exp2f(0.5f * (mv - m));
        return float2{half, half * 0x1p-15f};          // 2^-kPbHead
    }
};

// 32 TILES scores a row (16 TILES a lane) of NG blocks to weights
template <int TILES, int NG>
__device__ __forceinline__ void softmax_step(float16v (&s)[TILES], const BlockScale (&b)[NG], bool apart, RowState &st, half8 (&wb)[2 * TILES])
{
    constexpr int kOf = 16 * TILES / NG;               // scores of a block
    float top = -INFINITY, top_v = -INFINITY;
#pragma unroll
    for (int k = 0; k < NG; ++k) {
        float mx = -INFINITY;
#pragma unroll
        for (int e = k * kOf; e < (k + 1) * kOf; ++e) mx = fmaxf(mx, s[e >> 4][e & 15]);
        top_v = fmaxf(top_v, __builtin_fmaf(mx, b[k].ck, b[k].add));
        top = fmaxf(top, __builtin_fmaf(mx, b[k].ck, b[k].add_m));
    }
    auto both = [&](float v) {                         // (the other half-wave holds the row's other keys)
        const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
    };
    top = both(top), top_v = both(top_v);
    if (__any(top > st.m)) {
        const float to = fmaxf(top, st.m);
        st.l *= __builtin_amdgcn_exp2f(st.m - to), st.m = to;
    }
    if (apart || __any(top_v > st.mv)) {
        const float to = fmaxf(top_v, st.mv), alpha = __builtin_amdgcn_exp2f(st.mv - to);
        st.mv = to;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) st.o[db][i] *= alpha;
        if (apart)                                     // (in here, as a branch of its own costs 3 %)
#pragma unroll
            for (int k = 0; k < NG; ++k)
                if (b[k].sum == -INFINITY)
#pragma unroll
                    for (int e = k * kOf; e < (k + 1) * kOf; ++e) st.l += __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 4][e & 15], b[k].ck, b[k].add_m - st.m));
    }
#pragma unroll
    for (int k = 0; k < NG; ++k) {
        const float off = b[k].add - st.mv + kPbHead;
        float sum = 0.0f;
#pragma unroll
        for (int e = k * kOf; e < (k + 1) * kOf; ++e) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 4][e & 15], b[k].ck, off));
            sum += w, wb[e >> 3][e & 7] = (_Float16)w;
        }
        st.l = __builtin_fmaf(sum, __builtin_amdgcn_exp2f(st.mv - st.m + b[k].sum), st.l);
    }
}

// 16 KEYS tokens' weights times their values, in a tile of local memory
template <int KEYS>
__device__ __forceinline__ void add_values(const _Float16 *Vt, const int (&v_place)[4], const half8 (&wb)[KEYS], RowState &st)
{
#pragma unroll
    for (int k = 0; k < KEYS; ++k)
#pragma unroll
        for (int db = 0; db < 4; ++db) {
            const _Float16 *p = Vt + k * 16 * kPfD + v_place[db];
            const half4 lo = read_transposed(p), hi = read_transposed(p + 8 * kPfD);
            st.o[db] = mfma32<false>(half8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}, wb[k], st.o[db]);
        }
}

// The requests' blocks as a walk sees them
struct Pages {
    const uint8_t *K, *V;
    const float *Ks, *Vs;
    const int32_t *table;                              // the request's row
    int entries, n_blocks, Hkv, kvh, shift, L;
    __device__ __forceinline__ int id(int token) const { return table[min(token >> shift, entries - 1)]; }
    __device__ __forceinline__ bool there(int id) const { return (uint32_t)id < (uint32_t)n_blocks; }
    __device__ __forceinline__ int64_t head(int id) const { return (int64_t)(there(id) ? id : 0) * Hkv + kvh; }
};

// A tile of 64 tokens on its way: a thread has 16 channels of tokens tid / 8 and tid / 8 + 32.  NG: blocks that a tile may hold (4, 2, 1 of 16, 32,
// 64 and 128 tokens).
template <int NG> struct Tile {
    u4b k[2], v[2];
    float ks, vs;                                      // of block lane % NG
    int id;                                            // the same; of the tile two further on, once this one's codes have been requested
};

// Tiles are requested two steps before they are in local memory: a step is about as long as a round trip to memory
template <bool BF16, int NG>
__device__ __forceinline__ void walk_wide(const PromptBlkArgs &a, const Pages &pg, _Float16 *tiles, int t0, int t1, int wt1, int full, int last, const half8 (&qf)[8],
                                          RowState &st)
{
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int key0 = tid >> 3, chunk = tid & 7, in_block = (1 << pg.shift) - 1, mine = lane % NG * (64 / NG);
    auto granule = [&](int j) { return NG == 4 ? 2 * j + (wave >> 1) : NG == 2 ? j : 0; };       // of the thread's token j, the same for the whole wave
    // (a token's place in its block, in a part of the tile's that is the same for all and one that does not change: addresses are a scalar and a register)
    const unsigned lane_off = (unsigned)((NG == 4 ? key0 & 15 : key0) * kD + chunk * 16);
    auto load = [&](Tile<NG> &x, int n) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int id = __builtin_amdgcn_readlane(x.id, granule(j)), first = NG == 1 ? ((n * 64) & in_block) + 32 * j : 0;
            const int64_t off = ((pg.head(id) << pg.shift) + first) * kD;
            x.k[j] = *(const u4b *)(pg.K + off + lane_off), x.v[j] = *(const u4b *)(pg.V + off + lane_off);
        }
        const int64_t at = pg.head(x.id);
        const float ks = pg.Ks[at], vs = pg.Vs[at];
        x.ks = ks, x.vs = pg.there(x.id) ? vs : -1.0f;
        if (n + 2 < t1) x.id = pg.id((n + 2) * 64 + mine);
    };
    int put_key[2], put_value[2];                      // where the thread's 16 bytes go in a tile (32 rows on: the same swizzle)
#pragma unroll
    for (int e = 0; e < 2; ++e) put_key[e] = tile_place(key0, 2 * chunk + e), put_value[e] = key0 * kPfD + (((2 * chunk + e) ^ v_swizzle(key0)) << 3);
    BlockScale scale[NG];                              // of the tile in local memory
    bool apart;
    float most = -1.0e30f;
    auto store = [&](const Tile<NG> &x, int n, auto odd) {             // (odd: which of the two buffers, known when compiling)
        uint32_t none;
        apart = block_scales<NG>(x.ks, x.vs, a.c, most, scale, none);
        const bool plain = !none && n * 64 + 64 <= pg.L;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = key0 + 32 * j;
            u4b k = x.k[j], v = x.v[j], w[2];
            if (!plain) {
                const bool in = n * 64 + key < pg.L && !(none >> granule(j) & 1);
#pragma unroll
                for (int e = 0; e < 4; ++e) k[e] = in ? k[e] : 0, v[e] = in ? v[e] : 0;
            }
            _Float16 *Kt = tiles + (decltype(odd)::value * 2 * kPfTile + 32 * j * kPfD), *Vt = Kt + kPfTile;
            widen<BF16>(k, w);
#pragma unroll
            for (int e = 0; e < 2; ++e) *(u4b *)(Kt + put_key[e]) = w[e];
            widen<false>(v, w);
#pragma unroll
            for (int e = 0; e < 2; ++e) *(u4b *)(Vt + put_value[e]) = w[e];
        }
    };
    int k_place[8], v_place[4];
#pragma unroll
    for (int s = 0; s < 8; ++s) k_place[s] = tile_place(r, 2 * s + g);
    value_places(v_place);

    auto step = [&](Tile<NG> &x, const Tile<NG> &y, int n, auto odd, auto even) {         // tile n; n + 2 into x, n + 1 from y
        if (n + 2 < t1) load(x, n + 2);
        if (n < wt1) {
            const _Float16 *Kt = tiles + decltype(odd)::value * 2 * kPfTile, *Vt = Kt + kPfTile;
            float16v s[2];
            half8 wb[4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) s[t] = mfma32<BF16>(*(const half8 *)(Kt + t * 32 * kPfD + k_place[k]), qf[k], s[t]);
            }
            if (n >= full) {
                const int rel = last - n * 64 - 4 * g;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (t * 32 + acc_row(i, 0) > rel) s[t][i] = -INFINITY;
            }
            softmax_step<2, NG>(s, scale, apart, st, wb);
            add_values<4>(Vt, v_place, wb, st);
        }
        if (n + 1 < t1) store(y, n + 1, even);
        __syncthreads();
    };
    const std::integral_constant<int, 0> first;
    const std::integral_constant<int, 1> second;
    Tile<NG> x, y;
    x.id = pg.id(t0 * 64 + mine), y.id = pg.id(min(t0 + 1, t1 - 1) * 64 + mine);
    load(x, t0);
    load(y, min(t0 + 1, t1 - 1));
    store(x, t0, first);
    __syncthreads();
    for (int n = t0; n < t1; n += 2) {
        step(x, y, n, first, second);
        if (n + 1 < t1) step(y, x, n + 1, second, first);
    }
}

// A wave's 32 tokens on their way: a lane has channels 64 g .. 64 g + 63 of key r, and 16 channels of the values of tokens lane / 8 + 8 j
template <int NG> struct Unit {
    u4b k[4], v[4];
    float ks, vs;                                      // of block lane % NG
    int id;                                            // the same; of the unit eight further on, once this one's codes have been requested
};

// Units of 32 tokens u0, u0 + 4, ... below u1.  qf: Q[row][64 g + 8 s ..], the channels in the order in which a lane has the keys'.  NG: 2 blocks of 16
// tokens, or 1.  ALONE: no other block of the request reads the tokens, and the call reads more than caches hold: values are loaded with the streaming hint
// (16 x 8 tokens behind 16384 98.4 -> 91.8 us, 64 x 4 behind one shared prefix of 8192 103 each; for 44 requests of up to 1841 tokens, which stay in
// caches between calls, it would cost 17.7 -> 19.8, with six blocks a request 33.0 -> 34.3).  A row of keys takes four loads, which the hint would make
// as many trips to memory (119 us).
template <bool BF16, int NG, bool ALONE>
__device__ __forceinline__ void walk_narrow(const PromptBlkArgs &a, const Pages &pg, _Float16 *Vt, int u0, int u1, int full, int last, const half8 (&qf)[8],
                                            RowState &st)
{
    const int lane = threadIdx.x & 63, r = lane & 31, g = lane >> 5, key0 = lane >> 3, chunk = lane & 7, in_block = (1 << pg.shift) - 1;
    const int mine = lane % NG * 16;
    const unsigned k_off = (NG == 1 ? r : r & 15) * kD + 64 * g, v_off = key0 * kD + chunk * 16;
    int v_place[4];
    value_places(v_place);
    float most = -1.0e30f;
    auto load = [&](Unit<NG> &x, int u) {
        int ids[NG];
#pragma unroll
        for (int b = 0; b < NG; ++b) ids[b] = __builtin_amdgcn_readlane(x.id, b);
        int64_t base[NG];                              // of the blocks' rows, or of the 32 in a larger one
#pragma unroll
        for (int b = 0; b < NG; ++b) base[b] = ((pg.head(ids[b]) << pg.shift) + (NG == 1 ? (u * 32) & in_block : 0)) * kD;
        const uint8_t *K = pg.K + (NG == 1 ? base[0] : r & 16 ? base[NG - 1] : base[0]) + k_off;
#pragma unroll
        for (int j = 0; j < 4; ++j) x.k[j] = *(const u4b *)(K + 16 * j);
        auto values = [&](int j) { return (const u4b *)(pg.V + base[j * NG / 4] + (NG == 1 ? 8 * j : 8 * (j & 1)) * kD + v_off); };
#pragma unroll
        for (int j = 0; j < 4; ++j) x.v[j] = ALONE ? __builtin_nontemporal_load(values(j)) : *values(j);
        const int64_t at = pg.head(x.id);
        const float ks = pg.Ks[at], vs = pg.Vs[at];
        x.ks = ks, x.vs = pg.there(x.id) ? vs : -1.0f;
        if (u + 8 < u1) x.id = pg.id((u + 8) * 32 + mine);
    };
    auto step = [&](Unit<NG> &x, int u) {
        BlockScale scale[NG];
        uint32_t none;
        const bool apart = block_scales<NG>(x.ks, x.vs, a.c, most, scale, none);
        const bool plain = !none && u * 32 + 32 <= pg.L;
        float16v s[1];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[0][i] = 0.0f;
        if (!plain) {
            const bool no_key = u * 32 + r >= pg.L || (none >> (NG == 1 ? 0 : r >> 4) & 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool no_value = u * 32 + key0 + 8 * j >= pg.L || (none >> (j * NG / 4) & 1);
#pragma unroll
                for (int e = 0; e < 4; ++e) x.k[j][e] = no_key ? 0 : x.k[j][e], x.v[j][e] = no_value ? 0 : x.v[j][e];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u4b w[2];
            widen<BF16>(x.k[j], w);
            s[0] = mfma32<BF16>(__builtin_bit_cast(half8, w[0]), qf[2 * j], s[0]);
            s[0] = mfma32<BF16>(__builtin_bit_cast(half8, w[1]), qf[2 * j + 1], s[0]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int key = key0 + 8 * j;
            u4b w[2];
            widen<false>(x.v[j], w);
#pragma unroll
            for (int e = 0; e < 2; ++e) *(u4b *)(Vt + key * kPfD + (((2 * chunk + e) ^ v_swizzle(key)) << 3)) = w[e];
        }
        if (u + 8 < u1) load(x, u + 8);                // (what was in the registers has been taken)
        if (u >= full) {
            const int rel = last - u * 32 - 4 * g;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (acc_row(i, 0) > rel) s[0][i] = -INFINITY;
        }
        half8 wb[2];
        softmax_step<1, NG>(s, scale, apart, st, wb);
        wave_order();                                  // (other lanes' values, and their places for the next ones)
        add_values<2>(Vt, v_place, wb, st);
        wave_order();
    };
    Unit<NG> x, y;
    if (u0 < u1) x.id = pg.id(u0 * 32 + mine);
    if (u0 + 4 < u1) y.id = pg.id((u0 + 4) * 32 + mine);
    if (u0 < u1) load(x, u0);
    if (u0 + 4 < u1) load(y, u0 + 4);
    for (int u = u0; u < u1; u += 8) {
        step(x, u);
        if (u + 4 < u1) step(y, u + 4);
    }
}

template <bool BF16, int NG>
__global__ __launch_bounds__(kPbThreads, 2) void prompt_blk_kernel(PromptBlkArgs a)
{
    // tiles [buffer][K, V] of a wide block, or each wave's values of a narrow one; at the end the waves' rows
    __shared__ __align__(16) _Float16 tiles[4 * kPfTile];
    __shared__ float2 wave_ml[4][32];
    __shared__ int ticket;
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t idx = fast_div(blockIdx.x, a.hkv_magic, a.hkv_shift);
    const int kvh = (int)(blockIdx.x - idx * a.Hkv);                   // (neighbours on a die walk through the same head)
    PromptItem it;
    if (!find_item(a, idx, it)) return;

    const int M = it.n * a.rep, rows = min(M - it.row0, it.narrow ? kPbNarrow : kPbRows), base = it.L - it.n;        // rows of the block; token of the first new one
    auto query_of = [&](int row) { return (int)fast_div(row, a.rep_magic, a.rep_shift); };
    const int seen = (base + query_of(it.row0 + rows - 1) + 64) >> 6;  // tiles that the block's last row sees (0 or less where it has no token)
    const int parts = it.parts > 1 ? min(max((seen + it.chunk - 1) / it.chunk, 1), it.parts) : 1;
    if (it.part >= parts) return;
    const int share = (seen + parts - 1) / parts, t0 = it.part * share, t1 = min(t0 + share, seen);

    const int w0 = it.row0 + (it.narrow ? 0 : 32 * wave);              // the wave's first row; a lane's own (behind the last one: that again, not stored)
    const int row = min(w0 + r, M - 1), query = query_of(row), last = base + query;              // the last token that the row sees
    const int low = base + query_of(min(w0, M - 1)), high = base + query_of(min(w0 + 31, M - 1));       // of the wave's first and last row
    half8 qf[8];
    {
        const uint16_t *qp = a.q + (int64_t)(it.at + query) * a.q_stride + (kvh * a.rep + row - query * a.rep) * kD;
#pragma unroll
        for (int s = 0; s < 8; ++s) qf[s] = *(const half8 *)(qp + (it.narrow ? 64 * g + 8 * s : 16 * s + 8 * g));
    }
    const Pages pg{a.K, a.V, a.Ks, a.Vs, a.table + (int64_t)it.r * a.width, (it.L + (1 << a.shift) - 1) >> a.shift, a.n_blocks, a.Hkv, kvh, a.shift, it.L};
    RowState st;
    st.clear();
    if (it.narrow && it.stream && M <= kPbNarrow)
        walk_narrow<BF16, NG == 4 ? 2 : 1, true>(a, pg, tiles + wave * kPfTile / 2, 2 * t0 + wave, 2 * t1, (low + 1) >> 5, last, qf, st);
    else if (it.narrow)
        walk_narrow<BF16, NG == 4 ? 2 : 1, false>(a, pg, tiles + wave * kPfTile / 2, 2 * t0 + wave, 2 * t1, (low + 1) >> 5, last, qf, st);
    else if (t0 < t1)
        walk_wide<BF16, NG>(a, pg, tiles, t0, t1, w0 < M ? min(t1, (high + 64) >> 6) : t0, (low + 1) >> 6, last, qf, st);

    // the waves' rows in local memory, 16 bytes of channels at place (channels / 4) ^ row, so that writes of 32 rows and reads of one use all banks
    float *rows_of = (float *)tiles;
    __syncthreads();
    {
        const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(st.l), __float_as_uint(st.l), false, false);
        if (g == 0) wave_ml[wave][r] = float2{st.m, __uint_as_float(h[0]) + __uint_as_float(h[1])};
        const float2 by = st.by();
        auto weighed = [&](float v) { return v * by.x * by.y; };
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *(float4 *)(rows_of + (wave * 32 + r) * kD + (((db * 8 + (i >> 1) + g) ^ r) << 2)) =
                    float4{weighed(st.o[db][i]), weighed(st.o[db][i + 1]), weighed(st.o[db][i + 2]), weighed(st.o[db][i + 3])};
    }
    __syncthreads();
    const int quad = tid & 31;                         // a thread's four channels, of rows tid / 32 + 8 k
    auto finish = [&](int i, float m, float l, float4 o) {
        const int row = it.row0 + i, query = query_of(row);
        const int64_t to = (int64_t)(it.at + query) * a.Hq + kvh * a.rep + row - query * a.rep;
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        *(half4 *)(a.out + to * kD + quad * 4) = half4{to16<BF16>(o.x * inv), to16<BF16>(o.y * inv), to16<BF16>(o.z * inv), to16<BF16>(o.w * inv)};
        if (a.lse && quad == 0) a.lse[to] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    };
    auto keep = [&](int slot, int i, float m, float l, float4 o) {
        const int64_t at = (int64_t)slot * a.part_rows + i;
        if (quad == 0) pb_store(a.ml + at * 2, m, l);
        pb_store(a.o + at * kD + quad * 4, o.x, o.y), pb_store(a.o + at * kD + quad * 4 + 2, o.z, o.w);
    };
    auto slot_of = [&](int part) { return (it.slot + part) * a.Hkv + kvh; };
    for (int i = tid >> 5; i < rows; i += 8) {
        float m, l;
        float4 o;
        if (it.narrow) {
            float2 ml[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) ml[w] = wave_ml[w][i];
            m = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)), l = 0.0f, o = float4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = __builtin_amdgcn_exp2f(ml[w].x - m);
                const float4 v = *(const float4 *)(rows_of + (w * 32 + i) * kD + ((quad ^ i) << 2));
                l = __builtin_fmaf(ml[w].y, f, l);
                o.x = __builtin_fmaf(v.x, f, o.x), o.y = __builtin_fmaf(v.y, f, o.y), o.z = __builtin_fmaf(v.z, f, o.z), o.w = __builtin_fmaf(v.w, f, o.w);
            }
        } else {
            const float2 ml = wave_ml[i >> 5][i & 31];
            m = ml.x, l = ml.y, o = *(const float4 *)(rows_of + i * kD + ((quad ^ (i & 31)) << 2));
        }
        if (parts == 1) finish(i, m, l, o);
        else keep(slot_of(it.part), i, m, l, o);
    }
    // joins: step is how many parts each of up to eight results stands for
    for (int step = 1, level = 0; step < parts; step *= kPbJoin, ++level) {
        const int first = it.part / (step * kPbJoin) * (step * kPbJoin), n = min((parts - first + step - 1) / step, kPbJoin);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");               // this wave's results are where every die sees them
        __syncthreads();
        if (n > 1) {
            if (tid == 0) {
                int *t = a.tickets + level * 2 * kPbSlots + slot_of(first);
                ticket = __hip_atomic_fetch_add(t, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (ticket == n - 1) __hip_atomic_store(t, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);     // ready for the next call
            }
            __syncthreads();
            if (ticket != n - 1) return;
            const bool done = step * kPbJoin >= parts;
            // each row's references and sums first, a factor for each of its results, then four rows a round trip
            float *factor = (float *)tiles;            // [row][kPbJoin], then m and l
            float2 *sums = (float2 *)(factor + kPbRows * kPbJoin);
            if (tid < rows) {
                float2 ml[kPbJoin];
#pragma unroll
                for (int j = 0; j < kPbJoin; ++j) ml[j] = pb_pair(pb_load(a.ml + ((int64_t)slot_of(first + min(j, n - 1) * step) * a.part_rows + tid) * 2));
                float m = kPbNone, l = 0.0f;
#pragma unroll
                for (int j = 0; j < kPbJoin; ++j) m = fmaxf(m, ml[j].x);
#pragma unroll
                for (int j = 0; j < kPbJoin; ++j) {
                    const float f = j < n ? __builtin_amdgcn_exp2f(ml[j].x - m) : 0.0f;
                    factor[tid * kPbJoin + j] = f, l = __builtin_fmaf(ml[j].y, f, l);
                }
                sums[tid] = float2{m, l};
            }
            __syncthreads();
            for (int i0 = tid >> 5; i0 < rows; i0 += 32) {
                float2 lo[4][kPbJoin], hi[4][kPbJoin];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i0 + 8 * e < rows)
#pragma unroll
                        for (int j = 0; j < kPbJoin; ++j)
                            if (j < n) {
                                const float *o = a.o + ((int64_t)slot_of(first + j * step) * a.part_rows + i0 + 8 * e) * kD + quad * 4;
                                lo[e][j] = pb_pair(pb_load(o)), hi[e][j] = pb_pair(pb_load(o + 2));
                            }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = i0 + 8 * e;
                    if (i >= rows) break;
                    float4 o = float4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < kPbJoin; ++j) {
                        if (j >= n) break;
                        const float f = factor[i * kPbJoin + j];
                        o.x = __builtin_fmaf(lo[e][j].x, f, o.x), o.y = __builtin_fmaf(lo[e][j].y, f, o.y);
                        o.z = __builtin_fmaf(hi[e][j].x, f, o.z), o.w = __builtin_fmaf(hi[e][j].y, f, o.w);
                    }
                    if (done) finish(i, sums[i].x, sums[i].y, o);
                    else keep(slot_of(first), i, sums[i].x, sums[i].y, o);
                }
            }
        }
    }
}

static int part_rows(const minikv_blk_shape &s, int32_t T)
{
    const int64_t rows = (int64_t)T * (s.Hq / s.Hkv);
    return (int)(rows < kPbRows ? rows : kPbRows);
}

// [tickets][(m, l) of the parts' rows][their outputs], for twice as many parts as there can be
size_t prompt_blk_workspace_bytes(const minikv_blk_shape &s, int32_t T)
{
    return (size_t)2 * kPbSlots * (3 * sizeof(int) + (size_t)part_rows(s, T) * (2 + kD) * sizeof(float));
}

int launch_prompt_blk(const minikv_blk_shape &s, int32_t T, const void *q, int64_t q_stride, const minikv_blk_cache &c, const int32_t *table,
                      const int32_t *q_len, const int32_t *cu, float sm_scale, void *out, float *lse, void *workspace, hipStream_t st)
{
    PromptBlkArgs a;
    a.q = (const uint16_t *)q, a.q_stride = q_stride, a.K = c.K, a.V = c.V, a.Ks = c.Ks, a.Vs = c.Vs;
    a.table = table, a.q_len = q_len, a.cu = cu, a.out = (uint16_t *)out, a.lse = lse;
    a.R = s.R, a.T = T, a.Hq = s.Hq, a.Hkv = s.Hkv, a.rep = s.Hq / s.Hkv, a.n_blocks = s.n_blocks, a.width = s.max_blocks;
    a.shift = __builtin_ctz(s.block), a.c = sm_scale * kLog2e, a.part_rows = part_rows(s, T);
    a.tickets = (int *)workspace, a.ml = (float *)(a.tickets + 3 * 2 * kPbSlots), a.o = a.ml + (size_t)2 * kPbSlots * a.part_rows * 2;
    fast_div_setup((uint32_t)s.Hkv, a.hkv_magic, a.hkv_shift);
    fast_div_setup((uint32_t)a.rep, a.rep_magic, a.rep_shift);
    // The grid: the most items that find_item can count.  Row blocks: 128 rows each and up to two for the rest of each request that has rows, and never
    // more than blocks of 32 rows would be; or those, kPbFine of them at most.  Parts: by the longest walk that the table has room for, and kPbSlots more
    // than there are blocks.  (Workgroups without an item cost: a step of 3 requests of 75 tokens 8.4 us with 528 of them, 11.5 with 2560.)
    const int64_t requests = s.R < T ? s.R : T, fine = (int64_t)T * a.rep / kPbNarrow + requests;
    const int64_t coarse = (int64_t)T * a.rep / kPbRows + 2 * requests;
    int64_t blocks = (coarse < fine ? coarse : fine) * s.Hkv;
    const int64_t small = fine * s.Hkv < kPbFine ? fine * s.Hkv : kPbFine;
    if (blocks < small) blocks = small;
    const int64_t tiles = ((int64_t)s.max_blocks * s.block + 63) / 64;
    const int64_t parts = tiles < kPbWholeNarrow ? 1 : (tiles + kPbLeastNarrow - 1) / kPbLeastNarrow;
    const int64_t items = blocks * parts < blocks + kPbSlots ? blocks * parts : blocks + kPbSlots;
    if (items > 0x7fffff || blocks / s.Hkv > (int64_t)kPbCut - kPbSlots) return MINIKV_EINVAL;
    const dim3 grid((unsigned)items), threads(kPbThreads);
    const bool bf16 = s.dtype == MINIKV_BF16;
#define LAUNCH(NG)                                                                                        \
    if (bf16) hipLaunchKernelGGL((prompt_blk_kernel<true, NG>), grid, threads, 0, st, a);                  \
    else hipLaunchKernelGGL((prompt_blk_kernel<false, NG>), grid, threads, 0, st, a)
    if (s.block == 16) {
        LAUNCH(4);
    } else if (s.block == 32) {
        LAUNCH(2);
    } else {
        LAUNCH(1);
    }
#undef LAUNCH
    return hipGetLastError() == hipSuccess ? MINIKV_OK : MINIKV_ELAUNCH;
}

}  // namespace minikv
