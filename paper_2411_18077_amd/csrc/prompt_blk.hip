// Attention of several new tokens of each request over its tokens in the paged 8-bit cache (minikv_prompt_attn_blk).
//
// The rows of one KV head of a request are its new tokens times the query heads of that head: row i * rep + h.  A workgroup of four waves
// takes 128 of them, 32 a wave, and walks the request's tokens in tiles of 64, all it sees or a part of them.  A tile's codes go from
// memory through registers to local memory as 16-bit operands, every code once per workgroup (keys in the queries' type, values in fp16: e4m3 is
// exact in both).  Scores are computed transposed, S^T = K Q^T on the 32x32x16 instruction, so that a lane holds one row: maximum and
// sum of the softmax are the lane's own, and its weights are the B operand of O^T = V^T P^T as they are.
//
// The scales of a block are factors of whole keys and values: that of K is part of the factor that takes a score to a power of two, that
// of V becomes part of the weight, as its logarithm in the exponent: w = 2^(s c Ks + log2 Vs - m'), m' the largest such exponent of the row so far.  So
// the second product takes codes as they are, and no weight loses bits to a large scale without weight.  w, times 2^15, is rounded to fp16:
// 11 bits down to 2^-29 of the row's largest.  The sum of the weights without Vs is kept over a reference of its own, the largest score.
#include "decode_common.h"
#include "attn_tile.h"

namespace minikv {

constexpr int kPbRows = 128;                           // rows of a workgroup
constexpr int kPbThreads = 256;
constexpr float kPbNone = -3.0e38f;                    // references before the first token: finite, so that no difference is NaN
constexpr float kPbHead = 15.0f;                       // log2 of the largest weight
constexpr float kPbRange = 60.0f;                      // V scales further below the largest one, as powers of two, count as 0
constexpr int kPbLeast = 2;                            // tiles that a part of a walk has at least

struct PromptBlkArgs {
    const uint16_t *q;
    int64_t q_stride;
    const uint8_t *K, *V;
    const float *Ks, *Vs;
    const int32_t *table, *q_len, *cu;
    uint16_t *out;
    float *lse;
    int *header;                                       // parts of walks in this call
    int4 *parts;                                       // of each: first row of q, rows of the request, first row | KV head, parts (0: not a first one)
    float *ml, *o;                                     // [part][row] (m, l) and [part][row][128]
    int part_rows;
    float c;                                           // sm_scale * log2(e)
    int R, T, Hq, Hkv, rep, n_blocks, width, shift, slots;
    uint32_t hkv_magic, hkv_shift, rep_magic, rep_shift;
};

// What a workgroup works on.
struct PromptItem {
    int r, at, n, L;                                   // request, its first row of q, new tokens, tokens held
    int block, part, parts, slot;                      // row block; which part of the walk, of how many; its place in the workspace (part 0's for parts > 1)
    int chunk;                                         // tiles of a part
};

// The requests' rows in blocks of 128, each block's walk in parts of about as many tiles as there are for a slot (of workgroups at
// once).  A block has ceil(tiles / chunk) parts, tiles the request's, chunk = ceil(all tiles of all blocks / slots): at most slots more
// than there are blocks, and at most twice slots where there are two or more.  Every workgroup counts all that for itself.
__device__ inline bool find_item(const PromptBlkArgs &a, uint32_t idx, uint64_t *lds, PromptItem &it)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (a.R + kPbThreads - 1) / kPbThreads, r0 = min(tid * per, a.R), r1 = min(r0 + per, a.R);
    auto request = [&](int r, int &at, int &n, int &L) {
        at = a.cu[r];
        const int end = a.cu[r + 1];
        n = at >= 0 && end > at && end <= a.T ? end - at : 0;
        L = (int)min((int64_t)max(a.q_len[r], 0), (int64_t)a.width << a.shift);
    };
    auto blocks = [&](int n) { return (uint32_t)((n * a.rep + kPbRows - 1) / kPbRows); };
    auto tiles = [&](int L) { return (uint32_t)max((L + 63) >> 6, 1); };
    uint32_t *sums = (uint32_t *)(lds + 1);            // [2][4] of the waves
    PromptItem *found = (PromptItem *)(lds + 8);
    if (tid == 0) lds[0] = 0, found->r = -1;
    __syncthreads();
    uint64_t all = 0;
    int at, n, L;
    for (int r = r0; r < r1; ++r) {
        request(r, at, n, L);
        all += (uint64_t)blocks(n) * tiles(L);
    }
    if (all) atomicAdd((unsigned long long *)lds, (unsigned long long)all);
    __syncthreads();
    all = lds[0] * a.Hkv;
    const uint32_t chunk = max((uint32_t)((all + a.slots - 1) / a.slots), (uint32_t)kPbLeast);
    uint32_t items = 0, split = 0;
    for (int r = r0; r < r1; ++r) {
        request(r, at, n, L);
        const uint32_t b = blocks(n), p = (tiles(L) + chunk - 1) / chunk;
        items += b * p, split += p > 1 ? b * p : 0;
    }
    uint32_t v[2] = {items, split};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t u = __shfl_up(v[k], d, 64);
            if (lane >= d) v[k] += u;
        }
        if (lane == 63) sums[k * 4 + wave] = v[k];
    }
    __syncthreads();
    uint32_t first = v[0] - items, slot = v[1] - split;
    for (int w = 0; w < wave; ++w) first += sums[w], slot += sums[4 + w];
    if (blockIdx.x == 0 && tid == 0) a.header[0] = (int)((sums[4] + sums[5] + sums[6] + sums[7]) * a.Hkv);
    if (idx >= first && idx - first < items)
        for (int r = r0; r < r1; ++r) {
            request(r, at, n, L);
            const uint32_t b = blocks(n), p = (tiles(L) + chunk - 1) / chunk;
            if (idx - first < b * p) {
                const uint32_t k = (idx - first) / p;
                found->at = at, found->n = n, found->L = L, found->r = r;
                found->block = (int)(b - 1 - k), found->part = (int)(idx - first - k * p), found->parts = (int)p;      // the longest walks first
                found->slot = (int)(slot + k * p), found->chunk = (int)chunk;
                break;
            }
            first += b * p, slot += p > 1 ? b * p : 0;
        }
    __syncthreads();
    it = *found;
    __syncthreads();
    it.r = __builtin_amdgcn_readfirstlane(it.r), it.at = __builtin_amdgcn_readfirstlane(it.at), it.n = __builtin_amdgcn_readfirstlane(it.n);
    it.L = __builtin_amdgcn_readfirstlane(it.L), it.block = __builtin_amdgcn_readfirstlane(it.block), it.part = __builtin_amdgcn_readfirstlane(it.part);
    it.parts = __builtin_amdgcn_readfirstlane(it.parts), it.slot = __builtin_amdgcn_readfirstlane(it.slot), it.chunk = __builtin_amdgcn_readfirstlane(it.chunk);
    return it.r >= 0;
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

// NG: blocks that a tile of 64 tokens may hold (4, 2, 1 of 16, 32, 64 and 128 tokens).
template <bool BF16, int NG>
__global__ __launch_bounds__(kPbThreads, 2) void prompt_blk_kernel(PromptBlkArgs a)
{
    __shared__ __align__(16) _Float16 tiles[2][2][kPfTile];            // [buffer][K, V]
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t idx = fast_div(blockIdx.x, a.hkv_magic, a.hkv_shift);
    const int kvh = (int)(blockIdx.x - idx * a.Hkv);                   // (neighbours on a die walk through the same head)
    PromptItem it;
    if (!find_item(a, idx, (uint64_t *)tiles, it)) return;

    const int M = it.n * a.rep, row0 = it.block * kPbRows, rows = min(M - row0, kPbRows), base = it.L - it.n;        // token of the first new one
    auto token_of = [&](int row) { return base + (int)fast_div(row, a.rep_magic, a.rep_shift); };
    const int seen = (token_of(row0 + rows - 1) + 64) >> 6;            // tiles that the block's last row sees (0 where it has no token)
    const int parts = it.parts > 1 ? min(max((seen + it.chunk - 1) / it.chunk, 1), it.parts) : 1;
    const int share = (seen + parts - 1) / parts, t0 = it.part * share, t1 = min(t0 + share, seen);
    const int slot = (it.slot + it.part) * a.Hkv + kvh;
    if (it.parts > 1 && tid == 0)
        a.parts[slot] = int4{it.at, M, row0, it.part == 0 && parts > 1 ? kvh | parts << 16 : 0};
    if (it.part >= parts) return;

    const int w0 = row0 + 32 * wave;                   // the wave's first row; a lane's own (behind the last one: that again, not stored)
    const bool works = w0 < M;
    const int row = min(w0 + r, M - 1), query = (int)fast_div(row, a.rep_magic, a.rep_shift), head = kvh * a.rep + row - query * a.rep;
    const int last = base + query;                     // the last token that the row sees
    const int wt1 = works ? min(t1, (token_of(min(w0 + 31, M - 1)) + 64) >> 6) : t0, full = (token_of(min(w0, M - 1)) + 1) >> 6;     // tiles the wave sees, and whole
    half8 qf[8];
    {
        const uint16_t *qp = a.q + (int64_t)(it.at + query) * a.q_stride + head * kD + g * 8;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qf[ks] = *(const half8 *)(qp + ks * 16);
    }

    // tile loads: thread tid has 16 channels of tokens tid / 8 and tid / 8 + 32
    const int32_t *table = a.table + (int64_t)it.r * a.width;
    const int entries = (it.L + (1 << a.shift) - 1) >> a.shift, key0 = tid >> 3, chunk = tid & 7, in_block = (1 << a.shift) - 1;
    int ids[NG];
    float ks[NG], vs[NG];                              // of the tile whose codes are on the way
    u4b kraw[2], vraw[2];
    auto load_ids = [&](int n) {
#pragma unroll
        for (int b = 0; b < NG; ++b) ids[b] = __builtin_amdgcn_readfirstlane(table[min((n * 64 + b * (64 / NG)) >> a.shift, entries - 1)]);
    };
    // what belongs to the block of the thread's token j (the same for the whole wave)
    auto of_token = [&](const auto &v, int j) { return NG == 4 ? (wave >> 1 ? v[(2 * j + 1) % NG] : v[2 * j % NG]) : v[j % NG]; };
    auto load = [&](int n) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int id = of_token(ids, j);
            const int64_t at = ((int64_t)((uint32_t)id < (uint32_t)a.n_blocks ? id : 0) * a.Hkv + kvh) << a.shift;
            const int64_t off = (at + ((n * 64 + key0 + 32 * j) & in_block)) * kD + chunk * 16;
            kraw[j] = *(const u4b *)(a.K + off), vraw[j] = *(const u4b *)(a.V + off);
        }
#pragma unroll
        for (int b = 0; b < NG; ++b) {
            const bool there = (uint32_t)ids[b] < (uint32_t)a.n_blocks;
            const int64_t at = (int64_t)(there ? ids[b] : 0) * a.Hkv + kvh;
            ks[b] = there ? a.Ks[at] : -1.0f, vs[b] = there ? a.Vs[at] : -1.0f;
        }
    };
    float ck[NG], lv[NG], add[NG];                     // of the tile in local memory: score to power of two, log2 Vs, and what is added (-inf: absent)
    float most = -1.0e30f;                             // the largest log2 Vs so far
    auto store = [&](int n) {
        bool zero[NG];
#pragma unroll
        for (int b = 0; b < NG; ++b)
            if (vs[b] > 0.0f) most = fmaxf(most, log2_scale(vs[b]));
#pragma unroll
        for (int b = 0; b < NG; ++b) {
            const float l = vs[b] > 0.0f ? log2_scale(vs[b]) : kPbNone;
            zero[b] = !(l >= most - kPbRange);
            lv[b] = !zero[b] ? l : most > -1.0e29f ? most : 0.0f;
            add[b] = vs[b] < 0.0f ? -INFINITY : lv[b];
            ck[b] = fmaxf(ks[b], 0x1p-126f) * a.c;     // (not 0: a masked score is -inf)
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = key0 + 32 * j;
            const bool in = n * 64 + key < it.L, none = of_token(vs, j) < 0.0f, nil = of_token(zero, j);
            u4b k = kraw[j], v = vraw[j], x[2];
#pragma unroll
            for (int e = 0; e < 4; ++e) k[e] = in && !none ? k[e] : 0, v[e] = in && !nil ? v[e] : 0;
            _Float16 *Kt = tiles[n & 1][0] + key * kPfD, *Vt = tiles[n & 1][1] + key * kPfD;
            widen<BF16>(k, x);
#pragma unroll
            for (int e = 0; e < 2; ++e) *(u4b *)(Kt + (((2 * chunk + e) ^ (key & 15)) << 3)) = x[e];
            widen<false>(v, x);
#pragma unroll
            for (int e = 0; e < 2; ++e) *(u4b *)(Vt + (((2 * chunk + e) ^ v_swizzle(key)) << 3)) = x[e];
        }
    };

    // fragment places
    int k_place[8], v_place[4];
#pragma unroll
    for (int s = 0; s < 8; ++s) k_place[s] = tile_place(r, 2 * s + g);
    {
        const int i = lane & 15, row = 4 * g + (i >> 2), c0 = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
#pragma unroll
        for (int db = 0; db < 4; ++db) v_place[db] = row * kPfD + (((4 * db + c0) ^ v_swizzle(row)) << 3) + (i & 1) * 4;
    }

    float16v o[4];                                     // O^T: o[db][i] = out[row][32 db + acc_row(i, g)]
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] = 0.0f;
    float mv = kPbNone, m = kPbNone, l = 0.0f;         // references of the weights with and without Vs; sum of the weights without, of this half's keys

    auto compute = [&](int n) {
        const _Float16 *Kt = tiles[n & 1][0], *Vt = tiles[n & 1][1];
        float16v s[2];
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
        constexpr int kOf = 32 / NG;                   // scores of a block
        float top = -INFINITY, top_v = -INFINITY;
#pragma unroll
        for (int b = 0; b < NG; ++b) {
            float mx = -INFINITY;
#pragma unroll
            for (int e = b * kOf; e < (b + 1) * kOf; ++e) mx = fmaxf(mx, s[e >> 4][e & 15]);
            top_v = fmaxf(top_v, __builtin_fmaf(mx, ck[b], add[b]));
            top = fmaxf(top, __builtin_fmaf(mx, ck[b], add[b] - lv[b]));
        }
        auto both = [&](float v) {                     // (the other half-wave holds the row's other keys)
            const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
        };
        top = both(top), top_v = both(top_v);
        if (__any(top > m)) {
            const float to = fmaxf(top, m);
            l *= __builtin_amdgcn_exp2f(m - to), m = to;
        }
        if (__any(top_v > mv)) {
            const float to = fmaxf(top_v, mv), alpha = __builtin_amdgcn_exp2f(mv - to);
            mv = to;
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
        }
        half8 wb[4];
#pragma unroll
        for (int b = 0; b < NG; ++b) {
            const float off = add[b] - mv + kPbHead;
            float sum = 0.0f;
#pragma unroll
            for (int e = b * kOf; e < (b + 1) * kOf; ++e) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 4][e & 15], ck[b], off));
                sum += w, wb[e >> 3][e & 7] = (_Float16)w;
            }
            l = __builtin_fmaf(sum, __builtin_amdgcn_exp2f(mv - m - lv[b] - kPbHead), l);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const _Float16 *p = Vt + k * 16 * kPfD + v_place[db];
                const half4 lo = read_transposed(p), hi = read_transposed(p + 8 * kPfD);
                o[db] = mfma32<false>(half8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}, wb[k], o[db]);
            }
    };

    if (t0 < t1) {
        load_ids(t0);
        load(t0);
        if (t0 + 1 < t1) load_ids(t0 + 1);
        store(t0);
        __syncthreads();
        for (int n = t0; n < t1; ++n) {
            if (n + 1 < t1) {
                load(n + 1);
                if (n + 2 < t1) load_ids(n + 2);
            }
            if (n < wt1) compute(n);
            if (n + 1 < t1) store(n + 1);
            __syncthreads();
        }
    }
    if (w0 + r >= M) return;

    {
        const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(h[0]) + __uint_as_float(h[1]);
    }
    const float by = __builtin_amdgcn_exp2f(mv - m - kPbHead);         // of o, to the weights over m
    if (parts > 1) {
        const int64_t at = (int64_t)slot * a.part_rows + (row - row0);
        if (g == 0) *(float2 *)(a.ml + at * 2) = float2{m, l};
        float *p = a.o + at * kD + g * 4;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *(float4 *)(p + db * 32 + (i >> 2) * 8) = float4{o[db][i] * by, o[db][i + 1] * by, o[db][i + 2] * by, o[db][i + 3] * by};
        return;
    }
    const float inv = l > 0.0f ? by / l : 0.0f;
    const int64_t to = (int64_t)(it.at + query) * a.Hq + head;
    if (a.lse && g == 0) a.lse[to] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    uint16_t *p = a.out + to * kD + g * 4;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            half4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = to16<BF16>(o[db][i + e] * inv);
            *(half4 *)(p + db * 32 + (i >> 2) * 8) = v;
        }
}

// The rows whose walk was made in parts: a wave a row, two channels a lane.
constexpr int kPbJoinRows = 16;                        // of a workgroup

template <bool BF16>
__global__ __launch_bounds__(kPbThreads) void prompt_join_kernel(PromptBlkArgs a, int groups)
{
    const int slot = (int)blockIdx.x / groups, group = (int)blockIdx.x % groups, lane = threadIdx.x & 63;
    if (slot >= a.header[0]) return;
    const int4 d = a.parts[slot];
    const int parts = d.w >> 16, kvh = d.w & 0xffff, M = d.y, row0 = d.z;
    // (a call whose cu is not what it has to be may leave parts without a description of their own)
    if (parts < 2 || kvh >= a.Hkv || (int64_t)slot + (int64_t)(parts - 1) * a.Hkv >= a.header[0] || d.x < 0 || row0 < 0) return;
    const int end = min(M - row0, min((group + 1) * kPbJoinRows, a.part_rows));
    for (int i = group * kPbJoinRows + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < end; i += 4) {
        auto at = [&](int j) { return ((int64_t)slot + (int64_t)j * a.Hkv) * a.part_rows + i; };
        float m = kPbNone, l = 0.0f, x = 0.0f, y = 0.0f;
        for (int j0 = 0; j0 < parts; j0 += 64) {
            float2 ml = float2{kPbNone, 0.0f};
            if (j0 + lane < parts) ml = *(const float2 *)(a.ml + at(j0 + lane) * 2);
            float top = ml.x;
#pragma unroll
            for (int s = 32; s; s >>= 1) top = fmaxf(top, __shfl_xor(top, s, 64));
            top = fmaxf(top, m);
            const float old = __builtin_amdgcn_exp2f(m - top), f = __builtin_amdgcn_exp2f(ml.x - top);
            float sum = ml.y * f;
#pragma unroll
            for (int s = 32; s; s >>= 1) sum += __shfl_xor(sum, s, 64);
            m = top, l = l * old + sum, x *= old, y *= old;
            const int n = min(parts - j0, 64);
            for (int j = 0; j < n; j += 8) {
                float2 v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = *(const float2 *)(a.o + at(j0 + min(j + k, n - 1)) * kD + lane * 2);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float w = j + k < n ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), min(j + k, n - 1))) : 0.0f;
                    x = __builtin_fmaf(v[k].x, w, x), y = __builtin_fmaf(v[k].y, w, y);
                }
            }
        }
        const int row = row0 + i, query = (int)fast_div(row, a.rep_magic, a.rep_shift);
        if (query >= a.T - d.x) return;
        const int64_t to = (int64_t)(d.x + query) * a.Hq + kvh * a.rep + row - query * a.rep;
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        const _Float16 p = to16<BF16>(x * inv), q = to16<BF16>(y * inv);
        *(half2p *)(a.out + to * kD + lane * 2) = half2p{p, q};
        if (a.lse && lane == 0) a.lse[to] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    }
}

constexpr int kPbSlots = 2 * kComputeUnits;            // workgroups at once

static int part_rows(const minikv_blk_shape &s, int32_t T)
{
    const int64_t rows = (int64_t)T * (s.Hq / s.Hkv);
    return (int)(rows < kPbRows ? rows : kPbRows);
}

// [header][parts][(m, l) of the parts' rows][their outputs]
size_t prompt_blk_workspace_bytes(const minikv_blk_shape &s, int32_t T)
{
    return 64 + (size_t)2 * kPbSlots * (sizeof(int4) + (size_t)part_rows(s, T) * (2 + kD) * sizeof(float));
}

int launch_prompt_blk(const minikv_blk_shape &s, int32_t T, const void *q, int64_t q_stride, const minikv_blk_cache &c, const int32_t *table,
                      const int32_t *q_len, const int32_t *cu, float sm_scale, void *out, float *lse, void *workspace, hipStream_t st)
{
    PromptBlkArgs a;
    a.q = (const uint16_t *)q, a.q_stride = q_stride, a.K = c.K, a.V = c.V, a.Ks = c.Ks, a.Vs = c.Vs;
    a.table = table, a.q_len = q_len, a.cu = cu, a.out = (uint16_t *)out, a.lse = lse;
    a.R = s.R, a.T = T, a.Hq = s.Hq, a.Hkv = s.Hkv, a.rep = s.Hq / s.Hkv, a.n_blocks = s.n_blocks, a.width = s.max_blocks;
    a.shift = __builtin_ctz(s.block), a.c = sm_scale * kLog2e, a.slots = kPbSlots, a.part_rows = part_rows(s, T);
    a.header = (int *)workspace, a.parts = (int4 *)((char *)workspace + 64);
    a.ml = (float *)(a.parts + 2 * kPbSlots), a.o = a.ml + (size_t)2 * kPbSlots * a.part_rows * 2;
    fast_div_setup((uint32_t)s.Hkv, a.hkv_magic, a.hkv_shift);
    fast_div_setup((uint32_t)a.rep, a.rep_magic, a.rep_shift);
    const int64_t blocks = (int64_t)T * a.rep / kPbRows + (s.R < T ? s.R : T), items = blocks * s.Hkv + kPbSlots;
    if (items > 0x7fffff) return MINIKV_EINVAL;
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
    const int groups = (a.part_rows + kPbJoinRows - 1) / kPbJoinRows;
    const dim3 join(2 * kPbSlots * groups);
    if (bf16) hipLaunchKernelGGL((prompt_join_kernel<true>), join, threads, 0, st, a, groups);
    else hipLaunchKernelGGL((prompt_join_kernel<false>), join, threads, 0, st, a, groups);
    return hipGetLastError() == hipSuccess ? MINIKV_OK : MINIKV_ELAUNCH;
}

}  // namespace minikv
