// Blocks of the paged 8-bit cache that requests share, lose or move: forks of requests (kv_fork_blk), the copies that forks and
// moves ask for (kv_copy_blk), the blocks that no request names any more (kv_free_blk), and the used blocks moved to the front of the
// pool (kv_compact_blk).  See include/minikv.h for what they compute.
#include "decode_common.h"
#include "scan.h"

namespace minikv {

constexpr int kPgSegment = 1024;                       // table entries that a wave takes at once, sixteen a lane

// The waves of a launch take the requests' table rows in segments, one after the other: row and first entry of each.
struct Rows {
    int R, width, segments;
    uint32_t magic, shift;                             // division by segments
};
static Rows rows_of(const minikv_blk_shape &s)
{
    Rows r;
    r.R = s.R, r.width = s.max_blocks, r.segments = (s.max_blocks + kPgSegment - 1) / kPgSegment;
    fast_div_setup((uint32_t)r.segments, r.magic, r.shift);
    return r;
}
template <typename F> __device__ inline void each_segment(const Rows &a, int wave, int waves, F take)
{
    const uint32_t items = (uint32_t)a.R * a.segments;          // (far below 2^31 by the shape's rules)
    for (uint32_t i = wave; i < items; i += waves) {
        const int r = (int)fast_div(i, a.magic, a.shift);
        take(r, (int)(i - (uint32_t)r * a.segments) * kPgSegment);
    }
}
__device__ inline uint32_t blocks_of(int64_t tokens, int shift) { return (uint32_t)((tokens + (1 << shift) - 1) >> shift); }
__device__ inline int64_t clamped(int len, int width, int shift) { return min((int64_t)max(len, 0), (int64_t)width << shift); }

// =====================================================================================================================
// kv_fork_blk

struct ForkArgs {
    const int32_t *q_len, *parent, *n_keep, *table, *ring, *state;
    int32_t *q_len_next, *table_next, *state_next, *src, *dst;
    Rows rows;
    int N, shift;
};

constexpr int kFkMost = kMaxRequests / kScanThreads;   // requests of a thread, consecutive ones

// The waves of the grid copy table rows, whole blocks only.  The first workgroup settles the last blocks: who inherits each parent's (the
// lowest request that keeps all of it; a minimum, so in whatever order), who needs a fresh one (one scan), which of the ring's it gets.  Three round
// trips to memory: the requests, their last blocks and rows, the ring.
__global__ __launch_bounds__(kScanThreads) void fork_blk_kernel(ForkArgs a)
{
    extern __shared__ int lds[];
    const int R = a.rows.R, width = a.rows.width;
    int *heir = lds, *from = lds + R, *keep_of = lds + 2 * R, *held = lds + 3 * R;     // keep_of: without a fresh last block's tokens
    __shared__ uint32_t part[1][kScanThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), unit = (1 << a.shift) - 1;
    const int head = min(max(a.state[0], 0), a.N - 1), n_free = min(max(a.state[1], 0), a.N);
    const int per = (R + kScanThreads - 1) / kScanThreads, r0 = min(tid * per, R), mine = min(R - r0, per);

    for (int r = tid; r < R; r += kScanThreads) {
        const int p = a.parent[r], n = a.n_keep[r];
        held[r] = (int)clamped(a.q_len[r], width, a.shift);
        heir[r] = 0x7fffffff, from[r] = (uint32_t)p < (uint32_t)R ? p : -1, keep_of[r] = max(n, 0);
    }
    __syncthreads();
    for (int r = tid; r < R; r += kScanThreads) keep_of[r] = from[r] < 0 ? 0 : min(keep_of[r], held[from[r]]);
    __syncthreads();
    int keep[kFkMost], tail[kFkMost];                  // tail: the last block, partly filled
    bool whole[kFkMost];
    if (blockIdx.x == 0)
#pragma unroll
        for (int j = 0; j < kFkMost; ++j)
            if (j < mine) {
                const int r = r0 + j, p = from[r];
                keep[j] = keep_of[r], tail[j] = -1, whole[j] = false;
                if (keep[j] & unit) tail[j] = a.table[(int64_t)p * width + (keep[j] >> a.shift)], whole[j] = keep[j] == held[p];
                if (whole[j]) atomicMin(&heir[p], p == r ? -1 : r);
            }
    each_segment(a.rows, blockIdx.x * (kScanThreads / 64) + wave, gridDim.x * (kScanThreads / 64), [&](int r, int first) {
        const int whole_blocks = keep_of[r] >> a.shift;
        if (first >= whole_blocks) return;
        const int32_t *in = a.table + (int64_t)from[r] * width;
        int32_t *out = a.table_next + (int64_t)r * width;
#pragma unroll 4
        for (int i = first + lane; i < min(whole_blocks, first + kPgSegment); i += 64) out[i] = in[i];
    });
    if (blockIdx.x) return;
    __syncthreads();
    uint32_t need[1] = {0}, total[1];
    bool wants[kFkMost];
#pragma unroll
    for (int j = 0; j < kFkMost; ++j)
        if (j < mine) {
            const int r = r0 + j;
            wants[j] = (keep[j] & unit) && (uint32_t)tail[j] < (uint32_t)a.N && !(whole[j] && heir[from[r]] == (from[r] == r ? -1 : r));
            need[0] += wants[j];
        }
    block_scan(need, {0x7fffffffu}, part, total);
    uint32_t taken = need[0];
#pragma unroll
    for (int j = 0; j < kFkMost; ++j)
        if (j < mine) {
            const int r = r0 + j;
            int got = -1, old = -1;
            if (wants[j]) {
                if (taken < (uint32_t)n_free) {
                    const uint32_t at = (uint32_t)head + taken;
                    got = a.ring[at >= (uint32_t)a.N ? at - a.N : at], old = tail[j];
                } else {
                    keep[j] &= ~unit;
                }
                ++taken;
            }
            if (keep[j] & unit) a.table_next[(int64_t)r * width + (keep[j] >> a.shift)] = old >= 0 ? got : tail[j];
            a.q_len_next[r] = keep[j], a.src[r] = old, a.dst[r] = got;
        }
    if (tid == 0) {
        const uint32_t given = min(total[0], (uint32_t)n_free), at = (uint32_t)head + given;
        a.state_next[0] = (int)(at >= (uint32_t)a.N ? at - a.N : at), a.state_next[1] = n_free - (int)given;
    }
}

int launch_fork_blk(const minikv_blk_shape &s, const int32_t *q_len, const int32_t *parent, const int32_t *n_keep, const int32_t *table,
                    const int32_t *ring, const int32_t *state, int32_t *q_len_next, int32_t *table_next, int32_t *state_next, int32_t *src,
                    int32_t *dst, hipStream_t st)
{
    ForkArgs a;
    a.q_len = q_len, a.parent = parent, a.n_keep = n_keep, a.table = table, a.ring = ring, a.state = state;
    a.q_len_next = q_len_next, a.table_next = table_next, a.state_next = state_next, a.src = src, a.dst = dst;
    a.rows = rows_of(s), a.N = s.n_blocks, a.shift = __builtin_ctz(s.block);
    const int64_t items = (int64_t)s.R * a.rows.segments, grid = (items + kScanThreads / 64 - 1) / (kScanThreads / 64);
    hipLaunchKernelGGL(fork_blk_kernel, dim3((unsigned)(grid < kComputeUnits ? grid : kComputeUnits)), dim3(kScanThreads),
                       4 * s.R * sizeof(int), st, a);
    return hipGetLastError() == hipSuccess ? MINIKV_OK : MINIKV_ELAUNCH;
}

// =====================================================================================================================
// kv_copy_blk

constexpr int kCpCaches = 64;                          // caches of a launch (their pointers are its arguments)
constexpr int kCpRound = 2048;                         // pairs looked at between two barriers
constexpr int kCpThreads = 256;

struct CopyArgs {
    minikv_blk_cache caches[kCpCaches];
    const int32_t *src, *dst;
    int64_t block_bytes;                               // of K, and of V, of one block: its heads lie one behind the other
    int n_pairs, N, Hkv, n_caches, chunk, chunks;      // a workgroup copies `chunk` bytes at a time
};

typedef uint32_t u4p __attribute__((ext_vector_type(4)));

// Memory: 0.19 GB of 1500 moved blocks read and written 41 us, 4.8 TB/s; 0.38 GB of copies of one block per layer 80 us.  Stores carry the streaming
// hint, loads do not: forks behind one prefix read the same block many times (with the hint on both 113 us and 43, on neither 101 and 49).
// Pairs come with holes.  Every workgroup lists the pairs of a round that are none in local memory, in their order, and takes
// its share of (pair, cache, K or V, chunk), counted through all rounds, so that the shares are even wherever the holes are.
__global__ __launch_bounds__(kCpThreads) void copy_blk_kernel(CopyArgs a)
{
    __shared__ int2 list[kCpRound];
    __shared__ int counts[kCpRound / kCpThreads][kCpThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t per = (uint32_t)a.n_caches * 2 * a.chunks;
    uint32_t next = blockIdx.x;                        // the workgroup's next item, counted from the round's first
    for (int base = 0; base < a.n_pairs; base += kCpRound) {
        int2 pair[kCpRound / kCpThreads];
        uint64_t live[kCpRound / kCpThreads];
#pragma unroll
        for (int j = 0; j < kCpRound / kCpThreads; ++j) {
            const int64_t i = (int64_t)base + j * kCpThreads + tid;
            pair[j] = i < a.n_pairs ? int2{a.src[i], a.dst[i]} : int2{-1, -1};
        }
#pragma unroll
        for (int j = 0; j < kCpRound / kCpThreads; ++j) {
            live[j] = __ballot((uint32_t)pair[j].x < (uint32_t)a.N && (uint32_t)pair[j].y < (uint32_t)a.N && pair[j].x != pair[j].y);
            if (lane == 0) counts[j][wave] = __builtin_popcountll(live[j]);
        }
        __syncthreads();
        int at = 0;
#pragma unroll
        for (int j = 0; j < kCpRound / kCpThreads; ++j) {
            int before = at;
#pragma unroll
            for (int w = 0; w < kCpThreads / 64; ++w) {
                if (w < wave) before += counts[j][w];
                at += counts[j][w];
            }
            if (live[j] >> lane & 1)
                list[before + __builtin_amdgcn_mbcnt_hi((uint32_t)(live[j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)live[j], 0))] = pair[j];
        }
        __syncthreads();
        const uint32_t items = (uint32_t)at * per;
        for (; next < items; next += gridDim.x) {
            const uint32_t i = __builtin_amdgcn_readfirstlane(next), p = i / per, u = i - p * per, c = u / (2 * a.chunks), v = u - c * (2 * a.chunks);
            const bool is_v = v >= (uint32_t)a.chunks;
            const uint32_t part = v - (is_v ? a.chunks : 0);
            const int from = __builtin_amdgcn_readfirstlane(list[p].x), to = __builtin_amdgcn_readfirstlane(list[p].y);
            const minikv_blk_cache &m = a.caches[c];
            uint8_t *codes = is_v ? m.V : m.K;
            const int64_t first = (int64_t)part * a.chunk;
            const int n = (int)min((int64_t)a.chunk, a.block_bytes - first);
            const uint8_t *in = codes + from * a.block_bytes + first;
            uint8_t *out = codes + to * a.block_bytes + first;
            for (int o = tid * 16; o < n; o += 4 * kCpThreads * 16) {
                u4p x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (o + k * kCpThreads * 16 < n) x[k] = *(const u4p *)(in + o + k * kCpThreads * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (o + k * kCpThreads * 16 < n) __builtin_nontemporal_store(x[k], (u4p *)(out + o + k * kCpThreads * 16));
            }
            if (part == 0) {
                float *scales = is_v ? m.Vs : m.Ks;
                for (int h = tid; h < a.Hkv; h += kCpThreads) scales[(int64_t)to * a.Hkv + h] = scales[(int64_t)from * a.Hkv + h];
            }
        }
        next -= items;
        __syncthreads();                               // the list has been read
    }
}

int launch_copy_blk(const minikv_blk_shape &s, int32_t n_caches, const minikv_blk_cache *caches, int32_t n_pairs, const int32_t *src,
                    const int32_t *dst, hipStream_t st)
{
    CopyArgs a;
    a.src = src, a.dst = dst, a.n_pairs = n_pairs, a.N = s.n_blocks, a.Hkv = s.Hkv;
    a.block_bytes = (int64_t)s.Hkv * s.block * kD;
    // 16 KB at a time, or what makes 64 chunks of a block: a round's items are counted in 32 bits
    a.chunk = 16384;
    while (a.block_bytes > (int64_t)a.chunk * 64) a.chunk *= 2;
    a.chunks = (int)((a.block_bytes + a.chunk - 1) / a.chunk);
    for (int32_t first = 0; first < n_caches; first += kCpCaches) {
        a.n_caches = n_caches - first < kCpCaches ? n_caches - first : kCpCaches;
        for (int32_t i = 0; i < a.n_caches; ++i) a.caches[i] = caches[first + i];
        const int64_t items = (int64_t)n_pairs * a.n_caches * 2 * a.chunks;
        hipLaunchKernelGGL(copy_blk_kernel, dim3((unsigned)(items < kComputeUnits * 8 ? items : kComputeUnits * 8)), dim3(kCpThreads), 0, st, a);
        if (hipGetLastError() != hipSuccess) return MINIKV_ELAUNCH;
    }
    return MINIKV_OK;
}

// =====================================================================================================================
// kv_free_blk, kv_compact_blk

// Workspace: a ticket, the numbers of moves and of used blocks, and PoolWords for 1024 blocks each, at the same places for every shape.
struct PoolWords {
    uint32_t bits[32];                                 // the blocks that a table names (zero between calls)
    uint2 kept[32];                                    // for the new rows: bits, and how many used blocks lie below them
};
constexpr int kPlHeader = 128;
struct PoolArgs {
    const int32_t *q_len, *table;
    int32_t *table_next, *ring, *state, *src, *dst;
    int *header;                                       // ticket, moves, used blocks
    PoolWords *marks;
    Rows rows;
    int N, words, shift, n_pairs;
    __device__ uint32_t &bits(int w) const { return marks[w >> 5].bits[w & 31]; }
    __device__ uint2 &kept(int w) const { return marks[w >> 5].kept[w & 31]; }
};

constexpr int kPlPer = 4;                              // blocks of a thread of the second launch
constexpr int kPlBlocks = kPlPer * kScanThreads, kPlWords = kPlBlocks / 32;

__global__ __launch_bounds__(256) void mark_blk_kernel(PoolArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    each_segment(a.rows, blockIdx.x * 4 + wave, gridDim.x * 4, [&](int r, int first) {
        const int32_t *row = a.table + (int64_t)r * a.rows.width;
        const int len = a.q_len[r], end = min(a.rows.width, first + kPgSegment);
        auto mark = [&](int b) {
            if ((uint32_t)b < (uint32_t)a.N) atomicOr(&a.bits(b >> 5), 1u << (b & 31));
        };
        int b[4];                                      // (the first entries come with the length)
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = first + lane + 64 * j < end ? row[first + lane + 64 * j] : -1;
        const int n = min((int)blocks_of(clamped(len, a.rows.width, a.shift), a.shift), end);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (first + lane + 64 * j < n) mark(b[j]);
#pragma unroll 4
        for (int i = first + lane + 256; i < n; i += 64) mark(row[i]);
    });
}

// A workgroup has 4096 blocks and counts for itself what lies below them (a bit a block: 7.5 KB for 60000 of them).  With U blocks used, the
// used ones from U on move, the highest first, each to the lowest block that is left: of a used block count those above, of a free one those
// below, and it moves, or is moved into, if that is less than the number of moves.  The ring's place of a block follows from the same counts.
// The last workgroup clears the bits for the next call.
__global__ __launch_bounds__(kScanThreads) void sweep_blk_kernel(PoolArgs a)
{
    __shared__ uint32_t part[2][kScanThreads / 64], here[kPlWords], below_of[kPlWords], last;
    const int tid = threadIdx.x, first = blockIdx.x * kPlWords;
    uint32_t sums[2] = {0, 0}, totals[2];
    const uint32_t word = tid < kPlWords && first + tid < a.words ? a.bits(first + tid) : 0;
    for (int w = tid; w < a.words; w += kScanThreads) {
        const uint32_t n = __builtin_popcount(a.bits(w));
        sums[0] += n, sums[1] += w < first ? n : 0;
    }
    block_scan(sums, {0x7fffffffu, 0x7fffffffu}, part, totals);
    const int used = (int)totals[0], below = (int)totals[1];
    int moves = 0;
    if (a.n_pairs) {
        uint32_t n[1] = {0}, total[1];
        for (int w = (used >> 5) + tid; w < a.words; w += kScanThreads)
            n[0] += __builtin_popcount(a.bits(w) & (w == used >> 5 ? ~0u << (used & 31) : ~0u));
        __syncthreads();
        block_scan(n, {0x7fffffffu}, part, total);
        moves = min((int)total[0], a.n_pairs);
    }
    uint32_t n[1] = {(uint32_t)__builtin_popcount(word)}, total[1];
    __syncthreads();
    block_scan(n, {0x7fffffffu}, part, total);
    if (tid < kPlWords) here[tid] = word, below_of[tid] = n[0];
    if (a.table_next && tid < kPlWords && first + tid < a.words) a.kept(first + tid) = uint2{word, below + n[0]};
    __syncthreads();
    if (tid == 0) last = atomicAdd(&a.header[0], 1) == (int)gridDim.x - 1;

    const uint32_t bits = here[tid * kPlPer >> 5];
#pragma unroll
    for (int j = 0; j < kPlPer; ++j) {
        const int at = tid * kPlPer + j, b = first * 32 + at;
        if (b >= a.N) break;
        const bool is_used = bits >> (at & 31) & 1;
        const int low = below + (int)below_of[at >> 5] + __builtin_popcount(bits & ((1u << (at & 31)) - 1));      // used blocks below b
        const int free_low = b - low, above = used - low - is_used;
        const bool gone = is_used && above < moves, taken = !is_used && free_low < moves;
        if (gone) a.src[above] = b;
        if (taken) a.dst[free_low] = b;
        // free afterwards below b: the free ones that were not taken, and the moved ones
        if (gone || (!is_used && !taken)) a.ring[free_low - min(moves, free_low) + moves - min(moves, used - low)] = b;
    }
    for (int64_t k = (int64_t)blockIdx.x * kScanThreads + tid + moves; k < a.n_pairs; k += (int64_t)gridDim.x * kScanThreads) a.src[k] = a.dst[k] = -1;
    if (blockIdx.x == 0 && tid == 0) a.state[0] = 0, a.state[1] = a.N - used, a.header[1] = moves, a.header[2] = used;
    __syncthreads();
    if (last) {                                        // (everybody has read the bits)
        for (int w = tid; w < a.words; w += kScanThreads) a.bits(w) = 0;
        if (tid == 0) a.header[0] = 0;
    }
}

__global__ __launch_bounds__(256) void retable_blk_kernel(PoolArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int moves = a.header[1], used = a.header[2], lowest = moves ? a.src[moves - 1] : a.N;          // named blocks from there on have moved
    each_segment(a.rows, blockIdx.x * 4 + wave, gridDim.x * 4, [&](int r, int first) {
        const int n = (int)blocks_of(clamped(a.q_len[r], a.rows.width, a.shift), a.shift);
        const int32_t *in = a.table + (int64_t)r * a.rows.width;
        int32_t *out = a.table_next + (int64_t)r * a.rows.width;
#pragma unroll 4
        for (int i = first + lane; i < min(n, first + kPgSegment); i += 64) {
            int b = in[i];
            if (b >= lowest && b < a.N) {
                const uint2 k = a.kept(b >> 5);
                b = a.dst[used - 1 - (int)(k.y + __builtin_popcount(k.x & ((1u << (b & 31)) - 1)))];            // (by the used blocks above it)
            }
            out[i] = b;
        }
    });
}

// The whole of it in one workgroup, with nothing but local memory between the steps, where tables and pool are small: what costs then are launches
// and round trips to memory, one for lengths and table.
constexpr int kPlSmall = 16384;                        // entries of all rows, and blocks

__global__ __launch_bounds__(kScanThreads) void small_pool_blk_kernel(PoolArgs a)
{
    extern __shared__ int lds[];
    __shared__ uint32_t part[1][kScanThreads / 64];
    uint32_t *bits = (uint32_t *)lds, *below_of = bits + a.words, *count = bits + 2 * a.words, *to = count + a.rows.R;       // to: of each move
    const int tid = threadIdx.x, entries = a.rows.R * a.rows.width;
    uint32_t mine = 0;                                 // the thread's entries that count
    for (int w = tid; w < a.words; w += kScanThreads) bits[w] = 0;
    for (int r = tid; r < a.rows.R; r += kScanThreads) count[r] = blocks_of(clamped(a.q_len[r], a.rows.width, a.shift), a.shift);
    constexpr int kMine = kPlSmall / kScanThreads;     // entries of a thread
    int entry[kMine];
#pragma unroll
    for (int j = 0; j < kMine; ++j) entry[j] = tid + j * kScanThreads < entries ? a.table[tid + j * kScanThreads] : -1;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        const int i = tid + j * kScanThreads;
        if (i >= entries) break;
        const int r = (int)fast_div(i, a.rows.magic, a.rows.shift);                   // (by the width)
        const bool counts = i - r * a.rows.width < (int)count[r], there = (uint32_t)entry[j] < (uint32_t)a.N;
        mine |= (uint32_t)counts << j;
        if (counts && there) atomicOr(&bits[entry[j] >> 5], 1u << (entry[j] & 31));
    }
    __syncthreads();
    uint32_t n[1] = {tid < a.words ? (uint32_t)__builtin_popcount(bits[tid]) : 0}, total[1];            // (at most 512 words)
    block_scan(n, {0x7fffffffu}, part, total);
    if (tid < a.words) below_of[tid] = n[0];
    __syncthreads();
    const int used = (int)total[0];
    auto below = [&](int b) { return (int)below_of[b >> 5] + __builtin_popcount(bits[b >> 5] & ((1u << (b & 31)) - 1)); };        // used blocks below b < N
    const int moves = used < a.N ? min(used - below(used), a.n_pairs) : 0;
    for (int b = tid; b < a.N; b += kScanThreads) {
        const bool is_used = bits[b >> 5] >> (b & 31) & 1;
        const int low = below(b), free_low = b - low, above = used - low - is_used;
        const bool gone = is_used && above < moves, taken = !is_used && free_low < moves;
        if (gone) a.src[above] = b;
        if (taken) a.dst[free_low] = b, to[free_low] = b;
        if (gone || (!is_used && !taken)) a.ring[free_low - min(moves, free_low) + moves - min(moves, used - low)] = b;      // (as in sweep_blk_kernel)
    }
    for (int k = tid + moves; k < a.n_pairs; k += kScanThreads) a.src[k] = a.dst[k] = -1;
    if (tid == 0) a.state[0] = 0, a.state[1] = a.N - used;
    if (!a.table_next) return;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMine; ++j)
        if (mine >> j & 1) {
            const int above = (uint32_t)entry[j] < (uint32_t)a.N ? used - below(entry[j]) - 1 : moves;
            a.table_next[tid + j * kScanThreads] = above < moves ? (int)to[above] : entry[j];
        }
}

size_t pool_workspace_bytes(const minikv_blk_shape &s)
{
    return kPlHeader + ((size_t)s.n_blocks + 1023) / 1024 * sizeof(PoolWords);
}

int launch_pool_blk(const minikv_blk_shape &s, const int32_t *q_len, const int32_t *table, int32_t *table_next, int32_t *ring, int32_t *state,
                    int32_t n_pairs, int32_t *src, int32_t *dst, void *workspace, hipStream_t st)
{
    PoolArgs a;
    a.q_len = q_len, a.table = table, a.table_next = table_next, a.ring = ring, a.state = state, a.src = src, a.dst = dst;
    a.rows = rows_of(s), a.N = s.n_blocks, a.words = (s.n_blocks + 31) / 32, a.shift = __builtin_ctz(s.block), a.n_pairs = n_pairs;
    a.header = (int *)workspace, a.marks = (PoolWords *)((char *)workspace + kPlHeader);
    if ((int64_t)s.R * s.max_blocks <= kPlSmall && s.n_blocks <= kPlSmall) {
        fast_div_setup((uint32_t)s.max_blocks, a.rows.magic, a.rows.shift);
        const size_t lds = (size_t)(2 * a.words + s.R + (n_pairs < s.n_blocks / 2 ? n_pairs : s.n_blocks / 2)) * sizeof(uint32_t);
        hipLaunchKernelGGL(small_pool_blk_kernel, dim3(1), dim3(kScanThreads), lds, st, a);
        return hipGetLastError() == hipSuccess ? MINIKV_OK : MINIKV_ELAUNCH;
    }
    const int64_t items = (int64_t)s.R * a.rows.segments, grid = (items + 3) / 4;
    const dim3 rows((unsigned)(grid < kComputeUnits * 8 ? grid : kComputeUnits * 8)), pool((unsigned)((s.n_blocks + kPlBlocks - 1) / kPlBlocks));
    hipLaunchKernelGGL(mark_blk_kernel, rows, dim3(256), 0, st, a);
    hipLaunchKernelGGL(sweep_blk_kernel, pool, dim3(kScanThreads), 0, st, a);
    if (table_next) hipLaunchKernelGGL(retable_blk_kernel, rows, dim3(256), 0, st, a);
    return hipGetLastError() == hipSuccess ? MINIKV_OK : MINIKV_ELAUNCH;
}

}  // namespace minikv
