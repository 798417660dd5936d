// The paged 8-bit cache: block tables and slot maps from lengths on the device (kv_assign_blk), and the filing of new rows
// as e4m3 codes with one power-of-two scale per (block, head) (kv_quantize_blk).  See include/minikv.h for what they compute.
#include "decode_common.h"

namespace minikv {

// =====================================================================================================================
// kv_assign_blk

struct AssignArgs {
    const int32_t *q_len, *n_new, *state;
    int32_t *table, *ring, *q_len_next, *state_next, *cu, *slots;
    int R, N, width, shift, n_slots;
};

constexpr int kAsThreads = 1024;
constexpr int kAsMost = kMaxRequests / kAsThreads;     // requests of a thread, consecutive ones
constexpr int kAsFew = 3;                              // rows of all its requests that a thread writes the slots of itself
constexpr uint32_t kRefused = 0x80000000u;

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
__device__ inline void block_scan(uint32_t (&v)[N], const uint32_t (&cap)[N], uint32_t (*part)[kAsThreads / 64], uint32_t (&total)[N])
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
        const uint32_t sums = wave_scan(lane < kAsThreads / 64 ? part[i][lane] : 0, cap[i]);
        total[i] = __builtin_amdgcn_readlane(sums, kAsThreads / 64 - 1);
        const uint32_t before = wave ? (uint32_t)__shfl((int)sums, wave - 1, 64) : 0;
        const uint32_t ex = __builtin_amdgcn_update_dpp(0, in[i], 0x138, 0xf, 0xf, false);     // wave_shr 1
        v[i] = sat_add(before, lane ? ex : 0, cap[i]);
    }
}

// last i in [0, n) with (v[i] without its top bit) <= x; v ascends, v[0] = 0
__device__ inline int find(const uint32_t *v, int n, uint32_t x)
{
    int lo = 0;
    for (int step = n > 1 ? 1 << (31 - __builtin_clz(n - 1)) : 0; step; step >>= 1)
        if (lo + step < n && (v[lo + step] & ~kRefused) <= x) lo += step;
    return lo;
}

// Every workgroup scans all the requests (two scans: rows first, because a request whose rows do not fit asks for no blocks).
// Where no thread has more than kAsFew new rows in all (at most so many each of its one to eight requests), a decoding step, it writes
// their slots and table entries itself; else three prefix sums in local memory make slots, table entries and returned blocks three
// flat loops over the grid, each element finding its request by bisection.  Us, own thread / loops: 256 requests of 1 row 3.9 / 5.2,
// of 3 4.8 / 5.4, of 4 5.2 / 5.5, of 8 7.5 / 6.0; 1024 of 3 6.3 / 6.5, of 4 7.6 / 6.7; 1500 of 1 5.5 / 6.5, of 2 7.1 / 6.8; 3000 of 1 7.5 /
// 7.8; 8192 of 1 27.8 / 20.9, of 8 103 / 22.  New slots are computed from the ring, not from the table entries that another
// workgroup may not have written yet, so one launch does it all and nothing waits for anything.  What bounds it is latency, two
// dependent loads and the scans: 4.2 us for a step of 256 requests, 6.4 for 64 prompts of 131072 tokens, 9 for 1000 of 100000.
__global__ __launch_bounds__(kAsThreads) void assign_blk_kernel(AssignArgs a)
{
    extern __shared__ uint32_t lds[];
    uint32_t *rows = lds, *need = lds + a.R, *over = lds + 2 * a.R;     // exclusive prefix sums per request
    __shared__ uint32_t part[3][kAsThreads / 64], popped, many;
    const int tid = threadIdx.x, gtid = blockIdx.x * kAsThreads + tid, gsize = gridDim.x * kAsThreads;
    const int64_t most = (int64_t)a.width << a.shift;
    const int head = min(max(a.state[0], 0), a.N - 1), n_free = min(max(a.state[1], 0), a.N);
    const uint32_t kRows = 0x7fffffff, back = a.N - n_free;            // blocks that can come back
    const uint32_t unit = (1u << a.shift) - 1;

    auto len_of = [&](int r) { return (int)min((int64_t)max(a.q_len[r], 0), most); };
    auto blocks = [&](uint32_t tokens) { return (tokens + unit) >> a.shift; };       // (at most 2^30 + 2^31)
    // (of a block outside the pool: outside the pool as well, never another block's)
    auto slot_in = [&](int id, int pos) { return (uint32_t)id <= 0x7fffffffu >> a.shift ? (id << a.shift) + (pos & (int)unit) : -1; };
    auto wrap = [&](uint32_t i) { return i >= (uint32_t)a.N ? i - a.N : i; };          // i < 2 N

    const int per = (a.R + kAsThreads - 1) / kAsThreads, r0 = min(tid * per, a.R), mine = min(a.R - r0, per);
    int len[kAsMost], add[kAsMost];
    uint32_t sum[1] = {0}, total[1], sums[2] = {0, 0}, totals[2], largest = 0;
    if (tid == 0) popped = many = 0;
#pragma unroll
    for (int j = 0; j < kAsMost; ++j)
        if (j < mine) {
            len[j] = len_of(r0 + j), add[j] = a.n_new[r0 + j];
            sum[0] = sat_add(sum[0], max(add[j], 0), kRows), largest = max(largest, (uint32_t)max(add[j], 0));
        }
    block_scan(sum, {kRows}, part, total);
    if (largest > kAsFew || largest * per > kAsFew) many = 1;
    int end = a.R;                                     // requests from here on lie behind the slots although the saturated sum does not tell
    if (total[0] == kRows && (uint32_t)a.n_slots == kRows) {
        int64_t exact = 0;
        for (end = 0; end < a.R && (exact += max(a.n_new[end], 0)) <= kRows; ++end);
    }
    uint32_t row[kAsMost], nd[kAsMost], ov[kAsMost], at = sum[0];
#pragma unroll
    for (int j = 0; j < kAsMost; ++j)                  // (need <= new rows <= n_slots in all: no overflow)
        if (j < mine) {
            const uint32_t more = max(add[j], 0), after = blocks((uint32_t)len[j] + more), held = blocks(len[j]);
            row[j] = at, at = sat_add(at, more, kRows);
            const bool fits = add[j] >= 0 && after <= (uint32_t)a.width && at <= (uint32_t)a.n_slots && r0 + j < end;
            nd[j] = fits ? after - held : kRefused;
            ov[j] = add[j] < 0 ? min(held, back) : 0;
            sums[0] += nd[j] & ~kRefused, sums[1] = sat_add(sums[1], ov[j], back);
        }
    block_scan(sums, {kRows, back}, part + 1, totals);
    const bool few = !many;
    uint32_t take = sums[0], give = sums[1], pop = 0;
#pragma unroll
    for (int j = 0; j < kAsMost; ++j)
        if (j < mine) {
            const int r = r0 + j;
            const uint32_t n = nd[j] & ~kRefused, first = take;
            take += n;
            const bool ok = !(nd[j] & kRefused) && (n == 0 || take <= (uint32_t)n_free);
            if (ok && n) pop = take;                   // (ascending in the accepted ones)
            if (!few) rows[r] = row[j], need[r] = first | (ok ? 0u : kRefused);
            if (totals[1]) over[r] = give;
            give = sat_add(give, ov[j], back);
            if (blockIdx.x == 0) {
                a.q_len_next[r] = add[j] < 0 ? 0 : ok ? len[j] + add[j] : len[j];
                a.cu[r] = (int)row[j];
                if (few) {
                    const int held = (int)blocks(len[j]);
                    int32_t *entry = a.table + (int64_t)r * a.width;
                    for (int i = 0; i < add[j]; ++i) {
                        const int pos = len[j] + i, b = pos >> a.shift;
                        int slot = -1;
                        if (ok) {
                            const int id = b < held ? entry[b] : a.ring[wrap(head + first + (b - held))];
                            if (b >= held) entry[b] = id;
                            slot = slot_in(id, pos);
                        }
                        if (row[j] + i < (uint32_t)a.n_slots) a.slots[row[j] + i] = slot;
                    }
                }
            }
        }
    if (pop) atomicMax(&popped, pop);
    __syncthreads();
    pop = popped;
    if (blockIdx.x == 0 && tid == 0) {
        a.cu[a.R] = (int)total[0];
        a.state_next[0] = (int)wrap(head + pop), a.state_next[1] = n_free - (int)pop + (int)totals[1];
    }
    if (few) {
        for (int64_t t = (int64_t)total[0] + gtid; t < a.n_slots; t += gsize) a.slots[t] = -1;
    } else {
        for (int64_t at = gtid; at < a.n_slots; at += gsize) {
            const int t = (int)at;
            int slot = -1;
            const int r = find(rows, a.R, t);
            if ((uint32_t)t < total[0] && !(need[r] & kRefused)) {
                const int len = len_of(r), pos = len + (t - (int)rows[r]);
                const int b = pos >> a.shift, held = (int)blocks(len);
                const int id = b < held ? a.table[(int64_t)r * a.width + b] : a.ring[wrap(head + need[r] + (b - held))];
                slot = slot_in(id, pos);
            }
            a.slots[t] = slot;
        }
        for (uint32_t p = gtid; p < pop; p += gsize) {
            const int r = find(need, a.R, p);
            a.table[(int64_t)r * a.width + blocks(len_of(r)) + (p - need[r])] = a.ring[wrap(head + p)];
        }
    }
    for (uint32_t p = gtid; p < totals[1]; p += gsize) {
        const int r = find(over, a.R, p);
        a.ring[wrap(wrap(head + n_free) + p)] = a.table[(int64_t)r * a.width + (p - over[r])];
    }
}

int launch_assign_blk(const minikv_blk_shape &s, const int32_t *q_len, const int32_t *n_new, int32_t *table, int32_t *ring,
                      const int32_t *state, int32_t *q_len_next, int32_t *state_next, int32_t *cu, int32_t *slots,
                      int32_t n_slots, hipStream_t st)
{
    AssignArgs a;
    a.q_len = q_len, a.n_new = n_new, a.state = state, a.table = table, a.ring = ring;
    a.q_len_next = q_len_next, a.state_next = state_next, a.cu = cu, a.slots = slots;
    a.R = s.R, a.N = s.n_blocks, a.width = s.max_blocks, a.shift = __builtin_ctz(s.block), a.n_slots = n_slots;
    const int64_t grid = ((int64_t)n_slots + kAsThreads - 1) / kAsThreads;
    hipLaunchKernelGGL(assign_blk_kernel, dim3((unsigned)(grid < 1 ? 1 : grid < kComputeUnits ? grid : kComputeUnits)),
                       dim3(kAsThreads), 3 * s.R * sizeof(uint32_t), st, a);
    return hipGetLastError() == hipSuccess ? MINIKV_OK : MINIKV_ELAUNCH;
}

// =====================================================================================================================
// kv_quantize_blk

typedef float float2v __attribute__((ext_vector_type(2)));

struct FileArgs {
    const uint16_t *X[2];                              // K and V rows
    int64_t stride[2];
    uint8_t *codes[2];
    float *scales[2];
    const int32_t *slots;
    int n_tok, Hkv, shift, rows, chunk;                // rows = n_blocks * block
    uint32_t heads_magic, heads_shift;                 // division by 2 Hkv
};

typedef uint32_t u4v __attribute__((ext_vector_type(4)));

__device__ inline uint32_t wave_max_u32(uint32_t v)    // the same in every lane
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));     // row_shr 1, 2, 4, 8
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));     // row_bcast 15, 31
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ inline uint32_t max_u16x2(uint32_t a, uint32_t b)
{
    typedef uint16_t ushort2v __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, a), __builtin_bit_cast(ushort2v, b)));
}
template <bool BF16> __device__ inline float from16(uint32_t bits)
{
    if (BF16) return __uint_as_float(bits << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

// The smallest power of two s >= 2^-126 with amax <= 448 s: 448 = 1.75 * 2^8, so from the exponent of amax alone, one more
// where its mantissa is beyond 1.75.
__device__ inline float scale_for(float amax)
{
    if (amax == 0.0f) return 0.0f;
    const uint32_t bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000);
    return __uint_as_float((uint32_t)(max(e, -126) + 127) << 23);
}

// p is the binary32 number nearest to a value and r that value less p (or 0): of the two numbers next to the value the one whose
// last bit is set, p itself if it is the value.  Rounded on to fewer bits this gives what the value gives (p could lie on a tie that the value misses).
__device__ inline float to_odd(float p, float r)
{
    const uint32_t b = __float_as_uint(p);
    if (r == 0.0f || (b & 1)) return p;
    return __uint_as_float((r > 0.0f) != (b >> 31) ? b + 1 : b - 1);
}

// A wave takes the runs (consecutive tokens of one block) that begin among its `chunk` tokens, for one head and one of K
// and V (neighbouring waves take the heads of the same tokens, which lie side by side), so that a block's scale has one
// owner and no barrier or atomic is needed.  Sixteen lanes hold a row, four rows an instruction; up to ROWS rows, a block,
// stay in registers between the maximum (on the 16-bit magnitudes, whose order is that of the unsigned integers for fp16
// and bf16 alike) and the rounding.  Two dependent round trips: the slots of the chunk and the 64 behind it, which lanes
// then pass on, and the rows.  32768 tokens of 8 heads 38.7 us, 5.2 TB/s (44.3 with the slots read again for each run and
// each row); with 128 rows there are no registers for the offsets too, and those slots are read again (51 us instead of 43).
template <int ROWS, bool BF16>
__global__ __launch_bounds__(256) void quantize_blk_kernel(FileArgs a)
{
    const int lane = threadIdx.x & 63, c = lane & 15, sub = lane >> 4;
    const uint32_t item = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t part = fast_div(item, a.heads_magic, a.heads_shift), of = item - part * 2 * a.Hkv;
    const int64_t begin = (int64_t)part * a.chunk;
    if (begin >= a.n_tok) return;
    const int first = (int)begin, which = of >= (uint32_t)a.Hkv, h = (int)of - (which ? a.Hkv : 0);
    const uint16_t *X = (which ? a.X[1] : a.X[0]) + (int64_t)h * kD + c * 8;
    const int64_t stride = which ? a.stride[1] : a.stride[0];
    auto slot_of = [&](int64_t i) { return i >= 0 && i < a.n_tok ? a.slots[i] : -1; };
    auto block_of = [&](int slot) { return (uint32_t)slot < (uint32_t)a.rows ? slot >> a.shift : -1; };      // -1: none
    // the slots of the wave's tokens, of the one before, and of as many behind as one look at a run takes: one round trip
    const int before = slot_of(begin + lane - 1), window[2] = {slot_of(begin + lane), slot_of(begin + 64 + lane)};
    const bool begins = lane < a.chunk && block_of(window[0]) >= 0 && block_of(before) != block_of(window[0]);
    for (uint64_t todo = __ballot(begins); todo; todo &= todo - 1) {
        const int o = __builtin_ctzll(todo), i = first + o, blk = block_of(__builtin_amdgcn_readlane(window[0], o));
        int n = 0;                                     // rows of the run
        int mine_at = 0;                               // slot of its token `lane`
        bool fresh = false;                            // one of them is the block's first
        for (uint64_t same = ~0ull; same == ~0ull; n += same == ~0ull ? 64 : __builtin_ctzll(~same)) {
            int slot;
            if (n == 0) {
                const int lo = __shfl(window[0], (o + lane) & 63, 64), hi = __shfl(window[1], (o + lane) & 63, 64);
                slot = mine_at = o + lane < 64 ? lo : hi;
            } else {
                slot = slot_of((int64_t)i + n + lane);
            }
            const bool mine = (uint32_t)slot < (uint32_t)a.rows && slot >> a.shift == blk;
            same = __ballot(mine);
            const uint64_t run = same == ~0ull ? ~0ull : (1ull << __builtin_ctzll(~same)) - 1;
            fresh |= (__ballot(mine && (slot & ((1 << a.shift) - 1)) == 0) & run) != 0;
        }
        const int64_t at = (int64_t)blk * a.Hkv + h;
        float *scale = (which ? a.scales[1] : a.scales[0]) + at;
        uint8_t *codes = (which ? a.codes[1] : a.codes[0]) + ((at << a.shift) * kD);
        const float old = *scale;
        u4v x[ROWS / 4];
        auto load = [&](int base) {                    // (with the streaming hint: each row is this wave's alone)
#pragma unroll
            for (int k = 0; k < ROWS / 4; ++k)
                if (base + 4 * k < n) x[k] = __builtin_nontemporal_load((const u4v *)(X + (int64_t)(i + min(base + 4 * k + sub, n - 1)) * stride));
        };
        uint32_t mx = 0;
        for (int base = 0; base < n; base += ROWS) {
            load(base);
#pragma unroll
            for (int k = 0; k < ROWS / 4; ++k)
                if (base + 4 * k < n) {
                    const uint32_t lo = max_u16x2(x[k][0] & 0x7fff7fff, x[k][1] & 0x7fff7fff);
                    const uint32_t hi = max_u16x2(x[k][2] & 0x7fff7fff, x[k][3] & 0x7fff7fff);
                    mx = max_u16x2(mx, max_u16x2(lo, hi));
                }
        }
        mx = wave_max_u32(max(mx & 0xffff, mx >> 16));
        float s = scale_for(from16<BF16>(mx));
        if (!fresh) {
            if (old > s) s = old;
            if (s != old) {                            // every row of the block under the new scale
                const float ratio = old / s;           // (s is a power of two)
                auto scaled = [&](float c) { return to_odd(c * ratio, __builtin_fmaf(c, ratio, -(c * ratio))); };
                for (int k = lane; k < (8 << a.shift); k += 64) {
                    uint4 w = ((const uint4 *)codes)[k];
                    uint32_t *p = &w.x;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8(p[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(p[j], true);
                        int v = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(lo[0]), scaled(lo[1]), 0, false);
                        p[j] = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(hi[0]), scaled(hi[1]), v, true);
                    }
                    ((uint4 *)codes)[k] = w;
                }
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // before the new rows go to places among them
            }
        }
        if (__builtin_amdgcn_readfirstlane(__float_as_uint(s)) & 0x7fffff) {         // the block came with a scale that is no power of two (filed ones never have it)
            const float up = s < 1.0f ? 0x1p64f : 1.0f, by = s * up;   // (so that no remainder is subnormal)
            auto over = [&](uint32_t bits) {
                const float v = from16<BF16>(bits) * up, p = v / by;
                return to_odd(p, __builtin_fmaf(-p, by, v));
            };
#pragma unroll 1
            for (int row = sub; row < n; row += 4) {
                const u4v w = *(const u4v *)(X + (int64_t)(i + row) * stride);
                int v[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    v[j] = __builtin_amdgcn_cvt_pk_fp8_f32(over(w[2 * j] & 0xffff), over(w[2 * j] >> 16), 0, false);
                    v[j] = __builtin_amdgcn_cvt_pk_fp8_f32(over(w[2 * j + 1] & 0xffff), over(w[2 * j + 1] >> 16), v[j], true);
                }
                *(int2 *)(codes + (a.slots[i + row] & ((1 << a.shift) - 1)) * kD + c * 8) = int2{v[0], v[1]};
            }
            if (lane == 0) *scale = s;
            continue;
        }
        const float inv = s > 0.0f ? 1.0f / s : 0.0f;
        for (int base = 0; base < n; base += ROWS) {
            if (n > ROWS) load(base);
#pragma unroll
            for (int k = 0; k < ROWS / 4; ++k) {
                const int row = base + 4 * k + sub, at = ROWS == 64 ? __shfl(mine_at, row & 63, 64) : 0;      // (in front of the branch: from all lanes)
                if (base + 4 * k < n && row < n) {
                    int v[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t lo = x[k][2 * j], hi = x[k][2 * j + 1];
                        v[j] = __builtin_amdgcn_cvt_pk_fp8_f32(from16<BF16>(lo & 0xffff) * inv, from16<BF16>(lo >> 16) * inv, 0, false);
                        v[j] = __builtin_amdgcn_cvt_pk_fp8_f32(from16<BF16>(hi & 0xffff) * inv, from16<BF16>(hi >> 16) * inv, v[j], true);
                    }
                    const int off = (ROWS > 64 || base ? a.slots[i + row] : at) & ((1 << a.shift) - 1);
                    *(int2 *)(codes + off * kD + c * 8) = int2{v[0], v[1]};
                }
            }
        }
        if (lane == 0) *scale = s;
    }
}

int launch_quantize_blk(const minikv_blk_shape &s, int32_t n_tok, const void *K, int64_t k_stride, const void *V,
                        int64_t v_stride, const int32_t *slots, const minikv_blk_cache &c, hipStream_t st)
{
    FileArgs a;
    a.X[0] = (const uint16_t *)K, a.X[1] = (const uint16_t *)V, a.stride[0] = k_stride, a.stride[1] = v_stride;
    a.codes[0] = c.K, a.codes[1] = c.V, a.scales[0] = c.Ks, a.scales[1] = c.Vs, a.slots = slots;
    a.n_tok = n_tok, a.Hkv = s.Hkv, a.shift = __builtin_ctz(s.block), a.rows = s.n_blocks * s.block;
    // A wave takes about as many tokens as a run has, a request's share of them or a block's worth: one each in a decoding step,
    // whose runs are single tokens, and few waves without a run of their own for prompts.  Us by the share, 8 KV heads, blocks of 64: 256 prompts of
    // 3 tokens 5.0 with 3 tokens a wave, 6.1 with 6, 37 with 64; 200 of 2 6.3 with 3, 7.0 with one, 53 with 64; 2 of 400 7.3 with 64, 5.6 with 12, 6.6 with
    // 3 (of a batch of 256 places), 9.3 with one; 2 of 8192 20.9 with 64, 40.6 with 16 (of 1024 places), 82 with 2 (of 8192).
    const int64_t heads = 2 * (int64_t)s.Hkv;
    const int run = s.block < 64 ? s.block : 64, share = n_tok / s.R;
    a.chunk = share < 1 ? 1 : share < run ? share : run;
    // (a launch holds less than 2^26 waves: more tokens each where there are that many)
    if (n_tok * heads > 0x7fffffff) return MINIKV_EINVAL;
    const int least = (int)(n_tok * heads >> 25) + 1;
    if (a.chunk < least) a.chunk = least < 64 ? least : 64;
    fast_div_setup((uint32_t)heads, a.heads_magic, a.heads_shift);
    const int64_t waves = ((int64_t)n_tok + a.chunk - 1) / a.chunk * heads;
    const dim3 grid((unsigned)((waves + 3) / 4));
    const bool bf16 = s.dtype == MINIKV_BF16;
    if (s.block <= 64 && bf16) hipLaunchKernelGGL((quantize_blk_kernel<64, true>), grid, dim3(256), 0, st, a);
    else if (s.block <= 64) hipLaunchKernelGGL((quantize_blk_kernel<64, false>), grid, dim3(256), 0, st, a);
    else if (bf16) hipLaunchKernelGGL((quantize_blk_kernel<128, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((quantize_blk_kernel<128, false>), grid, dim3(256), 0, st, a);
    return hipGetLastError() == hipSuccess ? MINIKV_OK : MINIKV_ELAUNCH;
}

}  // namespace minikv
