// Attention of a step's new tokens over a paged cache: any mix of requests with one token and with thousands, in one launch of
// workgroups that share the work (span_attn.h has the rows, the tiles and the arithmetic).  `Cache` says how a workgroup gets at the keys and
// values of a request's pages: page_attn.hip (FP16), qpage_attn.hip (8 bits).
//
// Work.  A request's rows of a KV head (tokens x G) are blocks of 32 to a wave; a block costs its key tiles and a constant for coming
// and going.  Laid end to end, the costs of all blocks are cut into equal shares, one for each of the workgroups that the chip holds at a
// time (the KV heads on their own XCDs), wherever the cuts fall: the middle of a long context, or behind a few short
// ones.  Every workgroup derives the same cuts from the requests' lengths.  A block that is cut leaves partial sums, which the
// last of its workgroups to end adds up.  Long prompts in one go are many long blocks: each is a workgroup of its own (Params::unit).
//
// Wide blocks, of more than 32 rows: the waves have 32 rows each and share the key tiles (Cache::wide_sums).
// Narrow blocks (a token or a few of a request): there is one tile of rows, and memory is what bounds it.  Every wave streams key tiles
// of its own (Cache::narrow_sums); the waves' sums meet in LDS.
#pragma once

#include "span_attn.h"

namespace antkv {

namespace paged {

using namespace span;

constexpr int kNarrow = 32;
constexpr int kTurnNarrow = 1024;                                   // key tiles of a narrow block whose pages are looked up at a time
constexpr int kWindow = 64;                                         // requests that a wave looks at at a time
constexpr int kWindows = kMapRequests / kWindow;
constexpr int kWaves = 2048;                                        // that the chip holds at a time: two to a SIMD

__device__ __forceinline__ Request request_of(const Params& p, int r)
{
    const int64_t a = p.q_start[r], e = p.q_start[r + 1], ctx = p.ctx_len[r];
    const int64_t T = p.T, t0 = a < 0 ? 0 : a < T ? a : T, t1 = e < t0 ? t0 : e < T ? e : T;
    const int64_t have = p.table_cap << p.shift;
    int64_t p0 = ctx - (e > a ? e - a : 0) + (t0 - a);
    if (p0 < -(1 << 30)) p0 = -(1 << 30);
    if (p0 > 0x7fffffffLL - T) p0 = 0x7fffffffLL - T;
    return {(int)t0, (int)(t1 - t0), (int)p0, (int)(ctx < 0 ? 0 : ctx < have ? ctx : have)};
}

// ---- the plan --------------------------------------------------------------------------------------------------------------------

// Costs of a request's blocks, last one (the longest) first: a, a - step, a - 2 step, ..
template <class Cache, int NW>
struct Cost {
    static constexpr int kRows = 32 * NW;                           // of a block
    int blocks, a, step;
    __device__ __forceinline__ Cost(const Params& p, const Request& q)
    {
        const int rows = q.n << p.gs;
        blocks = (rows + kRows - 1) / kRows;
        a = step = 0;
        if (blocks > 0) {
            const int first = (blocks - 1) * (kRows >> p.gs);
            a = (span_of(q.p0 + first, q.p0 + q.n - 1, q.limit, p.window, p.n_sink).n << shift(rows)) + idle(rows);
            // causal: each block sees as many tiles less as it has tokens / 32; not so in a window, or where the table ends early
            if (p.window == 0 && q.p0 >= 0 && q.p0 + q.n <= q.limit) step = kRows / 32 >> p.gs << shift(rows);
        }
    }
    // of a key tile, as a power of two; of coming and going: looking up pages, the first loads, partial sums
    __device__ __forceinline__ static int shift(int rows) { return rows <= kNarrow ? Cache::kShiftNarrow : Cache::kShiftWide; }
    __device__ __forceinline__ static int idle(int rows) { return rows <= kNarrow ? Cache::kIdleNarrow : Cache::kIdleWide; }
    __device__ __forceinline__ int before(int k) const { return k * a - step * (k * (k - 1) / 2); }      // of blocks 0 .. k - 1
    __device__ __forceinline__ int all() const { return before(blocks); }
    __device__ __forceinline__ int block_at(int x) const            // the block in which x lies
    {
        int k;
        if (blocks == 1) k = 0;
        else if (step == 0) k = x / a;
        else {
            const float u = 2.f * a + step;
            k = (int)((u - sqrtf(fmaxf(u * u - 8.f * step * (float)x, 0.f))) / (2.f * step));
            k = k < 0 ? 0 : k < blocks ? k : blocks - 1;
            while (k > 0 && before(k) > x) --k;
            while (k + 1 < blocks && before(k + 1) <= x) ++k;
        }
        return k;
    }
};

__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

// Where a workgroup is in the laid-out blocks: 64 requests at a time, one to a lane.  All other members are the same in every lane.
template <class Cache, int NW>
struct Cursor {
    Request q;                                                      // the lane's request
    int upto;                                                       // and the costs up to its end, from the window's start on
    int window, base;                                               // first request / 64, costs before it
    __device__ __forceinline__ void look(const Params& p)
    {
        const int r = window * kWindow + (threadIdx.x & 63);
        q = r < p.R ? request_of(p, r) : Request{0, 0, 0, 0};
        const Cost<Cache, NW> c(p, q);
        upto = wave_scan(p.unit ? c.blocks : c.all());              // (unit: every block costs 1)
    }
};

// ---- partial sums ----------------------------------------------------------------------------------------------------------------

// 8 bytes, past the caches of the die that wrote them: the workgroup that merges may sit on another
__device__ __forceinline__ float2_t load_part(const float* x)
{
    return __builtin_bit_cast(float2_t, __hip_atomic_load((const unsigned long long*)x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ void store_part(float* x, float a, float b)
{
    __hip_atomic_store((unsigned long long*)x, __builtin_bit_cast(unsigned long long, float2_t{a, b}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The pieces of a block that is cut: shares first .. last.  A share has at most one piece that goes on from the share before (slot
// 2 share) and one that begins a block and does not end it (slot 2 share + 1).
struct Pieces {
    int first, last, start;                                         // start: the share in which the block's cost begins
    __device__ __forceinline__ int64_t slot(const Params& p, int share, int g) const { return (int64_t)(2 * share + (share == start ? 1 : 0)) * p.Hkv + g; }
};

// Each wave waits until its stores are acknowledged, the barrier collects the waves, then one thread arrives: the last arrival reads
// partial sums that have all reached the level its loads read from.  It leaves the word as (tag, 0): a captured launch that is
// replayed over other lengths, and so other numbers of pieces, finds no arrivals.
__device__ __forceinline__ bool last_to_arrive(unsigned long long* word, uint64_t tag, int pieces, int* s_flag)
{
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (threadIdx.x == 0) {
        const bool last = (int)(__hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & kArrivalMask) + 1 == pieces;
        if (last) __hip_atomic_store(word, (unsigned long long)tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *s_flag = last;
    }
    __syncthreads();
    return scalar(*s_flag) != 0;
}

// Weight of sums at reference `from` beside others at `to` >= from.  Never 0, which would make NaN of an infinity that is among the sums: what
// 2^-126 leaves of finite ones, at most 2^61, is nothing beside a weight of 2^8 or more, that of the largest score.
__device__ __forceinline__ float weight(float from, float to) { return fmaxf(fast_exp2(from - to), 1.17549435e-38f); }

// Adds the partial sums of a row of a narrow block: a wave, two channels to a lane.
template <class Cache>
__device__ __forceinline__ void merge_row(const Params& p, const Pieces& pc, int row, int g, int64_t t, int h, int lane)
{
    const int S = pc.last - pc.first + 1;
    auto at = [&](int s) { return pc.slot(p, pc.first + s, g) * p.rows_cap + row; };
    constexpr int kBatch = Cache::kBatch;
    float m = kNegBig, s_max = kMasked, l = 0.f, o0 = 0.f, o1 = 0.f;
    for (int s0 = 0; s0 < S; s0 += 64) {                            // lane: piece s0 + lane
        float2_t x = {kNegBig, 0.f}, y = {kMasked, 0.f};
        if (s0 + lane < S) {
            const float* stat = p.part_stat + 4 * at(s0 + lane);
            x = load_part(stat);
            y = load_part(stat + 2);
        }
        const int most = S - s0 < 64 ? S - s0 : 64;
        float2_t v[kBatch];
        auto fetch = [&](int s1) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j) v[j] = load_part(p.part_out + at(s0 + (s1 + j < most ? s1 + j : most - 1)) * kD + 2 * lane);
        };
        fetch(0);
        s_max = fmaxf(s_max, wave_max(y[0]));
        const float m_new = fmaxf(m, wave_max(x[0])), back = weight(m, m_new), w = weight(x[0], m_new);
        m = m_new;
        l = l * back + wave_sum(x[1] * w);
        o0 *= back;
        o1 *= back;
        for (int s1 = 0; s1 < most; s1 += kBatch) {
            if (s1 > 0) fetch(s1);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const float ws = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), (s1 + j) & 63));
                const bool there = s1 + j < most;                   // (what was read again for pieces that are none may be infinite)
                o0 = fmaf(there ? v[j][0] : 0.f, there ? ws : 0.f, o0);
                o1 = fmaf(there ? v[j][1] : 0.f, there ? ws : 0.f, o1);
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *(half2_t*)(p.out + t * p.os_t + h * p.os_h + 2 * lane) = half2_t{(half_t)(o0 * inv), (half_t)(o1 * inv)};
    if (lane == 0 && p.row_max) {
        p.row_max[h * p.st_h + t] = s_max * p.c1 * (1.f / kLog2e);
        p.row_sum[h * p.st_h + t] = l == 0.f ? 0.f : l * fast_exp2(fmaf(-s_max, p.c1, m));
    }
}

// Wide blocks leave their registers as they are, 64 lanes x 8 bytes at a time: whole lines, which is what goes past the caches well.
__device__ __forceinline__ float* wide_part(const Params& p, int64_t slot, int wave, int i, int lane)
{
    return p.part_out + slot * p.rows_cap * kD + ((wave * 32 + i) * 64 + lane) * 2;
}
__device__ __forceinline__ void store_wide(const Params& p, const Sums& x, int64_t slot, int wave, int lane)
{
#pragma unroll
    for (int i = 0; i < 32; ++i) store_part(wide_part(p, slot, wave, i, lane), x.o[i >> 3][2 * (i & 7)], x.o[i >> 3][2 * (i & 7) + 1]);
    if (lane < 32) {
        float* stat = p.part_stat + 4 * (slot * p.rows_cap + 32 * wave + lane);
        store_part(stat, x.m_ref, x.l);
        store_part(stat + 2, x.s_max, 0.f);
    }
}
__device__ __forceinline__ void merge_wide(const Params& p, Sums& x, const Pieces& pc, int share, int g, int wave, int lane)
{
    Sums all;
    all.clear();
    for (int s = pc.first; s <= pc.last; ++s) {                     // always in the order of the keys
        float2_t u = {x.m_ref, x.l}, v = {x.s_max, 0.f}, o[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = float2_t{x.o[i >> 3][2 * (i & 7)], x.o[i >> 3][2 * (i & 7) + 1]};
        if (s != share) {                                           // (its own are in registers still)
            const int64_t slot = pc.slot(p, s, g);
            const float* stat = p.part_stat + 4 * (slot * p.rows_cap + 32 * wave + (lane & 31));
            u = load_part(stat);
            v = load_part(stat + 2);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = load_part(wide_part(p, slot, wave, i, lane));
        }
        const float m_new = fmaxf(all.m_ref, u[0]), back = weight(all.m_ref, m_new), w = weight(u[0], m_new);
        all.m_ref = m_new;
        all.s_max = fmaxf(all.s_max, v[0]);
        all.l = all.l * back + u[1] * w;
#pragma unroll
        for (int i = 0; i < 32; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) all.o[i >> 3][2 * (i & 7) + e] = fmaf(o[i][e], w, all.o[i >> 3][2 * (i & 7) + e] * back);
    }
    x = all;
}

// ---- the kernel ------------------------------------------------------------------------------------------------------------------

template <class Cache, int NW>
__global__ __launch_bounds__(NW * 64, 2) void page_attn_kernel(const Params p)
{
    constexpr int kThreads = NW * 64, kRows = 32 * NW;
    using At = typename Cache::template Lds<NW>;
    __shared__ __attribute__((aligned(1024))) unsigned char s_all[At::total];
    __shared__ int s_cost[kWindows], s_odd, s_flag;
    __shared__ float s_tokens;
    Note* s_notes = (Note*)(s_all + At::notes);
    float4_t* s_stat = (float4_t*)(s_all + At::stat);
    const int tid = threadIdx.x, lane = tid & 63, wave = scalar(tid >> 6);
    const int share = blockIdx.x / p.Hkv, g = blockIdx.x % p.Hkv;      // (heads fastest: 8 heads, one per XCD)

    // the costs of all requests
    Cursor<Cache, NW> cur;
    cur.window = cur.base = 0;
    const int windows = (p.R + kWindow - 1) / kWindow;
    int total = 0, wide = 0;
    float tokens;                                                   // of all requests: more than the batch has only if they overlap
    if (windows == 1) {
        cur.look(p);
        total = last_lane(cur.upto);
        tokens = wave_sum((float)cur.q.n);
        wide = __any((cur.q.n << p.gs) > kNarrow);
    } else {
        if (tid == 0) {
            s_flag = 0;
            s_tokens = 0.f;
        }
        __syncthreads();
        for (int w = wave; w < windows; w += NW) {
            cur.window = w;
            cur.look(p);
            const int cost = last_lane(cur.upto);
            const float some = wave_sum((float)cur.q.n);
            const bool any = __any((cur.q.n << p.gs) > kNarrow);
            if (lane == 0) {
                s_cost[w] = cost;
                atomicAdd(&s_tokens, some);
                if (any) s_flag = 1;
            }
        }
        __syncthreads();
        wide = s_flag;
        tokens = s_tokens;
        for (int w = 0; w < windows; ++w) total += scalar(s_cost[w]);
    }
    // All of the plan is the same in every lane, and has to be so to the compiler too: values that come out of a shuffle are not, and a
    // loop over pieces on such values would be run under a mask of lanes.
    total = scalar(total);
    wide = scalar(wide);
    if (scalar(tokens > 1.01f * (float)p.T)) return;                // costs that might not fit
    int size = 1, x = share, end = total;                           // the share: costs x .. end - 1 (unit: block x)
    if (!p.unit) {
        size = (total + p.shares - 1) / p.shares;
        const int least = Cache::least(wide, total);                // less is not worth the partial sums
        if (size < least) size = least;
        x = share < p.shares ? share * size : total;
        end = x + size < total ? x + size : total;
    }
    if (x >= end) return;
    if (windows > 1) {                                              // the window of requests in which the share begins
        int w = 0, before = 0;
        for (int c = scalar(s_cost[0]); w + 1 < windows && x >= before + c; c = scalar(s_cost[w])) {
            before += c;
            ++w;
        }
        cur.window = w;
        cur.base = before;
        cur.look(p);
    }

    for (;;) {
        const int tid = own_thread(), lane = tid & 63, wave = scalar(tid >> 6);
        // the request in which x lies, its block, the block's pieces
        while (x >= cur.base + last_lane(cur.upto)) {
            if (cur.window + 1 >= windows) return;
            cur.base += last_lane(cur.upto);
            ++cur.window;
            cur.look(p);
        }
        const int l = __builtin_ctzll(__ballot(x < cur.base + cur.upto));
        Piece pc;
        pc.b = 0;
        pc.g = g;
        pc.r = cur.window * kWindow + l;
        pc.rq = {__builtin_amdgcn_readlane(cur.q.t0, l), __builtin_amdgcn_readlane(cur.q.n, l), __builtin_amdgcn_readlane(cur.q.p0, l), __builtin_amdgcn_readlane(cur.q.limit, l)};
        const Request rq = pc.rq;
        const Cost<Cache, NW> cost(p, rq);
        const int rows = rq.n << p.gs;
        const int begin = cur.base + __builtin_amdgcn_readlane(cur.upto, l) - (p.unit ? cost.blocks : cost.all());      // of the request
        const int k = scalar(p.unit ? x - begin : cost.block_at(x - begin));
        const int c0 = begin + (p.unit ? k : cost.before(k)), len = p.unit ? 1 : cost.a - cost.step * k;              // of the block
        pc.row0 = (cost.blocks - 1 - k) * kRows;
        const bool narrow = rows <= kNarrow;
        const int last_row = (pc.row0 + kRows < rows ? pc.row0 + kRows : rows) - 1;
        const Span span = span_of(rq.p0 + (pc.row0 >> p.gs), rq.p0 + (last_row >> p.gs), rq.limit, p.window, p.n_sink);
        pc.from = 0;
        pc.to = span.n;
        Pieces all = {share, share, share};
        bool some = true;                                           // the piece has tiles, or is the only one
        if (!p.unit) {
            // cost offset -> tile: what lies behind the idle part, cut at every fourth (wide blocks are worked on four at a time)
            const int idle = Cost<Cache, NW>::idle(rows), shift = Cost<Cache, NW>::shift(rows), round = 4;
            auto tile_at = [&](int off) { const int t = (off - idle) >> shift; return t <= 0 ? 0 : off >= len ? span.n : t / round * round < span.n ? t / round * round : span.n; };
            all.start = c0 >= share * size ? share : c0 / size;
            all.last = c0 + len <= (share + 1) * size ? share : (c0 + len - 1) / size;
            all.first = (c0 + idle + (Cache::kFirst << shift) + size - 1) / size - 1;   // the first with so many tiles
            if (all.first < all.start) all.first = all.start;
            if (all.first > all.last) all.first = all.last;
            some = share >= all.first;
            pc.from = share == all.first ? 0 : tile_at(share * size - c0);
            pc.to = share == all.last ? span.n : tile_at((share + 1) * size - c0);
        }
        if (some) {
            const int pieces = all.last - all.first + 1;
            unsigned long long* word = p.done + ((int64_t)all.last * p.Hkv + g) * Cache::kWordApart;
            unsigned long long seen = 0;
            if (pieces > 1 && tid == 0) seen = __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            Sums sums;
            sums.clear();
            // An arrival word that another launch, or anything else, has left is replaced by (tag, 0) by whoever gets there first.
            auto claim = [&]() {
                if (pieces > 1 && tid == 0 && arrivals_are_stale(seen, p.tag, 1u << kArrivalBits))
                    __hip_atomic_compare_exchange_strong(word, &seen, (unsigned long long)p.tag, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            };
            const int64_t slot = all.slot(p, share, g);
            if (narrow) {
                Cache::template narrow_sums<NW>(sums, p, pc, span, s_all + At::tiles, (int*)s_notes);
                claim();
                // the waves' sums meet: rows of 32 x 16 bytes per wave, turned by the row (banks)
                const int n = lane & 31, kh = lane >> 5;
                float4_t* s_sum = (float4_t*)(s_all + At::tiles);
                if (n < rows) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int c4 = 8 * (i >> 2) + 2 * (i & 3) + kh;
                        s_sum[(wave * kNarrow + n) * 32 + ((c4 + n) & 31)] =
                            float4_t{sums.o[i >> 2][4 * (i & 3)], sums.o[i >> 2][4 * (i & 3) + 1], sums.o[i >> 2][4 * (i & 3) + 2], sums.o[i >> 2][4 * (i & 3) + 3]};
                    }
                    if (kh == 0) s_stat[wave * kNarrow + n] = float4_t{sums.m_ref, sums.l, sums.s_max, 0.f};
                }
                __syncthreads();
                for (int u = tid; u < rows * (kD / 2); u += kThreads) {             // two channels to a lane
                    const int row = u >> 6, c2 = u & 63, t = rq.t0 + (row >> p.gs), h = (g << p.gs) + (row & (p.G - 1));
                    float m = kNegBig, s_max = kMasked, sum = 0.f;
                    float4_t st[NW];
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        st[w] = s_stat[w * kNarrow + row];
                        m = fmaxf(m, st[w][0]);
                        s_max = fmaxf(s_max, st[w][2]);
                    }
                    float2_t o = {0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        const float f = weight(st[w][0], m);
                        sum = fmaf(st[w][1], f, sum);
                        const float2_t v = ((const float2_t*)&s_sum[(w * kNarrow + row) * 32 + (((c2 >> 1) + row) & 31)])[c2 & 1];
                        o[0] = fmaf(v[0], f, o[0]);
                        o[1] = fmaf(v[1], f, o[1]);
                    }
                    if (pieces == 1) {
                        const float inv = sum == 0.f ? 0.f : 1.f / sum;
                        *(half2_t*)(p.out + t * p.os_t + h * p.os_h + 2 * c2) = half2_t{(half_t)(o[0] * inv), (half_t)(o[1] * inv)};
                        if (c2 == 0 && p.row_max) {
                            p.row_max[h * p.st_h + t] = s_max * p.c1 * (1.f / kLog2e);
                            p.row_sum[h * p.st_h + t] = sum == 0.f ? 0.f : sum * fast_exp2(fmaf(-s_max, p.c1, m));
                        }
                    } else {
                        const int64_t at = slot * p.rows_cap + row;
                        store_part(p.part_out + at * kD + 2 * c2, o[0], o[1]);
                        if (c2 == 0) {
                            store_part(p.part_stat + 4 * at, m, sum);
                            store_part(p.part_stat + 4 * at + 2, s_max, 0.f);
                        }
                    }
                }
                if (pieces > 1 && last_to_arrive(word, p.tag, pieces, &s_flag))
                    for (int row = wave; row < rows; row += NW) merge_row<Cache>(p, all, row, g, rq.t0 + (row >> p.gs), (g << p.gs) + (row & (p.G - 1)), lane);
            } else {
                Cache::template wide_sums<NW>(sums, p, pc, span, s_all + At::tiles, &s_odd, s_notes);
                claim();
                const int row = pc.row0 + 32 * wave + (lane & 31);
                const bool active = pc.row0 + 32 * wave < rows;
                bool mine = true;
                if (pieces > 1) {
                    if (active) store_wide(p, sums, slot, wave, lane);
                    mine = last_to_arrive(word, p.tag, pieces, &s_flag);
                    if (mine && active) merge_wide(p, sums, all, share, g, wave, lane);
                }
                if (mine && row < rows) write_row(p, sums, 0, rq.t0 + (row >> p.gs), (g << p.gs) + (row & (p.G - 1)), lane >> 5);
            }
            __syncthreads();                                        // LDS is free for the next piece
        }
        x = c0 + len;
        if (p.unit || x >= end) return;
    }
}

// Long chunks: 8 waves read a key tile for 256 rows; fewer tokens: 4 waves, two workgroups to a CU, one works while the other comes or
// goes.  With 8 and 4 waves, FP16 pages, 32 heads on 8: a chunk of 2048 on 32768 keys 998 and 1125 us, 8192 on 32768 3510 and 3645, 8 prompts of 1024 120 and 127,
// 64 of 256 154 and 147, one of 300 on 2000 keys 38 and 35; 4 of 100 on 1000 38 and 32, 64 tokens on 4096 keys 45 and 34, 16 requests with 2048 tokens
// among them (500 for four of them, one for the others) on up to 8192 keys 93 and 83, one token on 4096 14.5 and 13.2.
// The lengths are on the device, so that the host goes by the mean.  One long chunk among many short requests is on the slower side then, 2048 tokens on
// 32768 keys beside 63 single tokens on 2000 each 1129 and 1185, beside 63 requests without a token 1018 and 1104; the same 63 beside 2048 tokens on
// 4096 keys 220 and 192, beside 512 on 8192 183 and 149, 31 on 500 .. 16000 beside 2048 on 2048 275 and 219.
template <class Cache>
inline int waves_of(const Geom& g, int64_t T) { return T * g.G >= (int64_t)g.B * Cache::kRowsOfEight ? 8 : 4; }
// Shares per KV head: the chip's workgroups, or one each.
inline int shares_of(const Geom& g, int nw) { return g.Hkv < kWaves / nw ? kWaves / nw / g.Hkv : 1; }
// A batch has no block of more rows than it has itself.
inline int rows_cap_of(const Geom& g, int64_t T, int nw) { return T * g.G < 32 * nw ? ((int)(T * g.G) + 31) / 32 * 32 : 32 * nw; }

// A workgroup per block, where prompts are long and blocks two to a workgroup at least, so that nothing has to be cut: blocks of a prompt
// that run at the same time are then on about the same keys, which come out of the L2.  In shares and in blocks, FP16 pages, 32 heads on 8: 16384
// tokens 2108 and 2067 us, 8192 on 32768 keys 3618 and 3510, 4 x 4096 616 and 595, 8 x 2048 369 and 350, 4 x 2048 on 2048 .. 16384 834 and 789, but
// 8 x 1024 123 and 132, 1000 x 100 838 and 1201, 4096 tokens on 100 keys each 539 and 1540.  Also where the costs of all blocks might not
// fit an int.
template <class Cache>
inline bool unit_blocks(const Geom& g, int64_t T, int64_t most, int64_t longest)
{
    return (T >= 2048 * (int64_t)g.B && T * g.G / 256 * g.Hkv >= 2 * kWaves / 8) || most > (1LL << 30) / ((longest / 32 + 32) << Cache::kShiftWide);
}

// What either would need: a workspace made for many tokens then does for fewer.
template <class Cache>
inline size_t workspace_bytes(const Geom& g, int64_t T)
{
    size_t most = 0;
    for (int nw = 4; nw <= 8; nw += 4) {
        const size_t pairs = (size_t)shares_of(g, nw) * g.Hkv;
        const size_t n = align_up(pairs * sizeof(unsigned long long) * Cache::kWordApart) + 2 * pairs * rows_cap_of(g, T, nw) * (kD + 4) * sizeof(float);
        most = most < n ? n : most;
    }
    return most;
}

template <class Cache, int NW>
inline hipError_t launch_waves(const Geom& g, Params& p, int64_t T, void* ws, hipStream_t st)
{
    p.shares = shares_of(g, NW);
    p.rows_cap = rows_cap_of(g, T, NW);
    const int64_t pairs = (int64_t)p.shares * g.Hkv;
    p.tag = next_launch_tag();
    p.done = (unsigned long long*)ws;
    p.part_out = (float*)((char*)ws + align_up((size_t)pairs * sizeof(unsigned long long) * Cache::kWordApart));
    p.part_stat = p.part_out + 2 * pairs * p.rows_cap * kD;
    const int64_t most = T * g.G / (32 * NW) + (g.B < T ? g.B : T);         // blocks that there can be
    p.unit = unit_blocks<Cache>(g, T, most, p.table_cap << p.shift);
    hipLaunchKernelGGL((page_attn_kernel<Cache, NW>), dim3((unsigned)((p.unit ? most : p.shares) * g.Hkv)), dim3(NW * 64), 0, st, p);
    return hipGetLastError();
}

template <class Cache>
inline hipError_t launch(const Geom& g, const Pages& pg, const PageAttnArgs& a, void* ws, hipStream_t st)
{
    Params p = {};
    p.q = a.q; p.k = a.k_pages; p.v = a.v_pages; p.out = a.out; p.row_max = a.row_max; p.row_sum = a.row_sum;
    p.qs_t = a.qs_t; p.qs_h = a.qs_h; p.os_t = (int64_t)g.Hq * kD; p.os_h = kD; p.st_h = a.T;
    p.c1 = a.scale * kLog2e; p.Hkv = g.Hkv; p.G = g.G; p.gs = log2_of(g.G); p.window = a.window; p.n_sink = a.n_sink;
    p.q_start = a.q_start; p.ctx_len = a.ctx_len; p.table = a.table; p.table_cap = a.table_cap; p.n_pages = pg.n;
    p.T = (int)a.T; p.R = g.B; p.shift = pg.shift; p.k_scales = a.k_scales; p.v_scales = a.v_scales;
    return waves_of<Cache>(g, a.T) == 8 ? launch_waves<Cache, 8>(g, p, a.T, ws, st) : launch_waves<Cache, 4>(g, p, a.T, ws, st);
}

}  // namespace paged

}  // namespace antkv
