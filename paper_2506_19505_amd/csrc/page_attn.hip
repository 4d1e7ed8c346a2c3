// Attention of new tokens over a paged cache (one token to thousands a request, a ragged batch in one launch), and over a dense
// prompt, both with an optional window: a query at position p sees keys j <= p with j > p - window or j < n_sink.
//
// Rows.  The query rows of a request and KV head are its tokens x the G heads of the group, heads fastest: 32 consecutive rows are
// a wave's tile (32 / G tokens), NW such tiles a block, which one workgroup handles over a range of keys.  So one token of a
// group of four is a tile of four rows (memory is what bounds it), and a long chunk fills 8 x 32 rows per key tile that is read.
//
// Keys.  Tiles of 32 keys go from global memory straight into LDS (16 bytes per lane, no registers), four tiles of K and of V in
// flight or in use, shared by the workgroup's waves.  The page of every 16 keys of the range is looked up once, into LDS.
//   scores   S^T tile (keys on the MFMA row axis, queries on the column axis): lane (n, kh) owns query row n and 16 of the
//            tile's 32 keys, so the running softmax is lane-local; the two half-waves of a row meet only when the
//            reference moves and at the end.
//   output   O^T += V^T P^T: the B operand is the lane's own 16 probabilities (fp16), the A operand comes out of the V tile
//            through ds_read_b64_tr_b16.
// Probabilities are exp2 against a per-row reference kLift below the largest score when it was set: it moves when a score comes
// more than kPMax above it.  Rounded to fp16 they then keep 11 bits down to 2^-22 of the largest one and 2^-32 as a step, so that
// many small weights beside a large one are not lost; their sum is taken before the rounding, in fp32.
//
// Tiles that every row of a wave sees whole go four at a time through a loop that works on three at once (softmax of t, scores of
// t + 1, value product of t - 1).  Tiles that some row sees in part (the diagonal, the window's left edge, the end of the sinks,
// the end of the context, a page that is not one) go one by one: scores are masked, and where the tile's V is not finite the
// value product keeps hidden rows out of the sum (0 x inf) by counting what each query sees of them.
//
// Split.  Few rows over long contexts leave CUs idle: the key tiles of a block are cut into ranges of about the same
// work over all requests (every workgroup derives the plan from the lengths), partial sums meet in a second kernel.
#include "lds_tile.h"

#include <type_traits>

namespace antkv {

namespace {

constexpr int kRing = 4;                                // tiles of K, and of V, in LDS
constexpr int kRingBytes = 2 * kRing * kTileBytes;
constexpr int kChunk = 1024;                            // key tiles whose pages are looked up at a time
constexpr float kPMax = 15.f, kLift = 8.f;
constexpr float kMasked = -INFINITY;                    // a score that takes no part

struct Params {
    const half_t *q, *k, *v;
    half_t* out;
    float *row_max, *row_sum;
    int64_t qs_b, qs_t, qs_h, os_b, os_t, os_h, st_b, st_h;         // strides in elements: q, out, statistics (per token 1)
    float c1;
    int Hkv, G, gs;                                                 // gs = log2 G
    int window, n_sink;
    // dense
    int N, Nq, q_blocks;
    // paged
    const int32_t *q_start, *ctx_len, *table;
    int64_t table_cap, n_pages;
    int T, R, shift, target;                                        // target: key ranges over all requests, per KV head
    int4_t* plan;                                                   // [T]: ranges, rows of the request, its first partial row, the token's first row
    float4_t* part_stat;                                            // [partial rows]: reference, sum, largest score
    float* part_out;                                                // [partial rows][D]
    int64_t part_rows;
};

__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }      // of a value that is the same in every lane
__device__ __forceinline__ float max3f(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

// Key tiles that rows at positions lo .. hi of a context see: tiles 0 .. sink_tiles - 1, then from sink_tiles + gap on.
struct Span {
    int keys;                                                       // positions below this one are seen, at most
    int sink_tiles, gap, n;
    __device__ __forceinline__ int tile(int u) const { return u < sink_tiles ? u : u + gap; }
};
__device__ __forceinline__ Span span_of(int lo, int hi, int limit, int window, int n_sink)
{
    Span s;
    s.keys = hi + 1 < limit ? hi + 1 : limit;
    if (s.keys < 0) s.keys = 0;
    const int end = (int)(((uint32_t)s.keys + 31u) >> 5);
    s.sink_tiles = 0;
    s.gap = 0;
    if (window > 0) {
        int from = lo - window + 1;
        from = from > 0 ? from >> 5 : 0;
        if (from > end) from = end;
        const int sinks = n_sink < s.keys ? n_sink : s.keys;
        s.sink_tiles = (int)(((uint32_t)sinks + 31u) >> 5);
        s.gap = from > s.sink_tiles ? from - s.sink_tiles : 0;
    }
    s.n = end - s.gap;
    return s;
}

// One request: its tokens in the packed batch and where they stand.
struct Request {
    int t0, n, p0, limit;                                           // first token, tokens, position of the first, keys that exist
};
__device__ __forceinline__ Request request_of(const Params& p, int r)
{
    const int64_t a = p.q_start[r], e = p.q_start[r + 1], ctx = p.ctx_len[r];
    const int64_t T = p.T, t0 = a < 0 ? 0 : a < T ? a : T, t1 = e < t0 ? t0 : e < T ? e : T;
    const int64_t have = p.table_cap << p.shift;
    int64_t p0 = ctx - (e > a ? e - a : 0) + (t0 - a);
    if (p0 < -(1 << 30)) p0 = -(1 << 30);
    if (p0 > 0x7fffffffLL - T) p0 = 0x7fffffffLL - T;
    Request q;
    q.t0 = (int)t0;
    q.n = (int)(t1 - t0);
    q.p0 = (int)p0;
    q.limit = (int)(ctx < 0 ? 0 : ctx < have ? ctx : have);
    return q;
}

// What a workgroup works on.
struct Item {
    Request rq;
    int r, block, range, ranges, from, to;                          // key tiles from .. to - 1 of the block's span
    int64_t part;                                                   // first partial row of the request
};

// ranges of a request: about `most` tiles each, at least so many that partial sums stay cheap beside them
template <int NW>
__device__ __forceinline__ int ranges_of(const Request& q, const Span& s, int gs, int most)
{
    const int rows = q.n << gs, wide = rows < 32 * NW ? rows : 32 * NW;
    int least = wide >> 3;
    least = least < 4 ? 4 : least;
    const int len = most > least ? most : least;
    const int n = (s.n + len - 1) / len;
    return n < 1 ? 1 : n;
}

// Work item of this workgroup out of the lengths of all requests; false if there is none.  Every workgroup makes the same plan.
template <int NW>
__device__ bool find_item(const Params& p, int group, Item& it)
{
    constexpr int kT = NW * 64;
    __shared__ int64_t s_sum[2][NW];
    __shared__ int s_item[4];
    __shared__ int64_t s_part;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto look = [&](int r, Request& q, Span& s) {
        q = request_of(p, r);
        const int blocks = ((q.n << p.gs) + 32 * NW - 1) / (32 * NW);
        const int first = blocks > 0 ? (blocks - 1) * (32 * NW >> p.gs) : 0;
        s = span_of(q.p0 + first, q.p0 + q.n - 1, q.limit, p.window, p.n_sink);
        return blocks;
    };
    int64_t work = 0;
    for (int r = tid; r < p.R; r += kT) {
        Request q;
        Span s;
        work += (int64_t)look(r, q, s) * s.n;
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) work += __shfl_xor(work, off, 64);
    if (lane == 0) s_sum[0][wave] = work;
    if (tid == 0) s_item[0] = -1;
    __syncthreads();
    work = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) work += s_sum[0][w];
    const int64_t each = (work + p.target - 1) / p.target;
    const int most = (int)(each < 0x7fffffff ? each : 0x7fffffff);
    __syncthreads();
    int64_t run_g = 0, run_p = 0;
    for (int base = 0; base < p.R; base += kT) {
        const int r = base + tid;
        Request q;
        Span s;
        int64_t groups = 0, part = 0;
        int blocks = 0, ranges = 1;
        if (r < p.R) {
            blocks = look(r, q, s);
            ranges = ranges_of<NW>(q, s, p.gs, most);
            groups = (int64_t)blocks * ranges;
            part = ranges > 1 ? (int64_t)ranges * p.Hkv * (q.n << p.gs) : 0;
        }
        int64_t a = groups, b = part;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int64_t u = __shfl_up(a, off, 64), v = __shfl_up(b, off, 64);
            if (lane >= off) { a += u; b += v; }
        }
        if (lane == 63) { s_sum[0][wave] = a; s_sum[1][wave] = b; }
        __syncthreads();
        int64_t all_g = 0, all_p = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < wave) { a += s_sum[0][w]; b += s_sum[1][w]; }
            all_g += s_sum[0][w];
            all_p += s_sum[1][w];
        }
        const int64_t g0 = run_g + a - groups;
        if (groups > 0 && group >= g0 && group < g0 + groups) {     // one thread of the workgroup
            const int at = (int)(group - g0);
            s_item[0] = r;
            s_item[1] = blocks - 1 - at / ranges;                   // longest first
            s_item[2] = at % ranges;
            s_item[3] = ranges;
            s_part = run_p + b - part;
        }
        run_g += all_g;
        run_p += all_p;
        __syncthreads();
        if (run_g > group) break;                                   // (the same for every thread)
    }
    if (s_item[0] < 0) return false;
    it.r = scalar(s_item[0]);
    it.block = scalar(s_item[1]);
    it.range = scalar(s_item[2]);
    it.ranges = scalar(s_item[3]);
    it.part = (int64_t)(uint32_t)scalar((int)s_part) | (int64_t)scalar((int)(s_part >> 32)) << 32;
    it.rq = request_of(p, it.r);
    it.rq.t0 = scalar(it.rq.t0);
    it.rq.n = scalar(it.rq.n);
    it.rq.p0 = scalar(it.rq.p0);
    it.rq.limit = scalar(it.rq.limit);
    // a batch whose starts are not ascending can ask for more than the workspace holds: its ranges are not cut then
    if (it.ranges > 1 && it.part + (int64_t)it.ranges * p.Hkv * (it.rq.n << p.gs) > p.part_rows) {
        if (it.range > 0) return false;
        it.ranges = 1;
    }
    return true;
}

template <int NW, bool kPaged>                          // waves of a workgroup: 8 or 4
__global__ __launch_bounds__(NW * 64, 2) void span_attn_kernel(const Params p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char s_kv[];    // K ring, V ring; paged: pages of the range
    constexpr int kParts = 8 / NW;                                  // pieces of 1 KB of a tile that a wave moves
    lds_byte* lds = (lds_byte*)s_kv;
    int* s_page = (int*)(s_kv + kRingBytes);                        // [key tiles][2]: place of 16 keys in the pool, -1 if there is none
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);      // scalar, so that per-wave conditions are scalar branches
    const int n = lane & 31, kh = lane >> 5;
    Item it;
    int g, b;
    if (kPaged) {
        g = blockIdx.x % p.Hkv;                                     // heads fastest: 8 heads, one per XCD
        b = 0;
        if (!find_item<NW>(p, blockIdx.x / p.Hkv, it)) return;
    } else {
        const int bgs = gridDim.x / p.q_blocks, bg = blockIdx.x % bgs;
        b = bg / p.Hkv;
        g = bg % p.Hkv;
        it.rq = {0, p.Nq, p.N - p.Nq, p.N};
        it.r = 0;
        it.block = p.q_blocks - 1 - blockIdx.x / bgs;               // longest rows first
        it.range = 0;
        it.ranges = 1;
        it.part = 0;
    }
    const Request rq = it.rq;
    const int rows = rq.n << p.gs, row0 = it.block * 32 * NW;
    const int last_row = (row0 + 32 * NW < rows ? row0 + 32 * NW : rows) - 1;        // of the workgroup
    const Span span = span_of(rq.p0 + (row0 >> p.gs), rq.p0 + (last_row >> p.gs), rq.limit, p.window, p.n_sink);
    {
        // every block of the request is cut at the same tiles, those of its longest
        const int first = ((rows - 1) / (32 * NW)) * (32 * NW >> p.gs);
        const Span longest = span_of(rq.p0 + first, rq.p0 + rq.n - 1, rq.limit, p.window, p.n_sink);
        const int len = (longest.n + it.ranges - 1) / it.ranges;
        it.from = it.range * len < span.n ? it.range * len : span.n;
        it.to = it.range == it.ranges - 1 ? span.n : it.from + len < span.n ? it.from + len : span.n;
    }
    // the wave's rows: positions, and the keys a lane's row sees
    const int w_row = row0 + 32 * wave;
    const bool active = w_row < rows;
    const int w_last = w_row + 31 < rows ? w_row + 31 : rows - 1;
    const int w_lo = rq.p0 + (w_row >> p.gs), w_hi = rq.p0 + (w_last >> p.gs);
    const int row = w_row + n < rows ? w_row + n : rows - 1;        // (rows behind the last repeat it and are not written)
    const int tok = row >> p.gs, h = (g << p.gs) + (row & (p.G - 1));
    const int pos = rq.p0 + tok;
    const int key_hi = pos < rq.limit ? pos : rq.limit - 1;         // visible: j <= key_hi and (j >= key_lo or j < n_sink)
    const int key_lo = p.window > 0 && pos - p.window + 1 > 0 ? pos - p.window + 1 : 0;
    const int w_all = w_lo < rq.limit ? w_lo : rq.limit - 1;        // last key up to which every row sees what its window holds
    // the keys of a tile that the lane's row sees, one bit each, from bit 0 on those of the half-wave: key 8 a + 4 kh + c at 8 a + c
    auto below = [](int x) { return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1u; };      // bits 0 .. x - 1
    auto seen_of = [&](int tile, uint32_t bits) {
        const int at = tile * 32;
        const uint32_t w = below(key_hi + 1 - at) & (~below(key_lo - at) | below(p.n_sink - at));
        return (w & ~((bits & 1 ? 0xffffu : 0u) | (bits & 2 ? 0xffff0000u : 0u))) >> (4 * kh);
    };
    auto bit_of = [](int r) { return 1u << (8 * (r >> 2) + (r & 3)); };                   // of accumulator register r
    auto sees_all = [&](int tile) {                                 // every row of the wave sees every key of the tile
        if (!active || tile * 32 + 31 > w_all) return false;
        return p.window == 0 || tile * 32 > w_hi - p.window || tile * 32 + 31 < p.n_sink;
    };

    // staging: a wave moves kParts x 4 rows of a tile, a lane the chunk that belongs at its place of the 1 KB; rows behind the
    // last key that the workgroup sees repeat it
    const int last_tile = (span.keys - 1) >> 5, last_key = (span.keys - 1) & 31;
    uint32_t soff[kParts], soff_last[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        const int part = wave * kParts + i, r4 = 4 * part, r4l = r4 < (last_key & ~3) ? r4 : last_key & ~3;
        const uint32_t chunk = ((lane & 15) ^ swz(r4 + (lane >> 4))) << 4;
        const int in = lane >> 4, inl = in < last_key - r4l ? in : last_key - r4l;
        soff[i] = ((kPaged ? r4 & 15 : r4) + in) * 256 + chunk;
        soff_last[i] = ((kPaged ? r4l & 15 : r4l) + inl) * 256 + chunk;
    }
    const int half = wave * kParts * 4 >> 4;                        // which 16 keys of a tile this wave moves
    const unsigned char* kbase = (const unsigned char*)(kPaged ? p.k : p.k + (int64_t)(b * p.Hkv + g) * p.N * kD);
    const unsigned char* vbase = (const unsigned char*)(kPaged ? p.v : p.v + (int64_t)(b * p.Hkv + g) * p.N * kD);
    const uint32_t to0 = (uint32_t)(uintptr_t)lds + wave * (kParts * 1024);
    auto stage_at = [&](const unsigned char* base, int64_t off, bool last, uint32_t slot) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) load_to_lds16(base + off, last ? soff_last[i] : soff[i], to0 + slot * kTileBytes + 1024 * i);
    };
    // operand addresses inside a tile: K row n, channels 16 s + 8 kh .. + 7; V transposed: inside a 16-lane block, lane
    // 4 e + c reads key row e of the lane's four, channels 4 c .. 4 c + 3 of 16; blocks 0/1 cover the two channel halves
    // of a 32-channel group, blocks 2/3 the same for the other key half
    uint32_t k_at[8], v_at[4][2];
#pragma unroll
    for (int s = 0; s < 8; ++s) { k_at[s] = tile_at(n, s, kh); pin(k_at[s]); }
    {
        const int e = (lane & 15) >> 2, c = lane & 3, blk = (lane >> 4) & 1;
#pragma unroll
        for (int cg = 0; cg < 4; ++cg)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = 8 * j + 4 * kh + e;
                v_at[cg][j] = kRing * kTileBytes + r * 256 + (((4 * cg + 2 * blk + (c >> 1)) ^ swz(r)) << 4) + 8 * (c & 1);
                pin(v_at[cg][j]);
            }
    }
    half8_t tq[8];
    {
        const half_t* qp = p.q + b * p.qs_b + (int64_t)(rq.t0 + tok) * p.qs_t + h * p.qs_h + 8 * kh;
#pragma unroll
        for (int s = 0; s < 8; ++s) tq[s] = *(const half8_t*)(qp + 16 * s);
#pragma unroll
        for (int s = 0; s < 8; ++s) pin(tq[s]);
    }

    float16_t o[4], sc[2];
    half8_t pr[2][2];
#pragma unroll
    for (int cg = 0; cg < 4; ++cg)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[cg][r] = 0.f;
    float m_ref = kNegBig, s_max = kMasked, l_run = 0.f;            // reference (log2 units), largest raw score, sum
    auto k_op = [&](int s, int slot) { return *(lds_half8*)(lds + k_at[s] + slot * kTileBytes); };
    auto v_op = [&](int i, int slot) {                              // i = 4 * (16-key half) + channel group
        const lds_byte* at = lds + slot * kTileBytes + (i >> 2) * 16 * 256;
        const half4_t a = __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(at + v_at[i & 3][0])));
        const half4_t c = __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(at + v_at[i & 3][1])));
        return half8_t{a[0], a[1], a[2], a[3], c[0], c[1], c[2], c[3]};
    };
    // accumulator register r of a score tile, and k-slot r & 7 of 16-key half r >> 3, is key 8 (r >> 2) + 4 kh + (r & 3)

    for (int ua = it.from; ua < it.to; ua += kChunk) {
        const int m = it.to - ua < kChunk ? it.to - ua : kChunk;    // tiles of this turn; i counts them
        auto tile_of = [&](int i) { return span.tile(ua + (i < m ? i : m - 1)); };
        // A page's place is counted in 16 keys of one head.  bad: two bits a tile (its 16-key halves), tile i at the bottom
        uint32_t bad = 0;
        int page_ahead[2] = {0, 0};                                 // of the tile that the next step asks for
        int pv[2] = {0, 0}, pk = 0;                                 // places of tiles i + 2, i + 3 (V) and i + 4 (K)
        __syncthreads();                                            // the turn before has been read
        if (kPaged) {
            const int32_t* row_of = p.table + (int64_t)it.r * p.table_cap;
            for (int x = tid; x < 2 * m; x += NW * 64) {
                int at = span.tile(ua + (x >> 1)) * 32 + 16 * (x & 1);
                if (at > ((span.keys - 1) & ~15)) at = (span.keys - 1) & ~15;
                const int64_t page = row_of[at >> p.shift];
                s_page[x] = page >= 0 && page < p.n_pages
                                ? (int)(((page * p.Hkv + g) << (p.shift - 4)) + ((at & ((1 << p.shift) - 1)) >> 4)) : -1;
            }
            __syncthreads();
        }
        auto pages_of = [&](int i, int& a, int& c) {
            const int x = i < m ? i : m - 1;
            a = s_page[2 * x];
            c = s_page[2 * x + 1];
        };
        auto offset_of = [&](int i, int place) -> int64_t {
            if (kPaged) return (int64_t)(place > 0 ? place : 0) * (16 * kD * 2);
            return (int64_t)tile_of(i) * kTileBytes;
        };
        auto place_of = [&](int i) { return kPaged ? __builtin_amdgcn_readfirstlane(s_page[2 * (i < m ? i : m - 1) + half]) : 0; };
        for (int i = 0; i < 4; ++i) stage_at(kbase, offset_of(i, place_of(i)), tile_of(i) == last_tile, i);
        for (int i = 0; i < 2; ++i) stage_at(vbase, offset_of(i, place_of(i)), tile_of(i) == last_tile, kRing + i);
        if (kPaged) {
            for (int i = 0; i < 5; ++i) {
                int a, c;
                pages_of(i, a, c);
                bad |= (uint32_t)((a < 0 ? 1 : 0) | (c < 0 ? 2 : 0)) << (2 * i);
            }
            bad = __builtin_amdgcn_readfirstlane(bad);
            pv[0] = place_of(2);
            pv[1] = place_of(3);
            pk = place_of(4);
            pages_of(5, page_ahead[0], page_ahead[1]);
        }
        // the V slot of "tile -1" is multiplied with zero probabilities: it has to be finite
#pragma unroll
        for (int i = 0; i < kParts; ++i) *(uint4_t*)(s_kv + (2 * kRing - 1) * kTileBytes + (i * NW * 64 + tid) * 16) = uint4_t{0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) pr[1][i][j] = (half_t)0.f;
        wait_all_loads();
        __syncthreads();

        // stages for step i and brings the places one tile on
        auto stage_ahead = [&](int i) __attribute__((always_inline)) {
            stage_at(kbase, offset_of(i + 4, pk), tile_of(i + 4) == last_tile, i & 3);
            stage_at(vbase, offset_of(i + 2, pv[0]), tile_of(i + 2) == last_tile, kRing + ((i + 2) & 3));
            if (kPaged) {
                const int a = __builtin_amdgcn_readfirstlane(page_ahead[0]), c = __builtin_amdgcn_readfirstlane(page_ahead[1]);
                pv[0] = pv[1];
                pv[1] = pk;
                pk = half ? c : a;
                bad = bad >> 2 | (uint32_t)((a < 0 ? 1 : 0) | (c < 0 ? 2 : 0)) << 8;          // now of tiles i + 1 .. i + 5
                pages_of(i + 6, page_ahead[0], page_ahead[1]);
            }
        };
        auto scores = [&](float16_t& s, int slot) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(k_op(j, slot), tq[j], s, 0, 0, 0);
        };
        // largest score and reference before the exponentials of a tile; true if it moves (o has to be rescaled by alpha)
        auto open_tile = [&](float16_t& s, float& alpha) __attribute__((always_inline)) {
            s_max = max3f(s_max, s[0], s[1]);
#pragma unroll
            for (int r = 2; r < 16; r += 2) s_max = max3f(s_max, s[r], s[r + 1]);
            alpha = 1.f;
            const bool moves = __any(fmaf(s_max, p.c1, -m_ref) > kPMax);
            if (__builtin_expect(moves, 0)) {                       // the reference moves to the largest score so far
                const float m_new = fmaf(fmaxf(s_max, __shfl_xor(s_max, 32, 64)), p.c1, -kLift);
                if (m_new + kLift - m_ref > kPMax) {
                    alpha = fast_exp2(m_ref - m_new);
                    l_run *= alpha;
                    m_ref = m_new;
                }
            }
            return moves;
        };
        auto rescale = [&](float alpha) __attribute__((always_inline)) {
#pragma unroll
            for (int cg = 0; cg < 4; ++cg)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[cg][r] *= alpha;
        };
        // value product of a tile whose probabilities are pr[1].  edge: some key of it is hidden from some row (seen: the lane's word), and
        // counts as nothing for that row whatever its V holds: V that is not finite is left out, and comes back as inf, -inf or
        // NaN where a row sees it
        auto product = [&](int slot, bool edge, uint32_t seen) __attribute__((always_inline)) {
            uint32_t odd = 0;
            if (edge) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint4_t x = __builtin_bit_cast(uint4_t, v_op(i, slot));
#pragma unroll
                    for (int j = 0; j < 4; ++j) odd |= ((x[j] & 0x7c007c00u) + 0x04000400u) & 0x80008000u;
                }
            }
            if (__builtin_expect(__any(odd != 0), 0)) {
#pragma unroll
                for (int cg = 0; cg < 4; ++cg) {
                    float16_t c;
#pragma unroll
                    for (int r = 0; r < 16; ++r) c[r] = 0.f;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint4_t x = __builtin_bit_cast(uint4_t, v_op(4 * i + cg, slot)), kind, sees;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {               // two values at a time; 1: inf, 64: -inf, 4096: NaN (sums of 32 keep apart)
                            uint32_t all = 0, ones = 0;
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const uint32_t y = x[j] >> (16 * e) & 0xffffu;
                                const uint32_t of = (y & 0x7fffu) < 0x7c00u ? 0u : (y & 0x7fffu) > 0x7c00u ? 0x6c00u : y >> 15 ? 0x5400u : 0x3c00u;
                                all |= of << (16 * e);
                                if (seen & bit_of(8 * i + 2 * j + e)) ones |= 0x3c00u << (16 * e);
                                if (of) x[j] &= e ? 0x0000ffffu : 0xffff0000u;
                            }
                            kind[j] = all;
                            sees[j] = ones;
                        }
                        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, kind), __builtin_bit_cast(half8_t, sees), c, 0, 0, 0);
                        o[cg] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, x), pr[1][i], o[cg], 0, 0, 0);
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int count = (int)c[r];
                        o[cg][r] += (count & 63 ? INFINITY : 0.f) - (count >> 6 & 63 ? INFINITY : 0.f) + (count >> 12 ? NAN : 0.f);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v_op(i, slot), pr[1][i >> 2], o[i & 3], 0, 0, 0);
            }
        };

        bool was_edge = false;                                      // some row does not see some key of tile i - 1
        uint32_t seen = 0;                                          // its keys that the lane's row sees, where that is so
        if (active) scores(sc[0], 0);
        __syncthreads();                                            // step 0 stages over the tile that has just been read
        int i = 0;
        if (!active)                                                // a wave without rows stages for the others
            for (; i < m; ++i) {
                stage_ahead(i);
                landed_but<4 * kParts>();
            }
#pragma unroll 1
        for (; i < m; ++i) {
            const int tile = tile_of(i);
            const uint32_t bits = bad & 3;
            stage_ahead(i);
            product((i + 3) & 3, was_edge, seen);
            was_edge = bits != 0 || !sees_all(tile);
            if (was_edge) {
                seen = seen_of(tile, bits);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(seen & bit_of(r))) sc[0][r] = kMasked;
            }
            float alpha;
            if (open_tile(sc[0], alpha)) rescale(alpha);
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float e = fast_exp2(fmaf(sc[0][r], p.c1, -m_ref));
                sum[r & 1] += e;
                pr[1][r >> 3][r & 7] = (half_t)e;
            }
            l_run += sum[0] + sum[1];
            scores(sc[0], (i + 1) & 3);
            __builtin_amdgcn_sched_barrier(0);                      // (K and V have been read before another wave stages over them)
            landed_but<4 * kParts>();
        }
        if (active) product((m + 3) & 3, was_edge, seen);
        wait_all_loads();                                           // nothing may land in LDS after the turn, or the workgroup's end
    }

    const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
    s_max = fmaxf(s_max, __shfl_xor(s_max, 32, 64));
    if (it.ranges > 1) {
        if (active && w_row + n < rows) {
            const int64_t at = it.part + ((int64_t)it.range * p.Hkv + g) * rows + row;
            float* op = p.part_out + at * kD + 4 * kh;
            if (l_tot != 0.f)                                       // (also where it is NaN)
#pragma unroll
                for (int cg = 0; cg < 4; ++cg)
#pragma unroll
                    for (int qd = 0; qd < 4; ++qd)
                        *(float4_t*)(op + 32 * cg + 8 * qd) = float4_t{o[cg][4 * qd], o[cg][4 * qd + 1], o[cg][4 * qd + 2], o[cg][4 * qd + 3]};
            if (kh == 0) p.part_stat[at] = float4_t{m_ref, l_tot, s_max, 0.f};
        }
    } else if (active && w_row + n < rows) {
        const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;         // a row that sees nothing is zero
        half_t* op = p.out + b * p.os_b + (int64_t)(rq.t0 + tok) * p.os_t + h * p.os_h + 4 * kh;
#pragma unroll
        for (int cg = 0; cg < 4; ++cg)
#pragma unroll
            for (int qd = 0; qd < 4; ++qd) {                        // accumulator rows 8 qd + 4 kh + e = channels of group cg
                half4_t w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = (half_t)(o[cg][4 * qd + e] * inv);
                *(half4_t*)(op + 32 * cg + 8 * qd) = w;
            }
        if (kh == 0 && p.row_max) {
            const int64_t at = b * p.st_b + h * p.st_h + rq.t0 + tok;
            p.row_max[at] = s_max * p.c1 * (1.f / kLog2e);
            p.row_sum[at] = l_tot == 0.f ? 0.f : l_tot * fast_exp2(fmaf(-s_max, p.c1, m_ref));
        }
    }
    if (kPaged && g == 0 && it.range == 0)                          // for the second kernel
        for (int x = (row0 >> p.gs) + tid; x <= last_row >> p.gs; x += NW * 64)
            p.plan[rq.t0 + x] = int4_t{it.ranges, rows, (int)(it.part & 0x7fffffff), x << p.gs};
}

// Adds the partial sums of a row: a wave per row, two channels to a lane.
constexpr int kMergeThreads = 256;

__global__ __launch_bounds__(kMergeThreads) void merge_kernel(const Params p, int n_rows)
{
    const int lane = threadIdx.x & 63, Hq = p.Hkv << p.gs;
    const int at = blockIdx.x * (kMergeThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (at >= n_rows) return;
    const int t = at / Hq, h = at - t * Hq, g = h >> p.gs;
    const int4_t plan = p.plan[t];
    if (t < p.q_start[0] || t >= p.q_start[p.R]) return;            // a token that no request has
    const int S = plan[0], rows = plan[1], row = plan[3] + (h & (p.G - 1));
    const int64_t first = plan[2], stride = (int64_t)p.Hkv * rows;
    if (S < 2 || S > p.part_rows || rows < 1 || row < 0 || row >= rows || first + S * stride > p.part_rows) return;
    const float4_t* stat = p.part_stat + first + (int64_t)g * rows + row;
    const float* part = p.part_out + (first + (int64_t)g * rows + row) * kD + 2 * lane;
    float m = kNegBig, s_max = kMasked;
    for (int s = lane; s < S; s += 64) {
        const float4_t x = stat[s * stride];
        if (x[1] != 0.f) m = fmaxf(m, x[0]);
        s_max = fmaxf(s_max, x[2]);
    }
    m = wave_max(m);
    s_max = wave_max(s_max);
    float l = 0.f, o0 = 0.f, o1 = 0.f;
    for (int s0 = 0; s0 < S; s0 += 64) {
        float w = 0.f;
        if (s0 + lane < S) {
            const float4_t x = stat[(s0 + lane) * stride];
            if (x[1] != 0.f) {
                w = fast_exp2(x[0] - m);
                l += x[1] * w;
            }
        }
        const int most = S - s0 < 64 ? S - s0 : 64;
        for (int s1 = 0; s1 < most; s1 += 8) {
            float a[8], c[8];
            float ws[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                ws[j] = s1 + j < most ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), (s1 + j) & 63)) : 0.f;
                a[j] = c[j] = 0.f;
                if (ws[j] != 0.f) {                                 // (a range that nothing is seen of has written no sums)
                    const float* x = part + (s0 + s1 + j) * stride * kD;
                    a[j] = x[0];
                    c[j] = x[1];
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) { o0 = fmaf(a[j], ws[j], o0); o1 = fmaf(c[j], ws[j], o1); }
        }
    }
    l = wave_sum(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    half_t* op = p.out + (int64_t)t * p.os_t + h * p.os_h + 2 * lane;
    *(half2_t*)op = half2_t{(half_t)(o0 * inv), (half_t)(o1 * inv)};
    if (lane == 0 && p.row_max) {
        p.row_max[h * p.st_h + t] = s_max * p.c1 * (1.f / kLog2e);
        p.row_sum[h * p.st_h + t] = l == 0.f ? 0.f : l * fast_exp2(fmaf(-s_max, p.c1, m));
    }
}

template <int NW, bool kPaged>
hipError_t launch_t(const Params& p, int64_t grid, hipStream_t st)
{
    constexpr size_t lds = kRingBytes + (kPaged ? 2 * kChunk * sizeof(int) : 0);
    static OncePerDevice once;
    const hipError_t e = allow_lds(once, (const void*)span_attn_kernel<NW, kPaged>, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((span_attn_kernel<NW, kPaged>), dim3((unsigned)grid), dim3(NW * 64), lds, st, p);
    return hipGetLastError();
}

int log2_of(int G) { return G == 4 ? 2 : G == 2 ? 1 : 0; }

}  // namespace

// Key ranges, per KV head, that the plan aims at.
static int64_t target_of(const Geom& g)
{
    const int64_t t = (512 + g.Hkv - 1) / g.Hkv;
    return t < 1 ? 1 : t;
}

// Rows of partial sums: a request with S > 1 ranges has S <= 2 tiles / each of them, and `each` is work / target or more, so that
// all S x rows of one KV head come to twice target x the rows of a block at most, and a batch has no block of more rows than it has itself.
static int64_t part_rows_of(const Geom& g, int64_t T)
{
    const int64_t wide = T * g.G < 256 ? T * g.G : 256;
    return 2 * target_of(g) * wide * g.Hkv + 2 * g.Hkv * wide;
}

size_t page_attn_workspace_bytes(const Geom& g, int64_t T)
{
    return align_up((size_t)T * sizeof(int4_t)) + (size_t)part_rows_of(g, T) * (sizeof(float4_t) + kD * sizeof(float));
}

hipError_t launch_page_attn(const Geom& g, const Pages& pg, const PageAttnArgs& a, void* ws, hipStream_t st)
{
    Params p = {};
    p.q = a.q; p.k = a.k_pages; p.v = a.v_pages; p.out = a.out; p.row_max = a.row_max; p.row_sum = a.row_sum;
    p.qs_t = a.qs_t; p.qs_h = a.qs_h; p.os_t = (int64_t)g.Hq * kD; p.os_h = kD; p.st_h = a.T;
    p.c1 = a.scale * kLog2e; p.Hkv = g.Hkv; p.G = g.G; p.gs = log2_of(g.G); p.window = a.window; p.n_sink = a.n_sink;
    p.q_start = a.q_start; p.ctx_len = a.ctx_len; p.table = a.table; p.table_cap = a.table_cap; p.n_pages = pg.n;
    p.T = (int)a.T; p.R = g.B; p.shift = pg.shift; p.target = (int)target_of(g);
    p.part_rows = part_rows_of(g, a.T);
    p.plan = (int4_t*)ws;
    p.part_stat = (float4_t*)((char*)ws + align_up((size_t)a.T * sizeof(int4_t)));
    p.part_out = (float*)(p.part_stat + p.part_rows);
    const int64_t rows = a.T * g.G, some = g.B < a.T ? g.B : a.T;
    auto grid = [&](int nw) { return (p.target + rows / (32 * nw) + some + 1) * g.Hkv; };
    const bool wide = rows * g.Hkv >= 256 * 64;
    const hipError_t e = wide ? launch_t<8, true>(p, grid(8), st) : launch_t<4, true>(p, grid(4), st);
    if (e != hipSuccess) return e;
    const int64_t n = a.T * g.Hq;
    hipLaunchKernelGGL(merge_kernel, dim3((unsigned)((n + kMergeThreads / 64 - 1) / (kMergeThreads / 64))), dim3(kMergeThreads), 0, st, p, (int)n);
    return hipGetLastError();
}

hipError_t launch_prefill_attn_window(const Geom& g, const half_t* q, const half_t* k, const half_t* v, int64_t N, int64_t Nq, float scale,
                                      int window, int n_sink, half_t* out, float* row_max, float* row_sum, hipStream_t st)
{
    Params p = {};
    p.q = q; p.k = k; p.v = v; p.out = out; p.row_max = row_max; p.row_sum = row_sum;
    p.qs_t = p.os_t = kD; p.qs_h = p.os_h = Nq * kD; p.qs_b = p.os_b = g.Hq * Nq * kD; p.st_h = Nq; p.st_b = g.Hq * Nq;
    p.c1 = scale * kLog2e; p.Hkv = g.Hkv; p.G = g.G; p.gs = log2_of(g.G); p.window = window; p.n_sink = n_sink;
    p.N = (int)N; p.Nq = (int)Nq;
    const int64_t pairs = (int64_t)g.B * g.Hkv, rows = Nq * g.G;
    const bool wide = (rows + 255) / 256 * pairs >= 384;
    const int span = wide ? 256 : 128;
    p.q_blocks = (int)((rows + span - 1) / span);
    return wide ? launch_t<8, false>(p, p.q_blocks * pairs, st) : launch_t<4, false>(p, p.q_blocks * pairs, st);
}

}  // namespace antkv
