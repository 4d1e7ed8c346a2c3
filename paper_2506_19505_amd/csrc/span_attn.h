// Attention of query rows over a span of keys, by one workgroup: what the paged and the windowed kernel share.
//
// A query at position p sees keys j <= p, with a window only those with j > p - window or j < n_sink.
//
// Rows.  The query rows of a sequence and KV head are its tokens x the G heads of the group, heads fastest: 32 consecutive rows are a
// wave's tile (32 / G tokens), NW such tiles a block.
//
// Keys.  Tiles of 32 keys go from global memory straight into LDS (16 bytes per lane, no registers), shared by the workgroup's waves, four
// tiles of K and of V in flight or in use.
//   scores   S^T tile (keys on the MFMA row axis, queries on the column axis): lane (n, kh) owns query row n and 16 of the
//            tile's 32 keys, so the running softmax is lane-local; the two half-waves of a row meet only when the
//            reference moves and at the end.
//   output   O^T += V^T P^T: the B operand is the lane's own 16 probabilities (fp16), the A operand comes out of the V tile
//            through ds_read_b64_tr_b16.
// Probabilities are exp2 against a per-row reference kLift below the largest score when it was set: it moves when a score comes
// more than kPMax above it.  Rounded to fp16 they then keep 11 bits down to 2^-22 of the largest one and 2^-32 as a step, so that
// many small weights beside a large one are not lost; their sum is taken before the rounding, in fp32.  The reference itself is rounded to fp32:
// at scores of 2^27 log2 units to multiples of 16, which may lie 8 too low, and fp16 ends at 2^16.
//
// One step of the loop works on three tiles at once: the softmax of tile t (VALU) is interleaved with the scores of tile t + 1 and the
// value product of tile t - 1 (16 MFMAs), none of which waits for it.  Tiles that some row sees in part (the diagonal, the window's
// left edge, the end of the sinks or of the context, a page that is none) are masked, and their V is looked at: what is not finite
// must not reach the product of a row that does not see it (0 x inf).
//
// Values that are not finite.  A row that sees one has it in its result, whatever the weight; but a weight below 2^-25 is 0 in
// fp16, one far enough below the largest 0 in fp32 too, and 0 x inf is NaN.  Tiles that all rows see are not looked at: their infinities leave
// some sum that is not finite (none turns finite again), which is looked for once at the end.  Then, or where the tiles that were looked at held
// some, V is gone through a second time, and the rows get inf, -inf or NaN by counting (add_odd): the result does not depend on where tiles begin.
#pragma once

#include "lds_tile.h"

namespace antkv {

namespace span {

constexpr int kRing = 4;                                // tiles of K, and of V, in LDS
constexpr int kRingBytes = 2 * kRing * kTileBytes;
constexpr int kTurn = 512;                              // key tiles that are looked up at a time
constexpr int kNotes = kTurn + 8;                       // and what lies behind them: see Note
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
    int T, R, shift;
    int shares, rows_cap;                                           // shares of the work per KV head; rows of a piece's partial sums
    int unit;                                                       // a workgroup per block instead of per share
    unsigned long long* done;                                       // [shares][Hkv] arrival words (launch_tag.h) of the blocks that end there
    uint64_t tag;
    float *part_out, *part_stat;                                    // [2 shares][Hkv][rows_cap] x D sums, x 4: reference, sum, largest score
};

__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }      // of a value that is the same in every lane
// threadIdx.x, not known to be the same from one piece to the next: what a piece makes of it stays in the piece, where the compiler would
// take it out of the loop over pieces and, all at once being too much, put it on the stack
__device__ __forceinline__ int own_thread()
{
    int t = threadIdx.x;
    pin(t);
    return t;
}
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

// One sequence: its tokens in the batch and where they stand.
struct Request {
    int t0, n, p0, limit;                                           // first token, tokens, position of the first, keys that exist
};

// What a workgroup works on: a block of rows and a range of its key tiles.
struct Piece {
    Request rq;
    int b, r, g;                                                    // sequence (dense) or request (paged), KV head
    int row0;                                                       // first row of the block
    int from, to;                                                   // key tiles of the block's span
};

// The sums of a lane's row over a range of keys: register [cg][4 qd + e] is channel 32 cg + 8 qd + 4 kh + e.
struct Sums {
    float16_t o[4];
    float m_ref, s_max, l;                                          // reference (log2 units), largest raw score, sum of the half-wave's keys

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int cg = 0; cg < 4; ++cg)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[cg][r] = 0.f;
        m_ref = kNegBig;
        s_max = kMasked;
        l = 0.f;
    }
    // Largest score and reference before the exponentials of a tile's scores; true if the reference moves (o has to be rescaled by alpha).
    __device__ __forceinline__ bool open(const float16_t& s, float c1, float& alpha)
    {
        s_max = max3f(s_max, s[0], s[1]);
#pragma unroll
        for (int r = 2; r < 16; r += 2) s_max = max3f(s_max, s[r], s[r + 1]);
        alpha = 1.f;
        const bool moves = __any(fmaf(s_max, c1, -m_ref) > kPMax);
        if (__builtin_expect(moves, 0)) {                           // the reference moves to the largest score so far
            const float m_new = fmaf(fmaxf(s_max, __shfl_xor(s_max, 32, 64)), c1, -kLift);
            if (m_new + kLift - m_ref > kPMax) {
                alpha = fast_exp2(m_ref - m_new);
                l *= alpha;
                m_ref = m_new;
            }
        }
        return moves;
    }
    __device__ __forceinline__ void rescale(float alpha)
    {
#pragma unroll
        for (int cg = 0; cg < 4; ++cg)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[cg][r] *= alpha;
    }
    // the two half-waves of the row
    __device__ __forceinline__ void join_halves()
    {
        l += __shfl_xor(l, 32, 64);
        s_max = fmaxf(s_max, __shfl_xor(s_max, 32, 64));
    }
    // Some sum is not finite although the row's weights are numbers (halves joined): a value that the row sees is not.  Sums of finite
    // values are at most 2^15 x 2^16 x 2^30.
    __device__ __forceinline__ bool odd() const
    {
        float t = 0.f;
#pragma unroll
        for (int cg = 0; cg < 4; ++cg)
#pragma unroll
            for (int r = 0; r < 16; ++r) t = fmaf(o[cg][r], 0.f, t);
        return t != t && l == l;
    }
    __device__ __forceinline__ void drop_odd()
    {
#pragma unroll
        for (int cg = 0; cg < 4; ++cg)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[cg][r] = l == l && !(fabsf(o[cg][r]) < INFINITY) ? 0.f : o[cg][r];
    }
};

// What rows see.
struct Sight {
    int key_lo, key_hi, n_sink, window;                             // the lane's row: j <= key_hi and (j >= key_lo or j < n_sink)

    __device__ __forceinline__ Sight(const Params& p, int pos, int limit)
        : key_lo(p.window > 0 && pos - p.window + 1 > 0 ? pos - p.window + 1 : 0), key_hi(pos < limit ? pos : limit - 1), n_sink(p.n_sink), window(p.window)
    {
    }
    __device__ __forceinline__ static uint32_t below(int x) { return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1u; }      // bits 0 .. x - 1
    // The keys of a tile that the lane's row sees, one bit each, those of half-wave kh from bit 0 on: key 8 a + 4 kh + c at 8 a + c.
    // bad: 16-key halves of the tile that lie on no page
    __device__ __forceinline__ uint32_t of_tile(int tile, uint32_t bad, int kh) const
    {
        const int at = tile * 32;
        const uint32_t w = below(key_hi + 1 - at) & (~below(key_lo - at) | below(n_sink - at));
        return (w & ~((bad & 1 ? 0xffffu : 0u) | (bad & 2 ? 0xffff0000u : 0u))) >> (4 * kh);
    }
    // every one of a range of rows sees the whole tile: `all` is the last key that the first row sees, `hi` the last row's position
    __device__ __forceinline__ bool whole(int tile, int all, int hi) const
    {
        return tile * 32 + 31 <= all && (window == 0 || tile * 32 > hi - window || tile * 32 + 31 < n_sink);
    }
};
// bit, in such a word, of accumulator register r of a score tile: that of key 8 (r >> 2) + 4 kh + (r & 3), which also is k-slot r & 7 of 16-key half r >> 3
__device__ __forceinline__ constexpr uint32_t bit_of(int r) { return 1u << (8 * (r >> 2) + (r & 3)); }

__device__ __forceinline__ void mask(float16_t& s, uint32_t seen)
{
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if (!(seen & bit_of(r))) s[r] = kMasked;
}

// Operand addresses inside a tile at LDS address `at`: K row n, channels 16 s + 8 kh .. + 7; V transposed: inside a 16-lane block, lane
// 4 e + c reads key row e of the lane's four, channels 4 c .. 4 c + 3 of 16; blocks 0/1 cover the two channel halves
// of a 32-channel group, blocks 2/3 the same for the other key half
struct Operands {
    uint32_t k[8], v[4][2];

    __device__ __forceinline__ Operands(uint32_t k_at, uint32_t v_at, int lane)
    {
        const int n = lane & 31, kh = lane >> 5, e = (lane & 15) >> 2, c = lane & 3, blk = (lane >> 4) & 1;
#pragma unroll
        for (int s = 0; s < 8; ++s) { k[s] = k_at + tile_at(n, s, kh); pin(k[s]); }
#pragma unroll
        for (int cg = 0; cg < 4; ++cg)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = 8 * j + 4 * kh + e;
                v[cg][j] = v_at + r * 256 + (((4 * cg + 2 * blk + (c >> 1)) ^ swz(r)) << 4) + 8 * (c & 1);
                pin(v[cg][j]);
            }
    }
    __device__ __forceinline__ half8_t k_op(int s, int slot) const { return *(lds_half8*)(uintptr_t)(k[s] + slot * kTileBytes); }
    __device__ __forceinline__ half8_t v_op(int i, int slot) const                      // i = 4 * (16-key half) + channel group
    {
        const uint32_t at = slot * kTileBytes + (i >> 2) * 16 * 256;
        const half4_t a = __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(uintptr_t)(v[i & 3][0] + at)));
        const half4_t b = __builtin_bit_cast(half4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(uintptr_t)(v[i & 3][1] + at)));
        return half8_t{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
};

// Two fp16 values of V: which of them are not finite (their sign bits set), and the two without those.
__device__ __forceinline__ uint32_t not_finite(uint32_t two) { return ((two & 0x7c007c00u) + 0x04000400u) & 0x80008000u; }
__device__ __forceinline__ uint32_t without(uint32_t two, uint32_t odd) { return two & ~((odd & 0x8000u ? 0xffffu : 0u) | (odd & 0x80000000u ? 0xffff0000u : 0u)); }

// Values of a V tile that are not finite, as inf, -inf or NaN to the rows that see them: each row's number of them per channel is a
// matrix product of its own, in which fp16 1 stands for inf, 64 for -inf and 4096 for NaN (sums of 32 keep apart).
__device__ __forceinline__ void add_odd(Sums& x, const Operands& at, int slot, uint32_t seen)
{
#pragma unroll
    for (int cg = 0; cg < 4; ++cg) {
        float16_t n_odd;
#pragma unroll
        for (int r = 0; r < 16; ++r) n_odd[r] = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint4_t two = __builtin_bit_cast(uint4_t, at.v_op(4 * k + cg, slot));
            uint4_t kind, sees;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                kind[j] = sees[j] = 0;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t y = two[j] >> (16 * e) & 0xffffu;
                    const uint32_t of = (y & 0x7fffu) < 0x7c00u ? 0u : (y & 0x7fffu) > 0x7c00u ? 0x6c00u : y >> 15 ? 0x5400u : 0x3c00u;
                    kind[j] |= of << (16 * e);
                    if (seen & bit_of(8 * k + 2 * j + e)) sees[j] |= 0x3c00u << (16 * e);
                }
            }
            n_odd = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, kind), __builtin_bit_cast(half8_t, sees), n_odd, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int count = (int)n_odd[r];
            x.o[cg][r] += (count & 63 ? INFINITY : 0.f) - (count >> 6 & 63 ? INFINITY : 0.f) + (count >> 12 ? NAN : 0.f);
        }
        pin(x.o[cg]);                                               // (one channel group after the other: registers)
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The query row of each lane (row n of the tile that starts at row w_row; rows behind the last repeat it)
__device__ __forceinline__ void load_query(half8_t (&tq)[8], const Params& p, const Piece& x, int row, int lane)
{
    const int tok = row >> p.gs, h = (x.g << p.gs) + (row & (p.G - 1));
    const half_t* qp = p.q + x.b * p.qs_b + (int64_t)(x.rq.t0 + tok) * p.qs_t + h * p.qs_h + 8 * (lane >> 5);
#pragma unroll
    for (int s = 0; s < 8; ++s) tq[s] = *(const half8_t*)(qp + 16 * s);
#pragma unroll
    for (int s = 0; s < 8; ++s) pin(tq[s]);
}

// What the loop has to know of a key tile, looked up for a whole turn at once.  Behind the turn's last tile follow copies of it
// that nobody sees: the loop works on four tiles at a time and asks for the next ones ahead.
struct Note {
    int place[2];                                                   // of its 16-key halves, in 16 keys of a head, x 4; bits 0: the context's last tile, 1: no page
    int edge;                                                       // bit w: some row of wave w does not see some key, kEdgeAny: some row of the workgroup, kHidden: nobody sees any
    int unused;
};
constexpr int kLast = 1, kBad = 2, kEdgeAny = 1 << 8, kHidden = 1 << 9;

// Place in the pools, counted in 16 keys of a head, of the 16 keys of a request from position `at` on; -1 if they lie on no page
__device__ __forceinline__ int place_of(const Params& p, const int32_t* row_of, int g, int at)
{
    const int64_t page = row_of[at >> p.shift];
    return page >= 0 && page < p.n_pages ? (int)(((page * p.Hkv + g) << (p.shift - 4)) + ((at & ((1 << p.shift) - 1)) >> 4)) : -1;
}

// Sums of the piece's rows, 32 to a wave, over its key tiles.  s_kv: kRingBytes of LDS; s_odd: a word; notes: kNotes of them.
// Every wave of the workgroup takes part; its LDS is free again when all have come back and met at a barrier.
template <int NW, bool kPaged>
__device__ __forceinline__ void wide_sums(Sums& sums, const Params& p, const Piece& x, const Span& span, unsigned char* s_kv, int* s_odd, Note* notes)
{
    constexpr int kParts = 8 / NW;                                  // pieces of 1 KB of a tile that a wave moves
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)s_kv;
    const int tid = own_thread(), lane = tid & 63, n = lane & 31, kh = lane >> 5;
    const int wave = scalar(tid >> 6);                              // so that per-wave conditions are scalar branches
    const Request rq = x.rq;
    const int rows = rq.n << p.gs;
    // first and last row of wave w, or of the workgroup: the last key that the first sees, the last one's position
    auto sees_to = [&](int row) { const int pos = rq.p0 + (row >> p.gs); return pos < rq.limit ? pos : rq.limit - 1; };
    auto stands_at = [&](int row) { return rq.p0 + ((row < rows ? row : rows - 1) >> p.gs); };
    const int w_row = x.row0 + 32 * wave;
    const bool active = w_row < rows;
    const int row = w_row + n < rows ? w_row + n : rows - 1;
    const Sight sight(p, rq.p0 + (row >> p.gs), rq.limit);

    // staging: a wave moves kParts x 4 rows of a tile, a lane the chunk that belongs at its place of the 1 KB; rows behind the
    // last key that the workgroup sees repeat it
    const int last_tile = (span.keys - 1) >> 5, last_key = (span.keys - 1) & 31;
    uint32_t soff[kParts], soff_last[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        const int part = wave * kParts + i, r4 = 4 * part, r4l = r4 < (last_key & ~3) ? r4 : last_key & ~3;
        const uint32_t chunk = ((lane & 15) ^ swz(r4 + (lane >> 4))) << 4;
        const int in = lane >> 4, inl = in < last_key - r4l ? in : last_key - r4l;
        soff[i] = ((r4 & 15) + in) * 256 + chunk;
        soff_last[i] = ((r4l & 15) + inl) * 256 + chunk;
    }
    const int half = wave * kParts * 4 >> 4;                        // which 16 keys of a tile this wave moves
    const unsigned char* kbase = (const unsigned char*)(kPaged ? p.k : p.k + (int64_t)(x.b * p.Hkv + x.g) * p.N * kD);
    const unsigned char* vbase = (const unsigned char*)(kPaged ? p.v : p.v + (int64_t)(x.b * p.Hkv + x.g) * p.N * kD);
    const uint32_t to0 = lds0 + wave * (kParts * 1024);
    auto stage = [&](const unsigned char* base, int place, uint32_t slot) __attribute__((always_inline)) {
        base += (uint64_t)(uint32_t)(place & ~3) << 10;             // x 16 rows x 256 bytes
        const bool last = place & kLast;
#pragma unroll
        for (int i = 0; i < kParts; ++i) load_to_lds16(base, last ? soff_last[i] : soff[i], to0 + slot * kTileBytes + 1024 * i);
    };
    const Operands at(lds0, lds0 + kRing * kTileBytes, lane);
    half8_t tq[8], pr[2][2];
    load_query(tq, p, x, row, lane);
    float16_t sc[2];
    auto place_at = [&](int tile, int j) {                          // of 16-key half j, -1: no page
        int key = tile * 32 + 16 * j;
        if (key > ((span.keys - 1) & ~15)) key = (span.keys - 1) & ~15;
        return kPaged ? place_of(p, p.table + (int64_t)x.r * p.table_cap, x.g, key) : key >> 4;
    };
    auto noted = [&](int place, int tile) { return (place < 0 ? kBad : place << 2) | (tile == last_tile ? kLast : 0); };
    auto seen_by_all = [&](int tile) { return sight.whole(tile, sees_to(x.row0), stands_at(x.row0 + 32 * NW - 1)); };
    if (tid == 0) *s_odd = 0;

    for (int ua = x.from; ua < x.to; ua += kTurn) {
        const int m = x.to - ua < kTurn ? x.to - ua : kTurn;        // tiles of this turn; i counts them
        auto tile_of = [&](int i) { return span.tile(ua + i); };
        __syncthreads();                                            // the turn before has been read
        for (int i = tid; i < m + 8; i += NW * 64) {
            const int tile = tile_of(i < m ? i : m - 1);
            Note note;
            note.edge = i < m ? 0 : kHidden | kEdgeAny | 255;
            int bad = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int place = place_at(tile, j);
                bad |= place < 0;
                note.place[j] = noted(place, tile);
            }
            if (bad || !seen_by_all(tile)) {
                note.edge |= kEdgeAny;
                for (int w = 0; w < NW; ++w)
                    if (bad || !sight.whole(tile, sees_to(x.row0 + 32 * w), stands_at(x.row0 + 32 * w + 31))) note.edge |= 1 << w;
            }
            note.unused = 0;
            notes[i] = note;
        }
        // the V slot of "tile -1" is multiplied with zero probabilities: it has to be finite
#pragma unroll
        for (int i = 0; i < kParts; ++i) *(uint4_t*)(s_kv + (2 * kRing - 1) * kTileBytes + (i * NW * 64 + tid) * 16) = uint4_t{0u, 0u, 0u, 0u};
        wait_all_loads();
        __syncthreads();
        auto own_place = [&](int i) { return scalar(notes[i].place[half]); };
        // two bits a tile, from tile i on: edge of the wave, of the workgroup
        auto edges = [&](int edge) { return (uint32_t)(edge >> wave & 1) | (uint32_t)(edge & kEdgeAny) >> 7; };
        uint32_t hist = 0;
        int pk[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            pk[i] = own_place(i);
            stage(kbase, pk[i], i);
        }
        stage(vbase, pk[0], kRing);
        stage(vbase, pk[1], kRing + 1);
        int v_next = pk[2], v_then = pk[3], k_next = own_place(4);  // places of tiles i + 2, i + 3 (V) and i + 4 (K)
#pragma unroll
        for (int i = 0; i < 5; ++i) hist |= edges(scalar(notes[i].edge)) << (2 * i);
        int ahead_place = notes[5].place[half], ahead_edge = notes[5].edge;      // of the tile that the next step asks for
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) pr[1][i][j] = (half_t)0.f;
        wait_all_loads();
        __syncthreads();

        // stages for step i and brings the places one tile on; returns tile i's edges
        auto stage_ahead = [&](int i, int T) __attribute__((always_inline)) {
            stage(kbase, k_next, T);
            stage(vbase, v_next, kRing + ((T + 2) & 3));
            v_next = v_then;
            v_then = k_next;
            k_next = scalar(ahead_place);
            const uint32_t now = hist & 3;
            hist = hist >> 2 | edges(scalar(ahead_edge)) << 8;
            ahead_place = notes[i + 6].place[half];
            ahead_edge = notes[i + 6].edge;
            return now;
        };
        auto seen_of = [&](int i) {
            const Note note = notes[i];
            const uint32_t bad = scalar((note.place[0] >> 1 & 1) | (note.place[1] & kBad));
            return scalar(note.edge) & kHidden ? 0u : sight.of_tile(tile_of(i), bad, kh);
        };
        // A hidden key counts as nothing whatever its V holds, but 0 x inf is NaN: in a tile of which some row of the workgroup does not
        // see some key, V that is not finite is cleared in LDS, by the wave that has staged it, and looked at again at the end.
        const uint32_t own = lds0 + (kRing * kTileBytes) + wave * (kParts * 1024) + lane * 16;       // what the lane has staged of a V tile
        auto clear_odd = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
                lds_uint4* to = (lds_uint4*)(uintptr_t)(own + slot * kTileBytes + 1024 * i);
                uint4_t two = *to;
                uint32_t any = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t odd = not_finite(two[j]);
                    two[j] = without(two[j], odd);
                    any |= odd;
                }
                if (any) {
                    *to = two;
                    *s_odd = 1;
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        };
        // waits for the tiles of two steps ago; tile i's V is among them
        auto land = [&](int slot, uint32_t edge) __attribute__((always_inline)) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * kParts) : "memory");
            if (__builtin_expect(edge & 2, 0)) clear_odd(slot);
            asm volatile("s_barrier" ::: "memory");
        };

        if (active) {
            float16_t z;
#pragma unroll
            for (int r = 0; r < 16; ++r) z[r] = 0.f;
            sc[0] = z;
#pragma unroll
            for (int s = 0; s < 8; ++s) sc[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(at.k_op(s, 0), tq[s], sc[0], 0, 0, 0);
        }
        __syncthreads();                                            // step 0 stages over the tile that has just been read

        // step i: softmax of tile i (its scores s, slot T), scores y of i + 1, value product of i - 1 with its probabilities before
        auto step = [&](int i, int T, float16_t& s, float16_t& y, half8_t(&now)[2], const half8_t(&before)[2]) __attribute__((always_inline)) {
            const int next = (T + 1) & 3, prev = (T + 3) & 3;
            const uint32_t edge = stage_ahead(i, T);
            if (__builtin_expect(edge & 1, 0)) mask(s, seen_of(i));
            float alpha;
            const bool moves = sums.open(s, p.c1, alpha);
            half8_t ka[8], va[8];
            ka[0] = at.k_op(0, next); va[0] = at.v_op(0, prev);
            ka[1] = at.k_op(1, next); va[1] = at.v_op(1, prev);
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int r = 0; r < 16; ++r) y[r] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j + 2 < 8) { ka[j + 2] = at.k_op(j + 2, next); va[j + 2] = at.v_op(j + 2, prev); }
                y = __builtin_amdgcn_mfma_f32_32x32x16_f16(ka[j], tq[j], y, 0, 0, 0);                               // rows = keys, cols = queries
                float p0 = fast_exp2(fmaf(s[2 * j], p.c1, -sums.m_ref));
                sum[0] += p0;
                sums.o[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va[j], before[j >> 2], sums.o[j & 3], 0, 0, 0);   // rows = channels
                float p1 = fast_exp2(fmaf(s[2 * j + 1], p.c1, -sums.m_ref));
                sum[1] += p1;
                pin(sum[0]);                                        // (the products must not sink below the loop)
                pin(sum[1]);
                now[j >> 2][(2 * j) & 7] = (half_t)p0;
                now[j >> 2][(2 * j + 1) & 7] = (half_t)p1;
                __builtin_amdgcn_sched_barrier(0);
            }
            sums.l += sum[0] + sum[1];
            if (__builtin_expect(moves, 0)) sums.rescale(alpha);
            land(T, edge);
        };
        if (active) {
#pragma unroll 1
            for (int i = 0; i < m; i += 4) {
                step(i, 0, sc[0], sc[1], pr[0], pr[1]);
                step(i + 1, 1, sc[1], sc[0], pr[1], pr[0]);
                step(i + 2, 2, sc[0], sc[1], pr[0], pr[1]);
                step(i + 3, 3, sc[1], sc[0], pr[1], pr[0]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sums.o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(at.v_op(i, 3), pr[1][i >> 2], sums.o[i & 3], 0, 0, 0);
        } else {                                                    // a wave without rows stages for the others
#pragma unroll 1
            for (int i = 0; i < ((m + 3) & ~3); ++i) {
                const uint32_t edge = stage_ahead(i, i & 3);
                land(i & 3, edge);
            }
        }
        wait_all_loads();                                           // nothing may land in LDS after the turn, or the workgroup's end
    }
    sums.join_halves();
    // values that are not finite, to the rows that see them: 1, some were cleared; 2, some sum is not finite
    if (active && __any(sums.odd())) *s_odd = 2;
    __syncthreads();
    const int odd = scalar(*s_odd);
    if (__builtin_expect(odd, 0)) {
        if (odd == 2) sums.drop_odd();
#pragma unroll 1
        for (int u = x.from; u < x.to; ++u) {
            const int tile = span.tile(u), p0 = scalar(place_at(tile, 0)), p1 = scalar(place_at(tile, 1));
            const uint32_t bad = (p0 < 0 ? 1 : 0) | (p1 < 0 ? 2 : 0);
            if (odd == 1 && bad == 0 && seen_by_all(tile)) continue;
            stage(vbase, noted(half ? p1 : p0, tile), kRing);
            wait_all_loads();
            __syncthreads();
            if (active) add_odd(sums, at, 0, sight.of_tile(tile, bad, kh));
            __syncthreads();                                        // the tile has been read
        }
    }
}

// A row's result: fp16 channels 32 cg + 8 qd + 4 kh .. + 3 and, from half-wave 0, its statistics.  A row that sees nothing is zero.
__device__ __forceinline__ void write_row(const Params& p, const Sums& x, int64_t b, int64_t t, int h, int kh)
{
    const float inv = x.l == 0.f ? 0.f : 1.f / x.l;
    half_t* op = p.out + b * p.os_b + t * p.os_t + h * p.os_h + 4 * kh;
#pragma unroll
    for (int cg = 0; cg < 4; ++cg)
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
            half4_t w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = (half_t)(x.o[cg][4 * qd + e] * inv);
            *(half4_t*)(op + 32 * cg + 8 * qd) = w;
        }
    if (kh == 0 && p.row_max) {
        const int64_t at = b * p.st_b + h * p.st_h + t;
        p.row_max[at] = x.s_max * p.c1 * (1.f / kLog2e);
        p.row_sum[at] = x.l == 0.f ? 0.f : x.l * fast_exp2(fmaf(-x.s_max, p.c1, x.m_ref));
    }
}

inline int log2_of(int G) { return G == 4 ? 2 : G == 2 ? 1 : 0; }

}  // namespace span

}  // namespace antkv
