// Attention over a cache in pages of 8 bits (page_attn.h has the work and how it is shared, bytes.h what the pages hold).
//
// A value x its scale is an fp16 number, so that the arithmetic is the FP16 cache's on half the bytes: K and V become fp16 on their way into
// the matrix units, four of them in two instructions that apply the scale as well.
//
// Narrow blocks: a wave streams key tiles of its own, two of them (K, V and their scales, 8.25 KB each) in flight or in use, and makes
// halves of the operands that it reads.  Two k-steps of an operand are 16 bytes of a key: the query's channels are in that order.
// Wide blocks: the tiles' bytes go straight into LDS, four tiles of K and of V in flight; each wave makes halves of the 1 KB pieces that it
// has staged itself, two tiles of K and of V at a time, once for all waves (8 conversions per lane and step, of four waves 16, where
// converting operands would be 64).
#include "bytes.h"
#include "page_attn.h"

namespace antkv {

namespace {

using namespace paged;

constexpr int kByteTile = 32 * kD;                                  // bytes of a tile's K, or V

// 4 bytes per lane from the lane's address to LDS address `to` + 4 * lane
__device__ __forceinline__ void gather_to_lds4(const float* from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "m0", "memory");
}

// Rows of a byte tile are 8 chunks of 16 bytes; chunk c of row r sits at place c ^ turn(r).  The 16-byte reads of 16 rows and the 8 rows x 32
// bytes of a transposed read then fall on 64 different banks.
__device__ __forceinline__ int turn(int r) { return (r >> 2 & 1) | (r & 2) | (r >> 1 & 4); }

typedef __attribute__((address_space(3))) uint2_t lds_uint2;
typedef int int2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) int2_t lds_int2;
typedef __attribute__((address_space(3))) float lds_float;

// Operands of a narrow block out of byte tiles: K row n, channels 32 s + 16 kh .. + 15 for k-steps 2 s and 2 s + 1; V transposed: inside a
// 16-lane block, lane 2 e + c reads key e of the lane's eight (4 kh + 0 .. 3 and 8 + 4 kh + 0 .. 3), channels 8 c .. 8 c + 7 of 16.
struct ByteOperands {
    uint32_t k[4], v[4], scale;                                     // LDS addresses
    float v_scale[2];                                               // of the tile's 16-key halves

    __device__ __forceinline__ ByteOperands(uint32_t at, uint32_t scales, int lane)
    {
        const int n = lane & 31, kh = lane >> 5, e = (lane & 15) >> 1, c = lane & 1, blk = lane >> 4 & 1;
        const int r = 4 * kh + (e & 3) + 8 * (e >> 2);
#pragma unroll
        for (int s = 0; s < 4; ++s) { k[s] = at + n * kD + (((2 * s + kh) ^ turn(n)) << 4); pin(k[s]); }
#pragma unroll
        for (int cg = 0; cg < 4; ++cg) { v[cg] = at + kByteTile + r * kD + (((2 * cg + blk) ^ turn(r)) << 4) + 8 * c; pin(v[cg]); }
        scale = scales;
    }
    // slots of a wave: two tiles; of its scales: 64 words each
    __device__ __forceinline__ uint4_t k_bytes(int s, int slot) const { return *(lds_uint4*)(uintptr_t)(k[s] + slot * 2 * kByteTile); }
    __device__ __forceinline__ float scale_at(int place, int slot) const { return *(lds_float*)(uintptr_t)(scale + slot * 256 + 64 * place); }
    __device__ __forceinline__ half8_t v_op(int i, int slot) const                      // i = 4 * (16-key half) + channel group
    {
        const uint32_t at = v[i & 3] + slot * 2 * kByteTile + (i >> 2) * 16 * kD;
        return halves_of(__builtin_bit_cast(uint2_t, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_int2*)(uintptr_t)at)), v_scale[i >> 2]);
    }
};

struct BytePages {
    // Costs of key tiles, 2 and 4: four waves share a narrow block's, a workgroup each works on 0.25 and 1.0 us a tile side by side (a
    // narrow one 0.5 where all are).  As one and as half: 16 requests with 2048 tokens among them 87 and 81 us, 300 x 20 on 40 .. 1500 144 and 126, 64
    // tokens on 1 .. 32768 keys each 87 and 85.
    static constexpr int kShiftNarrow = 1, kShiftWide = 2;
    // Of coming and going: 10 and 15 us a block (pages, scales, first tiles 5, partial sums 4).  Narrow, 32 and 40: 64 tokens on 1 .. 32768 keys 88 and 85 us
    static constexpr int kIdleNarrow = 40, kIdleWide = 64;
    // The smallest shares.  Narrow blocks, 20, 24, 32, 40: a token on 1024 keys 11.3, 11.9, 12.0, 12.6 us, on 4096 12.1, 12.5, 12.7, 12.8, but on 16384 20.5, 20.0, 17.7, 17.0
    // (each piece arrives at the same word, and is asked for by the last one), 16 on 300 each 10.5, 11.7, 11.1, 10.6, 4 on 2048 13.5, 13.3, 13.7, 13.8.
    // Wide ones, 96 and 144: 300 tokens on 2000 keys 42 and 52.  All of these are of 32 heads on 8, 64 shares of a KV head.  Of 32 on 32, 16 shares, narrow 20, 32, 40: a
    // token on 1024 keys 11.4, 12.0, 12.6, on 4096 16.7, 15.6, 14.8 (12 % that the rule leaves there), on 16384 34.9 and on 32768 57.5 with any; wide 48, 96, 144: 300 on 2000
    // 38, 35, 43, 4 x 100 on 1000 32.9, 33.8, 37.3.  The rules around this one make no difference there (1 % at most, from kFirst 4, kIdleNarrow 32, words 8 bytes
    // apart, kRowsOfEight 512)
    __device__ __forceinline__ static int least(bool wide, int total) { return wide ? 96 : total < 480 ? 20 : 32; }
    // Key tiles of a block's first piece, at least.  4 and 8: 16 tokens on 300 keys each 13.6 and 12.7 us, 4 x 100 on 1000 36.3 and 34.9
    static constexpr int kFirst = 8;
    // Partial sums of a row that are asked for together (more are padded).  8, 12, 16, 32: 40 single tokens on 300 keys 11.2, 11.5, 11.9, 13.3 us, one on 4096 12.3, 12.0,
    // 12.3, 14.0, on 16384 22.7, 22.5, 22.8, 24.1
    static constexpr int kBatch = 8;
    // Arrival words, in 8 bytes apart.  1 and 16, a line each: a token on 32768 keys 31.3 and 25.2 us, on 16384 22.7 and 20.0, on 4096 12.3 and 12.5
    static constexpr int kWordApart = 16;
    // 1024 and 512: 16 requests with 2048 tokens among them 88 and 102 us; 1024 and 256: 64 tokens on 4096 keys 39 and 50
    static constexpr int kRowsOfEight = 1024;

    template <int NW>                                   // waves of a workgroup: 8 or 4
    struct Lds {
        static constexpr int tiles = 0;                                 // narrow: two K and V tiles per wave; wide: the rings
        static constexpr int scales = NW * 4 * kByteTile;               // narrow: of the two tiles, per wave
        static constexpr int notes = scales + NW * 512;                 // what is known of the turn's key tiles; narrow: [kTurnNarrow][2] places
        static constexpr int stat = notes + kByteNotes * (int)sizeof(Note);     // [NW][kNarrow][4]: reference, sum, largest score
        static constexpr int total = stat + NW * kNarrow * 16;
        static_assert(4 * kTileBytes + 8 * kByteTile <= notes && NW * kNarrow * kD * 4 <= scales && kTurnNarrow * 8 <= stat - notes &&
                      (total + kWindows * 8 + 1024) * (8 / NW) <= 163840, "LDS of a CU");
    };

    // Sums of up to 32 rows over the wave's share of the piece's key tiles: every NWth.
    template <int NW>
    __device__ __forceinline__ static void narrow_sums(Sums& sums, const Params& p, const Piece& x, const Span& span, unsigned char* s_tiles, int* s_place)
    {
        const int tid = own_thread(), lane = tid & 63, n = lane & 31, kh = lane >> 5, wave = scalar(tid >> 6);
        const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)s_tiles, own = lds0 + wave * (4 * kByteTile), scales = lds0 + Lds<NW>::scales + wave * 512;
        const Request rq = x.rq;
        const int rows = rq.n << p.gs, row = n < rows ? n : rows - 1;
        const int hi = rq.p0 + rq.n - 1, all = rq.p0 < rq.limit ? rq.p0 : rq.limit - 1;
        const Sight sight(p, rq.p0 + (row >> p.gs), rq.limit);
        const int last_tile = (span.keys - 1) >> 5, last_key = (span.keys - 1) & 31;
        // staging: 1 KB, eight rows, per load; rows behind the last key repeat it
        const int l8 = lane >> 3;
        uint32_t soff[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) soff[j] = ((8 * j + l8) & 15) * kD + (((lane & 7) ^ turn(8 * j + l8)) << 4);
        const float* const scale_of = lane < 32 ? p.k_scales : p.v_scales;
        constexpr int kLoads = 9;                                   // of a tile
        auto stage = [&](int a, int c, bool last, int slot) __attribute__((always_inline)) {
            a = a > 0 ? a : 0;
            c = c > 0 ? c : 0;
            const unsigned char* pools[2] = {(const unsigned char*)p.k, (const unsigned char*)p.v};
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t off = soff[j];
                    if (last) {
                        const int at = 8 * j + l8;
                        off = ((at < last_key ? at : last_key) & 15) * kD + (off & (kD - 1));
                    }
                    load_to_lds16(pools[u] + (int64_t)(j < 2 ? a : c) * (16 * kD), off, own + slot * 2 * kByteTile + u * kByteTile + 1024 * j);
                }
            gather_to_lds4(scale_of + (lane & 16 ? c : a), scales + 256 * slot);
        };
        ByteOperands at(own, scales, lane);
        half8_t tq[8];
        load_query<true>(tq, p, x, row, lane);
        const int32_t* row_of = p.table + (int64_t)x.r * p.table_cap;
        auto place_at = [&](int tile, int j) {                      // of 16-key half j, -1: no page
            int key = tile * 32 + 16 * j;
            if (key > ((span.keys - 1) & ~15)) key = (span.keys - 1) & ~15;
            return place_of(p, row_of, x.g, key);
        };
        bool odd = false;                                           // some edge tile's V was not finite
        for (int ua = x.from; ua < x.to; ua += kTurnNarrow) {
            const int m = x.to - ua < kTurnNarrow ? x.to - ua : kTurnNarrow;
            if (ua > x.from) __syncthreads();                       // the turn before has been read
            for (int k = tid; k < 2 * m; k += NW * 64) s_place[k] = place_at(span.tile(ua + (k >> 1)), k & 1);
            wait_all_loads();
            __syncthreads();
            const int mine = (m - wave + NW - 1) / NW;              // tiles wave, wave + NW, .. of the turn
            if (mine <= 0) continue;
            auto tile_of = [&](int i) { return span.tile(ua + wave + NW * i); };
            auto places = [&](int i, int& a, int& c) {
                const int k = 2 * (wave + NW * (i < mine ? i : mine - 1));
                a = scalar(s_place[k]);
                c = scalar(s_place[k + 1]);
            };
            auto ask = [&](int i, int a, int c, int slot) __attribute__((always_inline)) { stage(a, c, tile_of(i < mine ? i : mine - 1) == last_tile, slot); };
            int a, c, na, nc;                                       // places of tiles i and i + 1
            places(0, a, c);
            ask(0, a, c, 0);
            places(1, na, nc);
            ask(1, na, nc, 1);                                      // (behind the last tile: it once more, which keeps the counts)
            // tile i, in slot i & 1
            auto step = [&](int i, int slot) __attribute__((always_inline)) {
                const int tile = tile_of(i);
                const uint32_t bits = (a < 0 ? 1 : 0) | (c < 0 ? 2 : 0);
                int pa, pc;
                places(i + 2, pa, pc);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");                // the tile has landed
                const float k_scale = at.scale_at(n >> 4, slot);
                at.v_scale[0] = at.scale_at(2, slot);
                at.v_scale[1] = at.scale_at(3, slot);
                float16_t s;
                uint4_t bytes[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) bytes[j] = at.k_bytes(j, slot);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    s = __builtin_amdgcn_mfma_f32_32x32x16_f16(halves_of(uint2_t{bytes[j >> 1][2 * (j & 1)], bytes[j >> 1][2 * (j & 1) + 1]}, k_scale), tq[j], s, 0, 0, 0);
                const bool edge = bits != 0 || !sight.whole(tile, all, hi);
                if (__builtin_expect(edge, 0)) mask(s, sight.of_tile(tile, bits, kh));
                float alpha;
                if (sums.open(s, p.c1, alpha)) sums.rescale(alpha);
                float sum[2] = {0.f, 0.f};
                half8_t pr[2], op[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) op[j] = at.v_op(j, slot);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float e = fast_exp2(fmaf(s[r], p.c1, -sums.m_ref));
                    sum[r & 1] += e;
                    pr[r >> 3][r & 7] = (half_t)e;
                }
                sums.l += sum[0] + sum[1];
                if (__builtin_expect(edge, 0)) {                    // hidden or not, what is not finite waits until the end
                    uint32_t any = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        uint4_t two = __builtin_bit_cast(uint4_t, op[j]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t is = not_finite(two[e]);
                            two[e] = without(two[e], is);
                            any |= is;
                        }
                        op[j] = __builtin_bit_cast(half8_t, two);
                    }
                    odd = odd || __any(any != 0);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) sums.o[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(op[j], pr[j >> 2], sums.o[j & 3], 0, 0, 0);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile has been read
                a = na;
                c = nc;
                na = pa;
                nc = pc;
                ask(i + 2, na, nc, slot);
            };
#pragma unroll 1
            for (int i = 0; i < mine; i += 2) {
                step(i, 0);
                if (i + 1 < mine) step(i + 1, 1);
            }
            wait_all_loads();                                       // nothing may land in LDS after the turn
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        sums.join_halves();
        // values that are not finite, to the rows that see them: of the wave's edge tiles, or of all where some sum is not finite
        const bool every = __any(sums.odd());
        if (__builtin_expect(odd || every, 0)) {
            if (every) sums.drop_odd();
#pragma unroll 1
            for (int u = x.from + wave; u < x.to; u += NW) {
                const int tile = span.tile(u), a = scalar(place_at(tile, 0)), c = scalar(place_at(tile, 1));
                const uint32_t bits = (a < 0 ? 1 : 0) | (c < 0 ? 2 : 0);
                if (!every && bits == 0 && sight.whole(tile, all, hi)) continue;
                stage(a, c, tile == last_tile, 0);
                wait_all_loads();
                at.v_scale[0] = at.scale_at(2, 0);
                at.v_scale[1] = at.scale_at(3, 0);
                add_odd(sums, at, 0, sight.of_tile(tile, bits, kh));
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile has been read
            }
        }
    }

    // Sums of the piece's rows, 32 to a wave, over its key tiles.  s_kv: two tiles of K and of V in halves, then four of each in bytes; s_odd: a
    // word; notes: kByteNotes of them.  Step i works on tile i as span::wide_sums does (scores of tile i + 1, values of tile i - 1), makes
    // halves of K of tile i + 2 and of V of tile i, and asks for the bytes of K of tile i + 6 and of V of tile i + 4.
    template <int NW>
    __device__ __forceinline__ static void wide_sums(Sums& sums, const Params& p, const Piece& x, const Span& span, unsigned char* s_kv, int* s_odd, Note* notes)
    {
        // a tile's K, and V, is four pieces of 1 KB, eight rows: of four waves each has a piece of K and one of V, of eight four have K and four V
        constexpr int kStreams = NW == 8 ? 1 : 2;
        const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte*)s_kv;
        const int tid = own_thread(), lane = tid & 63, n = lane & 31, kh = lane >> 5;
        const int wave = scalar(tid >> 6);                          // so that per-wave conditions are scalar branches
        const Request rq = x.rq;
        const int rows = rq.n << p.gs;
        // first and last row of wave w, or of the workgroup: the last key that the first sees, the last one's position
        auto sees_to = [&](int row) { const int pos = rq.p0 + (row >> p.gs); return pos < rq.limit ? pos : rq.limit - 1; };
        auto stands_at = [&](int row) { return rq.p0 + ((row < rows ? row : rows - 1) >> p.gs); };
        const int w_row = x.row0 + 32 * wave;
        const bool active = w_row < rows;
        const int row = w_row + n < rows ? w_row + n : rows - 1;
        const Sight sight(p, rq.p0 + (row >> p.gs), rq.limit);

        // staging: lane's row of the piece's eight and 16 bytes of it.  Eight lanes have four pieces each of two rows four apart: what they write
        // together, every other 16 bytes of the halves, then falls on different banks (of 128 bytes at a time).  Rows behind the last key that the
        // workgroup sees repeat it
        const int part = wave & 3, half = part >> 1, r = 8 * part + (lane >> 4) + 4 * (lane >> 2 & 1), chunk = (lane & 3) + 4 * (lane >> 3 & 1);
        const int last_tile = (span.keys - 1) >> 5, last_key = (span.keys - 1) & 31;
        const uint32_t soff = (r & 15) * kD + chunk * 16, soff_last = ((r < last_key ? r : last_key) & 15) * kD + chunk * 16;
        const uint32_t bytes0 = lds0 + 4 * kTileBytes + part * 1024;                       // of K in slot 0; V 4 tiles on
        const uint32_t to[2] = {lds0 + r * 256 + (((2 * chunk) ^ swz(r)) << 4), lds0 + r * 256 + (((2 * chunk + 1) ^ swz(r)) << 4)};
        // which of the two the wave's stream u is, 0: K, 1: V; how far ahead of the step its halves are made
        auto kind = [&](int u) { return NW == 8 ? wave >> 2 : u; };
        auto ahead = [&](int u) { return kind(u) ? 0 : 2; };
        auto stage = [&](int v, int place, int slot) __attribute__((always_inline)) {
            const unsigned char* base = (const unsigned char*)(v ? p.v : p.k) + ((uint64_t)(uint32_t)(place & ~3) << 9);      // x 16 rows x 128 bytes
            load_to_lds16(base, place & kLast ? soff_last : soff, bytes0 + (4 * v + slot) * kByteTile);
        };
        auto fetch = [&](int v, int slot) { return *(lds_uint4*)(uintptr_t)(bytes0 + (4 * v + slot) * kByteTile + lane * 16); };
        // halves of the lane's 16 bytes to slot `slot`; clean: without what is not finite, which is noted
        auto put = [&](int v, const uint4_t& b, int exponents, int slot, bool clean) __attribute__((always_inline)) {
            const float scale = __builtin_bit_cast(float, (exponents >> (16 * v + 8 * half) & 255) << 23);
            uint4_t two[2] = {__builtin_bit_cast(uint4_t, halves_of(uint2_t{b[0], b[1]}, scale)), __builtin_bit_cast(uint4_t, halves_of(uint2_t{b[2], b[3]}, scale))};
            if (__builtin_expect(clean, 0)) {
                uint32_t any = 0;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t is = not_finite(two[j][e]);
                        two[j][e] = without(two[j][e], is);
                        any |= is;
                    }
                if (any) *s_odd = 1;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) *(lds_uint4*)(uintptr_t)(to[j] + (2 * v + slot) * kTileBytes) = two[j];
        };
        const Operands at(lds0, lds0 + 2 * kTileBytes, lane);
        half8_t tq[8], pr[2][2];
        load_query<false, false>(tq, p, x, row, lane);              // on its way under the first look at the pages
        float16_t sc[2];
        auto place_at = [&](int tile, int j) {                      // of 16-key half j, -1: no page
            int key = tile * 32 + 16 * j;
            if (key > ((span.keys - 1) & ~15)) key = (span.keys - 1) & ~15;
            return place_of(p, p.table + (int64_t)x.r * p.table_cap, x.g, key);
        };
        auto noted = [&](int place, int tile) { return (place < 0 ? kBad : place << 2) | (tile == last_tile ? kLast : 0); };
        auto exponent = [&](const float* scales, int place) { return (int)(__builtin_bit_cast(uint32_t, scales[place < 0 ? 0 : place]) >> 23 & 255); };
        auto exponents_of = [&](int p0, int p1) { return exponent(p.k_scales, p0) | exponent(p.k_scales, p1) << 8 | exponent(p.v_scales, p0) << 16 | exponent(p.v_scales, p1) << 24; };
        auto seen_by_all = [&](int tile) { return sight.whole(tile, sees_to(x.row0), stands_at(x.row0 + 32 * NW - 1)); };
        if (tid == 0) *s_odd = 0;

        for (int ua = x.from; ua < x.to; ua += kTurn) {
            const int m = x.to - ua < kTurn ? x.to - ua : kTurn;    // tiles of this turn; i counts them
            auto tile_of = [&](int i) { return span.tile(ua + i); };
            __syncthreads();                                        // the turn before has been read
            for (int i = tid; i < m + kByteNotes - kTurn; i += NW * 64) {
                const int tile = tile_of(i < m ? i : m - 1), p0 = place_at(tile, 0), p1 = place_at(tile, 1);
                Note note;
                note.edge = i < m ? 0 : kHidden | kEdgeAny | 255;
                note.place[0] = noted(p0, tile);
                note.place[1] = noted(p1, tile);
                note.exponents = exponents_of(p0, p1);
                const bool bad = p0 < 0 || p1 < 0;
                if (bad || !seen_by_all(tile)) {
                    note.edge |= kEdgeAny;
                    for (int w = 0; w < NW; ++w)
                        if (bad || !sight.whole(tile, sees_to(x.row0 + 32 * w), stands_at(x.row0 + 32 * w + 31))) note.edge |= 1 << w;
                }
                notes[i] = note;
            }
            // the V slot of "tile -1" is multiplied with zero probabilities: it has to be finite
#pragma unroll
            for (int i = 0; i < 8 / NW; ++i) *(uint4_t*)(s_kv + 3 * kTileBytes + (i * NW * 64 + tid) * 16) = uint4_t{0u, 0u, 0u, 0u};
#pragma unroll
            for (int s = 0; s < 8; ++s) pin(tq[s]);
            wait_all_loads();
            __syncthreads();
            auto own_place = [&](int i) { return scalar(notes[i].place[half]); };
            // two bits a tile, from tile i on: edge of the wave, of the workgroup
            auto edges = [&](int edge) { return (uint32_t)(edge >> wave & 1) | (uint32_t)(edge & kEdgeAny) >> 7; };
            uint32_t hist = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int u = 0; u < kStreams; ++u) stage(kind(u), own_place(i), i);
#pragma unroll
            for (int i = 0; i < 5; ++i) hist |= edges(scalar(notes[i].edge)) << (2 * i);
            int ahead_edge = notes[5].edge;                         // of the tile that the next step asks for
            int place[kStreams], exps[kStreams];                    // what step i asks for, and the scales of what it makes halves of
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) pr[1][i][j] = (half_t)0.f;
            wait_all_loads();
#pragma unroll
            for (int i = 0; i < 2; ++i) {                           // K of tiles 0 and 1
#pragma unroll
                for (int u = 0; u < kStreams; ++u)
                    if (kind(u) == 0) put(0, fetch(0, i), scalar(notes[i].exponents), i, false);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            // as steps -2 and -1 would: K of tiles 4 and 5 (V of 2 and 3 is there, but the loads are counted)
#pragma unroll
            for (int i = -2; i < 0; ++i)
#pragma unroll
                for (int u = 0; u < kStreams; ++u) stage(kind(u), own_place(i + 4 + ahead(u)), (i + 4 + ahead(u)) & 3);
#pragma unroll
            for (int u = 0; u < kStreams; ++u) {
                place[u] = notes[4 + ahead(u)].place[half];
                exps[u] = notes[ahead(u)].exponents;
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");

            uint4_t bytes[kStreams];
            uint32_t edge;
            // step i: the bytes that become halves, out of LDS
            auto take = [&](int i, int T) __attribute__((always_inline)) {
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * kStreams) : "memory");          // those that step i - 4 asked for
#pragma unroll
                for (int u = 0; u < kStreams; ++u) bytes[u] = fetch(kind(u), (T + ahead(u)) & 3);
                edge = hist & 3;
                hist = hist >> 2 | edges(scalar(ahead_edge)) << 8;
                ahead_edge = notes[i + 6].edge;
            };
            auto make = [&](int u, int T) __attribute__((always_inline)) { put(kind(u), bytes[u], scalar(exps[u]), T & 1, kind(u) && edge & 2); };
            auto end = [&](int i, int T) __attribute__((always_inline)) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (the bytes have been read, the halves written)
#pragma unroll
                for (int u = 0; u < kStreams; ++u) {
                    stage(kind(u), scalar(place[u]), (T + ahead(u)) & 3);
                    place[u] = notes[i + 5 + ahead(u)].place[half];
                    exps[u] = notes[i + 1 + ahead(u)].exponents;
                }
                asm volatile("s_barrier" ::: "memory");
            };
            auto seen_of = [&](int i) {
                const Note note = notes[i];
                const uint32_t bad = scalar((note.place[0] >> 1 & 1) | (note.place[1] & kBad));
                return scalar(note.edge) & kHidden ? 0u : sight.of_tile(tile_of(i), bad, kh);
            };

            if (active) {
                float16_t z;
#pragma unroll
                for (int r = 0; r < 16; ++r) z[r] = 0.f;
                sc[0] = z;
#pragma unroll
                for (int s = 0; s < 8; ++s) sc[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(at.k_op(s, 0), tq[s], sc[0], 0, 0, 0);
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");                  // step 0 writes over the tile that has just been read

            // step i: softmax of tile i (its scores s), scores y of i + 1, value product of i - 1 with its probabilities before
            auto step = [&](int i, int T, float16_t& s, float16_t& y, half8_t(&now)[2], const half8_t(&before)[2]) __attribute__((always_inline)) {
                take(i, T);
                if (__builtin_expect(edge & 1, 0)) mask(s, seen_of(i));
                tile_step(sums, at, tq, p.c1, (T + 1) & 1, (T + 1) & 1, s, y, now, before, [&](int j) __attribute__((always_inline)) {
                    if (j == (kStreams > 1 ? 4 : 3)) make(0, T);
                    if (kStreams > 1 && j == 6) make(1, T);
                });
                end(i, T);
            };
            // Two workgroups of a CU: the one that came first would have the matrix units first as well, and be done long before the other (16 requests with
            // 2048 tokens among them 83 us, 300 x 20 tokens on 40 .. 1500 keys 127; 78 and 119 this way round)
            if (NW == 4 && (blockIdx.x >> 8 & 1)) __builtin_amdgcn_s_setprio(1);
            if (active) {
#pragma unroll 1
                for (int i = 0; i < m; i += 4) {
                    step(i, 0, sc[0], sc[1], pr[0], pr[1]);
                    step(i + 1, 1, sc[1], sc[0], pr[1], pr[0]);
                    step(i + 2, 2, sc[0], sc[1], pr[0], pr[1]);
                    step(i + 3, 3, sc[1], sc[0], pr[1], pr[0]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) sums.o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(at.v_op(i, 1), pr[1][i >> 2], sums.o[i & 3], 0, 0, 0);
            } else {                                                // a wave without rows stages for the others
#pragma unroll 1
                for (int i = 0; i < ((m + 3) & ~3); ++i) {
                    take(i, i);
#pragma unroll
                    for (int u = 0; u < kStreams; ++u) make(u, i);
                    end(i, i);
                }
            }
            if (NW == 4) __builtin_amdgcn_s_setprio(0);
            wait_all_loads();                                       // nothing may land in LDS after the turn, or the workgroup's end
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
                if (wave < 4) {
                    stage(1, noted(half ? p1 : p0, tile), 0);
                    wait_all_loads();
                    put(1, fetch(1, 0), scalar(exponents_of(p0, p1)), 0, false);
                }
                __syncthreads();
                if (active) add_odd(sums, at, 0, sight.of_tile(tile, bad, kh));
                __syncthreads();                                    // the tile has been read
            }
        }
    }
};

}  // namespace

size_t qpage_attn_workspace_bytes(const Geom& g, int64_t T) { return paged::workspace_bytes<BytePages>(g, T); }

hipError_t launch_qpage_attn(const Geom& g, const Pages& pg, const PageAttnArgs& a, void* ws, hipStream_t st) { return paged::launch<BytePages>(g, pg, a, ws, st); }

}  // namespace antkv
