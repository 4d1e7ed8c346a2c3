// Attention over a paged FP16 cache (page_attn.h has the work and how it is shared).
//
// Narrow blocks: a wave streams key tiles of its own through 16 KB of LDS, K of the next tile under the softmax of this one and V under the
// scores of the next, without a barrier.
//
// Bound: many tokens, the matrix units (2048 on 32768 keys, 32 heads on 8, 1.00 to 1.03 ms by card, 1.03 to 1.07 PFLOP/s); one token each, HBM (64 requests on 1 .. 32768
// keys 147 us, 5.5 TB/s); few keys or requests, the chain plan - pages - first tiles - meeting - partial sums - their sum, 1 to 3 us
// each (one token on 4096 keys 13 us, of which its tiles take 5).
#include "page_attn.h"

namespace antkv {

namespace {

using namespace paged;

struct Fp16Pages {
    static constexpr int kShiftNarrow = 0, kShiftWide = 0;          // a key tile costs 1
    // What a block costs beside its key tiles.  Narrow 14, 20, 28: 16 tokens on 300 keys each 11.0, 15.0, 16.2 us, 63 tokens beside one chunk of 100 on 2000
    // keys each 105, 106, 118, 64 on 1 .. 32768 keys 147, 148, 147 (4, measured earlier: 208 where 20 took 176).  Wide 12, 16, 20: 300 tokens on 2000
    // keys 46, 38, 46, 8 prompts of 1024 131, 121, 119
    static constexpr int kIdleNarrow = 14, kIdleWide = 16;
    // The smallest shares.  8, 12, 16: a token on 4096 keys 14.7, 13.2, 13.8 us, one each of 4 requests on 2048 keys 16.6, 14.5, 14.9; 16, 24, 32: 64
    // tokens on 4096 keys 32.5, 33.9, 36.0, 300 on 2000 39.4, 38.1, 46.2, 4 x 100 on 1000 32.1, 31.4, 32.0
    __device__ __forceinline__ static int least(bool wide, int) { return wide ? 24 : 12; }
    static constexpr int kWordApart = 1;                            // arrival words: 8 bytes apart
    static constexpr int kBatch = 16;                               // partial sums of a row that are asked for together
    static constexpr int kFirst = 4;                                // key tiles of a block's first piece, at least
    static constexpr int kRowsOfEight = 1024;                       // of a request on average, and a KV head: for workgroups of eight waves

    template <int NW>                                       // waves of a workgroup: 8 or 4
    struct Lds {
        static constexpr int tiles = 0;                                 // narrow: a K and a V tile per wave; wide: the rings
        static constexpr int notes = NW * 2 * kTileBytes;               // what is known of the turn's key tiles; narrow: [kTurnNarrow][2] places
        static constexpr int stat = notes + kNotes * (int)sizeof(Note); // [NW][kNarrow][4]: reference, sum, largest score
        static constexpr int total = stat + NW * kNarrow * 16;
        static_assert(kRingBytes <= notes && kTurnNarrow * 8 <= stat - notes && (total + kWindows * 8 + 1024) * (8 / NW) <= 163840, "LDS of a CU");
    };

    // ---- narrow blocks ---------------------------------------------------------------------------------------------------------------

    // Sums of up to 32 rows over the wave's share of the piece's key tiles: every NWth.
    template <int NW>
    __device__ __forceinline__ static void narrow_sums(Sums& sums, const Params& p, const Piece& x, const Span& span, unsigned char* s_tiles, int* s_place)
    {
        const int tid = own_thread(), lane = tid & 63, n = lane & 31, kh = lane >> 5, wave = scalar(tid >> 6);
        const uint32_t k_at = (uint32_t)(uintptr_t)(lds_byte*)s_tiles + wave * (2 * kTileBytes), v_at = k_at + kTileBytes;
        const Request rq = x.rq;
        const int rows = rq.n << p.gs, row = n < rows ? n : rows - 1;
        const int hi = rq.p0 + rq.n - 1, all = rq.p0 < rq.limit ? rq.p0 : rq.limit - 1;
        const Sight sight(p, rq.p0 + (row >> p.gs), rq.limit);
        const int last_tile = (span.keys - 1) >> 5, last_key = (span.keys - 1) & 31;
        // staging: 1 KB, four rows, per load; rows behind the last key repeat it
        const int l4 = lane >> 4;
        uint32_t soff[4];
    #pragma unroll
        for (int j = 0; j < 4; ++j) soff[j] = (4 * j + l4) * 256 + (((lane & 15) ^ swz(4 * j + l4)) << 4);
        auto stage = [&](const half_t* pool, int a, int c, bool last, uint32_t to) __attribute__((always_inline)) {
            const unsigned char* base[2] = {(const unsigned char*)pool + (int64_t)(a > 0 ? a : 0) * (16 * kD * 2), (const unsigned char*)pool + (int64_t)(c > 0 ? c : 0) * (16 * kD * 2)};
    #pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t off = soff[j & 3];
                if (last) {
                    const int at = 4 * j + l4;
                    off = ((at < last_key ? at : last_key) & 15) * 256 + (off & 255);
                }
                load_to_lds16(base[j >> 2], off, to + 1024 * j);
            }
        };
        const Operands at(k_at, v_at, lane);
        half8_t tq[8];
        load_query(tq, p, x, row, lane);
        const int32_t* row_of = p.table + (int64_t)x.r * p.table_cap;
        auto place_at = [&](int tile, int j) {                          // of 16-key half j, -1: no page
            int key = tile * 32 + 16 * j;
            if (key > ((span.keys - 1) & ~15)) key = (span.keys - 1) & ~15;
            return place_of(p, row_of, x.g, key);
        };
        bool odd = false;                                               // some edge tile's V was not finite
        for (int ua = x.from; ua < x.to; ua += kTurnNarrow) {
            const int m = x.to - ua < kTurnNarrow ? x.to - ua : kTurnNarrow;
            if (ua > x.from) __syncthreads();                           // the turn before has been read
            for (int k = tid; k < 2 * m; k += NW * 64) s_place[k] = place_at(span.tile(ua + (k >> 1)), k & 1);
            wait_all_loads();
            __syncthreads();
            const int mine = (m - wave + NW - 1) / NW;                  // tiles wave, wave + NW, .. of the turn
            if (mine <= 0) continue;
            auto tile_of = [&](int i) { return span.tile(ua + wave + NW * i); };
            auto places = [&](int i, int& a, int& c) {
                const int k = 2 * (wave + NW * (i < mine ? i : mine - 1));
                a = s_place[k];
                c = s_place[k + 1];
            };
            int a, c, va, vc;                                           // places of the tile that K, and V, are asked for next
            places(0, a, c);
            va = a = scalar(a);
            vc = c = scalar(c);
            stage(p.k, a, c, tile_of(0) == last_tile, k_at);
            stage(p.v, a, c, tile_of(0) == last_tile, v_at);
    #pragma unroll 1
            for (int i = 0; i < mine; ++i) {
                const int tile = tile_of(i);
                const bool more_last = tile_of(i + 1 < mine ? i + 1 : i) == last_tile;
                const uint32_t bits = (a < 0 ? 1 : 0) | (c < 0 ? 2 : 0);
                int na, nc;
                places(i + 1, na, nc);
                asm volatile("s_waitcnt vmcnt(8)" ::: "memory");         // K has landed
                float16_t s;
                half8_t op[8];
    #pragma unroll
                for (int j = 0; j < 8; ++j) op[j] = at.k_op(j, 0);
    #pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = 0.f;
    #pragma unroll
                for (int j = 0; j < 8; ++j) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(op[j], tq[j], s, 0, 0, 0);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // and has been read
                a = scalar(na);
                c = scalar(nc);
                stage(p.k, a, c, more_last, k_at);                       // (behind the last tile: once more, which keeps the counts)
                const bool edge = bits != 0 || !sight.whole(tile, all, hi);
                if (__builtin_expect(edge, 0)) mask(s, sight.of_tile(tile, bits, kh));
                float alpha;
                if (sums.open(s, p.c1, alpha)) sums.rescale(alpha);
                float sum[2] = {0.f, 0.f};
                half8_t pr[2];
    #pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float e = fast_exp2(fmaf(s[r], p.c1, -sums.m_ref));
                    sum[r & 1] += e;
                    pr[r >> 3][r & 7] = (half_t)e;
                }
                sums.l += sum[0] + sum[1];
                asm volatile("s_waitcnt vmcnt(8)" ::: "memory");         // V has landed
                if (__builtin_expect(edge, 0)) {                        // hidden or not, what is not finite waits until the end
    #pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        lds_uint4* to = (lds_uint4*)(uintptr_t)(v_at + 1024 * j + lane * 16);
                        uint4_t two = *to;
                        uint32_t any = 0;
    #pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t is = not_finite(two[e]);
                            two[e] = without(two[e], is);
                            any |= is;
                        }
                        if (any) *to = two;
                        odd = odd || __any(any != 0);
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
    #pragma unroll
                for (int j = 0; j < 8; ++j) op[j] = at.v_op(j, 0);
    #pragma unroll
                for (int j = 0; j < 8; ++j) sums.o[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(op[j], pr[j >> 2], sums.o[j & 3], 0, 0, 0);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                va = a;
                vc = c;
                stage(p.v, va, vc, more_last, v_at);
            }
            wait_all_loads();                                           // nothing may land in LDS after the turn
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
                stage(p.v, a, c, tile == last_tile, v_at);
                wait_all_loads();
                add_odd(sums, at, 0, sight.of_tile(tile, bits, kh));
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the tile has been read
            }
        }
    }

    template <int NW>
    __device__ __forceinline__ static void wide_sums(Sums& sums, const Params& p, const Piece& x, const Span& span, unsigned char* s_kv, int* s_odd, Note* notes)
    {
        span::wide_sums<NW, true>(sums, p, x, span, s_kv, s_odd, notes);
    }
};
}  // namespace

size_t page_attn_workspace_bytes(const Geom& g, int64_t T) { return paged::workspace_bytes<Fp16Pages>(g, T); }

hipError_t launch_page_attn(const Geom& g, const Pages& pg, const PageAttnArgs& a, void* ws, hipStream_t st) { return paged::launch<Fp16Pages>(g, pg, a, ws, st); }

}  // namespace antkv
