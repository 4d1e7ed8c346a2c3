// Rows of K and V into pages of 8 bits, and out of them (bytes.h has the numbers, page_rows.hip the pages).
//
// Storing.  The unit is a block of kScaleRows slots of a KV head: its rows lie within 16 rows of the batch, so a wave has them all, up to 16 x 128
// values of K and of V in its registers, 16 lanes to a row.  It takes their largest value, makes the scale and writes bytes.  A block of which
// the batch holds no first row goes on: its scale grows if it has to, and the rows that are there are rounded to the new one.  No two waves
// touch the same block: nothing is waited for and nothing is atomic.
// A wave looks at `span` rows of the batch for the first rows of blocks: 16 in long batches (about one block), 1 in short ones, where each row may
// be a request of its own.
// Bound: HBM in long batches (32768 tokens of 8 heads 42.5 us, 4.7 TB/s read and written); in short ones (64 tokens of 64 requests 4.0 us a call in a captured loop,
// 4.5 in a trace) a chain: slots, rows, then K's scale (behind the rows' largest value, and only where the block goes on) and K's bytes, then V's scale and bytes.
//
// Loading is a copy: 8 bytes in, 16 out per lane, 16 lanes to a row, K and V by the same thread.  Bound: HBM.
#include "bytes.h"

namespace antkv {

namespace {

constexpr int kThreads = 256, kWavesOf = kThreads / 64;
constexpr int kLanes = 16;                                          // of a row
constexpr int kRows = 2;                                            // of a thread, loading
constexpr int kSpan = kThreads / kLanes * kRows;                    // of a workgroup, loading
constexpr int kMostRows = 65535;                                    // of workgroups, the second axis of a grid

// row of slot `slot`, head g, in 16 x 8 bytes
__device__ __forceinline__ int64_t byte_row(int64_t slot, int g, int Hkv, int shift)
{
    return ((((slot >> shift) * Hkv + g) << shift) + (slot & ((1 << shift) - 1))) * kLanes;
}

__device__ __forceinline__ uint32_t scalar(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }      // of a value that is the same in every lane

// Bits of the least scale from 2^-32 to 2^8 through which the fp16 value of bits `top` is at most 448 = 1.75 x 2^8
__device__ __forceinline__ uint32_t scale_bits(uint32_t top)
{
    const uint32_t x = __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(half_t, (uint16_t)top));
    const uint32_t s = ((x + 0x1fffffu) & 0x7f800000u) - (8u << 23);            // up from 1.75 on
    return x < kLeastScale + (8u << 23) ? kLeastScale : s < kMostScale ? s : kMostScale;
}

// Four fp16 values / scale as e4m3, what is not finite as NaN; no other is beyond 448 scale in size
__device__ __forceinline__ uint32_t bytes_of(uint2_t four, float scale)
{
    const uint32_t lo = four[0], hi = four[1];                      // (a bit cast of a vector's element takes the first one)
    short2_t r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(half2_t, lo), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(half2_t, hi), scale, true);
    return __builtin_bit_cast(uint32_t, r);
}
// sizes beyond 61440 (0x7b80) as that, infinities and NaN as they are
__device__ __forceinline__ uint32_t within(uint32_t two)
{
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t x = two >> (16 * e) & 0xffffu, size = x & 0x7fffu;
        r |= (size > 0x7b80u && size < 0x7c00u ? (x & 0x8000u) | 0x7b80u : x) << (16 * e);
    }
    return r;
}

typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b)              // of two 16-bit numbers each
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2_t, a), __builtin_bit_cast(ushort2_t, b)));
}

struct StoreParams {
    const uint4_t* x[2];                                            // K, V
    int64_t xs_t, xs_h, T, n_slots;                                 // strides in 16 bytes
    const int32_t* slot;
    uint2_t* pages[2];
    float* scales[2];
    int Hkv, shift, span, units;                                    // units: workgroups for all heads
};

// of 16 lanes, by rotations, then of the four sixteens
template <int kBy>
__device__ __forceinline__ uint32_t rotated(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + kBy, 0xf, 0xf, false); }
__device__ __forceinline__ uint32_t wave_top(uint32_t m)
{
    m = max_of(m, rotated<8>(m));
    m = max_of(m, rotated<4>(m));
    m = max_of(m, rotated<2>(m));
    m = max_of(m, rotated<1>(m));
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = __builtin_amdgcn_readlane(m, 16 * i), a = two & 0xffffu, b = two >> 16, most = a > b ? a : b;
        top = top > most ? top : most;
    }
    return top;
}

__global__ __launch_bounds__(kThreads) void qpage_store_kernel(const StoreParams p)
{
    const int lane = threadIdx.x & 63, g = blockIdx.x % p.units * kWavesOf + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (g >= p.Hkv) return;
    const int64_t t0 = (int64_t)(blockIdx.x / p.units) * p.span;
    // lane l: row t0 - 15 + l and its block
    constexpr int kNear = kScaleRows - 1;                           // rows before, and behind, a row that may be of the same block
    const int64_t t = t0 - kNear + lane;
    int at = -1;
    if (t >= 0 && t < p.T && lane < p.span + 2 * kNear) at = p.slot[t];
    if (at >= p.n_slots) at = -1;
    const int block = at < 0 ? -1 : at / kScaleRows;
    const bool goes_on = lane > 0 && block == __shfl_up(block, 1, 64);
    unsigned long long first = __ballot(lane >= kNear && lane < kNear + p.span && block >= 0 && !goes_on);
    const unsigned long long starts = __ballot(at >= 0 && (at & (kScaleRows - 1)) == 0);
    const int row4 = lane >> 4, c = lane & 15;
    while (first) {
        const int l = __builtin_ctzll(first);
        first &= first - 1;
        const unsigned long long of_block = __ballot(block == __builtin_amdgcn_readlane(block, l));
        if (of_block >> (l - kNear) & ((1ull << kNear) - 1)) continue;              // (not its first row)
        const uint32_t rows = (uint32_t)(of_block >> l) & 0xffffu;                  // those of rows l .. l + 15 that are
        const bool anew = (of_block & starts) >> l & 0xffffu;
        uint4_t x[2][4];
        const int64_t from = (t0 - kNear + l + row4) * p.xs_t + g * p.xs_h + c;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                x[v][j] = uint4_t{0u, 0u, 0u, 0u};
                if (rows >> (4 * j + row4) & 1) x[v][j] = p.x[v][from + 4 * j * p.xs_t];
            }
        const int64_t slot0 = __builtin_amdgcn_readlane(at, l) & ~(kScaleRows - 1), base = byte_row(slot0, g, p.Hkv, p.shift);     // of the block
        int to[4];                                                  // places in the block, of 8 bytes
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = (__shfl(at, l + 4 * j + row4, 64) & (kScaleRows - 1)) * kLanes + c;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) m = max_of(m, x[v][j][e] & 0x7fff7fffu);
            uint32_t top = wave_top(m);
            if (__builtin_expect(top >= 0x7c00u, 0)) {              // of what is finite
                m = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) m = max_of(m, without(x[v][j][e] & 0x7fff7fffu, not_finite(x[v][j][e])));
                top = wave_top(m);
            }
            uint32_t is = scale_bits(top);
            float* const scale_at = p.scales[v] + base / (kLanes * kScaleRows);
            uint2_t* const block_at = p.pages[v] + base;
            if (!anew) {                                            // the block goes on
                uint32_t was = scalar(__builtin_bit_cast(uint32_t, *scale_at));
                if (was < kLeastScale || was > kMostScale || (was & 0x7fffffu)) was = kLeastScale;
                if (was >= is) is = was;
                else {
                    const float grows = __builtin_bit_cast(float, (127u << 23) + (is - was));
                    uint32_t fresh = 0;                             // which of the block's rows are new
                    for (int i = 0; i < kScaleRows; ++i)
                        if (rows >> i & 1) fresh |= 1u << (__builtin_amdgcn_readlane(at, l + i) & (kScaleRows - 1));
                    uint4_t* const held = (uint4_t*)block_at;
                    uint4_t b[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) b[j] = held[64 * j + lane];                    // row 8 j + lane / 8
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (!(fresh >> (8 * j + (lane >> 3)) & 1)) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) b[j][e] = bytes_of(halves_of(b[j][e], 1.f), grows);
                            held[64 * j + lane] = b[j];
                        }
                }
            }
            if (__builtin_expect(is == kMostScale, 0)) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[v][j][e] = within(x[v][j][e]);
            }
            const float scale = __builtin_bit_cast(float, is);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (rows >> (4 * j + row4) & 1)
                    block_at[to[j]] = uint2_t{bytes_of(uint2_t{x[v][j][0], x[v][j][1]}, scale), bytes_of(uint2_t{x[v][j][2], x[v][j][3]}, scale)};
            if (lane == 0) *scale_at = scale;
        }
    }
}

__global__ __launch_bounds__(kThreads) void qpage_load_kernel(const uint2_t* __restrict__ k_pages, const uint2_t* __restrict__ v_pages,
                                                              const float* __restrict__ k_scales, const float* __restrict__ v_scales, int64_t n_pages,
                                                              int shift, const int32_t* __restrict__ table, int64_t table_cap,
                                                              const int32_t* __restrict__ ctx_len, int64_t first, int64_t N, int B, int Hkv,
                                                              half8_t* __restrict__ k, half8_t* __restrict__ v, int64_t xs_b, int64_t xs_h, int64_t xs_t, int clear)
{
    const int lane = threadIdx.x % kLanes;
    for (int pair = blockIdx.y; pair < B * Hkv; pair += gridDim.y) {
        const int b = pair / Hkv, g = pair % Hkv;
        int64_t end = first + N;
        if (ctx_len && ctx_len[b] < end) end = ctx_len[b];
        const int64_t to = b * xs_b + g * xs_h + lane;
        for (int64_t t0 = (int64_t)blockIdx.x * kSpan + threadIdx.x / kLanes; t0 < N; t0 += (int64_t)gridDim.x * kSpan) {
            uint2_t x[kRows], y[kRows];
            float ks[kRows], vs[kRows];
            bool have[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int64_t pos = first + t0 + i * (kThreads / kLanes);
                have[i] = clear && t0 + i * (kThreads / kLanes) < N;           // a row of zeros, as far as is known
                x[i] = y[i] = uint2_t{0u, 0u};
                ks[i] = vs[i] = 1.f;
                if (pos < end) {
                    const int64_t page = table[b * table_cap + (pos >> shift)];
                    if (page >= 0 && page < n_pages) {
                        const int64_t from = byte_row((page << shift) + (pos & ((1 << shift) - 1)), g, Hkv, shift) + lane;
                        x[i] = k_pages[from];
                        y[i] = v_pages[from];
                        ks[i] = k_scales[from / (kLanes * kScaleRows)];
                        vs[i] = v_scales[from / (kLanes * kScaleRows)];
                        have[i] = true;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kRows; ++i)
                if (have[i]) {
                    const int64_t at = to + (t0 + i * (kThreads / kLanes)) * xs_t;
                    k[at] = halves_of(x[i], ks[i]);
                    v[at] = halves_of(y[i], vs[i]);
                }
        }
    }
}

// Workgroups for all heads; rows of the batch that a wave looks at.
int units_of(int Hkv) { return (Hkv + kWavesOf - 1) / kWavesOf; }
// A wave goes through its blocks one after the other, 1.6 us each: a step of single tokens has one for every row, a prompt one for 16.  Spans
// of 1, 2, 8 and 16, 8 heads, a prompt and as many requests of a token: 500 tokens 5.1, 4.6, 3.7, 5.1 us and 5.2, 6.2, 15, 27; 1024 8.6, 6.3, 5.6, 4.9
// and 7.8, 7.5, 15, 28; 2048 14, 9.6, 6.9, 5.7 and 13, 12, 17, 29; 4096 25, 16, 8.5, 7.6 and 23, 21, 22, 32; 32768 (a prompt) 246, 135, 49, 42.
// 32 heads: 128 tokens 4.6, 3.8, 5.0, 5.0 and 5.2, 6.2, 15, 28; 512 7.7, 6.6, 5.9, 5.8 and 13, 13, 18, 30; 1024 12.6, 10.5, 7.3, 7.9 and 23, 22, 22, 34; 4096 50, 44, 25,
// 20 and 90, 80, 82, 86; 32768 376, 324, 177, 154
int span_of(int64_t T, int Hkv)
{
    const int64_t n = T * units_of(Hkv);
    return n <= 1024 ? 1 : n <= 4096 ? 2 : n <= 8192 ? 8 : kScaleRows;
}

}  // namespace

hipError_t launch_qpage_store(int Hkv, const Pages& pg, const half_t* k, const half_t* v, int64_t xs_t, int64_t xs_h, int64_t T, const int32_t* slot,
                              uint8_t* k_pages, uint8_t* v_pages, float* k_scales, float* v_scales, hipStream_t st)
{
    StoreParams p;
    p.x[0] = (const uint4_t*)k; p.x[1] = (const uint4_t*)v; p.xs_t = xs_t / 8; p.xs_h = xs_h / 8; p.T = T; p.n_slots = pg.n << pg.shift; p.slot = slot;
    p.pages[0] = (uint2_t*)k_pages; p.pages[1] = (uint2_t*)v_pages; p.scales[0] = k_scales; p.scales[1] = v_scales; p.Hkv = Hkv; p.shift = pg.shift;
    p.span = span_of(T, Hkv);
    p.units = units_of(Hkv);
    hipLaunchKernelGGL(qpage_store_kernel, dim3((unsigned)((T + p.span - 1) / p.span * p.units)), dim3(kThreads), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_qpage_load(int B, int Hkv, const Pages& pg, const uint8_t* k_pages, const uint8_t* v_pages, const float* k_scales, const float* v_scales,
                             const int32_t* table, int64_t table_cap, const int32_t* ctx_len, int64_t first, int64_t N, half_t* k, half_t* v, int64_t xs_b,
                             int64_t xs_h, int64_t xs_t, bool clear, hipStream_t st)
{
    int64_t blocks = (N + kSpan - 1) / kSpan;
    if (blocks > 1 << 20) blocks = 1 << 20;
    const int pairs = B * Hkv < kMostRows ? B * Hkv : kMostRows;
    hipLaunchKernelGGL(qpage_load_kernel, dim3((unsigned)blocks, (unsigned)pairs), dim3(kThreads), 0, st, (const uint2_t*)k_pages, (const uint2_t*)v_pages,
                       k_scales, v_scales, pg.n, pg.shift, table, table_cap, ctx_len, first, N, B, Hkv, (half8_t*)k, (half8_t*)v, xs_b / 8, xs_h / 8, xs_t / 8, (int)clear);
    return hipGetLastError();
}

}  // namespace antkv
