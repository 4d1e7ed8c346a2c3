// Rows of K and V into pages of 8 bits, and out of them (bytes.h has the numbers, page_rows.hip the pages).
//
// Storing.  The unit is a block of kScaleRows slots of a KV head, of K or of V: its rows lie within 16 rows of the batch, so a wave has them
// all, up to 16 x 128 values in its registers, 16 lanes to a row.  It takes their largest value, makes the scale and writes bytes.  A block of which
// the batch holds no first row goes on: its scale grows if it has to, and the rows that are there are rounded to the new one.  No two waves
// touch the same block: nothing is waited for and nothing is atomic.
// A wave looks at `span` rows of the batch for the first rows of blocks: 16 in long batches (about one block), 1 in short ones, where each row may
// be a request of its own.
// Bound: HBM in long batches, in short ones a chain of slot - rows and scale - bytes.
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

// Bits of the least scale from 2^-32 to 2^8 through which the fp16 value of bits `top` is at most 448 = 1.75 x 2^8
__device__ __forceinline__ uint32_t scale_bits(uint32_t top)
{
    const uint32_t x = __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(half_t, (uint16_t)top));
    const uint32_t s = ((x + 0x1fffffu) & 0x7f800000u) - (8u << 23);            // up from 1.75 on
    return x < kLeastScale + (8u << 23) ? kLeastScale : s < kMostScale ? s : kMostScale;
}

// Two fp16 values / scale as e4m3 in the low 16 bits; what is not finite is NaN, what is beyond `most` in size counts as that
__device__ __forceinline__ uint32_t bytes_of(uint32_t two, float inv, float most)
{
    const half2_t h = __builtin_bit_cast(half2_t, two);
    float a = (float)h[0] * inv, b = (float)h[1] * inv;
    a = fabsf(a) <= most ? a : (two & 0x7fffu) >= 0x7c00u ? NAN : copysignf(most, a);
    b = fabsf(b) <= most ? b : (two >> 16 & 0x7fffu) >= 0x7c00u ? NAN : copysignf(most, b);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
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
    int Hkv, shift, span, units;                                    // units: workgroups for the heads of K and V
};

__global__ __launch_bounds__(kThreads) void qpage_store_kernel(const StoreParams p)
{
    const int lane = threadIdx.x & 63, unit = blockIdx.x % p.units * kWavesOf + (threadIdx.x >> 6);
    if (unit >= 2 * p.Hkv) return;
    const int v = unit >= p.Hkv, g = v ? unit - p.Hkv : unit;
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
    const int row4 = lane >> 4, c = lane & 15;
    while (first) {
        const int l = __builtin_ctzll(first);
        first &= first - 1;
        const unsigned long long of_block = __ballot(block == __builtin_amdgcn_readlane(block, l));
        if (of_block >> (l - kNear) & ((1ull << kNear) - 1)) continue;              // (not its first row)
        const uint32_t rows = (uint32_t)(of_block >> l) & 0xffffu;                  // those of rows l .. l + 15 that are
        uint4_t x[4];
        int to[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = 4 * j + row4;
            to[j] = __shfl(at, l + i, 64);
            x[j] = uint4_t{0u, 0u, 0u, 0u};
            if (rows >> i & 1) x[j] = p.x[v][(t0 - kNear + l + i) * p.xs_t + g * p.xs_h + c];
            else to[j] = -1;
        }
        const int64_t slot0 = __builtin_amdgcn_readlane(at, l) & ~(kScaleRows - 1);            // of the block
        float* const scale_at = p.scales[v] + byte_row(slot0, g, p.Hkv, p.shift) / (kLanes * kScaleRows);
        const uint32_t there = __builtin_bit_cast(uint32_t, *scale_at);
        // which of the block's rows are new
        uint32_t fresh = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (to[j] >= 0) fresh |= 1u << (to[j] & (kScaleRows - 1));
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = max_of(top, without(x[j][e] & 0x7fff7fffu, not_finite(x[j][e])));
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) {
            top = max_of(top, __shfl_xor(top, off, 64));
            fresh |= __shfl_xor(fresh, off, 64);
        }
        const uint32_t need = scale_bits(max_of(top, top >> 16) & 0xffffu);
        uint32_t is = need;
        uint2_t* const pages = p.pages[v];
        if (!(fresh & 1)) {                                         // the block goes on
            const uint32_t was = there >= kLeastScale && there <= kMostScale && !(there & 0x7fffffu) ? there : kLeastScale;
            if (was >= need) is = was;
            else {
                const float down = __builtin_bit_cast(float, (127u << 23) - (need - was));     // was / need
                uint4_t* const held = (uint4_t*)(pages + byte_row(slot0, g, p.Hkv, p.shift));
                uint4_t b[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) b[j] = held[64 * j + lane];                        // row 8 j + lane / 8
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (!(fresh >> (8 * j + (lane >> 3)) & 1)) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint2_t h = halves_of(b[j][e], down);
                            b[j][e] = bytes_of(h[0], 1.f, 448.f) | bytes_of(h[1], 1.f, 448.f) << 16;
                        }
                        held[64 * j + lane] = b[j];
                    }
            }
        }
        const float inv = __builtin_bit_cast(float, (254u << 23) - is), most = is == kMostScale ? 240.f : 448.f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (to[j] >= 0)
                pages[byte_row(to[j], g, p.Hkv, p.shift) + c] = uint2_t{bytes_of(x[j][0], inv, most) | bytes_of(x[j][1], inv, most) << 16,
                                                                        bytes_of(x[j][2], inv, most) | bytes_of(x[j][3], inv, most) << 16};
        if (lane == 0) *scale_at = __builtin_bit_cast(float, is);
    }
}

__global__ __launch_bounds__(kThreads) void qpage_load_kernel(const uint2_t* __restrict__ k_pages, const uint2_t* __restrict__ v_pages,
                                                              const float* __restrict__ k_scales, const float* __restrict__ v_scales, int64_t n_pages,
                                                              int shift, const int32_t* __restrict__ table, int64_t table_cap,
                                                              const int32_t* __restrict__ ctx_len, int64_t first, int64_t N, int B, int Hkv,
                                                              half8_t* __restrict__ k, half8_t* __restrict__ v, int64_t xs_b, int64_t xs_h, int64_t xs_t)
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
                have[i] = false;
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

// Workgroups for the heads of K and V; rows of the batch that a wave looks at.
int units_of(int Hkv) { return (2 * Hkv + kWavesOf - 1) / kWavesOf; }
int span_of(int64_t T, int Hkv) { return T * units_of(Hkv) <= 4096 ? 1 : kScaleRows; }

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
                             int64_t xs_h, int64_t xs_t, hipStream_t st)
{
    int64_t blocks = (N + kSpan - 1) / kSpan;
    if (blocks > 1 << 20) blocks = 1 << 20;
    const int pairs = B * Hkv < kMostRows ? B * Hkv : kMostRows;
    hipLaunchKernelGGL(qpage_load_kernel, dim3((unsigned)blocks, (unsigned)pairs), dim3(kThreads), 0, st, (const uint2_t*)k_pages, (const uint2_t*)v_pages,
                       k_scales, v_scales, pg.n, pg.shift, table, table_cap, ctx_len, first, N, B, Hkv, (half8_t*)k, (half8_t*)v, xs_b / 8, xs_h / 8, xs_t / 8);
    return hipGetLastError();
}

}  // namespace antkv
