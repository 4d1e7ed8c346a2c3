// Rows of K and V into the pages of a cache, and out of them.
//
// A page holds `size` tokens of every KV head, [n_pages][Hkv][size][D]: the rows of one head lie together, so that 32 keys of a
// head are 8 KB in one piece (or two, of 16 tokens), which is the tile that attention moves.
//
// Both are copies: 16 bytes per lane, 16 lanes to a row, K and V by the same thread.  A thread has its loads of kRows rows in
// flight before it stores.  Bound: HBM, store 32768 tokens of 8 heads 55 us (4.85 TB/s read and written), load 4 x 32712 204 us
// (5.26 TB/s); few rows: a launch and two dependent loads (64 tokens 2.8 us, 4099 6.4 us).
#include "common.h"

namespace antkv {

namespace {

constexpr int kThreads = 256;
constexpr int kLanes = kD * 2 / 16;                                 // lanes of a row
constexpr int kRows = 2;                                            // rows of a thread
constexpr int kSpan = kThreads / kLanes * kRows;                    // rows of a workgroup
constexpr int kMostRows = 65535;                                    // of workgroups, the second axis of a grid

// row of slot `slot`, head g, in 16-byte pieces
__device__ __forceinline__ int64_t page_row(int64_t page, int off, int g, int Hkv, int shift)
{
    return ((((page * Hkv + g) << shift) + off)) * kLanes;
}

__global__ __launch_bounds__(kThreads) void page_store_kernel(const uint4_t* __restrict__ k, const uint4_t* __restrict__ v, int64_t xs_t,
                                                              int64_t xs_h, int64_t n_rows, const int32_t* __restrict__ slot, int64_t n_slots,
                                                              int Hkv, int shift, uint4_t* __restrict__ k_pages, uint4_t* __restrict__ v_pages)
{
    const int lane = threadIdx.x % kLanes;
    const int64_t row0 = (int64_t)blockIdx.x * kSpan + threadIdx.x / kLanes;      // rows: heads of a token one after the other
    uint4_t a[kRows], b[kRows];
    int64_t to[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int64_t row = row0 + i * (kThreads / kLanes);
        to[i] = -1;
        if (row < n_rows) {
            const int64_t t = row / Hkv;
            const int g = (int)(row - t * Hkv);
            const int64_t from = t * xs_t + g * xs_h + lane;
            a[i] = k[from];
            b[i] = v[from];
            const int64_t s = slot[t];
            if (s >= 0 && s < n_slots) to[i] = page_row(s >> shift, (int)(s & ((1 << shift) - 1)), g, Hkv, shift) + lane;
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        if (to[i] >= 0) {
            k_pages[to[i]] = a[i];
            v_pages[to[i]] = b[i];
        }
}

__global__ __launch_bounds__(kThreads) void page_load_kernel(const uint4_t* __restrict__ k_pages, const uint4_t* __restrict__ v_pages, int64_t n_pages,
                                                             int shift, const int32_t* __restrict__ table, int64_t table_cap,
                                                             const int32_t* __restrict__ ctx_len, int64_t first, int64_t N, int B, int Hkv,
                                                             uint4_t* __restrict__ k, uint4_t* __restrict__ v, int64_t xs_b, int64_t xs_h,
                                                             int64_t xs_t)
{
    const int lane = threadIdx.x % kLanes;
    for (int pair = blockIdx.y; pair < B * Hkv; pair += gridDim.y) {
        const int b = pair / Hkv, g = pair % Hkv;
        int64_t end = first + N;
        if (ctx_len && ctx_len[b] < end) end = ctx_len[b];
        const int64_t to = b * xs_b + g * xs_h + lane;
        for (int64_t t0 = (int64_t)blockIdx.x * kSpan + threadIdx.x / kLanes; t0 < N; t0 += (int64_t)gridDim.x * kSpan) {
            uint4_t x[kRows], y[kRows];
            bool have[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int64_t pos = first + t0 + i * (kThreads / kLanes);
                have[i] = false;
                if (pos < end) {
                    const int64_t page = table[b * table_cap + (pos >> shift)];
                    if (page >= 0 && page < n_pages) {
                        const int64_t from = page_row(page, (int)(pos & ((1 << shift) - 1)), g, Hkv, shift) + lane;
                        x[i] = k_pages[from];
                        y[i] = v_pages[from];
                        have[i] = true;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kRows; ++i)
                if (have[i]) {
                    const int64_t at = to + (t0 + i * (kThreads / kLanes)) * xs_t;
                    k[at] = x[i];
                    v[at] = y[i];
                }
        }
    }
}

}  // namespace

hipError_t launch_page_store(int Hkv, const Pages& pg, const half_t* k, const half_t* v, int64_t xs_t, int64_t xs_h, int64_t T,
                             const int32_t* slot, half_t* k_pages, half_t* v_pages, hipStream_t st)
{
    const int64_t rows = T * Hkv, grid = (rows + kSpan - 1) / kSpan;
    hipLaunchKernelGGL(page_store_kernel, dim3((unsigned)grid), dim3(kThreads), 0, st, (const uint4_t*)k, (const uint4_t*)v, xs_t / 8, xs_h / 8, rows,
                       slot, pg.n << pg.shift, Hkv, pg.shift, (uint4_t*)k_pages, (uint4_t*)v_pages);
    return hipGetLastError();
}

hipError_t launch_page_load(int B, int Hkv, const Pages& pg, const half_t* k_pages, const half_t* v_pages, const int32_t* table, int64_t table_cap,
                            const int32_t* ctx_len, int64_t first, int64_t N, half_t* k, half_t* v, int64_t xs_b, int64_t xs_h, int64_t xs_t,
                            hipStream_t st)
{
    int64_t blocks = (N + kSpan - 1) / kSpan;
    if (blocks > 1 << 20) blocks = 1 << 20;
    const int pairs = B * Hkv < kMostRows ? B * Hkv : kMostRows;
    hipLaunchKernelGGL(page_load_kernel, dim3((unsigned)blocks, (unsigned)pairs), dim3(kThreads), 0, st, (const uint4_t*)k_pages,
                       (const uint4_t*)v_pages, pg.n, pg.shift, table, table_cap, ctx_len, first, N, B, Hkv, (uint4_t*)k, (uint4_t*)v, xs_b / 8, xs_h / 8,
                       xs_t / 8);
    return hipGetLastError();
}

}  // namespace antkv
