// Block tables and slot maps of a step, from the lengths of its requests.
//
// Two prefix sums over the requests say everything: of the new tokens (where a request's rows start in the packed batch) and of
// the pages it takes (where its pages start in the list of free ones).  Every workgroup makes both for itself (8 bytes a request,
// out of the L2) and keeps them in LDS, with the lengths; it then writes its share of the slots, and of the new table entries.  A
// slot in a new page comes from the free list, one in a page held before from an entry that no thread writes: one launch, nothing
// to wait for between workgroups.
// Bound: latency, a launch and two dependent loads (256 requests of a token each 4.3 us, 48 prompts of 65536 tokens 5.0).
#include "common.h"

namespace antkv {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int64_t kMost = 0x7fffffffLL;

struct MapParams {
    const int32_t *held, *fresh, *free_pages, *free_at;
    int32_t *table, *ctx_len, *q_start, *slot, *status;
    int64_t table_cap, n_pages, n_free, T_cap;
    int R, shift;
};

// index of the last of the ascending s[0 .. n] that is <= x, given s[0] <= x < s[n]
__device__ __forceinline__ int last_at_most(const int* s, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// inclusive sum over the wave of 31-bit numbers, in halves that cannot overflow
__device__ __forceinline__ int64_t wave_scan31(int x) { return ((int64_t)wave_scan(x >> 16) << 16) + wave_scan(x & 0xffff); }

template <int kPer>                                     // slots of a thread: 4 where a request has many, which then are of one or two pages
__global__ __launch_bounds__(kThreads) void page_map_kernel(const MapParams p)
{
    extern __shared__ int s_pre[];                                  // [R + 1] first tokens, [R + 1] first pages of the free list, [R] lengths
    __shared__ int64_t s_wave[2][kWaves];
    __shared__ int s_short;
    int* s_tok = s_pre;
    int* s_page = s_pre + p.R + 1;
    int* s_held = s_page + p.R + 1;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t size = 1ll << p.shift;
    const int64_t at0 = p.free_at ? (*p.free_at > 0 ? *p.free_at : 0) : 0;
    if (tid == 0) s_short = 0;

    auto has = [&](int64_t h) { const int64_t n = (h + size - 1) >> p.shift; return n < p.table_cap ? n : p.table_cap; };
    int64_t run_tok = 0, run_page = 0;
    for (int base = 0; base < p.R; base += kThreads) {
        const int r = base + tid;
        int64_t n = 0, take = 0;
        if (r < p.R) {
            const int u = p.held[r], v = p.fresh[r], h = u > 0 ? u : 0;
            s_held[r] = h;
            n = v > 0 ? v : 0;
            take = has(h + n) - has(h);
        }
        int64_t a = wave_scan31((int)n), b = wave_scan31((int)take);
        if (lane == 63) { s_wave[0][wave] = a; s_wave[1][wave] = b; }
        __syncthreads();
        int64_t all_tok = 0, all_page = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) { a += s_wave[0][w]; b += s_wave[1][w]; }
            all_tok += s_wave[0][w];
            all_page += s_wave[1][w];
        }
        if (r < p.R) {
            const int64_t tok = run_tok + a - n, page = run_page + b - take;
            s_tok[r] = (int)(tok < kMost ? tok : kMost);
            s_page[r] = (int)(page < kMost ? page : kMost);
        }
        run_tok += all_tok;
        run_page += all_page;
        __syncthreads();
    }
    if (tid == 0) {
        s_tok[p.R] = (int)(run_tok < kMost ? run_tok : kMost);
        s_page[p.R] = (int)(run_page < kMost ? run_page : kMost);
    }
    __syncthreads();

    auto valid = [&](int64_t page) { return page >= 0 && page < p.n_pages; };
    auto from_list = [&](int64_t i) -> int64_t {                    // entry i of what this call takes
        const int64_t at = at0 + i;
        if (at >= p.n_free) return -1;
        const int64_t page = p.free_pages[at];
        return valid(page) ? page : -1;
    };
    // page of index `pi` of request r, -1 if it has none
    auto page_of = [&](int r, int64_t h, int64_t pi) -> int64_t {
        if (pi >= p.table_cap) return -1;
        const int64_t old = has(h);
        if (pi >= old) return from_list(s_page[r] + (pi - old));
        const int64_t page = p.table[(int64_t)r * p.table_cap + pi];
        return valid(page) ? page : -1;
    };

    // slots
    const int total = s_tok[p.R];
    for (int64_t t = ((int64_t)blockIdx.x * kThreads + tid) * kPer; t < p.T_cap; t += (int64_t)gridDim.x * kThreads * kPer) {
        int out[kPer];
        int r = 0, next = 0;                                        // request of the last token, first token behind it
        int64_t h = 0, pi = -1, page = -1;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            out[i] = -1;
            if (t + i >= total) continue;
            if (i == 0 || t + i >= next) {
                r = last_at_most(s_tok, p.R, (int)(t + i));
                next = s_tok[r + 1];
                h = s_held[r];
                pi = -1;
            }
            const int64_t pos = h + (t + i - s_tok[r]);
            if (pos >> p.shift != pi) {
                pi = pos >> p.shift;
                page = page_of(r, h, pi);
            }
            if (page >= 0) out[i] = (int)((page << p.shift) + (pos & (size - 1)));
        }
        if (kPer == 4 && t + kPer <= p.T_cap && ((uintptr_t)p.slot & 15) == 0)
            *(int4_t*)(p.slot + t) = int4_t{out[0], out[1 % kPer], out[2 % kPer], out[3 % kPer]};
        else
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (t + i < p.T_cap) p.slot[t + i] = out[i];
    }
    // new table entries
    const int pages = s_page[p.R];
    for (int64_t i = (int64_t)blockIdx.x * kThreads + tid; i < pages; i += (int64_t)gridDim.x * kThreads) {
        const int r = last_at_most(s_page, p.R, (int)i);
        p.table[(int64_t)r * p.table_cap + has(s_held[r]) + (i - s_page[r])] = (int)from_list(i);
    }
    // lengths, starts, what is left
    if (blockIdx.x != 0) return;
    int missing = 0;
    for (int r = tid; r < p.R; r += kThreads) {
        const int64_t h = s_held[r], n = p.fresh[r] > 0 ? p.fresh[r] : 0, ctx = h + n;
        p.ctx_len[r] = (int)(ctx < kMost ? ctx : kMost);
        p.q_start[r] = s_tok[r];
        if (n > 0) {
            const int64_t take = has(ctx) - has(h);
            bool room = s_tok[r] + n <= p.T_cap && ctx <= p.table_cap << p.shift && (take == 0 || at0 + s_page[r] + take <= p.n_free);
            if (room && (h & (size - 1)) != 0) room = page_of(r, h, h >> p.shift) >= 0;
            missing += !room;
        }
    }
    if (tid == 0) p.q_start[p.R] = total;
    if (missing) atomicAdd(&s_short, missing);
    __syncthreads();
    if (tid == 0) {
        const int64_t left = at0 + pages;
        p.status[0] = (int)(left < p.n_free ? left : p.n_free);
        p.status[1] = s_short;
    }
}

}  // namespace

hipError_t launch_page_map(const Pages& pg, int R, const int32_t* held, const int32_t* fresh, int32_t* table, int64_t table_cap,
                           const int32_t* free_pages, int64_t n_free, const int32_t* free_at, int64_t T_cap, int32_t* ctx_len, int32_t* q_start,
                           int32_t* slot, int32_t* status, hipStream_t st)
{
    MapParams p;
    p.held = held; p.fresh = fresh; p.free_pages = free_pages; p.free_at = free_at;
    p.table = table; p.ctx_len = ctx_len; p.q_start = q_start; p.slot = slot; p.status = status;
    p.table_cap = table_cap; p.n_pages = pg.n; p.n_free = n_free; p.T_cap = T_cap; p.R = R; p.shift = pg.shift;
    auto launch = [&](const void* at, auto kernel, int per, OncePerDevice& once) {
        int64_t blocks = (T_cap + kThreads * per - 1) / (kThreads * per);
        if (blocks < 1) blocks = 1;
        if (blocks > 1024) blocks = 1024;
        const size_t lds = (3 * (size_t)R + 2) * sizeof(int);
        if (lds > 60 * 1024) {
            const hipError_t e = allow_lds(once, at, (3 * (size_t)kMapRequests + 2) * sizeof(int));
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), lds, st, p);
        return hipGetLastError();
    };
    static OncePerDevice once1, once4;
    return T_cap >= 8 * (int64_t)R ? launch((const void*)page_map_kernel<4>, page_map_kernel<4>, 4, once4)
                                   : launch((const void*)page_map_kernel<1>, page_map_kernel<1>, 1, once1);
}

}  // namespace antkv
