// Attention over a dense prompt in which a query sees a window of recent keys and a few first ones (span_attn.h): a workgroup per
// block of rows, longest first.
#include "span_attn.h"

namespace antkv {

namespace {

using namespace span;

// Matrix instructions bound it where windows are long, coming and going (the query rows, the first tiles, the last ones) where they are
// short.  Waves of a workgroup: four, so that a CU holds two and one computes while the other comes or goes; 8 and 4 measured, us, 32 heads:
// 8192 tokens, 8 KV heads, window 1024: 183 and 177 (129 GFLOP, 730 TFLOP/s; 174 on another card); 16384, window 4096: 1026 and 993 (969 TFLOP/s); 2 x 1531, 32 KV heads,
// window 256: 60 and 50; 4096, 32 KV heads, window 128: 67 and 56; 16384, window 16384: 2170 and 2123 (1036 TFLOP/s).
constexpr int NW = 4;

__global__ __launch_bounds__(NW * 64, 2) void window_attn_kernel(const Params p)
{
    __shared__ __attribute__((aligned(1024))) unsigned char s_kv[kRingBytes];
    __shared__ __attribute__((aligned(16))) Note s_notes[kNotes];
    __shared__ int s_odd;
    const int bgs = gridDim.x / p.q_blocks, bg = blockIdx.x % bgs;              // (heads fastest: 8 heads, one per XCD)
    Piece x;
    x.b = bg / p.Hkv;
    x.g = bg % p.Hkv;
    x.r = 0;
    x.rq = {0, p.Nq, p.N - p.Nq, p.N};
    x.row0 = (p.q_blocks - 1 - blockIdx.x / bgs) * 32 * NW;
    const int rows = p.Nq << p.gs, last_row = (x.row0 + 32 * NW < rows ? x.row0 + 32 * NW : rows) - 1;
    const Span span = span_of(x.rq.p0 + (x.row0 >> p.gs), x.rq.p0 + (last_row >> p.gs), p.N, p.window, p.n_sink);
    x.from = 0;
    x.to = span.n;
    Sums sums;
    sums.clear();
    wide_sums<NW, false>(sums, p, x, span, s_kv, &s_odd, s_notes);
    const int lane = threadIdx.x & 63, row = x.row0 + 32 * scalar(threadIdx.x >> 6) + (lane & 31);
    if (row < rows) write_row(p, sums, x.b, row >> p.gs, (x.g << p.gs) + (row & (p.G - 1)), lane >> 5);
}

}  // namespace

hipError_t launch_prefill_attn_window(const Geom& g, const half_t* q, const half_t* k, const half_t* v, int64_t N, int64_t Nq, float scale,
                                      int window, int n_sink, half_t* out, float* row_max, float* row_sum, hipStream_t st)
{
    Params p = {};
    p.q = q; p.k = k; p.v = v; p.out = out; p.row_max = row_max; p.row_sum = row_sum;
    p.qs_t = p.os_t = kD; p.qs_h = p.os_h = Nq * kD; p.qs_b = p.os_b = g.Hq * Nq * kD; p.st_h = Nq; p.st_b = g.Hq * Nq;
    p.c1 = scale * kLog2e; p.Hkv = g.Hkv; p.G = g.G; p.gs = log2_of(g.G); p.window = window; p.n_sink = n_sink;
    p.N = (int)N; p.Nq = (int)Nq;
    const int64_t pairs = (int64_t)g.B * g.Hkv, rows = Nq * g.G;
    p.q_blocks = (int)((rows + 32 * NW - 1) / (32 * NW));
    hipLaunchKernelGGL(window_attn_kernel, dim3((unsigned)(p.q_blocks * pairs)), dim3(NW * 64), 0, st, p);
    return hipGetLastError();
}

}  // namespace antkv
