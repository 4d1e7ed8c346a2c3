// Rotary positions: pairs of channels turned by the position times a frequency.
//
//   y_a = amplitude (x_a cos - x_b sin),  y_b = amplitude (x_b cos + x_a sin),  angle = position x freqs[i]  (inverse: the negative angle)
//
// of pair i = 0 .. rot / 2 - 1: channels (2 i, 2 i + 1) in style 0, (i, i + rot / 2) in style 1; channels from rot on are copied.
//
// A workgroup takes a few tokens with all of their heads.  A wave works out a token's 64 angles, one to a lane: the product with the position
// and its reduction to a turn in fp64 (far positions turn thousands of times: fp32 would leave an error of 0.01 at 10^5), then sine and cosine
// in fp32, and leaves them in LDS.  A thread turns 16 channels (eight pairs) of a head: 32 bytes in, 32 out, fp32 in between, rounded once.
// Bound: HBM in long batches (32768 tokens of 40 heads 119 us, 5.7 TB/s read and written); in short ones (64 tokens of 64 requests 3.8 us a call in a captured
// loop, 4.4 in a trace) the launch and five loads one behind the other: the search of q_start, the request's two starts, its length, the frequency and, behind
// the barrier, the rows.  The frequency and the rows need none of the others.
#include "common.h"

namespace antkv {

namespace {

constexpr int kThreads = 256;
constexpr int kUnits = kD / 16;                                     // threads of a head's row
constexpr int kPass = kThreads / kUnits;                            // rows of a pass
constexpr int kTokens = 32;                                         // of a workgroup, at most
constexpr int64_t kCaches = 32LL << 20;                             // bytes of the eight L2s
constexpr int kMostGroups = 1 << 20;
constexpr double kTurn = 0.15915494309189533576888376337251;        // 1 / (2 pi)

// The request whose rows hold row t: the last r < R with q_start[r] <= t (64 looked at at a time)
__device__ __forceinline__ int request_at(const int32_t* q_start, int R, int64_t t, int lane)
{
    int lo = 0, n = R;
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        const bool here = lane == 0 || (at < n && q_start[lo + (at < n ? at : 0)] <= t);
        const int c = __builtin_popcountll(__ballot(here)) - 1;
        lo += c * step;
        n = n - c * step < step ? n - c * step : step;
    }
    return lo;
}

template <bool kStream>                                             // the output goes past the caches
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeArgs p, int tokens, int64_t groups)
{
    __shared__ float2_t s_turn[kTokens][kD / 2];                    // cosine, sine
    __shared__ int s_live[kTokens];                                 // somebody's row
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int H = p.Hq + p.Hkv, unit = tid % kUnits, pairs = p.rot / 2;
    const int half = p.rot / 16;                                    // 16-byte pieces between the channels of a pair, style 1
    // the unit's two 16-byte pieces
    const bool turns = 16 * unit < p.rot;
    const int a = p.style == 1 && turns ? unit : 2 * unit, b = p.style == 1 && turns ? unit + half : 2 * unit + 1;
    const int rows = tokens * H;
    for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
        const int64_t first = group * tokens;                       // token of all B x T
        if (group != blockIdx.x) __syncthreads();
        for (int i = wave; i < tokens; i += kThreads / 64) {
            const int64_t u = first + i;
            bool live = u < p.B * p.T;
            int64_t pos = 0;
            if (live && p.q_start) {
                const int r = request_at(p.q_start, p.R, u, lane);
                const int64_t from = p.q_start[r], end = p.q_start[r + 1];
                live = u >= from && u < end;
                pos = p.ctx_len[r] - end + u;
            } else if (live) {
                pos = p.pos ? p.pos[u] : p.pos0 + (p.B > 1 ? (int64_t)((uint32_t)u % (uint32_t)p.T) : u);
            }
            if (live && lane < pairs) {
                const double turn = (double)pos * p.freqs[lane] * kTurn;
                float s, c;
                sincospif(2.f * (float)(turn - rint(turn)), &s, &c);
                s_turn[i][lane] = float2_t{c * p.amplitude, s * (p.inverse ? -p.amplitude : p.amplitude)};
            }
            if (lane == 0) s_live[i] = live;
        }
        __syncthreads();
        for (int row = tid / kUnits; row < rows; row += kPass) {
            const int i = row / H, h = row - i * H;
            uint4_t x, y;
            uint4_t* to = nullptr;
            if (first + i < p.B * p.T) {                            // asked for before it is known whether the row is somebody's
                // (values are selected: a selected address is loaded through, a chain of its own in front of the row, 32768 tokens 119 -> 127 us)
                const uint32_t u = (uint32_t)(first + i), n = p.B > 1 ? u / (uint32_t)p.T : 0, t = u - n * (uint32_t)p.T;
                const bool of_q = h < p.Hq;
                const int hh = of_q ? h : h - p.Hq;
                const half_t* from_rows = of_q ? p.q.x : p.k.x;
                half_t* to_rows = of_q ? p.q.y : p.k.y;
                const int64_t xs_b = of_q ? p.q.xs_b : p.k.xs_b, xs_t = of_q ? p.q.xs_t : p.k.xs_t, xs_h = of_q ? p.q.xs_h : p.k.xs_h;
                const int64_t ys_b = of_q ? p.q.ys_b : p.k.ys_b, ys_t = of_q ? p.q.ys_t : p.k.ys_t, ys_h = of_q ? p.q.ys_h : p.k.ys_h;
                const uint4_t* from = (const uint4_t*)(from_rows + n * xs_b + t * xs_t + hh * xs_h);
                to = (uint4_t*)(to_rows + n * ys_b + t * ys_t + hh * ys_h);
                x = from[a];
                y = from[b];
            }
            if (!to || !s_live[i]) continue;
            if (turns) {
                const float4_t* cs = (const float4_t*)&s_turn[i][8 * unit];
                float c[8], s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    c[e] = cs[e >> 1][2 * (e & 1)];
                    s[e] = cs[e >> 1][2 * (e & 1) + 1];
                }
                half8_t u = __builtin_bit_cast(half8_t, x), w = __builtin_bit_cast(half8_t, y), yu, yw;
                if (p.style == 1) {                                 // pair e: channel e of either piece
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        yu[e] = (half_t)((float)u[e] * c[e] - (float)w[e] * s[e]);
                        yw[e] = (half_t)((float)w[e] * c[e] + (float)u[e] * s[e]);
                    }
                } else {                                            // pair e: channels 2 e, 2 e + 1 of the sixteen
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        yu[2 * e] = (half_t)((float)u[2 * e] * c[e] - (float)u[2 * e + 1] * s[e]);
                        yu[2 * e + 1] = (half_t)((float)u[2 * e + 1] * c[e] + (float)u[2 * e] * s[e]);
                        yw[2 * e] = (half_t)((float)w[2 * e] * c[4 + e] - (float)w[2 * e + 1] * s[4 + e]);
                        yw[2 * e + 1] = (half_t)((float)w[2 * e + 1] * c[4 + e] + (float)w[2 * e] * s[4 + e]);
                    }
                }
                x = __builtin_bit_cast(uint4_t, yu);
                y = __builtin_bit_cast(uint4_t, yw);
            }
            if (kStream) {
                __builtin_nontemporal_store(x, to + a);
                __builtin_nontemporal_store(y, to + b);
            } else {
                to[a] = x;
                to[b] = y;
            }
        }
    }
}

__global__ void rope_freqs_kernel(int rot, double base, double factor, double trained, double slow, double fast, double* freqs)
{
    const int i = threadIdx.x;
    if (i >= rot / 2) return;
    const double f = pow(base, -2.0 * i / rot);
    double w = 0.0;                                                 // share of the frequency that stays
    if (trained > 0.0) {
        w = (trained * f * kTurn - slow) / (fast - slow);
        w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
    }
    freqs[i] = f * (w + (1.0 - w) / factor);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, hipStream_t st)
{
    const int H = a.Hq + a.Hkv;
    const int64_t all = a.B * a.T;
    // A workgroup's tokens: those of one pass, fewer where that leaves CUs without a workgroup.  One, two and four rows of a thread in flight, 32768
    // tokens of 40 heads 124, 125 and 129 us, of 8 heads 32, 34 and 37; workgroups of twice the size, one row, 157 and 35; loads ahead of the angles (more
    // registers, fewer waves) 147 and 37 (not tried on short batches alone, where no waves are missing).
    int tokens = kPass / H;
    tokens = tokens < 1 ? 1 : tokens < kTokens ? tokens : kTokens;
    while (tokens > 1 && all / tokens < 1024) tokens /= 2;
    const int64_t groups = (all + tokens - 1) / tokens;
    // More than the L2s hold goes past them: 32768 tokens 124 us through them and 118 past them, of 8 heads 32 and 22.
    const auto kernel = all * H * (kD * 2) > kCaches ? rope_kernel<true> : rope_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(groups < kMostGroups ? groups : kMostGroups)), dim3(kThreads), 0, st, a, tokens, groups);
    return hipGetLastError();
}

hipError_t launch_rope_freqs(int rot, double base, double factor, double trained, double slow, double fast, double* freqs, hipStream_t st)
{
    hipLaunchKernelGGL(rope_freqs_kernel, dim3(1), dim3(kD / 2), 0, st, rot, base, factor, trained, slow, fast, freqs);
    return hipGetLastError();
}

}  // namespace antkv
