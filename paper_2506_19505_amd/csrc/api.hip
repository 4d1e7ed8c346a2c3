// extern "C" boundary of the AnTKV library: argument validation, workspace layout, kernel launches.
#include "common.h"

#include <mutex>

using namespace antkv;

namespace {

constexpr int64_t kMostPairs = 65535;                   // B * Hkv: the second axis of a grid
constexpr int64_t kMostPagedPairs = 1LL << 20;          // of the calls on pages: 8192 requests of 128 KV heads

int check_geom(const antkv_geom* gm, Geom& g, int64_t most_pairs = kMostPairs)
{
    if (!gm) return ANTKV_EINVAL;
    if (gm->B < 0 || gm->Hq <= 0 || gm->Hkv <= 0 || gm->D <= 0 || gm->d_sub <= 0 || gm->n_centroids <= 0)
        return ANTKV_EINVAL;
    if (gm->Hq % gm->Hkv != 0) return ANTKV_EINVAL;
    if (gm->D != kD) return ANTKV_EUNSUPPORTED;
    const bool wide = gm->n_centroids == 4096 && (gm->d_sub == 32 || gm->d_sub == 16);   // 12-bit codes
    const bool byte_codes = gm->n_centroids == kC && (gm->d_sub == 4 || gm->d_sub == 8 || gm->d_sub == 16);
    if (!wide && !byte_codes) return ANTKV_EUNSUPPORTED;
    const int G = gm->Hq / gm->Hkv;
    if (G != 1 && G != 2 && G != 4) return ANTKV_EUNSUPPORTED;
    if ((int64_t)gm->B * gm->Hkv > most_pairs) return ANTKV_EUNSUPPORTED;
    g.B = gm->B; g.Hq = gm->Hq; g.Hkv = gm->Hkv; g.G = G; g.d = gm->d_sub; g.M = kD / gm->d_sub;
    g.C = gm->n_centroids;
    g.code_bytes = wide ? 3 * g.M / 2 : g.M;
    return ANTKV_OK;
}

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// n_pages pages of page_size tokens; every slot number fits 32 bits
int check_pages(int64_t n_pages, int32_t page_size, Pages& pg)
{
    if (n_pages < 1 || page_size < 1) return ANTKV_EINVAL;
    if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0) return ANTKV_EUNSUPPORTED;
    if (n_pages > 0x7fffffffLL / page_size) return ANTKV_EINVAL;
    pg.n = n_pages;
    pg.shift = __builtin_ctz((unsigned)page_size);
    return ANTKV_OK;
}
constexpr int64_t kMostBlocks = (1LL << 24) - 1;        // of 256 threads: a grid has fewer than 2^32 threads
// a block table of so many entries a row; positions stay below 2^30
inline bool bad_table(int64_t table_cap, const Pages& pg) { return table_cap < 1 || table_cap > (1LL << 30) >> pg.shift; }

// channels that turn: whole units of eight pairs
inline bool bad_rot(int32_t rot) { return rot < 16 || rot > kD || (rot & 15) != 0; }
// q or k of a call on rotary positions: 16-byte pieces; rows of the output do not overlap, in place means the same rows
bool bad_rope_rows(const RopeRows& z, int64_t B, int64_t T, int heads)
{
    const int64_t x[3] = {z.xs_b, z.xs_t, z.xs_h}, y[3] = {z.ys_b, z.ys_t, z.ys_h}, n[3] = {B, T, heads};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && ((x[i] & 7) || x[i] < 0 || (y[i] & 7) || y[i] < kD || (z.x == z.y && x[i] != y[i]))) return true;
    return misaligned(z.x, 16) || misaligned(z.y, 16);
}

struct SelPlan {
    size_t off_score, off_topk, total;
};

// room: what the call can use; otherwise what it does not refuse
SelPlan sel_plan(const Geom& g, int64_t N, int64_t Nq, int64_t k, bool room)
{
    SelPlan p;
    p.off_score = 0;
    p.off_topk = align_up(anchor_score_workspace_bytes(g, N, Nq, room));
    p.total = p.off_topk + align_up(topk_workspace_bytes(2 * (int64_t)g.B * g.Hkv, N, k));   // K and V rows in one go
    return p;
}

struct DecPlan {
    size_t off_dec, off_topk, total;
};

DecPlan dec_plan(const Geom& g, int64_t N, int64_t k_k, int64_t k_v, int64_t k_resel, bool want_ans)
{
    DecPlan p;
    p.off_dec = 0;
    p.off_topk = align_up(decode_workspace_bytes(g, N, k_k, k_v, want_ans));
    p.total = p.off_topk + (k_resel > 0 ? align_up(topk_workspace_bytes(2 * (int64_t)g.B * g.Hkv, N, k_resel)) : 0);
    return p;
}

int decode_attn_impl(const antkv_geom* geom, const void* q, float scale, const uint8_t* codes_k,
                      const uint8_t* codes_v, int64_t N, int64_t N_cap, const void* cb_k, const void* cb_v,
                      const int32_t* idx_k, const void* rows_k, int64_t k_k, const int32_t* idx_v, const void* rows_v,
                      int64_t k_v, void* out, float* ans_k, float* ans_v, int32_t* resel_idx_k, int32_t* resel_idx_v,
                      int64_t k_resel, void* workspace, size_t workspace_bytes, void* stream,
                      const float* given_scores = nullptr)
{
    Geom g;
    int rc = check_geom(geom, g);
    if (rc) return rc;
    if (N < 0 || N_cap < N || k_k < 0 || k_v < 0 || k_k > N || k_v > N || k_resel < 0 || k_resel > N ||
        N > 0x7fffffffLL)
        return ANTKV_EINVAL;
    const bool wide = g.C != kC;                                 // 12-bit codes
    if (g.B == 0) return ANTKV_OK;
    if (!q || !out || misaligned(q, 16) || misaligned(out, 16)) return ANTKV_EINVAL;
    if (!(scale > 0.f)) return ANTKV_EINVAL;
    if (N > 0) {
        if (!codes_k || !codes_v || !cb_k || !cb_v) return ANTKV_EINVAL;
        if (misaligned(codes_k, 16) || misaligned(codes_v, 16) || misaligned(cb_k, 16) || misaligned(cb_v, 16))
            return ANTKV_EINVAL;
        if (k_k > 0 && (!idx_k || !rows_k || misaligned(rows_k, 16))) return ANTKV_EINVAL;
        if (k_v > 0 && (!idx_v || !rows_v || misaligned(rows_v, 16))) return ANTKV_EINVAL;
    }
    if ((resel_idx_k && !ans_k) || (resel_idx_v && !ans_v)) return ANTKV_EINVAL;
    const bool want_ans = ans_k || ans_v;
    if (want_ans && !(ans_k && ans_v)) return ANTKV_EINVAL;   // the two scores are produced together
    if (wide) {
        const size_t topk_bytes = k_resel > 0 ? align_up(topk_workspace_bytes(2 * (int64_t)g.B * g.Hkv, N, k_resel)) : 0;
        const size_t least = align_up(decode12_workspace_least(g, N)), best = align_up(decode12_workspace_bytes(g, N, k_v));
        if (!workspace || misaligned(workspace, 256) || workspace_bytes < least + topk_bytes) return ANTKV_EWORKSPACE;
        const size_t off_topk = workspace_bytes < best + topk_bytes ? least : best;
        hipStream_t st = (hipStream_t)stream;
        DecodeArgs a;
        a.q = (const half_t*)q; a.scale = scale; a.codes_k = codes_k; a.codes_v = codes_v; a.N = N; a.N_cap = N_cap;
        a.cb_k = (const half_t*)cb_k; a.cb_v = (const half_t*)cb_v; a.idx_k = idx_k; a.rows_k = (const half_t*)rows_k;
        a.k_k = k_k; a.idx_v = idx_v; a.rows_v = (const half_t*)rows_v; a.k_v = k_v; a.out = (half_t*)out;
        a.ans_k = ans_k; a.ans_v = ans_v;
        a.given_scores = given_scores;
        // with both index sets wanted, the score pass counts its scores into the selection's first histogram
        const bool fused = N > 0 && k_resel > 0 && resel_idx_k && resel_idx_v;
        a.topk = fused ? topk2_begin((int64_t)g.B * g.Hkv, N, (char*)workspace + off_topk) : TopkCounts{nullptr, 0};
        if (launch_decode12(g, a, workspace, off_topk, st) != hipSuccess) return ANTKV_ELAUNCH;
        if (N > 0 && k_resel > 0 && (resel_idx_k || resel_idx_v)) {
            char* w = (char*)workspace;
            const int64_t rows = (int64_t)g.B * g.Hkv;
            const hipError_t e =
                (resel_idx_k && resel_idx_v)
                    ? launch_topk2_finish(ans_k, resel_idx_k, ans_v, resel_idx_v, rows, N, k_resel, w + off_topk, st)
                    : launch_topk(resel_idx_k ? ans_k : ans_v, rows, N, k_resel, resel_idx_k ? resel_idx_k : resel_idx_v,
                                  w + off_topk, st);
            if (e != hipSuccess) return ANTKV_ELAUNCH;
        }
        return ANTKV_OK;
    }
    const DecPlan dp = dec_plan(g, N, k_k, k_v, k_resel, true);
    if (N > 0 && (!workspace || misaligned(workspace, 256) || workspace_bytes < dp.total)) return ANTKV_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    DecodeArgs a;
    a.q = (const half_t*)q; a.scale = scale; a.codes_k = codes_k; a.codes_v = codes_v; a.N = N; a.N_cap = N_cap;
    a.cb_k = (const half_t*)cb_k; a.cb_v = (const half_t*)cb_v; a.idx_k = idx_k; a.rows_k = (const half_t*)rows_k;
    a.k_k = k_k; a.idx_v = idx_v; a.rows_v = (const half_t*)rows_v; a.k_v = k_v; a.out = (half_t*)out;
    a.ans_k = ans_k; a.ans_v = ans_v;
    a.given_scores = given_scores;
    // with both index sets wanted, the score pass counts its scores into the selection's first histogram
    const bool fused = N > 0 && k_resel > 0 && resel_idx_k && resel_idx_v;
    a.topk = fused ? topk2_begin((int64_t)g.B * g.Hkv, N, (char*)workspace + dp.off_topk) : TopkCounts{nullptr, 0};
    hipError_t e = launch_decode_attn(g, a, workspace, st);
    if (e != hipSuccess) return ANTKV_ELAUNCH;
    if (N > 0 && k_resel > 0) {
        char* w = (char*)workspace;
        const int64_t rows = (int64_t)g.B * g.Hkv;
        if (resel_idx_k && resel_idx_v) {
            e = launch_topk2_finish(ans_k, resel_idx_k, ans_v, resel_idx_v, rows, N, k_resel, w + dp.off_topk, st);
            if (e != hipSuccess) return ANTKV_ELAUNCH;
        } else if (resel_idx_k || resel_idx_v) {
            e = launch_topk(resel_idx_k ? ans_k : ans_v, rows, N, k_resel, resel_idx_k ? resel_idx_k : resel_idx_v,
                            w + dp.off_topk, st);
            if (e != hipSuccess) return ANTKV_ELAUNCH;
        }
    }
    return ANTKV_OK;
}


// ---- scratch of the entry point that takes no workspace --------------------------------------------------------
// One array per GPU, held from the moment the library is loaded on it until the process ends.  Host code never
// uses the array's name as an address: the device address is asked for once per device and kept.
static __device__ __align__(256) unsigned char scratch[ANTKV_STATIC_SCRATCH_BYTES];
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

int static_scratch(void** out)
{
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return ANTKV_ELAUNCH;
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch_ptr[dev]) {
        void* ptr = nullptr;
        if (hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch)) != hipSuccess || !ptr) return ANTKV_ELAUNCH;
        g_scratch_ptr[dev] = ptr;
    }
    *out = g_scratch_ptr[dev];
    return ANTKV_OK;
}

}  // namespace

extern "C" {

int antkv_version(void) { return 1; }

const char* antkv_strerror(int code)
{
    switch (code) {
    case ANTKV_OK: return "ok";
    case ANTKV_EINVAL: return "invalid argument";
    case ANTKV_EUNSUPPORTED: return "unsupported geometry";
    case ANTKV_EWORKSPACE: return "workspace missing or too small";
    case ANTKV_ELAUNCH: return "HIP launch failed";
    default: return "unknown error";
    }
}

int antkv_encode(const antkv_geom* geom, const void* x, int64_t xs_b, int64_t xs_h, int64_t xs_t, int64_t n_tok,
                 const void* codebook, uint8_t* codes, int64_t N_cap, int64_t token_offset, void* stream)
{
    Geom g;
    int rc = check_geom(geom, g);
    if (rc) return rc;
    if (n_tok < 0 || N_cap < 0 || token_offset < 0 || token_offset + n_tok > N_cap) return ANTKV_EINVAL;
    if (n_tok == 0 || g.B == 0) return ANTKV_OK;
    if (!x || !codebook || !codes) return ANTKV_EINVAL;
    if (misaligned(x, 16) || misaligned(codebook, 16) || misaligned(codes, 16)) return ANTKV_EINVAL;
    if (xs_t < kD || (xs_b & 7) || (xs_h & 7) || (xs_t & 7) || xs_b < 0 || xs_h < 0) return ANTKV_EINVAL;
    const hipError_t e =
        g.C == 4096 ? launch_encode12(g, (const half_t*)x, xs_b, xs_h, xs_t, n_tok, (const half_t*)codebook, codes, N_cap,
                                      token_offset, (hipStream_t)stream)
                    : launch_encode(g, (const half_t*)x, xs_b, xs_h, xs_t, n_tok, (const half_t*)codebook, codes, N_cap,
                                    token_offset, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

size_t antkv_topk_workspace(int64_t n_rows, int64_t N, int64_t k)
{
    if (n_rows < 0 || N < 0 || k < 0) return 0;
    return topk_workspace_bytes(n_rows, N, k);
}

int antkv_topk(const float* scores, int64_t n_rows, int64_t N, int64_t k, int32_t* idx, void* workspace,
               size_t workspace_bytes, void* stream)
{
    if (n_rows < 0 || N < 0 || k < 0 || k > N || N > 0x7fffffffLL || n_rows > 65535) return ANTKV_EINVAL;
    if (k == 0 || n_rows == 0) return ANTKV_OK;
    if (!scores || !idx) return ANTKV_EINVAL;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < topk_workspace_bytes(n_rows, N, k))
        return ANTKV_EWORKSPACE;
    hipError_t e = launch_topk(scores, n_rows, N, k, idx, workspace, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

size_t antkv_anchor_select_workspace(const antkv_geom* geom, int64_t N, int64_t Nq, int64_t k)
{
    Geom g;
    if (check_geom(geom, g) || N <= 0 || Nq <= 0 || Nq > N || k < 0) return 0;
    return sel_plan(g, N, Nq, k, true).total;
}

size_t antkv_kmeans_step_workspace(const antkv_geom* geom)
{
    Geom g;
    if (check_geom(geom, g)) return 0;
    return kmeans_workspace_bytes(g);
}

int antkv_kmeans_step(const antkv_geom* geom, const void* x, const float* w, int64_t n_tok, const void* codebook_in,
                      void* codebook_out, uint8_t* codes, float* wsum, double* objective, void* workspace,
                      size_t workspace_bytes, void* stream)
{
    Geom g;
    int rc = check_geom(geom, g);
    if (rc) return rc;
    if (n_tok < 0 || n_tok > 0x7fffffffLL) return ANTKV_EINVAL;
    if (!codebook_in || !codebook_out || codebook_in == codebook_out) return ANTKV_EINVAL;
    if (misaligned(codebook_in, 16) || misaligned(codebook_out, 16) || misaligned(objective, 8)) return ANTKV_EINVAL;
    const bool have_tokens = n_tok > 0 && g.B > 0;
    if (have_tokens && (!x || !w || !codes || misaligned(x, 16) || misaligned(codes, 16) || misaligned(w, 4)))
        return ANTKV_EINVAL;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < kmeans_workspace_bytes(g)) return ANTKV_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    if (have_tokens) {
        const hipError_t e =
            g.C == kC ? launch_encode(g, (const half_t*)x, (int64_t)g.Hkv * n_tok * kD, n_tok * kD, kD, n_tok,
                                      (const half_t*)codebook_in, codes, n_tok, 0, st, kmeans_clear(g, n_tok, workspace))
                      : launch_encode12(g, (const half_t*)x, (int64_t)g.Hkv * n_tok * kD, n_tok * kD, kD, n_tok,
                                        (const half_t*)codebook_in, codes, n_tok, 0, st);
        if (e != hipSuccess) return ANTKV_ELAUNCH;
    }
    const hipError_t e = launch_kmeans_update(g, (const half_t*)x, w, have_tokens ? n_tok : 0, (const half_t*)codebook_in,
                                              (half_t*)codebook_out, codes, wsum, objective, workspace, st);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_prefill_attn(const antkv_geom* geom, const void* q, const void* k, const void* v, int64_t N, int64_t Nq,
                       float scale, void* out, float* row_max, float* row_sum, void* stream)
{
    Geom g;
    int rc = check_geom(geom, g);
    if (rc) return rc;
    if (N <= 0 || Nq <= 0 || Nq > N || N > 0x7fffffffLL) return ANTKV_EINVAL;
    if ((row_max == nullptr) != (row_sum == nullptr)) return ANTKV_EINVAL;
    if (g.B == 0) return ANTKV_OK;
    if (!q || !k || !v || !out) return ANTKV_EINVAL;
    if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16)) return ANTKV_EINVAL;
    if (!(scale > 0.f)) return ANTKV_EINVAL;
    const hipError_t e = launch_prefill_attn(g, (const half_t*)q, (const half_t*)k, (const half_t*)v, N, Nq, scale,
                                             (half_t*)out, row_max, row_sum, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_prefill_attn_window(const antkv_geom* geom, const void* q, const void* k, const void* v, int64_t N, int64_t Nq, float scale,
                              int64_t window, int64_t n_sink, void* out, float* row_max, float* row_sum, void* stream)
{
    Geom g;
    const int rc = check_geom(geom, g);
    if (rc) return rc;
    if (N <= 0 || Nq <= 0 || Nq > N || N > 1LL << 30 || window < 1 || n_sink < 0) return ANTKV_EINVAL;
    if (Nq * g.G > 0x7fffffffLL || (Nq * g.G + 127) / 128 * g.B * g.Hkv > kMostBlocks) return ANTKV_EINVAL;
    if ((row_max == nullptr) != (row_sum == nullptr)) return ANTKV_EINVAL;
    if (g.B == 0) return ANTKV_OK;
    if (!q || !k || !v || !out) return ANTKV_EINVAL;
    if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16)) return ANTKV_EINVAL;
    if (!(scale > 0.f)) return ANTKV_EINVAL;
    const hipError_t e = launch_prefill_attn_window(g, (const half_t*)q, (const half_t*)k, (const half_t*)v, N, Nq, scale,
                                                    (int)(window < N ? window : N), (int)(n_sink < N ? n_sink : N), (half_t*)out, row_max,
                                                    row_sum, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_page_map(int64_t R, const int32_t* held_len, const int32_t* new_len, int32_t* table, int64_t table_cap, int64_t n_pages,
                   int32_t page_size, const int32_t* free_pages, int64_t n_free, const int32_t* free_at, int64_t T, int32_t* ctx_len,
                   int32_t* q_start, int32_t* slot, int32_t* status, void* stream)
{
    Pages pg;
    const int rc = check_pages(n_pages, page_size, pg);
    if (rc) return rc;
    if (R < 0 || bad_table(table_cap, pg) || n_free < 0 || n_free > 0x7fffffffLL || T < 0 || T > 0x7fffffffLL) return ANTKV_EINVAL;
    if (R > kMapRequests) return ANTKV_EUNSUPPORTED;
    if (!q_start || !status || status == free_at || (T > 0 && !slot) || (n_free > 0 && !free_pages)) return ANTKV_EINVAL;
    if (R > 0 && (!held_len || !new_len || !table || !ctx_len || ctx_len == held_len || ctx_len == new_len)) return ANTKV_EINVAL;
    const hipError_t e = launch_page_map(pg, (int)R, held_len, new_len, table, table_cap, free_pages, n_free, free_at, T, ctx_len, q_start, slot,
                                         status, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_page_store(const antkv_geom* geom, const void* k, const void* v, int64_t xs_t, int64_t xs_h, int64_t T, const int32_t* slot,
                     void* k_pages, void* v_pages, int64_t n_pages, int32_t page_size, void* stream)
{
    Geom g;
    int rc = check_geom(geom, g, kMostPagedPairs);
    if (rc) return rc;
    Pages pg;
    rc = check_pages(n_pages, page_size, pg);
    if (rc) return rc;
    if (T < 0 || T > kMostBlocks * 32 / g.Hkv) return ANTKV_EINVAL;      // (a workgroup has 32 rows)
    if (T == 0) return ANTKV_OK;
    if (!k || !v || !slot || !k_pages || !v_pages || k_pages == v_pages) return ANTKV_EINVAL;
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_pages, 16) || misaligned(v_pages, 16)) return ANTKV_EINVAL;
    if ((xs_t & 7) || (xs_h & 7) || xs_t < 0 || xs_h < 0) return ANTKV_EINVAL;
    const hipError_t e = launch_page_store(g.Hkv, pg, (const half_t*)k, (const half_t*)v, xs_t, xs_h, T, slot, (half_t*)k_pages, (half_t*)v_pages,
                                           (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_page_load(const antkv_geom* geom, const void* k_pages, const void* v_pages, int64_t n_pages, int32_t page_size,
                    const int32_t* table, int64_t table_cap, const int32_t* ctx_len, int64_t first, int64_t N, void* k, void* v,
                    int64_t xs_b, int64_t xs_h, int64_t xs_t, void* stream)
{
    Geom g;
    int rc = check_geom(geom, g, kMostPagedPairs);
    if (rc) return rc;
    Pages pg;
    rc = check_pages(n_pages, page_size, pg);
    if (rc) return rc;
    if (bad_table(table_cap, pg) || first < 0 || N < 0 || first > table_cap << pg.shift || N > (table_cap << pg.shift) - first) return ANTKV_EINVAL;
    if (N == 0 || g.B == 0) return ANTKV_OK;
    if (!k_pages || !v_pages || !table || !k || !v || k == v) return ANTKV_EINVAL;
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_pages, 16) || misaligned(v_pages, 16)) return ANTKV_EINVAL;
    if (xs_t < kD || (xs_b & 7) || (xs_h & 7) || (xs_t & 7) || xs_b < 0 || xs_h < 0) return ANTKV_EINVAL;
    const hipError_t e = launch_page_load(g.B, g.Hkv, pg, (const half_t*)k_pages, (const half_t*)v_pages, table, table_cap, ctx_len, first, N,
                                          (half_t*)k, (half_t*)v, xs_b, xs_h, xs_t, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

size_t antkv_page_attn_workspace(const antkv_geom* geom, int64_t T)
{
    Geom g;
    if (check_geom(geom, g, kMostPagedPairs) || g.B > kMapRequests || T < 1 || T > (1LL << 30) / g.Hq || g.B == 0) return 0;
    return page_attn_workspace_bytes(g, T);
}

size_t antkv_qpage_attn_workspace(const antkv_geom* geom, int64_t T)
{
    Geom g;
    if (check_geom(geom, g, kMostPagedPairs) || g.B > kMapRequests || T < 1 || T > (1LL << 30) / g.Hq || g.B == 0) return 0;
    return qpage_attn_workspace_bytes(g, T);
}

// scales: of pages of 8 bits, or none
static int page_attn_impl(const antkv_geom* geom, const void* q, int64_t qs_t, int64_t qs_h, int64_t T, const int32_t* q_start,
                          const int32_t* ctx_len, const int32_t* table, int64_t table_cap, const void* k_pages, const void* v_pages,
                          bool bytes, const float* k_scales, const float* v_scales, int64_t n_pages, int32_t page_size, float scale, int64_t window,
                          int64_t n_sink, void* out, float* row_max, float* row_sum, void* workspace, size_t workspace_bytes, void* stream)
{
    Geom g;
    int rc = check_geom(geom, g, kMostPagedPairs);
    if (rc) return rc;
    Pages pg;
    rc = check_pages(n_pages, page_size, pg);
    if (rc) return rc;
    if (g.B > kMapRequests) return ANTKV_EUNSUPPORTED;
    if (T < 0 || T > (1LL << 30) / g.Hq || bad_table(table_cap, pg) || window < 0 || window > 1LL << 30 || n_sink < 0) return ANTKV_EINVAL;
    if (n_pages * g.Hkv > 0x0fffffffLL / (page_size / 16)) return ANTKV_EINVAL;      // places of 16 rows: below 2^28, 1 TB
    if ((row_max == nullptr) != (row_sum == nullptr) || !(scale > 0.f)) return ANTKV_EINVAL;
    if (T == 0 || g.B == 0) return ANTKV_OK;
    if (!q || !q_start || !ctx_len || !table || !k_pages || !v_pages || !out || (bytes && (!k_scales || !v_scales))) return ANTKV_EINVAL;
    if (misaligned(q, 16) || misaligned(k_pages, 16) || misaligned(v_pages, 16) || misaligned(out, 16)) return ANTKV_EINVAL;
    if (bytes && (misaligned(k_scales, 4) || misaligned(v_scales, 4))) return ANTKV_EINVAL;
    if ((qs_t & 7) || (qs_h & 7) || qs_t < 0 || qs_h < 0) return ANTKV_EINVAL;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < (bytes ? qpage_attn_workspace_bytes(g, T) : page_attn_workspace_bytes(g, T))) return ANTKV_EWORKSPACE;
    PageAttnArgs a;
    a.q = (const half_t*)q; a.qs_t = qs_t; a.qs_h = qs_h; a.T = T; a.q_start = q_start; a.ctx_len = ctx_len; a.table = table;
    a.table_cap = table_cap; a.k_pages = (const half_t*)k_pages; a.v_pages = (const half_t*)v_pages; a.scale = scale;
    a.window = (int)window; a.n_sink = (int)(n_sink < 1LL << 30 ? n_sink : 1LL << 30);
    a.out = (half_t*)out; a.row_max = row_max; a.row_sum = row_sum;
    a.k_scales = k_scales; a.v_scales = v_scales;
    const hipError_t e = bytes ? launch_qpage_attn(g, pg, a, workspace, (hipStream_t)stream) : launch_page_attn(g, pg, a, workspace, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_page_attn(const antkv_geom* geom, const void* q, int64_t qs_t, int64_t qs_h, int64_t T, const int32_t* q_start,
                    const int32_t* ctx_len, const int32_t* table, int64_t table_cap, const void* k_pages, const void* v_pages,
                    int64_t n_pages, int32_t page_size, float scale, int64_t window, int64_t n_sink, void* out, float* row_max,
                    float* row_sum, void* workspace, size_t workspace_bytes, void* stream)
{
    return page_attn_impl(geom, q, qs_t, qs_h, T, q_start, ctx_len, table, table_cap, k_pages, v_pages, false, nullptr, nullptr, n_pages, page_size, scale,
                          window, n_sink, out, row_max, row_sum, workspace, workspace_bytes, stream);
}

int antkv_qpage_attn(const antkv_geom* geom, const void* q, int64_t qs_t, int64_t qs_h, int64_t T, const int32_t* q_start, const int32_t* ctx_len,
                     const int32_t* table, int64_t table_cap, const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales,
                     int64_t n_pages, int32_t page_size, float scale, int64_t window, int64_t n_sink, void* out, float* row_max, float* row_sum,
                     void* workspace, size_t workspace_bytes, void* stream)
{
    return page_attn_impl(geom, q, qs_t, qs_h, T, q_start, ctx_len, table, table_cap, k_pages, v_pages, true, k_scales, v_scales, n_pages, page_size, scale,
                          window, n_sink, out, row_max, row_sum, workspace, workspace_bytes, stream);
}

int antkv_rope_freqs(int32_t rot_dim, double base, double factor, double trained_len, double slow_turns, double fast_turns, double* freqs, void* stream)
{
    if (bad_rot(rot_dim)) return rot_dim < 2 || rot_dim > kD || (rot_dim & 1) ? ANTKV_EINVAL : ANTKV_EUNSUPPORTED;
    const double most = 1e30;
    if (!(base > 1.0 && base <= most) || !(factor > 0.0 && factor <= most) || !(trained_len >= 0.0 && trained_len <= most)) return ANTKV_EINVAL;
    if (trained_len > 0.0 && !(slow_turns >= 0.0 && fast_turns > slow_turns && fast_turns <= most)) return ANTKV_EINVAL;
    if (!freqs || misaligned(freqs, 8)) return ANTKV_EINVAL;
    const hipError_t e = launch_rope_freqs(rot_dim, base, factor, trained_len, slow_turns, fast_turns, freqs, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_rope(const antkv_geom* geom, const void* q, int64_t qs_b, int64_t qs_t, int64_t qs_h, const void* k, int64_t ks_b, int64_t ks_t, int64_t ks_h,
               int64_t T, const int32_t* pos, const int32_t* q_start, const int32_t* ctx_len, int64_t pos0, const double* freqs, int32_t rot_dim,
               int32_t rope_style, float amplitude, int32_t inverse, void* q_out, int64_t qo_b, int64_t qo_t, int64_t qo_h, void* k_out, int64_t ko_b,
               int64_t ko_t, int64_t ko_h, void* stream)
{
    Geom g;
    const int rc = check_geom(geom, g, kMostPagedPairs);
    if (rc) return rc;
    if (bad_rot(rot_dim)) return rot_dim < 2 || rot_dim > kD || (rot_dim & 1) ? ANTKV_EINVAL : ANTKV_EUNSUPPORTED;
    if (rope_style != 0 && rope_style != 1) return ANTKV_EINVAL;
    if ((q_start == nullptr) != (ctx_len == nullptr) || (q_start && pos) || pos0 < 0 || pos0 > 1LL << 40 || !(fabsf(amplitude) < INFINITY)) return ANTKV_EINVAL;
    if (q_start && g.B > kMapRequests) return ANTKV_EUNSUPPORTED;
    RopeArgs a;
    a.B = q_start ? 1 : g.B;
    a.R = g.B;
    if (T < 0 || T > 0x7fffffffLL || a.B * T > 0x7fffffffLL) return ANTKV_EINVAL;
    if (T == 0 || g.B == 0) return ANTKV_OK;
    if ((!q && !k) || (q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr) || !freqs || misaligned(freqs, 8)) return ANTKV_EINVAL;
    a.Hq = q ? g.Hq : 0;
    a.Hkv = k ? g.Hkv : 0;
    a.q = {(const half_t*)q, (half_t*)q_out, qs_b, qs_t, qs_h, qo_b, qo_t, qo_h};
    a.k = {(const half_t*)k, (half_t*)k_out, ks_b, ks_t, ks_h, ko_b, ko_t, ko_h};
    if ((q && bad_rope_rows(a.q, a.B, T, g.Hq)) || (k && bad_rope_rows(a.k, a.B, T, g.Hkv)) || (q && k && (q_out == k_out || q_out == k || k_out == q)))
        return ANTKV_EINVAL;
    a.T = T;
    a.pos = pos; a.q_start = q_start; a.ctx_len = ctx_len; a.pos0 = pos0;
    a.freqs = freqs; a.rot = rot_dim; a.style = rope_style; a.inverse = inverse != 0; a.amplitude = amplitude;
    return launch_rope(a, (hipStream_t)stream) == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_qpage_store(const antkv_geom* geom, const void* k, const void* v, int64_t xs_t, int64_t xs_h, int64_t T, const int32_t* slot, void* k_pages,
                      void* v_pages, float* k_scales, float* v_scales, int64_t n_pages, int32_t page_size, void* stream)
{
    Geom g;
    int rc = check_geom(geom, g, kMostPagedPairs);
    if (rc) return rc;
    Pages pg;
    rc = check_pages(n_pages, page_size, pg);
    if (rc) return rc;
    if (T < 0 || T > 0x7fffffffLL || (T + 15) / 16 * ((g.Hkv + 3) / 4) > kMostBlocks) return ANTKV_EINVAL;      // (a workgroup has 16 rows of four heads)
    if (T == 0) return ANTKV_OK;
    if (!k || !v || !slot || !k_pages || !v_pages || k_pages == v_pages || !k_scales || !v_scales || k_scales == v_scales) return ANTKV_EINVAL;
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_pages, 16) || misaligned(v_pages, 16) || misaligned(k_scales, 4) || misaligned(v_scales, 4)) return ANTKV_EINVAL;
    if ((xs_t & 7) || (xs_h & 7) || xs_t < 0 || xs_h < 0) return ANTKV_EINVAL;
    const hipError_t e = launch_qpage_store(g.Hkv, pg, (const half_t*)k, (const half_t*)v, xs_t, xs_h, T, slot, (uint8_t*)k_pages, (uint8_t*)v_pages, k_scales,
                                            v_scales, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_qpage_load(const antkv_geom* geom, const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales, int64_t n_pages,
                     int32_t page_size, const int32_t* table, int64_t table_cap, const int32_t* ctx_len, int64_t first, int64_t N, void* k, void* v,
                     int64_t xs_b, int64_t xs_h, int64_t xs_t, int32_t clear, void* stream)
{
    Geom g;
    int rc = check_geom(geom, g, kMostPagedPairs);
    if (rc) return rc;
    Pages pg;
    rc = check_pages(n_pages, page_size, pg);
    if (rc) return rc;
    if (bad_table(table_cap, pg) || first < 0 || N < 0 || first > table_cap << pg.shift || N > (table_cap << pg.shift) - first) return ANTKV_EINVAL;
    if (N == 0 || g.B == 0) return ANTKV_OK;
    if (!k_pages || !v_pages || !k_scales || !v_scales || !table || !k || !v || k == v) return ANTKV_EINVAL;
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_pages, 16) || misaligned(v_pages, 16) || misaligned(k_scales, 4) || misaligned(v_scales, 4)) return ANTKV_EINVAL;
    if (xs_t < kD || (xs_b & 7) || (xs_h & 7) || (xs_t & 7) || xs_b < 0 || xs_h < 0) return ANTKV_EINVAL;
    const hipError_t e = launch_qpage_load(g.B, g.Hkv, pg, (const uint8_t*)k_pages, (const uint8_t*)v_pages, k_scales, v_scales, table, table_cap, ctx_len, first,
                                           N, (half_t*)k, (half_t*)v, xs_b, xs_h, xs_t, clear != 0, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_anchor_select(const antkv_geom* geom, const void* q, const void* k_fp16, int64_t N, int64_t Nq, float scale,
                        int64_t k, const float* row_max, const float* row_sum, float* ans_k, float* ans_v,
                        int32_t* idx_k, int32_t* idx_v, void* workspace, size_t workspace_bytes, void* stream)
{
    Geom g;
    int rc = check_geom(geom, g);
    if (rc) return rc;
    if (N <= 0 || Nq <= 0 || Nq > N || k < 0 || k > N || N > 0x7fffffffLL) return ANTKV_EINVAL;
    if ((row_max == nullptr) != (row_sum == nullptr)) return ANTKV_EINVAL;
    if (g.B == 0) return ANTKV_OK;
    if (!q || !k_fp16) return ANTKV_EINVAL;
    if (misaligned(q, 16) || misaligned(k_fp16, 16)) return ANTKV_EINVAL;
    if (!(scale > 0.f)) return ANTKV_EINVAL;
    const bool room = workspace_bytes >= sel_plan(g, N, Nq, k, true).total;
    const SelPlan sp = sel_plan(g, N, Nq, k, room);
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < sp.total) return ANTKV_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    char* w = (char*)workspace;
    // scores default to the tail of the score workspace
    const size_t as_bytes = anchor_score_workspace_bytes(g, N, Nq, room);
    const size_t score_bytes = align_up((size_t)g.B * g.Hkv * N * sizeof(float));
    float* sk = ans_k ? ans_k : (float*)(w + as_bytes - 2 * score_bytes);
    float* sv = ans_v ? ans_v : (float*)(w + as_bytes - score_bytes);
    hipError_t e = launch_anchor_score(g, (const half_t*)q, (const half_t*)k_fp16, N, Nq, scale, row_max, row_sum, sk, sv,
                                       w + sp.off_score, room, st);
    if (e != hipSuccess) return ANTKV_ELAUNCH;
    const int64_t rows = (int64_t)g.B * g.Hkv;
    if (idx_k && idx_v && k > 0) {
        e = launch_topk2(sk, idx_k, sv, idx_v, rows, N, k, w + sp.off_topk, st);
        if (e != hipSuccess) return ANTKV_ELAUNCH;
    } else if ((idx_k || idx_v) && k > 0) {
        e = launch_topk(idx_k ? sk : sv, rows, N, k, idx_k ? idx_k : idx_v, w + sp.off_topk, st);
        if (e != hipSuccess) return ANTKV_ELAUNCH;
    }
    return ANTKV_OK;
}

int antkv_gather_rows(const antkv_geom* geom, const void* x, int64_t N, const int32_t* idx, int64_t k, void* rows_out,
                      void* stream)
{
    Geom g;
    int rc = check_geom(geom, g);
    if (rc) return rc;
    if (N < 0 || k < 0 || k > N) return ANTKV_EINVAL;
    if (k == 0 || g.B == 0) return ANTKV_OK;
    if (!x || !idx || !rows_out || misaligned(x, 16) || misaligned(rows_out, 16)) return ANTKV_EINVAL;
    hipError_t e = launch_gather_rows(g, (const half_t*)x, N, idx, k, (half_t*)rows_out, (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

int antkv_append_token(const antkv_geom* geom, const void* k_new, const void* v_new, int64_t N, int64_t W,
                       const void* cb_k, const void* cb_v, uint8_t* codes_k, uint8_t* codes_v, int64_t N_cap,
                       int32_t* idx_k, void* rows_k, int64_t k_k, int32_t* idx_v, void* rows_v, int64_t k_v,
                       void* stream)
{
    Geom g;
    int rc = check_geom(geom, g);
    if (rc) return rc;
    if (N < 0 || W < 0 || W > N || N + 1 > N_cap || k_k < W || k_v < W) return ANTKV_EINVAL;
    if (W > 64) return ANTKV_EUNSUPPORTED;
    if (g.B == 0) return ANTKV_OK;
    if (!k_new || !v_new || !cb_k || !cb_v || !codes_k || !codes_v || misaligned(k_new, 16) || misaligned(v_new, 16) ||
        misaligned(cb_k, 16) || misaligned(cb_v, 16) || misaligned(codes_k, 16) || misaligned(codes_v, 16))
        return ANTKV_EINVAL;
    if (W > 0 && (!idx_k || !rows_k || !idx_v || !rows_v || misaligned(rows_k, 16) || misaligned(rows_v, 16)))
        return ANTKV_EINVAL;
    hipError_t e = launch_append(g, (const half_t*)k_new, (const half_t*)v_new, (const half_t*)cb_k, (const half_t*)cb_v,
                                 codes_k, codes_v, N_cap, idx_k, (half_t*)rows_k, k_k, idx_v, (half_t*)rows_v, k_v, N, (int)W,
                                 (hipStream_t)stream);
    return e == hipSuccess ? ANTKV_OK : ANTKV_ELAUNCH;
}

// least: what the call does not refuse; otherwise what it can use
static size_t decode_need(const antkv_geom* geom, int64_t N, int64_t k_k, int64_t k_v, int64_t k_resel, bool least)
{
    Geom g;
    if (check_geom(geom, g) || N < 0 || k_k < 0 || k_v < 0 || k_resel < 0) return 0;
    if (g.C != kC)
        return align_up(least ? decode12_workspace_least(g, N) : decode12_workspace_bytes(g, N, k_v)) +
               (k_resel > 0 ? align_up(topk_workspace_bytes(2 * (int64_t)g.B * g.Hkv, N, k_resel)) : 0);
    return dec_plan(g, N, k_k, k_v, k_resel, true).total;
}

size_t antkv_decode_attn_workspace(const antkv_geom* geom, int64_t N, int64_t k_k, int64_t k_v, int64_t k_resel)
{
    return decode_need(geom, N, k_k, k_v, k_resel, false);
}

int antkv_decode_attn(const antkv_geom* geom, const void* q, float scale, const uint8_t* codes_k,
                      const uint8_t* codes_v, int64_t N, int64_t N_cap, const void* cb_k, const void* cb_v,
                      const int32_t* idx_k, const void* rows_k, int64_t k_k, const int32_t* idx_v, const void* rows_v,
                      int64_t k_v, void* out, float* ans_k, float* ans_v, int32_t* resel_idx_k, int32_t* resel_idx_v,
                      int64_t k_resel, void* workspace, size_t workspace_bytes, void* stream)
{
    return decode_attn_impl(geom, q, scale, codes_k, codes_v, N, N_cap, cb_k, cb_v, idx_k, rows_k, k_k, idx_v, rows_v, k_v,
                            out, ans_k, ans_v, resel_idx_k, resel_idx_v, k_resel, workspace, workspace_bytes, stream);
}

int antkv_set_decode_options(int options) { return set_decode_options(options); }

// bytes of the K side's scores that the pre-RoPE path keeps in its workspace: 16 per token and KV head (one-byte codes:
// tokens rounded up to 64, the decode kernel reads whole tiles)
static size_t prerope_score_bytes(const Geom& g, int64_t N)
{
    const int64_t n = g.C == kC ? (N + 63) / 64 * 64 : N;
    return align_up((size_t)g.B * g.Hkv * (size_t)n * 16);
}

size_t antkv_decode_attn_prerope_workspace(const antkv_geom* geom, int64_t N, int64_t k_v)
{
    Geom g;
    if (check_geom(geom, g) || N < 0 || k_v < 0) return 0;
    return prerope_score_bytes(g, N) + align_up(antkv_decode_attn_workspace(geom, N, 0, k_v, 0));
}

int antkv_decode_attn_prerope(const antkv_geom* geom, const void* q, float scale, const uint8_t* codes_k,
                              const uint8_t* codes_v, int64_t N, int64_t N_cap, const void* cb_k, const void* cb_v,
                              const int32_t* idx_k, const void* rows_k, int64_t k_k, const int32_t* idx_v,
                              const void* rows_v, int64_t k_v, float rope_base, int rope_style, int64_t pos0, void* out,
                              void* workspace, size_t workspace_bytes, void* stream)
{
    Geom g;
    const int rc = check_geom(geom, g);
    if (rc) return rc;
    if (N < 0 || N_cap < N || k_k < 0 || k_v < 0 || k_k > N || k_v > N || N > 0x7fffffffLL) return ANTKV_EINVAL;
    if (!(rope_base > 1.f) || (rope_style != 0 && rope_style != 1) || pos0 < 0 || pos0 > (1LL << 40)) return ANTKV_EINVAL;
    if (g.B == 0) return ANTKV_OK;
    if (N == 0)   // nothing to rotate: the plain call writes the zeros
        return decode_attn_impl(geom, q, scale, codes_k, codes_v, 0, N_cap, cb_k, cb_v, nullptr, nullptr, 0, nullptr, nullptr, 0,
                                out, nullptr, nullptr, nullptr, nullptr, 0, workspace, workspace_bytes, stream);
    if (!codes_k || !cb_k || misaligned(codes_k, 16) || misaligned(cb_k, 16)) return ANTKV_EINVAL;
    if (k_k > 0 && (!idx_k || !rows_k || misaligned(rows_k, 16))) return ANTKV_EINVAL;
    if (!q || misaligned(q, 16) || !(scale > 0.f)) return ANTKV_EINVAL;
    const size_t need = prerope_score_bytes(g, N) + align_up(decode_need(geom, N, 0, k_v, 0, true));
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < need) return ANTKV_EWORKSPACE;
    // The rotated keys are never written out: a first pass leaves q . RoPE(K_eff) of every token and head (FP16 anchor
    // rows included) in the workspace, and the decode kernels take their scores from there instead of from a table.
    char* w = (char*)workspace;
    const size_t sc_b = prerope_score_bytes(g, N);
    if (launch_rope_scores(g, (const half_t*)q, scale, codes_k, N, N_cap, (const half_t*)cb_k, idx_k, (const half_t*)rows_k, k_k,
                           (double)rope_base, rope_style, pos0, (float*)w, (hipStream_t)stream) != hipSuccess)
        return ANTKV_ELAUNCH;
    return decode_attn_impl(geom, q, scale, codes_k, codes_v, N, N_cap, cb_k, cb_v, nullptr, nullptr, 0, idx_v, rows_v, k_v, out,
                            nullptr, nullptr, nullptr, nullptr, 0, w + sc_b, workspace_bytes - sc_b, stream, (const float*)w);
}

int antkv_decode_attn_static(const antkv_geom* geom, const void* q, float scale, const uint8_t* codes_k,
                             const uint8_t* codes_v, int64_t N, int64_t N_cap, const void* cb_k, const void* cb_v,
                             const int32_t* idx_k, const void* rows_k, int64_t k_k, const int32_t* idx_v,
                             const void* rows_v, int64_t k_v, void* out, void* stream)
{
    Geom g;
    const int rc = check_geom(geom, g);
    if (rc) return rc;
    if (N < 0 || k_k < 0 || k_v < 0) return ANTKV_EINVAL;
    const size_t need = decode_need(geom, N, k_k, k_v, 0, true);
    if (need > (size_t)ANTKV_STATIC_SCRATCH_BYTES) return ANTKV_EWORKSPACE;   // shape beyond the built-in scratch
    void* ws = nullptr;
    const int rs = static_scratch(&ws);
    if (rs) return rs;
    return decode_attn_impl(geom, q, scale, codes_k, codes_v, N, N_cap, cb_k, cb_v, idx_k, rows_k, k_k, idx_v, rows_v, k_v,
                            out, nullptr, nullptr, nullptr, nullptr, 0, ws, (size_t)ANTKV_STATIC_SCRATCH_BYTES, stream);
}

}  // extern "C"
