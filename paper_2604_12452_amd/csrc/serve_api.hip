// Entry points of the serving operators (include/lca_serve.h): argument validation, workspace carving, dispatch.  The rules of
// lca_api.hip hold here too: no allocation, no synchronisation, no state beyond the thread's error message.
#include <algorithm>
#include <climits>
#include <cmath>

#include "api_checks.h"
#include "serve_internal.h"

namespace {

using lca::check_ptr;
using lca::fail;
using lca::FastDiv;
using lca::ServeDims;

enum { TABLES = 1, CACHE = 2 };           // what a call reads of the descriptor

lca_status make_dims(const lca_serve_desc *desc, int what, ServeDims &d)
{
    if (desc == nullptr) return fail(LCA_ERR_INVALID_ARG, "desc is NULL");
    if (desc->B <= 0 || desc->H <= 0 || desc->S <= 0) return fail(LCA_ERR_INVALID_ARG, "B, H, S must be positive");
    if (desc->T < 0) return fail(LCA_ERR_INVALID_ARG, "T must not be negative");
    if (desc->H % desc->S != 0) return fail(LCA_ERR_INVALID_ARG, "H (%d) must be a multiple of S (%d)", desc->H, desc->S);
    if ((long long)desc->T * desc->H >= (1ll << 30)) return fail(LCA_ERR_UNSUPPORTED, "T*H must be below 2^30");
    if (desc->B >= (1 << 24) || (long long)desc->B * desc->S >= (1ll << 24)) return fail(LCA_ERR_UNSUPPORTED, "B*S must be below 2^24");
    if (desc->dtype != LCA_BF16 && desc->dtype != LCA_F32 && desc->dtype != LCA_F16) return fail(LCA_ERR_INVALID_ARG, "unknown dtype %d", desc->dtype);
    if (desc->window < 0) return fail(LCA_ERR_INVALID_ARG, "window must be >= 0");
    if (desc->max_q < 0 || desc->max_kv < 0) return fail(LCA_ERR_INVALID_ARG, "max_q and max_kv must be >= 0");
    if (!std::isfinite(desc->scale)) return fail(LCA_ERR_INVALID_ARG, "scale is not a finite number");
    if (!std::isfinite(desc->softcap) || desc->softcap < 0.f) return fail(LCA_ERR_INVALID_ARG, "softcap must be a finite number >= 0");
    if (!lca::in_fp32(lca::score_rule(desc->scale, desc->softcap, desc->window)))
        return fail(LCA_ERR_INVALID_ARG, "scale (%g) and softcap (%g): the scores' factors leave fp32", (double)desc->scale, (double)desc->softcap);
    if (desc->softcap > lca::LARGEST_CAP && desc->dtype != LCA_F32)
        return fail(LCA_ERR_UNSUPPORTED, "softcap (%g) above %g is not supported for the 16-bit types", (double)desc->softcap, (double)lca::LARGEST_CAP);
    const int mult = desc->dtype == LCA_F32 ? 4 : 8;
    if (desc->d_pool <= 0 || desc->d_sel <= 0 || desc->d_pool % mult || desc->d_sel % mult)
        return fail(LCA_ERR_INVALID_ARG, "d_pool and d_sel must be positive multiples of %d", mult);
    if (desc->d_pool > 1024 || desc->d_sel > 1024) return fail(LCA_ERR_UNSUPPORTED, "d_pool and d_sel above 1024 are not supported");
    const int64_t rows[3] = {desc->q_row, desc->sel_row, desc->pool_row};
    const int64_t least[3] = {(int64_t)desc->H * desc->d_sel, (int64_t)desc->S * desc->d_sel, (int64_t)desc->S * desc->d_pool};
    size_t row[3];
    for (int i = 0; i < 3; ++i) {
        static const char *const names[3] = {"q_row", "sel_row", "pool_row"};
        if (rows[i] != 0 && (rows[i] < least[i] || rows[i] % mult != 0 || rows[i] >= ((int64_t)1 << 32)))
            return fail(LCA_ERR_INVALID_ARG, "%s (%lld) must be 0 or a multiple of %d from %lld to below 2^32", names[i], (long long)rows[i], mult, (long long)least[i]);
        row[i] = (size_t)(rows[i] != 0 ? rows[i] : least[i]);
    }
    d.B = desc->B; d.T = desc->T; d.H = desc->H; d.S = desc->S; d.hps = desc->H / desc->S;
    d.d_pool = desc->d_pool; d.d_sel = desc->d_sel; d.dtype = desc->dtype;
    d.page = desc->page; d.n_blocks = desc->n_blocks; d.max_blocks = desc->max_blocks;
    d.window = desc->window; d.scale = desc->scale; d.softcap = desc->softcap;
    d.q_row = row[0]; d.sel_row = row[1]; d.pool_row = row[2];
    if (what & (TABLES | CACHE)) {
        if (desc->page < 16 || desc->page > 1024 || desc->page % 16 != 0) return fail(LCA_ERR_INVALID_ARG, "page (%d) must be a multiple of 16 in [16, 1024]", desc->page);
        if (desc->n_blocks <= 0 || (long long)desc->n_blocks * desc->page >= (1ll << 31))
            return fail(LCA_ERR_INVALID_ARG, "n_blocks (%d) must be positive, n_blocks * page below 2^31", desc->n_blocks);
        if (desc->max_blocks <= 0 || (long long)desc->max_blocks * desc->page > (1ll << 30))
            return fail(LCA_ERR_INVALID_ARG, "max_blocks (%d) must be positive, max_blocks * page at most 2^30", desc->max_blocks);
    }
    if (what & CACHE) {
        if (desc->dtype == LCA_F32) return fail(LCA_ERR_UNSUPPORTED, "the 8-bit cache takes the 16-bit types");
        if (desc->d_pool % 16 || desc->d_sel % 16 || desc->d_pool > 256 || desc->d_sel > 256)
            return fail(LCA_ERR_UNSUPPORTED, "the 8-bit cache takes widths that are multiples of 16 up to 256");
    }
    d.by_hps = FastDiv(d.hps); d.by_S = FastDiv(d.S); d.by_page = FastDiv(d.page); d.by_strips = FastDiv(d.page / 16);
    const int capacity = (int)std::min<int64_t>(std::max<int64_t>((int64_t)desc->max_blocks * desc->page, 0), 1 << 30);
    d.max_q = desc->max_q == 0 || desc->max_q > desc->T ? desc->T : desc->max_q;
    d.max_kv = desc->max_kv == 0 || desc->max_kv > capacity ? capacity : desc->max_kv;
    return LCA_OK;
}

size_t round_up(size_t n) { return (n + 255) & ~(size_t)255; }

// Requests of few rows are split over their keys, those of many share tiles in LDS.  Where the hint says that there are none
// of the second kind only the first kernel runs, and takes what comes.
bool long_requests(const ServeDims &d) { return (long long)d.max_q * d.hps > lca::PAGE_DECODE_COLUMNS; }

size_t paged_bytes(const ServeDims &d)
{
    const size_t few = lca::page_decode_workspace_bytes(d), many = long_requests(d) ? lca::scored_tile_workspace_bytes(d, true) : 0;
    return round_up(std::max(few, many));                // (one kernel after the other)
}
size_t packed_bytes(const ServeDims &d) { return d.T > 0 && lca::scored_tile_supported(d) ? round_up(lca::scored_tile_workspace_bytes(d, false)) : 0; }
// (a descriptor that the cache calls refuse needs no workspace for them)
size_t attn_bytes(const lca_serve_desc *desc)
{
    ServeDims d;
    return make_dims(desc, CACHE, d) == LCA_OK && d.T > 0 ? paged_bytes(d) : 0;
}
size_t tables_bytes(const ServeDims &d) { return round_up((size_t)d.B * sizeof(int32_t)); }

lca_status check_i32(const void *p, const char *name, bool required = true)
{
    if (p == nullptr) return required ? fail(LCA_ERR_INVALID_ARG, "%s is NULL", name) : LCA_OK;
    if (reinterpret_cast<uintptr_t>(p) & 3) return fail(LCA_ERR_INVALID_ARG, "%s is not 4-byte aligned", name);
    return LCA_OK;
}

lca_status check_ws(size_t need, const void *ws, size_t ws_bytes)
{
    if (need == 0) return LCA_OK;
    if (ws == nullptr) return fail(LCA_ERR_WORKSPACE, "workspace is NULL, %zu bytes needed", need);
    LCA_TRY(check_ptr(ws, "workspace"));
    if (ws_bytes < need) return fail(LCA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
    return LCA_OK;
}

}  // namespace

extern "C" {

lca_status lca_serve_workspace_size(const lca_serve_desc *desc, size_t *bytes)
{
    ServeDims d;
    LCA_TRY(make_dims(desc, 0, d));
    if (bytes == nullptr) return fail(LCA_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = std::max({tables_bytes(d), packed_bytes(d), attn_bytes(desc)});
    return LCA_OK;
}

lca_status lca_page_tables(const lca_serve_desc *desc, const int32_t *cached_len, const int32_t *new_len, const int32_t *free_list, const int32_t *free_count,
                           int32_t *free_left, int32_t *block_table, int32_t *q_start, int32_t *seq_len, int32_t *slot, int32_t *position, int32_t *request,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    ServeDims d;
    LCA_TRY(make_dims(desc, TABLES, d));
    LCA_TRY(check_i32(cached_len, "cached_len"));
    LCA_TRY(check_i32(new_len, "new_len"));
    LCA_TRY(check_i32(free_list, "free_list"));
    LCA_TRY(check_i32(free_count, "free_count"));
    LCA_TRY(check_i32(free_left, "free_left"));
    LCA_TRY(check_i32(block_table, "block_table"));
    LCA_TRY(check_i32(q_start, "q_start"));
    LCA_TRY(check_i32(seq_len, "seq_len"));
    LCA_TRY(check_i32(slot, "slot", d.T > 0));
    LCA_TRY(check_i32(position, "position", d.T > 0));
    LCA_TRY(check_i32(request, "request", d.T > 0));
    LCA_TRY(check_ws(tables_bytes(d), workspace, workspace_bytes));
    const lca::TablesArgs a{d, cached_len, new_len, free_list, free_count, free_left, block_table, q_start, seq_len, slot, position, request,
                            static_cast<int32_t *>(workspace)};
    return LCA_LAUNCH(lca::launch_page_tables(a, static_cast<hipStream_t>(stream)), "lca_page_tables");
}

lca_status lca_page_release(const lca_serve_desc *desc, const int32_t *finished, int32_t *cached_len, int32_t *block_table, int32_t *free_list,
                            int32_t *free_count, void *stream)
{
    ServeDims d;
    LCA_TRY(make_dims(desc, TABLES, d));
    LCA_TRY(check_i32(finished, "finished"));
    LCA_TRY(check_i32(cached_len, "cached_len"));
    LCA_TRY(check_i32(block_table, "block_table"));
    LCA_TRY(check_i32(free_list, "free_list"));
    LCA_TRY(check_i32(free_count, "free_count"));
    const lca::ReleaseArgs a{d, finished, cached_len, block_table, free_list, free_count};
    return LCA_LAUNCH(lca::launch_page_release(a, static_cast<hipStream_t>(stream)), "lca_page_release");
}

lca_status lca_page_store_q8(const lca_serve_desc *desc, const void *SEL, const void *POOL, const int32_t *slot, uint8_t *sel_q8, uint8_t *pool_q8,
                             float *scales, void *stream)
{
    ServeDims d;
    LCA_TRY(make_dims(desc, CACHE, d));
    LCA_TRY(check_ptr(SEL, "SEL", d.T > 0));
    LCA_TRY(check_ptr(POOL, "POOL", d.T > 0));
    LCA_TRY(check_i32(slot, "slot", d.T > 0));
    LCA_TRY(check_ptr(sel_q8, "sel_q8"));
    LCA_TRY(check_ptr(pool_q8, "pool_q8"));
    LCA_TRY(check_i32(scales, "scales"));
    if (d.T == 0) return LCA_OK;
    const lca::StoreArgs a{d, SEL, POOL, slot, sel_q8, pool_q8, scales};
    return LCA_LAUNCH(lca::launch_page_store_q8(a, static_cast<hipStream_t>(stream)), "lca_page_store_q8");
}

lca_status lca_page_attn_q8(const lca_serve_desc *desc, const void *q, const int32_t *q_start, const int32_t *seq_len, const int32_t *prefix_len,
                            const float *slopes, const int32_t *block_table, const uint8_t *sel_q8, const uint8_t *pool_q8, const float *scales, void *O,
                            float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    ServeDims d;
    LCA_TRY(make_dims(desc, CACHE, d));
    LCA_TRY(check_ptr(q, "q", d.T > 0));
    LCA_TRY(check_i32(q_start, "q_start"));
    LCA_TRY(check_i32(seq_len, "seq_len"));
    LCA_TRY(check_i32(prefix_len, "prefix_len", false));
    LCA_TRY(check_i32(slopes, "slopes", false));
    LCA_TRY(check_i32(block_table, "block_table"));
    LCA_TRY(check_ptr(sel_q8, "sel_q8"));
    LCA_TRY(check_ptr(pool_q8, "pool_q8"));
    LCA_TRY(check_i32(scales, "scales"));
    LCA_TRY(check_ptr(O, "O", d.T > 0));
    LCA_TRY(check_i32(lse, "lse", false));
    if (d.T == 0) return LCA_OK;
    LCA_TRY(check_ws(paged_bytes(d), workspace, workspace_bytes));
    lca::ScoredArgs a{};
    a.d = d; a.Q = q; a.q_start = q_start; a.seq_len = seq_len; a.prefix_len = prefix_len; a.slopes = slopes; a.block_table = block_table;
    a.sel_q8 = sel_q8; a.pool_q8 = pool_q8; a.scales = scales; a.O = O; a.lse = lse; a.part = static_cast<float *>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    LCA_TRY(LCA_LAUNCH(lca::launch_page_decode(a, long_requests(d) ? lca::PAGE_DECODE_COLUMNS : INT_MAX, st), "lca_page_attn_q8"));
    return long_requests(d) ? LCA_LAUNCH(lca::launch_scored_tile_paged(a, lca::PAGE_DECODE_COLUMNS + 1, st), "lca_page_attn_q8") : LCA_OK;
}

lca_status lca_packed_attn(const lca_serve_desc *desc, const void *Q, const void *SEL, const void *POOL, const int32_t *doc_start,
                           const int32_t *prefix_len, const float *slopes, void *O, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    ServeDims d;
    LCA_TRY(make_dims(desc, 0, d));
    LCA_TRY(check_ptr(Q, "Q", d.T > 0));
    LCA_TRY(check_ptr(SEL, "SEL", d.T > 0));
    LCA_TRY(check_ptr(POOL, "POOL", d.T > 0));
    LCA_TRY(check_i32(doc_start, "doc_start"));
    LCA_TRY(check_i32(prefix_len, "prefix_len", false));
    LCA_TRY(check_i32(slopes, "slopes", false));
    LCA_TRY(check_ptr(O, "O", d.T > 0));
    LCA_TRY(check_i32(lse, "lse", false));
    if (d.T == 0) return LCA_OK;
    LCA_TRY(check_ws(packed_bytes(d), workspace, workspace_bytes));
    lca::ScoredArgs a{};
    a.d = d; a.Q = Q; a.SEL = SEL; a.POOL = POOL; a.q_start = doc_start; a.prefix_len = prefix_len; a.slopes = slopes; a.O = O; a.lse = lse;
    a.part = static_cast<float *>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (lca::scored_tile_supported(d)) return LCA_LAUNCH(lca::launch_scored_tile(a, st), "lca_packed_attn");
    return LCA_LAUNCH(lca::launch_scored_rows(a, st), "lca_packed_attn");
}

}  // extern "C"
