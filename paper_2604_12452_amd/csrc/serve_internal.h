// Internal declarations of the serving operators (include/lca_serve.h): validated sizes, arguments, launchers, and the
// few device functions that their kernels share.
#pragma once
#include <cmath>

#include "lanes.h"
#include "lca_internal.h"
#include "lca_serve.h"

namespace lca {

// x / d for 0 <= x < 2^31 by one multiplication: with s = ceil(log2 d) and mul = ceil(2^(31 + s) / d), mul d exceeds 2^(31 + s)
// by less than d <= 2^s, which x < 2^31 keeps below one quotient.  (A division of the ALU's own is some thirty dependent
// instructions, and a short call has a dozen.)
struct FastDiv {
    unsigned mul, shift;                          // mul = 0: d = 1
    FastDiv() = default;
    explicit FastDiv(int d) : mul(0), shift(0)
    {
        if (d <= 1) return;
        unsigned s = 0;
        while ((1ull << s) < (unsigned long long)d) ++s;
        mul = (unsigned)(((1ull << (31 + s)) + d - 1) / d);
        shift = s - 1;
    }
    __device__ __forceinline__ int operator()(int x) const { return mul == 0 ? x : (int)(__umulhi((unsigned)x, mul) >> shift); }
};

// A validated lca_serve_desc; rows resolved, hints resolved (max_kv <= max_blocks * page, max_q <= T).
struct ServeDims {
    int B, T, H, S, hps, d_pool, d_sel, dtype;
    int page, n_blocks, max_blocks, max_q, max_kv, window;
    float scale, softcap;
    size_t q_row, sel_row, pool_row;
    FastDiv by_hps, by_S, by_page, by_strips;     // strips: page / 16
};

struct TablesArgs {
    ServeDims d;
    const int32_t *cached_len, *new_len, *free_list, *free_count;
    int32_t *free_left, *block_table, *q_start, *seq_len, *slot, *position, *request;
    int32_t *base;                 // workspace, [B]
};
hipError_t launch_page_tables(const TablesArgs &a, hipStream_t st);

struct ReleaseArgs {
    ServeDims d;
    const int32_t *finished;
    int32_t *cached_len, *block_table, *free_list, *free_count;
};
hipError_t launch_page_release(const ReleaseArgs &a, hipStream_t st);

struct StoreArgs {
    ServeDims d;
    const void *SEL, *POOL;
    const int32_t *slot;
    uint8_t *sel_q8, *pool_q8;
    float *scales;
};
hipError_t launch_page_store_q8(const StoreArgs &a, hipStream_t st);

// Both attention calls: packed (block_table == NULL: keys and values are SEL, POOL) or over the cache.
struct ScoredArgs {
    ServeDims d;
    const void *Q, *SEL, *POOL;
    const int32_t *q_start, *seq_len, *prefix_len, *block_table;
    const float *slopes;
    const uint8_t *sel_q8, *pool_q8;
    const float *scales;
    void *O;
    float *lse;
    float *part;                   // workspace: split partials
};
hipError_t launch_scored_rows(const ScoredArgs &a, hipStream_t st);

// Requests of up to this many (row, query head) pairs per KV head are page_decode.hip's, the others scored_tile.h's.  16 requests of 8000 tokens,
// 8 rows each, 128 / 128: 32 pairs 39 us in the first kernel and 142 in the second, 64 pairs 62 and 142; of 500 tokens 15 and 25.
constexpr int PAGE_DECODE_COLUMNS = 64;
size_t page_decode_workspace_bytes(const ServeDims &d);
// Requests of at most `most` pairs (the others are left alone).
hipError_t launch_page_decode(const ScoredArgs &a, int most, hipStream_t st);
// Many rows: packed prompts, and over the cache the requests of at least `least` pairs (scored_tile.h).
bool scored_tile_supported(const ServeDims &d);
size_t scored_tile_workspace_bytes(const ServeDims &d, bool paged);
hipError_t launch_scored_tile(const ScoredArgs &a, hipStream_t st);
hipError_t launch_scored_tile_paged(const ScoredArgs &a, int least, hipStream_t st);

// ---- device functions ----

constexpr float LOG2E = 1.4426950408889634f;

// The score rule in base 2: what the kernels need per call.  With a cap, cap * tanh(x) = cap - 2 cap / (1 + e^(2x)): two
// hardware instructions at a quarter rate, exact to a few 2^-24 of the cap, and its limits are right at infinities.  Small against the
// rounding of 16-bit weights while the cap is at most LARGEST_CAP (2^-12 of a logit); fp32 takes a tanh that is exact to a few 2^-24 of itself.
constexpr float LARGEST_CAP = 1024.f;
struct ScoreRule {
    float scale_log2;              // no cap: logit (base 2) = dot * scale_log2
    float pre, cap_log2;           // cap: logit = cap_log2 - 2 cap_log2 / (1 + 2^(dot * pre)); cap_log2 = 0: no cap
    int window;                    // INT_MAX: none
};
inline ScoreRule score_rule(float scale, float softcap, int window)
{
    ScoreRule r;
    r.scale_log2 = scale * LOG2E;
    r.cap_log2 = softcap * LOG2E;
    r.pre = softcap > 0.f ? 2.f * scale / softcap * LOG2E : 0.f;
    r.window = window > 0 ? window : 0x7FFFFFFF;
    return r;
}
inline ScoreRule score_rule(const ServeDims &d) { return score_rule(d.scale, d.softcap, d.window); }
inline bool in_fp32(const ScoreRule &r) { return std::isfinite(r.scale_log2) && std::isfinite(2.f * r.cap_log2) && std::isfinite(r.pre); }
// Below a quarter of the cap the difference would lose what the score has: tanh's series there (next term 2^-26 of the score), a few 2^-24 of the score
// itself.  Tiles of 64 keys that every row sees whole do without: their sums hide it (24 requests, window 4096: 14.1 us, 14.7 with the series in all).
__device__ __forceinline__ float capped_among_many(float dot, const ScoreRule &r)
{
    return fmaf(-2.f * r.cap_log2, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(dot * r.pre)), r.cap_log2);
}
template <bool CAP> __device__ __forceinline__ float capped(float dot, const ScoreRule &r)
{
    if constexpr (!CAP) return dot * r.scale_log2;
    const float u = dot * r.pre * (0.5f / LOG2E), v = u * u;
    const float series = fmaf(v, fmaf(v, fmaf(v, fmaf(v, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
    return v < 0.0625f ? dot * r.scale_log2 * series : capped_among_many(dot, r);
}

// The request whose rows hold row t: the last one that starts at or in front of t (empty ones share their start with the
// next), or -1 in front of the first and behind the last.
__device__ __forceinline__ int request_of(const int32_t *q_start, int B, int t)
{
    int lo = 0, hi = B + 1;                      // number of starts <= t lies in [lo, hi]
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (q_start[mid] <= t) lo = mid + 1;
        else hi = mid;
    }
    return lo >= 1 && lo <= B ? lo - 1 : -1;
}

// A request as the kernels see it, its numbers brought into range whatever the arrays hold.
struct Request {
    int first, rows;                             // packed rows [first, first + rows), 0 <= first, first + rows <= T
    int n, pos0, prefix;                         // tokens, position of its first row (may be negative), visible prefix (<= n)
};
__device__ __forceinline__ Request make_request(const int32_t *q_start, const int32_t *seq_len, const int32_t *prefix_len, int b, int T, int capacity)
{
    Request r;
    const int lo = min(max(q_start[b], 0), T), hi = min(max(q_start[b + 1], 0), T);
    r.first = lo;
    r.rows = max(hi - lo, 0);
    r.n = seq_len != nullptr ? min(max(seq_len[b], 0), capacity) : r.rows;
    r.pos0 = r.n - r.rows;
    r.prefix = prefix_len != nullptr ? min(max(prefix_len[b], 0), r.n) : 0;
    return r;
}

}  // namespace lca
