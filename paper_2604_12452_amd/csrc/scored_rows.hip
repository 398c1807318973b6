// The scored attention of packed prompts (include/lca_serve.h) row by row, one wavefront per (row, query head): fp32, widths above 256, tokens
// farther apart than a buffer descriptor reaches.  2048 tokens, 16 heads over 4, 128 / 128, fp32: 2.9 ms.
#include "serve_row.h"

namespace lca {
namespace {

struct RowsParams {
    const void *Q, *SEL, *POOL;
    void *O;
    float *lse;
    const int32_t *q_start, *prefix_len;
    const float *slopes;
    ServeDims d;
    ScoreRule rule;
};

template <typename T, int NV>
__global__ __launch_bounds__(256) void scored_rows_kernel(const RowsParams kp)
{
    const ServeDims &d = kp.d;
    const int lane = threadIdx.x & 63;
    const long u = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = (int)(u / d.H), h = (int)(u - (long)t * d.H), s = h / d.hps;
    if (t >= d.T) return;
    const int b = request_of(kp.q_start, d.B, t);
    if (b < 0) return;
    const Request r = make_request(kp.q_start, nullptr, kp.prefix_len, b, d.T, 0);
    if (t < r.first || t >= r.first + r.rows) return;
    const int i = r.pos0 + t - r.first;
    const float slope = kp.slopes != nullptr ? kp.slopes[h] * LOG2E : 0.f;
    const T *q = (const T *)kp.Q + (size_t)t * d.q_row + (size_t)h * d.d_sel;
    T *O = (T *)kp.O + ((size_t)t * d.H + h) * d.d_pool;
    float *lse = kp.lse != nullptr ? kp.lse + (size_t)t * d.H + h : nullptr;
    const PackedSource<T> src{(const T *)kp.SEL + (size_t)r.first * d.sel_row + (size_t)s * d.d_sel,
                              (const T *)kp.POOL + (size_t)r.first * d.pool_row + (size_t)s * d.d_pool, d.sel_row, d.pool_row};
    scored_row<T, NV>(src, q, r, i, slope, kp.rule, d.d_sel, d.d_pool, O, lse, lane);
}

template <typename T> void run_rows(const RowsParams &kp, hipStream_t st)
{
    const unsigned grid = (unsigned)(((long)kp.d.T * kp.d.H + 3) / 4);
    if (kp.d.d_pool <= 256) scored_rows_kernel<T, 4><<<grid, 256, 0, st>>>(kp);
    else scored_rows_kernel<T, 16><<<grid, 256, 0, st>>>(kp);
}

}  // namespace

hipError_t launch_scored_rows(const ScoredArgs &a, hipStream_t st)
{
    const RowsParams kp{a.Q, a.SEL, a.POOL, a.O, a.lse, a.q_start, a.prefix_len, a.slopes, a.d, score_rule(a.d)};
    if (a.d.dtype == LCA_F32) run_rows<float>(kp, st);
    else if (a.d.dtype == LCA_F16) run_rows<f16_t>(kp, st);
    else run_rows<uint16_t>(kp, st);
    return hipGetLastError();
}

}  // namespace lca
