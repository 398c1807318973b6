// Attention of a few rows per request over the paged 8-bit cache (include/lca_serve.h): single tokens, speculative ones.
// Up to 16 NCT (row, query head) pairs of a KV head are the columns of 16x16x32 MFMAs:
//   S^T[key, column] = K Q^T     A = keys,   B = the queries, in registers throughout
//   O^T[dv, column] += V^T P^T   A = values, B = P^T = exp2(S^T - m)
// Bound by reading the codes, once per request and KV head.  They go from memory straight into the registers that the
// products read, without LDS, a barrier or a transpose, because the cache is laid out for it and the products' inner
// index may be counted in any order that both operands agree on:
//   keys    a lane takes 16 columns of a key in one load: the halves are its 8 elements of two k-steps, and the queries
//           are loaded in that order;
//   values  sixteen tokens of a column lie next to each other: a lane's 16 bytes are its 8 keys of two k-steps;
//   P^T     row 4 q + r of S^T's block t (of four) is key 16 q + 4 t + r of the 64, so that a lane's sixteen weights
//           are those of the sixteen tokens whose values it holds.
// A code becomes a 16-bit element with the block's scale in one conversion of two (exact: powers of two).
// A wavefront takes every W-th tile of 64 keys of its workgroup's part on its own (four of them, eight where a workgroup has a request and
// a CU to itself); the loads of its next tile are issued as soon as the registers of this one are free.  Softmax with a running maximum, sums in fp32 of the
// weights before they are rounded.  Parts of long requests are joined by page_merge_kernel.
// 32 requests of 65536 tokens, 32 heads over 8, 128 / 128: 0.68 to 0.73 ms, 5.9 to 6.3 TB/s, what a plain read reaches (4.33 GB fetched, 4.30 needed).
// One of 500 tokens, 28 heads over 4: 8.9 us, a chain of launch, starts, table, codes, join.
#include <algorithm>

#include "serve_row.h"

namespace lca {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ floatx4 mfma_16x16x32(bf16x8 a, bf16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx4 mfma_16x16x32(f16x8 a, f16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

template <typename E> struct Store;                        // the row code's tag of the element type
template <> struct Store<__bf16> { typedef uint16_t type; };
template <> struct Store<_Float16> { typedef f16_t type; };

// Eight codes times a power of two as eight elements.
template <typename E> __device__ __forceinline__ unsigned convert2(unsigned w, float scale, bool high);
template <> __device__ __forceinline__ unsigned convert2<__bf16>(unsigned w, float scale, bool high)
{
    return high ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))
                : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
}
template <> __device__ __forceinline__ unsigned convert2<_Float16>(unsigned w, float scale, bool high)
{
    return high ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true))
                : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false));
}
template <typename E> __device__ __forceinline__ auto convert8(unsigned lo, unsigned hi, float scale)
{
    typedef E ex8 __attribute__((ext_vector_type(8)));
    const uint4 v = make_uint4(convert2<E>(lo, scale, false), convert2<E>(lo, scale, true), convert2<E>(hi, scale, false), convert2<E>(hi, scale, true));
    return __builtin_bit_cast(ex8, v);
}

struct DecodeParams {
    const void *q;
    void *O;
    float *lse, *part;
    const int32_t *q_start, *seq_len, *prefix_len, *block_table;
    const float *slopes;
    const uint8_t *sel_q8, *pool_q8;
    const float *scales;
    ServeDims d;
    ScoreRule rule;
    int parts;                            // workgroups of a (request, KV head, group of columns)
    int groups;                           // groups of 16 NCT columns
    FastDiv by_parts, by_groups, by_pairs;
    int most;                             // requests of more columns are left to the chunk kernel (INT_MAX: none)
};

constexpr int TILE = 64;
constexpr int LEAST_TILES = 8;            // of a part (24 requests of 4 rows, window 4096, in up to ten parts: 13.7 us, 14.3 with four, 16.9 with sixteen; 14.1 since)
// Whether a wavefront needs the registers of two.
constexpr bool heavy(int dv, int nct) { return dv * nct >= 256; }

// What a request's rows see, in tiles: [0, pre) and [from, to), numbered one behind the other.
struct Tiles { int pre, from, count; };
__device__ __forceinline__ Tiles make_tiles(const Request &r, int window)
{
    Tiles t;
    const int first = max(r.pos0, 0);                                          // first row's position
    const int lo = first >= window ? first - window + 1 : 0;                   // first key any row sees by the window
    const int end = (r.n + TILE - 1) / TILE;
    t.pre = min((r.prefix + TILE - 1) / TILE, end);
    t.from = max(t.pre, lo / TILE);
    t.count = t.pre + max(end - t.from, 0);
    return t;
}

// A column computed again over what its row sees alone (serve_row.h).
template <typename E, int DV> __device__ __forceinline__ void row_again(const DecodeParams &kp, const Request &r, int b, int s, int column, int lane)
{
    typedef typename Store<E>::type T;
    const ServeDims &d = kp.d;
    const int row = d.by_hps(column), h = s * d.hps + (column - row * d.hps), t = r.first + row;
    const PagedSource<T> src{kp.block_table + (size_t)b * d.max_blocks, kp.sel_q8, kp.pool_q8, kp.scales, d.page, d.n_blocks, d.S, s, d.d_sel, d.d_pool, d.by_page};
    scored_row<T, DV / 64>(src, (const T *)kp.q + (size_t)t * d.q_row + (size_t)h * d.d_sel, r, r.pos0 + row, kp.slopes != nullptr ? kp.slopes[h] * LOG2E : 0.f, kp.rule, d.d_sel,
                           d.d_pool, (T *)kp.O + ((size_t)t * d.H + h) * d.d_pool, kp.lse != nullptr ? kp.lse + (size_t)t * d.H + h : nullptr, lane);
}

// Output columns [first, first + N) of a column from its sums, the softmax's sum and maximum (base 2); whether they are finite numbers.
template <typename E, int N>
__device__ __forceinline__ bool write_column(const DecodeParams &kp, const Request &r, int s, int column, int first, const float (&sum)[N], float l, float m)
{
    typedef typename Store<E>::type T;
    const ServeDims &d = kp.d;
    const int row = d.by_hps(column), h = s * d.hps + (column - row * d.hps);
    const size_t at = (size_t)(r.first + row) * d.H + h;
    T *O = (T *)kp.O + at * d.d_pool + first;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bool fine = true;
    T o[N];
#pragma unroll
    for (int v = 0; v < N; ++v) {
        const float x = sum[v] * inv;
        fine = fine && fabsf(x) < INFINITY;
        o[v] = from_float<T>(x);
    }
    if (first < d.d_pool) __builtin_memcpy(__builtin_assume_aligned(O, N * sizeof(T)), o, N * sizeof(T));        // (N divides 16, and 16 the width)
    if (kp.lse != nullptr && first == 0) kp.lse[at] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    return fine;
}

template <typename E, int DK, int DV, int NCT, int W>
__global__ __launch_bounds__(64 * W, heavy(DV, NCT) ? 1 : 2) void page_decode_kernel(const DecodeParams kp)
{
    typedef E ex8 __attribute__((ext_vector_type(8)));
    constexpr int NK = DK / 64, NV = DV / 16, ROW = DV + 4;
    __shared__ __attribute__((aligned(16))) float outs[W][16][ROW];
    __shared__ float stats[W][16][2];

    const ServeDims &d = kp.d;
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, q4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // first part 0 of all pairs, then part 1: what is split by a hint of long requests and has short ones still falls on every XCD (workgroups go to
    // them in turn: 32 requests of 4000 tokens with room for 131072, 32 heads over 8, 123 us with a pair's parts next to each other, 51 so)
    const int outer = kp.by_pairs((int)blockIdx.x), pair = blockIdx.x - outer * (d.B * d.S), part = kp.by_groups(outer), group = outer - part * kp.groups;
    const int unit = pair * kp.groups + group, b = d.by_S(pair), s = pair - b * d.S;
    const Request r = make_request(kp.q_start, kp.seq_len, kp.prefix_len, b, d.T, d.max_blocks * d.page);
    const int columns = r.rows * d.hps;
    if (columns == 0 || columns > kp.most) return;
    const Tiles tiles = make_tiles(r, kp.rule.window);
    // more columns than there are groups for (a hint that was too small): the first part takes them all, unsplit
    const bool many = columns > kp.groups * 16 * NCT;
    const int parts = many ? 1 : kp.parts;
    if (part >= parts) return;
    const int per = max(LEAST_TILES, many ? tiles.count : kp.by_parts(tiles.count + kp.parts - 1));
    const int lo = part * per, hi = many ? tiles.count : min(lo + per, tiles.count);
    if (lo >= hi && part > 0) return;                                          // (nothing to see at all: part 0 writes it)
    const bool whole = lo == 0 && hi == tiles.count;                           // this workgroup has the request to itself

    const int32_t *table = kp.block_table + (size_t)b * d.max_blocks;
    const int strips = d.page >> 4, strip_end = (r.n + 15) >> 4;               // strips of 16 tokens: of a block, of the request
    const int chunks = d.d_sel >> 4, cols16 = d.d_pool >> 4;

    for (int cg = group; cg * 16 * NCT < columns; cg += kp.groups) {
        const int c0 = cg * 16 * NCT;
        // the columns' rows and heads; the queries in the order of the keys' loads
        int pos[NCT];
        float slope[NCT];
        ex8 qf[NCT][2 * NK];
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
            const int c = min(c0 + 16 * ct + col, columns - 1), row = d.by_hps(c), h = s * d.hps + (c - row * d.hps);
            pos[ct] = r.pos0 + row;
            slope[ct] = kp.slopes != nullptr ? kp.slopes[h] * LOG2E : 0.f;
            const E *qp = (const E *)kp.q + (size_t)(r.first + row) * d.q_row + (size_t)h * d.d_sel;
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
                    qf[ct][2 * k + hf] = q4 + 4 * k < chunks ? *reinterpret_cast<const ex8 *>(qp + 16 * (q4 + 4 * k) + 8 * hf) : ex8{0, 0, 0, 0, 0, 0, 0, 0};
        }
        floatx4 acc[NCT][NV];
        float m_run[NCT], l_run[NCT];
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
            m_run[ct] = -INFINITY;
            l_run[ct] = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) acc[ct][v] = floatx4{0.f, 0.f, 0.f, 0.f};
        }

        auto tile_at = [&](int x) { return x < tiles.pre ? x : x - tiles.pre + tiles.from; };
        // the blocks of a lane's two strips of tile x: the one its key rows lie in, the one of its values; -1: none
        auto block_of = [&](int strip) {
            const int blk = table[d.by_strips(min(strip, strip_end - 1))];
            return strip < strip_end && (unsigned)blk < (unsigned)d.n_blocks ? blk : -1;
        };
        uint4 kreg[4][NK], vreg[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) vreg[v] = make_uint4(0, 0, 0, 0);        // (columns behind d_pool stay so)
        float k_scale = 1.f, v_scale = 1.f;
        int k_blk = -1, v_blk = -1, k_next = -1, v_next = -1;
        auto fetch_blocks = [&](int x) {
            const int strip = 4 * tile_at(x);
            k_next = block_of(strip + (col >> 2));
            v_next = block_of(strip + q4);
        };
        auto load_keys = [&](int x) {
            const int strip = 4 * tile_at(x) + (col >> 2);
            k_blk = k_next;
            const size_t u = (size_t)max(k_blk, 0) * d.S + s;
            const uint8_t *p = kp.sel_q8 + (u * d.page + (strip - d.by_strips(strip) * strips) * 16 + (col & 3)) * d.d_sel + 16 * q4;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int k = 0; k < NK; ++k)
                    kreg[t][k] = q4 + 4 * k < chunks ? *reinterpret_cast<const uint4 *>(p + (size_t)4 * t * d.d_sel + 64 * k) : make_uint4(0, 0, 0, 0);
            k_scale = kp.scales[2 * u + 1];
        };
        auto load_values = [&](int x) {
            const int strip = 4 * tile_at(x) + q4;
            v_blk = v_next;
            const size_t u = (size_t)max(v_blk, 0) * d.S + s;
            const uint8_t *p = kp.pool_q8 + ((u * strips + strip - d.by_strips(strip) * strips) * d.d_pool + col) * 16;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (v < cols16) vreg[v] = *reinterpret_cast<const uint4 *>(p + 256 * v);
            v_scale = kp.scales[2 * u];
        };

        const int pos_lo = max(r.pos0, 0), pos_hi = r.n - 1;                   // of the request's rows
        int x = lo + wave;
        if (x < hi) {
            fetch_blocks(x);
            load_keys(x);
            load_values(x);
            if (x + W < hi) fetch_blocks(x + W);
        }
        for (; x < hi; x += W) {
            const int j0 = tile_at(x) * TILE + 16 * q4;                        // first key of the lane's strip
            const int blk = v_blk;                                            // (its scores are those of the strip whose values it holds)
            // S^T
            floatx4 sacc[NCT][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                ex8 kf[2 * NK];
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    kf[2 * k] = convert8<E>(kreg[t][k].x, kreg[t][k].y, k_scale);
                    kf[2 * k + 1] = convert8<E>(kreg[t][k].z, kreg[t][k].w, k_scale);
                }
#pragma unroll
                for (int ct = 0; ct < NCT; ++ct) {
                    sacc[ct][t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < 2 * NK; ++k) sacc[ct][t] = mfma_16x16x32(kf[k], qf[ct][k], sacc[ct][t]);
                }
            }
            if (x + W < hi) load_keys(x + W);

            // does every row see the whole tile?
            const int j_lo = tile_at(x) * TILE, j_hi = j_lo + TILE - 1;
            const bool inside = j_hi <= pos_lo && (j_hi < r.prefix || pos_hi - j_lo < kp.rule.window);
            const bool full = inside && __builtin_amdgcn_ballot_w64(blk < 0) == 0;
            ex8 pb[NCT][2];
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) {
                float lg[16], mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < 16; ++i) lg[i] = sacc[ct][i >> 2][i & 3];
                if (kp.rule.cap_log2 > 0.f && full) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) lg[i] = capped_among_many(lg[i], kp.rule);
                } else if (kp.rule.cap_log2 > 0.f) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) lg[i] = capped<true>(lg[i], kp.rule);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) lg[i] = capped<false>(lg[i], kp.rule);
                }
                if (kp.slopes != nullptr) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) lg[i] = fmaf(-slope[ct], fabsf((float)(pos[ct] - j0 - i)), lg[i]);
                }
                if (!full) {
                    const int p = pos[ct];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int j = j0 + i;
                        const bool seen = blk >= 0 && p >= 0 && j < r.n && ((j <= p && p - j < kp.rule.window) || j < r.prefix);
                        lg[i] = seen ? lg[i] : -INFINITY;
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, lg[i]);
                mx = fmaxf(m_run[ct], lanes::across32(lanes::across16(mx, lanes::Max()), lanes::Max()));
                if (__builtin_amdgcn_ballot_w64(mx > m_run[ct]) != 0) {
                    const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[ct] - mx);
                    m_run[ct] = mx;
                    l_run[ct] *= f;
#pragma unroll
                    for (int v = 0; v < NV; ++v)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[ct][v][i] *= f;
                }
                const float ref = m_run[ct] == -INFINITY ? 0.f : m_run[ct];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float p = __builtin_amdgcn_exp2f(lg[i] - ref);
                    l_run[ct] += p;
                    pb[ct][i >> 3][i & 7] = (E)p;
                }
            }
            // values that no row sees do not enter, whatever they are
            if (!full) {
                const int lo_all = pos_lo >= kp.rule.window ? pos_lo - kp.rule.window + 1 : 0;
                unsigned keep[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    keep[w] = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = j0 + 4 * w + i;
                        if (blk >= 0 && j < r.n && (j >= lo_all || j < r.prefix)) keep[w] |= 0xFFu << (8 * i);
                    }
                }
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    vreg[v].x &= keep[0]; vreg[v].y &= keep[1]; vreg[v].z &= keep[2]; vreg[v].w &= keep[3];
                }
            }
            // O^T
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const ex8 v0 = convert8<E>(vreg[v].x, vreg[v].y, v_scale), v1 = convert8<E>(vreg[v].z, vreg[v].w, v_scale);
#pragma unroll
                for (int ct = 0; ct < NCT; ++ct) {
                    acc[ct][v] = mfma_16x16x32(v0, pb[ct][0], acc[ct][v]);
                    acc[ct][v] = mfma_16x16x32(v1, pb[ct][1], acc[ct][v]);
                }
            }
            if (x + W < hi) load_values(x + W);
            if (x + 2 * W < hi) fetch_blocks(x + 2 * W);
        }

        // the wavefronts' results, 16 columns at a time
        for (int ct = 0; ct < NCT; ++ct) {
            if (c0 + 16 * ct >= columns) break;
            float m_ct = 0.f, l_ct = 0.f;
#pragma unroll
            for (int k = 0; k < NCT; ++k)
                if (k == ct) {
#pragma unroll
                    for (int v = 0; v < NV; ++v) *reinterpret_cast<floatx4 *>(&outs[wave][col][16 * v + 4 * q4]) = acc[k][v];
                    m_ct = m_run[k];
                    l_ct = l_run[k];
                }
            l_ct = lanes::across32(lanes::across16(l_ct, lanes::Sum()), lanes::Sum());
            if (q4 == 0) { stats[wave][col][0] = m_ct; stats[wave][col][1] = l_ct; }
            __syncthreads();
            {
                // 4 W lanes take a column, N outputs each
                constexpr int LANES = 4 * W, N = DV / LANES;
                const int k = tid / LANES, column = c0 + 16 * ct + k, first = (tid % LANES) * N;
                float m = -INFINITY, l = 0.f, sum[N], f[W];
#pragma unroll
                for (int w = 0; w < W; ++w) m = fmaxf(m, stats[w][k][0]);
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    f[w] = stats[w][k][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stats[w][k][0] - m);
                    l = fmaf(stats[w][k][1], f[w], l);
                }
#pragma unroll
                for (int v = 0; v < N; ++v) sum[v] = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    float y[N];
                    __builtin_memcpy(y, __builtin_assume_aligned(&outs[w][k][first], 4 * (N < 4 ? N : 4)), 4 * N);
#pragma unroll
                    for (int v = 0; v < N; ++v) sum[v] = fmaf(y[v], f[w], sum[v]);
                }
                if (whole) {
                    const bool fine = column >= columns || write_column<E, N>(kp, r, s, column, first, sum, l, m);
                    unsigned long long odd = __builtin_amdgcn_ballot_w64(!fine);
                    while (__builtin_expect(odd != 0, 0)) {
                        const int g = __builtin_ctzll(odd) / LANES;
                        row_again<E, DV>(kp, r, b, s, c0 + 16 * ct + wave * (64 / LANES) + g, lane);
                        odd &= ~(((1ull << LANES) - 1) << (LANES * g));
                    }
                } else {
                    float *dst = kp.part + (((size_t)unit * kp.parts + part) * 16 * NCT + 16 * ct + k) * (DV + 2);
#pragma unroll
                    for (int v = 0; v < N; v += 2) *reinterpret_cast<float2 *>(dst + 2 + first + v) = float2{sum[v], sum[v + 1]};
                    if (first == 0) *reinterpret_cast<float2 *>(dst) = float2{m, l};
                }
            }
            __syncthreads();
        }
    }
}

// Joins the parts of every column that has more than one: one wavefront per column.
template <typename E, int DV, int NCT>
__global__ __launch_bounds__(256) void page_merge_kernel(const DecodeParams kp)
{
    constexpr int V = DV / 64, columns_per_unit = 16 * NCT;
    const ServeDims &d = kp.d;
    const int lane = threadIdx.x & 63;
    const int c = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = c / columns_per_unit, k = c % columns_per_unit;         // (a power of two)
    const int pair = kp.by_groups(unit), group = unit - pair * kp.groups, b = d.by_S(pair), s = pair - b * d.S;
    if (b >= d.B) return;
    const Request r = make_request(kp.q_start, kp.seq_len, kp.prefix_len, b, d.T, d.max_blocks * d.page);
    const int columns = r.rows * d.hps, column = group * columns_per_unit + k;
    if (column >= columns || columns > kp.most || columns > kp.groups * columns_per_unit) return;
    const Tiles tiles = make_tiles(r, kp.rule.window);
    const int per = max(LEAST_TILES, kp.by_parts(tiles.count + kp.parts - 1));
    if (tiles.count <= per) return;                                            // one part: it has written the output
    const int parts = (tiles.count + per - 1) / per;
    const float *src = kp.part + ((size_t)unit * kp.parts * columns_per_unit + k) * (DV + 2);
    float m, l, sum[V];
    merge_parts<V>(src, (size_t)columns_per_unit * (DV + 2), parts, lane, m, l, sum);
    const bool fine = write_column<E, V>(kp, r, s, column, lane * V, sum, l, m);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!fine) != 0, 0)) row_again<E, DV>(kp, r, b, s, column, lane);
}

struct Plan { int nct, groups, parts, waves; };

// How a call is split, from its sizes and hints.
Plan make_plan(const ServeDims &d)
{
    Plan p;
    const int dv = d.d_pool <= 64 && d.d_sel <= 64 ? 64 : d.d_pool <= 128 && d.d_sel <= 192 ? 128 : 256;
    const int columns = (int)std::min<long>((long)d.max_q * d.hps, PAGE_DECODE_COLUMNS);
    const int most = dv == 64 ? 4 : dv == 128 ? 2 : 1;                // (what the registers hold)
    p.nct = columns <= 16 ? 1 : columns <= 32 ? 2 : 4;
    if (p.nct > most) p.nct = most;
    p.groups = (columns + 16 * p.nct - 1) / (16 * p.nct);
    long keys = d.max_kv;
    if (d.window > 0) keys = std::min<long>(keys, (long)d.window + d.max_q + TILE);
    const long tiles = std::max<long>(1, (keys + TILE - 1) / TILE), units = (long)d.B * d.S * p.groups;
    // Twice the workgroups that run at a time: requests are of different lengths, and the parts of the long ones fill in behind the
    // short ones (20 requests of up to 9000 tokens, 32 heads over 8: 30 us, 41 with half as many; 4 of 30000 each 48 and 45).  Where a
    // wavefront needs the registers of two, one for each CU: 8 requests of 16000, 40 heads over one, 23 us, 27 with twice as many, 38 with
    // four times.  Up to 16 tiles, and up to 64 where there is a workgroup per CU without it, nothing is split and there is nothing to join: 500
    // tokens, 28 heads over 4, 9.9 us, 11.4 in two parts; 64 requests of up to 1500, 17 us, 25 in two.
    const long target = heavy(dv, p.nct) ? 256 : 1024;
    p.parts = tiles <= 16 || (units >= 256 && tiles <= 64) ? 1 : (int)std::max<long>(1, std::min<long>(target / units, (tiles + 3) / 4));
    // Eight wavefronts where all of them run at once and nothing is split: 500 tokens 9.1 us with four, 8.6 with eight; where there are more
    // workgroups than CUs (64 requests of up to 1500) 17 and 21, where parts are joined (one request of 2000) 11.2 and 12.2.
    p.waves = !heavy(dv, p.nct) && p.parts == 1 && units <= 256 && tiles > 4 ? 8 : 4;
    return p;
}

template <typename E, int DK, int DV, int NCT> void run(const DecodeParams &kp, const Plan &p, hipStream_t st)
{
    const long units = (long)kp.d.B * kp.d.S * kp.groups;
    if constexpr (!heavy(DV, NCT))
        if (p.waves == 8) return page_decode_kernel<E, DK, DV, NCT, 8><<<(unsigned)units, 512, 0, st>>>(kp);          // (one part)
    page_decode_kernel<E, DK, DV, NCT, 4><<<(unsigned)(units * kp.parts), 256, 0, st>>>(kp);
    if (kp.parts > 1) page_merge_kernel<E, DV, NCT><<<(unsigned)(units * 4 * NCT), 256, 0, st>>>(kp);
}
template <typename E, int DK, int DV> void run_columns(const DecodeParams &kp, const Plan &p, hipStream_t st)
{
    if constexpr (DV == 64)
        if (p.nct == 4) return run<E, DK, DV, 4>(kp, p, st);
    if constexpr (DV <= 128)
        if (p.nct == 2) return run<E, DK, DV, 2>(kp, p, st);
    run<E, DK, DV, 1>(kp, p, st);
}

template <typename E> void run_widths(const DecodeParams &kp, const Plan &p, hipStream_t st)
{
    const int dk = kp.d.d_sel, dv = kp.d.d_pool;
    if (dk <= 64 && dv <= 64) run_columns<E, 64, 64>(kp, p, st);
    else if (dk <= 128 && dv <= 128) run_columns<E, 128, 128>(kp, p, st);
    else if (dk <= 192 && dv <= 128) run_columns<E, 192, 128>(kp, p, st);
    else run_columns<E, 256, 256>(kp, p, st);
}

}  // namespace

size_t page_decode_workspace_bytes(const ServeDims &d)
{
    const Plan p = make_plan(d);
    const int dv = d.d_pool <= 64 && d.d_sel <= 64 ? 64 : d.d_pool <= 128 && d.d_sel <= 192 ? 128 : 256;
    return p.parts > 1 ? (size_t)d.B * d.S * p.groups * p.parts * 16 * p.nct * (dv + 2) * sizeof(float) : 0;
}

hipError_t launch_page_decode(const ScoredArgs &a, int most, hipStream_t st)
{
    const Plan p = make_plan(a.d);
    const DecodeParams kp{a.Q, a.O, a.lse, a.part, a.q_start, a.seq_len, a.prefix_len, a.block_table, a.slopes, a.sel_q8, a.pool_q8, a.scales, a.d, score_rule(a.d),
                          p.parts, p.groups, FastDiv(p.parts), FastDiv(p.groups), FastDiv(a.d.B * a.d.S), most};
    if (a.d.dtype == LCA_F16) run_widths<_Float16>(kp, p, st);
    else run_widths<__bf16>(kp, p, st);
    return hipGetLastError();
}

}  // namespace lca
