// One row of the scored attention by one wavefront: the plain order of the definition, over the visible keys alone.  It
// serves every width and type, and the rows whose tile holds a value that is not finite: on the matrix cores a masked
// entry's weight of zero times an infinity is no number, here an entry that the row does not see is never read.
// Keys: a lane takes a key of a block of 64 and adds up its whole product (16-byte loads of rows 64 apart in the cache);
// values: the lanes take columns and go over the 64 keys.  Far from any bound, which is not what it is for.
#pragma once
#include "serve_internal.h"

namespace lca {

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<uint16_t>(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
template <> __device__ __forceinline__ float to_float<f16_t>(f16_t v) { return f16_bits_to_float(v.bits); }
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ uint16_t from_float<uint16_t>(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
template <> __device__ __forceinline__ f16_t from_float<f16_t>(float v) { return f16_t{float_to_f16_bits(v)}; }
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }

// Keys and values of one request and KV head, packed rows: the element at (key, column), 0 <= key < n.
template <typename T> struct PackedSource {
    const T *sel, *pool;
    size_t sel_row, pool_row;
    __device__ __forceinline__ bool has(int) const { return true; }
    __device__ __forceinline__ float dot(const T *q, int key, int d) const
    {
        constexpr int W = 16 / sizeof(T);
        const T *k = sel + (size_t)key * sel_row;
        float sum = 0.f;
        for (int c = 0; c < d; c += W) {
            T kv[W], qv[W];
            __builtin_memcpy(kv, __builtin_assume_aligned(k + c, 16), 16);
            __builtin_memcpy(qv, __builtin_assume_aligned(q + c, 16), 16);
#pragma unroll
            for (int i = 0; i < W; ++i) sum = fmaf(to_float(kv[i]), to_float(qv[i]), sum);
        }
        return sum;
    }
    __device__ __forceinline__ float value(int key, int c, int) const { return to_float(pool[(size_t)key * pool_row + c]); }
};

__device__ __forceinline__ float decode_e4m3(unsigned code) { return __builtin_amdgcn_cvt_f32_fp8((int)code, 0); }

// The same over the paged cache.
template <typename T> struct PagedSource {
    const int32_t *table;                        // the request's row of the block table
    const uint8_t *sel_q8, *pool_q8;
    const float *scales;
    int page, n_blocks, S, s, d_sel, d_pool;
    FastDiv by_page;
    __device__ __forceinline__ int block(int key) const { return table[by_page(key)]; }
    __device__ __forceinline__ bool has(int key) const { return (unsigned)block(key) < (unsigned)n_blocks; }
    __device__ __forceinline__ float dot(const T *q, int key, int d) const
    {
        const size_t unit = (size_t)block(key) * S + s;
        const uint8_t *k = sel_q8 + (unit * page + key - by_page(key) * page) * d_sel;
        float sum = 0.f;
        for (int c = 0; c < d; c += 8) {
            T qv[8];
            __builtin_memcpy(qv, __builtin_assume_aligned(q + c, 16), 16);
            const uint2 kv = *reinterpret_cast<const uint2 *>(k + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(decode_e4m3((i < 4 ? kv.x : kv.y) >> (8 * (i & 3)) & 0xFF), to_float(qv[i]), sum);
        }
        return sum * scales[2 * unit + 1];
    }
    __device__ __forceinline__ float value(int key, int c, int d) const
    {
        const size_t unit = (size_t)block(key) * S + s;
        const int at = key - by_page(key) * page;
        return decode_e4m3(pool_q8[((unit * (page >> 4) + (at >> 4)) * d + c) * 16 + (at & 15)]) * scales[2 * unit];
    }
};

// A column's partial results [max (base 2), sum, 64 V outputs], `step` floats apart, joined by one wavefront: each 16 lanes take
// every fourth, 4 V outputs a lane, and are added up by exchanges; lane l ends with outputs l V .. l V + V - 1.
template <int V> __device__ __forceinline__ void merge_parts(const float *src, size_t step, int parts, int lane, float &m, float &l, float (&out)[V])
{
    const int q4 = lane >> 4, first = (lane & 15) * 4 * V;
    m = -INFINITY;
    for (int p = lane; p < parts; p += 64) m = fmaxf(m, src[p * step]);
    m = lanes::over_group<64>(m, lanes::Max());
    float sum[4 * V];
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * V; ++i) sum[i] = 0.f;
#pragma unroll 2
    for (int p = q4; p < parts; p += 4) {
        const float *x = src + p * step;
        const float f = x[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[0] - m);
        l = fmaf(x[1], f, l);
#pragma unroll
        for (int i = 0; i < 4 * V; i += 2) {
            const float2 y = *reinterpret_cast<const float2 *>(x + 2 + first + i);
            sum[i] = fmaf(y.x, f, sum[i]);
            sum[i + 1] = fmaf(y.y, f, sum[i + 1]);
        }
    }
    l = lanes::across32(lanes::across16(l, lanes::Sum()), lanes::Sum());
#pragma unroll
    for (int i = 0; i < 4 * V; ++i) sum[i] = lanes::across32(lanes::across16(sum[i], lanes::Sum()), lanes::Sum());
    // lane l has columns first + 0 .. 4 V - 1 of its l & 15; its own are those of lane l / 4, from (l & 3) V on
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = __shfl(sum[k * V + v], lane >> 2, 64);
        out[v] = (lane & 3) == 0 ? y[0] : (lane & 3) == 1 ? y[1] : (lane & 3) == 2 ? y[2] : y[3];
    }
}

// Row at position i (< r.n) of request r: its output to O (d_pool elements) and lse (may be NULL).  All 64 lanes take
// part, everything but the lane is the same for all of them.  NV: columns per lane (64 NV >= d_pool).
template <typename T, int NV, class Source>
__device__ __forceinline__ void scored_row(const Source &src, const T *q, const Request &r, int i, float slope, const ScoreRule &rule, int d_sel, int d_pool,
                                           T *O, float *lse, int lane)
{
    // the visible keys: [0, pre) and [from, to)
    const int pre = i >= 0 ? r.prefix : 0;
    const int from = max(pre, i >= rule.window ? i - rule.window + 1 : 0), to = max(from, min(i + 1, r.n));
    const int count = pre + (to - from);
    float m = -INFINITY, l = 0.f, acc[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) acc[u] = 0.f;
    for (int x0 = 0; x0 < count; x0 += 64) {
        const int x = x0 + lane, j = x < pre ? x : x - pre + from;
        float s = -INFINITY;
        if (x < count && src.has(j)) {
            const float dot = src.dot(q, j, d_sel);
            if constexpr (sizeof(T) == 4) s = rule.cap_log2 > 0.f ? rule.cap_log2 * tanhf(dot * rule.pre * (0.5f / LOG2E)) : capped<false>(dot, rule);
            else s = rule.cap_log2 > 0.f ? capped<true>(dot, rule) : capped<false>(dot, rule);
            s = fmaf(-slope, fabsf((float)(i - j)), s);
        }
        const float top = fmaxf(m, lanes::over_group<64>(s, lanes::Max()));
        const float ref = top == -INFINITY ? 0.f : top, old = __builtin_amdgcn_exp2f(m - ref);
        const float p = __builtin_amdgcn_exp2f(s - ref);
        l = fmaf(l, old, lanes::over_group<64>(p, lanes::Sum()));
        m = top;
#pragma unroll
        for (int u = 0; u < NV; ++u) acc[u] *= old;
        const unsigned long long live = __builtin_amdgcn_ballot_w64(s != -INFINITY);     // (a NaN is live)
        for (unsigned long long todo = live; todo != 0; todo &= todo - 1) {
            const int y = __builtin_ctzll(todo);
            const float pj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(p), y));
            const int jj = __builtin_amdgcn_readlane(j, y);
#pragma unroll
            for (int u = 0; u < NV; ++u)
                if (lane + 64 * u < d_pool) acc[u] = fmaf(pj, src.value(jj, lane + 64 * u, d_pool), acc[u]);
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int u = 0; u < NV; ++u)
        if (lane + 64 * u < d_pool) O[lane + 64 * u] = from_float<T>(acc[u] * inv);
    if (lse != nullptr && lane == 0) *lse = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

}  // namespace lca
