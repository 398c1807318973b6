// New keys and values into the paged 8-bit cache (include/lca_serve.h): one E4M3 code per element, one power-of-two scale
// per block of tokens, KV head and component.
//
// Unit = the tokens of one block in this call, one KV head; one workgroup takes both components of it, so that nobody else
// reads or writes its codes and scales.  Two passes over the unit's new values, largest magnitude, then codes: the second reads
// what the first has brought into the caches.  A power-of-two scale makes x / scale exact, the only rounding is the
// conversion's.  When the block's scale rises, the codes in front of the new tokens are converted again, old / new being a
// power of two as well: exact but for codes that leave E4M3's normal range.
// Values lie sixteen tokens of a column next to each other: a thread takes sixteen tokens of a pair of columns, reads them
// four bytes at a time (a wavefront: 256 bytes of a row) and writes two whole 16-byte pieces; a piece that holds older
// tokens, or places behind the new ones, is read first and keeps them.
// Bound by memory: two bytes read and one written per element.
#include "serve_internal.h"

namespace lca {
namespace {

struct StoreParams {
    const void *SEL, *POOL;
    const int32_t *slot;
    uint8_t *sel_q8, *pool_q8;
    float *scales;
    int T, S, d_pool, d_sel, page, n_blocks, window;       // window: packed rows a workgroup looks for starts of units in
    size_t sel_row, pool_row;
};

template <typename T> struct Range;                      // exponents of a block's scale: the decoded codes stay finite numbers of the type
template <> struct Range<uint16_t> { static constexpr int LO = -100, HI = 119; };
template <> struct Range<f16_t> { static constexpr int LO = -15, HI = 7; };

// Two 16-bit elements of a word.
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<uint16_t>(uint32_t w) { return float2{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)}; }
template <> __device__ __forceinline__ float2 unpack2<f16_t>(uint32_t w) { return float2{f16_bits_to_float((uint16_t)w), f16_bits_to_float((uint16_t)(w >> 16))}; }

template <typename T> __device__ __forceinline__ int scale_exponent(float amax)
{
    if (!(amax > 0.f)) return Range<T>::LO;
    if (amax == INFINITY) return Range<T>::HI;
    int e;
    const float f = frexpf(amax, &e);                    // amax = f 2^e, f in [0.5, 1); 448 = 0.875 * 2^9
    return min(max(f <= 0.875f ? e - 9 : e - 8, Range<T>::LO), Range<T>::HI);
}
// x / 2^e within E4M3's range (a NaN stays one).
__device__ __forceinline__ float in_range(float x, float inv)
{
    const float y = x * inv;
    return y > 448.f ? 448.f : y < -448.f ? -448.f : y;
}
__device__ __forceinline__ unsigned encode4(float a, float b, float c, float d)
{
    unsigned w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// Four codes times a power of two, encoded again.
__device__ __forceinline__ unsigned recode4(unsigned w, float factor)
{
    return encode4(in_range(__builtin_amdgcn_cvt_f32_fp8((int)w, 0), factor), in_range(__builtin_amdgcn_cvt_f32_fp8((int)w, 1), factor),
                   in_range(__builtin_amdgcn_cvt_f32_fp8((int)w, 2), factor), in_range(__builtin_amdgcn_cvt_f32_fp8((int)w, 3), factor));
}

template <typename T>
__device__ __forceinline__ void store_unit(const StoreParams &kp, int t0, int block, int off, int n, int s, float (&maxima)[2][4], int tid)
{
    const int lane = tid & 63, wave = tid >> 6;
    const size_t unit = (size_t)block * kp.S + s;
    const uint16_t *sel = (const uint16_t *)kp.SEL + (size_t)t0 * kp.sel_row + (size_t)s * kp.d_sel;
    const uint16_t *pool = (const uint16_t *)kp.POOL + (size_t)t0 * kp.pool_row + (size_t)s * kp.d_pool;
    const float2 old = *reinterpret_cast<const float2 *>(kp.scales + 2 * unit);      // (pooled, selected)

    // largest magnitudes (fmaxf drops a NaN)
    auto largest = [&](const uint16_t *x, size_t row, int d) {
        const int pieces = d / 8;
        float m = 0.f;
        for (int u = tid; u < n * pieces; u += 256) {
            const int t = u / pieces, c = u - t * pieces;
            const uint4 v = *reinterpret_cast<const uint4 *>(x + (size_t)t * row + 8 * c);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = unpack2<T>(w[i]);
                m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
        }
        return lanes::over_group<64>(m, lanes::Max());
    };
    const float m_pool = largest(pool, kp.pool_row, kp.d_pool), m_sel = largest(sel, kp.sel_row, kp.d_sel);
    __syncthreads();                                     // (the unit before is done with `maxima`; the scales have been read)
    if (lane == 0) { maxima[0][wave] = m_pool; maxima[1][wave] = m_sel; }
    __syncthreads();
    float scale[2], inv[2], factor[2];
    bool raised[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const float m = fmaxf(fmaxf(maxima[c][0], maxima[c][1]), fmaxf(maxima[c][2], maxima[c][3]));
        const int e = scale_exponent<T>(m);
        const float before = c == 0 ? old.x : old.y, fresh = ldexpf(1.f, e);
        raised[c] = off > 0 && !(before >= fresh);
        scale[c] = off > 0 && before >= fresh ? before : fresh;
        inv[c] = 1.f / scale[c];
        factor[c] = before * inv[c];
    }
    if (tid == 0) *reinterpret_cast<float2 *>(kp.scales + 2 * unit) = float2{scale[0], scale[1]};

    // keys: 16 codes at a time; older tokens only when the scale rose
    {
        const int pieces = kp.d_sel / 16, first = raised[1] ? 0 : off;
        uint8_t *dst = kp.sel_q8 + unit * kp.page * kp.d_sel;
        for (int u = tid; u < (off + n - first) * pieces; u += 256) {
            const int at = u / pieces, c = u - at * pieces, token = first + at;
            uint4 *p = reinterpret_cast<uint4 *>(dst + (size_t)token * kp.d_sel + 16 * c);
            uint4 out;
            if (token < off) {
                const uint4 v = *p;
                out = make_uint4(recode4(v.x, factor[1]), recode4(v.y, factor[1]), recode4(v.z, factor[1]), recode4(v.w, factor[1]));
            } else {
                const uint4 *x = reinterpret_cast<const uint4 *>(sel + (size_t)(token - off) * kp.sel_row + 16 * c);
                const uint4 a = x[0], b = x[1];
                const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = unpack2<T>(w[2 * i]), g = unpack2<T>(w[2 * i + 1]);
                    o[i] = encode4(in_range(f.x, inv[1]), in_range(f.y, inv[1]), in_range(g.x, inv[1]), in_range(g.y, inv[1]));
                }
                out = make_uint4(o[0], o[1], o[2], o[3]);
            }
            *p = out;
        }
    }
    // values: sixteen tokens of two columns at a time
    {
        const int pairs = kp.d_pool / 2, first = raised[0] ? 0 : off >> 4, last = (off + n - 1) >> 4;
        uint8_t *dst = kp.pool_q8 + unit * kp.page * kp.d_pool;
        for (int u = tid; u < (last - first + 1) * pairs; u += 256) {
            const int at = u / pairs, c = u - at * pairs, strip = first + at;
            uint4 *p = reinterpret_cast<uint4 *>(dst + ((size_t)strip * kp.d_pool + 2 * c) * 16);
            const int lo = off - 16 * strip, hi = lo + n;       // the new tokens' places in the strip, cut to [0, 16)
            unsigned o[2][4];
            if (lo > 0 || hi < 16) {                            // some places keep what they hold, those of older tokens perhaps recoded
                const uint4 v[2] = {p[0], p[1]};
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const unsigned w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        unsigned r = raised[0] ? recode4(w[i], factor[0]) : w[i];
                        // places at and behind the first new one are not recoded
                        const int keep = min(max(lo - 4 * i, 0), 4);
                        const unsigned mask = keep == 4 ? 0xFFFFFFFFu : (1u << (8 * keep)) - 1;
                        o[k][i] = (r & mask) | (w[i] & ~mask);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) o[0][i] = o[1][i] = 0;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 f[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int place = 4 * i + j;
                    f[j] = float2{0.f, 0.f};
                    if (place >= lo && place < hi) f[j] = unpack2<T>(*reinterpret_cast<const uint32_t *>(pool + (size_t)(place - lo) * kp.pool_row + 2 * c));
                }
                const int from = min(max(lo - 4 * i, 0), 4), to = min(max(hi - 4 * i, 0), 4);
                const unsigned upto_to = to == 4 ? 0xFFFFFFFFu : (1u << (8 * to)) - 1, upto_from = from == 4 ? 0xFFFFFFFFu : (1u << (8 * from)) - 1;
                const unsigned mask = upto_to & ~upto_from;     // bytes of the new tokens
                const unsigned c0 = encode4(in_range(f[0].x, inv[0]), in_range(f[1].x, inv[0]), in_range(f[2].x, inv[0]), in_range(f[3].x, inv[0]));
                const unsigned c1 = encode4(in_range(f[0].y, inv[0]), in_range(f[1].y, inv[0]), in_range(f[2].y, inv[0]), in_range(f[3].y, inv[0]));
                o[0][i] = (o[0][i] & ~mask) | (c0 & mask);
                o[1][i] = (o[1][i] & ~mask) | (c1 & mask);
            }
            p[0] = make_uint4(o[0][0], o[0][1], o[0][2], o[0][3]);
            p[1] = make_uint4(o[1][0], o[1][1], o[1][2], o[1][3]);
        }
    }
}

// A workgroup takes the units that start among `window` packed rows, one KV head.  A unit starts where a token's slot does not
// follow the slot of the token in front of it, or opens a block, and ends where either happens again.
template <typename T>
__global__ __launch_bounds__(256) void page_store_kernel(const StoreParams kp)
{
    __shared__ float maxima[2][4];
    const int tid = threadIdx.x, lane = tid & 63;
    const int win = blockIdx.x / kp.S, s = blockIdx.x - win * kp.S;
    const int slots = kp.n_blocks * kp.page;
    const int lo = win * kp.window, hi = min(lo + kp.window, kp.T);          // at most 64 rows
    const int t = lo + lane;
    const int mine = t < hi ? kp.slot[t] : -1, before = t < hi && t > 0 ? kp.slot[t - 1] : -1;
    const bool valid = (unsigned)mine < (unsigned)slots;
    unsigned long long starts = __builtin_amdgcn_ballot_w64(valid && (mine % kp.page == 0 || before < 0 || mine != before + 1));
    for (; starts != 0; starts &= starts - 1) {                              // (the same for every wavefront)
        const int at = __builtin_ctzll(starts), first = __builtin_amdgcn_readlane(mine, at), t0 = lo + at;
        const int block = first / kp.page, off = first - block * kp.page;
        const int most = min(kp.page - off, kp.T - t0);                      // >= 1
        int n = 0;
        for (;;) {                                                           // tokens of the unit, 64 at a time
            const int k = n + lane;
            const unsigned long long follow = __builtin_amdgcn_ballot_w64(k < most && kp.slot[t0 + min(k, most - 1)] == first + k);
            const int run = follow == ~0ull ? 64 : __builtin_ctzll(~follow);
            n += run;
            if (run < 64) break;
        }
        store_unit<T>(kp, t0, block, off, n, s, maxima, tid);
    }
}

}  // namespace

hipError_t launch_page_store_q8(const StoreArgs &a, hipStream_t st)
{
    const ServeDims &d = a.d;
    // A workgroup per token where requests bring a few (each is a unit of its own), else one per block's worth of tokens: most
    // of them start one unit, and a workgroup per token would be started for nothing page - 1 times of page.
    const int window = d.max_q <= 8 ? 1 : d.page < 64 ? d.page : 64;
    const StoreParams kp{a.SEL, a.POOL, a.slot, a.sel_q8, a.pool_q8, a.scales, d.T, d.S, d.d_pool, d.d_sel, d.page, d.n_blocks, window, d.sel_row, d.pool_row};
    const unsigned grid = (unsigned)(((long)d.T + window - 1) / window * d.S);
    if (grid == 0) return hipSuccess;
    if (d.dtype == LCA_F16) page_store_kernel<f16_t><<<grid, 256, 0, st>>>(kp);
    else page_store_kernel<uint16_t><<<grid, 256, 0, st>>>(kp);
    return hipGetLastError();
}

}  // namespace lca
