// New keys and values into the paged 8-bit cache (include/lca_serve.h): one E4M3 code per element, one power-of-two scale
// per block of tokens, KV head and component.
//
// Unit = the tokens of one block in this call, one KV head; one wavefront takes a component of it, so that nobody else reads or
// writes its codes and scale, and nothing is shared but lanes.  The unit's new values are read once and held in registers
// from the largest magnitude to the codes (up to 8192 of them, 64 tokens of 128; larger units are read twice).  A power-of-two
// scale makes x / scale exact, the only rounding is the conversion's.  When the block's scale rises, the codes in front of the new
// tokens are converted again, old / new being a power of two as well: exact but for codes that leave E4M3's normal range.
// Keys: a lane takes sixteen columns of a token, 32 bytes in, 16 out.  Values lie sixteen tokens of a column next to each other: a lane
// takes sixteen tokens of a pair of columns, reads them four bytes at a time (a wavefront: 256 bytes of a row) and writes two
// whole 16-byte pieces; a piece that holds older tokens, or places behind the new ones, is read first and keeps them.
// Bound by memory: two bytes read and one written per element.  50064 tokens, 8 heads of 128 + 128, blocks of 64: 74 us, 4.16 TB/s (a copy: 4.75).
// 32 single tokens into blocks of 16: 5.3 to 5.8 us, latency.
#include "serve_internal.h"

namespace lca {
namespace {

struct StoreParams {
    const void *SEL, *POOL;
    const int32_t *slot;
    uint8_t *sel_q8, *pool_q8;
    float *scales;
    int T, S, d_pool, d_sel, page, n_blocks, window;       // window: packed rows a wavefront looks for starts of units in
    FastDiv by_pieces, by_pairs, by_S2, by_page;           // d_sel / 16, d_pool / 2, 2 S
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

// The unit's scale and what becomes of the older codes.
struct Scale { float value, inv, factor; bool raised; };
template <typename T> __device__ __forceinline__ Scale new_scale(float amax, float old, int off)
{
    const float fresh = ldexpf(1.f, scale_exponent<T>(lanes::over_group<64>(amax, lanes::Max())));
    Scale c;
    const bool keep = off > 0 && old >= fresh;
    c.value = keep ? old : fresh;
    c.inv = 1.f / c.value;
    c.raised = off > 0 && !keep;
    c.factor = old * c.inv;
    return c;
}
template <typename T> __device__ __forceinline__ float largest8(const uint4 &v, float m)     // (fmaxf drops a NaN)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<T>(w[i]);
        m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
    }
    return m;
}
template <typename T> __device__ __forceinline__ uint2 encode8(const uint4 &v, float inv)
{
    const float2 a = unpack2<T>(v.x), b = unpack2<T>(v.y), c = unpack2<T>(v.z), d = unpack2<T>(v.w);
    return uint2{encode4(in_range(a.x, inv), in_range(a.y, inv), in_range(b.x, inv), in_range(b.y, inv)),
                 encode4(in_range(c.x, inv), in_range(c.y, inv), in_range(d.x, inv), in_range(d.y, inv))};
}

constexpr int K_HELD = 8, V_HELD = 4;                      // items of a lane that registers hold

// Keys: item u = 16 columns of a new token.
template <typename T> __device__ __forceinline__ void store_keys(const StoreParams &kp, int t0, int block, int off, int n, int s, int lane)
{
    const size_t unit = (size_t)block * kp.S + s;
    const uint16_t *x = (const uint16_t *)kp.SEL + (size_t)t0 * kp.sel_row + (size_t)s * kp.d_sel;
    uint8_t *dst = kp.sel_q8 + (unit * kp.page + off) * kp.d_sel;
    float *scale = kp.scales + 2 * unit + 1;
    const int pieces = kp.d_sel / 16, total = n * pieces;
    const bool held = total <= 64 * K_HELD;
    auto source = [&](int u) {
        const int t = kp.by_pieces(u);
        return reinterpret_cast<const uint4 *>(x + (size_t)t * kp.sel_row + 16 * (u - t * pieces));
    };
    auto target = [&](int u) { return reinterpret_cast<uint4 *>(dst + 16 * (size_t)u); };      // (tokens of a block follow one another)
    uint4 a[K_HELD], b[K_HELD];
    float m = 0.f;
    const float old = off > 0 ? *scale : 0.f;
    if (held) {
#pragma unroll
        for (int i = 0; i < K_HELD; ++i) {
            a[i] = b[i] = make_uint4(0, 0, 0, 0);
            if (64 * i + lane < total) { const uint4 *p = source(64 * i + lane); a[i] = p[0]; b[i] = p[1]; }
        }
#pragma unroll
        for (int i = 0; i < K_HELD; ++i) m = largest8<T>(b[i], largest8<T>(a[i], m));
    } else {
        for (int u = lane; u < total; u += 64) { const uint4 *p = source(u); m = largest8<T>(p[1], largest8<T>(p[0], m)); }
    }
    const Scale c = new_scale<T>(m, old, off);
    auto put = [&](int u, const uint4 &lo, const uint4 &hi) {
        const uint2 e = encode8<T>(lo, c.inv), f = encode8<T>(hi, c.inv);
        *target(u) = make_uint4(e.x, e.y, f.x, f.y);
    };
    if (held) {
#pragma unroll
        for (int i = 0; i < K_HELD; ++i)
            if (64 * i + lane < total) put(64 * i + lane, a[i], b[i]);
    } else {
        for (int u = lane; u < total; u += 64) { const uint4 *p = source(u); put(u, p[0], p[1]); }
    }
    if (c.raised)                                          // the older tokens lie in front
        for (int u = -1 - lane; u >= -off * pieces; u -= 64) {
            const uint4 v = *target(u);
            *target(u) = make_uint4(recode4(v.x, c.factor), recode4(v.y, c.factor), recode4(v.z, c.factor), recode4(v.w, c.factor));
        }
    if (lane == 0) *scale = c.value;
}

// Values: item u = the sixteen tokens of a strip, two columns; strips from the first one with a new token on.
template <typename T> __device__ __forceinline__ void store_values(const StoreParams &kp, int t0, int block, int off, int n, int s, int lane)
{
    const size_t unit = (size_t)block * kp.S + s;
    const int first = off >> 4, pairs = kp.d_pool / 2, total = (((off + n - 1) >> 4) - first + 1) * pairs;
    const uint16_t *x = (const uint16_t *)kp.POOL + (size_t)s * kp.d_pool;
    uint8_t *dst = kp.pool_q8 + unit * kp.page * kp.d_pool;
    float *scale = kp.scales + 2 * unit;
    const bool held = total <= 64 * V_HELD;
    struct Item { uint32_t w[16]; uint4 old[2]; };         // new values of the places that have one, what the two pieces hold
    // places of strip `strip` that get a new token: [lo, hi)
    auto places = [&](int strip, int &lo, int &hi) { lo = off - 16 * strip; hi = lo + n; };
    auto target = [&](int strip, int pair) { return reinterpret_cast<uint4 *>(dst + ((size_t)strip * kp.d_pool + 2 * pair) * 16); };
    auto load = [&](int u, Item &it) {
        const int at = kp.by_pairs(u), strip = first + at, pair = u - at * pairs;
        int lo, hi;
        places(strip, lo, hi);
        const uint16_t *p = x + (size_t)(t0 - lo) * kp.pool_row + 2 * pair;          // of place 0 (read from the first new one on)
        if (lo <= 0 && hi >= 16) {
#pragma unroll
            for (int i = 0; i < 16; ++i) it.w[i] = *reinterpret_cast<const uint32_t *>(p + (size_t)i * kp.pool_row);
            it.old[0] = it.old[1] = make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) it.w[i] = i >= lo && i < hi ? *reinterpret_cast<const uint32_t *>(p + (ptrdiff_t)i * (ptrdiff_t)kp.pool_row) : 0;
            it.old[0] = target(strip, pair)[0];
            it.old[1] = target(strip, pair)[1];
        }
    };
    auto largest = [&](const Item &it, float m) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 f = unpack2<T>(it.w[i]);
            m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
        return m;
    };
    auto put = [&](int u, const Item &it, const Scale &c) {
        const int at = kp.by_pairs(u), strip = first + at, pair = u - at * pairs;
        int lo, hi;
        places(strip, lo, hi);
        unsigned o[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float2 f[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = unpack2<T>(it.w[4 * i + j]);
            o[0][i] = encode4(in_range(f[0].x, c.inv), in_range(f[1].x, c.inv), in_range(f[2].x, c.inv), in_range(f[3].x, c.inv));
            o[1][i] = encode4(in_range(f[0].y, c.inv), in_range(f[1].y, c.inv), in_range(f[2].y, c.inv), in_range(f[3].y, c.inv));
        }
        if (lo > 0 || hi < 16) {                           // older tokens (recoded if the scale rose) and places behind the new ones stay
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int from = min(max(lo - 4 * i, 0), 4), to = min(max(hi - 4 * i, 0), 4);
                const unsigned older = from == 4 ? 0xFFFFFFFFu : (1u << (8 * from)) - 1, upto = to == 4 ? 0xFFFFFFFFu : (1u << (8 * to)) - 1;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const unsigned h = i == 0 ? it.old[k].x : i == 1 ? it.old[k].y : i == 2 ? it.old[k].z : it.old[k].w;
                    const unsigned front = c.raised ? recode4(h, c.factor) : h;
                    o[k][i] = (front & older) | (o[k][i] & upto & ~older) | (h & ~(upto | older));
                }
            }
        }
        uint4 *p = target(strip, pair);
        p[0] = make_uint4(o[0][0], o[0][1], o[0][2], o[0][3]);
        p[1] = make_uint4(o[1][0], o[1][1], o[1][2], o[1][3]);
    };
    Item it[V_HELD];
    float m = 0.f;
    const float old = off > 0 ? *scale : 0.f;
    if (held) {
#pragma unroll
        for (int i = 0; i < V_HELD; ++i)
            if (64 * i + lane < total) load(64 * i + lane, it[i]);
            else
#pragma unroll
                for (int j = 0; j < 16; ++j) it[i].w[j] = 0;
#pragma unroll
        for (int i = 0; i < V_HELD; ++i) m = largest(it[i], m);
    } else {
        for (int u = lane; u < total; u += 64) { load(u, it[0]); m = largest(it[0], m); }
    }
    const Scale c = new_scale<T>(m, old, off);
    if (held) {
#pragma unroll
        for (int i = 0; i < V_HELD; ++i)
            if (64 * i + lane < total) put(64 * i + lane, it[i], c);
    } else {
        for (int u = lane; u < total; u += 64) { load(u, it[0]); put(u, it[0], c); }
    }
    if (c.raised)                                          // strips of older tokens alone
        for (int u = lane; u < first * kp.d_pool; u += 64) {
            uint4 *p = reinterpret_cast<uint4 *>(dst) + u;
            const uint4 v = *p;
            *p = make_uint4(recode4(v.x, c.factor), recode4(v.y, c.factor), recode4(v.z, c.factor), recode4(v.w, c.factor));
        }
    if (lane == 0) *scale = c.value;
}

// A wavefront takes the units that start among `window` packed rows, one KV head, one component.  A unit starts where a token's slot
// does not follow the slot of the token in front of it, or opens a block, and ends where either happens again.
template <typename T>
__global__ __launch_bounds__(256) void page_store_kernel(const StoreParams kp)
{
    const int lane = threadIdx.x & 63;
    const int job = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);     // (T * S < 2^30)
    const int win = kp.by_S2(job), s = (job - win * 2 * kp.S) >> 1;
    const bool keys = (job & 1) != 0;
    const int slots = kp.n_blocks * kp.page;
    const int lo = win * kp.window, hi = min(lo + kp.window, kp.T);          // at most 64 rows
    const int t = lo + lane;
    const int mine = t < hi ? kp.slot[t] : -1, before = t < hi && t > 0 ? kp.slot[t - 1] : -1;
    const bool valid = (unsigned)mine < (unsigned)slots;
    unsigned long long starts = __builtin_amdgcn_ballot_w64(valid && (mine == kp.by_page(mine) * kp.page || before < 0 || mine != before + 1));
    for (; starts != 0; starts &= starts - 1) {
        const int at = __builtin_ctzll(starts), first = __builtin_amdgcn_readlane(mine, at), t0 = lo + at;
        const int block = kp.by_page(first), off = first - block * kp.page;
        const int most = min(kp.page - off, kp.T - t0);                      // >= 1
        int n = 0;
        for (;;) {                                                           // tokens of the unit, 64 at a time
            const int k = n + lane;
            const unsigned long long follow = __builtin_amdgcn_ballot_w64(k < most && kp.slot[t0 + min(k, most - 1)] == first + k);
            const int run = follow == ~0ull ? 64 : __builtin_ctzll(~follow);
            n += run;
            if (run < 64) break;
        }
        if (keys) store_keys<T>(kp, t0, block, off, n, s, lane);
        else store_values<T>(kp, t0, block, off, n, s, lane);
    }
}

// Rows of a wavefront's window.  A unit takes it about 2.8 us, one after the other, and a wavefront that finds none 1.5 ns of the chip's time, so that
// the better window is as long as the runs of new tokens: 64 requests of 8 tokens, 8 heads, 19.5 us with one row, 6.5 with four, 5.4 with eight, 24.5 with 64;
// 32 of one token 5.0, 13.2, 24.3, 89; 8 of 2000, blocks of 64, 162, 110, 99, 25.  Units of a window: those of runs of max_q tokens (or blocks), and
// as many shorter ones as the batch can hold (of B requests T / max_q are long).
int make_window(const ServeDims &d)
{
    const int run = d.max_q < d.page ? d.max_q : d.page, shorter = d.B - (int)((d.T + d.max_q - 1) / d.max_q);
    int best = 1;
    float least = INFINITY;
    for (int w = 1; w <= 64; w *= 2) {
        const float units = (float)(shorter < 0 ? 0 : shorter < w ? shorter : w) + (float)w / (float)run;
        const float time = 2.8f * units + 1.5e-3f * 2.f * (float)d.T * (float)d.S / (float)w;
        if (time < least) { least = time; best = w; }
    }
    return best;
}

}  // namespace

hipError_t launch_page_store_q8(const StoreArgs &a, hipStream_t st)
{
    const ServeDims &d = a.d;
    const int window = make_window(d);
    const StoreParams kp{a.SEL, a.POOL, a.slot, a.sel_q8, a.pool_q8, a.scales, d.T, d.S, d.d_pool, d.d_sel, d.page, d.n_blocks, window,
                         FastDiv(d.d_sel / 16), FastDiv(d.d_pool / 2), FastDiv(2 * d.S), d.by_page, d.sel_row, d.pool_row};
    const unsigned grid = (unsigned)((((long)d.T + window - 1) / window * d.S * 2 + 3) / 4);
    if (grid == 0) return hipSuccess;
    if (d.dtype == LCA_F16) page_store_kernel<f16_t><<<grid, 256, 0, st>>>(kp);
    else page_store_kernel<uint16_t><<<grid, 256, 0, st>>>(kp);
    return hipGetLastError();
}

}  // namespace lca
