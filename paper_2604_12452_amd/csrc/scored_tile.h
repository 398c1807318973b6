// Scored attention of many rows (include/lca_serve.h) on the matrix cores: packed prompts (scored_tile.hip), and chunks of
// prompts over the paged 8-bit cache (scored_tile_paged.hip).
//
// The (row, query head) pairs of a request and KV head are columns, row after row, whatever the number of heads: a wavefront
// takes 32 of them, and a workgroup's wavefronts (four, over the cache eight) share the tiles of 64 keys and values in LDS.
//   S^T[key, column] = K Q^T      32x32x16 MFMAs, A = keys from LDS, B = the queries, in registers throughout
//   O^T[dv, column] += V^T P^T    A = values, B = P^T = exp2(S^T - m)
// A lane holds 16 of 32 scores of one column (the lane 32 further the others), so that maxima and sums are the lane's own
// but for one exchange, and masks, bias and positions are per lane.  Row m of S^T's 32 is key pi(m), pi exchanging bits 2
// and 3, which makes the registers of S^T the B fragments of the second product as they are.
// Tiles of packed rows are copied into LDS by buffer loads (rows behind the document's end, and columns behind the
// width, read as zeros); tiles of the cache go through registers, where the codes are converted.  16-byte pieces of a row are
// permuted by the row, so that neither the key reads nor the transposing value reads meet on a bank.
// Software pipeline over halves of 32 keys: a slot takes the weights of half H while the matrix core adds the values of half
// H - 1 and computes the scores of half H + 1.  Keys and values have two buffers each, one barrier between the two slots of a tile:
// behind it the next tile's keys are read for the first time, and everybody is done with the last tile's values.  Two
// workgroups of a CU fill each other's waits.
// Tiles are taken from the rows' own positions backwards.  The first one that a column sees anything of gives its reference,
// the largest score there; tiles that the whole wavefront sees then need no maximum: weights are 2^(score - reference)
// whatever they are.  When a sum of them passes 2^10 the references are raised with the next tile.  fp16 ends at 2^16, and a
// sum beyond 2^15 makes the workgroup repeat the item with a maximum for every half; bf16's end is fp32's (a column that
// gets there is computed row by row, like every one that does not come out as finite numbers).
// Sums are in fp32 of the weights before they are rounded.
// Bound by the matrix core and the vector ALU, which take turns more than they overlap.  16384 tokens in three documents, 16 heads over 4, 192 / 128:
// 0.48 ms, 1.11 PFLOP/s (matrix core 59 % of the cycles, vector ALU 43 %; a plain product of 16384^3 reaches 1.33).  8192 tokens, 32 heads over 8, 128 / 128,
// capped: 0.60 to 0.65 ms, 0.9 PFLOP/s (42 and 67 %).  Over the cache, 700 rows against 9000 tokens and five smaller requests, 32 heads over 8: 167 us, 0.61 PFLOP/s.
#pragma once
#include <algorithm>
#include <type_traits>
#include <utility>

#include "serve_row.h"

namespace lca {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));

// Nothing is scheduled across.
#define LCA_FENCE() __builtin_amdgcn_sched_barrier(0)

__device__ __forceinline__ floatx16 mfma_32x32x16(bf16x8 a, bf16x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx16 mfma_32x32x16(f16x8 a, f16x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ bf16x4 lds_read_tr16(__attribute__((address_space(3))) bf16x4 *p) { return __builtin_amdgcn_ds_read_tr16_b64_v4bf16(p); }
__device__ __forceinline__ f16x4 lds_read_tr16(__attribute__((address_space(3))) f16x4 *p)
{
    typedef __fp16 fp16x4 __attribute__((__vector_size__(4 * sizeof(__fp16))));     // the builtin's own spelling of four halves
    return __builtin_bit_cast(f16x4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) fp16x4 *)p));
}

template <typename E> struct Store;
template <> struct Store<__bf16> { typedef uint16_t type; };
template <> struct Store<_Float16> { typedef f16_t type; };

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
template <typename E> __device__ __forceinline__ uint4 convert8(unsigned lo, unsigned hi, float scale)
{
    return make_uint4(convert2<E>(lo, scale, false), convert2<E>(lo, scale, true), convert2<E>(hi, scale, false), convert2<E>(hi, scale, true));
}

// f(0), f(1), .. with the numbers as constants.
template <int... I, typename F> __device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F &&f) { (f(std::integral_constant<int, I>()), ...); }
template <int N, typename F> __device__ __forceinline__ void each(F &&f) { each_of(std::make_integer_sequence<int, N>(), f); }

struct TileParams {
    const void *Q, *SEL, *POOL;
    void *O;
    float *lse;
    const int32_t *q_start, *seq_len, *prefix_len, *block_table;
    const float *slopes;
    const uint8_t *sel_q8, *pool_q8;
    const float *scales;
    ServeDims d;
    ScoreRule rule;
    int items;                                    // numbers of work items, per KV head
    bool by_slots;                                // how they are counted (request_of_item)
    int least;                                    // requests of fewer (row, head) pairs per KV head are another kernel's
    int parts;                                    // workgroups of an item
    FastDiv by_parts, by_units;                   // items * S
    float *part;                                  // their results, [slot, KV head, part, BM, DV + 2]
};

// Wavefronts per workgroup (32 columns each): over the cache eight, so that a tile's codes are converted for 256 columns, unless
// the width takes the registers of two wavefronts per SIMD (the chunks above 187 us, 210 with four, before later steps).
constexpr int wavefronts(bool paged, int dv) { return paged && dv <= 128 ? 8 : 4; }
constexpr int BN = 64;                            // keys of a tile
constexpr int LEAST_TILES = 8;                    // of a part
constexpr float LAZY = 8.f;                       // where maxima are taken, the reference may lag them this much (base 2)
// A lane's 16 weights of a half may add up to this: in fp16 none of them is then beyond 65504; fp32 and bf16 end at 2^127.  Past
// CALM the references are brought up with the next tile.
template <typename E> struct Limit { static constexpr float value = 0x1p100f; };
template <> struct Limit<_Float16> { static constexpr float value = 0x1p15f; };
constexpr float CALM = 0x1p10f;
constexpr int RSRC_WORD3 = 0x00020000;            // raw buffer of dwords, gfx9 layout
constexpr unsigned NOWHERE = 0x80000000u;         // a buffer offset behind every end

__device__ __forceinline__ constexpr int pi(int m) { return (m & 0x13) | ((m & 4) << 1) | ((m & 8) >> 1); }
// Where 16-byte piece c of a row lies: c ^ key(row).  Keys: the 32 rows of an MFMA operand (or 16 of them) on different
// banks; values: four rows, two 16-column tiles each.
template <int D> __device__ __forceinline__ int key_swizzle(int row) { return D % 128 == 0 ? row & 15 : (row >> 1) & 7; }
template <int D> __device__ __forceinline__ int value_swizzle(int row) { return D % 128 == 0 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; }

__device__ __forceinline__ unsigned lds_address(const void *p) { return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const char *)p; }

// 64 x 16 bytes from buffer offsets `voff` of the lanes into LDS bytes [at, at + 1024).  Inline assembly because the
// compiler would make every later LDS read wait for a load into LDS that it knows of; the waits are by hand.
// Up to four of them follow one another: the instruction's offset moves both ends, and the lanes' offsets take it back (they
// are counted from COPY_ROOM bytes in front of the buffer for that).
constexpr int COPY_ROOM = 3 * 1024;
template <int N> __device__ __forceinline__ void copies(const unsigned *voff, const int4v &rs, unsigned at)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(voff[0]), "s"(rs), "s"(at) : "memory");
    if constexpr (N > 1) asm volatile("buffer_load_dwordx4 %0, %1, 0 offen offset:%2 lds" : : "v"(voff[1]), "s"(rs), "n"(1 * 1024) : "memory");
    if constexpr (N > 2) asm volatile("buffer_load_dwordx4 %0, %1, 0 offen offset:%2 lds" : : "v"(voff[2]), "s"(rs), "n"(2 * 1024) : "memory");
    if constexpr (N > 3) asm volatile("buffer_load_dwordx4 %0, %1, 0 offen offset:%2 lds" : : "v"(voff[3]), "s"(rs), "n"(3 * 1024) : "memory");
    if constexpr (N > 4) copies<N - 4>(voff + 4, rs, at + 4096);
}

// The request of work item x (counted from the first); 64 starts are looked at at a time.  Request b's items start at floor(q_start[b] * hps / BM) + b, which
// leaves each at least as many numbers as it has items; over the cache, where that is fewer numbers, at floor(q_start[b] * hps / 64): requests that are this
// kernel's have 65 columns and more, room for their items, and those before and after them, however many, take no numbers of theirs (256 requests of one
// token over 2000, max_q not known: 284 us, 357 by the first; 700 rows over 9000 tokens and five smaller requests 169.5, 166 by the first).
constexpr int SLOT = 64;
static_assert(PAGE_DECODE_COLUMNS >= SLOT, "floor(n / 64) >= ceil(n / 128) for n above 64");
template <int BM> __device__ __forceinline__ int request_of_item(const int32_t *q_start, const ServeDims &d, bool by_slots, int x, int lane, int &first)
{
    auto start = [&](int b) __attribute__((always_inline)) {
        const long column = (long)min(max(q_start[b], 0), d.T) * d.hps;
        return by_slots ? (int)(column / SLOT) : (int)(column / BM) + b;
    };
    int lo = 0, n = d.B;                          // the request is one of [lo, lo + n): the last that starts at or before x
    while (n > 1) {
        const int step = (n + 63) / 64, b = min(lo + lane * step, lo + n - 1);
        const unsigned long long at_or_before = __builtin_amdgcn_ballot_w64(lane * step < n && start(b) <= x);
        const int k = max(0, 63 - __builtin_clzll(at_or_before | 1));
        n = min(step, n - k * step);
        lo += k * step;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    first = start(lo);
    return lo;
}

// What an item's rows see, in tiles: [0, pre) and [from, ..), numbered one behind the other.
struct Tiles { int pre, from, count; };
template <int BM> __device__ __forceinline__ Tiles make_tiles(const ServeDims &d, const ScoreRule &rule, const Request &r, int c_first, int columns)
{
    const int lo = max(r.pos0 + d.by_hps(c_first), 0), hi = r.pos0 + d.by_hps(min(c_first + BM - 1, columns - 1));      // positions of its rows
    Tiles t;
    t.pre = hi >= 0 ? (r.prefix + BN - 1) / BN : 0;
    t.from = max(t.pre, (lo >= rule.window ? lo - rule.window + 1 : 0) / BN);
    t.count = t.pre + max((hi + BN) / BN - t.from, 0);
    return t;
}

// Where the parts of item k of a request lie (packed rows too: only documents of more than 64 LEAST_TILES rows are split).
__device__ __forceinline__ size_t slot_of(const ServeDims &d, const Request &r, int k) { return (size_t)((long)r.first * d.hps / SLOT + k); }

// A column that did not come out as finite numbers: again, over what its row sees alone (serve_row.h).
template <typename E, int DV, bool PAGED>
__device__ __forceinline__ void row_again(const TileParams &kp, const Request &r, int b, int s, int c, int lane)
{
    typedef typename Store<E>::type T;
    const ServeDims &d = kp.d;
    const int row = d.by_hps(c), head = s * d.hps + (c - row * d.hps), t = r.first + row;
    const T *q = (const T *)kp.Q + (size_t)t * d.q_row + (size_t)head * d.d_sel;
    T *O = (T *)kp.O + ((size_t)t * d.H + head) * d.d_pool;
    float *lse = kp.lse != nullptr ? kp.lse + (size_t)t * d.H + head : nullptr;
    const float slope = kp.slopes != nullptr ? kp.slopes[head] * LOG2E : 0.f;
    if constexpr (PAGED) {
        const PagedSource<T> src{kp.block_table + (size_t)b * d.max_blocks, kp.sel_q8, kp.pool_q8, kp.scales, d.page, d.n_blocks, d.S, s, d.d_sel, d.d_pool, d.by_page};
        scored_row<T, DV / 64>(src, q, r, r.pos0 + row, slope, kp.rule, d.d_sel, d.d_pool, O, lse, lane);
    } else {
        const PackedSource<T> src{(const T *)kp.SEL + (size_t)r.first * d.sel_row + (size_t)s * d.d_sel, (const T *)kp.POOL + (size_t)r.first * d.pool_row + (size_t)s * d.d_pool,
                                  d.sel_row, d.pool_row};
        scored_row<T, DV / 64>(src, q, r, r.pos0 + row, slope, kp.rule, d.d_sel, d.d_pool, O, lse, lane);
    }
}

template <typename E, int DK, int DV, bool PAGED, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * wavefronts(PAGED, DV), DV <= 128 ? 2 : 1) void scored_tile_kernel(const TileParams kp)
{
    typedef typename Store<E>::type T;
    typedef E ex8 __attribute__((ext_vector_type(8)));
    typedef E ex4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) ex4 *lds_b64_ptr;
    typedef const __attribute__((address_space(3))) ex8 *lds_b128_ptr;
    constexpr int NW = wavefronts(PAGED, DV), BM = 32 * NW, NKS = DK / 16, NDV = DV / 32;
    constexpr int RBK = 2 * DK, RBV = 2 * DV;     // bytes of a row of keys and of values in LDS
    constexpr int RBT = 2 * BN;                   // PAGED: the values lie transposed, a row per column
    constexpr int K_BYTES = BN * RBK, V_BYTES = BN * RBV, V_AT = 2 * K_BYTES;        // two buffers of keys, then two of values
    constexpr int K_COPIES = K_BYTES / 1024 / NW, V_COPIES = BN * RBV / 1024 / NW;
    static_assert(PAGED || (K_BYTES % (1024 * NW) == 0 && V_BYTES % (1024 * NW) == 0), "whole copies");
    extern __shared__ __attribute__((aligned(1024))) char lds[];

    const ServeDims &d = kp.d;
    const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, h32 = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // first part 0 of all items (every XCD has some of those that are not split); one KV head's items follow one another at a distance of S (an XCD sees
    // few heads), the last rows first
    const int part = kp.by_units((int)blockIdx.x), u = blockIdx.x - part * (kp.items * d.S), y = d.by_S(u), x = kp.items - 1 - y, s = u - y * d.S;
    int item0;
    const int b = request_of_item<BM>(kp.q_start, d, kp.by_slots, x, lane, item0);
    const Request r = make_request(kp.q_start, kp.seq_len, kp.prefix_len, b, d.T, d.max_blocks * d.page);
    const int columns = r.rows * d.hps, item = x - item0;
    if (item < 0 || item >= (columns + BM - 1) / BM || columns < kp.least) return;
    const int c_first = item * BM;

    // this lane's column
    const int c_lane = c_first + 32 * wave + n32, c = min(c_lane, columns - 1), row = d.by_hps(c), head = s * d.hps + (c - row * d.hps);
    const int pos = r.pos0 + row, pre_lane = pos >= 0 ? r.prefix : 0, lo_lane = pos >= kp.rule.window ? pos - kp.rule.window + 1 : 0;
    const float slope = kp.slopes != nullptr ? kp.slopes[head] * LOG2E : 0.f;
    // positions of the wavefront's and of the item's rows
    const int w_lo = __builtin_amdgcn_readfirstlane(r.pos0 + d.by_hps(min(c_first + 32 * wave, columns - 1)));
    const int w_hi = __builtin_amdgcn_readfirstlane(r.pos0 + d.by_hps(min(c_first + 32 * wave + 31, columns - 1)));
    const Tiles tiles = make_tiles<BM>(d, kp.rule, r, c_first, columns);
    const int per = max(LEAST_TILES, kp.by_parts(tiles.count + kp.parts - 1)), t_lo = part * per, n_tiles = min(tiles.count - t_lo, per);
    if (n_tiles <= 0 && part > 0) return;         // (nothing to see at all: part 0 writes it)
    const bool whole = n_tiles == tiles.count;
    // step t takes tile t_lo + t, counted backwards
    auto first_key = [&](int t) __attribute__((always_inline)) {
        const int k = tiles.count - 1 - t_lo - t;
        return (k < tiles.pre ? k : k - tiles.pre + tiles.from) * BN;
    };

    // Q^T fragments: lane (column, h) holds elements 16 k + 8 h .. + 7
    ex8 qf[NKS];
    {
        const E *qp = (const E *)kp.Q + (size_t)(r.first + row) * d.q_row + (size_t)head * d.d_sel + 8 * h32;
#pragma unroll
        for (int k = 0; k < NKS; ++k) qf[k] = 16 * k + 8 * h32 < d.d_sel ? *reinterpret_cast<const ex8 *>(qp + 16 * k) : ex8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < NKS; ++k) asm volatile("" : "+v"(qf[k]));          // here before the loop (its waits count copies)
    }

    // ---- tiles into LDS ----
    const unsigned lds0 = lds_address(lds);
    unsigned k_voff[PAGED ? 1 : K_COPIES], v_voff[PAGED ? 1 : V_COPIES];
    const char *k_base = nullptr, *v_base = nullptr;
    const unsigned k_row = (unsigned)d.sel_row * 2, v_row = (unsigned)d.pool_row * 2;
    if constexpr (!PAGED) {
        k_base = (const char *)kp.SEL + ((size_t)r.first * d.sel_row + (size_t)s * d.d_sel) * 2;
        v_base = (const char *)kp.POOL + ((size_t)r.first * d.pool_row + (size_t)s * d.d_pool) * 2;
#pragma unroll
        for (int i = 0; i < K_COPIES; ++i) {      // LDS row m of a block of 32 keys holds key pi(m)
            const int at = ((wave * K_COPIES + i) * 64 + lane) * 16, m = at / RBK, piece = (at % RBK / 16) ^ key_swizzle<DK>(m);
            k_voff[i] = 8 * piece < d.d_sel ? ((m & 32) + pi(m & 31)) * k_row + 16 * piece + COPY_ROOM - (i & 3) * 1024 : NOWHERE;
        }
#pragma unroll
        for (int i = 0; i < V_COPIES; ++i) {
            const int at = ((wave * V_COPIES + i) * 64 + lane) * 16, m = at / RBV, piece = (at % RBV / 16) ^ value_swizzle<DV>(m);
            v_voff[i] = 8 * piece < d.d_pool ? m * v_row + 16 * piece + COPY_ROOM - (i & 3) * 1024 : NOWHERE;
        }
    }
    // tile of keys j0 .. into buffer t & 1; `rows` of it lie behind the first
    auto copy_keys = [&](int t, int j0, int rows) __attribute__((always_inline)) {
        const unsigned long long at = (unsigned long long)k_base + (size_t)j0 * k_row - COPY_ROOM;
        const int4v rs = int4v{(int)(unsigned)at, (int)((unsigned)(at >> 32) & 0xFFFFu), (int)(rows * k_row + 2 * d.d_sel + COPY_ROOM), RSRC_WORD3};
        copies<K_COPIES>(k_voff, rs, lds0 + (t & 1) * K_BYTES + wave * K_COPIES * 1024);
    };
    auto copy_values = [&](int t, int j0, int rows) __attribute__((always_inline)) {
        const unsigned long long at = (unsigned long long)v_base + (size_t)j0 * v_row - COPY_ROOM;
        const int4v rs = int4v{(int)(unsigned)at, (int)((unsigned)(at >> 32) & 0xFFFFu), (int)(rows * v_row + 2 * d.d_pool + COPY_ROOM), RSRC_WORD3};
        copies<V_COPIES>(v_voff, rs, lds0 + V_AT + (t & 1) * V_BYTES + wave * V_COPIES * 1024);
    };
    // The cache: a thread takes 16 codes of a key, 16 tokens of a column; a tile's blocks are looked up a step before its
    // keys are loaded, its values follow a step behind.
    constexpr int K_TOTAL = BN * DK / 16, V_TOTAL = 4 * DV, THREADS = 64 * NW;
    constexpr int K_PIECES = PAGED ? (K_TOTAL + THREADS - 1) / THREADS : 1, V_PIECES = PAGED ? (V_TOTAL + THREADS - 1) / THREADS : 1;
    uint4 kreg[K_PIECES], vreg[V_PIECES];
    float k_scale[K_PIECES], v_scale[V_PIECES];
    int k_block = -1, v_block = -1;               // lane: block of strip lane & 3 of the next tile of keys and of values to be loaded
    unsigned valid = 0;                           // strips that exist, four bits a tile: of tile t in the lowest when step t begins
    const int strips = PAGED ? d.page >> 4 : 1, strip_end = (r.n + 15) >> 4;
    auto find_blocks = [&](int t) __attribute__((always_inline)) {
        const int strip = first_key(t) / 16 + (lane & 3);
        const int blk = kp.block_table[(size_t)b * d.max_blocks + d.by_strips(min(strip, strip_end - 1))];
        k_block = strip < strip_end && (unsigned)blk < (unsigned)d.n_blocks ? blk : -1;
    };
    // (a strip's DK or DV threads are whole wavefronts: its block and addresses are a wavefront's)
    auto load_keys = [&](int t) __attribute__((always_inline)) {
        const int strip0 = first_key(t) / 16;
#pragma unroll
        for (int i = 0; i < K_PIECES; ++i) {
            const int u = i * THREADS + tid, j = u / (DK / 16) & 15, piece = u % (DK / 16), st = (i * THREADS + 64 * wave) / DK, strip = strip0 + st;
            const size_t unit = (size_t)max(__builtin_amdgcn_readlane(k_block, st & 3), 0) * d.S + s;
            const uint8_t *at = kp.sel_q8 + (unit * d.page + (strip - d.by_strips(strip) * strips) * 16) * d.d_sel;
            kreg[i] = make_uint4(0, 0, 0, 0);
            if (st < 4 && 16 * piece < d.d_sel) kreg[i] = *reinterpret_cast<const uint4 *>(at + (unsigned)(j * d.d_sel + 16 * piece));
            k_scale[i] = kp.scales[2 * unit + 1];
        }
    };
    auto load_values = [&](int t) __attribute__((always_inline)) {
        const int strip0 = first_key(t) / 16;
#pragma unroll
        for (int i = 0; i < V_PIECES; ++i) {
            const int u = i * THREADS + tid, col = u % DV, st = (i * THREADS + 64 * wave) / DV, strip = strip0 + st;
            const int blk = __builtin_amdgcn_readlane(v_block, st & 3);
            const size_t unit = (size_t)max(blk, 0) * d.S + s;
            const uint8_t *at = kp.pool_q8 + (unit * strips + strip - d.by_strips(strip) * strips) * 16 * d.d_pool;
            vreg[i] = make_uint4(0, 0, 0, 0);
            if (st < 4 && col < d.d_pool && blk >= 0) vreg[i] = *reinterpret_cast<const uint4 *>(at + (unsigned)(16 * col));
            v_scale[i] = kp.scales[2 * unit];
        }
    };
    auto write_keys = [&](int t) __attribute__((always_inline)) {
        char *kb = lds + (t & 1) * K_BYTES;
#pragma unroll
        for (int i = 0; i < K_PIECES; ++i) {
            const int u = i * THREADS + tid, j = u / (DK / 16), piece = u % (DK / 16), m = (j & 32) + pi(j & 31);       // (pi is its own inverse)
            if (K_TOTAL % THREADS != 0 && u >= K_TOTAL) break;
            *reinterpret_cast<uint4 *>(kb + m * RBK + (((2 * piece) ^ key_swizzle<DK>(m)) << 4)) = convert8<E>(kreg[i].x, kreg[i].y, k_scale[i]);
            *reinterpret_cast<uint4 *>(kb + m * RBK + (((2 * piece + 1) ^ key_swizzle<DK>(m)) << 4)) = convert8<E>(kreg[i].z, kreg[i].w, k_scale[i]);
        }
    };
    auto write_values = [&](int t) __attribute__((always_inline)) {
        char *vb = lds + V_AT + (t & 1) * V_BYTES;
        const int strip0 = first_key(t) / 16;
#pragma unroll
        for (int i = 0; i < V_PIECES; ++i) {
            const int u = i * THREADS + tid, st = u / DV, col = u % DV, real = r.n - (strip0 + st) * 16;        // tokens of the strip that the request has
            if (V_TOTAL % THREADS != 0 && u >= V_TOTAL) break;
            if (real < 16) {
                unsigned w[4] = {vreg[i].x, vreg[i].y, vreg[i].z, vreg[i].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int keep = min(max(real - 4 * k, 0), 4);
                    w[k] &= keep == 4 ? 0xFFFFFFFFu : (1u << (8 * keep)) - 1;
                }
                vreg[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
            *reinterpret_cast<uint4 *>(vb + col * RBT + (((2 * st) ^ key_swizzle<BN>(col)) << 4)) = convert8<E>(vreg[i].x, vreg[i].y, v_scale[i]);
            *reinterpret_cast<uint4 *>(vb + col * RBT + (((2 * st + 1) ^ key_swizzle<BN>(col)) << 4)) = convert8<E>(vreg[i].z, vreg[i].w, v_scale[i]);
        }
    };

    // ---- operand reads ----
    // One LDS address per lane and operand: a fragment's is that one with a constant exchanged in the permuted bits of the piece's
    // number, plus a constant.  (Held as one address each and opaque to the compiler, which would otherwise keep them all, and has no registers for it.)
    constexpr int K_BITS = (DK % 128 == 0 ? 15 : 7) << 4;                      // the bits that key_swizzle touches, in bytes
    unsigned k_lane = lds0 + n32 * RBK + ((h32 ^ key_swizzle<DK>(n32)) << 4);
    unsigned v_lane;
    if constexpr (PAGED) {
        v_lane = lds0 + V_AT + n32 * RBT + ((h32 ^ key_swizzle<BN>(n32)) << 4);
    } else {
        // each 16 lanes: four keys (lane >> 2) by 16 columns (4 of a lane); lane c of them gets column c of the four
        const int key = 8 * h32 + ((lane >> 2) & 3), piece = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        v_lane = lds0 + V_AT + key * RBV + ((piece ^ value_swizzle<DV>(key)) << 4) + 8 * (lane & 1);
    }
    auto key_fragment = [&](unsigned base, auto HF, int k) __attribute__((always_inline)) {        // rows 32 half + n32, elements 16 k + 8 h ..
        const int c = 2 * k << 4;
        return *(lds_b128_ptr)(uintptr_t)((base ^ (c & K_BITS)) + (c & ~K_BITS) + 32 * HF * RBK);
    };
    auto value_fragment = [&](unsigned base, auto HF, int j, int v) __attribute__((always_inline)) {   // columns 32 v + n32, keys 32 half + 16 j + 8 h ..
        if constexpr (PAGED) {
            return *(lds_b128_ptr)(uintptr_t)((base ^ ((4 * HF + 2 * j) << 4)) + 32 * v * RBT);
        } else {
            constexpr int V_BITS = (DV % 128 == 0 ? 12 : 4) << 4;
            const int c = 4 * v << 4;
            const unsigned at = (base ^ (c & V_BITS)) + (c & ~V_BITS) + (32 * HF + 16 * j) * RBV;
            const ex4 lo = lds_read_tr16((lds_b64_ptr)(uintptr_t)at), hi = lds_read_tr16((lds_b64_ptr)(uintptr_t)(at + 4 * RBV));      // (key + 4: the same permutation)
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    };

    floatx16 acc[NDV];
#pragma unroll
    for (int v = 0; v < NDV; ++v)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[v][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f, m_seen = -INFINITY;
    bool unset = true;                            // (wave-uniform) a column has no reference yet
    bool over = false, again = false;             // a sum passed the limit; the item is being repeated

    floatx16 sv[2];                               // scores and weights of a tile's two halves
    uint4v pb[2][2];                              // (two weights a word)
    // S^T of half HF of tile t.  Register i of lane half h holds key 16 (i / 8) + 8 h + i % 8 of the 32.
    auto scores = [&](auto HF, int t) __attribute__((always_inline)) {
        unsigned kb = k_lane + (t & 1) * K_BYTES;
        asm volatile("" : "+v"(kb));
#pragma unroll
        for (int k = 0; k < NKS; ++k) sv[HF] = mfma_32x32x16(key_fragment(kb, HF, k), qf[k], k == 0 ? floatx16{} : sv[HF]);
    };
    auto add_values = [&](auto HF, int t) __attribute__((always_inline)) {
        unsigned vb = v_lane + (t & 1) * V_BYTES;
        asm volatile("" : "+v"(vb));
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < NDV; ++v) acc[v] = mfma_32x32x16(value_fragment(vb, HF, j, v), __builtin_bit_cast(ex8, pb[HF][j]), acc[v]);
    };
    auto pack = [&](float a, float b) __attribute__((always_inline)) {
        typedef E ex2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(unsigned, ex2{(E)a, (E)b});
    };
    // Any half: masked, with its maximum, the output rescaled where a reference grew.
    auto weights_masked = [&](auto HF, int j0) __attribute__((always_inline)) {
        const int jl = j0 + 8 * h32;
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int j = jl + (i & 7) + 16 * (i >> 3);
            float x = capped<CAP>(sv[HF][i], kp.rule);
            if constexpr (BIAS) x = fmaf(-slope, fabsf((float)(pos - j)), x);
            bool seen = (j >= lo_lane && j <= pos) || j < pre_lane;
            if constexpr (PAGED) seen = seen && (valid >> (2 * HF + (i >> 3)) & 1) != 0;
            sv[HF][i] = seen ? x : -INFINITY;
            mx = fmaxf(mx, sv[HF][i]);
        }
        mx = lanes::across32(fmaxf(mx, m_seen), lanes::Max());
        m_seen = -INFINITY;
        if (__builtin_amdgcn_ballot_w64(mx > m_run + LAZY) != 0) {
            const float m_new = fmaxf(m_run, mx), f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= f;
#pragma unroll
            for (int v = 0; v < NDV; ++v)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[v][i] *= f;
        }
        unset = __builtin_amdgcn_ballot_w64(m_run == -INFINITY) != 0;
        const float ref = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float p0 = __builtin_amdgcn_exp2f(sv[HF][i] - ref), p1 = __builtin_amdgcn_exp2f(sv[HF][i + 1] - ref);
            l_run += p0 + p1;
            pb[HF][i >> 3][(i & 7) >> 1] = pack(p0, p1);
        }
    };
    // Whether the whole wavefront sees all of tile t (of keys j0 ..), and all of it has references: it lies in front of every row and
    // in every row's window, or in the prefix (in front of the rows as well where the distance counts: it is taken without its sign).
    const int before = w_lo - BN + 1, window_from = w_hi - kp.rule.window, prefix_below = BIAS ? min(r.prefix - BN + 1, before + 1) : w_lo >= 0 ? r.prefix - BN + 1 : 0;
    auto is_fast = [&](int t, int j0) __attribute__((always_inline)) {
        bool fast = t + 1 < n_tiles && !unset && !again && ((j0 <= before && j0 > window_from) || j0 < prefix_below);
        if constexpr (PAGED) fast = fast && (valid & 0xF) == 0xF;
        return fast;
    };
    // Slot of half HF of a tile that is: weights to the references as they are.  A score goes through its stages in as many steps
    // (one MFMA each), so that nothing waits for the instruction in front of it: A its logit, with a cap the exponential in it,
    // B the cap's reciprocal, C the weight, D sum and rounding.  Operands are requested RING MFMAs ahead.  Returns the lane's sum.
    constexpr int MFMAS = NKS + 2 * NDV, RING = 3, LAST = CAP ? 3 : 2;
    auto fast_slot = [&](auto HF, int t, int j0) __attribute__((always_inline)) {
        constexpr int hf = decltype(HF)::value;
        constexpr std::integral_constant<int, hf ^ 1> OTHER;
        unsigned kb = k_lane + ((t + hf) & 1) * K_BYTES, vb = v_lane + ((t - 1 + hf) & 1) * V_BYTES;
        asm volatile("" : "+v"(kb), "+v"(vb));
        auto request = [&](int i) __attribute__((always_inline)) { return i < 2 * NDV ? value_fragment(vb, OTHER, i / NDV, i % NDV) : key_fragment(kb, OTHER, i - 2 * NDV); };
        ex8 ring[RING];
#pragma unroll
        for (int i = 0; i < RING; ++i) ring[i] = request(i);
        float sum[2] = {0.f, 0.f}, x[16];
        const float top = (CAP ? kp.rule.cap_log2 : 0.f) - m_run, bias = BIAS ? fmaf(slope, (float)(j0 + 32 * hf + 8 * h32 - pos), top) : top;
        LCA_FENCE();
        each<MFMAS>([&](auto I) __attribute__((always_inline)) {
            constexpr int i = decltype(I)::value;
            if constexpr (i < 2 * NDV) acc[i % NDV] = mfma_32x32x16(ring[i % RING], __builtin_bit_cast(ex8, pb[hf ^ 1][i / NDV]), acc[i % NDV]);
            else sv[hf ^ 1] = mfma_32x32x16(ring[i % RING], qf[i - 2 * NDV], i == 2 * NDV ? floatx16{} : sv[hf ^ 1]);
            if constexpr (i + RING < MFMAS) ring[i % RING] = request(i + RING);
            each<16>([&](auto C) __attribute__((always_inline)) {
                constexpr int c = decltype(C)::value, at = i - c * (MFMAS - LAST) / 16;        // steps since this score's first
                const float off = BIAS ? fmaf(slope, (float)((c & 7) + 16 * (c >> 3)), bias) : bias;
                if constexpr (at == LAST) {
                    sum[c & 1] += x[c];
                    if constexpr (c & 1) {
                        unsigned w = pack(x[c - 1], x[c]);
                        asm volatile("" : "+v"(w));                            // (here, and not where it is used)
                        pb[hf][c >> 3][(c & 7) >> 1] = w;
                    }
                }
                if constexpr (at == LAST - 1) x[c] = __builtin_amdgcn_exp2f(CAP ? fmaf(-2.f * kp.rule.cap_log2, x[c], off) : x[c]);
                if constexpr (CAP && at == 1) x[c] = __builtin_amdgcn_rcpf(1.f + x[c]);
                if constexpr (at == 0) x[c] = CAP ? __builtin_amdgcn_exp2f(sv[hf][c] * kp.rule.pre) : fmaf(sv[hf][c], kp.rule.scale_log2, off);
            });
            LCA_FENCE();
        });
        asm volatile("" : "+v"(sum[0]), "+v"(sum[1]));
        return sum[0] + sum[1];
    };
    auto slow_weights = [&](auto HF, int j0) __attribute__((always_inline)) {
        if (j0 + 32 * HF > w_hi && j0 + 32 * HF >= r.prefix) pb[HF][0] = pb[HF][1] = uint4v{0, 0, 0, 0};      // (wave-uniform) no column sees any of it
        else weights_masked(HF, j0 + 32 * HF);
    };
    // Between the slots of a tile.
    int j_next = 0;                               // first key of tile t + 1 (packed rows)
    auto exchange = [&](int t) __attribute__((always_inline)) {
        if constexpr (!PAGED) asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // this wavefront's part of keys t + 1 and values t has landed
        __syncthreads();                                                       // everybody's has, and everybody is done with keys t and values t - 1
        if constexpr (PAGED) {
            if (t + 2 < n_tiles) {
                write_keys(t + 2);
                v_block = k_block;
            }
            if (t + 1 < n_tiles) write_values(t + 1);
            if (t + 2 < n_tiles) load_values(t + 2);
            if (t + 3 < n_tiles) {
                find_blocks(t + 3);
                valid |= (unsigned)(__builtin_amdgcn_ballot_w64(k_block >= 0) & 0xF) << 12;
                load_keys(t + 3);
            }
        } else {
            // (only the first tile may end behind the document)
            if (t + 1 < n_tiles) copy_values(t + 1, j_next, BN - 1);
            j_next = first_key(t + 2);
            if (t + 2 < n_tiles) copy_keys(t + 2, j_next, BN - 1);
        }
    };
    constexpr std::integral_constant<int, 0> FIRST;
    constexpr std::integral_constant<int, 1> SECOND;

    auto run_tiles = [&]() __attribute__((always_inline)) {
        if constexpr (PAGED) {
            // keys 0 and 1 and values 0 go to LDS, keys 2 and values 1 are on their way
            valid = 0;
            for (int t = 0; t < 3 && t < n_tiles; ++t) {
                find_blocks(t);
                valid |= (unsigned)(__builtin_amdgcn_ballot_w64(k_block >= 0) & 0xF) << (4 * t);
                load_keys(t);
                if (t < 2) {
                    write_keys(t);
                    v_block = k_block;
                    load_values(t);
                    if (t == 0) write_values(0);
                }
            }
        } else {
            const int j0 = first_key(0), rows = min(r.n - j0, BN) - 1;
            j_next = first_key(1);
            copy_keys(0, j0, rows);
            copy_values(0, j0, rows);
            if (n_tiles > 1) copy_keys(1, j_next, BN - 1);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        __syncthreads();
        scores(FIRST, 0);
        for (int t = 0, j0 = first_key(0); t < n_tiles; ++t) {
            float s0 = 0.f, s1 = 0.f;
            bool calm = true;
#pragma clang loop unroll(disable)
            for (; is_fast(t, j0) && calm; ++t) {
                s0 = fast_slot(FIRST, t, j0);
                exchange(t);
                s1 = fast_slot(SECOND, t, j0);
                l_run += s0 + s1;
                if constexpr (std::is_same<E, _Float16>::value) over = over || !(s0 <= Limit<E>::value && s1 <= Limit<E>::value);
                calm = __builtin_amdgcn_ballot_w64(!(s0 + s1 <= CALM)) == 0;
                j0 = first_key(t + 1);
                valid >>= 4;
            }
            m_seen = s0 + s1 <= CALM ? -INFINITY : m_run + __builtin_amdgcn_logf(s0 > s1 ? s0 : s1);
            if (t > 0) add_values(SECOND, t - 1);
            scores(SECOND, t);
            slow_weights(FIRST, j0);
            exchange(t);
            add_values(FIRST, t);
            if (t + 1 < n_tiles) scores(FIRST, t + 1);
            slow_weights(SECOND, j0);
            j0 = first_key(t + 1);
            valid >>= 4;
        }
        add_values(SECOND, n_tiles - 1);
    };
    while (n_tiles > 0) {
        run_tiles();
        if (!std::is_same<E, _Float16>::value || again) break;
        int *flags = reinterpret_cast<int *>(lds);
        __syncthreads();
        if (tid < NW) flags[tid] = 0;
        __syncthreads();
        if (over) flags[wave] = 1;
        __syncthreads();
        int any = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) any |= flags[w];
        again = __builtin_amdgcn_readfirstlane(any) != 0;
        if (__builtin_expect(!again, 1)) break;
        __syncthreads();
        m_run = m_seen = -INFINITY;
        l_run = 0.f;
        unset = true;
#pragma unroll
        for (int v = 0; v < NDV; ++v)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[v][i] = 0.f;
    }

    // ---- output ----
    l_run = lanes::across32(l_run, lanes::Sum());
    if (!whole) {
        float *dst = kp.part + (((slot_of(d, r, item) * d.S + s) * kp.parts + part) * BM + 32 * wave + n32) * (DV + 2);
        if (h32 == 0) { dst[0] = m_run; dst[1] = l_run; }
#pragma unroll
        for (int v = 0; v < NDV; ++v)
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    *reinterpret_cast<float2 *>(dst + 2 + 32 * v + 8 * g + 4 * h32 + 2 * i) = float2{acc[v][4 * g + 2 * i], acc[v][4 * g + 2 * i + 1]};
        return;
    }
    const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
    const bool real = c_lane < columns;
    bool fine = true;
#pragma unroll
    for (int v = 0; v < NDV; ++v)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            acc[v][i] *= inv;
            fine = fine && fabsf(acc[v][i]) < INFINITY;
        }
    T *O = (T *)kp.O + ((size_t)(r.first + row) * d.H + head) * d.d_pool;
    float *lse = kp.lse != nullptr ? kp.lse + (size_t)(r.first + row) * d.H + head : nullptr;
    if (real) {
#pragma unroll
        for (int v = 0; v < NDV; ++v)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = 32 * v + 8 * g + 4 * h32;
                if (col < d.d_pool) {
                    const ex4 o = ex4{(E)acc[v][4 * g], (E)acc[v][4 * g + 1], (E)acc[v][4 * g + 2], (E)acc[v][4 * g + 3]};
                    *reinterpret_cast<ex4 *>(O + col) = o;
                }
            }
        if (lse != nullptr && h32 == 0) *lse = l_run == 0.f ? -INFINITY : (m_run + __builtin_amdgcn_logf(l_run)) * 0.6931471805599453f;
    }
    // columns that are not finite numbers: again, over what their rows see alone
    unsigned long long odd = __builtin_amdgcn_ballot_w64(real && !fine);
    odd = (odd | odd >> 32) & 0xFFFFFFFFull;
    for (; __builtin_expect(odd != 0, 0); odd &= odd - 1) {
        const int k = __builtin_ctzll(odd);
        row_again<E, DV, PAGED>(kp, r, b, s, c_first + 32 * wave + k, lane);
    }
}

// Joins the parts of every column of the items that have more than one: sixteen lanes a column, DV / 16 outputs each.
template <typename E, int DV, bool PAGED>
__global__ __launch_bounds__(256) void scored_merge_kernel(const TileParams kp)
{
    typedef typename Store<E>::type T;
    constexpr int N = DV / 16, BM = 32 * wavefronts(PAGED, DV);
    const ServeDims &d = kp.d;
    const int lane = threadIdx.x & 63, l16 = lane & 15, u = blockIdx.x / (BM / 16);
    const int k = (blockIdx.x % (BM / 16)) * 16 + (threadIdx.x >> 4);
    const int y = d.by_S(u), x = kp.items - 1 - y, s = u - y * d.S;
    int item0;
    const int b = request_of_item<BM>(kp.q_start, d, kp.by_slots, x, lane, item0);
    const Request r = make_request(kp.q_start, kp.seq_len, kp.prefix_len, b, d.T, d.max_blocks * d.page);
    const int columns = r.rows * d.hps, item = x - item0;
    if (item < 0 || item >= (columns + BM - 1) / BM || columns < kp.least) return;
    const int c_first = item * BM;
    const Tiles tiles = make_tiles<BM>(d, kp.rule, r, c_first, columns);
    const int per = max(LEAST_TILES, kp.by_parts(tiles.count + kp.parts - 1));
    if (tiles.count <= per) return;               // one part: it has written the output
    const int parts = (tiles.count + per - 1) / per, c = c_first + k;
    const float *src = kp.part + ((slot_of(d, r, item) * d.S + s) * kp.parts * BM + k) * (DV + 2);
    constexpr size_t STEP = (size_t)BM * (DV + 2);
    float m = -INFINITY, l = 0.f, sum[N];
    for (int p = l16; p < parts; p += 16) m = fmaxf(m, src[p * STEP]);
    m = lanes::over_group<16>(m, lanes::Max());
#pragma unroll
    for (int v = 0; v < N; ++v) sum[v] = 0.f;
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
        const float *part = src + p * STEP;
        const float2 ml = *reinterpret_cast<const float2 *>(part);
        const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
        l = fmaf(ml.y, f, l);
#pragma unroll
        for (int v = 0; v < N; v += 2) {
            const float2 w = *reinterpret_cast<const float2 *>(part + 2 + l16 * N + v);
            sum[v] = fmaf(w.x, f, sum[v]);
            sum[v + 1] = fmaf(w.y, f, sum[v + 1]);
        }
    }
    bool fine = true;
    if (c < columns) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int row = d.by_hps(c), head = s * d.hps + (c - row * d.hps);
        const size_t at = (size_t)(r.first + row) * d.H + head;
        T o[N];
#pragma unroll
        for (int v = 0; v < N; ++v) {
            const float w = sum[v] * inv;
            fine = fine && fabsf(w) < INFINITY;
            o[v] = from_float<T>(w);
        }
        T *O = (T *)kp.O + at * d.d_pool + l16 * N;
        // (widths are multiples of 8: pieces of 4 or 8 outputs lie inside or outside; of 16, half of one may)
#pragma unroll
        for (int v = 0; v < N; v += 8)
            if (l16 * N + v < d.d_pool) __builtin_memcpy(__builtin_assume_aligned(O + v, (N < 8 ? N : 8) * sizeof(T)), o + v, (N < 8 ? N : 8) * sizeof(T));
        if (kp.lse != nullptr && l16 == 0) kp.lse[at] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    }
    unsigned long long odd = __builtin_amdgcn_ballot_w64(!fine);
    while (__builtin_expect(odd != 0, 0)) {
        const int g = __builtin_ctzll(odd) >> 4;
        row_again<E, DV, PAGED>(kp, r, b, s, __builtin_amdgcn_readlane(c, 16 * g), lane);
        odd &= ~(0xFFFFull << (16 * g));
    }
}

// The widths kernels are built for: 64 / 64, 128 / 128, 192 / 128, 256 / 256.
constexpr int width_class(int dk, int dv) { return dk <= 64 && dv <= 64 ? 0 : dk <= 128 && dv <= 128 ? 1 : dk <= 192 && dv <= 128 ? 2 : 3; }
constexpr int CLASS_DV[4] = {64, 128, 128, 256};

// How a call is split, from its sizes and hints: items of BM columns, and where they alone do not fill the chip their tiles.
struct Plan { int items, parts; bool by_slots; };
Plan make_plan(const ServeDims &d, bool paged)
{
    const int BM = 32 * wavefronts(paged, CLASS_DV[width_class(d.d_sel, d.d_pool)]);
    Plan p;
    const int apart = (int)((long)d.T * d.hps / BM) + d.B, slots = (int)((long)d.T * d.hps / SLOT) + 1;
    p.by_slots = paged && slots < apart;
    p.items = p.by_slots ? slots : apart;
    const long keys = paged ? d.max_kv : d.max_q;
    const long tiles = std::max<long>(1, ((d.window > 0 ? std::min<long>(keys, (long)d.window + BM) : keys) + BN - 1) / BN);
    const long busy = std::max<long>(1, (long)d.T * d.hps / BM) * d.S;         // items that have work, about
    // As many workgroups as run at a time (eight wavefronts: one per CU, four: two), of eight tiles at least.  700 rows over 9000 tokens and five smaller
    // requests, 32 heads over 8: 167 us so (two parts), 215 with three, 193 with six: rounds that end with few of them.
    p.parts = (int)std::max<long>(1, std::min<long>(1024 / (BM / 32) * 2 / busy, tiles / LEAST_TILES));
    return p;
}

template <typename E, int DK, int DV, bool PAGED> void run(const TileParams &kp, hipStream_t st)
{
    constexpr size_t bytes = 2 * (size_t)BN * 2 * (DK + DV);
    constexpr int NW = wavefronts(PAGED, DV), BM = 32 * NW;
    const unsigned grid = (unsigned)((long)kp.items * kp.d.S * kp.parts);
    const bool cap = kp.rule.cap_log2 > 0.f, bias = kp.slopes != nullptr;
    if (cap && bias) scored_tile_kernel<E, DK, DV, PAGED, true, true><<<grid, 64 * NW, bytes, st>>>(kp);
    else if (cap) scored_tile_kernel<E, DK, DV, PAGED, true, false><<<grid, 64 * NW, bytes, st>>>(kp);
    else if (bias) scored_tile_kernel<E, DK, DV, PAGED, false, true><<<grid, 64 * NW, bytes, st>>>(kp);
    else scored_tile_kernel<E, DK, DV, PAGED, false, false><<<grid, 64 * NW, bytes, st>>>(kp);
    if (kp.parts > 1) scored_merge_kernel<E, DV, PAGED><<<(unsigned)((long)kp.items * kp.d.S * (BM / 16)), 256, 0, st>>>(kp);
}

template <typename E, bool PAGED> void run_widths(const TileParams &kp, hipStream_t st)
{
    switch (width_class(kp.d.d_sel, kp.d.d_pool)) {
    case 0: run<E, 64, 64, PAGED>(kp, st); break;
    case 1: run<E, 128, 128, PAGED>(kp, st); break;
    case 2: run<E, 192, 128, PAGED>(kp, st); break;
    default: run<E, 256, 256, PAGED>(kp, st); break;
    }
}

template <bool PAGED> hipError_t launch(const ScoredArgs &a, int least, hipStream_t st)
{
    const Plan p = make_plan(a.d, PAGED);
    const TileParams kp{a.Q, a.SEL, a.POOL, a.O, a.lse, a.q_start, a.seq_len, a.prefix_len, a.block_table, a.slopes, a.sel_q8, a.pool_q8, a.scales, a.d,
                        score_rule(a.d), p.items, p.by_slots, least, p.parts, FastDiv(p.parts), FastDiv((int)((long)p.items * a.d.S)), a.part};
    if (a.d.dtype == LCA_F16) run_widths<_Float16, PAGED>(kp, st);
    else run_widths<__bf16, PAGED>(kp, st);
    return hipGetLastError();
}

}  // namespace
}  // namespace lca
