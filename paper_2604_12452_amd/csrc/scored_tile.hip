// Scored attention of many rows (include/lca_serve.h) on the matrix cores: packed prompts, and chunks of prompts over the
// paged 8-bit cache.
//
// The (row, query head) pairs of a request and KV head are columns, row after row, whatever the number of heads: a wavefront
// takes 32 of them, a workgroup of four 128, and all of them share the tiles of 64 keys and values in LDS.
//   S^T[key, column] = K Q^T      32x32x16 MFMAs, A = keys from LDS, B = the queries, in registers throughout
//   O^T[dv, column] += V^T P^T    A = values, B = P^T = exp2(S^T - m)
// A lane holds 16 of 32 scores of one column (the lane 32 further the others), so that maxima and sums are the lane's own
// but for one exchange, and masks, bias and positions are per lane.  Row m of S^T's 32 is key pi(m), pi exchanging bits 2
// and 3, which makes the registers of S^T the B fragments of the second product as they are.
// Two workgroups of a CU fill each other's waits: while one's wavefront takes exponentials the other's has the matrix core.
// Tiles of packed rows are copied into LDS by buffer loads (rows behind the document's end, and columns behind the
// width, read as zeros); tiles of the cache go through registers, where the codes are converted.  Two stages, one barrier per tile.
// 16-byte pieces of a row are permuted by the row, so that neither the key reads nor the transposing value reads meet
// on a bank.
// Softmax with a running maximum that the output is rescaled for only when it grew by more than 2^8; sums in fp32 of the
// weights before they are rounded.
#include <algorithm>

#include "serve_row.h"

namespace lca {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef int int4v __attribute__((ext_vector_type(4)));

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
    int items;                                    // per KV head
    int least;                                    // requests of fewer (row, head) pairs per KV head are another kernel's
};

constexpr int NW = 4;                             // wavefronts per workgroup
constexpr int BM = 32 * NW;                       // columns of an item
constexpr int BN = 64;                            // keys of a tile
constexpr float LAZY = 8.f;                       // the running maximum may lag this much (base 2)
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
__device__ __forceinline__ void copy_1k(unsigned voff, const int4v &rs, unsigned at)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(voff), "s"(rs), "s"(at) : "memory");
}

// The request of work item x (counted from the first): request b's items start at floor(q_start[b] * hps / BM) + b, which leaves
// each at least as many numbers as it has items; 64 starts are looked at at a time.
__device__ __forceinline__ int request_of_item(const int32_t *q_start, const ServeDims &d, int x, int lane, int &first)
{
    auto start = [&](int b) { return (int)((long)min(max(q_start[b], 0), d.T) * d.hps / BM) + b; };
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

template <typename E, int DK, int DV, bool PAGED>
__global__ __launch_bounds__(64 * NW, DV <= 128 ? 2 : 1) void scored_tile_kernel(const TileParams kp)
{
    typedef typename Store<E>::type T;
    typedef E ex8 __attribute__((ext_vector_type(8)));
    typedef E ex4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) ex4 *lds_b64_ptr;
    constexpr int NKS = DK / 16, NDV = DV / 32;
    constexpr int RBK = 2 * DK, RBV = 2 * DV;     // bytes of a row of keys and of values in LDS
    constexpr int RBT = 2 * BN;                   // PAGED: the values lie transposed, a row per column
    constexpr int K_BYTES = BN * RBK, STAGE = K_BYTES + BN * RBV;
    constexpr int K_COPIES = K_BYTES / 1024 / NW, V_COPIES = BN * RBV / 1024 / NW;
    static_assert(K_BYTES % (1024 * NW) == 0 && (BN * RBV) % (1024 * NW) == 0, "whole copies");
    extern __shared__ __attribute__((aligned(1024))) char lds[];

    const ServeDims &d = kp.d;
    const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, h32 = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // one KV head's items follow one another at a distance of S (an XCD sees few heads), the last rows first
    const int x = kp.items - 1 - (int)(blockIdx.x / d.S), s = blockIdx.x % d.S;
    int item0;
    const int b = request_of_item(kp.q_start, d, x, lane, item0);
    const Request r = make_request(kp.q_start, kp.seq_len, kp.prefix_len, b, d.T, d.max_blocks * d.page);
    const int columns = r.rows * d.hps, c_first = (x - item0) * BM;
    if (x < item0 || c_first >= columns || columns < kp.least) return;

    // this lane's column
    const int c_lane = c_first + 32 * wave + n32, c = min(c_lane, columns - 1), row = c / d.hps, head = s * d.hps + (c - row * d.hps);
    const int pos = r.pos0 + row, pre_lane = pos >= 0 ? r.prefix : 0, lo_lane = pos >= kp.rule.window ? pos - kp.rule.window + 1 : 0;
    const float slope = kp.slopes != nullptr ? kp.slopes[head] * LOG2E : 0.f;
    // positions of the wavefront's and of the item's rows
    const int w_lo = __builtin_amdgcn_readfirstlane(r.pos0 + min(c_first + 32 * wave, columns - 1) / d.hps);
    const int w_hi = __builtin_amdgcn_readfirstlane(r.pos0 + min(c_first + 32 * wave + 31, columns - 1) / d.hps);
    const int i_lo = max(r.pos0 + c_first / d.hps, 0), i_hi = r.pos0 + min(c_first + BM - 1, columns - 1) / d.hps;
    // tiles that any row of the item sees: [0, pre) and [from, ..), numbered one behind the other
    const int pre_tiles = i_hi >= 0 ? (r.prefix + BN - 1) / BN : 0;
    const int from = max(pre_tiles, (i_lo >= kp.rule.window ? i_lo - kp.rule.window + 1 : 0) / BN);
    const int n_tiles = pre_tiles + max((i_hi + BN) / BN - from, 0);
    auto first_key = [&](int t) { return (t < pre_tiles ? t : t - pre_tiles + from) * BN; };

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
            k_voff[i] = 8 * piece < d.d_sel ? ((m & 32) + pi(m & 31)) * k_row + 16 * piece : NOWHERE;
        }
#pragma unroll
        for (int i = 0; i < V_COPIES; ++i) {
            const int at = ((wave * V_COPIES + i) * 64 + lane) * 16, m = at / RBV, piece = (at % RBV / 16) ^ value_swizzle<DV>(m);
            v_voff[i] = 8 * piece < d.d_pool ? m * v_row + 16 * piece : NOWHERE;
        }
    }
    auto issue_copies = [&](int t, int stage) {
        const int j0 = first_key(t), left = r.n - j0 - 1;                      // rows of the tile behind its first, to the document's end
        const unsigned long long ka = (unsigned long long)k_base + (size_t)j0 * k_row, va = (unsigned long long)v_base + (size_t)j0 * v_row;
        const int rows = min(left, BN - 1);
        const int4v ks = int4v{(int)(unsigned)ka, (int)((unsigned)(ka >> 32) & 0xFFFFu), (int)(rows * k_row + 2 * d.d_sel), RSRC_WORD3};
        const int4v vs = int4v{(int)(unsigned)va, (int)((unsigned)(va >> 32) & 0xFFFFu), (int)(rows * v_row + 2 * d.d_pool), RSRC_WORD3};
        const unsigned at = lds0 + stage * STAGE;
#pragma unroll
        for (int i = 0; i < K_COPIES; ++i) copy_1k(k_voff[i], ks, at + (wave * K_COPIES + i) * 1024);
#pragma unroll
        for (int i = 0; i < V_COPIES; ++i) copy_1k(v_voff[i], vs, at + K_BYTES + (wave * V_COPIES + i) * 1024);
    };
    // The cache: a thread takes 16 codes of a key, 16 tokens of a column; blocks are looked up a tile ahead.
    constexpr int K_PIECES = PAGED ? BN * DK / 16 / (64 * NW) : 1, V_PIECES = PAGED ? 4 * DV / (64 * NW) : 1;
    uint4 kreg[K_PIECES], vreg[V_PIECES];
    float k_scale[K_PIECES], v_scale[V_PIECES];
    int valid = 0xF, valid_next = 0xF;            // strips of 16 tokens of the tile that exist
    int strip_block = -1;                         // lane: block of strip lane & 3 of the tile to be loaded
    const int strips = PAGED ? d.page >> 4 : 1, strip_end = (r.n + 15) >> 4;
    auto find_blocks = [&](int t) {
        const int strip = first_key(t) / 16 + (lane & 3);
        const int blk = kp.block_table[(size_t)b * d.max_blocks + min(strip, strip_end - 1) / strips];
        strip_block = strip < strip_end && (unsigned)blk < (unsigned)d.n_blocks ? blk : -1;
    };
    auto load_codes = [&](int t) {
        const int strip0 = first_key(t) / 16;
        valid_next = (int)(__builtin_amdgcn_ballot_w64(strip_block >= 0) & 0xF);
#pragma unroll
        for (int i = 0; i < K_PIECES; ++i) {
            const int u = i * 64 * NW + tid, j = u / (DK / 16), piece = u % (DK / 16), strip = strip0 + (j >> 4);
            const int blk = __shfl(strip_block, j >> 4, 64);
            const size_t unit = (size_t)max(blk, 0) * d.S + s;
            kreg[i] = make_uint4(0, 0, 0, 0);
            if (16 * piece < d.d_sel) kreg[i] = *reinterpret_cast<const uint4 *>(kp.sel_q8 + (unit * d.page + (strip % strips) * 16 + (j & 15)) * d.d_sel + 16 * piece);
            k_scale[i] = kp.scales[2 * unit + 1];
        }
#pragma unroll
        for (int i = 0; i < V_PIECES; ++i) {
            const int u = i * 64 * NW + tid, strip = strip0 + u / DV, col = u % DV;
            const int blk = __shfl(strip_block, u / DV, 64);
            const size_t unit = (size_t)max(blk, 0) * d.S + s;
            vreg[i] = make_uint4(0, 0, 0, 0);
            if (col < d.d_pool && blk >= 0) {
                uint4 v = *reinterpret_cast<const uint4 *>(kp.pool_q8 + ((unit * strips + strip % strips) * d.d_pool + col) * 16);
                const int real = r.n - strip * 16;                             // tokens of the strip that the request has
                if (real < 16) {
                    unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int keep = min(max(real - 4 * k, 0), 4);
                        w[k] &= keep == 4 ? 0xFFFFFFFFu : (1u << (8 * keep)) - 1;
                    }
                    v = make_uint4(w[0], w[1], w[2], w[3]);
                }
                vreg[i] = v;
            }
            v_scale[i] = kp.scales[2 * unit];
        }
    };
    auto write_codes = [&](int stage) {
        char *kb = lds + stage * STAGE, *vb = kb + K_BYTES;
#pragma unroll
        for (int i = 0; i < K_PIECES; ++i) {
            const int u = i * 64 * NW + tid, j = u / (DK / 16), piece = u % (DK / 16), m = (j & 32) + pi(j & 31);       // (pi is its own inverse)
            *reinterpret_cast<uint4 *>(kb + m * RBK + (((2 * piece) ^ key_swizzle<DK>(m)) << 4)) = convert8<E>(kreg[i].x, kreg[i].y, k_scale[i]);
            *reinterpret_cast<uint4 *>(kb + m * RBK + (((2 * piece + 1) ^ key_swizzle<DK>(m)) << 4)) = convert8<E>(kreg[i].z, kreg[i].w, k_scale[i]);
        }
#pragma unroll
        for (int i = 0; i < V_PIECES; ++i) {
            const int u = i * 64 * NW + tid, st = u / DV, col = u % DV;
            *reinterpret_cast<uint4 *>(vb + col * RBT + (((2 * st) ^ key_swizzle<BN>(col)) << 4)) = convert8<E>(vreg[i].x, vreg[i].y, v_scale[i]);
            *reinterpret_cast<uint4 *>(vb + col * RBT + (((2 * st + 1) ^ key_swizzle<BN>(col)) << 4)) = convert8<E>(vreg[i].z, vreg[i].w, v_scale[i]);
        }
    };

    // ---- operand reads ----
    const int k_key = key_swizzle<DK>(n32);
    auto key_fragment = [&](const char *kb, int half, int k) {                 // rows 32 half + n32, elements 16 k + 8 h ..
        return *reinterpret_cast<const ex8 *>(kb + (32 * half + n32) * RBK + (((2 * k + h32) ^ k_key) << 4));
    };
    auto value_fragment = [&](const char *vb, int half, int j, int v) {        // columns 32 v + n32, keys 32 half + 16 j + 8 h ..
        if constexpr (PAGED) {
            const int col = 32 * v + n32;
            return *reinterpret_cast<const ex8 *>(vb + col * RBT + (((4 * half + 2 * j + h32) ^ key_swizzle<BN>(col)) << 4));
        } else {
            // each 16 lanes: four keys (lane >> 2) by 16 columns (4 of a lane); lane c of them gets column c of the four
            const int key = 32 * half + 16 * j + 8 * h32 + ((lane >> 2) & 3), piece = 4 * v + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
            const char *p = vb + key * RBV + ((piece ^ value_swizzle<DV>(key)) << 4) + 8 * (lane & 1);
            const ex4 lo = lds_read_tr16((lds_b64_ptr)p), hi = lds_read_tr16((lds_b64_ptr)(p + 4 * RBV));      // (key + 4: the same permutation)
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    };

    floatx16 acc[NDV];
#pragma unroll
    for (int v = 0; v < NDV; ++v)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[v][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;

    if (n_tiles > 0) {
        if constexpr (PAGED) {
            find_blocks(0);
            load_codes(0);
            valid = valid_next;
            write_codes(0);
            if (n_tiles > 1) { find_blocks(1); load_codes(1); }
            if (n_tiles > 2) find_blocks(2);
        } else {
            issue_copies(0, 0);
        }
    }
    for (int t = 0; t < n_tiles; ++t) {
        const int stage = t & 1;
        if constexpr (!PAGED) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wavefront's part of tile t has landed
        __syncthreads();                                                       // everybody's has, and everybody is done with tile t - 1
        if constexpr (!PAGED) {
            if (t + 1 < n_tiles) issue_copies(t + 1, stage ^ 1);
        }
        const char *kb = lds + stage * STAGE, *vb = kb + K_BYTES;
        const int j0 = first_key(t);
        const bool none = j0 > w_hi && j0 >= r.prefix;                         // (wave-uniform) no column sees any of it
        if (!none) {
            floatx16 sv[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sv[half][i] = 0.f;
#pragma unroll
                for (int k = 0; k < NKS; ++k) sv[half] = mfma_32x32x16(key_fragment(kb, half, k), qf[k], sv[half]);
            }
            // register i of lane half h holds key 16 (i / 8) + 8 h + i % 8 of the 32
            const bool full = (j0 + BN - 1 < r.prefix && w_lo >= 0) || (j0 + BN - 1 <= w_lo && w_hi - j0 < kp.rule.window);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (kp.rule.cap_log2 > 0.f) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) sv[half][i] = capped<true>(sv[half][i], kp.rule);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) sv[half][i] = capped<false>(sv[half][i], kp.rule);
                }
                const int jl = j0 + 32 * half + 8 * h32;
                if (kp.slopes != nullptr) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) sv[half][i] = fmaf(-slope, fabsf((float)(pos - jl - (i & 7) - 16 * (i >> 3))), sv[half][i]);
                }
                if (!full || (PAGED && valid != 0xF)) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int j = jl + (i & 7) + 16 * (i >> 3);
                        bool seen = (j >= lo_lane && j <= pos) || j < pre_lane;
                        if constexpr (PAGED) seen = seen && (valid >> (2 * half + (i >> 3)) & 1) != 0;
                        sv[half][i] = seen ? sv[half][i] : -INFINITY;
                    }
                }
            }
            float mx = fmaxf(sv[0][0], sv[1][0]);
#pragma unroll
            for (int i = 1; i < 16; ++i) mx = fmaxf(mx, fmaxf(sv[0][i], sv[1][i]));
            mx = lanes::across32(mx, lanes::Max());
            if (__builtin_amdgcn_ballot_w64(mx > m_run + LAZY) != 0) {
                const float m_new = fmaxf(m_run, mx), f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
                m_run = m_new;
                l_run *= f;
#pragma unroll
                for (int v = 0; v < NDV; ++v)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[v][i] *= f;
            }
            const float ref = m_run == -INFINITY ? 0.f : m_run;
            ex8 pb[2][2];
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float p = __builtin_amdgcn_exp2f(sv[half][i] - ref);
                    l_run += p;
                    pb[half][i >> 3][i & 7] = (E)p;
                }
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < NDV; ++v) acc[v] = mfma_32x32x16(value_fragment(vb, half, j, v), pb[half][j], acc[v]);
        }
        if constexpr (PAGED) {
            valid = valid_next;
            if (t + 1 < n_tiles) write_codes(stage ^ 1);                       // (everybody is done with tile t - 1: the barrier above)
            if (t + 2 < n_tiles) load_codes(t + 2);
            if (t + 3 < n_tiles) find_blocks(t + 3);
        }
    }

    // ---- output ----
    l_run = lanes::across32(l_run, lanes::Sum());
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
    unsigned long long again = __builtin_amdgcn_ballot_w64(real && !fine);
    again = (again | again >> 32) & 0xFFFFFFFFull;
    for (; __builtin_expect(again != 0, 0); again &= again - 1) {
        const int k = __builtin_ctzll(again), cc = c_first + 32 * wave + k, rr = cc / d.hps, hh = s * d.hps + (cc - rr * d.hps), tt = r.first + rr;
        const T *q = (const T *)kp.Q + (size_t)tt * d.q_row + (size_t)hh * d.d_sel;
        T *Or = (T *)kp.O + ((size_t)tt * d.H + hh) * d.d_pool;
        float *lr = kp.lse != nullptr ? kp.lse + (size_t)tt * d.H + hh : nullptr;
        const float sl = kp.slopes != nullptr ? kp.slopes[hh] * LOG2E : 0.f;
        if constexpr (PAGED) {
            const PagedSource<T> src{kp.block_table + (size_t)b * d.max_blocks, kp.sel_q8, kp.pool_q8, kp.scales, d.page, d.n_blocks, d.S, s, d.d_sel, d.d_pool};
            scored_row<T, DV / 64>(src, q, r, r.pos0 + rr, sl, kp.rule, d.d_sel, d.d_pool, Or, lr, lane);
        } else {
            const PackedSource<T> src{(const T *)kp.SEL + (size_t)r.first * d.sel_row + (size_t)s * d.d_sel, (const T *)kp.POOL + (size_t)r.first * d.pool_row + (size_t)s * d.d_pool,
                                      d.sel_row, d.pool_row};
            scored_row<T, DV / 64>(src, q, r, r.pos0 + rr, sl, kp.rule, d.d_sel, d.d_pool, Or, lr, lane);
        }
    }
}

template <typename E, int DK, int DV, bool PAGED> void run(const TileParams &kp, hipStream_t st)
{
    constexpr size_t bytes = 2 * (size_t)BN * 2 * (DK + DV);
    scored_tile_kernel<E, DK, DV, PAGED><<<(unsigned)((long)kp.items * kp.d.S), 64 * NW, bytes, st>>>(kp);
}

template <typename E, bool PAGED> void run_widths(const TileParams &kp, hipStream_t st)
{
    const int dk = kp.d.d_sel, dv = kp.d.d_pool;
    if (dk <= 64 && dv <= 64) run<E, 64, 64, PAGED>(kp, st);
    else if (dk <= 128 && dv <= 128) run<E, 128, 128, PAGED>(kp, st);
    else if (dk <= 192 && dv <= 128) run<E, 192, 128, PAGED>(kp, st);
    else run<E, 256, 256, PAGED>(kp, st);
}

}  // namespace

bool scored_tile_supported(const ServeDims &d)
{
    // (64 rows of a tile lie within the 2^31 bytes of a buffer descriptor)
    return d.dtype != LCA_F32 && d.d_sel <= 256 && d.d_pool <= 256 && d.sel_row < (1u << 23) && d.pool_row < (1u << 23);
}

hipError_t launch_scored_tile(const ScoredArgs &a, int least, hipStream_t st)
{
    const int items = (int)((long)a.d.T * a.d.hps / BM) + a.d.B;
    const TileParams kp{a.Q, a.SEL, a.POOL, a.O, a.lse, a.q_start, a.seq_len, a.prefix_len, a.block_table, a.slopes, a.sel_q8, a.pool_q8, a.scales, a.d,
                        score_rule(a.d), items, least};
    if (a.block_table != nullptr) {
        if (a.d.dtype == LCA_F16) run_widths<_Float16, true>(kp, st);
        else run_widths<__bf16, true>(kp, st);
    } else {
        if (a.d.dtype == LCA_F16) run_widths<_Float16, false>(kp, st);
        else run_widths<__bf16, false>(kp, st);
    }
    return hipGetLastError();
}

}  // namespace lca
