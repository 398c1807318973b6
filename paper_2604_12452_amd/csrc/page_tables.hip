// Block tables, slots and positions of a serving step on the GPU, and the release of finished requests' blocks
// (include/lca_serve.h).
//
// Requests: two prefix sums (rows, then blocks of those that fit) by one workgroup, 1024 requests at a time.  The sums are
// of numbers >= 0 that matter up to a limit only (T, the pool), so they saturate one above it and stay in 32 bits.
// Tokens: each finds its request among the starts and writes its slot, position and request; the first token of a new
// block also writes the block table, so that nothing walks the requests' blocks one after another.
// What bounds it is latency (a decode step moves a kilobyte), so there is one launch: every workgroup takes the sums of all requests
// for itself, into LDS, and then 1024 tokens (1000 requests, 131072 rows: 7 us, 9 in two launches).  Two launches are left for more requests than LDS
// holds, and for a free_left that is free_count itself, which the workgroups behind the first would still read.
#include <algorithm>

#include "serve_internal.h"

namespace lca {
namespace {

struct TablesParams {
    const int32_t *cached_len, *new_len, *free_list, *free_count;
    int32_t *free_left, *block_table, *q_start, *seq_len, *slot, *position, *request, *base;
    int B, T, page, n_blocks, max_blocks;
    FastDiv by_page;
};

constexpr int REFUSED = -1;                       // base of a request that gets nothing

// Inclusive prefix sum over the workgroup, saturating at `limit` (values >= 0, each <= limit, limit <= 2^30: two of them fit 32 bits without a sign).
__device__ __forceinline__ int add_up_to(int a, int b, int limit) { return (int)min((unsigned)a + (unsigned)b, (unsigned)limit); }
template <int WAVES> __device__ __forceinline__ int scan_up_to(int v, int limit, int *lds, int tid)
{
    const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int w = __shfl_up(v, o, 64);
        if (lane >= o) v = add_up_to(v, w, limit);
    }
    if constexpr (WAVES == 1) return v;
    if (lane == 63) lds[wave] = v;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
        if (w < wave) before = add_up_to(before, lds[w], limit);
    __syncthreads();
    return add_up_to(v, before, limit);
}

// A token's slot and request: t < T, b its request (its first row, its base) or -1.
__device__ __forceinline__ void write_token(const TablesParams &kp, int t, int b, int first, int base)
{
    int slot = -1, position = 0;
    if (b >= 0) {
        const int cached = max(kp.cached_len[b], 0);
        position = (int)((unsigned)cached + (unsigned)(t - first));
        if (base != REFUSED) {
            const int col = kp.by_page(position), have = kp.by_page(cached + kp.page - 1);
            int32_t *entry = kp.block_table + (size_t)b * kp.max_blocks + col;
            int block;
            if (col >= have) {                    // (0 <= base - (col - have): the stack held the request's blocks)
                block = kp.free_list[base - (col - have)];
                if (position == col * kp.page) *entry = block;
            } else {
                block = *entry;
            }
            if ((unsigned)block < (unsigned)kp.n_blocks) slot = block * kp.page + position - col * kp.page;
        }
    }
    kp.slot[t] = slot;
    kp.position[t] = position;
    kp.request[t] = b;
}

// The sums over all requests by one workgroup; put(b, rows up to and including b, seq_len, base) for each, the blocks taken returned to thread 0 as
// what is left.
template <int WAVES, typename Put> __device__ __forceinline__ int take_requests(const TablesParams &kp, int *lds, int tid, Put &&put)
{
    __shared__ int carry[2];
    const int T1 = kp.T + 1, P1 = kp.n_blocks + 1;
    const int free = min(max(kp.free_count[0], 0), kp.n_blocks);
    int rows = 0, blocks = 0, taken = 0;          // of the requests in front of this round
    for (int b0 = 0; b0 < kp.B; b0 += WAVES * 64) {
        const int b = b0 + tid;
        const bool real = b < kp.B;
        const int cached = real ? kp.cached_len[b] : 0, asked = real ? kp.new_len[b] : 0;
        const int add = min(max(asked, 0), T1);
        const int end = add_up_to(scan_up_to<WAVES>(add, T1, lds, tid), rows, T1);
        const long total = (long)cached + add;
        const bool fits = real && cached >= 0 && asked >= 0 && end <= kp.T && total <= (long)kp.max_blocks * kp.page;
        const int have = fits ? kp.by_page(cached + kp.page - 1) : 0;
        const int need = fits ? min(kp.by_page((int)total + kp.page - 1) - have, P1) : 0;
        const int upto = add_up_to(scan_up_to<WAVES>(need, P1, lds, tid), blocks, P1);
        const bool ok = fits && (need == 0 || upto <= free);
        if (real) put(b, min(end, kp.T), ok ? (int)total : 0, ok ? max(free - 1 - (upto - need), 0) : REFUSED);      // (needs none: any base but REFUSED)
        if (ok && need > 0) taken = upto;
        if (kp.B > b0 + WAVES * 64) {             // the last thread's sums go to all for the next round
            if (tid == WAVES * 64 - 1) { carry[0] = end; carry[1] = upto; }
            __syncthreads();
            rows = carry[0];
            blocks = carry[1];
            __syncthreads();
        }
    }
    // blocks taken: cum_b of the last request that got any (the sums only grow)
    for (int o = 32; o >= 1; o >>= 1) taken = max(taken, __shfl_xor(taken, o, 64));
    if constexpr (WAVES > 1) {
        if ((tid & 63) == 0) lds[tid >> 6] = taken;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) taken = max(taken, lds[w]);
    }
    return free - taken;
}

// Up to MOST requests, whose starts and bases stay in LDS; each workgroup every gridDim.x-th WAVES * 64 tokens.
template <int WAVES, int MOST> __global__ __launch_bounds__(WAVES * 64) void tables_kernel(const TablesParams kp)
{
    __shared__ int lds[WAVES], start[MOST + 1], base[MOST];
    const int tid = threadIdx.x;
    const bool first = blockIdx.x == 0;
    if (tid == 0) {
        start[0] = 0;
        if (first) kp.q_start[0] = 0;
    }
    const int left = take_requests<WAVES>(kp, lds, tid, [&](int b, int end, int len, int at) {
        start[b + 1] = end;
        base[b] = at;
        if (first) {
            kp.q_start[b + 1] = end;
            kp.seq_len[b] = len;
        }
    });
    if (first && tid == 0) kp.free_left[0] = left;
    __syncthreads();
    for (int t = blockIdx.x * (WAVES * 64) + tid; t < kp.T; t += gridDim.x * (WAVES * 64)) {
        const int b = request_of(start, kp.B, t);
        write_token(kp, t, b, b >= 0 ? start[b] : 0, b >= 0 ? base[b] : 0);
    }
}

__global__ __launch_bounds__(1024) void tables_requests_kernel(const TablesParams kp)
{
    __shared__ int lds[16];
    const int tid = threadIdx.x;
    if (tid == 0) kp.q_start[0] = 0;
    const int left = take_requests<16>(kp, lds, tid, [&](int b, int end, int len, int at) {
        kp.q_start[b + 1] = end;
        kp.seq_len[b] = len;
        kp.base[b] = at;
    });
    if (tid == 0) kp.free_left[0] = left;
}

__global__ __launch_bounds__(256) void tables_tokens_kernel(const TablesParams kp)
{
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= kp.T) return;
    const int b = request_of(kp.q_start, kp.B, t);
    write_token(kp, t, b, b >= 0 ? kp.q_start[b] : 0, b >= 0 ? kp.base[b] : 0);
}

struct ReleaseParams {
    const int32_t *finished;
    int32_t *cached_len, *block_table, *free_list, *free_count;
    int B, page, n_blocks, max_blocks;
};

// One workgroup: finished requests in order (64 flags at a time), the entries of one 1024 at a time (a ballot and a sum
// over the wavefronts say where each goes on the stack).
__global__ __launch_bounds__(1024) void release_kernel(const ReleaseParams kp)
{
    __shared__ int counts[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int top = min(max(kp.free_count[0], 0), kp.n_blocks);
    for (int b0 = 0; b0 < kp.B; b0 += 64) {
        unsigned long long todo = __builtin_amdgcn_ballot_w64(b0 + lane < kp.B && kp.finished[min(b0 + lane, kp.B - 1)] != 0);
        for (; todo != 0; todo &= todo - 1) {
            const int b = b0 + __builtin_ctzll(todo);
            const int held = min((int)(((long)max(kp.cached_len[b], 0) + kp.page - 1) / kp.page), kp.max_blocks);
            for (int c0 = 0; c0 < held; c0 += 1024) {
                const int col = c0 + tid;
                int32_t *entry = kp.block_table + (size_t)b * kp.max_blocks + col;
                const int block = col < held ? *entry : -1;
                const bool real = (unsigned)block < (unsigned)kp.n_blocks;
                const unsigned long long mask = __builtin_amdgcn_ballot_w64(real);
                if (lane == 0) counts[wave] = __builtin_popcountll(mask);
                __syncthreads();
                int at = top + __builtin_popcountll(mask & ((1ull << lane) - 1)), all = 0;
#pragma unroll
                for (int w = 0; w < 16; ++w) {
                    if (w < wave) at += counts[w];
                    all += counts[w];
                }
                if (real) {
                    if (at < kp.n_blocks) kp.free_list[at] = block;
                    *entry = -1;
                }
                top = min(top + all, kp.n_blocks);
                __syncthreads();
            }
            if (tid == 0) kp.cached_len[b] = 0;       // (every thread has read it: a barrier lies between, or held is 0)
        }
    }
    if (tid == 0) kp.free_count[0] = top;
}

}  // namespace

hipError_t launch_page_tables(const TablesArgs &a, hipStream_t st)
{
    const ServeDims &d = a.d;
    const TablesParams kp{a.cached_len, a.new_len, a.free_list, a.free_count, a.free_left, a.block_table, a.q_start, a.seq_len, a.slot, a.position, a.request,
                          a.base, d.B, d.T, d.page, d.n_blocks, d.max_blocks, d.by_page};
    constexpr int MOST = 4096;
    const bool in_place = a.free_left == a.free_count;
    if (d.B <= 64 && d.T <= 256) {
        tables_kernel<1, 64><<<1, 64, 0, st>>>(kp);
    } else if (d.B <= MOST && (!in_place || d.T <= 4096)) {
        tables_kernel<16, MOST><<<in_place ? 1 : (unsigned)std::max(1, (d.T + 1023) / 1024), 1024, 0, st>>>(kp);
    } else {
        tables_requests_kernel<<<1, 1024, 0, st>>>(kp);
        if (d.T > 0) tables_tokens_kernel<<<(unsigned)((d.T + 255) / 256), 256, 0, st>>>(kp);
    }
    return hipGetLastError();
}

hipError_t launch_page_release(const ReleaseArgs &a, hipStream_t st)
{
    const ServeDims &d = a.d;
    const ReleaseParams kp{a.finished, a.cached_len, a.block_table, a.free_list, a.free_count, d.B, d.page, d.n_blocks, d.max_blocks};
    release_kernel<<<1, 1024, 0, st>>>(kp);
    return hipGetLastError();
}

}  // namespace lca
