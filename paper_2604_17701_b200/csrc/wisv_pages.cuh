// Page bookkeeping of the paged cache, and the copy of new keys and values into it.
//
// pages_extend_kernel turns request lengths into everything a round needs: with c_b = ceil((len_b + n_b) / page) -
// blocks_b pages lacking (at least 0), prefix sums over the requests give each request its place among the new rows
// (n_b) and in the free list (c_b); every new page and every new row then finds its request by a binary search in those
// prefix sums, which shared memory holds.  pages_commit_kernel is the way back.
//
// What bounds them is latency: a launch, four dependent loads, two block-wide scans (extend and commit together 5.6 us for one
// request, 9.6 us for 512 with 5632 rows).  So everything happens in ONE launch: a single block for small rounds, a cluster of
// eight blocks for extensions of many rows and commits of many requests, each of which repeats the scan (cheaper than handing
// its result on) and takes its share of the pages and rows; the arrays that are both read and written are written after a
// cluster barrier.
#pragma once

#include "wisv_ptx.cuh"

namespace wisv {

constexpr int kPageThreads = 1024;
constexpr int kPagePer = 4;                       // requests per thread: 1024 * 4 = WISV_MAX_REQUESTS
constexpr int kPageCluster = 8;

struct PagesParams {
    int32_t B, T, n_uniform, page_shift, n_pages, max_blocks;
    const int32_t* n_new;
    const int32_t* new_len;
    int32_t *free_list, *n_free, *block_table, *n_blocks, *seq_len;
    int32_t *q_off, *kv_len, *positions, *status;
    int64_t* slot_map;
};

// Inclusive prefix sums over the block of each thread's two totals (a: rows, b: pages).
__device__ __forceinline__ void block_scan2(long long& a, long long& b, long long (&tot)[2][32])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
        if (lane >= o) { a += x; b += y; }
    }
    if (lane == 31) { tot[0][warp] = a; tot[1][warp] = b; }
    __syncthreads();
    if (warp == 0) {
        long long x = tot[0][lane], y = tot[1][lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
            if (lane >= o) { x += u; y += v; }
        }
        tot[0][lane] = x; tot[1][lane] = y;
    }
    __syncthreads();
    if (warp > 0) { a += tot[0][warp - 1]; b += tot[1][warp - 1]; }
}

// the last index b in [0, n) with first[b] <= x (first ascends, first[0] <= x)
__device__ __forceinline__ int last_at_most(const int32_t* first, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int32_t clamp_i32(long long x) { return x > 0x7fffffffLL ? 0x7fffffff : static_cast<int32_t>(x); }

template <bool kClustered>
__global__ void __launch_bounds__(kPageThreads) pages_extend_kernel(const PagesParams p)
{
    extern __shared__ int32_t sh[];
    int32_t* off = sh;                            // [B + 1] first row of a request
    int32_t* first = off + p.B + 1;               // [B] first of its pages among the pages taken
    int32_t* held = first + p.B;                  // [B] pages it held before
    int32_t* len = held + p.B;                    // [B] tokens it held before; ~len: it got no pages
    __shared__ long long tot[2][32];
    __shared__ int taken;
    const int rank = kClustered ? static_cast<int>(cluster_ctarank()) : 0;
    const int ctas = kClustered ? kPageCluster : 1;
    const int b0 = threadIdx.x * kPagePer;
    if (threadIdx.x == 0) taken = 0;
    griddep_wait();
    griddep_launch_dependents();
    int nv[kPagePer], sv[kPagePer], hv[kPagePer], cv[kPagePer];
    bool fits[kPagePer], bad[kPagePer];
    long long rows = 0, lack = 0;
    const int n_free = min(max(*p.n_free, 0), p.n_pages);
    const int page = 1 << p.page_shift;
#pragma unroll
    for (int u = 0; u < kPagePer; ++u) {
        const int b = b0 + u;
        nv[u] = sv[u] = hv[u] = cv[u] = 0; fits[u] = true; bad[u] = false;
        if (b >= p.B) continue;
        const int n = p.n_new ? p.n_new[b] : p.n_uniform, s = p.seq_len[b], h = p.n_blocks[b];
        bad[u] = n < 0 || s < 0 || h < 0 || h > p.max_blocks;
        nv[u] = max(n, 0); sv[u] = max(s, 0); hv[u] = min(max(h, 0), p.max_blocks);
        const long long want = (static_cast<long long>(sv[u]) + nv[u] + page - 1) >> p.page_shift;
        fits[u] = want <= p.max_blocks;
        cv[u] = fits[u] ? max(static_cast<int>(want) - hv[u], 0) : 0;
        rows += nv[u]; lack += cv[u];
    }
    if (kClustered) cluster_arrive();             // this block has read what block 0 rewrites at the end
    long long r_end = rows, c_end = lack;
    block_scan2(r_end, c_end, tot);
    long long r = r_end - rows, c = c_end - lack;
    bool good[kPagePer];
#pragma unroll
    for (int u = 0; u < kPagePer; ++u) {
        const int b = b0 + u;
        if (b >= p.B) continue;
        const long long upto = c + cv[u];
        good[u] = fits[u] && (cv[u] == 0 || upto <= n_free);
        if (good[u] && cv[u]) atomicMax(&taken, static_cast<int>(upto));
        off[b] = clamp_i32(r);
        first[b] = clamp_i32(c);
        held[b] = hv[u];
        len[b] = good[u] ? sv[u] : ~sv[u];
        r += nv[u]; c = upto;
        if (b == p.B - 1) off[p.B] = clamp_i32(r);
    }
    __syncthreads();
    const int N = taken;
    const int me = rank * kPageThreads + threadIdx.x, all = ctas * kPageThreads;
    // the pages taken: the j-th of them is free_list[n_free - N + j]
    for (int j = me; j < N; j += all) {
        const int b = last_at_most(first, p.B, j);
        p.block_table[static_cast<size_t>(b) * p.max_blocks + held[b] + (j - first[b])] = p.free_list[n_free - N + j];
    }
    // the rows
    for (int t = me; t < p.T; t += all) {
        int pos = -1;
        long long slot = -1;
        if (t < off[p.B]) {
            const int b = last_at_most(off, p.B, t);
            const int s = len[b] < 0 ? ~len[b] : len[b];
            pos = s + (t - off[b]);
            if (len[b] >= 0) {
                const int blk = pos >> p.page_shift;
                const int pg = blk < held[b] ? p.block_table[static_cast<size_t>(b) * p.max_blocks + blk]
                                             : p.free_list[n_free - N + first[b] + (blk - held[b])];
                slot = (static_cast<long long>(pg) << p.page_shift) + (pos & (page - 1));
            }
        }
        p.positions[t] = pos;
        p.slot_map[t] = slot;
    }
    if (kClustered) cluster_wait();               // every block has read n_free and n_blocks
    if (rank == 0) {
#pragma unroll
        for (int u = 0; u < kPagePer; ++u) {
            const int b = b0 + u;
            if (b >= p.B) continue;
            p.q_off[b] = off[b];
            p.kv_len[b] = good[u] ? sv[u] + nv[u] : 0;
            if (good[u] && cv[u]) p.n_blocks[b] = hv[u] + cv[u];
            if (p.status) p.status[b] = (good[u] ? 0 : WISV_ST_NO_PAGES) | (bad[u] ? WISV_ST_BAD_LENGTH : 0);
        }
        if (threadIdx.x == 0) { p.q_off[p.B] = off[p.B]; *p.n_free = n_free - N; }
    }
}

template <bool kClustered>
__global__ void __launch_bounds__(kPageThreads) pages_commit_kernel(const PagesParams p)
{
    extern __shared__ int32_t sh[];
    int32_t* first = sh;                          // [B] first of a request's pages among the pages returned
    int32_t* left = first + p.B;                  // [B] pages it keeps
    __shared__ long long tot[2][32];
    __shared__ int returned;
    const int rank = kClustered ? static_cast<int>(cluster_ctarank()) : 0;
    const int ctas = kClustered ? kPageCluster : 1;
    const int b0 = threadIdx.x * kPagePer;
    griddep_wait();
    griddep_launch_dependents();
    const int n_free = min(max(*p.n_free, 0), p.n_pages);
    int lv[kPagePer], kv[kPagePer], hv[kPagePer];
    bool bad[kPagePer];
    long long gone = 0, none = 0;
#pragma unroll
    for (int u = 0; u < kPagePer; ++u) {
        const int b = b0 + u;
        lv[u] = kv[u] = hv[u] = 0; bad[u] = false;
        if (b >= p.B) continue;
        const int h0 = p.n_blocks[b], want = p.new_len[b];
        const int h = min(max(h0, 0), p.max_blocks);
        const long long most = static_cast<long long>(h) << p.page_shift;
        bad[u] = want < 0 || want > most || h != h0;
        lv[u] = static_cast<int>(min(static_cast<long long>(max(want, 0)), most));
        kv[u] = static_cast<int>((static_cast<long long>(lv[u]) + (1 << p.page_shift) - 1) >> p.page_shift);
        hv[u] = h;
        gone += h - kv[u];
    }
    if (kClustered) cluster_arrive();
    long long end = gone;
    block_scan2(end, none, tot);
    long long c = end - gone;
#pragma unroll
    for (int u = 0; u < kPagePer; ++u) {
        const int b = b0 + u;
        if (b >= p.B) continue;
        first[b] = clamp_i32(c);
        left[b] = kv[u];
        c += hv[u] - kv[u];
        if (b == p.B - 1) returned = clamp_i32(c);
    }
    __syncthreads();
    const int G = min(returned, p.n_pages - n_free);      // a pool cannot hold more free pages than it has
    for (int j = rank * kPageThreads + threadIdx.x; j < returned; j += ctas * kPageThreads) {
        const int b = last_at_most(first, p.B, j);
        int32_t* e = p.block_table + static_cast<size_t>(b) * p.max_blocks + left[b] + (j - first[b]);
        if (j < G) p.free_list[n_free + j] = *e;
        *e = -1;
    }
    if (kClustered) cluster_wait();
    __syncthreads();
    if (rank == 0) {
#pragma unroll
        for (int u = 0; u < kPagePer; ++u) {
            const int b = b0 + u;
            if (b >= p.B) continue;
            p.n_blocks[b] = kv[u];
            p.seq_len[b] = lv[u];
            if (p.status) p.status[b] = bad[u] ? WISV_ST_BAD_LENGTH : 0;
        }
        if (threadIdx.x == 0) *p.n_free = n_free + G;
    }
}

// ---------------------------------------------------------------- append
// One thread moves 16 bytes of a key row and the same 16 bytes of the value row; a row of n_kv_heads * head_dim elements
// takes `vecs` threads.  A plain stream: bound by HBM for long chunks (8192 rows of 8 x 128: 67 MB in 11.7 us, 5.7 TB/s), by the launch
// for a window (1.6 us).
struct AppendParams {
    int32_t T, vecs, vec_shift, page_shift;       // vec_shift: log2 of 16-byte pieces per head
    int64_t n_slots;
    const uint4 *k, *v;                           // strides in 16-byte pieces
    int64_t kt, kh, vt, vh;
    uint4 *kp, *vp;
    int64_t kpp, kpt, kph, vpp, vpt, vph;
    const int64_t* slot_map;
};

constexpr int kAppendThreads = 256;

__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendParams p)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kAppendThreads + threadIdx.x;
    const int64_t t = i / p.vecs;
    griddep_wait();
    griddep_launch_dependents();
    if (t >= p.T) return;
    const int x = static_cast<int>(i - t * p.vecs);
    const int h = x >> p.vec_shift, e = x & ((1 << p.vec_shift) - 1);
    const int64_t slot = p.slot_map[t];
    if (slot < 0 || slot >= p.n_slots) return;
    const int64_t pg = slot >> p.page_shift, o = slot & ((1 << p.page_shift) - 1);
    const uint4 a = p.k[t * p.kt + h * p.kh + e];
    const uint4 b = p.v[t * p.vt + h * p.vh + e];
    p.kp[pg * p.kpp + o * p.kpt + h * p.kph + e] = a;
    p.vp[pg * p.vpp + o * p.vpt + h * p.vph + e] = b;
}

}  // namespace wisv
