// Attention of each request's new rows over its paged cache, on the tensor cores (tcgen05), and the merge of partial results.
//
// Mathematics.  Per (request, key head) the query heads that share the key head are stacked: row r of a tile is new token
// r / group, query head r % group.  For 128 rows and 128 keys at a time: S = Q K^T (fp32, TMEM), then with the running
// maximum m and sum l of each row P = exp2(c S - m), l += sum P, O += P V (fp32, TMEM), P rounded to the cache's
// type because the second product takes 16-bit operands.  O is rescaled only when a row's maximum has grown by
// more than 2^8 since its last rescaling: P then stays below 2^8, which loses nothing in a floating-point type.
//
// What bounds it.  A window of K + 1 rows has group * (K + 1) rows per key head, so up to some 64 of them the kernel moves
// 4 D bytes per key and does 4 D flops per row and key: bound by HBM as long as one 128-row MMA tile (1024 clocks for 128
// keys at D = 128) is faster than its 64 KB of keys and values (some 2800 clocks at a 148th of the measured copy
// rate).  Prompt chunks are bound by the MMAs and by the exponentials, 1024 clocks each per 128 x 128 tile.
//
// Roles.  One block per SM, persistent: a TMA warp, an MMA warp and two softmax warpgroups, each with its own S and O in
// TMEM (all 512 columns).  A work item is either "paired" - two row tiles of
// the same (request, key head), one per warpgroup, sharing each tile of keys - or, where a single row tile is left, "split":
// the warpgroups take the key tiles in turn and merge at the end.  Either way the jobs (row tile, key tile) alternate
// between the two warpgroups, and the MMA warp issues S of job j + 2 behind O of job j, so one warpgroup's
// exponentials run under the other's MMAs.
//
// Work split.  The key tiles of all items form one line, cut into equal contiguous ranges, one per block; every block finds
// its range from the lengths on the device, so the host knows no lengths and a captured graph stays balanced.  An item cut by a
// range boundary leaves fp32 partials (at most two per block) that attn_merge_kernel adds in block order.
//
// Keys and values come in 128-byte swizzled tiles laid out [8 tokens][D / 64][8][64]: one TMA per page (five dimensions: 64
// columns, 8 tokens, column halves, head, token groups), whatever the page size, with both the K-major view for the first product and
// the MN-major view for the second.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include "wisv_ptx.cuh"

namespace wisv {

constexpr int kAttnThreads = 384;
constexpr int kAttnTile = 128;                   // rows of a row tile, keys of a key tile
constexpr int kAttnMaxStages = 12;
constexpr int kAttnItemCost = 1;                 // key tiles that starting and finishing an item is worth
constexpr int kAttnSmem = 232448;                // all of an SM's shared memory that a block can have
constexpr int kAttnSmall = 2624;                 // barriers, the warpgroups' exchange of m and l
constexpr int kAttnSlack = 448;                  // for aligning the tiles to 1024 bytes
constexpr uint64_t kAttnWaitClocks = 4000000000ull;

struct AttnParams {
    int32_t B, T, max_new, n_kv, group, tpt, page_shift, n_pages, max_blocks, min_units;
    int32_t page_groups_k, page_groups_v;        // 8-token groups from one page to the next
    int32_t groups_k, groups_v;                  // 8-token groups in the whole pool: the first coordinate out of range
    int32_t uniform;                             // rows per request where q_off is NULL
    const int32_t *q_off, *kv_len, *block_table;
    int64_t table_stride;
    void* out; int64_t ot, oh;
    float* lse;
    float scale_log2;
    int32_t* err;
    float* part_o;                               // [2 * blocks][256][D]
    float2* part_ml;                             // [2 * blocks][256]
    int4* desc;                                  // [blocks][2]: the item whose merge starts with this block
};

template <typename E> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <typename E> struct is_bf16 { static constexpr bool value = false; };
template <> struct is_bf16<__nv_bfloat16> { static constexpr bool value = true; };

__device__ __forceinline__ float attn_ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---------------------------------------------------------------- instructions that only this kernel needs
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* m, int32_t a, int32_t b, int32_t c, int32_t d,
                                            int32_t e, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e)
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]: 16-bit A, two elements of K per 32-bit column
__device__ __forceinline__ void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                            uint32_t accumulate)
{
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
        "}\n"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// Shared-memory matrix descriptor, 128-byte swizzle, for a tile whose 8-row groups are `group_bytes` apart and whose
// 64-column chunks are 1024 bytes apart.  K-major operands use the group stride only; for an MN-major operand (rows along
// K) the leading offset is the step between 64-column chunks and the stride offset the step between 8-row groups.
__device__ __forceinline__ uint64_t attn_desc(uint32_t smem_addr, uint32_t group_bytes)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((smem_addr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>(1024 >> 4) << 16;
    d |= static_cast<uint64_t>(group_bytes >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}
// kind::f16, fp32 accumulator; bit 16 set: B is MN-major
template <typename E>
__device__ __forceinline__ uint32_t attn_idesc(uint32_t M, uint32_t N, bool b_mn)
{
    const uint32_t f = is_bf16<E>::value ? 1u : 0u;
    return (1u << 4) | (f << 7) | (f << 10) | (b_mn ? 1u << 16 : 0u) | ((N >> 3) << 17) | ((M >> 4) << 24);
}

// ---------------------------------------------------------------- work items
// One request as the kernel sees it; device-side lengths are clamped to what the arrays hold.
struct AttnReq { int q0, n, kv, items; };

__device__ __forceinline__ AttnReq attn_request(const AttnParams& p, int b)
{
    AttnReq r;
    if (p.q_off) {
        r.q0 = min(max(__ldg(p.q_off + b), 0), p.T);
        r.n = max(min(max(__ldg(p.q_off + b + 1), 0), p.T) - r.q0, 0);
    } else {
        r.q0 = b * p.uniform;
        r.n = p.uniform;
    }
    r.kv = min(max(__ldg(p.kv_len + b), 0), p.max_blocks << p.page_shift);
    r.items = ((r.n + p.tpt - 1) / p.tpt + 1) >> 1;
    return r;
}
// key tiles of item `it` of the request: up to the last key that its last row sees, at least one
__device__ __forceinline__ int attn_tiles(const AttnParams& p, const AttnReq& r, int it)
{
    const int last_tok = min((it + 1) * 2 * p.tpt, r.n) - 1;
    const int last_key = r.kv - r.n + last_tok;
    return last_key < 0 ? 1 : last_key / kAttnTile + 1;
}

// A stretch of one item's key tiles that this block works on
struct AttnSeg {
    int b, kvh, q0, tok0, lim0, kv;              // first row of the item in q; last key that its first token sees
    int rows[2];                                 // valid rows of its row tiles (rows[1] = 0: split)
    int t0, t1, nt;
    bool paired;
    __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == nt; }
    __device__ __forceinline__ int jobs() const { return paired ? 2 * (t1 - t0) : t1 - t0; }
};

struct AttnWalk {
    int b, kvh, it, pos, units;                  // position on the line of key tiles, and what is left of the range
    AttnReq r;

    __device__ __forceinline__ void start(const AttnParams& p, const int* s)
    {
        b = s[0]; kvh = s[1]; it = s[2]; pos = s[3]; units = s[4];
        if (units > 0) r = attn_request(p, b);
    }
    __device__ __forceinline__ bool next(const AttnParams& p, AttnSeg& s)
    {
        while (units > 0) {
            if (it >= r.items) {                 // (a request without rows)
                if (++b >= p.B) return false;
                kvh = it = pos = 0;
                r = attn_request(p, b);
                continue;
            }
            s.nt = attn_tiles(p, r, it);
            const int take = min(units, s.nt + kAttnItemCost - pos);
            s.t0 = pos;
            s.t1 = min(s.nt, pos + take);
            const bool some = s.t1 > s.t0;
            if (some) {
                s.b = b; s.kvh = kvh; s.kv = r.kv;
                s.tok0 = it * 2 * p.tpt;
                s.q0 = r.q0 + s.tok0;
                s.lim0 = r.kv - r.n + s.tok0;
                const int left = r.n - s.tok0;
                s.paired = left > p.tpt;
                s.rows[0] = min(left, p.tpt) * p.group;
                s.rows[1] = s.paired ? min(left - p.tpt, p.tpt) * p.group : 0;
            }
            units -= take;
            pos += take;
            if (pos == s.nt + kAttnItemCost) {
                pos = 0;
                if (++it == r.items) {
                    it = 0;
                    if (++kvh == p.n_kv) {
                        kvh = 0;
                        if (++b < p.B) r = attn_request(p, b);
                        else units = 0;
                    }
                }
            }
            if (some) return true;
        }
        return false;
    }
};

// Position in the ring of key and value tiles: tile g uses entries 2 g (keys) and 2 g + 1 (values).
struct AttnRing {
    int s = 0;
    uint32_t ph = 0;
    __device__ __forceinline__ void step(int stages) { if (++s == stages) { s = 0; ph ^= 1u; } }
};

template <int D> __host__ __device__ constexpr int attn_stage_bytes() { return kAttnTile * D * 2; }
template <int D> __host__ __device__ constexpr int attn_stages()
{
    return (kAttnSmem - kAttnSmall - kAttnSlack - 2 * attn_stage_bytes<D>()) / attn_stage_bytes<D>() < kAttnMaxStages
               ? (kAttnSmem - kAttnSmall - kAttnSlack - 2 * attn_stage_bytes<D>()) / attn_stage_bytes<D>() : kAttnMaxStages;
}

template <typename E, int D>
__global__ void __launch_bounds__(kAttnThreads, 1)
attn_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
            const __grid_constant__ CUtensorMap tmV, const AttnParams p)
{
    constexpr int kStages = attn_stages<D>();
    constexpr uint32_t kStage = attn_stage_bytes<D>();
    constexpr uint32_t kGroup = D / 64 * 1024;   // bytes of 8 tokens
    constexpr int kHalves = D / 64;

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;
    const uint32_t base = raw_addr + pad;
    const uint32_t q_buf = base, ring = base + 2 * kStage;
    const uint32_t small_off = pad + (2 + kStages) * kStage;
    uint8_t* small = smem_raw + small_off;
    const uint32_t bars = raw_addr + small_off;

    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (kAttnMaxStages + s); };
    auto q_full = [&](int s) { return bars + 8u * (2 * kAttnMaxStages + s); };
    auto q_empty = [&](int s) { return bars + 8u * (2 * kAttnMaxStages + 2 + s); };
    auto s_full = [&](int s) { return bars + 8u * (2 * kAttnMaxStages + 4 + s); };
    auto p_full = [&](int s) { return bars + 8u * (2 * kAttnMaxStages + 6 + s); };
    const uint32_t o_full = bars + 8u * (2 * kAttnMaxStages + 8);
    const uint32_t o_empty = o_full + 8, ml_full = o_full + 16, drain = o_full + 24;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(small + 8 * (2 * kAttnMaxStages + 12));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);       // [0] abort, [1] drain scratch
    int* start = reinterpret_cast<int*>(tmem_slot + 3);                              // [5] start of the range
    long long* totals = reinterpret_cast<long long*>(small + 432);                   // [12] scan over the warps
    float2* ml = reinterpret_cast<float2*>(small + 544);                             // [2][128]

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int lane = threadIdx.x & 31;

    if (small_off + kAttnSmall > static_cast<uint32_t>(kAttnSmem)) {          // (dynamic shared memory starts 1024-byte aligned)
        if (threadIdx.x == 0) { atomicOr(p.err, 2); p.desc[2 * blockIdx.x] = make_int4(0, 0, 0, 0); }
        return;
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(q_full(s), 1); mbar_init(q_empty(s), 1); mbar_init(s_full(s), 1); mbar_init(p_full(s), 4);
        }
        mbar_init(o_full, 1); mbar_init(o_empty, 8); mbar_init(ml_full, 8); mbar_init(drain, 1);
        abort_flag[0] = 0; abort_flag[1] = 0;
        for (int i = 0; i < 5; ++i) start[i] = 0;
        fence_barrier_init();
        tma_prefetch_desc(&tmQ);
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmV);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    griddep_wait();                              // lengths, tables and the cache itself come from kernels before this one
    griddep_launch_dependents();

    // ---- the block's range of the line of key tiles
    long long total;
    int blocks, me;
    {
        const int per = (p.B + kAttnThreads - 1) / kAttnThreads;
        const int b0 = min(static_cast<int>(threadIdx.x) * per, p.B), b1 = min(b0 + per, p.B);
        auto units_of = [&](const AttnReq& r) {
            long long u = 0;
            for (int i = 0; i < r.items; ++i) u += attn_tiles(p, r, i) + kAttnItemCost;
            return u;
        };
        long long mine = 0;
        for (int b = b0; b < b1; ++b) mine += units_of(attn_request(p, b)) * p.n_kv;
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        if (lane == 31) totals[warp] = upto;
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        total = 0;
        for (int w = 0; w < kAttnThreads / 32; ++w) {
            if (w < warp) upto += totals[w];
            total += totals[w];
        }
        const long long want = total / p.min_units;
        blocks = static_cast<int>(min(static_cast<long long>(gridDim.x), max(want, 1ll)));
        me = blockIdx.x;
        if (me < blocks && total > 0) {
            const long long lo = me * total / blocks, hi = (me + 1) * total / blocks;
            const long long first = upto - mine;
            if (mine > 0 && lo >= first && lo < upto) {          // one thread's requests hold the start
                long long x = lo - first;
                for (int b = b0; b < b1; ++b) {
                    const AttnReq r = attn_request(p, b);
                    const long long one = units_of(r);
                    if (x >= one * p.n_kv) { x -= one * p.n_kv; continue; }
                    const int h = static_cast<int>(x / one);
                    x -= h * one;
                    int it = 0;
                    for (; ; ++it) {
                        const int u = attn_tiles(p, r, it) + kAttnItemCost;
                        if (x < u) break;
                        x -= u;
                    }
                    start[0] = b; start[1] = h; start[2] = it; start[3] = static_cast<int>(x);
                    start[4] = static_cast<int>(hi - lo);
                    break;
                }
            }
        }
        __syncthreads();
    }
    const uint32_t tmem = *tmem_slot;
    const uint32_t tS = tmem, tO = tmem + 256;   // S of slot s at 128 s, P in the upper half of it, O at 256 + 128 s
    AttnWalk walk;
    walk.start(p, start);
    AttnSeg seg;
    long long issued = 0;                        // ring entries filled (producer warp; read again before the end)
    int q_issued = 0;

    if (warp < 4) {
        if (warp == 0) {
            // ------------------------------------------------------------ TMA
            AttnRing rg;
            bool ok = true;
            const int box_tok = min(1 << p.page_shift, kAttnTile);
            while (ok && walk.next(p, seg)) {
                // queries: one buffer per row tile
                for (int t = 0; ok && t < (seg.paired ? 2 : 1); ++t, ++q_issued) {
                    const int qb = q_issued & 1;
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(q_empty(qb), ((q_issued >> 1) & 1u) ^ 1u, abort_flag, kAttnWaitClocks));
                    if (ok && elect_one()) {
                        mbar_expect_tx(q_full(qb), static_cast<uint32_t>(p.tpt * p.group) * 128u * kHalves);
                        for (int h = 0; h < kHalves; ++h)
                            tma_load_5d(q_buf + qb * kStage + h * (kAttnTile * 128), &tmQ, 0, 0, seg.q0 + t * p.tpt, h, seg.kvh, q_full(qb));
                    }
                    __syncwarp();
                }
                const int32_t* table = p.block_table + seg.b * p.table_stride;
                for (int t = seg.t0; ok && t < seg.t1; ++t) {
                    // this tile's pages: lane i holds the i-th one's first token group, for keys and for values
                    const int tok0 = t * kAttnTile;
                    const int have = min(seg.kv - tok0, kAttnTile);       // keys that exist
                    const int pages = have <= 0 ? 0 : (have + box_tok - 1) / box_tok;
                    int gk = p.groups_k, gv = p.groups_v;
                    if (lane < pages) {
                        const int tok = tok0 + lane * box_tok;
                        const int pg = __ldg(table + (tok >> p.page_shift));
                        if (pg >= 0 && pg < p.n_pages) {
                            const int in = (tok & ((1 << p.page_shift) - 1)) >> 3;
                            gk = pg * p.page_groups_k + in;
                            gv = pg * p.page_groups_v + in;
                        }
                    }
                    for (int kv = 0; ok && kv < 2; ++kv) {
                        ok = __all_sync(0xffffffffu, mbar_wait_bounded(empty_bar(rg.s), rg.ph ^ 1u, abort_flag, kAttnWaitClocks));
                        if (!ok) break;
                        const uint32_t dst = ring + rg.s * kStage, bar = full_bar(rg.s);
                        const uint32_t box_bytes = static_cast<uint32_t>(box_tok) * (D * 2);
                        if (elect_one()) mbar_expect_tx(bar, static_cast<uint32_t>(pages) * box_bytes);
                        __syncwarp();
                        for (int i = 0; i < pages; ++i) {
                            const int g = __shfl_sync(0xffffffffu, kv ? gv : gk, i);
                            if (elect_one()) tma_load_5d(dst + i * box_bytes, kv ? &tmV : &tmK, 0, 0, 0, seg.kvh, g, bar);
                        }
                        __syncwarp();
                        ++issued;
                        rg.step(kStages);
                    }
                }
            }
        } else if (warp == 1) {
            // ------------------------------------------------------------ MMA
            const uint32_t idS = attn_idesc<E>(kAttnTile, kAttnTile, false);
            const uint32_t idO = attn_idesc<E>(kAttnTile, D, true);
            AttnWalk wq = walk;                  // the S side runs two jobs ahead of the O side
            AttnSeg sq, so;
            int jq = 0, jo = 0;                  // jobs issued on either side, over all items
            int nq = 0, no = 0;                  // job within the item
            int Jq = 0, Jo = 0;
            int q_used = 0;                      // query buffers released so far
            int items = 0;
            AttnRing rq, ro;                     // key entry of the S side's tile, value entry of the O side's
            ro.step(kStages);
            bool ok = true;

            auto issue_s = [&]() {
                if (nq == Jq) {
                    if (!wq.next(p, sq)) { Jq = nq = -1; return; }
                    nq = 0; Jq = sq.jobs();
                }
                if (Jq < 0) return;
                const int slot = jq & 1, half = sq.paired ? (nq & 1) : 0;
                const int qb = (q_used + half) & 1;
                if (nq < (sq.paired ? 2 : 1)) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(q_full(qb), ((q_used + half) >> 1) & 1u, abort_flag, kAttnWaitClocks));
                    if (!ok) return;
                }
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(full_bar(rq.s), rq.ph, abort_flag, kAttnWaitClocks));
                if (!ok) return;
                tc_fence_after();
                const bool last_use = !sq.paired || half == 1;
                const bool q_done = nq + (sq.paired ? 2 : 1) >= Jq;
                if (elect_one()) {
                    const uint64_t a0 = attn_desc(q_buf + qb * kStage, 1024);
                    const uint64_t b0 = attn_desc(ring + rq.s * kStage, kGroup);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t a = a0 + static_cast<uint64_t>(((k >> 2) * (kAttnTile * 128) + (k & 3) * 32) >> 4);
                        const uint64_t b = b0 + static_cast<uint64_t>(((k >> 2) * 1024 + (k & 3) * 32) >> 4);
                        umma_bf16(tS + slot * 128, a, b, idS, k != 0);
                    }
                    umma_commit(s_full(slot));
                    if (last_use) umma_commit(empty_bar(rq.s));
                    if (q_done) umma_commit(q_empty(qb));
                }
                __syncwarp();
                if (last_use) { rq.step(kStages); rq.step(kStages); }
                ++jq; ++nq;
                if (nq == Jq) q_used += sq.paired ? 2 : 1;
            };
            auto issue_o = [&]() -> bool {
                if (no == Jo) {
                    if (!walk.next(p, so)) return false;
                    no = 0; Jo = so.jobs();
                    if (items > 0) {             // the previous item's O has been read
                        ok = __all_sync(0xffffffffu, mbar_wait_bounded(o_empty, (items - 1) & 1u, abort_flag, kAttnWaitClocks));
                        if (!ok) return false;
                    }
                }
                const int slot = jo & 1, half = so.paired ? (no & 1) : 0;
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(p_full(slot), (jo >> 1) & 1u, abort_flag, kAttnWaitClocks));
                if (!ok) return false;
                if (half == 0) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(full_bar(ro.s), ro.ph, abort_flag, kAttnWaitClocks));
                    if (!ok) return false;
                }
                tc_fence_after();
                const bool last_use = !so.paired || half == 1;
                const bool first = no < 2;       // the slot's first job of this item
                if (elect_one()) {
                    const uint64_t b0 = attn_desc(ring + ro.s * kStage, kGroup);
#pragma unroll
                    for (int k = 0; k < kAttnTile / 16; ++k)
                        umma_f16_ts(tO + slot * 128, tS + slot * 128 + 64 + k * 8, b0 + static_cast<uint64_t>((k * 2 * kGroup) >> 4), idO,
                                    (!first || k != 0) ? 1u : 0u);
                    if (last_use) umma_commit(empty_bar(ro.s));
                    if (no + 1 == Jo) umma_commit(o_full);
                }
                __syncwarp();
                if (last_use) { ro.step(kStages); ro.step(kStages); }
                ++jo; ++no;
                if (no == Jo) ++items;
                return true;
            };
            issue_s();
            if (ok) issue_s();
            while (ok && issue_o()) issue_s();
            if (!ok) {
                if (elect_one()) umma_commit(drain);
                __syncwarp();
                mbar_wait_bounded(drain, 0, abort_flag + 1, kAttnWaitClocks);
            }
        }
    } else {
        // ---------------------------------------------------------------- softmax warpgroups
        const int slot = (warp - 4) >> 2, quad = warp & 3;
        const int row = quad * 32 + lane;        // row of the tile = TMEM lane
        const uint32_t lane_off = static_cast<uint32_t>(quad * 32) << 16;
        const uint32_t aS = tS + slot * 128 + lane_off, aO = tO + slot * 128 + lane_off;
        const uint32_t aO_other = tO + (slot ^ 1) * 128 + lane_off;
        const int my_tok = row / p.group, my_head = row % p.group;
        int jobs = 0, items = 0, splits = 0, tiles = 0;      // over all items of the block
        bool ok = true, described = false;
        while (ok && walk.next(p, seg)) {
            const int f = jobs & 1, n0 = slot ^ f, J = seg.jobs();
            const int tile_rows = seg.paired ? seg.rows[n0] : seg.rows[0];
            const bool warp_has_rows = quad * 32 < tile_rows;
            const int lim = seg.lim0 + my_tok + (seg.paired && n0 ? p.tpt : 0);     // last key that this row sees
            float m = -CUDART_INF_F, l = 0.0f;
            for (int n = n0; ok && n < J; n += 2) {
                const int tile = seg.t0 + (seg.paired ? n >> 1 : n);
                const uint32_t use = static_cast<uint32_t>((jobs + n) >> 1);
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(s_full(slot), use & 1u, abort_flag, kAttnWaitClocks));
                if (!ok) break;
                tc_fence_after();
                if (warp_has_rows) {
                    // The row in two halves of 64 columns, so that it fits the registers: maximum of the first, then of the second,
                    // which stays for its exponentials; the first is read again for its own.  P goes to the upper half of
                    // the slot's columns, which holds nothing that is still to be read.
                    uint32_t sr[64];
                    float* s = reinterpret_cast<float*>(sr);
                    const int cut = lim - tile * kAttnTile;                          // columns past it are masked
                    const bool masked = !__all_sync(0xffffffffu, cut >= kAttnTile - 1);
                    float mx[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
                    auto load_half = [&](int h) {
                        tmem_ld32(aS + h * 64, sr);
                        tmem_ld32(aS + h * 64 + 32, sr + 32);
                        tmem_wait_ld();
                        if (masked) {
#pragma unroll
                            for (int c = 0; c < 64; ++c) s[c] = h * 64 + c <= cut ? s[c] : -CUDART_INF_F;
                        }
                    };
                    auto max_half = [&]() {
#pragma unroll
                        for (int c = 0; c < 64; ++c) mx[c & 3] = fmaxf(mx[c & 3], s[c]);
                    };
                    load_half(0);
                    max_half();
                    load_half(1);
                    max_half();
                    const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
                    const bool grow = mt > m + 8.0f;
                    if (__any_sync(0xffffffffu, grow)) {
                        const float m_new = grow ? mt : m;
                        const float a = grow ? attn_ex2(m - m_new) : 1.0f;
                        l *= a;
                        m = m_new;
                        if (n >= 2) {
#pragma unroll
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                tmem_ld16(aO + c, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * a);
                                tmem_st16(aO + c, o);
                            }
                        }
                    }
                    const float base_m = m == -CUDART_INF_F ? 0.0f : m;
                    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    auto exp_half = [&](int h) {
#pragma unroll
                        for (int c = 0; c < 64; c += 32) {
                            uint32_t pk[16];
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const float x = attn_ex2(fmaf(s[c + i], p.scale_log2, -base_m));
                                const float y = attn_ex2(fmaf(s[c + i + 1], p.scale_log2, -base_m));
                                sum[i & 2] += x;
                                sum[(i & 2) + 1] += y;
                                pk[i / 2] = pack2<E>(x, y);
                            }
                            tmem_st16(aS + 64 + h * 32 + c / 2, pk);
                        }
                    };
                    exp_half(1);
                    load_half(0);
                    exp_half(0);
                    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    tmem_wait_st();
                }
                const int have = max(seg.kv - tile * kAttnTile, 0);
                if (have < kAttnTile) {
                    // Value rows behind the last key: their probabilities are 0, but 0 times what happens to lie there could be
                    // NaN.  (Both warpgroups of a paired item clear them: zeros over zeros.)  Row r of a tile lies in group r / 8
                    // at 128 (r % 8), once per 64 columns.  The stage cannot be recycled before this job's second product.
                    const int e = 2 * (tiles + tile - seg.t0) + 1, st = e % kStages;
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(full_bar(st), static_cast<uint32_t>(e / kStages) & 1u, abort_flag, kAttnWaitClocks));
                    if (!ok) break;
                    for (int i = row; i < (kAttnTile - have) * kHalves * 8; i += 128) {
                        const int r = have + i / (kHalves * 8), c = i % (kHalves * 8);
                        const uint32_t at = ring + st * kStage + (r >> 3) * kGroup + (c >> 3) * 1024 + (r & 7) * 128 + (c & 7) * 16;
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
                    }
                    fence_proxy_async();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(slot));
            }
            if (!ok) break;

            // ---- the item (or its stretch) is done: O of both slots is complete.  A split item's two halves are put
            // together here, each warpgroup taking one half of the columns of both accumulators.
            if (!seg.paired) {
                ml[slot * 128 + row] = make_float2(m, l);
                __syncwarp();
                if (lane == 0) mbar_arrive(ml_full);
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(ml_full, static_cast<uint32_t>(splits & 1), abort_flag, kAttnWaitClocks));
                if (!ok) break;
                ++splits;
            }
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(o_full, static_cast<uint32_t>(items & 1), abort_flag, kAttnWaitClocks));
            if (!ok) break;
            tc_fence_after();
            if (warp_has_rows) {
                float wa = 1.0f, wb = 0.0f;      // weights of this slot's accumulator and of the other one's
                if (!seg.paired) {
                    const float2 o = ml[(slot ^ 1) * 128 + row];
                    const float mm = fmaxf(m, o.x);
                    wa = m == -CUDART_INF_F ? 0.0f : attn_ex2(m - mm);
                    wb = o.x == -CUDART_INF_F ? 0.0f : attn_ex2(o.x - mm);
                    l = l * wa + o.y * wb;
                    m = mm;
                }
                const bool valid = row < tile_rows, whole = seg.whole();
                const bool use_a = seg.paired || n0 < J, use_b = !seg.paired && (n0 ^ 1) < J;      // the slot had a job
                const int c0 = seg.paired ? 0 : slot * (D / 2), c1 = seg.paired ? D : c0 + D / 2;
                const int part = static_cast<int>(blockIdx.x) * 2 + (seg.t0 == 0 ? 1 : 0);
                const int part_row = part * 256 + (seg.paired ? n0 * 128 : 0) + row;
                const int tok = seg.q0 + my_tok + (seg.paired && n0 ? p.tpt : 0), head = seg.kvh * p.group + my_head;
                E* const dst = static_cast<E*>(p.out) + tok * p.ot + head * p.oh;
                float* const dst_part = p.part_o + static_cast<size_t>(part_row) * D;
                const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                if (whole) { wa *= inv; wb *= inv; }
                for (int c = c0; c < c1; c += 32) {
                    uint32_t o[32];
                    float x[32];
                    if (use_a) {
                        tmem_ld32(aO + c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(o[i]) * wa;
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = 0.0f;
                    }
                    if (use_b) {
                        tmem_ld32(aO_other + c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = fmaf(__uint_as_float(o[i]), wb, x[i]);
                    }
                    if (valid && whole) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            *reinterpret_cast<uint4*>(dst + c + i) =
                                make_uint4(pack2<E>(x[i], x[i + 1]), pack2<E>(x[i + 2], x[i + 3]), pack2<E>(x[i + 4], x[i + 5]),
                                           pack2<E>(x[i + 6], x[i + 7]));
                    } else if (valid) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            *reinterpret_cast<float4*>(dst_part + c + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
                    }
                }
                if (valid && (seg.paired || slot == 0)) {
                    if (!whole) p.part_ml[part_row] = make_float2(m, l);
                    else if (p.lse)
                        p.lse[static_cast<int64_t>(tok) * (p.n_kv * p.group) + head] =
                            l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -CUDART_INF_F;
                }
            }
            // what the merge kernel has to know of an item that starts here and ends in another block: this is the last stretch
            // of this block's range
            if (warp == 4 && lane == 0 && seg.t0 == 0 && seg.t1 < seg.nt) {
                const long long last = (me + 1) * total / blocks - seg.t1 + seg.nt - 1;           // its last key tile on the line
                const int parts = static_cast<int>(((last + 1) * blocks - 1) / total) - me + 1;
                p.desc[2 * me] = make_int4(parts, seg.q0, seg.kvh, seg.paired ? p.tpt : 0);
                p.desc[2 * me + 1] = make_int4(seg.rows[0], seg.rows[1], 0, 0);
                described = true;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_empty);
            jobs += J;
            tiles += seg.t1 - seg.t0;
            ++items;
        }
        if (warp == 4 && lane == 0 && !described) p.desc[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
    }

    __syncthreads();
    if (warp == 0 && lane == 0 && abort_flag[0] != 0) {
        // after a time-out: the copies still in flight have to land before this block's shared memory is given up
        for (long long i = issued > kStages ? issued - kStages : 0; i < issued; ++i)
            mbar_wait_bounded(full_bar(static_cast<int>(i % kStages)), static_cast<uint32_t>((i / kStages) & 1), abort_flag + 1, kAttnWaitClocks);
        for (int i = q_issued > 2 ? q_issued - 2 : 0; i < q_issued; ++i)
            mbar_wait_bounded(q_full(i & 1), static_cast<uint32_t>((i >> 1) & 1), abort_flag + 1, kAttnWaitClocks);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (threadIdx.x == 0 && abort_flag[0] != 0) atomicOr(p.err, 1);
}

// ---------------------------------------------------------------- merge of the items that several blocks share
// Block c looks after the item that starts in block c's range and ends in a later one; a warp takes a row: the partials' maxima
// and sums first, then D / 32 columns per lane, partials in block order (so the result does not depend on timing).
struct AttnMerge {
    const float* part_o;
    const float2* part_ml;
    const int4* desc;
    void* out; int64_t ot, oh;
    float* lse;
    int32_t group, n_heads;
};

constexpr int kMergeThreads = 128;

template <typename E, int D>
__global__ void __launch_bounds__(kMergeThreads) attn_merge_kernel(const AttnMerge p)
{
    griddep_wait();
    griddep_launch_dependents();
    const int c = blockIdx.x;
    const int4 d = p.desc[2 * c];
    const int parts = d.x;
    if (parts < 2) return;
    const int4 e = p.desc[2 * c + 1];
    const int lane = threadIdx.x & 31;
    constexpr int N = D / 32;
    for (int w = blockIdx.y * (kMergeThreads / 32) + (threadIdx.x >> 5); w < e.x + e.y; w += gridDim.y * (kMergeThreads / 32)) {
        const int second = w >= e.x ? 1 : 0;
        const int r = second ? w - e.x : w;
        const int at = second * 128 + r;
        auto row_of = [&](int j) { return (j == 0 ? 2 * c + 1 : 2 * (c + j)) * 256 + at; };
        float m = -CUDART_INF_F;
        for (int j = lane; j < parts; j += 32) m = fmaxf(m, p.part_ml[row_of(j)].x);
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        float l = 0.0f, acc[N] = {};
        for (int j0 = 0; j0 < parts; j0 += 32) {
            float wt = 0.0f, wl = 0.0f;
            if (j0 + lane < parts) {
                const float2 x = p.part_ml[row_of(j0 + lane)];
                wt = x.x == -CUDART_INF_F ? 0.0f : attn_ex2(x.x - m);
                wl = wt * x.y;
            }
            const int here = min(32, parts - j0);
#pragma unroll 4
            for (int u = 0; u < here; ++u) {
                const float f = __shfl_sync(0xffffffffu, wt, u);
                l += __shfl_sync(0xffffffffu, wl, u);
                const float* src = p.part_o + static_cast<size_t>(row_of(j0 + u)) * D + lane * N;
                if (N == 4) {
                    const float4 v = *reinterpret_cast<const float4*>(src);
                    acc[0] = fmaf(f, v.x, acc[0]); acc[1] = fmaf(f, v.y, acc[1]);
                    acc[2 % N] = fmaf(f, v.z, acc[2 % N]); acc[3 % N] = fmaf(f, v.w, acc[3 % N]);
                } else {
                    const float2 v = *reinterpret_cast<const float2*>(src);
                    acc[0] = fmaf(f, v.x, acc[0]); acc[1] = fmaf(f, v.y, acc[1]);
                }
            }
        }
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        const int tok = d.y + r / p.group + second * d.w, head = d.z * p.group + r % p.group;
        E* const dst = static_cast<E*>(p.out) + tok * p.ot + head * p.oh + lane * N;
        if (N == 4)
            *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<E>(acc[0] * inv, acc[1] * inv), pack2<E>(acc[2 % N] * inv, acc[3 % N] * inv));
        else
            *reinterpret_cast<uint32_t*>(dst) = pack2<E>(acc[0] * inv, acc[1] * inv);
        if (p.lse && lane == 0)
            p.lse[static_cast<int64_t>(tok) * p.n_heads + head] = l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -CUDART_INF_F;
    }
}

}  // namespace wisv
