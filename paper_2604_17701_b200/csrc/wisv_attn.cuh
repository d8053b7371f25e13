// Attention of each request's new rows over its paged cache, on the tensor cores (tcgen05), and the merge of partial results.
//
// Mathematics.  Per (request, key head) the query heads that share the key head are stacked: row r of a tile is new token
// r / group, query head r % group.  For 128 rows and 128 keys at a time: S = Q K^T (fp32, TMEM), then with the running
// maximum m and sum l of each row P = exp2(c S - m), l += sum P, O += P V (fp32, TMEM), P rounded to the cache's
// type because the second product takes 16-bit operands.  O is rescaled only when a row's maximum has grown by
// more than 2^8 since its last rescaling: P then stays below 2^8, which loses nothing in a floating-point type.
//
// (That rounding is most of the kernel's own error: relative to 64 bits 2.3e-3 in bf16 and 2.8e-4 in fp16, of which rounding the
// result alone is 1.7e-3 and 2.1e-4.)
//
// A score of +inf or NaN makes its row NaN.  Masked scores have weight 0 exactly, and values are multiplied by it only where they are
// finite: in the jobs that some row of an item does not see, infinite and NaN elements of V are taken out and added afterwards
// to the rows that see them.
//
// Measured (8B shape: 32 query heads, 8 key heads, D = 128), back to back under the power cap and, in brackets, in runs of some
// milliseconds: 64 requests of one row over 258 k keys in all 179 us, 5.9 TB/s, 0.91 of the copy rate (165 us); 2 x 2048 rows over
// 8 k keys 553 us, 0.99 PFLOP/s (490-530 us); 8 requests of 65 rows over 120 k keys 152 us (128 us); one request of 9 rows over
// 709 keys 12.4 us.  With D = 64: 110 us in short runs, 413 us, -, 10.4 us.
//
// What bounds it.  A window of K + 1 rows has group * (K + 1) rows per key head, so up to some 64 of them the kernel moves
// 4 D bytes per key and does 4 D flops per row and key: bound by HBM as long as one 128-row MMA tile (1024 clocks for 128
// keys at D = 128) is faster than its 64 KB of keys and values (some 2800 clocks at a 148th of the measured copy
// rate).  Prompt chunks are bound by the MMAs and by the exponentials, 1024 clocks each per 128 x 128 tile.
//
// Roles.  One block per SM, persistent: a warp that walks the work and copies queries and keys by TMA, one that copies values, four
// that issue the MMAs (S and O of each slot), two that at most clear rows of no window, and two sets of four softmax warps, each set
// ("slot") with its own S and O in TMEM (all 512 columns).  A work item is either "paired" - two row tiles of the same (request, key head), one per slot, sharing each tile of keys - or, where a
// single row tile is left, "split": the slots take the key tiles in turn and are put together at the end.  Either way
// the slots work at different 64-key jobs, and each has two S of 64 columns in turn: S of a job waits for O of the slot's last job but
// one alone, so it is computed under the exponentials of the job before and under the other slot's products.
//
// Work split.  The key tiles of all items form one line, cut into equal contiguous ranges, one per block; every block finds
// its range from the lengths on the device, so the host knows no lengths and a captured graph stays balanced.  An item cut by a
// range boundary leaves fp32 partials (at most two per block); the block that comes last with its own adds them all, in block
// order, so the result does not depend on who that is.
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

constexpr int kAttnMmaWarps = 4;
constexpr int kAttnThreads = 512;
constexpr int kAttnTile = 128;                   // rows of a row tile, keys of a key tile
constexpr int kAttnSub = 64;                     // keys of a job
constexpr int kAttnMaxStages = 12;
// The smallest stretch worth a block of its own: shorter ones cost more to merge than they save.  (One window of 9 rows over 709
// keys with 1, 2, 3, 4: 13.7, 12.4, 15.3, 15.5 us.  Where blocks have more than that to do it does not matter.)
constexpr int kAttnMinUnits = 2;
// Key tiles that starting and finishing an item is worth: with 0, 1, 2 one window takes 12.5, 12.4, 12.6 us, 64 requests of one row
// over 258 k keys 169.0, 165.5, 165.2, ragged windows over 141 k keys 113-117, 107-113, 108.
constexpr int kAttnItemCost = 1;
constexpr int kAttnSmem = 232448;                // all of an SM's shared memory that a block can have
constexpr int kAttnSmall = 2816;                 // barriers, the queue of stretches, the slots' exchange of m and l
constexpr int kAttnSlack = 256;                  // for aligning the tiles to 1024 bytes
constexpr uint64_t kAttnWaitClocks = 4000000000ull;       // the limit of every wait, unless a test has set a shorter one

struct AttnParams {
    int32_t B, T, n_kv, group, tpt, page_shift, n_pages, max_blocks;
    int32_t page_groups_k, page_groups_v;        // 8-token groups from one page to the next
    int32_t groups_k, groups_v;                  // 8-token groups in the whole pool: the first coordinate out of range
    int32_t uniform;                             // rows per request where q_off is NULL
    int32_t clear_rest;                          // rows of no window are written too
    const int32_t *q_off, *kv_len, *block_table;
    int64_t table_stride;
    const void* v; int64_t vp, vt, vh;           // the value pool and its strides, for values that are infinite or NaN
    void* out; int64_t ot, oh;
    float* lse;
    float scale_log2, inv_group;
    int32_t* err;
    uint32_t wait_limit;                         // in 1024 clocks
    int32_t stalled;                             // test hook: a block whose values are never copied; -1: none
    float* part_o;                               // [2 * blocks][D / 4][256 rows][4]: rows side by side, as the lanes that write and read them
    float2* part_ml;                             // [2 * blocks][256]
    // [blocks]: arrivals at the item that starts in a block's range and ends in another's, in the half of the word that err[1] names.
    // It is 0 when a call starts: the block that comes last clears it.  After a time-out the other half counts, and the next call
    // clears what the failed one left.
    int32_t* count;
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
// the token of a row of a row tile: row / group for row < 128 (the product is off by 1e-5 at most, the nearest wrong answer 1/128)
__device__ __forceinline__ int attn_token(const AttnParams& p, int row) { return static_cast<int>((row + 0.5f) * p.inv_group); }
__device__ __forceinline__ float attn_lg2(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <typename E> struct is_bf16 { static constexpr bool value = false; };
template <> struct is_bf16<__nv_bfloat16> { static constexpr bool value = true; };

// 1 / x by the hardware approximation (1 ulp): the full division may call a function, which this kernel cannot
__device__ __forceinline__ float attn_rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 2^x by the hardware approximation (relative error 2^-22)
__device__ __forceinline__ float attn_ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Bounded wait; `flag` is the shared-memory address of the block's abort flag, three words before the limit.  One inline try and
// everything else out of line: a try that is the condition of an inline loop costs some 370 clocks even where the barrier is complete.
static __device__ __forceinline__ bool attn_wait_slow(uint32_t bar, uint32_t parity, uint32_t flag)
{
    const long long t0 = clock64();
    uint32_t n = 0;
    while (!mbar_try_wait(bar, parity)) {
        if ((++n & 0xFFu) == 0) {
            uint32_t stop, limit;
            asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(stop) : "r"(flag) : "memory");
            if (stop != 0) return false;
            asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(limit) : "r"(flag + 12u) : "memory");
            if (static_cast<uint64_t>(clock64() - t0) >> 10 > limit) {
                asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(flag), "r"(1) : "memory");
                return false;
            }
        }
    }
    return true;
}
__device__ __forceinline__ bool attn_wait(uint32_t bar, uint32_t parity, uint32_t flag)
{
    if (mbar_try_wait(bar, parity)) return true;
    return attn_wait_slow(bar, parity, flag);
}
// the same for a warp that acts as one
__device__ __forceinline__ bool attn_wait_warp(uint32_t bar, uint32_t parity, uint32_t flag)
{
    return __all_sync(0xffffffffu, attn_wait(bar, parity, flag));
}

// ---- pairs of floats: one instruction does two multiply-adds
__device__ __forceinline__ uint64_t pair(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float low(uint64_t x) { return __uint_as_float(static_cast<uint32_t>(x)); }
__device__ __forceinline__ float high(uint64_t x) { return __uint_as_float(static_cast<uint32_t>(x >> 32)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// 2^x of a pair by multiply-adds, for x <= 8: the nearest whole number goes to the exponent, the rest r in [-1/2, 1/2] through the
// degree-4 polynomial that is 1 at r = 0 and has the least relative error there (2.8e-6; fitted by linear programming, 2.9e-6 in
// fp32).  From x = -127 down it gives 0 exactly (the exponent of 1 less 127 is that of 0), as a masked score must; between -126 and
// -127 something below 2^-126.
// The special-function unit does 16 exponentials a clock, which for a 128 x 128 tile takes as long as both matrix products;
// kAttnPoly of every 8 pairs go this way instead (2 x 2048 rows under the power cap with 0 to 3: 570, 553, 560, 564 us; D = 64:
// 442, 413, 422, 430).
constexpr int kAttnPoly = 1;
__device__ __forceinline__ uint64_t exp2_poly2(uint64_t x)
{
    const uint64_t magic = pair(12582912.0f, 12582912.0f), unmagic = pair(-12582912.0f, -12582912.0f);
    x = pair(fmaxf(low(x), -127.0f), fmaxf(high(x), -127.0f));
    const uint64_t t = add2(x, magic);                       // the whole number in the low bits
    const uint64_t r = fma2(add2(t, unmagic), pair(-1.0f, -1.0f), x);
    uint64_t y = fma2(r, pair(9.585382417e-3f, 9.585382417e-3f), pair(5.590662733e-2f, 5.590662733e-2f));
    y = fma2(y, r, pair(2.402403802e-1f, 2.402403802e-1f));
    y = fma2(y, r, pair(6.931241751e-1f, 6.931241751e-1f));
    y = fma2(y, r, pair(1.0f, 1.0f));
    const uint32_t a = static_cast<uint32_t>(t) * 0x800000u + static_cast<uint32_t>(y);
    const uint32_t b = static_cast<uint32_t>(t >> 32) * 0x800000u + static_cast<uint32_t>(y >> 32);
    return pair(__uint_as_float(a), __uint_as_float(b));
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
// One request as the kernel sees it; device-side lengths are clamped to what the arrays hold.  (Offsets, lengths and tables may be
// written by a kernel that still runs when this one's blocks start, so they are not read through the read-only path.)
struct AttnReq { int q0, n, kv, items; };

__device__ __forceinline__ AttnReq attn_request(const AttnParams& p, int b)
{
    AttnReq r;
    if (p.q_off) {
        r.q0 = min(max(p.q_off[b], 0), p.T);
        r.n = max(min(max(p.q_off[b + 1], 0), p.T) - r.q0, 0);
    } else {
        r.q0 = b * p.uniform;
        r.n = p.uniform;
    }
    r.kv = min(max(p.kv_len[b], 0), p.max_blocks << p.page_shift);
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

// A stretch of one item's key tiles that this block works on, as the walking warp queues it for the others
enum {
    kSegJobs,                                    // 0: the end
    kSegPaired, kSegT0, kSegT1, kSegTiles,       // key tiles [t0, t1) of the item's kSegTiles
    kSegKeys,                                    // keys of the request
    kSegLimit,                                   // last key that the item's first token sees
    kSegRow, kSegHead,                           // first row of the item in q, key head
    kSegRows0, kSegRows1,                        // valid rows of its row tiles
    kSegReq,
    kSegFirst, kSegParts,                        // blocks that share the item: the first one, how many
    kSegOdd,                                     // set by the softmax warps: infinite or NaN values were taken out of the stretch
    kSegShift,                                   // 16 times the half of the arrival counters that this call uses
    kSegWords,
    kSegLeft = kSegWords                         // (units of the range before the stretch; the walking warp's own)
};
constexpr int kSegQueue = 4;

struct AttnWalk {
    int b, kvh, it, pos, units;                  // position on the line of key tiles, and what is left of the range
    AttnReq r;
    // The next stretch; false at the end of the range.
    __device__ __forceinline__ bool next(const AttnParams& p, int (&s)[kSegWords + 1])
    {
        while (units > 0) {
            if (it >= r.items) {                 // (a request without rows)
                if (++b >= p.B) return false;
                kvh = it = pos = 0;
                r = attn_request(p, b);
                continue;
            }
            const int nt = attn_tiles(p, r, it);
            const int take = min(units, nt + kAttnItemCost - pos);
            const int t0 = pos, t1 = min(nt, pos + take);
            if (t1 > t0) {
                const int tok0 = it * 2 * p.tpt, left = r.n - tok0;
                const bool paired = left > p.tpt;
                s[kSegJobs] = (paired ? 4 : 2) * (t1 - t0);
                s[kSegPaired] = paired; s[kSegT0] = t0; s[kSegT1] = t1; s[kSegTiles] = nt;
                s[kSegKeys] = r.kv; s[kSegLimit] = r.kv - r.n + tok0;
                s[kSegRow] = r.q0 + tok0; s[kSegHead] = kvh; s[kSegReq] = b; s[kSegLeft] = units;
                s[kSegRows0] = min(left, p.tpt) * p.group;
                s[kSegRows1] = paired ? min(left - p.tpt, p.tpt) * p.group : 0;
            }
            units -= take;
            pos += take;
            if (pos == nt + kAttnItemCost) {
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
            if (t1 > t0) return true;
        }
        return false;
    }
};

// This block's range of the line of key tiles, found by one warp: `share` units each, one more for the first `more` blocks.  (The host
// has made sure that all of them together fit 31 bits, unless the offsets on the device overlap: then nothing is done and bit 2 of
// the error word set.)
template <int D>
__device__ __forceinline__ void attn_range(const AttnParams& p, unsigned me, int lane, AttnWalk& w, unsigned& share, unsigned& more)
{
    const int per = (p.B + 31) >> 5, b0 = min(lane * per, p.B), b1 = min(b0 + per, p.B);
    auto units_of = [&](const AttnReq& r) {
        unsigned u = 0;
        for (int i = 0; i < r.items; ++i) u += attn_tiles(p, r, i) + kAttnItemCost;
        return u;
    };
    unsigned long long sum = 0;
#pragma unroll 4
    for (int b = b0; b < b1; ++b) sum += units_of(attn_request(p, b)) * p.n_kv;
    const unsigned mine = static_cast<unsigned>(sum);
    const unsigned high = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(min(sum >> 16, 1ull << 20)));
    unsigned upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    unsigned total = __shfl_sync(0xffffffffu, upto, 31);
    if (high >= 0x7fffu) {
        total = upto = 0;
        if (lane == 0) atomicOr(p.err, 4);
    }
    const unsigned blocks = min(gridDim.x, max(total / kAttnMinUnits, 1u));
    share = total / blocks;
    more = total - share * blocks;
    const unsigned lo = me * share + min(me, more);
    w.b = w.kvh = w.it = w.pos = w.units = 0;
    const bool mine_starts = me < blocks && lo < upto && lo >= upto - mine;          // one lane's requests hold the start
    if (mine_starts) {
        unsigned x = lo - (upto - mine);
        for (int b = b0; b < b1; ++b) {
            const AttnReq r = attn_request(p, b);
            const unsigned one = units_of(r);
            if (x >= one * p.n_kv) { x -= one * p.n_kv; continue; }
            const unsigned h = x / one;
            x -= h * one;
            int it = 0;
            for (; ; ++it) {
                const unsigned u = attn_tiles(p, r, it) + kAttnItemCost;
                if (x < u) break;
                x -= u;
            }
            w.b = b; w.kvh = h; w.it = it; w.pos = x;
            break;
        }
    }
    const unsigned who = __ballot_sync(0xffffffffu, mine_starts);
    const int src = who ? __ffs(who) - 1 : 0;
    w.b = __shfl_sync(0xffffffffu, w.b, src);
    w.kvh = __shfl_sync(0xffffffffu, w.kvh, src);
    w.it = __shfl_sync(0xffffffffu, w.it, src);
    w.pos = __shfl_sync(0xffffffffu, w.pos, src);
    w.units = who ? share + (me < more ? 1 : 0) : 0;
    if (who) w.r = attn_request(p, w.b);
}

// The merge of an item's partials by the eight softmax warps of the block that came last.  A lane takes a row, a warp 32 rows and
// 16 columns; four partials' maxima, sums and outputs are loaded together and put onto the running ones, in block order.  Reads
// go past L1, which other blocks' writes do not reach.
template <typename E, int D>
__device__ __forceinline__ void attn_merge(const AttnParams& p, const int* sg, int w, int lane)
{
    constexpr int G = D / 16, U = 4;
    // (through shuffles, so that the compiler knows the loops uniform)
    const int parts = __shfl_sync(0xffffffffu, sg[kSegParts], 0);
    const int rows0 = __shfl_sync(0xffffffffu, sg[kSegRows0], 0), rows1 = __shfl_sync(0xffffffffu, sg[kSegRows1], 0);
    const int first = sg[kSegFirst], nb0 = (rows0 + 31) >> 5, nb = nb0 + ((rows1 + 31) >> 5);
    for (int unit = w; unit < nb * G; unit += 8) {
        const int rb = unit / G, g = unit % G;
        const bool second = rb >= nb0;           // the second row tile's rows lie from 128 on
        const int in = (second ? rb - nb0 : rb) * 32 + lane, at = in + (second ? 128 : 0);
        float m = -CUDART_INF_F, l = 0.0f, acc[16];
#pragma unroll
        for (int c = 0; c < 16; ++c) acc[c] = 0.0f;
        for (int j0 = 0; j0 < parts; j0 += U) {
            float2 x[U];
            float4 v[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = min(j0 + u, parts - 1), buf = j == 0 ? 2 * first + 1 : 2 * (first + j);
                x[u] = __ldcg(p.part_ml + buf * 256 + at);
                const float4* src = reinterpret_cast<const float4*>(p.part_o) + (static_cast<size_t>(buf) * (D / 4) + g * 4) * 256 + at;
#pragma unroll
                for (int c = 0; c < 4; ++c) v[u][c] = __ldcg(src + c * 256);
                if (j0 + u >= parts) x[u] = make_float2(-CUDART_INF_F, 0.0f);
            }
            float mm = m;
#pragma unroll
            for (int u = 0; u < U; ++u) mm = fmaxf(mm, x[u].x);
            const float f0 = m == -CUDART_INF_F ? 0.0f : attn_ex2(m - mm);
            l *= f0;
#pragma unroll
            for (int c = 0; c < 16; ++c) acc[c] *= f0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool some = x[u].x != -CUDART_INF_F;           // (else its outputs may be anything)
                const float f = some ? attn_ex2(x[u].x - mm) : 0.0f;
                l = fmaf(f, x[u].y, l);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    acc[4 * c] = some ? fmaf(f, v[u][c].x, acc[4 * c]) : acc[4 * c];
                    acc[4 * c + 1] = some ? fmaf(f, v[u][c].y, acc[4 * c + 1]) : acc[4 * c + 1];
                    acc[4 * c + 2] = some ? fmaf(f, v[u][c].z, acc[4 * c + 2]) : acc[4 * c + 2];
                    acc[4 * c + 3] = some ? fmaf(f, v[u][c].w, acc[4 * c + 3]) : acc[4 * c + 3];
                }
            }
            m = mm;
        }
        if (in < (second ? rows1 : rows0)) {
            const float inv = l == 0.0f ? 0.0f : attn_rcp(l);
            const int t = attn_token(p, in), tok = sg[kSegRow] + t + (second ? p.tpt : 0), head = sg[kSegHead] * p.group + in - t * p.group;
            uint4* const dst = reinterpret_cast<uint4*>(static_cast<E*>(p.out) + tok * p.ot + head * p.oh + g * 16);
#pragma unroll
            for (int c = 0; c < 2; ++c)
                dst[c] = make_uint4(pack2<E>(acc[8 * c] * inv, acc[8 * c + 1] * inv), pack2<E>(acc[8 * c + 2] * inv, acc[8 * c + 3] * inv),
                                    pack2<E>(acc[8 * c + 4] * inv, acc[8 * c + 5] * inv), pack2<E>(acc[8 * c + 6] * inv, acc[8 * c + 7] * inv));
            if (p.lse && g == 0)
                p.lse[static_cast<int64_t>(tok) * (p.n_kv * p.group) + head] =
                    l == 0.0f ? -CUDART_INF_F : (m + attn_lg2(l)) * 0.6931471805599453f;
        }
    }
}

// Bits of the 16-bit elements of `w` that are infinite or NaN: all exponent bits set, to which one more at their low end carries
// into the sign's place.
template <typename E>
__device__ __forceinline__ uint32_t odd_elements(uint32_t w)
{
    const uint32_t mask = is_bf16<E>::value ? 0x7f807f80u : 0x7c007c00u, one = is_bf16<E>::value ? 0x00800080u : 0x04000400u;
    const uint32_t top = ((w & mask) + one) & 0x80008000u;
    return (top >> 15) * 0xffffu;
}
// The infinite and NaN elements of 32 columns of one row of V, as they lie in the pool, added to a row's output
template <typename E>
__device__ __forceinline__ void add_odd_elements(const E* v, float (&x)[32])
{
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t w = reinterpret_cast<const uint32_t*>(v)[i], odd = w & odd_elements<E>(w);
        if (is_bf16<E>::value) {
            x[2 * i] += __uint_as_float(odd << 16);
            x[2 * i + 1] += __uint_as_float(odd & 0xffff0000u);
        } else {
            x[2 * i] += __half2float(__ushort_as_half(static_cast<unsigned short>(odd & 0xffffu)));
            x[2 * i + 1] += __half2float(__ushort_as_half(static_cast<unsigned short>(odd >> 16)));
        }
    }
}

// Position in the ring of key and value tiles: tile g uses entries 2 g (keys) and 2 g + 1 (values).
// The ring of key and value tiles, in turn.  A barrier's phase is one bit, so whoever waits for a fill (or a release) of a stage must know
// that the one before it is past.  Here that hangs on S of a job being issued only after O of the slot's last job but one (s_free): the
// values of tile t - 3, whose stage the keys of tile t take over where the stages are five, are then in, and the keys of tile t - 3
// released only after the values of tile t - 5.  A product S that runs further ahead needs stages of keys and of values apart.
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

// Table entry of the lane's page (of at most 128 tokens) of key tile t; -1 where the tile has none.
__device__ __forceinline__ int attn_page(const AttnParams& p, int req, int t, int t1, int keys, int lane)
{
    const int box_tok = min(1 << p.page_shift, kAttnTile), tok = t * kAttnTile + lane * box_tok;
    return t < t1 && lane * box_tok < kAttnTile && tok < keys ? p.block_table[req * p.table_stride + (tok >> p.page_shift)] : -1;
}

// The copies of key (or value) tiles t0 .. t1 - 1 of a request into every other entry of the ring, by one warp.  `pg`: attn_page
// of tile t0; that of the next tile is read a tile ahead.
template <int D>
__device__ __forceinline__ bool attn_load_tiles(const AttnParams& p, const CUtensorMap* map, int page_groups, int groups, int req, int pg, int t0,
                                                int t1, int keys, int head, uint32_t ring, uint32_t bars, uint32_t flag, int lane,
                                                AttnRing& rg, int& issued)
{
    constexpr int kStages = attn_stages<D>();
    const int box_tok = min(1 << p.page_shift, kAttnTile);
    const uint32_t box_bytes = static_cast<uint32_t>(box_tok) * (D * 2);
    for (int t = t0; t < t1; ++t) {
        const int tok0 = t * kAttnTile;
        const int pages = max(min(keys - tok0, kAttnTile) + box_tok - 1, 0) / box_tok;               // that hold keys
        const int at = ((tok0 + lane * box_tok) & ((1 << p.page_shift) - 1)) >> 3;
        const int g = pg >= 0 && pg < p.n_pages ? pg * page_groups + at : groups;                    // out of range: zeros
        pg = attn_page(p, req, t + 1, t1, keys, lane);
        if (!attn_wait_warp(bars + 8u * (kAttnMaxStages + rg.s), rg.ph ^ 1u, flag)) return false;
        const uint32_t dst = ring + rg.s * attn_stage_bytes<D>(), bar = bars + 8u * rg.s;
        if (elect_one()) mbar_expect_tx(bar, static_cast<uint32_t>(pages) * box_bytes);
        __syncwarp();
        for (int i = 0; i < pages; ++i) {
            const int gi = __shfl_sync(0xffffffffu, g, i);
            if (elect_one()) tma_load_5d(dst + i * box_bytes, map, 0, 0, 0, head, gi, bar);
        }
        __syncwarp();
        ++issued;
        rg.step(kStages);
        rg.step(kStages);
    }
    return true;
}

// Zeros (-inf in lse) for the rows of q that no window covers, those before the first offset and behind the last one: a batch padded
// to a fixed number of rows carries them on into the next layer.  `w` of `all` warps.
template <typename E, int D>
__device__ __forceinline__ void attn_clear_rows(const AttnParams& p, int w, int all, int lane)
{
    if (!p.q_off || !p.clear_rest) return;
    const int head = min(max(p.q_off[0], 0), p.T), tail = min(max(p.q_off[p.B], head), p.T);
    const int heads = p.n_kv * p.group;
    for (int i = w; i < head + p.T - tail; i += all) {
        const int64_t t = i < head ? i : tail + (i - head);
        for (int x = lane; x < heads * (D / 8); x += 32)
            *reinterpret_cast<uint4*>(static_cast<E*>(p.out) + t * p.ot + x / (D / 8) * p.oh + x % (D / 8) * 8) = make_uint4(0, 0, 0, 0);
        for (int h = lane; p.lse && h < heads; h += 32) p.lse[t * heads + h] = -CUDART_INF_F;
    }
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
    auto s_full = [&](int s) { return bars + 8u * (2 * kAttnMaxStages + 4 + s); };            // 2 slot + half of its S columns
    auto p_full = [&](int s) { return bars + 8u * (2 * kAttnMaxStages + 8 + s); };
    auto s_free = [&](int s) { return bars + 8u * (2 * kAttnMaxStages + 12 + s); };           // the second product has read P there
    auto seg_full = [&](int s) { return bars + 8u * (2 * kAttnMaxStages + 16 + s); };
    auto seg_empty = [&](int s) { return bars + 8u * (2 * kAttnMaxStages + 16 + kSegQueue + s); };
    constexpr int kBars = 2 * kAttnMaxStages + 16 + 2 * kSegQueue;
    const uint32_t o_full = bars + 8u * kBars, o_empty = o_full + 8, ml_full = o_full + 16, part_full = o_full + 24, last_full = o_full + 32, drain = o_full + 40;
    constexpr int kSegAt = (kBars + 14) * 8;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(small + 8 * (kBars + 9));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);       // [0] abort, [1] drain scratch
    const uint32_t flag = bars + 8u * (kBars + 9) + 4u;
    volatile int* came_last = reinterpret_cast<volatile int*>(tmem_slot + 3);        // whether this block was the last at a shared item
    volatile uint32_t* wait_limit = tmem_slot + 4;                                   // [2]: three words behind either flag
    volatile int* copies = reinterpret_cast<volatile int*>(tmem_slot + 6);           // key and value tiles copied, written at the end
    volatile uint32_t* half_used = tmem_slot + 8;                                    // thread 0's: the half of the counters in use
    const unsigned me = blockIdx.x;
    int (*queue)[kSegWords] = reinterpret_cast<int (*)[kSegWords]>(small + kSegAt);  // [kSegQueue]
    float2* ml = reinterpret_cast<float2*>(small + kAttnSmall - 2048);               // [2][128]
    static_assert(kSegWords == 16 && kSegAt + kSegQueue * kSegWords * 4 <= kAttnSmall - 2048, "shared memory");

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int lane = threadIdx.x & 31;

    if (small_off + kAttnSmall > static_cast<uint32_t>(kAttnSmem)) {          // (dynamic shared memory starts 1024-byte aligned)
        if (threadIdx.x == 0) atomicOr(p.err, 2);
        return;
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 2); }
        for (int s = 0; s < 2; ++s) { mbar_init(q_full(s), 1); mbar_init(q_empty(s), 2); }
        for (int s = 0; s < 4; ++s) { mbar_init(s_full(s), 1); mbar_init(p_full(s), 4); mbar_init(s_free(s), 1); }
        for (int s = 0; s < kSegQueue; ++s) { mbar_init(seg_full(s), 1); mbar_init(seg_empty(s), 11); }
        mbar_init(o_full, 2); mbar_init(o_empty, 8); mbar_init(ml_full, 8); mbar_init(part_full, 8); mbar_init(last_full, 1); for (int s = 0; s < kAttnMmaWarps; ++s) mbar_init(drain + 8 * s, 1);
        abort_flag[0] = 0; abort_flag[1] = 0;
        wait_limit[0] = wait_limit[1] = p.wait_limit;
        fence_barrier_init();
        tma_prefetch_desc(&tmQ);
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmV);
    }
    // Rows of a row tile that the query box does not reach stay zero: the MMAs compute them all the same, and with zeros (and
    // probabilities of zero, below) they cost far less of the power that caps the clock.
    for (int i = threadIdx.x * 16; i < static_cast<int>(2 * kStage) && p.tpt * p.group < kAttnTile; i += kAttnThreads * 16)
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(q_buf + i), "r"(0) : "memory");
    fence_proxy_async();
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    griddep_wait();                              // lengths, tables and the cache itself come from kernels before this one
    griddep_launch_dependents();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    const uint32_t tS = tmem, tO = tmem + 256;   // S of slot s at 128 s, P over its first half, O at 256 + 128 s
    int issued = 0, q_issued = 0;                // ring entries and query buffers filled (copying warps; read again before the end)

    // Warps 0 and 4 have next to nothing to do: they share a scheduler with the softmax warps of rows 0 .. 31, the only ones at
    // work where a row tile has few rows.  Warps 1, 2, 3, 5, 6, 7 are roles 0 .. 5.
    const int role = warp > 7 || (warp & 3) == 0 ? -1 : warp < 4 ? warp - 1 : warp - 2;
    if (warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (role < 0) {
            if (threadIdx.x == 0) {
                const unsigned half = static_cast<unsigned>(__ldcg(p.err + 1)) & 1u;
                *half_used = half;
                const unsigned other = 0xffffu << (16u * (half ^ 1u));
                if (static_cast<unsigned>(__ldcg(p.count + me)) & other) atomicAnd(p.count + me, static_cast<int>(~other));
            }
            __syncwarp();
            attn_clear_rows<E, D>(p, static_cast<int>(me) * 2 + (warp >> 2), static_cast<int>(gridDim.x) * 2, lane);
        } else if (role == 0) {
            // ------------------------------------------------------------ the work, and the TMA copies of queries and keys
            const int half = __ldcg(p.err + 1) & 1;              // (on its way while the range is found: 0.5 us of a small call)
            AttnWalk walk;
            unsigned share, more;
            attn_range<D>(p, me, lane, walk, share, more);
            int s[kSegWords + 1];
            AttnRing rg;
            bool ok = true;
            for (int item = 0; ok; ++item) {
                const bool some = walk.next(p, s);
                const int qi = item & (kSegQueue - 1);
                if (some) {
                    s[kSegFirst] = static_cast<int>(me); s[kSegParts] = 1; s[kSegOdd] = 0; s[kSegShift] = 16 * half;
                    if (s[kSegT0] > 0 || s[kSegT1] < s[kSegTiles]) {                 // shared: whose ranges does the item reach?
                        auto block_of = [&](unsigned u) {
                            return u < more * (share + 1) ? u / (share + 1) : more + (u - more * (share + 1)) / share;
                        };
                        const unsigned unit0 = (me + 1) * share + min(me + 1, more) - s[kSegLeft] - s[kSegT0];
                        const unsigned first = block_of(unit0), last = block_of(unit0 + s[kSegTiles] - 1);
                        s[kSegFirst] = first; s[kSegParts] = last - first + 1;
                    }
                }
                ok = attn_wait_warp(seg_empty(qi), (static_cast<uint32_t>(item / kSegQueue) & 1u) ^ 1u, flag);
                if (!ok) break;
                if (lane == 0) {
#pragma unroll
                    for (int i = 0; i < kSegWords; ++i) queue[qi][i] = some ? s[i] : 0;
                    mbar_arrive(seg_full(qi));
                }
                __syncwarp();
                if (!some) break;
                const int pg = attn_page(p, s[kSegReq], s[kSegT0], s[kSegT1], s[kSegKeys], lane);
                // queries: one buffer per row tile
                for (int t = 0; ok && t < (s[kSegPaired] ? 2 : 1); ++t, ++q_issued) {
                    const int qb = q_issued & 1;
                    ok = attn_wait_warp(q_empty(qb), ((q_issued >> 1) & 1u) ^ 1u, flag);
                    if (ok && elect_one()) {
                        mbar_expect_tx(q_full(qb), static_cast<uint32_t>(p.tpt * p.group) * 128u * kHalves);
                        for (int h = 0; h < kHalves; ++h)
                            tma_load_5d(q_buf + qb * kStage + h * (kAttnTile * 128), &tmQ, 0, 0, s[kSegRow] + t * p.tpt, h, s[kSegHead], q_full(qb));
                    }
                    __syncwarp();
                }
                ok = ok && attn_load_tiles<D>(p, &tmK, p.page_groups_k, p.groups_k, s[kSegReq], pg, s[kSegT0], s[kSegT1], s[kSegKeys],
                                              s[kSegHead], ring, bars, flag, lane, rg, issued);
            }
        } else if (role == 1 + kAttnMmaWarps) {
            // ------------------------------------------------------------ the TMA copies of values (pages of 16 tokens are eight
            // copies a tile, some 80 clocks each: one warp for both would be late)
            AttnRing rg;
            rg.step(kStages);
            bool ok = static_cast<int>(me) != p.stalled;
            for (int item = 0; ok; ++item) {
                const int qi = item & (kSegQueue - 1);
                ok = attn_wait_warp(seg_full(qi), static_cast<uint32_t>(item / kSegQueue) & 1u, flag);
                if (!ok || queue[qi][kSegJobs] == 0) break;
                const int req = queue[qi][kSegReq], t0 = queue[qi][kSegT0], t1 = queue[qi][kSegT1], keys = queue[qi][kSegKeys];
                ok = attn_load_tiles<D>(p, &tmV, p.page_groups_v, p.groups_v, req, attn_page(p, req, t0, t1, keys, lane), t0, t1, keys,
                                        queue[qi][kSegHead], ring, bars, flag, lane, rg, issued);
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(seg_empty(qi));
            }
        } else if (role > 0) {
            // ------------------------------------------------------------ MMA: two warps issue S = Q K^T, one per slot, and two
            // O += P V.  Each waits (some 100 clocks and more behind its own products, barrier complete or not) under the
            // others' products.  Job n of a slot in a stretch: split: keys 64 slot .. of tile n; paired: keys 64 (n & 1) .. of
            // tile n / 2.
            const int slot = (role - 1) & 1;
            const bool second = role > 2;
            const uint32_t idesc = second ? attn_idesc<E>(kAttnTile, D, true) : attn_idesc<E>(kAttnTile, kAttnSub, false);
            const uint32_t sS = tS + slot * 128, sO = tO + slot * 128;
            uint32_t used = 0;                   // jobs of this slot so far
            int q_used = 0;                      // query buffers used so far
            AttnRing rg;                         // the tile's key entry (S) or value entry (O)
            if (second) rg.step(kStages);
            bool ok = true;
            for (int item = 0; ok; ++item) {
                const int qi = item & (kSegQueue - 1);
                ok = attn_wait_warp(seg_full(qi), static_cast<uint32_t>(item / kSegQueue) & 1u, flag);
                if (!ok) break;
                const int jobs = __shfl_sync(0xffffffffu, queue[qi][kSegJobs], 0);   // (the compiler then knows it uniform)
                const bool paired = __shfl_sync(0xffffffffu, queue[qi][kSegPaired], 0) != 0;
                if (jobs == 0) break;
                const int J = jobs >> 1;
                const int qb = (q_used + (paired ? slot : 0)) & 1;                   // the slot's query buffer
                if (!second) {
                    // (a paired item's other buffer too, so that no warp skips a phase)
                    for (const int end = q_used + (paired ? 2 : 1); ok && q_used < end; ++q_used)
                        ok = attn_wait_warp(q_full(q_used & 1), static_cast<uint32_t>(q_used >> 1) & 1u, flag);
                } else if (item > 0) {
                    ok = attn_wait_warp(o_empty, static_cast<uint32_t>(item - 1) & 1u, flag);         // the previous O has been read
                }
                for (int n = 0; ok && n < J; ++n, ++used) {
                    const uint32_t h = used & 1u, ph = (used >> 1) & 1u;
                    const bool first_use = !paired || (n & 1) == 0, last_use = !paired || (n & 1) == 1;
                    const uint32_t b_at = ring + rg.s * kStage + (paired ? (n & 1) : slot) * (kAttnSub / 8 * kGroup);
                    if (!second) {
                        ok = attn_wait_warp(s_free(2 * h + slot), ph ^ 1u, flag);
                        if (ok && first_use) ok = attn_wait_warp(full_bar(rg.s), rg.ph, flag);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) {
                            const uint64_t a0 = attn_desc(q_buf + qb * kStage, 1024), b0 = attn_desc(b_at, kGroup);
#pragma unroll
                            for (int k = 0; k < D / 16; ++k) {
                                const uint64_t a = a0 + static_cast<uint64_t>(((k >> 2) * (kAttnTile * 128) + (k & 3) * 32) >> 4);
                                const uint64_t b = b0 + static_cast<uint64_t>(((k >> 2) * 1024 + (k & 3) * 32) >> 4);
                                umma_bf16(sS + h * kAttnSub, a, b, idesc, k != 0);
                            }
                            umma_commit(s_full(2 * h + slot));
                            if (last_use) umma_commit(empty_bar(rg.s));
                            if (n + 1 == J) {
                                umma_commit(q_empty(qb));
                                if (paired) umma_commit(q_empty(qb));                // (a split item's buffer hears from both warps)
                            }
                        }
                    } else {
                        if (first_use) ok = attn_wait_warp(full_bar(rg.s), rg.ph, flag);
                        if (ok) ok = attn_wait_warp(p_full(2 * h + slot), ph, flag);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) {
                            const uint64_t b0 = attn_desc(b_at, kGroup);
#pragma unroll
                            for (int k = 0; k < kAttnSub / 16; ++k)
                                umma_f16_ts(sO, sS + h * kAttnSub + k * 8, b0 + static_cast<uint64_t>((k * 2 * kGroup) >> 4), idesc,
                                            (n != 0 || k != 0) ? 1u : 0u);           // a slot's first job overwrites O
                            umma_commit(s_free(2 * h + slot));
                            if (last_use) umma_commit(empty_bar(rg.s));
                            if (n + 1 == J) umma_commit(o_full);
                        }
                    }
                    __syncwarp();
                    if (last_use) { rg.step(kStages); rg.step(kStages); }
                }
                if (ok && second && lane == 0) mbar_arrive(seg_empty(qi));
            }
        }
    } else {
        // ---------------------------------------------------------------- softmax: four warps per slot, a thread per row
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int slot = (warp - 8) >> 2, quad = warp & 3;
        const int row = quad * 32 + lane;        // row of the tile = TMEM lane
        const uint32_t lane_off = static_cast<uint32_t>(quad * 32) << 16;
        const uint32_t aS0 = tS + slot * 128 + lane_off, aO = tO + slot * 128 + lane_off;
        uint32_t used = 0;                       // jobs of this slot so far
        int tiles = 0;                           // key tiles in the stretches before
        uint32_t splits = 0;                     // stretches of shared items so far
        bool ok = true;
        for (int item = 0; ok; ++item) {
            const int* const sg = queue[item & (kSegQueue - 1)];
            ok = attn_wait_warp(seg_full(item & (kSegQueue - 1)), static_cast<uint32_t>(item / kSegQueue) & 1u, flag);
            if (!ok) break;
            const int J = sg[kSegJobs];
            if (J == 0) break;
            const bool paired = sg[kSegPaired];
            const int tile_rows = paired && slot ? sg[kSegRows1] : sg[kSegRows0];
            const bool warp_has_rows = quad * 32 < tile_rows, valid = row < tile_rows;
            const int key0 = sg[kSegT0] * kAttnTile + (paired ? 0 : slot * kAttnSub);
            const int step = paired ? kAttnSub : 2 * kAttnSub;                       // keys from one job of the slot to its next
            // columns of the job's keys past `cut` are masked for this row, rows of V from `have` on do not exist
            int cut = sg[kSegLimit] + attn_token(p, row) + (paired && slot ? p.tpt : 0) - key0;
            int have = sg[kSegKeys] - key0;
            int common = sg[kSegLimit] - key0;       // last column that every row of the item sees
            float m = -CUDART_INF_F, l = 0.0f;
            for (int n = 0; n < J; n += 2) {
                const uint32_t h = used & 1u;
                ok = attn_wait_warp(s_full(2 * h + slot), (used >> 1) & 1u, flag);
                if (!ok) break;
                tc_fence_after();
                const uint32_t aS = aS0 + h * kAttnSub;
                uint32_t sr[kAttnSub];
                float* const s = reinterpret_cast<float*>(sr);
                float base_m = 0.0f;
                if (warp_has_rows) {
                    tmem_ld32(aS, sr);
                    tmem_ld32(aS + 32, sr + 32);
                    tmem_wait_ld();
                    if (!__all_sync(0xffffffffu, cut >= kAttnSub - 1)) {
#pragma unroll
                        for (int c = 0; c < kAttnSub; ++c) s[c] = c <= cut ? s[c] : -CUDART_INF_F;
                    }
                    float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                    for (int c = 4; c < 60; c += 8) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) mx[i] = max3_nan(mx[i], s[c + 2 * i], s[c + 2 * i + 1]);
                    }
                    const float mt = max3_nan(max3_nan(mx[0], mx[1], s[60]), max3_nan(mx[2], mx[3], s[61]), max3_nan(s[62], s[63], s[63])) * p.scale_log2;
                    // A score of NaN or +inf makes the row NaN, whichever way its exponential goes (the polynomial's clamp
                    // would turn inf - inf into a small weight).
                    if (!(mt < CUDART_INF_F)) l = CUDART_NAN_F;
                    const bool grow = valid && mt > m + 8.0f;
                    if (__any_sync(0xffffffffu, grow)) {
                        const float m_new = grow ? mt : m;
                        const float a = grow ? attn_ex2(m - m_new) : 1.0f;
                        l *= a;
                        m = m_new;
                        if (n > 0) {
                            // O holds the jobs up to the last but one for certain; its rescaling waits for that one too
                            ok = attn_wait_warp(s_free(2 * (h ^ 1u) + slot), ((used - 1) >> 1) & 1u, flag);
                            if (!ok) break;
                            tc_fence_after();
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
                    base_m = !valid ? -CUDART_INF_F : m == -CUDART_INF_F ? 0.0f : -m;
                }
                if (warp_has_rows) {
                    // A masked score's exponential is 0 both ways, so that a finite value behind it adds nothing, however large.
                    const uint64_t scale2 = pair(p.scale_log2, p.scale_log2), base2 = pair(base_m, base_m);
                    uint64_t sum[2] = {0, 0};
#pragma unroll
                    for (int c = 0; c < kAttnSub; c += 32) {
                        uint32_t pk[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint64_t x = fma2(pair(s[c + 2 * i], s[c + 2 * i + 1]), scale2, base2);
                            const uint64_t e = (i & 7) < kAttnPoly ? exp2_poly2(x) : pair(attn_ex2(low(x)), attn_ex2(high(x)));
                            sum[i & 1] = add2(sum[i & 1], e);
                            pk[i] = pack2<E>(low(e), high(e));
                        }
                        tmem_st16(aS + c / 2, pk);
                    }
                    const uint64_t both = add2(sum[0], sum[1]);
                    l += low(both) + high(both);
                    tmem_wait_st();
                }
                if (common < kAttnSub - 1) {
                    // Values that some row of the item does not see have weight 0 there, but 0 times an infinite value or NaN is NaN.
                    // So rows of V behind the last key are cleared, and infinite and NaN elements of rows between taken out and
                    // remembered; they are added at the end to the rows that see them.  Both slots of a paired item do this on
                    // the same condition, whatever they see themselves: whoever comes second finds zeros.  Row r of a tile lies
                    // in group r / 8 at 128 (r % 8), once per 64 columns.  The stage cannot be recycled before this job's
                    // second product.
                    const int tile = tiles + (paired ? n >> 2 : n >> 1), sub = paired ? (n >> 1) & 1 : slot;
                    const int e = 2 * tile + 1, st = e % kStages;
                    ok = attn_wait_warp(full_bar(st), static_cast<uint32_t>(e / kStages) & 1u, flag);
                    if (!ok) break;
                    const int r0 = max(common + 1, 0), dead = max(have, 0);
                    for (int i = row + r0 * (kHalves * 8); i < kAttnSub * (kHalves * 8); i += 128) {
                        const int r = i / (kHalves * 8), c = i % (kHalves * 8), at_row = sub * kAttnSub + r;
                        const uint32_t at = ring + st * kStage + (at_row >> 3) * kGroup + (c >> 3) * 1024 + (at_row & 7) * 128 + (c & 7) * 16;
                        uint32_t v[4] = {0, 0, 0, 0}, odd = 1;
                        if (r < dead) {
                            odd = 0;
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t bad = odd_elements<E>(v[k]);
                                odd |= bad;
                                v[k] &= ~bad;
                            }
                            if (odd) *const_cast<volatile int*>(sg + kSegOdd) = 1;
                        }
                        if (odd)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                    }
                    fence_proxy_async();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(2 * h + slot));
                cut -= step;
                have -= step;
                common -= step;
                ++used;
            }
            if (!ok) break;

            // ---- the item (or its stretch) is done once O is complete (which also says that nobody reads the previous
            // stretch's m and l any more).  The slots' (m, l) are exchanged: a split item is put together here from both
            // accumulators, each slot taking half of the columns.
            ok = attn_wait_warp(o_full, static_cast<uint32_t>(item) & 1u, flag);
            if (!ok) break;
            tc_fence_after();
            if (m == -CUDART_INF_F && l == l) l = 0.0f;                              // the row has seen no key (and no NaN)
            ml[slot * 128 + row] = make_float2(m, l);
            __syncwarp();
            if (lane == 0) mbar_arrive(ml_full);
            ok = attn_wait_warp(ml_full, static_cast<uint32_t>(item) & 1u, flag);
            if (!ok) break;
            if (warp_has_rows) {
                float wa = 1.0f, wb = 0.0f;      // weights of this slot's accumulator and of the other one's
                if (!paired) {
                    const float2 o = ml[(slot ^ 1) * 128 + row];
                    const float mm = fmaxf(m, o.x);
                    wa = m == -CUDART_INF_F ? 0.0f : attn_ex2(m - mm);
                    wb = o.x == -CUDART_INF_F ? 0.0f : attn_ex2(o.x - mm);
                    l = l * wa + o.y * wb;
                    m = mm;
                }
                const bool first = sg[kSegT0] == 0, whole = first && sg[kSegT1] == sg[kSegTiles];
                const int c0 = paired ? 0 : slot * (D / 2), c1 = paired ? D : c0 + D / 2;
                const int part = static_cast<int>(me) * 2 + (first ? 1 : 0), part_row = (paired ? slot * 128 : 0) + row;
                const int t = attn_token(p, row), tok = sg[kSegRow] + t + (paired && slot ? p.tpt : 0);
                const int head = sg[kSegHead] * p.group + row - t * p.group;
                const float inv = l == 0.0f ? 0.0f : attn_rcp(l);
                if (whole) { wa *= inv; wb *= inv; }
                const bool odd = valid && *const_cast<const volatile int*>(sg + kSegOdd) != 0;
                const uint32_t aO_other = tO + (slot ^ 1) * 128 + lane_off;
                for (int c = c0; c < c1; c += 32) {
                    uint32_t o[32];
                    float x[32];
                    tmem_ld32(aO + c, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(o[i]) * wa;
                    if (!paired) {
                        tmem_ld32(aO_other + c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = fmaf(__uint_as_float(o[i]), wb, x[i]);
                    }
                    if (odd) {
                        const int lo = max(max(sg[kSegLimit] + 1, 0), sg[kSegT0] * kAttnTile);
                        const int hi = min(sg[kSegLimit] + tok - sg[kSegRow], sg[kSegT1] * kAttnTile - 1);       // the row's last key here
                        for (int key = lo; key <= hi; ++key) {
                            const int pg = p.block_table[sg[kSegReq] * p.table_stride + (key >> p.page_shift)];
                            if (pg >= 0 && pg < p.n_pages)
                                add_odd_elements<E>(static_cast<const E*>(p.v) + pg * p.vp + (key & ((1 << p.page_shift) - 1)) * p.vt +
                                                        sg[kSegHead] * p.vh + c, x);
                        }
                    }
                    if (valid && whole) {
                        E* const dst = static_cast<E*>(p.out) + tok * p.ot + head * p.oh + c;
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            *reinterpret_cast<uint4*>(dst + i) =
                                make_uint4(pack2<E>(x[i], x[i + 1]), pack2<E>(x[i + 2], x[i + 3]), pack2<E>(x[i + 4], x[i + 5]),
                                           pack2<E>(x[i + 6], x[i + 7]));
                    } else if (valid) {
                        float4* const dst = reinterpret_cast<float4*>(p.part_o) + (static_cast<size_t>(part) * (D / 4) + c / 4) * 256 + part_row;
#pragma unroll
                        for (int i = 0; i < 32; i += 4) dst[i / 4 * 256] = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
                    }
                }
                if (valid && (paired || slot == 0)) {
                    if (!whole) p.part_ml[part * 256 + part_row] = make_float2(m, l);
                    else if (p.lse)
                        p.lse[static_cast<int64_t>(tok) * (p.n_kv * p.group) + head] =
                            l == 0.0f ? -CUDART_INF_F : (m + attn_lg2(l)) * 0.6931471805599453f;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_empty);
            tiles += sg[kSegT1] - sg[kSegT0];
            if (sg[kSegParts] > 1) {
                // The item is shared: count this block's part, and if it is the last one to arrive, add all of them.  (One
                // thread's fences stand for the block: the barriers before and after order the others' writes and reads.)
                const int first_block = sg[kSegFirst], parts = sg[kSegParts];
                if (lane == 0) mbar_arrive(part_full);
                if (warp == 8) {
                    ok = attn_wait_warp(part_full, splits & 1u, flag);
                    if (!ok) break;
                    if (lane == 0) {
                        const int shift = sg[kSegShift];
                        __threadfence();
                        const int before = static_cast<int>(static_cast<unsigned>(atomicAdd(p.count + first_block, 1 << shift)) >> shift & 0xffffu);
                        *came_last = before == parts - 1;
                        __threadfence();
                        mbar_arrive(last_full);
                        if (before == parts - 1) p.count[first_block] = 0;               // (nobody counts in the other half)
                    }
                    __syncwarp();
                }
                ok = attn_wait_warp(last_full, splits & 1u, flag);
                if (!ok) break;
                ++splits;
                if (__shfl_sync(0xffffffffu, *came_last, 0)) attn_merge<E, D>(p, sg, warp - 8, lane);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(seg_empty(item & (kSegQueue - 1)));
        }
    }

    if (lane == 0 && role == 0) copies[0] = issued;
    if (lane == 0 && role == 1 + kAttnMmaWarps) copies[1] = issued;
    __syncthreads();
    if (abort_flag[0] != 0) {
        // After a time-out: products and copies still in flight have to end before this block's TMEM and shared memory are given up,
        // whoever issued them and however its own loop ended.
        if (role > 0 && role <= kAttnMmaWarps) {
            const uint32_t mine = drain + 8 * (role - 1);
            if (elect_one()) umma_commit(mine);
            __syncwarp();
            attn_wait(mine, 0, flag + 4);
        } else if (role == 0 && lane == 0) {
            // the last fill of each stage: earlier ones were complete before the stage was filled again
            const int n[2] = {copies[0], copies[1]}, end = 2 * max(n[0], n[1]);
            for (int e = max(end - 4 * kStages, 0); e < end; ++e) {
                const int again = e + kStages;
                if ((e >> 1) < ((e & 1) ? n[1] : n[0]) && (again >> 1) >= ((again & 1) ? n[1] : n[0]))
                    attn_wait(full_bar(e % kStages), static_cast<uint32_t>(e / kStages) & 1u, flag + 4);
            }
            for (int i = q_issued > 2 ? q_issued - 2 : 0; i < q_issued; ++i)
                attn_wait(q_full(i & 1), static_cast<uint32_t>((i >> 1) & 1), flag + 4);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (threadIdx.x == 0 && abort_flag[0] != 0) {
        atomicOr(p.err, 1);
        atomicExch(p.err + 1, static_cast<int>(*half_used ^ 1u));                    // (every block that gave up writes the same)
    }
}

}  // namespace wisv
