// Attention of each request's new rows over a paged cache of e4m3 codes, on the 8-bit tensor cores (tcgen05 kind::f8f6f4).
//
// Mathematics.  Keys and values are code * scale, one fp32 scale per token and key head (a for keys, b for values).  Per (request, key
// head) the query heads that share the key head are stacked: column n of a tile is new token n / group, query head n % group.
// With keys as the rows of the matrix products, for 128 keys and up to 64 columns at a time:
//     S = K Q^T,   x = c S a + log2 b - m,   P = exp2(x),   l += P / b,   O^T += V^T P,   out = O / l,
// where K and V are the codes as they lie in the cache and m is a reference of the column.  Taking log2 b into the exponent makes P the
// factor that a code of V is multiplied by, so that its largest value, and not the largest softmax weight, is what m follows: a
// token whose values are tiny (an attention sink) costs the others no precision.
//
// 8-bit operands without a loss.  The codes are operands of the products as they are.  The other operand is cut into e4m3 parts: a number's
// nearest e4m3 number, the nearest to what is left, and so on; each part takes 4 bits and the sign of the rest one more, so two parts carry
// the 8 bits of a bf16 and three the 11 of an fp16 number, above a floor: the last part's half step, 2^-10.  The parts lie side by side as columns,
// [part][column], so that a tile of K or V is read once for all of them, and each further part is scaled up by 16, since its sums are
// kept apart until they are read.  Queries share a power of two that brings the tile's largest element to [128, 256): the floor is 2^-21 of that element.  (Where
// three parts of S do not fit TMEM side by side they are added in one accumulator, unscaled: then every row has its own power of two, and the
// floor is 2^-17 of the row's largest element.)  Of P two parts keep 9 bits (and fp16's 11 on the way), half the error of a bf16 P, and three 14; its
// floor is 2^-14 (three parts: 2^-17) of its largest.  The products are exact, sums are fp32.
//
// References.  m grows only when a column's x passes 8.75 (P must stay below 448, the largest e4m3 number), then to the column's largest (one more
// where there are three parts, whose floor leaves room); l and O are scaled with it.  One vote of a slot's warps per tile says whether any
// column has to, and columns that have doubled follow.  (With 2^2 below the largest instead, half of the tiles of a prompt chunk grew some
// column: 1267 us instead of 1077.)
//
// What does not reach a column.  Masked keys have x = -inf and P = 0 exactly.  V behind the last key of a request is cleared in shared memory,
// since 0 times a code of NaN is NaN.  A scale of NaN (a token with infinite or NaN elements) makes x, and so the columns that see
// the token, NaN.  Values with a scale of 0 (or below 2^-40 of the largest of the tile) count as that small: their l needs a b that can be
// divided by.
//
// Roles.  One block per SM, persistent: a warp that walks the work and copies keys, one that copies values, one that copies scales and
// prepares them, four that issue the MMAs (S and O of each slot), one that at most clears rows of no window, and two sets of eight
// softmax warps ("slots"), a thread per key and half of the columns, which also cut the queries.  A
// work item is "paired" - two tiles of columns of the same (request, key head), one per slot, sharing every tile of keys - or, where one
// tile of columns is left, "split": the slots take the key tiles in turn and are put together at the end.  The line of key tiles, its cut
// over the blocks and the joining of shared items are those of the 16-bit cache (wisv_attn.cuh).
//
// What bounds it.  A tile of 128 keys has 2 * 128 D bytes, some 1400 clocks at a 148th of the measured copy rate (D = 128), and with keys as the
// rows its products take 32 + columns / 4 clocks per 32 of the inner dimension, what their operands take through shared memory: 320 clocks at
// 16 query rows, 1030 at 64.  One row per request is bound by HBM; from some 32 rows on by the instructions of the softmax warps (some 540 for 32 columns
// of a tile, half of them for waits, votes and addresses).
//
// Measured (8B shape: 32 query heads, 8 key heads, D = 128, pools with heads first; short runs): 64 requests of one row over 514 k keys
// 174 us, 6.2 TB/s, 0.95 of the copy rate; of 4, 8, 9 and 16 rows over 270 k keys 101, 111, 130 and 146 us (5.7 to 4.0 TB/s); one
// row over 131 k keys 54 us; one request of 9 rows over 709 keys 14.2 us, of which 3 us are the walk's first lookups, 1.5 the queries and 2 the merge.
#pragma once

#include <stddef.h>

#include "wisv_attn.cuh"

namespace wisv {

constexpr int kA8Cols = 64;                      // columns of a tile
constexpr int kA8Stages = 12;                    // at most, of keys and of values
constexpr int kA8Scales = 6;                     // tiles of scales in flight
constexpr int kA8ScaleBytes = 3 * 4 * kAttnTile; // of a tile: a, log2 b and 1 / b
constexpr int kA8Small = 9 * 1024;               // barriers, queue, tables of columns
constexpr int kA8Slack = 1024;
constexpr int kA8SoftWarps = 16;                 // eight per slot
constexpr int kA8Threads = 256 + 32 * kA8SoftWarps;
// Key tiles that starting and finishing an item is worth.  (With 1, 5, 8, 12: decoding 64 requests over 514 k keys 212, 173, 173, 176 us; windows
// of 5 to 17 rows over 270 k keys -, 175, 167, 171.)
constexpr int kA8ItemCost = 8;
constexpr float kA8Grow = 8.75f;                 // log2 of 430
template <typename E> __host__ __device__ constexpr float a8_room() { return is_bf16<E>::value ? 0.0f : -1.0f; }
constexpr float kA8Step = 16.0f;                 // from one part to the next

struct Attn8Params : AttnParams {
    const void* q; int64_t qt, qh;               // in elements
    const float *ks, *vs;                        // scales: tokens of a page and head side by side
    int64_t ksp, ksh, vsp, vsh;                  // strides of pages and heads, in floats
    int32_t rows;                                // query rows are rows of the products (wisv_attn8r.cuh)
    int32_t k_stages, v_stages;                  // even
    uint32_t q_bytes, p_bytes;                   // of a tile's queries, of a slot's P
};

template <typename E> struct a8_parts { static constexpr int n = is_bf16<E>::value ? 2 : 3; };

// TMEM: 256 columns a slot, O behind S.  O has columns for each part, so that V is read once for all of them and that the parts can have scales of
// their own; S too where that fits.
template <typename E> __host__ __device__ constexpr int a8_o_at() { return 256 - kA8Cols * a8_parts<E>::n; }
template <typename E> __host__ __device__ constexpr bool a8_s_stacked(int cols) { return a8_parts<E>::n * cols <= a8_o_at<E>(); }
// bytes of a slot's P: 64 columns of 128 keys in a piece
template <typename E> __host__ __device__ constexpr int a8_p_bytes(int cols) { return (a8_parts<E>::n * cols + 63) / 64 * 8192; }

// D[tmem] (+)= A[smem] * B[smem], e4m3 operands
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t"
        "}\n"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// kind::f8f6f4, e4m3 operands, fp32 sums; `mn`: both operands MN-major
__device__ __forceinline__ uint32_t a8_idesc(uint32_t M, uint32_t N, bool mn)
{
    return (1u << 4) | (mn ? 3u << 15 : 0u) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
// Descriptor of rows of `row` (128 or 64) bytes with the swizzle of that width; MN-major: `lead` bytes between row-wide pieces
__device__ __forceinline__ uint64_t a8_desc(uint32_t smem_addr, uint32_t row, uint32_t lead)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((smem_addr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>(lead >> 4) << 16;
    d |= static_cast<uint64_t>((8u * row) >> 4) << 32;
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(row == 128 ? 2 : 4) << 61;
    return d;
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* m, int32_t a, int32_t b, int32_t c, int32_t d, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(a), "r"(b), "r"(c), "r"(d)
        : "memory");
}
// 16 bytes, or zeros where `bytes` is 0
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ float warp_max_nan(float x)
{
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
// The e4m3 codes of four numbers (a word, the first in the low byte), and what is left of them, in fp16: 11 bits of the rest, where rounding the numbers
// themselves to fp16 would leave it 7.
__device__ __forceinline__ uint32_t a8_first(float x0, float x1, float x2, float x3, uint32_t& h0, uint32_t& h1)
{
    uint32_t c;
    float r0, r1, r2, r3;
    asm("{\n\t"
        ".reg .b16 e0, e1, b0, b1, b2, b3, one;\n\t"
        ".reg .b32 f0, f1;\n\t"
        "mov.b16 one, 0xbc00;\n\t"                                 // -1
        "cvt.rn.satfinite.e4m3x2.f32 e0, %6, %5;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 e1, %8, %7;\n\t"
        "mov.b32 %0, {e0, e1};\n\t"
        "cvt.rn.f16x2.e4m3x2 f0, e0;\n\t"
        "cvt.rn.f16x2.e4m3x2 f1, e1;\n\t"
        "mov.b32 {b0, b1}, f0;\n\t"
        "mov.b32 {b2, b3}, f1;\n\t"
        "fma.rn.f32.f16 %1, b0, one, %5;\n\t"
        "fma.rn.f32.f16 %2, b1, one, %6;\n\t"
        "fma.rn.f32.f16 %3, b2, one, %7;\n\t"
        "fma.rn.f32.f16 %4, b3, one, %8;\n\t"
        "}"
        : "=r"(c), "=f"(r0), "=f"(r1), "=f"(r2), "=f"(r3) : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h0) : "f"(r1), "f"(r0));
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h1) : "f"(r3), "f"(r2));
    return c;
}
// Four numbers below 448 in NP e4m3 parts each, largest first, each further part 16 times what is left where `kScaled`: a word of four codes,
// the first number in the low byte, for each part
template <int NP, bool kScaled, bool kLong>
__device__ __forceinline__ void a8_cut(float x0, float x1, float x2, float x3, uint32_t (&c)[NP])
{
    uint32_t h0, h1;
    if (kLong) {
        c[0] = a8_first(x0, x1, x2, x3, h0, h1);
        if (kScaled) {
            asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(h0) : "r"(0x4c004c00u));               // 16
            asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(h1) : "r"(0x4c004c00u));
        }
    } else {
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h0) : "f"(x1), "f"(x0));
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h1) : "f"(x3), "f"(x2));
    }
#pragma unroll
    for (int p = kLong ? 1 : 0; p < NP; ++p) {
        if (p + 1 < NP) {
            uint32_t b0, b1;
            asm("{\n\t"
                ".reg .b16 e0, e1;\n\t"
                "cvt.rn.satfinite.e4m3x2.f16x2 e0, %3;\n\t"
                "cvt.rn.satfinite.e4m3x2.f16x2 e1, %4;\n\t"
                "mov.b32 %0, {e0, e1};\n\t"
                "cvt.rn.f16x2.e4m3x2 %1, e0;\n\t"
                "cvt.rn.f16x2.e4m3x2 %2, e1;\n\t"
                "}"
                : "=r"(c[p]), "=r"(b0), "=r"(b1) : "r"(h0), "r"(h1));
            asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(h0) : "r"(b0));
            asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(h1) : "r"(b1));
            if (kScaled) {
                asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(h0) : "r"(0x4c004c00u));           // 16
                asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(h1) : "r"(0x4c004c00u));
            }
        } else {
            asm("{\n\t"
                ".reg .b16 e0, e1;\n\t"
                "cvt.rn.satfinite.e4m3x2.f16x2 e0, %1;\n\t"
                "cvt.rn.satfinite.e4m3x2.f16x2 e1, %2;\n\t"
                "mov.b32 %0, {e0, e1};\n\t"
                "}"
                : "=r"(c[p]) : "r"(h0), "r"(h1));
        }
    }
}

template <typename E> __device__ __forceinline__ void unpack2(uint32_t w, float& lo, float& hi);
template <> __device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t w, float& lo, float& hi)
{
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xffff0000u);
}
template <> __device__ __forceinline__ void unpack2<__half>(uint32_t w, float& lo, float& hi)
{
    lo = __half2float(__ushort_as_half(static_cast<unsigned short>(w & 0xffffu)));
    hi = __half2float(__ushort_as_half(static_cast<unsigned short>(w >> 16)));
}

template <typename E> __device__ __forceinline__ E a8_round(float x);
template <> __device__ __forceinline__ __nv_bfloat16 a8_round<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half a8_round<__half>(float x) { return __float2half_rn(x); }

// Waits and arrivals of whole warps, on a barrier OFF bytes behind `base`.  A wait for a barrier that is complete is a try, a vote and a branch
// that the warp takes as one; an arrival is one predicated instruction.  (As calls of attn_wait they were two fifths of a tile's
// instructions, and their loops, one to each place, a twentieth of the time: 24 warps in eight roles share the caches of instructions.)
// `flag`: see attn_wait.
template <int OFF>
__device__ __forceinline__ bool a8_try(uint32_t base, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1 + %3], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t"
        "}\n"
        : "=r"(ok) : "r"(base), "r"(parity), "n"(OFF) : "memory");
    return __all_sync(0xffffffffu, ok);
}
template <int OFF>
__device__ __forceinline__ bool a8_wait(uint32_t base, uint32_t parity, uint32_t flag)
{
    if (a8_try<OFF>(base, parity)) return true;
    const uint32_t t0 = static_cast<uint32_t>(clock64() >> 10);
#pragma unroll 1
    for (;;) {
        if (a8_try<OFF>(base, parity)) return true;
        uint32_t stop, limit;
        asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(stop) : "r"(flag) : "memory");
        asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(limit) : "r"(flag + 12u) : "memory");
        if (static_cast<uint32_t>(clock64() >> 10) - t0 > limit) {
            asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(flag), "r"(1) : "memory");
            stop = 1;
        }
        if (__any_sync(0xffffffffu, stop)) return false;
    }
}
template <int OFF>
__device__ __forceinline__ void a8_arrive(uint32_t base, int lane)
{
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.eq.s32 p, %1, 0;\n\t"
        "@p mbarrier.arrive.shared::cta.b64 _, [%0 + %2];\n\t"
        "}\n"
        ::"r"(base), "r"(lane), "n"(OFF) : "memory");
}
// A ring of `n` stages (n even), walked one or two entries at a time.  Slots of a split item take the tiles by the parity of their number, so
// the fill before the one that a warp waits for is of a tile that the same warp has seen: a barrier's one phase bit is enough.
struct A8Ring {
    int s = 0;
    uint32_t ph = 0;
    __device__ __forceinline__ void step(int n, int by) { s += by; if (s >= n) { s -= n; ph ^= 1u; } }
    __device__ __forceinline__ void jump(int n, int by)              // any number of entries
    {
        s += by;
        const int turns = s / n;
        s -= turns * n;
        ph ^= static_cast<uint32_t>(turns) & 1u;
    }
};

// Shared memory behind the tiles
struct A8Small {
    uint64_t k_full[kA8Stages], k_empty[kA8Stages], v_full[kA8Stages], v_empty[kA8Stages];
    uint64_t sc_full[kA8Scales], sc_empty[kA8Scales];
    uint64_t q_full[2], s_full[2], s_free[2], p_full[2], pv_done[2], vote[2];                        // slots
    uint64_t seg_full[kSegQueue], seg_empty[kSegQueue];
    uint64_t o_full, o_empty, ml_full, fin_full, part_full, last_full, drain[4];
    uint32_t tmem;
    uint32_t abort[2];                           // [1] is for the waits after a time-out
    uint32_t pad;
    uint32_t limit[2];                           // three words behind either flag
    int32_t came_last;
    uint32_t half;
    alignas(16) int32_t queue[kSegQueue][kSegWords];
    uint32_t grow[2][2];
    uint32_t top[2][2];                          // largest query element of a slot's tile, for even and odd items
    alignas(16) float rs[2][kA8Cols];            // of query columns: c over a column's power of two; with a common one 0, or NaN where the row is
    alignas(16) float m[2][kA8Cols];             // references
    alignas(16) float a[2][kA8Cols];             // factors when they grow; at the end those of a slot's own O
    alignas(16) float b[2][kA8Cols];             // at the end: of the other slot's O
    alignas(16) float mx[2][4][kA8Cols];         // maxima of the warps; at the end their l
    int64_t at[2][kA8Cols];                      // at the end: where a column's output lies
};
static_assert(sizeof(A8Small) <= kA8Small, "shared memory");
static_assert(offsetof(A8Small, limit) - offsetof(A8Small, abort) == 12, "attn_wait");

template <int D> __host__ __device__ constexpr uint32_t a8_tile_bytes() { return kAttnTile * D; }

// The copies of key (or value) tiles t0 .. t1 - 1 of a request into the ring, by one warp (see attn_load_tiles).
template <int D>
__device__ __forceinline__ bool a8_load_tiles(const Attn8Params& p, const CUtensorMap* map, int req, int pg, int t0, int t1, int keys, int head,
                                              uint32_t ring, uint32_t full, uint32_t empty, int stages, uint32_t flag, int lane, A8Ring& rg,
                                              int& issued)
{
    const int box_tok = min(1 << p.page_shift, kAttnTile);
    const uint32_t box_bytes = static_cast<uint32_t>(box_tok) * D;
    for (int t = t0; t < t1; ++t) {
        const int tok0 = t * kAttnTile;
        const int pages = max(min(keys - tok0, kAttnTile) + box_tok - 1, 0) / box_tok;               // that hold keys
        const int at = (tok0 + lane * box_tok) & ((1 << p.page_shift) - 1);
        const int g = pg >= 0 && pg < p.n_pages ? pg : p.n_pages;                                   // out of range: zeros
        pg = attn_page(p, req, t + 1, t1, keys, lane);
        if (!a8_wait<0>(empty + 8u * rg.s, rg.ph ^ 1u, flag)) return false;
        const uint32_t dst = ring + rg.s * a8_tile_bytes<D>(), bar = full + 8u * rg.s;
        if (elect_one()) mbar_expect_tx(bar, static_cast<uint32_t>(pages) * box_bytes);
        __syncwarp();
        for (int i = 0; i < pages; ++i) {
            const int gi = __shfl_sync(0xffffffffu, g, i), ai = __shfl_sync(0xffffffffu, at, i);
            if (elect_one()) tma_load_4d(dst + i * box_bytes, map, 0, ai, head, gi, bar);
        }
        __syncwarp();
        ++issued;
        rg.step(stages, 1);
    }
    return true;
}

// A slot's tile of queries, cut into parts by its eight warps: D / 16 lanes to a row of 16 elements, rows in groups of 32 / (D / 16).  Where the
// parts lie side by side (kCommon) the tile has one power of two, from its largest finite element, and each further part 16 times
// what is left, so that the half step is at most 2^-21 of that element; else every row has its own, and the step is 2^-17 of the row's
// largest.  Returns c over the common power of two.
template <typename E, int D, bool kCommon, typename Vote>
__device__ __forceinline__ bool a8_cut_queries(const Attn8Params& p, A8Small* sm, int slot, uint32_t item, int row0, int head, int rows, int cols, uint32_t dst,
                                               int w, int lane, Vote vote, float& common)
{
    constexpr int NP = a8_parts<E>::n, L = D / 16, R = 32 / L, U = 8 / R;            // U groups a warp: 64 columns by eight warps
    const int c = lane % L;
    uint4 v[U][2];
    uint32_t top[U], most = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int r = (u * 8 + w) * R + lane / L;
        v[u][0] = v[u][1] = make_uint4(0, 0, 0, 0);
        if (r < rows) {
            const int t = attn_token(p, r);
            const uint4* src = reinterpret_cast<const uint4*>(static_cast<const E*>(p.q) + (row0 + t) * p.qt + (head * p.group + r - t * p.group) * p.qh) + 2 * c;
            v[u][0] = src[0];
            v[u][1] = src[1];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t* d = reinterpret_cast<const uint32_t*>(v[u]);
        top[u] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float a, b;
            unpack2<E>(d[i], a, b);
            top[u] = max(top[u], max(__float_as_uint(a) & 0x7fffffffu, __float_as_uint(b) & 0x7fffffffu));
        }
#pragma unroll
        for (int o = 1; o < L; o <<= 1) top[u] = max(top[u], __shfl_xor_sync(0xffffffffu, top[u], o));
        if (top[u] < 0x7f800000u) most = max(most, top[u]);
    }
    if (kCommon) {
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) atomicMax(&sm->top[slot][item & 1u], most);
        if (!vote()) return false;
        most = *const_cast<volatile uint32_t*>(&sm->top[slot][item & 1u]);
        if (w == 0 && lane == 0) *const_cast<volatile uint32_t*>(&sm->top[slot][(item + 1) & 1u]) = 0;
    }
    // (0 and what is below 2^-119 are scaled alike)
    const uint32_t ec = max(most >> 23, 8u);
    common = p.scale_log2 * __uint_as_float((ec - 7u) << 23);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int r = (u * 8 + w) * R + lane / L;
        if ((u * 8 + w) * R >= cols) break;                          // (the warp as one)
        const uint32_t* d = reinterpret_cast<const uint32_t*>(v[u]);
        const bool fine = top[u] < 0x7f800000u;
        const uint32_t e = kCommon ? ec : fine ? max(top[u] >> 23, 8u) : 8u;
        const float up = __uint_as_float((261u - e) << 23);          // largest element to [128, 256)
        uint32_t out[NP][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[4];
            unpack2<E>(d[2 * i], x[0], x[1]);
            unpack2<E>(d[2 * i + 1], x[2], x[3]);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = fine ? x[k] * up : 0.0f;
            uint32_t f[NP];
            a8_cut<NP, kCommon, false>(x[0], x[1], x[2], x[3], f);
#pragma unroll
            for (int q = 0; q < NP; ++q) out[q][i] = f[q];
        }
#pragma unroll
        for (int q = 0; q < NP; ++q) {
            const int row = q * cols + r;
            const uint32_t at = dst + row * D + ((D == 128 ? c ^ (row & 7) : c ^ ((row >> 1) & 3)) << 4);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(out[q][0]), "r"(out[q][1]), "r"(out[q][2]), "r"(out[q][3]) : "memory");
        }
        if (c == 0) sm->rs[slot][r] = kCommon ? (fine ? 0.0f : CUDART_NAN_F) : r >= rows ? 0.0f : fine ? p.scale_log2 * __uint_as_float((e - 7u) << 23) : CUDART_NAN_F;
    }
    return true;
}

constexpr int kA8Tok1 = kSegOdd;                 // in a stretch: tokens of a paired item's first tile

// The merge of an item's partials by the softmax warps of the block that came last: a warp takes a column at a time, its lanes
// the D elements; four partials are loaded together and added in block order.  Reads go past L1, which other blocks'
// writes do not reach.
template <typename E, int D>
__device__ __forceinline__ void a8_merge(const Attn8Params& p, const int* sg, int w, int lane)
{
    constexpr int V = D / 32, U = 4;
    const int parts = __shfl_sync(0xffffffffu, sg[kSegParts], 0);
    const int rows0 = __shfl_sync(0xffffffffu, sg[kSegRows0], 0), rows = rows0 + __shfl_sync(0xffffffffu, sg[kSegRows1], 0);
    const int first = sg[kSegFirst];
    for (int r = w; r < rows; r += kA8SoftWarps) {
        const bool second = r >= rows0;
        const int in = second ? r - rows0 : r, at = in + (second ? kA8Cols : 0);
        float m = -CUDART_INF_F, l = 0.0f, acc[V];
#pragma unroll
        for (int c = 0; c < V; ++c) acc[c] = 0.0f;
        for (int j0 = 0; j0 < parts; j0 += U) {
            float2 x[U];
            float v[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = min(j0 + u, parts - 1), buf = j == 0 ? 2 * first + 1 : 2 * (first + j);
                x[u] = __ldcg(p.part_ml + buf * (2 * kA8Cols) + at);
                const float* src = p.part_o + (static_cast<size_t>(buf) * (2 * kA8Cols) + at) * D + lane * V;
                if (V == 4) {
                    const float4 q = __ldcg(reinterpret_cast<const float4*>(src));
                    v[u][0] = q.x; v[u][1] = q.y; v[u][V - 2] = q.z; v[u][V - 1] = q.w;
                } else {
                    const float2 q = __ldcg(reinterpret_cast<const float2*>(src));
                    v[u][0] = q.x; v[u][1] = q.y;
                }
                if (j0 + u >= parts) x[u] = make_float2(-CUDART_INF_F, 0.0f);
            }
            float mm = m;
#pragma unroll
            for (int u = 0; u < U; ++u) mm = fmaxf(mm, x[u].x);
            const float f0 = m == -CUDART_INF_F ? 0.0f : attn_ex2(m - mm);
            l *= f0;
#pragma unroll
            for (int c = 0; c < V; ++c) acc[c] *= f0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool some = x[u].x != -CUDART_INF_F;           // (else its outputs may be anything)
                const float f = some ? attn_ex2(x[u].x - mm) : 0.0f;
                l = fmaf(f, x[u].y, l);
#pragma unroll
                for (int c = 0; c < V; ++c) acc[c] = some ? fmaf(f, v[u][c], acc[c]) : acc[c];
            }
            m = mm;
        }
        const float inv = l == 0.0f ? 0.0f : attn_rcp(l);
        const int t = attn_token(p, in), tok = sg[kSegRow] + t + (second ? sg[kA8Tok1] : 0), head = sg[kSegHead] * p.group + in - t * p.group;
        E* const dst = static_cast<E*>(p.out) + tok * p.ot + head * p.oh + lane * V;
        if (V == 4)
            *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<E>(acc[0] * inv, acc[1] * inv), pack2<E>(acc[V - 2] * inv, acc[V - 1] * inv));
        else
            *reinterpret_cast<uint32_t*>(dst) = pack2<E>(acc[0] * inv, acc[1] * inv);
        if (p.lse && lane == 0)
            p.lse[static_cast<int64_t>(tok) * (p.n_kv * p.group) + head] = l == 0.0f ? -CUDART_INF_F : (m + attn_lg2(l)) * 0.6931471805599453f;
    }
}

// Columns that tiles of up to so many rows are computed with, all tiles of a call alike.  (Sixteen warps that change from one width's instructions to
// another's fetch them anew: windows of 8 or of 9 rows of 4 heads 121 and 141 us, mixed with a width for each 163, with one 141.)
__host__ __device__ __forceinline__ int a8_cols(int rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 48 ? 48 : kA8Cols; }

constexpr float kA8None = -3.402823466e38f;      // the reference of a column that has seen no key

// ---- the work: as in the 16-bit kernel, with tiles of paired items weighing two units, since their two slots have a product each.  Where
// rows are columns a paired item's tokens are halved, so that neither tile has columns to spare.
__device__ __forceinline__ int a8_weight(const Attn8Params& p, const AttnReq& r, int it) { return r.n - it * 2 * p.tpt > p.tpt ? 2 : 1; }
__device__ __forceinline__ unsigned a8_units(const Attn8Params& p, const AttnReq& r, int it)
{
    return a8_weight(p, r, it) * attn_tiles(p, r, it) + kA8ItemCost;
}

struct A8Walk {
    int b, kvh, it, pos, units;                  // position on the line of units, and what is left of the range
    AttnReq r;
    // The next stretch; false at the end of the range.  A tile belongs to the range that its first unit lies in.
    __device__ __forceinline__ bool next(const Attn8Params& p, int (&s)[kSegWords + 1])
    {
        while (units > 0) {
            if (it >= r.items) {                 // (a request without rows)
                if (++b >= p.B) return false;
                kvh = it = pos = 0;
                r = attn_request(p, b);
                continue;
            }
            const int nt = attn_tiles(p, r, it), wt = a8_weight(p, r, it), all = wt * nt + kA8ItemCost;
            const int take = min(units, all - pos);
            const int t0 = min(nt, (pos + wt - 1) / wt), t1 = min(nt, (pos + take + wt - 1) / wt);
            if (t1 > t0) {
                const int tok0 = it * 2 * p.tpt, here = min(r.n - tok0, 2 * p.tpt), tok1 = wt != 2 ? here : p.rows ? p.tpt : (here + 1) / 2;
                s[kSegJobs] = t1 - t0;
                s[kSegPaired] = wt == 2; s[kSegT0] = t0; s[kSegT1] = t1; s[kSegTiles] = nt;
                s[kSegKeys] = r.kv; s[kSegLimit] = r.kv - r.n + tok0;
                s[kSegRow] = r.q0 + tok0; s[kSegHead] = kvh; s[kSegReq] = b;
                s[kSegLeft] = units + pos;       // (from the item's first unit to the end of the range)
                s[kSegRows0] = tok1 * p.group;
                s[kSegRows1] = (here - tok1) * p.group;
                s[kA8Tok1] = tok1;
            }
            units -= take;
            pos += take;
            if (pos == all) {
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

// This block's range of the line of units, found by one warp (see attn_range).
__device__ __forceinline__ void a8_range(const Attn8Params& p, unsigned me, int lane, A8Walk& w, unsigned& share, unsigned& more)
{
    const int per = (p.B + 31) >> 5, b0 = min(lane * per, p.B), b1 = min(b0 + per, p.B);
    auto units_of = [&](const AttnReq& r) {
        unsigned u = 0;
        for (int i = 0; i < r.items; ++i) u += a8_units(p, r, i);
        return u;
    };
    unsigned long long sum = 0;
#pragma unroll 4
    for (int b = b0; b < b1; ++b) sum += static_cast<unsigned long long>(units_of(attn_request(p, b))) * p.n_kv;
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
                const unsigned u = a8_units(p, r, it);
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

// The scales of key tiles t0 .. t1 - 1 into their ring, by one warp, four tokens to a lane: copied four tiles ahead, then turned in place into
// a, log2 b and 1 / b.  A lane works on what it has copied itself.
template <typename Small>
__device__ __forceinline__ bool a8_scales(const Attn8Params& p, int req, int head, int t0, int t1, int keys, uint32_t ring, Small* sm, uint32_t flag,
                                          int lane, A8Ring& at, A8Ring& done)
{
    constexpr int kAhead = 4;
    const int mask = (1 << p.page_shift) - 1;
    auto page = [&](int t) {
        const int tok = t * kAttnTile + 4 * lane;
        return t < t1 && tok < keys ? p.block_table[req * p.table_stride + (tok >> p.page_shift)] : -1;
    };
    int pg = page(t0);
    for (int t = t0; t < t1 + kAhead; ++t) {
        if (t < t1) {
            const bool in = pg >= 0 && pg < p.n_pages;
            const int o = in ? (t * kAttnTile + 4 * lane) & mask : 0, from = in ? pg : 0;
            pg = page(t + 1);
            if (!a8_wait<0>(smem_u32(&sm->sc_empty[at.s]), at.ph ^ 1u, flag)) return false;
            const uint32_t dst = ring + at.s * kA8ScaleBytes + lane * 16;
            cp_async16(dst, p.ks + from * p.ksp + head * p.ksh + o, in ? 16 : 0);
            cp_async16(dst + 512, p.vs + from * p.vsp + head * p.vsh + o, in ? 16 : 0);
            at.step(kA8Scales, 1);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (t < t0 + kAhead) continue;
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
        const uint32_t src = ring + done.s * kA8ScaleBytes + lane * 16;
        float a[4], b[4], lb[4];
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(a[0]), "=f"(a[1]), "=f"(a[2]), "=f"(a[3]) : "r"(src) : "memory");
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(b[0]), "=f"(b[1]), "=f"(b[2]), "=f"(b[3]) : "r"(src + 512) : "memory");
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if ((t - kAhead) * kAttnTile + 4 * lane + i >= keys) a[i] = b[i] = 0.0f;                // (behind the last key: anything)
            if (b[i] > 0.0f && b[i] < CUDART_INF_F) top = max(top, __float_as_uint(b[i]));
        }
        const float least = fmaxf(__uint_as_float(__reduce_max_sync(0xffffffffu, top)) * 9.094947e-13f, 7.888609e-31f);          // 2^-40 of the largest, 2^-100
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float be = fmaxf(b[i], least);
            lb[i] = b[i] >= 0.0f ? attn_lg2(be) : CUDART_NAN_F;
            b[i] = attn_rcp(be);
        }
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(src), "f"(a[0]), "f"(a[1]), "f"(a[2]), "f"(a[3]) : "memory");
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(src + 512), "f"(lb[0]), "f"(lb[1]), "f"(lb[2]), "f"(lb[3]) : "memory");
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(src + 1024), "f"(b[0]), "f"(b[1]), "f"(b[2]), "f"(b[3]) : "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm->sc_full[done.s]));
        done.step(kA8Scales, 1);
    }
    return true;
}

#define A8_AT(member) static_cast<int>(offsetof(A8Small, member))

// What a softmax warp carries from stretch to stretch
struct A8Soft {
    int slot, half, quad, lane, row;             // half: of the columns; row: of the tile of keys
    uint32_t lane_off, tmem, q_smem, p_smem, ring_v, ring_sc, flag;
    uint32_t small, bars;                        // A8Small, and its barriers of this slot
    uint32_t jobs = 0, votes = 0;                // of this slot so far
    uint32_t tiles = 0;                          // of the block so far
    A8Ring v, sc;                                // the place of tile number `tiles`
};

// 8 or 16 columns of TMEM, and 8 or 16 bytes of an operand
template <int W> __device__ __forceinline__ void a8_tmem_ld(uint32_t at, uint32_t (&r)[W]);
template <> __device__ __forceinline__ void a8_tmem_ld<8>(uint32_t at, uint32_t (&r)[8]) { tmem_ld8(at, r); }
template <> __device__ __forceinline__ void a8_tmem_ld<16>(uint32_t at, uint32_t (&r)[16]) { tmem_ld16(at, r); }

// A stretch of an item's tiles with 2 C columns, up to and including its outputs or partials.  false: a wait ran out.
template <typename E, int D, int C>
__device__ __forceinline__ bool a8_stretch(const Attn8Params& p, A8Small* sm, A8Soft& w, const int* sg, uint32_t item)
{
    constexpr int NP = a8_parts<E>::n, N = 2 * C, W = C % 16 ? 8 : 16;               // W: columns at a time
    constexpr bool kCommon = a8_s_stacked<E>(N);                     // S has columns for each part, and the queries one power of two
    constexpr int kSParts = kCommon ? NP : 1;
    const int slot = w.slot, col0 = w.half * C, ts = w.half * 128 + w.row;
    const bool paired = sg[kSegPaired];
    const int nt = sg[kSegT1] - sg[kSegT0], keys = sg[kSegKeys];
    const int limit = sg[kSegLimit] + (paired && slot ? sg[kA8Tok1] : 0);  // last key that the tile's first token sees
    const int rows = paired && slot ? sg[kSegRows1] : sg[kSegRows0];
    const int tok0 = sg[kSegRow] + (paired && slot ? sg[kA8Tok1] : 0);
    const uint32_t aS = w.tmem + static_cast<uint32_t>(slot) * 256 + w.lane_off, aO = aS + a8_o_at<E>();
    const float* const rs = sm->rs[slot] + col0;
    float* const m = sm->m[slot];
    auto vote = [&]() {                                              // the slot's warps meet
        __syncwarp();
        a8_arrive<A8_AT(vote)>(w.bars, w.lane);
        const bool ok = a8_wait<A8_AT(vote)>(w.bars, w.votes & 1u, w.flag);
        ++w.votes;
        return ok;
    };
    // ---- queries (the products that read the last ones are complete: their S has been waited for)
    float common;
    if (!a8_cut_queries<E, D, kCommon>(p, sm, slot, item, tok0, sg[kSegHead], rows, N, w.q_smem, w.half * 4 + w.quad, w.lane, vote, common)) return false;
    fence_proxy_async();
    __syncwarp();
    a8_arrive<A8_AT(q_full)>(w.bars, w.lane);
    if (ts < N) m[ts] = kA8None;
    if (!vote()) return false;
    uint64_t l[C / 2];
#pragma unroll
    for (int i = 0; i < C / 2; ++i) l[i] = 0;

    const int i0 = paired ? 0 : static_cast<int>((w.tiles ^ static_cast<uint32_t>(slot)) & 1u), step = paired ? 1 : 2;
    A8Ring rv = w.v, rsc = w.sc;
    if (i0) { rv.step(p.v_stages, 1); rsc.step(kA8Scales, 1); }
    for (int i = i0; i < nt; i += step) {
        const int key0 = (sg[kSegT0] + i) * kAttnTile, key = key0 + w.row;
        // ---- the scales of this thread's key
        if (!a8_wait<A8_AT(sc_full)>(w.small + 8 * rsc.s, rsc.ph, w.flag)) return false;
        float ka, lb, rb;
        {
            const uint32_t at = w.ring_sc + rsc.s * kA8ScaleBytes + w.row * 4;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(ka) : "r"(at) : "memory");
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(lb) : "r"(at + 512) : "memory");
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(rb) : "r"(at + 1024) : "memory");
        }
        if (kCommon) {
            ka *= common;
            if (ka > 3.402823466e38f) ka = 3.402823466e38f;          // (times a column of zeros it must stay 0)
        }
        const uint64_t ka2 = pair(ka, ka), lb2 = pair(lb, lb);
        const bool masked = key0 + kAttnTile - 1 > limit;
        if (!a8_wait<A8_AT(s_full)>(w.bars, w.jobs & 1u, w.flag)) return false;
        tc_fence_after();
        float x[C];
        // Pass 0 finds x with the references as they are; where a column outgrows its own, pass 1 finds x + m for its maximum and pass 2 x
        // with the new references.  (The first tile of a stretch has none yet.)
        for (int pass = i == i0 ? 1 : 0; ; ++pass) {
            const float neg = pass == 1 ? 0.0f : -1.0f;
            const uint64_t neg2 = pair(neg, neg);
#pragma unroll
            for (int c = 0; c < C; c += W) {
                uint32_t s[kSParts][W];
#pragma unroll
                for (int q = 0; q < kSParts; ++q) a8_tmem_ld<W>(aS + q * N + col0 + c, s[q]);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < W; j += 4) {
                    const float4 m4 = *reinterpret_cast<const float4*>(m + col0 + c + j);
                    float4 r4 = make_float4(1.0f, 1.0f, 1.0f, 1.0f);
                    if (!kCommon) r4 = *reinterpret_cast<const float4*>(rs + c + j);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int k = j + 2 * h;
                        uint64_t v = pair(__uint_as_float(s[kSParts - 1][k]), __uint_as_float(s[kSParts - 1][k + 1]));
#pragma unroll
                        for (int q = kSParts - 2; q >= 0; --q)
                            v = fma2(v, pair(1.0f / kA8Step, 1.0f / kA8Step), pair(__uint_as_float(s[q][k]), __uint_as_float(s[q][k + 1])));
                        if (!kCommon) v = mul2(v, h ? pair(r4.z, r4.w) : pair(r4.x, r4.y));
                        v = fma2(v, ka2, fma2(h ? pair(m4.z, m4.w) : pair(m4.x, m4.y), neg2, lb2));
                        x[c + k] = low(v);
                        x[c + k + 1] = high(v);
                    }
                }
            }
            if (masked) {
                // columns from `vis` on see this key
                const int vis = (key >= keys ? 1 << 20 : min(max(key - limit, 0), kA8Cols + 1) * p.group) - col0;
#pragma unroll
                for (int n = 0; n < C; ++n) x[n] = n >= vis ? x[n] : -CUDART_INF_F;
            }
            if (pass == 2) break;
            if (pass == 0) {
                float worst[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                for (int n = 0; n < C; n += 4) {
                    worst[0] = max3_nan(worst[0], x[n], x[n + 1]);
                    worst[1] = max3_nan(worst[1], x[n + 2], x[n + 3]);
                }
                // (whoever has such a column writes the number of the vote: two places in turn, and nothing to clear)
                volatile uint32_t* const grow = &sm->grow[slot][w.votes & 1u];
                const uint32_t number = w.votes;
                if (!(worst[0] <= kA8Grow && worst[1] <= kA8Grow)) *grow = number;
                if (!vote()) return false;
                if (__all_sync(0xffffffffu, *grow != number)) break;
                continue;
            }
            // ---- the references grow
#pragma unroll
            for (int n = 0; n < C; ++n) sm->mx[slot][w.quad][col0 + n] = warp_max_nan(x[n]);
            if (!vote()) return false;
            if (ts < N) {
                const float (&mx)[4][kA8Cols] = sm->mx[slot];
                const float big = max3_nan(max3_nan(mx[0][ts], mx[1][ts], mx[2][ts]), mx[3][ts], mx[3][ts]);
                const float old = m[ts];
                // (once any column has to, those that have doubled follow)
                const bool grows = !(big - old <= a8_room<E>() + 1.0f), bad = !(big < CUDART_INF_F);             // (a score of NaN or +inf)
                const float now = !grows ? old : !bad ? big - a8_room<E>() : old == kA8None ? 0.0f : old;
                sm->a[slot][ts] = !grows ? 1.0f : bad ? CUDART_NAN_F : attn_ex2(old - now);
                m[ts] = now;
            }
            if (!vote()) return false;
            const float* const a = sm->a[slot];
            if (i != i0) {
                if (!a8_wait<A8_AT(pv_done)>(w.bars, (w.jobs - 1) & 1u, w.flag)) return false;
                tc_fence_after();
#pragma unroll
                for (int q = 0; q < NP; ++q) {
#pragma unroll
                    for (int c = 0; c < C; c += 8) {
                        uint32_t o[8];
                        tmem_ld8(aO + q * N + col0 + c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * a[col0 + c + j]);
                        tmem_st8(aO + q * N + col0 + c, o);
                    }
                }
                tmem_wait_st();
            }
#pragma unroll
            for (int n = 0; n < C; n += 2) l[n / 2] = mul2(l[n / 2], pair(a[col0 + n], a[col0 + n + 1]));
        }
        tc_fence_before();
        __syncwarp();
        a8_arrive<A8_AT(s_free)>(w.bars, w.lane);
        a8_arrive<A8_AT(sc_empty)>(w.small + 8 * rsc.s, w.lane);
        if (!paired) a8_arrive<A8_AT(sc_empty)>(w.small + 8 * rsc.s, w.lane);
        rsc.step(kA8Scales, step);

        // ---- P, once the product before has read the last one
        if (w.jobs) {
            if (!a8_wait<A8_AT(pv_done)>(w.bars, (w.jobs - 1) & 1u, w.flag)) return false;
        }
        if (key0 + kAttnTile > keys) {
            // (both slots of a paired item clear: whoever comes second writes zeros over zeros)
            if (!a8_wait<A8_AT(v_full)>(w.small + 8 * rv.s, rv.ph, w.flag)) return false;
            if (key >= keys) {
                const uint32_t at = w.ring_v + rv.s * a8_tile_bytes<D>() + w.row * D + w.half * (D / 2);
#pragma unroll
                for (int c = 0; c < D / 2; c += 16) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + c), "r"(0) : "memory");
            }
        }
        rv.step(p.v_stages, step);
        const uint64_t rb2 = pair(rb, rb);
        const uint32_t p_row = w.p_smem ^ (C % 16 ? 0 : col0);
#pragma unroll
        for (int c = 0; c < C; c += W) {
            uint32_t out[NP][W / 4];
#pragma unroll
            for (int j = 0; j < W / 4; ++j) {
                const int n = c + 4 * j;
                uint64_t y[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = n + 2 * h;
                    y[h] = pair(attn_ex2(x[k]), attn_ex2(x[k + 1]));
                    l[k / 2] = fma2(y[h], rb2, l[k / 2]);
                }
                uint32_t e[NP];
                a8_cut<NP, true, NP == 3>(low(y[0]), high(y[0]), low(y[1]), high(y[1]), e);
#pragma unroll
                for (int q = 0; q < NP; ++q) out[q][j] = e[q];
            }
#pragma unroll
            for (int q = 0; q < NP; ++q) {
                // column n of the operand, in rows of 64 bytes, swizzled.  (w.p_smem is the row's place with the swizzle of piece 0; where
                // a half's columns make whole pieces, its own bits do not carry into the others'.)
                const int n = q * N + c + (C % 16 ? col0 : 0);
                const uint32_t at = ((C % 16 ? w.p_smem : p_row) ^ (((n >> 4) & 3) << 4)) + (n >> 6) * 8192 + (n & 8);
                if (W == 16)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(out[q][0]), "r"(out[q][1]), "r"(out[q][W / 4 - 2]), "r"(out[q][W / 4 - 1]) : "memory");
                else
                    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(out[q][0]), "r"(out[q][1]) : "memory");
            }
        }
        fence_proxy_async();
        tc_fence_before();
        __syncwarp();
        a8_arrive<A8_AT(p_full)>(w.bars, w.lane);
        ++w.jobs;
    }

    // ---- sums over the keys: lanes first (a lane, or several, end with one column), then warps, then slots
    {
        float v[C];
#pragma unroll
        for (int i = 0; i < C / 2; ++i) { v[2 * i] = low(l[i]); v[2 * i + 1] = high(l[i]); }
        // halve the columns that a lane keeps while they are even in number; what is left (1, or 3 of 24) is added over the other lanes
        int len = C;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            if (len % 2 == 0) {
                len >>= 1;
                const bool up = (w.lane & o) != 0;
#pragma unroll
                for (int i = 0; i < C / 2; ++i) {
                    if (i < len) {
                        const float keep = up ? v[i + len] : v[i], send = up ? v[i] : v[i + len];
                        v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    if (i < len) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
                }
            }
        }
        constexpr int kLeft = C == 24 ? 3 : 1, kLanes = 32 * kLeft / C;              // columns a lane ends with, lanes that share them
        if (w.lane % kLanes == 0) {
#pragma unroll
            for (int i = 0; i < kLeft; ++i) sm->mx[slot][w.quad][col0 + w.lane / kLanes * kLeft + i] = v[i];
        }
    }
    __syncwarp();
    a8_arrive<A8_AT(ml_full)>(w.small, w.lane);
    if (!a8_wait<A8_AT(ml_full)>(w.small, item & 1u, w.flag)) return false;
    const bool first = sg[kSegT0] == 0, whole = first && sg[kSegT1] == sg[kSegTiles];
    const int part = static_cast<int>(blockIdx.x) * 2 + (first ? 1 : 0), part_row = paired ? slot * kA8Cols : 0;
    if (ts < N) {
        auto sum = [&](int s) { return (sm->mx[s][0][ts] + sm->mx[s][1][ts]) + (sm->mx[s][2][ts] + sm->mx[s][3][ts]); };
        float mm = m[ts], ll = sum(slot), wa = 1.0f, wb = 0.0f;
        if (!paired) {
            const float other = sm->m[slot ^ 1][ts], top = fmaxf(mm, other);
            wa = mm == kA8None ? 0.0f : attn_ex2(mm - top);
            wb = other == kA8None ? 0.0f : attn_ex2(other - top);
            ll = ll * wa + sum(slot ^ 1) * wb;
            mm = top;
        }
        if (mm == kA8None) { mm = -CUDART_INF_F; wa = 0.0f; }
        else if (kCommon) ll += sm->rs[slot][ts];
        if (whole) {
            const float inv = ll == 0.0f ? 0.0f : attn_rcp(ll);
            wa *= inv;
            wb *= inv;
        }
        sm->a[slot][ts] = wa;
        sm->b[slot][ts] = wb;
        const int t = attn_token(p, ts), head = sg[kSegHead] * p.group + ts - t * p.group;
        sm->at[slot][ts] = (tok0 + t) * p.ot + head * p.oh;
        if (ts < rows && (paired || slot == 0)) {
            if (!whole) p.part_ml[part * (2 * kA8Cols) + part_row + ts] = make_float2(mm, ll);
            else if (p.lse)
                p.lse[static_cast<int64_t>(tok0 + t) * (p.n_kv * p.group) + head] = ll == 0.0f ? -CUDART_INF_F : (mm + attn_lg2(ll)) * 0.6931471805599453f;
        }
    }
    __syncwarp();
    a8_arrive<A8_AT(fin_full)>(w.small, w.lane);
    if (!a8_wait<A8_AT(fin_full)>(w.small, item & 1u, w.flag)) return false;
    if (!a8_wait<A8_AT(o_full)>(w.small, item & 1u, w.flag)) return false;
    tc_fence_after();

    // ---- outputs: a thread has one element of every column; split: each slot does half of the columns, from both accumulators
    const int d = D == 128 ? w.row : w.quad * 16 + w.lane;
    const bool has = D == 128 || w.lane < 16;
    const uint32_t other = slot ? aO - 256 : aO + 256;
    // chunks of 8 columns, dealt out to the warps that share the lanes: two in a paired item, the four of both slots in a split one
    for (int c = 8 * (paired ? w.half : 2 * slot + w.half); c < rows; c += paired ? 16 : 32) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = 0.0f;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            if (side && paired) break;
            uint32_t o[NP][8];
#pragma unroll
            for (int q = 0; q < NP; ++q) tmem_ld8((side ? other : aO) + q * N + c, o[q]);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = side ? sm->b[slot][c + j] : sm->a[slot][c + j];
                float v = __uint_as_float(o[NP - 1][j]);
#pragma unroll
                for (int q = NP - 2; q >= 0; --q) v = fmaf(v, 1.0f / kA8Step, __uint_as_float(o[q][j]));
                if (f != 0.0f) y[j] = fmaf(v, f, y[j]);              // (an accumulator without a job may hold anything)
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (c + j >= rows || !has) continue;
            if (whole) static_cast<E*>(p.out)[sm->at[slot][c + j] + d] = a8_round<E>(y[j]);
            else p.part_o[(static_cast<size_t>(part) * (2 * kA8Cols) + part_row + c + j) * D + d] = y[j];
        }
    }
    w.tiles += static_cast<uint32_t>(nt);
    w.v.jump(p.v_stages, nt);
    w.sc.jump(kA8Scales, nt);
    return true;
}

template <typename E, int D, int N>
__global__ void __launch_bounds__(kA8Threads, 1)
attn8_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const Attn8Params p)
{
    constexpr int NP = a8_parts<E>::n;
    constexpr uint32_t kTile = a8_tile_bytes<D>();

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;
    const uint32_t q_buf = raw_addr + pad, p_buf = q_buf + 2 * p.q_bytes, ring_k = p_buf + 2 * p.p_bytes;
    const uint32_t ring_v = ring_k + p.k_stages * kTile, ring_sc = ring_v + p.v_stages * kTile;
    const uint32_t small_off = ring_sc + kA8Scales * kA8ScaleBytes - raw_addr;
    A8Small* const sm = reinterpret_cast<A8Small*>(smem_raw + small_off);
    auto bar = [](const uint64_t& b) { return smem_u32(&b); };
    const unsigned me = blockIdx.x;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int lane = threadIdx.x & 31;

    if (small_off + kA8Small > static_cast<uint32_t>(kAttnSmem)) {            // (dynamic shared memory starts 1024-byte aligned)
        if (threadIdx.x == 0) atomicOr(p.err, 2);
        return;
    }
    const uint32_t flag = smem_u32(&sm->abort[0]);
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.k_stages; ++s) { mbar_init(bar(sm->k_full[s]), 1); mbar_init(bar(sm->k_empty[s]), 2); }
        for (int s = 0; s < p.v_stages; ++s) { mbar_init(bar(sm->v_full[s]), 1); mbar_init(bar(sm->v_empty[s]), 2); }
        for (int s = 0; s < kA8Scales; ++s) { mbar_init(bar(sm->sc_full[s]), 1); mbar_init(bar(sm->sc_empty[s]), kA8SoftWarps); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(sm->q_full[s]), 8);
            mbar_init(bar(sm->s_full[s]), 1); mbar_init(bar(sm->s_free[s]), 8);
            mbar_init(bar(sm->p_full[s]), 8); mbar_init(bar(sm->pv_done[s]), 1);
            mbar_init(bar(sm->vote[s]), 8);
        }
        for (int s = 0; s < kSegQueue; ++s) { mbar_init(bar(sm->seg_full[s]), 1); mbar_init(bar(sm->seg_empty[s]), 6 + kA8SoftWarps); }
        mbar_init(bar(sm->o_full), 2); mbar_init(bar(sm->o_empty), kA8SoftWarps); mbar_init(bar(sm->ml_full), kA8SoftWarps);
        mbar_init(bar(sm->fin_full), kA8SoftWarps); mbar_init(bar(sm->part_full), kA8SoftWarps); mbar_init(bar(sm->last_full), 1);
        for (int s = 0; s < 4; ++s) mbar_init(bar(sm->drain[s]), 1);
        sm->abort[0] = 0; sm->abort[1] = 0;
        sm->top[0][0] = sm->top[0][1] = sm->top[1][0] = sm->top[1][1] = 0;
        sm->grow[0][0] = sm->grow[0][1] = sm->grow[1][0] = sm->grow[1][1] = 0xffffffffu;
        sm->limit[0] = sm->limit[1] = p.wait_limit;
        fence_barrier_init();
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmV);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&sm->tmem), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    griddep_wait();                              // lengths, tables and the cache itself come from kernels before this one
    griddep_launch_dependents();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sm->tmem, 0);
    int issued = 0;                              // tiles copied (copying warps; read again before the end)

    // warps 0: rows of no window; 1: the walk and keys; 2, 3: S of the slots; 4: scales; 5, 6: O of the slots; 7: values.  (The block starts with
    // 80 registers a thread: 8 warps at 32 and 16 at 104 take the same.)
    if (warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
        if (warp == 0) {
            if (lane == 0) {
                const unsigned half = static_cast<unsigned>(__ldcg(p.err + 1)) & 1u;
                sm->half = half;
                const unsigned other = 0xffffu << (16u * (half ^ 1u));
                if (static_cast<unsigned>(__ldcg(p.count + me)) & other) atomicAnd(p.count + me, static_cast<int>(~other));
            }
            __syncwarp();
            attn_clear_rows<E, D>(p, static_cast<int>(me), static_cast<int>(gridDim.x), lane);
        } else if (warp == 1) {
            const int half = __ldcg(p.err + 1) & 1;
            A8Walk walk;
            unsigned share, more;
            a8_range(p, me, lane, walk, share, more);
            int s[kSegWords + 1];
            A8Ring rg;
            bool ok = true;
            for (int item = 0; ok; ++item) {
                const bool some = walk.next(p, s);
                const int qi = item & (kSegQueue - 1);
                if (some) {
                    s[kSegFirst] = static_cast<int>(me); s[kSegParts] = 1; s[kSegShift] = 16 * half;
                    if (s[kSegT0] > 0 || s[kSegT1] < s[kSegTiles]) {                 // shared: whose ranges does the item reach?
                        auto block_of = [&](unsigned u) {
                            return u < more * (share + 1) ? u / (share + 1) : more + (u - more * (share + 1)) / share;
                        };
                        const unsigned unit0 = (me + 1) * share + min(me + 1, more) - s[kSegLeft];
                        const unsigned first = block_of(unit0), last = block_of(unit0 + (s[kSegTiles] - 1) * (s[kSegPaired] ? 2 : 1));
                        s[kSegFirst] = first; s[kSegParts] = last - first + 1;
                    }
                }
                ok = a8_wait<0>(bar(sm->seg_empty[qi]), (static_cast<uint32_t>(item / kSegQueue) & 1u) ^ 1u, flag);
                if (!ok) break;
                if (lane == 0) {
#pragma unroll
                    for (int i = 0; i < kSegWords; ++i) sm->queue[qi][i] = some ? s[i] : 0;
                    mbar_arrive(bar(sm->seg_full[qi]));
                }
                __syncwarp();
                if (!some) break;
                ok = a8_load_tiles<D>(p, &tmK, s[kSegReq], attn_page(p, s[kSegReq], s[kSegT0], s[kSegT1], s[kSegKeys], lane), s[kSegT0], s[kSegT1],
                                      s[kSegKeys], s[kSegHead], ring_k, bar(sm->k_full[0]), bar(sm->k_empty[0]), p.k_stages, flag, lane, rg, issued);
            }
        } else {
            const int slot = warp == 3 || warp == 6 ? 1 : 0;
            A8Ring rg, done;
            uint32_t tiles = 0, jobs = 0;        // of the block, of the slot
            bool ok = warp != 7 || static_cast<int>(me) != p.stalled;
            for (int item = 0; ok; ++item) {
                const int qi = item & (kSegQueue - 1);
                ok = a8_wait<0>(bar(sm->seg_full[qi]), static_cast<uint32_t>(item / kSegQueue) & 1u, flag);
                if (!ok) break;
                const int* const sg = sm->queue[qi];
                if (__shfl_sync(0xffffffffu, sg[kSegJobs], 0) == 0) break;           // (the compiler then knows it uniform)
                const bool paired = __shfl_sync(0xffffffffu, sg[kSegPaired], 0) != 0;
                const int t0 = __shfl_sync(0xffffffffu, sg[kSegT0], 0), t1 = __shfl_sync(0xffffffffu, sg[kSegT1], 0), nt = t1 - t0;
                if (warp == 7) {
                    // ------------------------------------------------ values
                    ok = a8_load_tiles<D>(p, &tmV, sg[kSegReq], attn_page(p, sg[kSegReq], t0, t1, sg[kSegKeys], lane), t0, t1, sg[kSegKeys], sg[kSegHead],
                                          ring_v, bar(sm->v_full[0]), bar(sm->v_empty[0]), p.v_stages, flag, lane, rg, issued);
                } else if (warp == 4) {
                    ok = a8_scales(p, sg[kSegReq], sg[kSegHead], t0, t1, sg[kSegKeys], ring_sc, sm, flag, lane, rg, done);
                } else {
                    // ------------------------------------------------ MMA: a warp per slot and product
                    const bool second = warp > 4;
                    const int stages = second ? p.v_stages : p.k_stages;
                    constexpr int kSParts = a8_s_stacked<E>(N) ? 1 : NP;             // products of S
                    const uint32_t sS = tmem + slot * 256, sO = sS + a8_o_at<E>();
                    const uint32_t idesc = second ? a8_idesc(D, NP * N, true) : a8_idesc(kAttnTile, kSParts == 1 ? NP * N : N, false);
                    ok = second ? item == 0 || a8_wait<0>(bar(sm->o_empty), static_cast<uint32_t>(item - 1) & 1u, flag)      // the previous O has been read
                                : a8_wait<0>(bar(sm->q_full[slot]), static_cast<uint32_t>(item) & 1u, flag);
                    const int i0 = paired ? 0 : static_cast<int>((tiles ^ static_cast<uint32_t>(slot)) & 1u), step = paired ? 1 : 2;
                    A8Ring r = rg;
                    if (i0) r.step(stages, 1);
                    for (int i = i0; ok && i < nt; i += step, ++jobs) {
                        if (!second) {
                            ok = a8_wait<0>(bar(sm->s_free[slot]), (jobs & 1u) ^ 1u, flag);
                            if (ok) ok = a8_wait<0>(bar(sm->k_full[r.s]), r.ph, flag);
                            if (!ok) break;
                            tc_fence_after();
                            if (elect_one()) {
                                const uint64_t a0 = a8_desc(ring_k + r.s * kTile, D, 16), b0 = a8_desc(q_buf + slot * p.q_bytes, D, 16);
#pragma unroll
                                for (int q = 0; q < kSParts; ++q) {
#pragma unroll
                                    for (int k = 0; k < D / 32; ++k) umma_f8(sS, a0 + 2 * k, b0 + 2 * k + q * (N * D / 16), idesc, q != 0 || k != 0);
                                }
                                umma_commit(bar(sm->s_full[slot]));
                                umma_commit(bar(sm->k_empty[r.s]));
                                if (!paired) umma_commit(bar(sm->k_empty[r.s]));
                            }
                        } else {
                            ok = a8_wait<0>(bar(sm->v_full[r.s]), r.ph, flag);
                            if (ok) ok = a8_wait<0>(bar(sm->p_full[slot]), jobs & 1u, flag);
                            if (!ok) break;
                            tc_fence_after();
                            if (elect_one()) {
                                const uint64_t a0 = a8_desc(ring_v + r.s * kTile, D, 8192), b0 = a8_desc(p_buf + slot * p.p_bytes, 64, 8192);
#pragma unroll
                                for (int k = 0; k < kAttnTile / 32; ++k)
                                    umma_f8(sO, a0 + k * (32 * D / 16), b0 + k * (32 * 64 / 16), idesc, i != i0 || k != 0);      // a slot's first tile overwrites O
                                umma_commit(bar(sm->pv_done[slot]));
                                umma_commit(bar(sm->v_empty[r.s]));
                                if (!paired) umma_commit(bar(sm->v_empty[r.s]));
                            }
                        }
                        __syncwarp();
                        r.step(stages, step);
                    }
                    if (ok && second && elect_one()) umma_commit(bar(sm->o_full));
                    __syncwarp();
                    tiles += static_cast<uint32_t>(nt);
                    rg.jump(stages, nt);
                }
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(bar(sm->seg_empty[qi]));
            }
            if (warp == 4) cp_async_wait_all();
        }
    } else {
        // ---------------------------------------------------------------- softmax: a thread per key and half of the columns
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        A8Soft w;
        w.slot = (warp - 8) >> 3; w.half = ((warp - 8) >> 2) & 1; w.quad = warp & 3; w.lane = lane; w.row = w.quad * 32 + lane;
        w.lane_off = static_cast<uint32_t>(w.quad * 32) << 16;
        w.small = smem_u32(sm); w.bars = w.small + 8 * w.slot;
        w.tmem = tmem; w.q_smem = q_buf + w.slot * p.q_bytes; w.p_smem = p_buf + w.slot * p.p_bytes + w.row * 64 + (((w.row >> 1) & 3) << 4); w.ring_v = ring_v; w.ring_sc = ring_sc; w.flag = flag;
        uint32_t splits = 0;                     // stretches of shared items so far
        for (uint32_t item = 0; ; ++item) {
            const int qi = item & (kSegQueue - 1);
            const int* const sg = sm->queue[qi];
            if (!a8_wait<0>(bar(sm->seg_full[qi]), (item / kSegQueue) & 1u, flag)) break;
            if (__shfl_sync(0xffffffffu, sg[kSegJobs], 0) == 0) break;
            const bool ok = a8_stretch<E, D, N / 2>(p, sm, w, sg, item);
            if (!ok) break;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm->o_empty));
            if (sg[kSegParts] > 1) {
                // The item is shared: count this block's part, and if it is the last one to arrive, add all of them.  (One
                // thread's fences stand for the block: the barriers before and after order the others' writes and reads.)
                const int first_block = sg[kSegFirst], parts = sg[kSegParts];
                if (lane == 0) mbar_arrive(bar(sm->part_full));
                if (warp == 8) {
                    if (!a8_wait<0>(bar(sm->part_full), splits & 1u, flag)) break;
                    if (lane == 0) {
                        const int shift = sg[kSegShift];
                        __threadfence();
                        const int before = static_cast<int>(static_cast<unsigned>(atomicAdd(p.count + first_block, 1 << shift)) >> shift & 0xffffu);
                        sm->came_last = before == parts - 1;
                        __threadfence();
                        mbar_arrive(bar(sm->last_full));
                        if (before == parts - 1) p.count[first_block] = 0;           // (nobody counts in the other half)
                    }
                    __syncwarp();
                }
                if (!a8_wait<0>(bar(sm->last_full), splits & 1u, flag)) break;
                ++splits;
                if (__shfl_sync(0xffffffffu, *const_cast<volatile int32_t*>(&sm->came_last), 0)) a8_merge<E, D>(p, sg, warp - 8, lane);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm->seg_empty[qi]));
        }
    }

    __syncthreads();
    volatile uint32_t* const aborted = sm->abort;
    if (aborted[0] != 0) {
        // After a time-out: products and copies still in flight have to end before this block's TMEM and shared memory are given up,
        // whoever issued them and however its own loop ended.
        if (warp == 2 || warp == 3 || warp == 5 || warp == 6) {
            const uint32_t mine = bar(sm->drain[warp < 4 ? warp - 2 : warp - 3]);
            if (elect_one()) umma_commit(mine);
            __syncwarp();
            attn_wait(mine, 0, flag + 4);
        } else if ((warp == 1 || warp == 7) && lane == 0) {
            // the last fill of each stage: earlier ones were complete before the stage was filled again
            const int n = warp == 1 ? p.k_stages : p.v_stages;
            const uint32_t full = warp == 1 ? bar(sm->k_full[0]) : bar(sm->v_full[0]);
            for (int e = max(issued - n, 0); e < issued; ++e) attn_wait(full + 8u * (e % n), static_cast<uint32_t>(e / n) & 1u, flag + 4);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (threadIdx.x == 0 && aborted[0] != 0) {
        atomicOr(p.err, 1);
        atomicExch(p.err + 1, static_cast<int>(sm->half ^ 1u));                      // (every block that gave up writes the same)
    }
}

}  // namespace wisv
