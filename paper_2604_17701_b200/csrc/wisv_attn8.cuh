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
// the 8 bits of a bf16 and three the 11 of an fp16 number, above a floor: with queries scaled by a power of two to a largest element in
// [128, 256) and P to a largest value of 64 or more, what is lost is at most 2^-10 (2^-18 of a query row's largest
// element, 2^-16 of a column's largest P).  The products are exact, sums are fp32.  (P is rounded to fp16 on the way, then to 9 bits where
// queries are bf16: half the error of a bf16 P.)  The parts lie side by side as columns, [part][column], so that a tile of K or V is
// read once for all of them.
//
// References.  m grows only when a column's x passes 8.75 (P must stay below 448, the largest e4m3 number), then to the column's largest
// minus 6; l and O are scaled with it.  One vote of the four warps a tile says whether any column has to.
//
// What does not reach a column.  Masked keys have x = -inf and P = 0 exactly.  V behind the last key of a request is cleared in shared memory,
// since 0 times a code of NaN is NaN.  A scale of NaN (a token with infinite or NaN elements) makes x, and so the columns that see
// the token, NaN.  Values with a scale of 0 (or below 2^-40 of the largest of the 32 keys around them) count as that small:
// their l needs a b that can be divided by.
//
// Roles.  One block per SM, persistent: a warp that walks the work and copies keys, one that copies values, one that copies scales, one that
// cuts queries, four that issue the MMAs (S and O of each slot), and two sets of four softmax warps ("slots"), a thread per key.  A
// work item is "paired" - two tiles of columns of the same (request, key head), one per slot, sharing every tile of keys - or, where one
// tile of columns is left, "split": the slots take the key tiles in turn and are put together at the end.  The line of key tiles, its cut
// over the blocks and the joining of shared items are those of the 16-bit cache (wisv_attn.cuh).
#pragma once

#include <stddef.h>

#include "wisv_attn.cuh"

namespace wisv {

constexpr int kA8Cols = 64;                      // columns of a tile
constexpr int kA8Stages = 12;                    // at most, of keys and of values
constexpr int kA8Scales = 8;                     // tiles of scales in flight
constexpr int kA8Small = 9 * 1024;               // barriers, queue, tables of columns
constexpr int kA8Slack = 1024;
constexpr float kA8Grow = 8.75f, kA8Room = 6.0f;

struct Attn8Params : AttnParams {
    const void* q; int64_t qt, qh;               // in elements
    const float *ks, *vs;                        // scales: tokens of a page and head side by side
    int64_t ksp, ksh, vsp, vsh;                  // strides of pages and heads, in floats
    int32_t cols;                                // 16, 32 or 64: no tile has more
    int32_t k_stages, v_stages;                  // even
    uint32_t q_bytes, p_bytes;                   // of a tile's queries, of a slot's P
};

template <typename E> struct a8_parts { static constexpr int n = is_bf16<E>::value ? 2 : 3; };

// TMEM: 256 columns a slot, S (at most 64 columns for each part) from the first, O behind it, with a column for each part where that fits:
// V then is read once for all parts (a product whose operand has to be turned takes 73 clocks whatever its columns, 16 to 128).
template <typename E> __host__ __device__ constexpr int a8_o_at() { return kA8Cols * a8_parts<E>::n; }
template <typename E> __host__ __device__ constexpr bool a8_stacked(int cols) { return a8_parts<E>::n * cols <= 256 - a8_o_at<E>(); }
// bytes of a slot's P: 64 columns of 128 keys in a piece
template <typename E> __host__ __device__ constexpr int a8_p_bytes(int cols) { return (a8_stacked<E>(cols) ? (a8_parts<E>::n * cols + 63) / 64 : a8_parts<E>::n) * 8192; }

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
// kind::f8f6f4, e4m3 operands, fp32 accumulator; `mn`: both operands MN-major
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
// an arrival on `bar` when the thread's copies so far are done
__device__ __forceinline__ void cp_async_arrive(uint32_t bar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
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
__device__ __forceinline__ float warp_max_nan(float x)
{
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
// Two numbers below 448 in NP e4m3 parts each, largest first; codes in pairs, the first number in the low byte
template <int NP>
__device__ __forceinline__ void a8_cut(float lo, float hi, uint32_t (&c)[NP])
{
    uint32_t h;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(hi), "f"(lo));
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        uint16_t e;
        asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(e) : "r"(h));
        c[p] = e;
        if (p + 1 < NP) {
            uint32_t back;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(back) : "h"(e));
            asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(h) : "r"(back));
        }
    }
}

template <typename E> __device__ __forceinline__ E a8_round(float x);
template <> __device__ __forceinline__ __nv_bfloat16 a8_round<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half a8_round<__half>(float x) { return __float2half_rn(x); }

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
    uint64_t q_full[2], q_empty[2];              // query buffers
    uint64_t s_full[2], s_free[2], p_full[2], pv_done[2], vote[2];          // slots
    uint64_t seg_full[kSegQueue], seg_empty[kSegQueue], rs_full[kSegQueue];
    uint64_t o_full, o_empty, ml_full, fin_full, part_full, last_full, drain[4];
    uint32_t tmem;
    uint32_t abort[2];                           // [1] is for the waits after a time-out
    uint32_t pad;
    uint32_t limit[2];                           // three words behind either flag
    int32_t came_last;
    uint32_t half;
    int32_t queue[kSegQueue][kSegWords];
    float rs[kSegQueue][2][kA8Cols];             // c over a query column's power of two
    float m[2][kA8Cols];                         // references
    float a[2][kA8Cols];                         // factors when they grow; at the end those of a slot's own O
    float b[2][kA8Cols];                         // at the end: of the other slot's O
    float mx[2][4][kA8Cols];                     // maxima of the warps; at the end their l
    int32_t grow[2][2][4];
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
        if (!attn_wait_warp(empty + 8u * rg.s, rg.ph ^ 1u, flag)) return false;
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

// A tile of queries cut into parts, by one warp: D / 16 lanes to a row of 16 elements each.
template <typename E, int D>
__device__ __forceinline__ void a8_cut_queries(const Attn8Params& p, int row0, int head, int rows, int cols, uint32_t dst, float* rs, int lane)
{
    constexpr int NP = a8_parts<E>::n, L = D / 16, R = 32 / L;
    const int c = lane % L;
    for (int r0 = 0; r0 < cols; r0 += 4 * R) {
        uint4 w[4][2];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = r0 + u * R + lane / L;
            w[u][0] = w[u][1] = make_uint4(0, 0, 0, 0);
            if (r < rows) {
                const int t = attn_token(p, r);
                const uint4* src = reinterpret_cast<const uint4*>(static_cast<const E*>(p.q) + (row0 + t) * p.qt + (head * p.group + r - t * p.group) * p.qh) + 2 * c;
                w[u][0] = src[0];
                w[u][1] = src[1];
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = r0 + u * R + lane / L;
            if (R == 8 && r0 + u * R >= cols) break;                                 // (16 columns: the warp as one)
            const uint32_t* v = reinterpret_cast<const uint32_t*>(w[u]);
            float x[16];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (is_bf16<E>::value) {
                    x[2 * i] = __uint_as_float(v[i] << 16);
                    x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
                } else {
                    x[2 * i] = __half2float(__ushort_as_half(static_cast<unsigned short>(v[i] & 0xffffu)));
                    x[2 * i + 1] = __half2float(__ushort_as_half(static_cast<unsigned short>(v[i] >> 16)));
                }
                top = max(top, max(__float_as_uint(x[2 * i]) & 0x7fffffffu, __float_as_uint(x[2 * i + 1]) & 0x7fffffffu));
            }
#pragma unroll
            for (int o = 1; o < L; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            const bool fine = top < 0x7f800000u;
            const uint32_t e = max(top >> 23, 8u);                                   // (0 and what is below 2^-119 are scaled alike)
            const float up = fine ? __uint_as_float((261u - e) << 23) : 0.0f;        // largest element to [128, 256)
            uint32_t out[NP][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t a[NP], b[NP];
                a8_cut<NP>(fine ? x[4 * i] * up : 0.0f, fine ? x[4 * i + 1] * up : 0.0f, a);
                a8_cut<NP>(fine ? x[4 * i + 2] * up : 0.0f, fine ? x[4 * i + 3] * up : 0.0f, b);
#pragma unroll
                for (int q = 0; q < NP; ++q) out[q][i] = a[q] | b[q] << 16;
            }
#pragma unroll
            for (int q = 0; q < NP; ++q) {
                const int row = q * cols + r;
                const uint32_t at = dst + row * D + ((D == 128 ? c ^ (row & 7) : c ^ ((row >> 1) & 3)) << 4);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(out[q][0]), "r"(out[q][1]), "r"(out[q][2]), "r"(out[q][3]) : "memory");
            }
            if (c == 0) rs[r] = r >= rows ? 0.0f : fine ? p.scale_log2 * __uint_as_float((e - 7u) << 23) : CUDART_NAN_F;
        }
    }
}

// The merge of an item's partials by the eight softmax warps of the block that came last: a warp takes a column at a time, its lanes
// the D elements; four partials are loaded together and added in block order.  Reads go past L1, which other blocks'
// writes do not reach.
template <typename E, int D>
__device__ __forceinline__ void a8_merge(const Attn8Params& p, const int* sg, int w, int lane)
{
    constexpr int V = D / 32, U = 4;
    const int parts = __shfl_sync(0xffffffffu, sg[kSegParts], 0);
    const int rows0 = __shfl_sync(0xffffffffu, sg[kSegRows0], 0), rows = rows0 + __shfl_sync(0xffffffffu, sg[kSegRows1], 0);
    const int first = sg[kSegFirst];
    for (int r = w; r < rows; r += 8) {
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
        const int t = attn_token(p, in), tok = sg[kSegRow] + t + (second ? p.tpt : 0), head = sg[kSegHead] * p.group + in - t * p.group;
        E* const dst = static_cast<E*>(p.out) + tok * p.ot + head * p.oh + lane * V;
        if (V == 4)
            *reinterpret_cast<uint2*>(dst) = make_uint2(pack2<E>(acc[0] * inv, acc[1] * inv), pack2<E>(acc[V - 2] * inv, acc[V - 1] * inv));
        else
            *reinterpret_cast<uint32_t*>(dst) = pack2<E>(acc[0] * inv, acc[1] * inv);
        if (p.lse && lane == 0)
            p.lse[static_cast<int64_t>(tok) * (p.n_kv * p.group) + head] = l == 0.0f ? -CUDART_INF_F : (m + attn_lg2(l)) * 0.6931471805599453f;
    }
}

// columns of the tiles of an item with so many rows in its larger tile
__device__ __forceinline__ int a8_cols(int rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : kA8Cols; }

// What a softmax warp carries from stretch to stretch
struct A8Soft {
    int slot, quad, lane, row;                   // row: of the tile of keys
    uint32_t lane_off, tmem, p_smem, ring_v, ring_sc, flag;
    uint32_t jobs = 0, votes = 0;                // of this slot so far
    uint32_t tiles = 0;                          // of the block so far
    A8Ring v, sc;                                // the place of tile number `tiles`
};

constexpr float kA8None = -3.402823466e38f;      // the reference of a column that has seen no key

// A stretch of an item's tiles with at most 16 NC columns, up to and including its outputs or partials.  false: a wait ran out.
template <typename E, int D, int NC>
__device__ __forceinline__ bool a8_stretch(const Attn8Params& p, A8Small* sm, A8Soft& w, const int* sg, int qi, uint32_t item)
{
    constexpr int NP = a8_parts<E>::n, N = 16 * NC;
    constexpr bool kStacked = a8_stacked<E>(N);                      // O has a column per part
    constexpr int kOAt = a8_o_at<E>(), kOParts = kStacked ? NP : 1;
    const int slot = w.slot;
    const bool paired = sg[kSegPaired];
    const int nt = sg[kSegT1] - sg[kSegT0], keys = sg[kSegKeys];
    const int limit = sg[kSegLimit] + (paired && slot ? p.tpt : 0);  // last key that the tile's first token sees
    const uint32_t aS = w.tmem + static_cast<uint32_t>(slot) * 256 + w.lane_off, aO = aS + kOAt;
    const float* const rs = sm->rs[qi][paired ? slot : 0];
    float* const m = sm->m[slot];
    auto vote = [&]() {                                              // the slot's four warps meet
        __syncwarp();
        if (w.lane == 0) mbar_arrive(smem_u32(&sm->vote[slot]));
        const bool ok = attn_wait_warp(smem_u32(&sm->vote[slot]), w.votes & 1u, w.flag);
        ++w.votes;
        return ok;
    };
    if (w.row < N) m[w.row] = kA8None;
    if (!attn_wait_warp(smem_u32(&sm->rs_full[qi]), static_cast<uint32_t>(item / kSegQueue) & 1u, w.flag)) return false;
    uint64_t l[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) l[i] = 0;

    const int i0 = paired ? 0 : static_cast<int>((w.tiles ^ static_cast<uint32_t>(slot)) & 1u), step = paired ? 1 : 2;
    A8Ring rv = w.v, rsc = w.sc;
    if (i0) { rv.step(p.v_stages, 1); rsc.step(kA8Scales, 1); }
    for (int i = i0; i < nt; i += step) {
        const int key0 = (sg[kSegT0] + i) * kAttnTile, key = key0 + w.row;
        // ---- the scales of this thread's key
        if (!attn_wait_warp(smem_u32(&sm->sc_full[rsc.s]), rsc.ph, w.flag)) return false;
        float ka, vb;
        {
            const uint32_t at = w.ring_sc + rsc.s * 1024 + w.row * 4;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(ka) : "r"(at) : "memory");
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(vb) : "r"(at + 512) : "memory");
        }
        __syncwarp();
        if (w.lane == 0) {
            mbar_arrive(smem_u32(&sm->sc_empty[rsc.s]));
            if (!paired) mbar_arrive(smem_u32(&sm->sc_empty[rsc.s]));
        }
        rsc.step(kA8Scales, step);
        if (key >= keys) { ka = 0.0f; vb = 0.0f; }
        const uint32_t top = __reduce_max_sync(0xffffffffu, vb > 0.0f && vb < CUDART_INF_F ? __float_as_uint(vb) : 0u);
        const float be = fmaxf(vb, fmaxf(__uint_as_float(top) * 9.094947e-13f, 7.888609e-31f));     // 2^-40 of the largest, 2^-100
        const float lb = vb == vb ? attn_lg2(be) : CUDART_NAN_F, rb = attn_rcp(be);
        const uint64_t ka2 = pair(ka, ka), lb2 = pair(lb, lb), rb2 = pair(rb, rb);
        // columns from `vis` on see this key
        const bool masked = key0 + kAttnTile - 1 > limit;
        const int vis = key >= keys ? 1 << 20 : min(max(key - limit, 0), kA8Cols + 1) * p.group;

        if (!attn_wait_warp(smem_u32(&sm->s_full[slot]), w.jobs & 1u, w.flag)) return false;
        tc_fence_after();
        float x[N];
        // Pass 0 finds x with the references as they are; where a column outgrows its own, pass 1 finds x + m for its maximum and pass 2 x
        // with the new references.  (The first tile of a stretch has none yet.)
        for (int pass = i == i0 ? 1 : 0; ; ++pass) {
            constexpr int W = N < 32 ? N : 32;
            const float neg = pass == 1 ? 0.0f : -1.0f;
            const uint64_t neg2 = pair(neg, neg);
#pragma unroll
            for (int c = 0; c < N; c += W) {
                uint32_t s[NP][W];
#pragma unroll
                for (int q = 0; q < NP; ++q) {
                    if (W == 32) tmem_ld32(aS + q * N + c, s[q]);
                    else tmem_ld16(aS + q * N + c, *reinterpret_cast<uint32_t (*)[16]>(s[q]));
                }
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < W; j += 4) {
                    const float4 r4 = *reinterpret_cast<const float4*>(rs + c + j), m4 = *reinterpret_cast<const float4*>(m + c + j);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int k = j + 2 * h;
                        uint64_t v = pair(__uint_as_float(s[0][k]), __uint_as_float(s[0][k + 1]));
#pragma unroll
                        for (int q = 1; q < NP; ++q) v = add2(v, pair(__uint_as_float(s[q][k]), __uint_as_float(s[q][k + 1])));
                        v = fma2(mul2(v, h ? pair(r4.z, r4.w) : pair(r4.x, r4.y)), ka2, lb2);
                        v = fma2(h ? pair(m4.z, m4.w) : pair(m4.x, m4.y), neg2, v);
                        x[c + k] = low(v);
                        x[c + k + 1] = high(v);
                    }
                }
            }
            if (masked) {
#pragma unroll
                for (int n = 0; n < N; ++n) x[n] = n >= vis ? x[n] : -CUDART_INF_F;
            }
            if (pass == 2) break;
            if (pass == 0) {
                float worst[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                for (int n = 0; n < N; n += 4) {
                    worst[0] = max3_nan(worst[0], x[n], x[n + 1]);
                    worst[1] = max3_nan(worst[1], x[n + 2], x[n + 3]);
                }
                const bool mine = __any_sync(0xffffffffu, !(worst[0] <= kA8Grow && worst[1] <= kA8Grow));
                volatile int32_t* const grow = sm->grow[slot][w.votes & 1u];
                if (w.lane == 0) grow[w.quad] = mine;
                if (!vote()) return false;
                if (!(grow[0] | grow[1] | grow[2] | grow[3])) break;
                continue;
            }
            // ---- the references grow
#pragma unroll
            for (int c = 0; c < N; c += W) {
                float keep = 0.0f;
#pragma unroll
                for (int n = 0; n < W; ++n) {
                    const float r = warp_max_nan(x[c + n]);
                    if (n == w.lane) keep = r;
                }
                if (w.lane < W) sm->mx[slot][w.quad][c + w.lane] = keep;
            }
            if (!vote()) return false;
            if (w.row < N) {
                const float (&mx)[4][kA8Cols] = sm->mx[slot];
                const float big = max3_nan(max3_nan(mx[0][w.row], mx[1][w.row], mx[2][w.row]), mx[3][w.row], mx[3][w.row]);
                const float old = m[w.row];
                const bool grows = !(big - old <= kA8Grow), bad = !(big < CUDART_INF_F);             // (a score of NaN or +inf)
                const float now = !grows ? old : !bad ? big - kA8Room : old == kA8None ? 0.0f : old;
                sm->a[slot][w.row] = !grows ? 1.0f : bad ? CUDART_NAN_F : attn_ex2(old - now);
                m[w.row] = now;
            }
            if (!vote()) return false;
            if (i != i0) {
                if (!attn_wait_warp(smem_u32(&sm->pv_done[slot]), (w.jobs - 1) & 1u, w.flag)) return false;
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < kOParts * N; c += 16) {
                    uint32_t o[16];
                    tmem_ld16(aO + c, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * sm->a[slot][c % N + j]);
                    tmem_st16(aO + c, o);
                }
                tmem_wait_st();
            }
#pragma unroll
            for (int n = 0; n < N; n += 2) l[n / 2] = mul2(l[n / 2], pair(sm->a[slot][n], sm->a[slot][n + 1]));
        }
        tc_fence_before();
        __syncwarp();
        if (w.lane == 0) mbar_arrive(smem_u32(&sm->s_free[slot]));

        // ---- P, once the product before has read the last one
        if (w.jobs) {
            if (!attn_wait_warp(smem_u32(&sm->pv_done[slot]), (w.jobs - 1) & 1u, w.flag)) return false;
        }
        if (key0 + kAttnTile > keys) {
            // (both slots of a paired item clear: whoever comes second writes zeros over zeros)
            if (!attn_wait_warp(smem_u32(&sm->v_full[rv.s]), rv.ph, w.flag)) return false;
            if (key >= keys) {
                const uint32_t at = w.ring_v + rv.s * a8_tile_bytes<D>() + w.row * D;
#pragma unroll
                for (int c = 0; c < D; c += 16) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + c), "r"(0) : "memory");
            }
        }
        rv.step(p.v_stages, step);
#pragma unroll
        for (int c = 0; c < N; c += 16) {
            uint32_t out[NP][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t e[2][NP];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int n = c + 4 * j + 2 * h;
                    const float e0 = attn_ex2(x[n]), e1 = attn_ex2(x[n + 1]);
                    l[n / 2] = fma2(pair(e0, e1), rb2, l[n / 2]);
                    a8_cut<NP>(e0, e1, e[h]);
                }
#pragma unroll
                for (int q = 0; q < NP; ++q) out[q][j] = e[0][q] | e[1][q] << 16;
            }
#pragma unroll
            for (int q = 0; q < NP; ++q) {
                const int n = q * (kStacked ? N : kA8Cols) + c;      // column of the operand; rows of 64 bytes, swizzled
                const uint32_t at = w.p_smem + (n >> 6) * 8192 + w.row * 64 + ((((n >> 4) & 3) ^ ((w.row >> 1) & 3)) << 4);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(out[q][0]), "r"(out[q][1]), "r"(out[q][2]), "r"(out[q][3]) : "memory");
            }
        }
        fence_proxy_async();
        tc_fence_before();
        __syncwarp();
        if (w.lane == 0) mbar_arrive(smem_u32(&sm->p_full[slot]));
        ++w.jobs;
    }

    // ---- sums over the keys: lanes first (a lane ends with N / 32 columns, or two lanes with one), then warps, then slots
    if (!attn_wait_warp(smem_u32(&sm->o_full), item & 1u, w.flag)) return false;
    tc_fence_after();
    {
        float v[N];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) { v[2 * i] = low(l[i]); v[2 * i + 1] = high(l[i]); }
        int len = N;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            if (len > 1) {
                len >>= 1;
                const bool up = (w.lane & o) != 0;
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    if (i < len) {
                        const float keep = up ? v[i + len] : v[i], send = up ? v[i] : v[i + len];
                        v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                    }
                }
            } else {
                v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
            }
        }
        float* const mine = sm->mx[slot][w.quad];
        if (NC == 4) { mine[2 * w.lane] = v[0]; mine[2 * w.lane + 1] = v[1]; }
        else if (NC == 2) mine[w.lane] = v[0];
        else if ((w.lane & 1) == 0) mine[w.lane >> 1] = v[0];
    }
    __syncwarp();
    if (w.lane == 0) mbar_arrive(smem_u32(&sm->ml_full));
    if (!attn_wait_warp(smem_u32(&sm->ml_full), item & 1u, w.flag)) return false;
    const int rows = paired && slot ? sg[kSegRows1] : sg[kSegRows0];
    const bool first = sg[kSegT0] == 0, whole = first && sg[kSegT1] == sg[kSegTiles];
    const int part = static_cast<int>(blockIdx.x) * 2 + (first ? 1 : 0), part_row = paired ? slot * kA8Cols : 0;
    const int tok0 = sg[kSegRow] + (paired && slot ? p.tpt : 0), head0 = sg[kSegHead] * p.group;
    if (w.row < N) {
        const int n = w.row;
        auto sum = [&](int s) { return (sm->mx[s][0][n] + sm->mx[s][1][n]) + (sm->mx[s][2][n] + sm->mx[s][3][n]); };
        float mm = m[n], ll = sum(slot), wa = 1.0f, wb = 0.0f;
        if (!paired) {
            const float other = sm->m[slot ^ 1][n], top = fmaxf(mm, other);
            wa = mm == kA8None ? 0.0f : attn_ex2(mm - top);
            wb = other == kA8None ? 0.0f : attn_ex2(other - top);
            ll = ll * wa + sum(slot ^ 1) * wb;
            mm = top;
        }
        if (mm == kA8None) { mm = -CUDART_INF_F; wa = 0.0f; }
        if (whole) {
            const float inv = ll == 0.0f ? 0.0f : attn_rcp(ll);
            wa *= inv;
            wb *= inv;
        }
        sm->a[slot][n] = wa;
        sm->b[slot][n] = wb;
        if (n < rows && (paired || slot == 0)) {
            if (!whole) p.part_ml[part * (2 * kA8Cols) + part_row + n] = make_float2(mm, ll);
            else if (p.lse) {
                const int t = attn_token(p, n);
                p.lse[static_cast<int64_t>(tok0 + t) * (p.n_kv * p.group) + head0 + n - t * p.group] =
                    ll == 0.0f ? -CUDART_INF_F : (mm + attn_lg2(ll)) * 0.6931471805599453f;
            }
        }
    }
    __syncwarp();
    if (w.lane == 0) mbar_arrive(smem_u32(&sm->fin_full));
    if (!attn_wait_warp(smem_u32(&sm->fin_full), item & 1u, w.flag)) return false;

    // ---- outputs: a thread has one element of every column; split: each slot does half of the columns, from both accumulators
    const int d = D == 128 ? w.row : w.quad * 16 + w.lane;
    const bool has = D == 128 || w.lane < 16;
    const uint32_t other = slot ? aO - 256 : aO + 256;
    const int c0 = paired ? 0 : slot * (N / 2), c1 = min(paired ? N : c0 + N / 2, rows);
    for (int c = c0; c < c1; c += 8) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = 0.0f;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            if (side && paired) break;
            uint32_t o[kOParts][8];
#pragma unroll
            for (int q = 0; q < kOParts; ++q) tmem_ld8((side ? other : aO) + q * N + c, o[q]);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = side ? sm->b[slot][c + j] : sm->a[slot][c + j];
                float v = __uint_as_float(o[0][j]);
#pragma unroll
                for (int q = 1; q < kOParts; ++q) v += __uint_as_float(o[q][j]);
                if (f != 0.0f) y[j] = fmaf(v, f, y[j]);              // (an accumulator without a job may hold anything)
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int n = c + j;
            if (n >= rows || !has) continue;
            if (whole) {
                const int t = attn_token(p, n);
                static_cast<E*>(p.out)[(tok0 + t) * p.ot + (head0 + n - t * p.group) * p.oh + d] = a8_round<E>(y[j]);
            } else {
                p.part_o[(static_cast<size_t>(part) * (2 * kA8Cols) + part_row + n) * D + d] = y[j];
            }
        }
    }
    w.tiles += static_cast<uint32_t>(nt);
    w.v.jump(p.v_stages, nt);
    w.sc.jump(kA8Scales, nt);
    return true;
}

template <typename E, int D>
__global__ void __launch_bounds__(kAttnThreads, 1)
attn8_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const Attn8Params p)
{
    constexpr int NP = a8_parts<E>::n;
    constexpr uint32_t kTile = a8_tile_bytes<D>();

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;
    const uint32_t q_buf = raw_addr + pad, p_buf = q_buf + 2 * p.q_bytes, ring_k = p_buf + 2 * p.p_bytes;
    const uint32_t ring_v = ring_k + p.k_stages * kTile, ring_sc = ring_v + p.v_stages * kTile;
    const uint32_t small_off = ring_sc + kA8Scales * 1024 - raw_addr;
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
        for (int s = 0; s < kA8Scales; ++s) { mbar_init(bar(sm->sc_full[s]), 32); mbar_init(bar(sm->sc_empty[s]), 8); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(sm->q_full[s]), 1); mbar_init(bar(sm->q_empty[s]), 2);
            mbar_init(bar(sm->s_full[s]), 1); mbar_init(bar(sm->s_free[s]), 4);
            mbar_init(bar(sm->p_full[s]), 4); mbar_init(bar(sm->pv_done[s]), 1);
            mbar_init(bar(sm->vote[s]), 4);
        }
        for (int s = 0; s < kSegQueue; ++s) { mbar_init(bar(sm->seg_full[s]), 1); mbar_init(bar(sm->seg_empty[s]), 15); mbar_init(bar(sm->rs_full[s]), 1); }
        mbar_init(bar(sm->o_full), 2); mbar_init(bar(sm->o_empty), 8); mbar_init(bar(sm->ml_full), 8); mbar_init(bar(sm->fin_full), 8);
        mbar_init(bar(sm->part_full), 8); mbar_init(bar(sm->last_full), 1);
        for (int s = 0; s < 4; ++s) mbar_init(bar(sm->drain[s]), 1);
        sm->abort[0] = 0; sm->abort[1] = 0;
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

    // warps 0: queries; 1: the walk and keys; 2, 3: S of the slots; 4: scales; 5, 6: O of the slots; 7: values
    if (warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 1) {
            const int half = __ldcg(p.err + 1) & 1;
            AttnWalk walk;
            unsigned share, more;
            attn_range<D>(p, me, lane, walk, share, more);
            int s[kSegWords + 1];
            A8Ring rg;
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
                ok = attn_wait_warp(bar(sm->seg_empty[qi]), (static_cast<uint32_t>(item / kSegQueue) & 1u) ^ 1u, flag);
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
            if (threadIdx.x == 0) {
                const unsigned half = static_cast<unsigned>(__ldcg(p.err + 1)) & 1u;
                sm->half = half;
                const unsigned other = 0xffffu << (16u * (half ^ 1u));
                if (static_cast<unsigned>(__ldcg(p.count + me)) & other) atomicAnd(p.count + me, static_cast<int>(~other));
            }
            __syncwarp();
            const int slot = warp == 3 || warp == 6 ? 1 : 0;
            A8Ring rg;
            uint32_t tiles = 0, jobs = 0;        // of the block, of the slot
            int q_used = 0;
            bool ok = warp != 7 || static_cast<int>(me) != p.stalled;
            for (int item = 0; ok; ++item) {
                const int qi = item & (kSegQueue - 1);
                ok = attn_wait_warp(bar(sm->seg_full[qi]), static_cast<uint32_t>(item / kSegQueue) & 1u, flag);
                if (!ok) break;
                const int* const sg = sm->queue[qi];
                if (__shfl_sync(0xffffffffu, sg[kSegJobs], 0) == 0) break;           // (the compiler then knows it uniform)
                const bool paired = __shfl_sync(0xffffffffu, sg[kSegPaired], 0) != 0;
                const int t0 = __shfl_sync(0xffffffffu, sg[kSegT0], 0), t1 = __shfl_sync(0xffffffffu, sg[kSegT1], 0), nt = t1 - t0;
                const int rows0 = __shfl_sync(0xffffffffu, sg[kSegRows0], 0), rows1 = __shfl_sync(0xffffffffu, sg[kSegRows1], 0);
                const int cols = a8_cols(max(rows0, rows1));
                const int req = sg[kSegReq], keys = sg[kSegKeys], head = sg[kSegHead];
                if (warp == 7) {
                    // ------------------------------------------------ values
                    ok = a8_load_tiles<D>(p, &tmV, req, attn_page(p, req, t0, t1, keys, lane), t0, t1, keys, head, ring_v, bar(sm->v_full[0]),
                                          bar(sm->v_empty[0]), p.v_stages, flag, lane, rg, issued);
                } else if (warp == 4) {
                    // ------------------------------------------------ scales: a lane copies those of four tokens
                    const int mask = (1 << p.page_shift) - 1;
                    auto page = [&](int t) {
                        const int tok = t * kAttnTile + 4 * lane;
                        return t < t1 && tok < keys ? p.block_table[req * p.table_stride + (tok >> p.page_shift)] : -1;
                    };
                    int pg = page(t0);
                    for (int t = t0; t < t1; ++t) {
                        const bool in = pg >= 0 && pg < p.n_pages;
                        const int at = in ? (t * kAttnTile + 4 * lane) & mask : 0, from = in ? pg : 0;
                        pg = page(t + 1);
                        ok = attn_wait_warp(bar(sm->sc_empty[rg.s]), rg.ph ^ 1u, flag);
                        if (!ok) break;
                        const uint32_t dst = ring_sc + rg.s * 1024 + lane * 16;
                        cp_async16(dst, p.ks + from * p.ksp + head * p.ksh + at, in ? 16 : 0);
                        cp_async16(dst + 512, p.vs + from * p.vsp + head * p.vsh + at, in ? 16 : 0);
                        cp_async_arrive(bar(sm->sc_full[rg.s]));
                        rg.step(kA8Scales, 1);
                    }
                } else if (warp == 0) {
                    // ------------------------------------------------ queries
                    for (int t = 0; ok && t < (paired ? 2 : 1); ++t, ++q_used) {
                        const int qb = q_used & 1;
                        ok = attn_wait_warp(bar(sm->q_empty[qb]), ((q_used >> 1) & 1u) ^ 1u, flag);
                        if (!ok) break;
                        a8_cut_queries<E, D>(p, sg[kSegRow] + t * p.tpt, head, t ? rows1 : rows0, cols, q_buf + qb * p.q_bytes, sm->rs[qi][t], lane);
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(sm->q_full[qb]));
                    }
                    if (ok && lane == 0) mbar_arrive(bar(sm->rs_full[qi]));
                } else {
                    // ------------------------------------------------ MMA: a warp per slot and product
                    const bool second = warp > 4;
                    const int qb = (q_used + (paired ? slot : 0)) & 1, stages = second ? p.v_stages : p.k_stages;
                    const bool stacked = a8_stacked<E>(cols);
                    const uint32_t sS = tmem + slot * 256, sO = sS + a8_o_at<E>();
                    const uint32_t idesc = second ? a8_idesc(D, stacked ? NP * cols : cols, true) : a8_idesc(kAttnTile, NP * cols, false);
                    if (!second) {
                        // (a paired item's other buffer too, so that no warp skips a phase)
                        for (const int end = q_used + (paired ? 2 : 1); ok && q_used < end; ++q_used)
                            ok = attn_wait_warp(bar(sm->q_full[q_used & 1]), static_cast<uint32_t>(q_used >> 1) & 1u, flag);
                    } else if (item > 0) {
                        ok = attn_wait_warp(bar(sm->o_empty), static_cast<uint32_t>(item - 1) & 1u, flag);   // the previous O has been read
                    }
                    const int i0 = paired ? 0 : static_cast<int>((tiles ^ static_cast<uint32_t>(slot)) & 1u), step = paired ? 1 : 2;
                    A8Ring r = rg;
                    if (i0) r.step(stages, 1);
                    for (int i = i0; ok && i < nt; i += step, ++jobs) {
                        if (!second) {
                            ok = attn_wait_warp(bar(sm->s_free[slot]), (jobs & 1u) ^ 1u, flag);
                            if (ok) ok = attn_wait_warp(bar(sm->k_full[r.s]), r.ph, flag);
                            if (!ok) break;
                            tc_fence_after();
                            if (elect_one()) {
                                const uint64_t a0 = a8_desc(ring_k + r.s * kTile, D, 16), b0 = a8_desc(q_buf + qb * p.q_bytes, D, 16);
#pragma unroll
                                for (int k = 0; k < D / 32; ++k) umma_f8(sS, a0 + 2 * k, b0 + 2 * k, idesc, k != 0);
                                umma_commit(bar(sm->s_full[slot]));
                                umma_commit(bar(sm->k_empty[r.s]));
                                if (!paired) umma_commit(bar(sm->k_empty[r.s]));
                            }
                        } else {
                            ok = attn_wait_warp(bar(sm->v_full[r.s]), r.ph, flag);
                            if (ok) ok = attn_wait_warp(bar(sm->p_full[slot]), jobs & 1u, flag);
                            if (!ok) break;
                            tc_fence_after();
                            if (elect_one()) {
                                const uint64_t a0 = a8_desc(ring_v + r.s * kTile, D, 8192), b0 = a8_desc(p_buf + slot * p.p_bytes, 64, 8192);
                                for (int q = 0; q < (stacked ? 1 : NP); ++q) {
#pragma unroll
                                    for (int k = 0; k < kAttnTile / 32; ++k)
                                        umma_f8(sO, a0 + k * (32 * D / 16), b0 + k * (32 * 64 / 16) + q * (8192 / 16), idesc,
                                                (i != i0 || q != 0 || k != 0) ? 1u : 0u);            // a slot's first tile overwrites O
                                }
                                umma_commit(bar(sm->pv_done[slot]));
                                umma_commit(bar(sm->v_empty[r.s]));
                                if (!paired) umma_commit(bar(sm->v_empty[r.s]));
                            }
                        }
                        __syncwarp();
                        r.step(stages, step);
                    }
                    if (ok && elect_one()) {
                        if (second) {
                            umma_commit(bar(sm->o_full));
                        } else {
                            umma_commit(bar(sm->q_empty[qb]));
                            if (paired) umma_commit(bar(sm->q_empty[qb]));           // (a split item's buffer hears from both warps)
                        }
                    }
                    __syncwarp();
                    tiles += static_cast<uint32_t>(nt);
                    rg.jump(stages, nt);
                }
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(bar(sm->seg_empty[qi]));
            }
            if (warp == 4) {
                cp_async_wait_all();
                attn_clear_rows<E, D>(p, static_cast<int>(me), static_cast<int>(gridDim.x), lane);
            }
        }
    } else {
        // ---------------------------------------------------------------- softmax: four warps per slot, a thread per key
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        A8Soft w;
        w.slot = (warp - 8) >> 2; w.quad = warp & 3; w.lane = lane; w.row = w.quad * 32 + lane;
        w.lane_off = static_cast<uint32_t>(w.quad * 32) << 16;
        w.tmem = tmem; w.p_smem = p_buf + w.slot * p.p_bytes; w.ring_v = ring_v; w.ring_sc = ring_sc; w.flag = flag;
        uint32_t splits = 0;                     // stretches of shared items so far
        for (uint32_t item = 0; ; ++item) {
            const int qi = item & (kSegQueue - 1);
            const int* const sg = sm->queue[qi];
            if (!attn_wait_warp(bar(sm->seg_full[qi]), (item / kSegQueue) & 1u, flag)) break;
            if (__shfl_sync(0xffffffffu, sg[kSegJobs], 0) == 0) break;
            const int cols = __shfl_sync(0xffffffffu, a8_cols(max(sg[kSegRows0], sg[kSegRows1])), 0);
            bool ok;
            if (cols == 16) ok = a8_stretch<E, D, 1>(p, sm, w, sg, qi, item);
            else if (cols == 32) ok = a8_stretch<E, D, 2>(p, sm, w, sg, qi, item);
            else ok = a8_stretch<E, D, 4>(p, sm, w, sg, qi, item);
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
                    if (!attn_wait_warp(bar(sm->part_full), splits & 1u, flag)) break;
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
                if (!attn_wait_warp(bar(sm->last_full), splits & 1u, flag)) break;
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
