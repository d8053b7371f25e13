// Attention over e4m3 codes where a key head has many query rows (long windows, prompt chunks): rows are the rows of the matrix products.
//
// Mathematics.  As in wisv_attn8.cuh, per 128 query rows and 64 keys: S = Q K^T, x = c S a + log2 b - m, P = exp2(x), l += P / b, O += P V, with
// codes as operands; here a thread has a row, so that its m and l are registers and the scales of the keys come from shared memory, and P
// is the TMEM operand of the second product.  m grows by the rule of the 16-bit kernel (by more than 2^8).
//
// Parts.  Both operands' parts are added in one accumulator, so they are not scaled.  The last one is e5m2, whose steps go down to 2^-16: with a
// largest element of a query row in [128, 256) two parts are exact for bf16 and three for fp16 down to 2^-24 of it; a P, whose largest is
// 1 or more, is rounded to 8 bits (bf16, fp16's 11 on the way) or 13 (fp16), down to 2^-17.
//
// Against the kernel with keys as rows it needs a thread per row whether the row exists or not, but no meeting of warps, no tables of columns and half
// of the instructions per element: 64 requests of 12, 16, 17 and 24 rows of 4 heads over 270 k keys take 200, 203, 208 and 211 us here and
// 132, 147, 235 and 243 there, where 17 tokens are two tiles.  Hence the rule: more than 64 rows to a request on the average.  The roles
// are those of wisv_attn8.cuh, slots and merge those of wisv_attn.cuh.
//
// Measured (8B shape, D = 128, short runs): 2 x 2048 rows over 8 k keys 612 us, 0.89 PFLOP/s of the formula's (each product is done twice, a
// part at a time); 8 requests of 65 rows of 7 heads over 120 k keys 155 us.  What bounds it: two softmax warps on each scheduler, which issue half of the
// time; the tensor pipe is active 39 %.
#pragma once

#include "wisv_attn8.cuh"

namespace wisv {

constexpr int kR8Small = 8 * 1024;
constexpr int kR8Fixed = kA8Slack + kR8Small + kA8Scales * kA8ScaleBytes;            // shared memory beside queries and tiles

struct R8Small {
    uint64_t k_full[kA8Stages], k_empty[kA8Stages], v_full[kA8Stages], v_empty[kA8Stages];
    uint64_t sc_full[kA8Scales], sc_empty[kA8Scales];
    uint64_t q_full[2], s_full[4], p_full[4], s_free[4];             // slots; 2 half + slot
    uint64_t seg_full[kSegQueue], seg_empty[kSegQueue];
    uint64_t turn[2][4];                         // at the exponentials: of slots, for the two warps of a scheduler
    uint64_t o_full, o_empty, ml_full, part_full, last_full, drain[4];
    uint32_t tmem;
    uint32_t abort[2];                           // [1] is for the waits after a time-out
    uint32_t pad;
    uint32_t limit[2];                           // three words behind either flag
    int32_t came_last;
    uint32_t half;
    alignas(16) int32_t queue[kSegQueue][kSegWords];
    float rs[2][kAttnTile];                      // of query rows: c over a row's power of two
    float2 ml[2][kAttnTile];
};
static_assert(sizeof(R8Small) <= kR8Small, "shared memory");
static_assert(offsetof(R8Small, limit) - offsetof(R8Small, abort) == 12, "attn_wait");

// Four numbers below 448 in NP parts each, the last e5m2, the others e4m3 (see a8_cut)
template <int NP, bool kLong>
__device__ __forceinline__ void r8_cut(float x0, float x1, float x2, float x3, uint32_t (&c)[NP])
{
    uint32_t h0, h1;
    if (kLong) {
        c[0] = a8_first(x0, x1, x2, x3, h0, h1);
    } else {
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h0) : "f"(x1), "f"(x0));
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h1) : "f"(x3), "f"(x2));
    }
#pragma unroll
    for (int p = kLong ? 1 : 0; p + 1 < NP; ++p) {
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
    }
    asm("{\n\t"
        ".reg .b16 e0, e1;\n\t"
        "cvt.rn.satfinite.e5m2x2.f16x2 e0, %1;\n\t"
        "cvt.rn.satfinite.e5m2x2.f16x2 e1, %2;\n\t"
        "mov.b32 %0, {e0, e1};\n\t"
        "}"
        : "=r"(c[NP - 1]) : "r"(h0), "r"(h1));
}
// D[tmem] (+)= A[tmem] * B[smem], 8-bit operands, four elements of K per 32-bit column of A
__device__ __forceinline__ void umma_f8_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t"
        "}\n"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// kind::f8f6f4, fp32 sums, B e4m3, A e4m3 or (last) e5m2; bit 16: B is MN-major
__device__ __forceinline__ uint32_t r8_idesc(uint32_t N, bool b_mn, bool last)
{
    return (1u << 4) | (last ? 1u << 7 : 0u) | (b_mn ? 1u << 16 : 0u) | ((N >> 3) << 17) | ((kAttnTile >> 4) << 24);
}
__device__ __forceinline__ uint64_t lds_pair(uint32_t at)
{
    uint64_t r;
    asm volatile("ld.shared.b64 %0, [%1];" : "=l"(r) : "r"(at) : "memory");
    return r;
}

// Rows 32 w .. 32 w + 31 of a slot's tile of queries, cut by warp w of its four: D / 16 lanes to a row of 16 elements.
template <typename E, int D>
__device__ __forceinline__ void r8_cut_queries(const Attn8Params& p, int row0, int head, int rows, uint32_t dst, float* rs, int w, int lane)
{
    constexpr int NP = a8_parts<E>::n, L = D / 16, R = 32 / L;
    const int c = lane % L;
#pragma unroll 1
    for (int r0 = 32 * w; r0 < 32 * w + 32; r0 += 4 * R) {
        if (r0 >= rows) {                        // no such rows: zeros
#pragma unroll
            for (int u = 0; u < 4; ++u) {
#pragma unroll
                for (int q = 0; q < NP; ++q)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst + q * (kAttnTile * D) + (r0 + u * R) * D + lane * 16), "r"(0) : "memory");
                if (c == 0) rs[r0 + u * R + lane / L] = 0.0f;
            }
            continue;
        }
        uint4 v[4][2];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = r0 + u * R + lane / L;
            v[u][0] = v[u][1] = make_uint4(0, 0, 0, 0);
            if (r < rows) {
                const int t = attn_token(p, r);
                const uint4* src = reinterpret_cast<const uint4*>(static_cast<const E*>(p.q) + (row0 + t) * p.qt + (head * p.group + r - t * p.group) * p.qh) + 2 * c;
                v[u][0] = src[0];
                v[u][1] = src[1];
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = r0 + u * R + lane / L;
            const uint32_t* d = reinterpret_cast<const uint32_t*>(v[u]);
            float x[16];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                unpack2<E>(d[i], x[2 * i], x[2 * i + 1]);
                top = max(top, max(__float_as_uint(x[2 * i]) & 0x7fffffffu, __float_as_uint(x[2 * i + 1]) & 0x7fffffffu));
            }
#pragma unroll
            for (int o = 1; o < L; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            const bool fine = top < 0x7f800000u;
            const uint32_t e = fine ? max(top >> 23, 8u) : 8u;       // (0 and what is below 2^-119 are scaled alike)
            const float up = __uint_as_float((261u - e) << 23);      // largest element to [128, 256)
            uint32_t out[NP][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t f[NP];
                r8_cut<NP, false>(fine ? x[4 * i] * up : 0.0f, fine ? x[4 * i + 1] * up : 0.0f, fine ? x[4 * i + 2] * up : 0.0f, fine ? x[4 * i + 3] * up : 0.0f, f);
#pragma unroll
                for (int q = 0; q < NP; ++q) out[q][i] = f[q];
            }
            const uint32_t at = dst + r * D + ((D == 128 ? c ^ (r & 7) : c ^ ((r >> 1) & 3)) << 4);
#pragma unroll
            for (int q = 0; q < NP; ++q)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + q * (kAttnTile * D)), "r"(out[q][0]), "r"(out[q][1]), "r"(out[q][2]), "r"(out[q][3]) : "memory");
            if (c == 0) rs[r] = fine ? p.scale_log2 * __uint_as_float((e - 7u) << 23) : CUDART_NAN_F;
        }
    }
}

template <typename E, int D>
__global__ void __launch_bounds__(kAttnThreads, 1)
attn8_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const Attn8Params p)
{
    constexpr int NP = a8_parts<E>::n;
    constexpr uint32_t kTile = a8_tile_bytes<D>(), kQ = NP * kAttnTile * D;
    constexpr int kStages = (kAttnSmem - kR8Fixed - 2 * static_cast<int>(kQ)) / static_cast<int>(kTile);
    constexpr int kV = (kStages + 1) / 2 < kA8Stages ? (kStages + 1) / 2 : kA8Stages, kK = kStages - kV < kA8Stages ? kStages - kV : kA8Stages;
    static_assert(kK >= 2 && kV >= 3, "shared memory");

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = ((raw_addr + 1023u) & ~1023u) - raw_addr;
    const uint32_t q_buf = raw_addr + pad, ring_k = q_buf + 2 * kQ, ring_v = ring_k + kK * kTile, ring_sc = ring_v + kV * kTile;
    const uint32_t small_off = ring_sc + kA8Scales * kA8ScaleBytes - raw_addr;
    R8Small* const sm = reinterpret_cast<R8Small*>(smem_raw + small_off);
    auto bar = [](const uint64_t& b) { return smem_u32(&b); };
    const unsigned me = blockIdx.x;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int lane = threadIdx.x & 31;

    if (small_off + kR8Small > static_cast<uint32_t>(kAttnSmem)) {            // (dynamic shared memory starts 1024-byte aligned)
        if (threadIdx.x == 0) atomicOr(p.err, 2);
        return;
    }
    const uint32_t flag = smem_u32(&sm->abort[0]);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kK; ++s) { mbar_init(bar(sm->k_full[s]), 1); mbar_init(bar(sm->k_empty[s]), 2); }
        for (int s = 0; s < kV; ++s) { mbar_init(bar(sm->v_full[s]), 1); mbar_init(bar(sm->v_empty[s]), 2); }
        for (int s = 0; s < kA8Scales; ++s) { mbar_init(bar(sm->sc_full[s]), 1); mbar_init(bar(sm->sc_empty[s]), 8); }
        for (int s = 0; s < 2; ++s) mbar_init(bar(sm->q_full[s]), 4);
        for (int s = 0; s < 4; ++s) { mbar_init(bar(sm->s_full[s]), 1); mbar_init(bar(sm->p_full[s]), 4); mbar_init(bar(sm->s_free[s]), 1); }
        for (int s = 0; s < kSegQueue; ++s) { mbar_init(bar(sm->seg_full[s]), 1); mbar_init(bar(sm->seg_empty[s]), 14); }
        mbar_init(bar(sm->o_full), 2); mbar_init(bar(sm->o_empty), 8); mbar_init(bar(sm->ml_full), 8); mbar_init(bar(sm->part_full), 8); mbar_init(bar(sm->last_full), 1);
        for (int s = 0; s < 4; ++s) mbar_init(bar(sm->drain[s]), 1);
        for (int s = 0; s < 8; ++s) mbar_init(bar(sm->turn[s >> 2][s & 3]), 1);
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
    const uint32_t tS = tmem, tO = tmem + 256;   // S of slot s at 128 s, two of 64 columns, P over either; O at 256 + 128 s
    int issued = 0;                              // tiles copied (copying warps; read again before the end)

    // warps 0: rows of no window; 1: the walk and keys; 2, 3: S of the slots; 4: scales; 5, 6: O of the slots; 7: values
    if (warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
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
                                      s[kSegKeys], s[kSegHead], ring_k, bar(sm->k_full[0]), bar(sm->k_empty[0]), kK, flag, lane, rg, issued);
            }
        } else {
            const int slot = warp == 3 || warp == 6 ? 1 : 0;
            A8Ring rg, done;                     // (done: of scales)
            uint32_t used = 0;                   // jobs of this slot so far
            bool ok = warp != 7 || static_cast<int>(me) != p.stalled;
            for (int item = 0; ok; ++item) {
                const int qi = item & (kSegQueue - 1);
                ok = a8_wait<0>(bar(sm->seg_full[qi]), static_cast<uint32_t>(item / kSegQueue) & 1u, flag);
                if (!ok) break;
                const int* const sg = sm->queue[qi];
                const int tiles = __shfl_sync(0xffffffffu, sg[kSegJobs], 0);         // (the compiler then knows it uniform)
                if (tiles == 0) break;
                const bool paired = __shfl_sync(0xffffffffu, sg[kSegPaired], 0) != 0;
                const int t0 = __shfl_sync(0xffffffffu, sg[kSegT0], 0), t1 = __shfl_sync(0xffffffffu, sg[kSegT1], 0);
                if (warp == 7) {
                    ok = a8_load_tiles<D>(p, &tmV, sg[kSegReq], attn_page(p, sg[kSegReq], t0, t1, sg[kSegKeys], lane), t0, t1, sg[kSegKeys], sg[kSegHead],
                                          ring_v, bar(sm->v_full[0]), bar(sm->v_empty[0]), kV, flag, lane, rg, issued);
                } else if (warp == 4) {
                    ok = a8_scales(p, sg[kSegReq], sg[kSegHead], t0, t1, sg[kSegKeys], ring_sc, sm, flag, lane, rg, done);
                } else {
                    // ------------------------------------------------ MMA: a warp per slot and product.  Job n of a slot in a stretch: split: keys 64
                    // slot .. of tile n; paired: keys 64 (n & 1) .. of tile n / 2.
                    const bool second = warp > 4;
                    const uint32_t sS = tS + slot * 128, sO = tO + slot * 128;
                    const int J = paired ? 2 * tiles : tiles;
                    ok = second ? item == 0 || a8_wait<0>(bar(sm->o_empty), static_cast<uint32_t>(item - 1) & 1u, flag)      // the previous O has been read
                                : a8_wait<0>(bar(sm->q_full[slot]), static_cast<uint32_t>(item) & 1u, flag);
                    for (int n = 0; ok && n < J; ++n, ++used) {
                        const uint32_t h = used & 1u, ph = (used >> 1) & 1u;
                        const bool first_use = !paired || (n & 1) == 0, last_use = !paired || (n & 1) == 1;
                        const uint32_t keys_at = (paired ? (n & 1) : slot) * (kAttnSub * D);
                        if (!second) {
                            ok = a8_wait<0>(bar(sm->s_free[2 * h + slot]), ph ^ 1u, flag);
                            if (ok && first_use) ok = a8_wait<0>(bar(sm->k_full[rg.s]), rg.ph, flag);
                            if (!ok) break;
                            tc_fence_after();
                            if (elect_one()) {
                                const uint64_t a0 = a8_desc(q_buf + slot * kQ, D, 16), b0 = a8_desc(ring_k + rg.s * kTile + keys_at, D, 16);
#pragma unroll
                                for (int q = 0; q < NP; ++q) {
#pragma unroll
                                    for (int k = 0; k < D / 32; ++k)
                                        umma_f8(sS + h * kAttnSub, a0 + 2 * k + q * (kAttnTile * D / 16), b0 + 2 * k, r8_idesc(kAttnSub, false, q == NP - 1), q != 0 || k != 0);
                                }
                                umma_commit(bar(sm->s_full[2 * h + slot]));
                                if (last_use) umma_commit(bar(sm->k_empty[rg.s]));
                            }
                        } else {
                            if (first_use) ok = a8_wait<0>(bar(sm->v_full[rg.s]), rg.ph, flag);
                            if (ok) ok = a8_wait<0>(bar(sm->p_full[2 * h + slot]), ph, flag);
                            if (!ok) break;
                            tc_fence_after();
                            if (elect_one()) {
                                const uint64_t b0 = a8_desc(ring_v + rg.s * kTile + keys_at, D, 8192);
#pragma unroll
                                for (int q = 0; q < NP; ++q) {
#pragma unroll
                                    for (int k = 0; k < kAttnSub / 32; ++k)
                                        umma_f8_ts(sO, sS + h * kAttnSub + q * 16 + k * 8, b0 + k * (32 * D / 16), r8_idesc(D, true, q == NP - 1),
                                                   (n != 0 || q != 0 || k != 0) ? 1u : 0u);          // a slot's first job overwrites O
                                }
                                umma_commit(bar(sm->s_free[2 * h + slot]));
                                if (last_use) umma_commit(bar(sm->v_empty[rg.s]));
                                if (n + 1 == J) umma_commit(bar(sm->o_full));
                            }
                        }
                        __syncwarp();
                        if (last_use) rg.step(second ? kV : kK, 1);
                    }
                }
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(bar(sm->seg_empty[qi]));
            }
            if (warp == 4) cp_async_wait_all();
        }
    } else {
        // ---------------------------------------------------------------- softmax: four warps per slot, a thread per row
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int slot = (warp - 8) >> 2, quad = warp & 3;
        const int row = quad * 32 + lane;        // row of the tile = TMEM lane
        const uint32_t lane_off = static_cast<uint32_t>(quad * 32) << 16;
        const uint32_t aS0 = tS + slot * 128 + lane_off, aO = tO + slot * 128 + lane_off;
        uint32_t used = 0;                       // jobs of this slot so far
        uint32_t splits = 0;                     // stretches of shared items so far
        A8Ring rv, rsc;                          // of values, of scales
        bool ok = true;
        for (int item = 0; ok; ++item) {
            const int* const sg = sm->queue[item & (kSegQueue - 1)];
            ok = a8_wait<0>(bar(sm->seg_full[item & (kSegQueue - 1)]), static_cast<uint32_t>(item / kSegQueue) & 1u, flag);
            if (!ok) break;
            if (__shfl_sync(0xffffffffu, sg[kSegJobs], 0) == 0) break;
            const bool paired = sg[kSegPaired];
            const int J = paired ? 2 * sg[kSegJobs] : sg[kSegJobs];
            const int tile_rows = paired && slot ? sg[kSegRows1] : sg[kSegRows0];
            const bool warp_has_rows = quad * 32 < tile_rows, valid = row < tile_rows;
            // ---- queries (the products that read the last ones are complete: their S has been waited for)
            r8_cut_queries<E, D>(p, sg[kSegRow] + (paired && slot ? p.tpt : 0), sg[kSegHead], tile_rows, q_buf + slot * kQ, sm->rs[slot], quad, lane);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm->q_full[slot]));
            const float rs = sm->rs[slot][row];
            const uint64_t rs2 = pair(rs, rs);
            const int key0 = sg[kSegT0] * kAttnTile + (paired ? 0 : slot * kAttnSub);
            const int step = paired ? kAttnSub : 2 * kAttnSub;                       // keys from one job of the slot to its next
            // columns of the job's keys past `cut` are masked for this row, rows of V from `have` on do not exist
            int cut = sg[kSegLimit] + attn_token(p, row) + (paired && slot ? p.tpt : 0) - key0;
            int have = sg[kSegKeys] - key0;
            float m = -CUDART_INF_F, l = 0.0f;
            for (int n = 0; n < J; ++n) {
                const uint32_t h = used & 1u;
                const int sub = paired ? n & 1 : slot;
                const bool first_use = !paired || sub == 0, last_use = !paired || sub == 1;
                if (first_use) {
                    ok = a8_wait<0>(bar(sm->sc_full[rsc.s]), rsc.ph, flag);
                    if (!ok) break;
                }
                ok = a8_wait<0>(bar(sm->s_full[2 * h + slot]), (used >> 1) & 1u, flag);
                if (!ok) break;
                tc_fence_after();
                const uint32_t aS = aS0 + h * kAttnSub, sc = ring_sc + rsc.s * kA8ScaleBytes + sub * (kAttnSub * 4);
                uint32_t sr[kAttnSub];
                float* const s = reinterpret_cast<float*>(sr);
                if (warp_has_rows) {
                    float base_m = 0.0f;
                    tmem_ld32(aS, sr);
                    tmem_ld32(aS + 32, sr + 32);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < kAttnSub; c += 2) {
                        const uint64_t t = fma2(mul2(pair(s[c], s[c + 1]), lds_pair(sc + c * 4)), rs2, lds_pair(sc + 512 + c * 4));
                        s[c] = low(t);
                        s[c + 1] = high(t);
                    }
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
                    const float mt = max3_nan(max3_nan(mx[0], mx[1], s[60]), max3_nan(mx[2], mx[3], s[61]), max3_nan(s[62], s[63], s[63]));
                    if (!(mt < CUDART_INF_F)) l = CUDART_NAN_F;                      // a score of NaN or +inf
                    const bool grow = valid && mt > m + 8.0f;
                    if (__any_sync(0xffffffffu, grow)) {
                        const float m_new = grow ? mt : m;
                        const float a = grow ? attn_ex2(m - m_new) : 1.0f;
                        l *= a;
                        m = m_new;
                        if (n > 0) {
                            // O holds the jobs up to the last but one for certain; its rescaling waits for that one too
                            ok = a8_wait<0>(bar(sm->s_free[2 * (h ^ 1u) + slot]), ((used - 1) >> 1) & 1u, flag);
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
                    // The slots' warps on a scheduler take turns at the exponentials (both have the same number of jobs): together they would queue for
                    // the special-function unit and leave it idle together.  (2 x 2048 rows 668 -> 612 us, 65 rows 168 -> 155.)
                    ok = a8_wait<0>(bar(sm->turn[slot][quad]), (used & 1u) ^ (slot ? 0u : 1u), flag);
                    if (!ok) break;
                    const uint64_t base2 = pair(base_m, base_m);
                    uint64_t sum[2] = {0, 0};
                    uint32_t pk[NP][16];
#pragma unroll
                    for (int c = 0; c < kAttnSub; c += 4) {
                        uint64_t y[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint64_t x = add2(pair(s[c + 2 * i], s[c + 2 * i + 1]), base2);
                            y[i] = pair(attn_ex2(low(x)), attn_ex2(high(x)));
                            sum[i] = fma2(y[i], lds_pair(sc + 1024 + (c + 2 * i) * 4), sum[i]);
                        }
                        uint32_t e[NP];
                        r8_cut<NP, NP == 3>(low(y[0]), high(y[0]), low(y[1]), high(y[1]), e);
#pragma unroll
                        for (int q = 0; q < NP; ++q) pk[q][c / 4] = e[q];
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(sm->turn[slot ^ 1][quad]));
#pragma unroll
                    for (int q = 0; q < NP; ++q) tmem_st16(aS + q * 16, pk[q]);
                    const uint64_t both = add2(sum[0], sum[1]);
                    l += low(both) + high(both);
                    tmem_wait_st();
                }
                if (!warp_has_rows) {
                    ok = a8_wait<0>(bar(sm->turn[slot][quad]), (used & 1u) ^ (slot ? 0u : 1u), flag);
                    if (!ok) break;
                    if (lane == 0) mbar_arrive(bar(sm->turn[slot ^ 1][quad]));
                    __syncwarp();
                }
                if (have < kAttnSub) {
                    // V behind the last key is cleared.  (Both slots of a paired item do: whoever comes second writes zeros over zeros.  The
                    // stage cannot be recycled before this job's second product.)
                    ok = a8_wait<0>(bar(sm->v_full[rv.s]), rv.ph, flag);
                    if (!ok) break;
                    for (int i = row + max(have, 0) * (D / 16); i < kAttnSub * (D / 16); i += 128)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ring_v + rv.s * kTile + sub * (kAttnSub * D) + i * 16), "r"(0) : "memory");
                    fence_proxy_async();
                }
                tc_fence_before();
                __syncwarp();
                a8_arrive<0>(bar(sm->p_full[2 * h + slot]), lane);
                if (last_use) a8_arrive<0>(bar(sm->sc_empty[rsc.s]), lane);
                if (last_use) { rsc.step(kA8Scales, 1); rv.step(kV, 1); }
                cut -= step;
                have -= step;
                ++used;
            }
            if (!ok) break;

            // ---- the item (or its stretch) is done once O is complete (which also says that nobody reads the previous
            // stretch's m and l any more).  The slots' (m, l) are exchanged: a split item is put together here from both
            // accumulators, each slot taking half of the columns.
            ok = a8_wait<0>(bar(sm->o_full), static_cast<uint32_t>(item) & 1u, flag);
            if (!ok) break;
            tc_fence_after();
            if (m == -CUDART_INF_F && l == l) l = 0.0f;                              // the row has seen no key (and no NaN)
            sm->ml[slot][row] = make_float2(m, l);
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm->ml_full));
            ok = a8_wait<0>(bar(sm->ml_full), static_cast<uint32_t>(item) & 1u, flag);
            if (!ok) break;
            if (warp_has_rows) {
                float wa = 1.0f, wb = 0.0f;      // weights of this slot's accumulator and of the other one's
                if (!paired) {
                    const float2 o = sm->ml[slot ^ 1][row];
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
            if (lane == 0) mbar_arrive(bar(sm->o_empty));
            if (sg[kSegParts] > 1) {
                // The item is shared: count this block's part, and if it is the last one to arrive, add all of them.  (One
                // thread's fences stand for the block: the barriers before and after order the others' writes and reads.)
                const int first_block = sg[kSegFirst], parts = sg[kSegParts];
                if (lane == 0) mbar_arrive(bar(sm->part_full));
                if (warp == 8) {
                    ok = a8_wait<0>(bar(sm->part_full), splits & 1u, flag);
                    if (!ok) break;
                    if (lane == 0) {
                        const int shift = sg[kSegShift];
                        __threadfence();
                        const int before = static_cast<int>(static_cast<unsigned>(atomicAdd(p.count + first_block, 1 << shift)) >> shift & 0xffffu);
                        sm->came_last = before == parts - 1;
                        __threadfence();
                        mbar_arrive(bar(sm->last_full));
                        if (before == parts - 1) p.count[first_block] = 0;               // (nobody counts in the other half)
                    }
                    __syncwarp();
                }
                ok = a8_wait<0>(bar(sm->last_full), splits & 1u, flag);
                if (!ok) break;
                ++splits;
                if (__shfl_sync(0xffffffffu, *const_cast<volatile int32_t*>(&sm->came_last), 0)) attn_merge<E, D>(p, sg, warp - 8, lane);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sm->seg_empty[item & (kSegQueue - 1)]));
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
            const int n = warp == 1 ? kK : kV;
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
