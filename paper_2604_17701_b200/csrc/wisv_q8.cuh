// Quantising keys and values as they are written into the cache, and reading them back.
//
// A head of a token is e4m3 codes and one fp32 scale: with T = max |x| over its D elements, scale = T / 448 and
// code = 448 x / T rounded to the nearest e4m3 number, ties to even.  The kernel gets that rounding exactly although it
// multiplies by an fp32 reciprocal: x and T have at most 11 bits, so a quotient 448 x / T is either on the border between two codes or at
// least 2^-16 of itself away from it, while x * (448 / T) in fp32 is off by at most 2^-23.  Rounding the product to 21 bits puts it
// on the border where it belongs there, and moves no other across.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include "wisv_attn8.cuh"

namespace wisv {

constexpr int kQ8Threads = 128;

struct Q8Pages {                                  // strides in 16-byte pieces of codes, in floats of scales
    uint4 *k, *v;
    float *ks, *vs;
    int64_t kp, kt, kh, vp, vt, vh, ksp, ksh, vsp, vsh;
    int64_t n_slots;
    int32_t page_shift;
};

struct Q8AppendParams {
    Q8Pages pg;
    int32_t T, vecs;                              // vecs: pieces of 16 elements per token
    const uint4 *k, *v;                           // strides in 16-byte pieces (8 elements)
    int64_t kt, kh, vt, vh;
    const int64_t* slot_map;
};

// 16 elements of a head that L lanes hold: their codes; returns the scale.  A head with an infinite element or NaN has the scale NaN and
// codes of 0.
template <typename E, int L>
__device__ __forceinline__ float q8_codes(const uint4 (&w)[2], uint4& out)
{
    const uint32_t* v = reinterpret_cast<const uint32_t*>(w);
    // the largest magnitude: 16-bit numbers without their sign order as whole numbers, infinity and NaN last
    uint32_t two = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) two = __vmaxu2(two, v[i] & 0x7fff7fffu);
    uint32_t top = max(two >> 16, two & 0xffffu);
#pragma unroll
    for (int o = 1; o < L; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const bool fine = top < (is_bf16<E>::value ? 0x7f80u : 0x7c00u);
    float t, none;
    unpack2<E>(top, t, none);
    out = make_uint4(0, 0, 0, 0);
    if (fine && top != 0) {
        // (below 2^-100 both are scaled by 2^64, which is exact, so that the reciprocal stays finite)
        const bool tiny = t < 7.888609e-31f;
        const float inv = __fdiv_rn(448.0f, tiny ? t * 1.8446744e19f : t);
        uint32_t c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[4];
            unpack2<E>(v[2 * i], x[0], x[1]);
            unpack2<E>(v[2 * i + 1], x[2], x[3]);
            if (tiny) {
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] *= 1.8446744e19f;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = __uint_as_float((__float_as_uint(x[k] * inv) + 4u) & ~7u);
            asm("{\n\t"
                ".reg .b16 e0, e1;\n\t"
                "cvt.rn.satfinite.e4m3x2.f32 e0, %2, %1;\n\t"
                "cvt.rn.satfinite.e4m3x2.f32 e1, %4, %3;\n\t"
                "mov.b32 %0, {e0, e1};\n\t"
                "}"
                : "=r"(c[i]) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]));
        }
        out = make_uint4(c[0], c[1], c[2], c[3]);
    }
    return fine ? __fdiv_rn(t, 448.0f) : CUDART_NAN_F;
}

// One thread takes 16 elements of a key row and the same 16 of the value row; D / 16 lanes share a head and find its maximum by
// shuffles.  A stream of 6 bytes per element of K and V: 8192 rows of 8 x 128 (51 MB) in 11.4 us, 4.5 TB/s with the launch, of which 3 us, and some
// 6 instructions an element; a window of 9 rows 1.8 us, the launch.
template <typename E, int D>
__global__ void __launch_bounds__(kQ8Threads) append_q8_kernel(const Q8AppendParams p)
{
    constexpr int L = D / 16;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kQ8Threads + threadIdx.x;
    const int64_t t = i / p.vecs;
    griddep_wait();
    griddep_launch_dependents();
    const int x = static_cast<int>(i - t * p.vecs), h = x / L, e = x % L;
    int64_t slot = -1;
    uint4 k[2], v[2];
    k[0] = k[1] = v[0] = v[1] = make_uint4(0, 0, 0, 0);
    if (t < p.T) {                                                // (the rows are read whatever the slot, which comes beside them)
        slot = p.slot_map[t];
        const uint4* a = p.k + t * p.kt + h * p.kh + 2 * e;
        const uint4* b = p.v + t * p.vt + h * p.vh + 2 * e;
        k[0] = a[0]; k[1] = a[1];
        v[0] = b[0]; v[1] = b[1];
    }
    uint4 kc, vc;
    const float ks = q8_codes<E, L>(k, kc), vs = q8_codes<E, L>(v, vc);
    if (slot < 0 || slot >= p.pg.n_slots) return;
    const int64_t pg = slot >> p.pg.page_shift, o = slot & ((1 << p.pg.page_shift) - 1);
    p.pg.k[pg * p.pg.kp + o * p.pg.kt + h * p.pg.kh + e] = kc;
    p.pg.v[pg * p.pg.vp + o * p.pg.vt + h * p.pg.vh + e] = vc;
    if (e == 0) p.pg.ks[pg * p.pg.ksp + h * p.pg.ksh + o] = ks;
    if (e == 1) p.pg.vs[pg * p.pg.vsp + h * p.pg.vsh + o] = vs;
}

// ---------------------------------------------------------------- reading back
struct Q8ReadParams {
    Q8Pages pg;
    int32_t B, T, vecs, tokens;                   // tokens: of a block
    int32_t uniform, max_blocks, n_pages, clear_rest;
    const int32_t *off, *start, *block_table;
    int64_t table_stride;
    uint4 *k, *v;                                 // strides in 16-byte pieces (8 elements)
    int64_t kt, kh, vt, vh;
};

constexpr int kQ8ReadTokens = 64;                 // of a block, at most

// Row t is token start[b] + t - off[b] of request b: its slot, -1 where there is none (zeros), -2 for a row of no request.  Found by one
// warp, which tests 32 offsets at a time.
__device__ __forceinline__ int64_t q8_slot(const Q8ReadParams& p, int t, int lane)
{
    int b, i;
    if (p.off) {
        if (p.off[0] > t) return -2;
        int lo = 0, n = p.B + 1;                  // the last offset that is at most t is one of n from lo on
        while (n > 1) {
            const int step = (n + 31) / 32, at = (lane + 1) * step;
            const int c = __popc(__ballot_sync(0xffffffffu, at < n && p.off[lo + at] <= t));
            lo += c * step;
            n = min(step, n - c * step);
        }
        if (lo >= p.B) return -2;
        b = lo;
        i = t - p.off[b];
    } else {
        b = t / p.uniform;
        i = t - b * p.uniform;
    }
    const int64_t pos = (p.start ? static_cast<int64_t>(p.start[b]) : 0) + i;
    if (pos < 0 || pos >= static_cast<int64_t>(p.max_blocks) << p.pg.page_shift) return -1;
    const int pg = p.block_table[b * p.table_stride + (pos >> p.pg.page_shift)];
    if (pg < 0 || pg >= p.n_pages) return -1;
    return (static_cast<int64_t>(pg) << p.pg.page_shift) + (pos & ((1 << p.pg.page_shift) - 1));
}

template <typename E>
__device__ __forceinline__ void q8_values(uint4 codes, float scale, uint4 (&out)[2])
{
    const uint32_t c[4] = {codes.x, codes.y, codes.z, codes.w};
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(c[i / 2] >> (16 * (i & 1)))));
        float a, b;
        unpack2<__half>(h, a, b);
        r[i] = pack2<E>(a * scale, b * scale);
    }
    out[0] = make_uint4(r[0], r[1], r[2], r[3]);
    out[1] = make_uint4(r[4], r[5], r[6], r[7]);
}

// A block first finds the slots of its rows, a warp at a time, then streams: a thread turns 16 codes of keys and 16 of values.  code *
// scale in fp32, rounded once to the cache's type.  Bound by HBM (3 bytes an element: 64 prefixes of 137 k tokens, 854 MB, in 140 us, 6.1 TB/s), for one
// request by its chain of lookups (709 tokens 3.4 us).
template <typename E, int D>
__global__ void __launch_bounds__(kQ8Threads) read_q8_kernel(const Q8ReadParams p)
{
    constexpr int L = D / 16;
    __shared__ int64_t slots[kQ8ReadTokens];
    const int t0 = blockIdx.x * p.tokens, n = min(p.tokens, p.T - t0);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    griddep_wait();
    griddep_launch_dependents();
    for (int j = warp; j < n; j += kQ8Threads / 32) {
        const int64_t s = q8_slot(p, t0 + j, lane);
        if (lane == 0) slots[j] = s;
    }
    __syncthreads();
    constexpr int U = 2;
    const int total = n * p.vecs;
    for (int i0 = threadIdx.x; i0 < total; i0 += U * kQ8Threads) {
        uint4 kc[U], vc[U];
        float ks[U], vs[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * kQ8Threads, j = min(i, total - 1) / p.vecs, x = min(i, total - 1) - j * p.vecs, h = x / L, e = x % L;
            const int64_t slot = slots[j];
            kc[u] = vc[u] = make_uint4(0, 0, 0, 0);
            ks[u] = vs[u] = 0.0f;
            if (i < total && slot >= 0) {
                const int64_t pg = slot >> p.pg.page_shift, o = slot & ((1 << p.pg.page_shift) - 1);
                kc[u] = p.pg.k[pg * p.pg.kp + o * p.pg.kt + h * p.pg.kh + e];
                vc[u] = p.pg.v[pg * p.pg.vp + o * p.pg.vt + h * p.pg.vh + e];
                ks[u] = p.pg.ks[pg * p.pg.ksp + h * p.pg.ksh + o];
                vs[u] = p.pg.vs[pg * p.pg.vsp + h * p.pg.vsh + o];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * kQ8Threads;
            if (i >= total) break;
            const int j = i / p.vecs, x = i - j * p.vecs, h = x / L, e = x % L;
            if (slots[j] == -2 && !p.clear_rest) continue;
            const int64_t t = t0 + j;
            uint4 a[2], b[2];
            q8_values<E>(kc[u], ks[u], a);
            q8_values<E>(vc[u], vs[u], b);
            uint4* const kd = p.k + t * p.kt + h * p.kh + 2 * e;
            uint4* const vd = p.v + t * p.vt + h * p.vh + 2 * e;
            kd[0] = a[0]; kd[1] = a[1];
            vd[0] = b[0]; vd[1] = b[1];
        }
    }
}

}  // namespace wisv
