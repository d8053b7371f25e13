// Attention of new tokens over the paged cache: one warp per (row, query head), 32 keys at a time.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "wisv_ptx.cuh"

namespace wisv {

struct AttnParams {
    int32_t B, T, max_new, n_heads, group, page_shift, n_pages, max_blocks;
    const int32_t *q_off, *kv_len, *block_table;
    int64_t table_stride;
    const void* q; int64_t qt, qh;
    const void *kp, *vp; int64_t kpp, kpt, kph, vpp, vpt, vph;
    void* out; int64_t ot, oh;
    float* lse;
    float scale;
};

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f(float x) { return __float2half_rn(x); }

template <typename E, int D>
__global__ void __launch_bounds__(128) attn_simple_kernel(const AttnParams p)
{
    __shared__ float qs[4][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + warp;
    if (item >= static_cast<int64_t>(p.T) * p.n_heads) return;
    const int t = static_cast<int>(item / p.n_heads), h = static_cast<int>(item % p.n_heads);
    int b = 0, lo = 0, n = p.max_new;
    if (p.q_off) {
        int l = 0, r = p.B;
        while (r - l > 1) { const int m = (l + r) >> 1; if (p.q_off[m] <= t) l = m; else r = m; }
        b = l; lo = p.q_off[b]; n = p.q_off[b + 1] - lo;
    } else {
        b = t / n; lo = b * n;
    }
    if (b >= p.B || t < lo || t >= lo + n) return;
    const E* q = static_cast<const E*>(p.q) + t * p.qt + h * p.qh;
    for (int e = lane; e < D; e += 32) qs[warp][e] = to_f(q[e]);
    __syncwarp();
    const int kv = min(max(p.kv_len[b], 0), p.max_blocks << p.page_shift);
    const int seen = max(kv - n + (t - lo) + 1, 0);
    const int kh = h / p.group;
    float m = -INFINITY, l = 0.0f, acc[D / 32] = {};
    for (int j0 = 0; j0 < seen; j0 += 32) {
        const int j = j0 + lane;
        float s = -INFINITY;
        int pg = -1;
        if (j < seen) {
            pg = p.block_table[b * p.table_stride + (j >> p.page_shift)];
            if (pg < 0 || pg >= p.n_pages) pg = -1;
            float x = 0.0f;
            if (pg >= 0) {
                const E* k = static_cast<const E*>(p.kp) + pg * p.kpp + (j & ((1 << p.page_shift) - 1)) * p.kpt + kh * p.kph;
                for (int e = 0; e < D; ++e) x = fmaf(qs[warp][e], to_f(k[e]), x);
            }
            s = x * p.scale;
        }
        float mx = s;
        for (int o = 16; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float mn = fmaxf(m, mx), c = m == -INFINITY ? 0.0f : exp2f((m - mn) * 1.4426950408889634f);
        const float w = j < seen ? exp2f((s - mn) * 1.4426950408889634f) : 0.0f;
        float ws = w;
        for (int o = 16; o; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
        l = l * c + ws; m = mn;
        for (int e = 0; e < D / 32; ++e) acc[e] *= c;
        for (int u = 0; u < 32 && j0 + u < seen; ++u) {
            const float wu = __shfl_sync(0xffffffffu, w, u);
            const int pu = __shfl_sync(0xffffffffu, pg, u);
            if (pu < 0) continue;
            const E* v = static_cast<const E*>(p.vp) + pu * p.vpp + ((j0 + u) & ((1 << p.page_shift) - 1)) * p.vpt + kh * p.vph;
            for (int e = 0; e < D / 32; ++e) acc[e] = fmaf(wu, to_f(v[e * 32 + lane]), acc[e]);
        }
    }
    E* o = static_cast<E*>(p.out) + t * p.ot + h * p.oh;
    for (int e = 0; e < D / 32; ++e) o[e * 32 + lane] = from_f<E>(seen ? acc[e] / l : 0.0f);
    if (p.lse && lane == 0) p.lse[static_cast<int64_t>(t) * p.n_heads + h] = seen ? m + logf(l) : -INFINITY;
}

}  // namespace wisv
