// wisv_verify_residual: accept drafted tokens against the target's probabilities (Eq. 1) and draw the correction token from
// the residual max(P - Q, 0) (Eq. 2), or the bonus token from P.
//
// One cluster of thread blocks per request, one launch, no workspace.  Every block of the cluster makes the acceptance
// test of the whole window (at most 64 pairs of gathered probabilities); that gives the ONE row of P, and of Q, which
// has to be read.  The row is cut into contiguous slices, one per warp of the cluster; a warp adds the weights of its
// slice, the blocks exchange their sums through distributed shared memory, and the one warp whose slice holds the goal reads its
// slice again (from L2) to find the token.  So the row crosses HBM once, and that is the bound: V (size(P) + size(Q))
// bytes per request.
//
// Weights are integers (2^-44 units, 64-bit sums): addition is exact in any order, so the token depends neither on the number
// of blocks nor on how the row was cut, and a row whose mass is spread over 2^18 tokens still leaves each token with
// the 24 bits that an fp32 probability of 2^-20 or more has.  A residual below 2^-44 has no weight; 2^18 of those would
// be 1.5e-8 of the mass, less than the rounding of one fp32 probability.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/wisv.h"
#include "wisv_ptx.cuh"

using namespace wisv;

namespace {

typedef unsigned long long u64;

constexpr int kResThreads = 512;
constexpr int kResWarps = kResThreads / 32;
constexpr int kResMaxCluster = 8;
constexpr float kFix = 17592186044416.0f;          // 2^44
constexpr int kQuiet = 0, kDense = 1, kTop = 2;    // the drafter's distribution: one token, dense, a list

struct ResidualParams {
    int32_t B, K, T, V, n_top, cluster;
    const int32_t* k_off;
    const void* P; int64_t p_stride;
    const void* Q; int64_t q_stride;
    const int32_t *ids, *tokens;
    const float *u, *u_draw;
    const int32_t* accept_in;
    int32_t *accept_len, *token, *status;
    float* mass;
};

__device__ __forceinline__ float as_f(float x) { return x; }
__device__ __forceinline__ float as_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_f(__half x) { return __half2float(x); }
// a probability as the draw sees it: NaN and negative values 0, at most 1
__device__ __forceinline__ float unit(float x) { return fminf(fmaxf(x, 0.0f), 1.0f); }
__device__ __forceinline__ u64 fix(float x) { return __float2ull_rz(x * kFix); }

// E consecutive elements from v on; E = 8 needs 16-byte aligned rows.  Elements past V are 0.
template <typename T, int E>
__device__ __forceinline__ void load_probs(const T* row, int v, int V, float (&x)[E])
{
    if (E == 8 && v + 8 <= V) {
        uint4 w[sizeof(T) / 2];
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) w[i] = __ldg(reinterpret_cast<const uint4*>(row + v) + i);
        const T* e = reinterpret_cast<const T*>(w);
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = unit(as_f(e[i]));
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = v + i < V ? unit(as_f(row[v + i])) : 0.0f;
    }
}

__device__ __forceinline__ u64 warp_sum(u64 x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

__device__ __forceinline__ void st_cluster_u64(uint32_t addr, u64 x)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(x) : "memory");
}

template <typename TP, typename TQ, int kForm, int E>
__global__ void __launch_bounds__(kResThreads) residual_kernel(const ResidualParams p)
{
    __shared__ u64 warp_mass[kResWarps];
    __shared__ u64 block_mass[2][kResMaxCluster];          // written by every block of the cluster
    __shared__ unsigned ok_bits[2];
    __shared__ int flag;
    __shared__ int list_v[kForm == kTop ? WISV_MAX_TOP : 1];
    __shared__ float list_q[kForm == kTop ? WISV_MAX_TOP : 1];
    __shared__ long long list_d[kForm == kTop ? WISV_MAX_TOP : 1];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = static_cast<int>(cluster_ctarank());
    const int b = blockIdx.x / p.cluster;
    if (tid == 0) { ok_bits[0] = ok_bits[1] = 0; flag = 0; }
    cluster_arrive();                                      // waited for before the first store to another block

    // ---- the window: offsets come from the device, so every index made of them is clamped
    int t0, K;
    if (p.k_off) {
        t0 = min(max(p.k_off[b], 0), p.T);
        K = min(max(p.k_off[b + 1], 0), p.T) - t0;
        if (tid == 0 && (K < 0 || K > WISV_MAX_K)) flag = WISV_ST_BAD_WINDOW;
        K = min(max(K, 0), WISV_MAX_K);
    } else {
        K = p.K; t0 = b * K;
    }
    const TP* P0 = static_cast<const TP*>(p.P) + static_cast<int64_t>(t0 + b) * p.p_stride;
    auto draft_at = [&](int i) {
        const int y = p.tokens[t0 + i];
        if (y < 0 || y >= p.V) atomicOr(&flag, WISV_ST_BAD_TOKEN);
        return min(max(y, 0), p.V - 1);
    };
    __syncthreads();

    int A;
    if (p.accept_in) {
        A = min(max(p.accept_in[b], 0), K);
    } else {
        if (kForm == kTop) {
            for (int i = warp; i < K; i += kResWarps) {    // a warp looks one token up in its list
                const int y = draft_at(i);
                float q = 0.0f;
                for (int j = lane; j < p.n_top; j += 32) {
                    const int64_t at = static_cast<int64_t>(t0 + i) * p.n_top + j;
                    if (p.ids[at] == y) q += static_cast<const float*>(p.Q)[static_cast<int64_t>(t0 + i) * p.q_stride + j];
                }
#pragma unroll
                for (int o = 16; o; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
                q = unit(q);
                const float a = unit(as_f(P0[static_cast<int64_t>(i) * p.p_stride + y]));
                const bool ok = p.u[t0 + i] < (q > 0.0f ? fminf(a / q, 1.0f) : (a > 0.0f ? 1.0f : 0.0f));
                if (lane == 0 && ok) atomicOr(&ok_bits[i >> 5], 1u << (i & 31));
            }
        } else if (tid < K) {
            const int y = draft_at(tid);
            const float a = unit(as_f(P0[static_cast<int64_t>(tid) * p.p_stride + y]));
            const float q = kForm == kDense
                                ? unit(as_f(static_cast<const TQ*>(p.Q)[static_cast<int64_t>(t0 + tid) * p.q_stride + y]))
                                : 1.0f;
            if (p.u[t0 + tid] < (q > 0.0f ? fminf(a / q, 1.0f) : (a > 0.0f ? 1.0f : 0.0f)))
                atomicOr(&ok_bits[tid >> 5], 1u << (tid & 31));
        }
        __syncthreads();
        const u64 ok = (static_cast<u64>(ok_bits[1]) << 32) | ok_bits[0];
        A = min(ok == ~0ull ? 64 : __ffsll(static_cast<long long>(~ok)) - 1, K);
    }

    const TP* P = P0 + static_cast<int64_t>(A) * p.p_stride;
    const TQ* Q = kForm == kDense ? static_cast<const TQ*>(p.Q) + static_cast<int64_t>(t0 + A) * p.q_stride : nullptr;
    const int y = A < K ? draft_at(A) : -1;
    const int m = static_cast<int>(fminf(unit(p.u_draw[b]) * 2147483648.0f, 2147483520.0f));

    // ---- slices: a warp owns `per` consecutive elements, a multiple of 32 * E
    const int warps = p.cluster * kResWarps;
    const int per = (p.V + warps * 32 * E - 1) / (warps * 32 * E) * (32 * E);
    const int64_t at0 = static_cast<int64_t>(rank * kResWarps + warp) * per;
    const int v0 = static_cast<int>(at0 < p.V ? at0 : p.V), v1 = min(v0 + per, p.V);

    for (int pass = 0; pass < 2; ++pass) {
        const bool rest = pass == 0 && A < K;              // the residual; then (or at once, for a bonus token) P alone
        auto weights = [&](int v, u64 (&w)[E]) {
            float a[E];
            load_probs<TP, E>(P, v, p.V, a);
            if (kForm == kDense && rest) {
                float q[E];
                load_probs<TQ, E>(Q, v, p.V, q);
#pragma unroll
                for (int i = 0; i < E; ++i) a[i] = fmaxf(a[i] - q[i], 0.0f);
            }
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (kForm == kQuiet && rest && v + i == y) a[i] = fmaxf(a[i] - 1.0f, 0.0f);
                w[i] = fix(a[i]);
            }
        };
        u64 sum = 0;
        constexpr int U = E == 8 ? 2 : 8;
        for (int v = v0 + lane * E; v < v1; v += 32 * E * U) {
            u64 w[U][E];
#pragma unroll
            for (int s = 0; s < U; ++s) {
                const int x = v + s * 32 * E;
                if (x < v1) weights(x, w[s]);
                else {
#pragma unroll
                    for (int i = 0; i < E; ++i) w[s][i] = 0;
                }
            }
#pragma unroll
            for (int s = 0; s < U; ++s)
#pragma unroll
                for (int i = 0; i < E; ++i) sum += w[s][i];
        }
        sum = warp_sum(sum);
        if (lane == 0) warp_mass[warp] = sum;
        if (kForm == kTop && rest) {
            // the listed tokens' weights, taken with Q = 0 above, are corrected by integers
            for (int j = tid; j < p.n_top; j += kResThreads) {
                const int v = p.ids[static_cast<int64_t>(t0 + A) * p.n_top + j];
                list_v[j] = v >= 0 && v < p.V ? v : -1;
                list_q[j] = static_cast<const float*>(p.Q)[static_cast<int64_t>(t0 + A) * p.q_stride + j];
            }
            __syncthreads();
            for (int j = tid; j < p.n_top; j += kResThreads) {
                const int v = list_v[j];
                float q = 0.0f;
                bool head = v >= 0;                        // the first entry of a token stands for all of them
                for (int k = 0; k < p.n_top; ++k)
                    if (list_v[k] == v) { if (k < j) head = false; q += list_q[k]; }
                long long d = 0;
                const int64_t slice = head ? v / per : -1;
                if (head) {
                    const float a = unit(as_f(P[v]));
                    d = static_cast<long long>(fix(fmaxf(a - unit(q), 0.0f))) - static_cast<long long>(fix(a));
                }
                list_d[j] = d;
                if (slice / kResWarps == rank && head)
                    atomicAdd(&warp_mass[slice % kResWarps], static_cast<u64>(d));
            }
        }
        __syncthreads();
        if (pass == 0) cluster_wait();                     // every block of the cluster is running
        if (warp == 0) {
            u64 x = lane < kResWarps ? warp_mass[lane] : 0;
            x = warp_sum(x);
            if (lane < p.cluster) st_cluster_u64(mapa_u32(smem_u32(&block_mass[pass][rank]), lane), x);
        }
        cluster_arrive();
        cluster_wait();
        u64 W = 0, before = 0;
        for (int r = 0; r < p.cluster; ++r) {
            if (r < rank) before += block_mass[pass][r];
            W += block_mass[pass][r];
        }
        if (W == 0 && rest) continue;                      // the same in every block
        if (rank == 0 && tid == 0) {
            p.accept_len[b] = A;
            if (p.mass) p.mass[b] = static_cast<float>(W) * (1.0f / kFix);
            if (p.status) p.status[b] = flag | (W == 0 ? WISV_ST_NO_MASS : 0);
            if (W == 0) p.token[b] = -1;
        }
        if (W == 0) break;
        const u64 mm = static_cast<u64>(m);
        const u64 goal = (W >> 31) * mm + (((W & 0x7fffffffull) * mm) >> 31);
        for (int k = 0; k < warp; ++k) before += warp_mass[k];
        if (goal < before || goal >= before + warp_mass[warp]) break;
        // ---- this warp's slice holds the goal: 32 * E elements at a time
        for (int v = v0; v < v1; v += 32 * E) {
            u64 w[E];
            const int mine = v + lane * E;
            if (mine < v1) weights(mine, w);
            else {
#pragma unroll
                for (int i = 0; i < E; ++i) w[i] = 0;
            }
            if (kForm == kTop && rest) {
                for (int j = 0; j < p.n_top; ++j) {
                    const int x = list_v[j] - mine;
#pragma unroll
                    for (int i = 0; i < E; ++i) if (x == i) w[i] += static_cast<u64>(list_d[j]);
                }
            }
            u64 s = 0;
#pragma unroll
            for (int i = 0; i < E; ++i) s += w[i];
            u64 upto = s;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 z = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += z;
            }
            const unsigned past = __ballot_sync(0xffffffffu, before + upto > goal);
            if (past) {
                if (lane == __ffs(past) - 1) {
                    u64 c = before + upto - s;
                    int tok = -1;
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        c += w[i];
                        if (tok < 0 && c > goal) tok = mine + i;
                    }
                    p.token[b] = tok;
                }
                break;
            }
            before += __shfl_sync(0xffffffffu, upto, 31);
        }
        break;
    }
}

template <typename TP, typename TQ, int kForm, int E>
int go(const ResidualParams& p, cudaStream_t st)
{
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)(p.B * p.cluster));
    cfg.blockDim = dim3(kResThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, residual_kernel<TP, TQ, kForm, E>, p) != cudaSuccess) {
        (void)cudaGetLastError();
        return WISV_ECUDA;
    }
    return WISV_OK;
}

template <typename TP, int E>
int by_form(const wisv_residual* r, const ResidualParams& p, cudaStream_t st)
{
    if (!r->draft_probs) return go<TP, float, kQuiet, E>(p, st);
    if (r->draft_ids) return go<TP, float, kTop, E>(p, st);
    switch (r->draft_dtype) {
        case WISV_DT_F32: return go<TP, float, kDense, E>(p, st);
        case WISV_DT_BF16: return go<TP, __nv_bfloat16, kDense, E>(p, st);
        default: return go<TP, __half, kDense, E>(p, st);
    }
}

template <int E>
int by_target(const wisv_residual* r, const ResidualParams& p, cudaStream_t st)
{
    switch (r->target_dtype) {
        case WISV_DT_F32: return by_form<float, E>(r, p, st);
        case WISV_DT_BF16: return by_form<__nv_bfloat16, E>(r, p, st);
        default: return by_form<__half, E>(r, p, st);
    }
}

bool known_dtype(int32_t d) { return d == WISV_DT_F32 || d == WISV_DT_BF16 || d == WISV_DT_F16; }
int size_of(int32_t d) { return d == WISV_DT_F32 ? 4 : 2; }
bool rows_aligned(const void* p, int64_t stride, int size, int to)
{
    return reinterpret_cast<uintptr_t>(p) % to == 0 && stride * size % to == 0;
}

}  // namespace

extern "C" int wisv_verify_residual(const wisv_residual* r, void* cuda_stream)
{
    if (!r || !known_dtype(r->target_dtype)) return WISV_EINVAL;
    if (r->B < 1 || r->T_total < 0 || r->V < 1 || r->V > WISV_STATIC_MAX_V || r->target_stride < r->V) return WISV_ESHAPE;
    if (!r->k_off && (r->K < 0 || r->K > WISV_MAX_K || (int64_t)r->B * r->K != r->T_total)) return WISV_ESHAPE;
    if ((int64_t)r->T_total + r->B > 0x7fffffffLL || (int64_t)r->B * kResMaxCluster > 0x7fffffffLL) return WISV_ESHAPE;
    if (!r->target_probs || !r->u_draw || !r->accept_len || !r->token) return WISV_EINVAL;
    if (r->T_total > 0 && (!r->draft_tokens || (!r->uniforms && !r->accept_in))) return WISV_EINVAL;
    if (r->draft_probs) {
        if (r->draft_ids) {
            if (r->n_top < 1 || r->n_top > WISV_MAX_TOP || r->draft_stride < r->n_top) return WISV_ESHAPE;
        } else {
            if (!known_dtype(r->draft_dtype)) return WISV_EINVAL;
            if (r->draft_stride < r->V) return WISV_ESHAPE;
        }
    } else if (r->draft_ids) {
        return WISV_EINVAL;
    }
    const bool dense = r->draft_probs && !r->draft_ids;
    const int ps = size_of(r->target_dtype), qs = dense ? size_of(r->draft_dtype) : 4;
    if (!rows_aligned(r->target_probs, 0, 1, ps) || (r->draft_probs && !rows_aligned(r->draft_probs, 0, 1, qs)))
        return WISV_EALIGN;
    int dev = 0, major = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return WISV_ECUDA;
    }
    if (major != 10) return WISV_EARCH;
    ResidualParams p;
    p.B = r->B; p.K = r->K; p.T = r->T_total; p.V = r->V; p.n_top = r->n_top;
    p.cluster = kResMaxCluster;
    p.k_off = r->k_off; p.P = r->target_probs; p.p_stride = r->target_stride;
    p.Q = r->draft_probs; p.q_stride = r->draft_stride; p.ids = r->draft_ids; p.tokens = r->draft_tokens;
    p.u = r->uniforms; p.u_draw = r->u_draw; p.accept_in = r->accept_in;
    p.accept_len = r->accept_len; p.token = r->token; p.status = r->status; p.mass = r->mass;
    const bool wide = rows_aligned(p.P, p.p_stride, ps, 16) && (!dense || rows_aligned(p.Q, p.q_stride, qs, 16));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return wide ? by_target<8>(r, p, st) : by_target<1>(r, p, st);
}
