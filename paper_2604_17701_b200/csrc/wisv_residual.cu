// wisv_verify_residual: accept drafted tokens against the target's probabilities (Eq. 1) and draw the correction token from
// the residual max(P - Q, 0) (Eq. 2), or the bonus token from P.
//
// One cluster of thread blocks per request, one launch, no workspace.  Every block of the cluster makes the acceptance
// test of the whole window (at most 64 pairs of gathered probabilities); that gives the ONE row of P, and of Q, which
// has to be read.  The row is cut into chunks of 512 tokens; a warp adds up the weights of a chunk and keeps the sum in shared
// memory, the blocks exchange their totals through distributed shared memory, and the block whose chunks hold the
// goal scans its sums and reads that one chunk again (from L2) to find the token.  So the row crosses HBM once, and that
// is the bound: V (size(P) + size(Q)) bytes per request.  (512 requests, 152064 bf16 with 64 listed drafts: 156 MB in 37 us, 4.2
// TB/s; in the median block the acceptance test is done after 4.6 us and the row read after 36, 5.0 TB/s between, and the last
// token is out 3 us behind the last row.  The same with a deterministic drafter 37 us; 64 requests with two bf16 rows of 128256
// 10.4 us; one with two fp32 rows 6.6 us.  Rows that are not 16-byte aligned are read by elements: 512 requests of 152065 75 us, 64
// of two rows of 128257 22 us.)
//
// Weights are integers (2^-44 units): addition is exact in any order, so the token depends neither on the number of
// blocks nor on how the row was cut, and a row whose mass is spread over 2^18 tokens still leaves each token with
// the 24 bits that an fp32 probability of 2^-20 or more has.  A residual below 2^-44 has no weight; 2^18 of those would
// be 1.5e-8 of the mass, less than the rounding of one fp32 probability.  In the inner loop a weight is a pair of integers below
// 2^22 and 2^23 that two fused multiply-adds with rounding towards zero leave in the low bits of a float (adding 2^23
// makes the spacing of floats 1): six full-rate instructions, where a conversion to 64 bits runs at an eighth of that rate.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "../../include/wisv.h"
#include "wisv_ptx.cuh"

using namespace wisv;

namespace {

typedef unsigned long long u64;

constexpr int kResThreads = 128;                   // (twice as many blocks as with 256 spread more evenly: 41 -> 37.5 us for 512 requests)
constexpr int kResWarps = kResThreads / 32;
constexpr int kResMaxCluster = 16;
constexpr int kChunk = 512;                        // tokens whose weights a warp adds into one sum: 512 (2^23 - 1) < 2^32
constexpr int kMaxChunks = WISV_STATIC_MAX_V / kChunk;
constexpr int kChunksPerThread = kMaxChunks / kResThreads;
constexpr int kResPerSm = 8;                       // blocks that run on an SM at once
constexpr float kFix = 17592186044416.0f;          // 2^44
constexpr int kQuiet = 0, kDense = 1, kTop = 2;    // the drafter's distribution: one token, dense, a list

struct ResidualParams {
    int32_t B, K, T, V, n_top, cluster, device;
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
__device__ __forceinline__ float unit(float x) { return __saturatef(x); }

// floor(2^44 x) of 0 <= x <= 1 as hi 2^23 + lo, both with a constant on top that the caller takes off: kHiBias and kLoBias
constexpr unsigned kBias = 0x4B000000u;            // the bits of 2^23
__device__ __forceinline__ void fix_parts(float x, unsigned& hi, unsigned& lo)
{
    const float t = __fmaf_rz(x, 2097152.0f, 8388608.0f);                     // 2^23 + floor(2^21 x)
    const float r = __fmaf_rn(x, 2097152.0f, 8388608.0f - t);                 // the rest, exact: 0 <= r < 1
    hi = __float_as_uint(t);
    lo = __float_as_uint(__fmaf_rz(r, 8388608.0f, 8388608.0f));               // 2^23 + floor(2^23 r)
}
__device__ __forceinline__ u64 fix(float x)
{
    unsigned hi, lo;
    fix_parts(x, hi, lo);
    return (static_cast<u64>(hi - kBias) << 23) + (lo - kBias);
}

// 16 of a chunk's 512 elements per lane, as they lie in memory.  kWide: two runs of 8 consecutive ones (16-byte aligned
// rows), at 8 lane and 256 + 8 lane; otherwise every 32nd.  Elements past V are 0.
template <typename T, bool kWide>
struct Piece {
    union { uint4 w[sizeof(T)]; unsigned raw[4 * sizeof(T)]; };               // 16 elements

    __device__ __forceinline__ void load(const T* row, int v, int V, int lane)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            constexpr int n = sizeof(T) / 2;                                  // 16-byte loads per run
            const int at = v + h * 256 + lane * 8;
            if (kWide && at + 8 <= V) {
#pragma unroll
                for (int i = 0; i < n; ++i) w[h * n + i] = reinterpret_cast<const uint4*>(row + at)[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int x = kWide ? at + i : v + (8 * h + i) * 32 + lane;
                    put(8 * h + i, x < V ? bits(row[x]) : 0u);
                }
            }
        }
    }
    static __device__ __forceinline__ unsigned bits(float x) { return __float_as_uint(x); }
    static __device__ __forceinline__ unsigned bits(__nv_bfloat16 x) { return __bfloat16_as_ushort(x); }
    static __device__ __forceinline__ unsigned bits(__half x) { return __half_as_ushort(x); }
    __device__ __forceinline__ void put(int i, unsigned x)
    {
        if (sizeof(T) == 4) raw[i] = x;
        else raw[i / 2] = (i & 1) ? raw[i / 2] | (x << 16) : x;
    }
    __device__ __forceinline__ float get(int i) const
    {
        if (sizeof(T) == 4) return __uint_as_float(raw[i]);
        const unsigned x = raw[i / 2];
        if (is_bf16(static_cast<T*>(nullptr))) return __uint_as_float((i & 1) ? x & 0xffff0000u : x << 16);
        return __half2float(__ushort_as_half(static_cast<unsigned short>((i & 1) ? x >> 16 : x & 0xffffu)));
    }
    static __device__ __forceinline__ bool is_bf16(const __nv_bfloat16*) { return true; }
    static __device__ __forceinline__ bool is_bf16(const void*) { return false; }
};

__device__ __forceinline__ void st_cluster_u64(uint32_t addr, u64 x)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(x) : "memory");
}

template <typename TP, typename TQ, int kForm, bool kWide>
__global__ void __launch_bounds__(kResThreads, kResPerSm) residual_kernel(const ResidualParams p)
{
    __shared__ u64 chunk_mass[kMaxChunks];
    __shared__ u64 warp_mass[kResWarps];
    __shared__ u64 block_mass[2][kResMaxCluster];          // written by every block of the cluster
    __shared__ unsigned ok_bits[2];
    __shared__ int flag, found;
    __shared__ u64 found_before;
    __shared__ int list_v[kForm == kTop ? WISV_MAX_TOP : 1];
    __shared__ float list_q[kForm == kTop ? WISV_MAX_TOP : 1];
    __shared__ long long list_d[kForm == kTop ? WISV_MAX_TOP : 1];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = static_cast<int>(cluster_ctarank());
    const int b = blockIdx.x / p.cluster;
    if (tid == 0) { ok_bits[0] = ok_bits[1] = 0; flag = 0; found = -1; }
    cluster_arrive();                                      // waited for before the first store to another block
    // Everything read below may come from the kernel before this one.  (No early launch_dependents: the next kernel's blocks would
    // take room from this one's, 512 requests 37.2 -> 40 us.)
    griddep_wait();

    // ---- the window: offsets come from the device, so every index made of them is clamped
    int t0, K;
    if (p.k_off) {
        t0 = min(max(p.k_off[b], 0), p.T);
        K = min(max(p.k_off[b + 1], 0), p.T) - t0;
    } else {
        K = p.K; t0 = b * K;
    }
    const unsigned m = static_cast<unsigned>(fminf(unit(p.u_draw[b]) * 2147483648.0f, 2147483520.0f));
    const bool bad_window = K < 0 || K > WISV_MAX_K;
    K = min(max(K, 0), WISV_MAX_K);
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
            // eight lanes look one token up in its list
            for (int i = tid >> 3; i < ((K + 3) & ~3); i += kResThreads / 8) {
                const int k = min(i, K - 1);               // (whole warps take part in the shuffles)
                const int y = draft_at(k);
                const int64_t at = static_cast<int64_t>(t0 + k) * p.n_top, aq = static_cast<int64_t>(t0 + k) * p.q_stride;
                const float a = unit(as_f(P0[static_cast<int64_t>(k) * p.p_stride + y]));
                const float u = p.u[t0 + k];
                float q = 0.0f;
#pragma unroll 4
                for (int j = lane & 7; j < p.n_top; j += 8) q += p.ids[at + j] == y ? static_cast<const float*>(p.Q)[aq + j] : 0.0f;
#pragma unroll
                for (int o = 4; o; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
                q = unit(q);
                if ((lane & 7) == 0 && i < K && u < (q > 0.0f ? fminf(a / q, 1.0f) : (a > 0.0f ? 1.0f : 0.0f)))
                    atomicOr(&ok_bits[i >> 5], 1u << (i & 31));
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
    if (kForm == kTop && A < K) {
        for (int j = tid; j < p.n_top; j += kResThreads) {
            const int v = p.ids[static_cast<int64_t>(t0 + A) * p.n_top + j];
            list_v[j] = v >= 0 && v < p.V ? v : -1;
            list_q[j] = static_cast<const float*>(p.Q)[static_cast<int64_t>(t0 + A) * p.q_stride + j];
        }
    }

    // ---- this block's chunks, a contiguous run of them
    const int all = (p.V + kChunk - 1) / kChunk, per = (all + p.cluster - 1) / p.cluster;
    const int first = min(rank * per, all), n_chunks = min(first + per, all) - first;

    for (int pass = 0; pass < 2; ++pass) {
        const bool rest = pass == 0 && A < K;              // the residual; then (or at once, for a bonus token) P alone
        auto residual = [&](float a, float q) { return kForm == kDense && rest ? __saturatef(unit(a) - unit(q)) : unit(a); };
        // chunks whose loads are under way together: some 128 bytes per lane
        constexpr int kBytes = static_cast<int>(sizeof(TP)) + (kForm == kDense ? static_cast<int>(sizeof(TQ)) : 0);
        constexpr int U = kBytes <= 2 ? 4 : kBytes <= 4 ? 2 : 1;
        for (int c0 = warp; c0 < n_chunks; c0 += U * kResWarps) {
            Piece<TP, kWide> a[U];
            Piece<TQ, kWide> q[kForm == kDense ? U : 1];
#pragma unroll
            for (int s = 0; s < U; ++s) {
                const int c = c0 + s * kResWarps;
                if (c < n_chunks) {
                    a[s].load(P, (first + c) * kChunk, p.V, lane);
                    if (kForm == kDense && rest) q[kForm == kDense ? s : 0].load(Q, (first + c) * kChunk, p.V, lane);
                }
            }
#pragma unroll
            for (int s = 0; s < U; ++s) {
                const int c = c0 + s * kResWarps;
                if (c >= n_chunks) break;
                unsigned hi = 0, lo = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float x = residual(a[s].get(i), kForm == kDense ? q[kForm == kDense ? s : 0].get(i) : 0.0f);
                    if (kForm == kQuiet && rest) {         // Q is 1 at the drafted token: nothing is left there
                        const int v = (first + c) * kChunk + (kWide ? (i >> 3) * 256 + lane * 8 + (i & 7) : i * 32 + lane);
                        x = v == y ? 0.0f : x;
                    }
                    unsigned h, l;
                    fix_parts(x, h, l);
                    hi += h; lo += l;
                }
                hi = __reduce_add_sync(0xffffffffu, hi - 16u * kBias);
                lo = __reduce_add_sync(0xffffffffu, lo - 16u * kBias);
                if (lane == 0) chunk_mass[c] = (static_cast<u64>(hi) << 23) + lo;
            }
        }
        __syncthreads();
        if (kForm == kTop && rest) {
            // the listed tokens' weights, taken with Q = 0 above, are corrected by integers
            for (int j = tid; j < p.n_top; j += kResThreads) {
                const int v = list_v[j];
                float q = 0.0f;
                bool head = v >= 0;                        // the first entry of a token stands for all of them
                for (int k = 0; k < p.n_top; ++k)
                    if (list_v[k] == v) { if (k < j) head = false; q += list_q[k]; }
                long long d = 0;
                if (head) {
                    const float a = unit(as_f(P[v]));
                    d = static_cast<long long>(fix(__saturatef(a - unit(q)))) - static_cast<long long>(fix(a));
                    const int c = v / kChunk - first;
                    if (c >= 0 && c < n_chunks) atomicAdd(&chunk_mass[c], static_cast<u64>(d));
                }
                list_d[j] = d;
            }
            __syncthreads();
        }
        // ---- exclusive prefix sums over the block's chunks
        u64 own[kChunksPerThread], sum = 0;
#pragma unroll
        for (int i = 0; i < kChunksPerThread; ++i) {
            const int c = tid * kChunksPerThread + i;
            own[i] = c < n_chunks ? chunk_mass[c] : 0;
            sum += own[i];
        }
        u64 upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        if (lane == 31) warp_mass[warp] = upto;
        __syncthreads();
        u64 total = 0;
#pragma unroll
        for (int w = 0; w < kResWarps; ++w) {
            if (w < warp) upto += warp_mass[w];
            total += warp_mass[w];
        }
        if (pass == 0) cluster_wait();                     // every block of the cluster is running
        if (tid < p.cluster) st_cluster_u64(mapa_u32(smem_u32(&block_mass[pass][rank]), tid), total);
        __syncwarp();
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
            if (p.status) p.status[b] = flag | (bad_window ? WISV_ST_BAD_WINDOW : 0) | (W == 0 ? WISV_ST_NO_MASS : 0);
            if (W == 0) p.token[b] = -1;
        }
        if (W == 0) break;
        const u64 goal = (W >> 31) * m + (((W & 0x7fffffffull) * m) >> 31);
        if (goal < before || goal >= before + total) break;                   // another block's
        u64 at = before + upto - sum;
#pragma unroll
        for (int i = 0; i < kChunksPerThread; ++i) {
            if (goal >= at && goal < at + own[i]) { found = tid * kChunksPerThread + i; found_before = at; }
            at += own[i];
        }
        __syncthreads();
        if (warp != 0) break;
        // ---- the chunk that holds the goal: 16 consecutive tokens per lane
        const int v0 = (first + found) * kChunk + lane * 16;
        u64 w[16], s = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int v = v0 + i;
            float x = 0.0f;
            if (v < p.V) {
                x = residual(as_f(P[v]), kForm == kDense && rest ? as_f(Q[v]) : 0.0f);
                if (kForm == kQuiet && rest && v == y) x = 0.0f;
            }
            w[i] = fix(x);
        }
        if (kForm == kTop && rest) {
            for (int j0 = 0; j0 < p.n_top; j0 += 32) {     // listed tokens of this chunk
                const int x = j0 + lane < p.n_top ? list_v[j0 + lane] : -1;
                unsigned hit = __ballot_sync(0xffffffffu, x >= 0 && x / kChunk == first + found);
                while (hit) {
                    const int j = j0 + __ffs(hit) - 1;
                    hit &= hit - 1;
                    const int e = list_v[j] - v0;
#pragma unroll
                    for (int i = 0; i < 16; ++i) if (e == i) w[i] += static_cast<u64>(list_d[j]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s += w[i];
        u64 run = s;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 x = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += x;
        }
        run += found_before;
        if (goal < run && goal >= run - s) {
            u64 c = run - s;
            int tok = -1;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                c += w[i];
                if (tok < 0 && c > goal) tok = v0 + i;
            }
            p.token[b] = tok;
        }
        break;
    }
}

template <typename TP, typename TQ, int kForm, bool kWide>
int go(const ResidualParams& p, cudaStream_t st)
{
    auto kernel = residual_kernel<TP, TQ, kForm, kWide>;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)(p.B * p.cluster));
    cfg.blockDim = dim3(kResThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    static std::atomic<unsigned long long> allowed{0};    // devices on which clusters of 16 have been allowed
    const unsigned long long bit = p.device < 64 ? 1ull << p.device : 0;
    if (p.cluster > 8 && !(allowed.load(std::memory_order_relaxed) & bit)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
            (void)cudaGetLastError();
            return WISV_ECUDA;
        }
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) {
        (void)cudaGetLastError();
        return WISV_ECUDA;
    }
    return WISV_OK;
}

template <typename TP, bool kWide>
int by_form(const wisv_residual* r, const ResidualParams& p, cudaStream_t st)
{
    if (!r->draft_probs) return go<TP, float, kQuiet, kWide>(p, st);
    if (r->draft_ids) return go<TP, float, kTop, kWide>(p, st);
    switch (r->draft_dtype) {
        case WISV_DT_F32: return go<TP, float, kDense, kWide>(p, st);
        case WISV_DT_BF16: return go<TP, __nv_bfloat16, kDense, kWide>(p, st);
        default: return go<TP, __half, kDense, kWide>(p, st);
    }
}

template <bool kWide>
int by_target(const wisv_residual* r, const ResidualParams& p, cudaStream_t st)
{
    switch (r->target_dtype) {
        case WISV_DT_F32: return by_form<float, kWide>(r, p, st);
        case WISV_DT_BF16: return by_form<__nv_bfloat16, kWide>(r, p, st);
        default: return by_form<__half, kWide>(r, p, st);
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
    int dev = 0, major = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return WISV_ECUDA;
    }
    if (major != 10) return WISV_EARCH;
    ResidualParams p;
    p.device = dev;
    p.B = r->B; p.K = r->K; p.T = r->T_total; p.V = r->V; p.n_top = r->n_top;
    // Blocks per request: as many as can run at once, so that a small batch uses the whole chip and a large one pays for the
    // acceptance test and the exchange once per request; 16 only while every block has an SM to itself (one request: 7.0 us
    // against 8.5 with 8; 64 requests: 12.0 against 11.0).
    p.cluster = r->B * kResMaxCluster <= sms ? kResMaxCluster : kResMaxCluster / 2;
    while (p.cluster > 1 && (int64_t)p.B * p.cluster > kResPerSm * sms) p.cluster >>= 1;
    p.k_off = r->k_off; p.P = r->target_probs; p.p_stride = r->target_stride;
    p.Q = r->draft_probs; p.q_stride = r->draft_stride; p.ids = r->draft_ids; p.tokens = r->draft_tokens;
    p.u = r->uniforms; p.u_draw = r->u_draw; p.accept_in = r->accept_in;
    p.accept_len = r->accept_len; p.token = r->token; p.status = r->status; p.mass = r->mass;
    const bool wide = rows_aligned(p.P, p.p_stride, ps, 16) && (!dense || rows_aligned(p.Q, p.q_stride, qs, 16));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return wide ? by_target<true>(r, p, st) : by_target<false>(r, p, st);
}
