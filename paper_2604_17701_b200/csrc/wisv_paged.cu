// Paged key/value cache: context, argument checks and launches (include/wisv.h).
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <new>

#include "../../include/wisv.h"
#include "wisv_pages.cuh"
#include "wisv_attn.cuh"

using namespace wisv;

struct wisv_cache {
    wisv_cache_config cfg;
    int device = 0;
    int sm_count = 0;
    int page_shift = 0;
    int64_t launches = 0;
    int32_t* err = nullptr;
};

namespace {

#define WISV_TRY_CUDA(call)                                                        \
    do {                                                                           \
        if ((call) != cudaSuccess) { (void)cudaGetLastError(); return WISV_ECUDA; } \
    } while (0)

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

int log2_exact(int x)
{
    for (int s = 0; s < 31; ++s) if ((1 << s) == x) return s;
    return -1;
}

// one kernel on `st`, as a cluster of `cluster` blocks when that is more than 1
template <typename P>
int launch(void (*kernel)(P), int grid, int block, size_t smem, int cluster, cudaStream_t st, const P& p)
{
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    if (cluster > 1) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)cluster;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
    WISV_TRY_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
    return WISV_OK;
}

int check_pages(const wisv_cache* c, const wisv_pages* pg, int32_t B)
{
    if (!c || !pg || !pg->free_list || !pg->n_free || !pg->block_table || !pg->n_blocks || !pg->seq_len) return WISV_EINVAL;
    if (B < 1) return WISV_ESHAPE;
    if (B > c->cfg.max_requests) return WISV_ECAPACITY;
    return WISV_OK;
}

void fill_pages(const wisv_cache* c, const wisv_pages* pg, int32_t B, PagesParams* p)
{
    memset(p, 0, sizeof *p);
    p->B = B;
    p->page_shift = c->page_shift;
    p->n_pages = c->cfg.n_pages;
    p->max_blocks = c->cfg.max_blocks;
    p->free_list = pg->free_list;
    p->n_free = pg->n_free;
    p->block_table = pg->block_table;
    p->n_blocks = pg->n_blocks;
    p->seq_len = pg->seq_len;
}

// rounds with more rows than this are laid out by a cluster of eight blocks
constexpr int kExtendOneBlockRows = 4096;
constexpr int kCommitOneBlockRequests = 64;

}  // namespace

extern "C" {

int wisv_cache_create(const wisv_cache_config* cfg, wisv_cache** out)
{
    if (out) *out = nullptr;
    if (!cfg || !out) return WISV_EINVAL;
    if (cfg->dtype != WISV_DT_BF16 && cfg->dtype != WISV_DT_F16) return WISV_EINVAL;
    if (cfg->n_kv_heads < 1 || cfg->n_heads < 1 || cfg->n_heads % cfg->n_kv_heads ||
        cfg->n_heads / cfg->n_kv_heads > WISV_MAX_GROUP || cfg->n_kv_heads > 1024 ||
        (cfg->head_dim != 64 && cfg->head_dim != 128) || cfg->page_size < 16 || cfg->page_size > 256 ||
        log2_exact(cfg->page_size) < 0 || cfg->n_pages < 1 || cfg->max_requests < 1 ||
        cfg->max_requests > WISV_MAX_REQUESTS || cfg->max_blocks < 1 ||
        (int64_t)cfg->max_blocks * cfg->page_size > 0x7fff0000LL || (int64_t)cfg->n_pages * cfg->page_size > 0x7fff0000LL)
        return WISV_ESHAPE;
    int dev = 0;
    WISV_TRY_CUDA(cudaGetDevice(&dev));
    int major = 0, sms = 0;       // attributes one by one: cudaGetDeviceProperties takes milliseconds
    WISV_TRY_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
    WISV_TRY_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    if (major != 10) return WISV_EARCH;
    wisv_cache* c = new (std::nothrow) wisv_cache;
    if (!c) return WISV_ENOMEM;
    c->cfg = *cfg;
    c->device = dev;
    c->sm_count = sms;
    c->page_shift = log2_exact(cfg->page_size);
    const int sh = (4 * WISV_MAX_REQUESTS + 1) * 4;
    if (cudaFuncSetAttribute(pages_extend_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, sh) != cudaSuccess ||
        cudaFuncSetAttribute(pages_extend_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, sh) != cudaSuccess) {
        (void)cudaGetLastError();
        delete c;
        return WISV_ECUDA;
    }
    if (cudaMalloc(&c->err, 256) != cudaSuccess) { (void)cudaGetLastError(); delete c; return WISV_ENOMEM; }
    if (cudaMemset(c->err, 0, 256) != cudaSuccess || cudaStreamSynchronize(0) != cudaSuccess) {
        (void)cudaGetLastError();
        cudaFree(c->err);
        delete c;
        return WISV_ECUDA;
    }
    *out = c;
    return WISV_OK;
}

int wisv_cache_destroy(wisv_cache* c)
{
    if (!c) return WISV_EINVAL;
    cudaFree(c->err);
    delete c;
    return WISV_OK;
}

int64_t wisv_cache_launch_count(const wisv_cache* c) { return c ? c->launches : 0; }

int wisv_cache_error(wisv_cache* c, void* cuda_stream, int32_t* flags)
{
    if (!c || !flags) return WISV_EINVAL;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    WISV_TRY_CUDA(cudaMemcpyAsync(flags, c->err, sizeof(int32_t), cudaMemcpyDeviceToHost, st));
    WISV_TRY_CUDA(cudaMemsetAsync(c->err, 0, sizeof(int32_t), st));
    WISV_TRY_CUDA(cudaStreamSynchronize(st));
    return WISV_OK;
}

int wisv_cache_extend(wisv_cache* c, const wisv_pages* pages, int32_t B, int32_t T_total, const int32_t* n_new,
                      int32_t n_uniform, const wisv_layout* out, void* cuda_stream)
{
    const int rc = check_pages(c, pages, B);
    if (rc != WISV_OK) return rc;
    if (!out || !out->q_off || !out->kv_len || (T_total > 0 && (!out->slot_map || !out->positions))) return WISV_EINVAL;
    if (T_total < 0 || (!n_new && (n_uniform < 0 || (int64_t)n_uniform * B > 0x7fffffffLL))) return WISV_ESHAPE;
    PagesParams p;
    fill_pages(c, pages, B, &p);
    p.T = T_total;
    p.n_new = n_new;
    p.n_uniform = n_uniform;
    p.q_off = out->q_off;
    p.kv_len = out->kv_len;
    p.slot_map = out->slot_map;
    p.positions = out->positions;
    p.status = out->status;
    const size_t smem = (size_t)(4 * B + 1) * 4;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int r = T_total > kExtendOneBlockRows
                      ? launch(pages_extend_kernel<true>, kPageCluster, kPageThreads, smem, kPageCluster, st, p)
                      : launch(pages_extend_kernel<false>, 1, kPageThreads, smem, 1, st, p);
    if (r == WISV_OK) ++c->launches;
    return r;
}

int wisv_cache_commit(wisv_cache* c, const wisv_pages* pages, int32_t B, const int32_t* new_len, int32_t* status,
                      void* cuda_stream)
{
    const int rc = check_pages(c, pages, B);
    if (rc != WISV_OK) return rc;
    if (!new_len) return WISV_EINVAL;
    PagesParams p;
    fill_pages(c, pages, B, &p);
    p.new_len = new_len;
    p.status = status;
    const size_t smem = (size_t)(2 * B) * 4;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int r = B > kCommitOneBlockRequests
                      ? launch(pages_commit_kernel<true>, kPageCluster, kPageThreads, smem, kPageCluster, st, p)
                      : launch(pages_commit_kernel<false>, 1, kPageThreads, smem, 1, st, p);
    if (r == WISV_OK) ++c->launches;
    return r;
}

int wisv_cache_append(wisv_cache* c, const wisv_append* a, void* cuda_stream)
{
    if (!c || !a) return WISV_EINVAL;
    if (a->T < 0) return WISV_ESHAPE;
    if (a->T == 0) return WISV_OK;
    if (!a->k || !a->v || !a->k_pages || !a->v_pages || !a->slot_map) return WISV_EINVAL;
    if (misaligned(a->k) || misaligned(a->v) || misaligned(a->k_pages) || misaligned(a->v_pages)) return WISV_EALIGN;
    const int64_t s[] = {a->k_token_stride, a->k_head_stride, a->v_token_stride, a->v_head_stride, a->kp_page_stride,
                         a->kp_token_stride, a->kp_head_stride, a->vp_page_stride, a->vp_token_stride, a->vp_head_stride};
    for (int64_t x : s) if (x % 8) return WISV_EALIGN;
    AppendParams p;
    p.T = a->T;
    p.vecs = c->cfg.n_kv_heads * c->cfg.head_dim / 8;
    p.vec_shift = c->cfg.head_dim == 128 ? 4 : 3;
    p.page_shift = c->page_shift;
    p.n_slots = (int64_t)c->cfg.n_pages << c->page_shift;
    p.k = static_cast<const uint4*>(a->k);
    p.v = static_cast<const uint4*>(a->v);
    p.kt = s[0] / 8; p.kh = s[1] / 8; p.vt = s[2] / 8; p.vh = s[3] / 8;
    p.kp = static_cast<uint4*>(a->k_pages);
    p.vp = static_cast<uint4*>(a->v_pages);
    p.kpp = s[4] / 8; p.kpt = s[5] / 8; p.kph = s[6] / 8; p.vpp = s[7] / 8; p.vpt = s[8] / 8; p.vph = s[9] / 8;
    p.slot_map = a->slot_map;
    const int64_t n = (int64_t)a->T * p.vecs;
    if (n > 0x7fffffffLL * 128) return WISV_ESHAPE;
    const int r = launch(append_kernel, (int)((n + kAppendThreads - 1) / kAppendThreads), kAppendThreads, 0, 1,
                         static_cast<cudaStream_t>(cuda_stream), p);
    if (r == WISV_OK) ++c->launches;
    return r;
}

int wisv_cache_attend(wisv_cache* c, const wisv_attend* a, void* cuda_stream)
{
    if (!c || !a) return WISV_EINVAL;
    if (a->B < 1 || a->T < 0 || a->max_new < 1 || a->max_blocks < 1 || a->table_stride < a->max_blocks ||
        (int64_t)a->max_blocks << c->page_shift > 0x7fff0000LL || (!a->q_off && (int64_t)a->B * a->max_new != a->T))
        return WISV_ESHAPE;
    if (a->B > c->cfg.max_requests) return WISV_ECAPACITY;
    if (a->T == 0) return WISV_OK;
    if (!a->q || !a->k_pages || !a->v_pages || !a->out || !a->kv_len || !a->block_table || !(a->scale >= 0.0f) ||
        isinf(a->scale))
        return WISV_EINVAL;
    if (misaligned(a->q) || misaligned(a->k_pages) || misaligned(a->v_pages) || misaligned(a->out)) return WISV_EALIGN;
    const int64_t s[] = {a->q_token_stride, a->q_head_stride, a->o_token_stride, a->o_head_stride, a->kp_page_stride,
                         a->kp_token_stride, a->kp_head_stride, a->vp_page_stride, a->vp_token_stride, a->vp_head_stride};
    for (int64_t x : s) if (x % 8 || x < 0) return WISV_EALIGN;
    if (a->kp_page_stride % (8 * a->kp_token_stride) || a->vp_page_stride % (8 * a->vp_token_stride)) return WISV_EALIGN;
    AttnParams p;
    p.B = a->B; p.T = a->T; p.max_new = a->max_new;
    p.n_heads = c->cfg.n_heads; p.group = c->cfg.n_heads / c->cfg.n_kv_heads;
    p.page_shift = c->page_shift; p.n_pages = c->cfg.n_pages; p.max_blocks = a->max_blocks;
    p.q_off = a->q_off; p.kv_len = a->kv_len; p.block_table = a->block_table; p.table_stride = a->table_stride;
    p.q = a->q; p.qt = s[0]; p.qh = s[1]; p.out = a->out; p.ot = s[2]; p.oh = s[3];
    p.kp = a->k_pages; p.vp = a->v_pages; p.kpp = s[4]; p.kpt = s[5]; p.kph = s[6]; p.vpp = s[7]; p.vpt = s[8]; p.vph = s[9];
    p.lse = a->lse;
    p.scale = a->scale > 0.0f ? a->scale : 1.0f / sqrtf((float)c->cfg.head_dim);
    const int64_t n = (int64_t)a->T * p.n_heads;
    const int grid = (int)((n + 3) / 4);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int r;
    if (c->cfg.dtype == WISV_DT_BF16)
        r = c->cfg.head_dim == 128 ? launch(attn_simple_kernel<__nv_bfloat16, 128>, grid, 128, 0, 1, st, p)
                                   : launch(attn_simple_kernel<__nv_bfloat16, 64>, grid, 128, 0, 1, st, p);
    else
        r = c->cfg.head_dim == 128 ? launch(attn_simple_kernel<__half, 128>, grid, 128, 0, 1, st, p)
                                   : launch(attn_simple_kernel<__half, 64>, grid, 128, 0, 1, st, p);
    if (r == WISV_OK) ++c->launches;
    return r;
}

}  // extern "C"
