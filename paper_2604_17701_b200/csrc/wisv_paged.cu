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

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct wisv_cache {
    wisv_cache_config cfg;
    int device = 0;
    int sm_count = 0;
    int page_shift = 0;
    int64_t launches = 0;
    // one allocation: [error word, half of the counters in use | arrival counters | partial maxima and sums | partial outputs]
    void* work = nullptr;         // NULL: the caller's
    int32_t* err = nullptr;
    int32_t* count = nullptr;
    float2* part_ml = nullptr;
    float* part_o = nullptr;
    EncodeTiledFn encode = nullptr;
    uint64_t wait_clocks = kAttnWaitClocks;       // wisv_debug_cache_waits
    int32_t stalled = -1;
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

// One kernel on `st`, as a cluster of `cluster` blocks when that is more than 1, with programmatic dependent launch: its blocks are
// set up while the kernel before it in the stream ends, and wait for it (griddepcontrol.wait) before they read anything.
template <typename P>
int launch(void (*kernel)(P), int grid, int block, size_t smem, int cluster, cudaStream_t st, const P& p)
{
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    WISV_TRY_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
    return WISV_OK;
}

// Five-dimensional map of 16-bit elements with the 128-byte swizzle; strides[i] in bytes for dimensions 1..4.
int encode_5d(const wisv_cache* c, CUtensorMap* out, const void* base, const cuuint64_t (&dims)[5],
              const cuuint64_t (&strides)[4], const cuuint32_t (&box)[5])
{
    const cuuint32_t one[5] = {1, 1, 1, 1, 1};
    const CUresult r = c->encode(out, c->cfg.dtype == WISV_DT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                                 5, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                 CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? WISV_OK : WISV_EINVAL;
}

// A pool of pages as (64 columns, 8 tokens, column halves, key head, 8-token group): one box is one page (or 128 tokens of
// a larger one) of one head, in shared memory [group][half][token][64].
int encode_pool(const wisv_cache* c, CUtensorMap* out, const void* base, int64_t page, int64_t token, int64_t head,
                int32_t* page_groups, int32_t* groups)
{
    const int64_t step = c->cfg.n_pages > 1 ? page / (8 * token) : 0;
    const int64_t n = (c->cfg.n_pages - 1) * step + c->cfg.page_size / 8;
    if (n > 0x7fffffffLL) return WISV_ESHAPE;
    *page_groups = (int32_t)step;
    *groups = (int32_t)n;
    const cuuint64_t dims[5] = {64, 8, (cuuint64_t)c->cfg.head_dim / 64, (cuuint64_t)c->cfg.n_kv_heads, (cuuint64_t)n};
    const cuuint64_t strides[4] = {(cuuint64_t)token * 2, 128, (cuuint64_t)(c->cfg.n_kv_heads > 1 ? head : 64) * 2, (cuuint64_t)token * 16};
    const cuuint32_t box[5] = {64, 8, (cuuint32_t)c->cfg.head_dim / 64, 1, (cuuint32_t)(c->cfg.page_size < kAttnTile ? c->cfg.page_size : kAttnTile) / 8};
    return encode_5d(c, out, base, dims, strides, box);
}

int check_config(const wisv_cache_config* cfg, int* dev, int* sms)
{
    if (cfg->dtype != WISV_DT_BF16 && cfg->dtype != WISV_DT_F16) return WISV_EINVAL;
    if (cfg->n_kv_heads < 1 || cfg->n_heads < 1 || cfg->n_heads % cfg->n_kv_heads ||
        cfg->n_heads / cfg->n_kv_heads > WISV_MAX_GROUP || cfg->n_kv_heads > 1024 ||
        (cfg->head_dim != 64 && cfg->head_dim != 128) || cfg->page_size < 16 || cfg->page_size > 256 ||
        log2_exact(cfg->page_size) < 0 || cfg->n_pages < 1 || cfg->max_requests < 1 ||
        cfg->max_requests > WISV_MAX_REQUESTS || cfg->max_blocks < 1 ||
        (int64_t)cfg->max_blocks * cfg->page_size > 0x7fff0000LL || (int64_t)cfg->n_pages * cfg->page_size > 0x7fff0000LL)
        return WISV_ESHAPE;
    int major = 0;       // attributes one by one: cudaGetDeviceProperties takes milliseconds
    WISV_TRY_CUDA(cudaGetDevice(dev));
    WISV_TRY_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev));
    WISV_TRY_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev));
    return major == 10 ? WISV_OK : WISV_EARCH;
}

// offsets in the workspace: error word at 0, arrival counters, partial maxima and sums, partial outputs
struct Workspace { int64_t count, ml, o, bytes; };
Workspace layout_of(const wisv_cache_config* cfg, int sms)
{
    Workspace w;
    const int64_t rows = (int64_t)sms * 2 * 256;
    w.count = 256;
    w.ml = (w.count + (int64_t)sms * 4 + 255) / 256 * 256;
    w.o = (w.ml + rows * 8 + 255) / 256 * 256;
    w.bytes = w.o + rows * cfg->head_dim * 4;
    return w;
}

// A cache's workspace and launch shapes are those of the device that it was created on.
int check_device(const wisv_cache* c)
{
    int dev = 0;
    WISV_TRY_CUDA(cudaGetDevice(&dev));
    return dev == c->device ? WISV_OK : WISV_EINVAL;
}

int check_pages(const wisv_cache* c, const wisv_pages* pg, int32_t B)
{
    if (!c || !pg || !pg->free_list || !pg->n_free || !pg->block_table || !pg->n_blocks || !pg->seq_len) return WISV_EINVAL;
    if (B < 1) return WISV_ESHAPE;
    if (B > c->cfg.max_requests) return WISV_ECAPACITY;
    return check_device(c);
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

// One block, or a cluster of eight that repeats the scan and shares the rest.  extend: a row per thread at most for one block (one / eight:
// 576 rows of 64 requests 4.15 / 4.23 us, 1088 rows 4.85 / 4.33, 4608 rows of 512 requests 8.1 / 4.6, 69632 of 4096 78 / 17).
constexpr int kExtendOneBlockRows = 1024;
// commit: the pages that go back are what the blocks share, and only the device knows how many (extend and commit with a commit of one
// / eight: 512 requests of 9 rows 9.66 / 9.96 us, 1024 of 9 11.9 / 12.3, 2048 of 9 16.9 / 16.5, 4096 of 2 17.4 / 17.7, of 17 32.9 / 28.4).
constexpr int kCommitOneBlockRequests = 1024;

// Programmatic dependent launch: the block set-up (barriers, TMEM) runs while the kernel before it in the stream ends.
template <typename E, int D>
int launch_attn(const wisv_cache* c, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const AttnParams& p,
                cudaStream_t st)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)c->sm_count);
    cfg.blockDim = dim3(kAttnThreads);
    cfg.dynamicSmemBytes = kAttnSmem;
    WISV_TRY_CUDA(cudaLaunchKernelEx(&cfg, attn_kernel<E, D>, tmQ, tmK, tmV, p));
    return WISV_OK;
}

}  // namespace

extern "C" {

int wisv_cache_workspace(const wisv_cache_config* cfg, int64_t* bytes)
{
    if (!cfg || !bytes) return WISV_EINVAL;
    int dev = 0, sms = 0;
    const int rc = check_config(cfg, &dev, &sms);
    if (rc == WISV_OK) *bytes = layout_of(cfg, sms).bytes;
    return rc;
}

int wisv_cache_create(const wisv_cache_config* cfg, wisv_cache** out)
{
    if (out) *out = nullptr;
    if (!cfg || !out) return WISV_EINVAL;
    int dev = 0, sms = 0;
    const int rc = check_config(cfg, &dev, &sms);
    if (rc != WISV_OK) return rc;
    const Workspace lay = layout_of(cfg, sms);
    if (cfg->workspace && (reinterpret_cast<uintptr_t>(cfg->workspace) & 255u)) return WISV_EALIGN;
    if (cfg->workspace && cfg->workspace_bytes < lay.bytes) return WISV_ECAPACITY;
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
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ready =
        cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) == cudaSuccess && fn &&
        cudaFuncSetAttribute(attn_kernel<__nv_bfloat16, 128>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAttnSmem) == cudaSuccess &&
        cudaFuncSetAttribute(attn_kernel<__nv_bfloat16, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAttnSmem) == cudaSuccess &&
        cudaFuncSetAttribute(attn_kernel<__half, 128>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAttnSmem) == cudaSuccess &&
        cudaFuncSetAttribute(attn_kernel<__half, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAttnSmem) == cudaSuccess;
    if (!ready) { (void)cudaGetLastError(); delete c; return WISV_ECUDA; }
    c->encode = reinterpret_cast<EncodeTiledFn>(fn);
    if (!cfg->workspace && cudaMalloc(&c->work, (size_t)lay.bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        delete c;
        return WISV_ENOMEM;
    }
    char* w = static_cast<char*>(cfg->workspace ? cfg->workspace : c->work);
    c->err = reinterpret_cast<int32_t*>(w);
    c->count = reinterpret_cast<int32_t*>(w + lay.count);
    c->part_ml = reinterpret_cast<float2*>(w + lay.ml);
    c->part_o = reinterpret_cast<float*>(w + lay.o);
    if (cudaMemset(c->err, 0, (size_t)lay.ml) != cudaSuccess || cudaStreamSynchronize(0) != cudaSuccess) {
        (void)cudaGetLastError();
        if (c->work) cudaFree(c->work);
        delete c;
        return WISV_ECUDA;
    }
    *out = c;
    return WISV_OK;
}

int wisv_cache_destroy(wisv_cache* c)
{
    if (!c) return WISV_EINVAL;
    if (c->work) cudaFree(c->work);
    delete c;
    return WISV_OK;
}

int64_t wisv_cache_launch_count(const wisv_cache* c) { return c ? c->launches : 0; }

int wisv_cache_error(wisv_cache* c, void* cuda_stream, int32_t* flags)
{
    if (!c || !flags) return WISV_EINVAL;
    const int rc = check_device(c);
    if (rc != WISV_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    WISV_TRY_CUDA(cudaMemcpyAsync(flags, c->err, sizeof(int32_t), cudaMemcpyDeviceToHost, st));
    WISV_TRY_CUDA(cudaMemsetAsync(c->err, 0, 256 + (size_t)c->sm_count * 4, st));
    WISV_TRY_CUDA(cudaStreamSynchronize(st));
    return WISV_OK;
}

int wisv_debug_cache_waits(wisv_cache* c, uint64_t limit_cycles, int32_t block)
{
    if (!c || limit_cycles > kAttnWaitClocks || block < -1) return WISV_EINVAL;
    c->wait_clocks = limit_cycles ? limit_cycles : kAttnWaitClocks;
    c->stalled = block;
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
    const int rc = check_device(c);
    if (rc != WISV_OK) return rc;
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
    if (!a->kp_token_stride || !a->vp_token_stride || a->kp_page_stride % (8 * a->kp_token_stride) || a->vp_page_stride % (8 * a->vp_token_stride)) return WISV_EALIGN;
    int r = check_device(c);
    if (r != WISV_OK) return r;
    const int group = c->cfg.n_heads / c->cfg.n_kv_heads, D = c->cfg.head_dim;
    AttnParams p;
    memset(&p, 0, sizeof p);
    CUtensorMap tmQ, tmK, tmV;
    r = encode_pool(c, &tmK, a->k_pages, s[4], s[5], s[6], &p.page_groups_k, &p.groups_k);
    if (r == WISV_OK) r = encode_pool(c, &tmV, a->v_pages, s[7], s[8], s[9], &p.page_groups_v, &p.groups_v);
    if (r != WISV_OK) return r;
    p.tpt = kAttnTile / group < a->max_new ? kAttnTile / group : a->max_new;
    {
        // (64 columns, head of the group, token, column halves, key head): a box is a row tile of one key head
        const cuuint64_t dims[5] = {64, (cuuint64_t)group, (cuuint64_t)a->T, (cuuint64_t)D / 64, (cuuint64_t)c->cfg.n_kv_heads};
        const cuuint64_t strides[4] = {(cuuint64_t)(c->cfg.n_heads > 1 ? s[1] : 64) * 2, (cuuint64_t)(a->T > 1 ? s[0] : 64) * 2, 128,
                                       (cuuint64_t)(c->cfg.n_heads > 1 ? s[1] : 64) * 2 * group};
        const cuuint32_t box[5] = {64, (cuuint32_t)group, (cuuint32_t)p.tpt, 1, 1};
        r = encode_5d(c, &tmQ, a->q, dims, strides, box);
        if (r != WISV_OK) return r;
    }
    // every key tile of every item has to count in 31 bits, whatever the lengths on the device say
    const int64_t items = (a->T + p.tpt - 1) / p.tpt + a->B, tiles = ((int64_t)a->max_blocks << c->page_shift) / kAttnTile + 2;
    if (items * tiles > 0x7ffe0000LL / c->cfg.n_kv_heads) return WISV_ESHAPE;
    p.B = a->B; p.T = a->T; p.n_kv = c->cfg.n_kv_heads; p.group = group;
    p.page_shift = c->page_shift; p.n_pages = c->cfg.n_pages; p.max_blocks = a->max_blocks;
    p.uniform = a->max_new; p.clear_rest = a->clear_rest; p.q_off = a->q_off; p.kv_len = a->kv_len; p.block_table = a->block_table;
    p.table_stride = a->table_stride;
    p.v = a->v_pages; p.vp = s[7]; p.vt = s[8]; p.vh = s[9];
    p.out = a->out; p.ot = s[2]; p.oh = s[3]; p.lse = a->lse;
    p.scale_log2 = (a->scale > 0.0f ? a->scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
    p.inv_group = 1.0f / (float)group;
    p.wait_limit = (uint32_t)((c->wait_clocks + 1023) >> 10); p.stalled = c->stalled;
    p.err = c->err; p.part_o = c->part_o; p.part_ml = c->part_ml; p.count = c->count;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool bf = c->cfg.dtype == WISV_DT_BF16;
    if (D == 128) r = bf ? launch_attn<__nv_bfloat16, 128>(c, tmQ, tmK, tmV, p, st) : launch_attn<__half, 128>(c, tmQ, tmK, tmV, p, st);
    else r = bf ? launch_attn<__nv_bfloat16, 64>(c, tmQ, tmK, tmV, p, st) : launch_attn<__half, 64>(c, tmQ, tmK, tmV, p, st);
    if (r == WISV_OK) ++c->launches;
    return r;
}

}  // extern "C"
