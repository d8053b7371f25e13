// The paged cache in 8 bits: argument checks and launches (include/wisv.h).
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "../../include/wisv.h"
#include "wisv_cache.cuh"
#include "wisv_attn8r.cuh"
#include "wisv_q8.cuh"

namespace wisv {

namespace {

template <typename E, int D>
bool prepare()
{
    auto set = [](const void* kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kAttnSmem) == cudaSuccess; };
    return set((const void*)attn8_kernel<E, D, 16>) && set((const void*)attn8_kernel<E, D, 32>) && set((const void*)attn8_kernel<E, D, 48>) &&
           set((const void*)attn8_kernel<E, D, 64>) && set((const void*)attn8_rows_kernel<E, D>);
}

}  // namespace

bool q8_prepare()
{
    return prepare<__nv_bfloat16, 128>() && prepare<__nv_bfloat16, 64>() && prepare<__half, 128>() && prepare<__half, 64>();
}

}  // namespace wisv

using namespace wisv;

namespace {

// Pools as the library takes them: 16-byte pieces of codes, 16-byte pieces of scales.
int check_pools(const wisv_cache* c, const wisv_q8_pages* g)
{
    if (!g->k || !g->v || !g->k_scale || !g->v_scale) return WISV_EINVAL;
    if (misaligned(g->k) || misaligned(g->v) || misaligned(g->k_scale) || misaligned(g->v_scale)) return WISV_EALIGN;
    const int64_t codes[] = {g->k_page_stride, g->k_token_stride, g->k_head_stride, g->v_page_stride, g->v_token_stride, g->v_head_stride};
    for (int64_t x : codes) if (x % 16) return WISV_EALIGN;
    const int64_t scales[] = {g->ks_page_stride, g->ks_head_stride, g->vs_page_stride, g->vs_head_stride};
    for (int64_t x : scales) if (x % 4) return WISV_EALIGN;
    return check_device(c);
}

Q8Pages pools_of(const wisv_cache* c, const wisv_q8_pages* g)
{
    Q8Pages p;
    p.k = static_cast<uint4*>(g->k); p.v = static_cast<uint4*>(g->v);
    p.ks = g->k_scale; p.vs = g->v_scale;
    p.kp = g->k_page_stride / 16; p.kt = g->k_token_stride / 16; p.kh = g->k_head_stride / 16;
    p.vp = g->v_page_stride / 16; p.vt = g->v_token_stride / 16; p.vh = g->v_head_stride / 16;
    p.ksp = g->ks_page_stride; p.ksh = g->ks_head_stride; p.vsp = g->vs_page_stride; p.vsh = g->vs_head_stride;
    p.n_slots = (int64_t)c->cfg.n_pages << c->page_shift;
    p.page_shift = c->page_shift;
    return p;
}

// A pool of codes as (element, token of the page, key head, page): one box is one page (or 128 tokens of a larger one) of one head, a row per
// token with the swizzle of its width.  (Fetched by 128 bytes: with 256 a pool with heads side by side gives twice what is asked for, one row each
// of 64 requests over 270 k keys 152 instead of 116 us.)
int encode_codes(const wisv_cache* c, CUtensorMap* out, const void* base, int64_t page, int64_t token, int64_t head)
{
    const cuuint64_t D = (cuuint64_t)c->cfg.head_dim;
    const cuuint64_t dims[4] = {D, (cuuint64_t)c->cfg.page_size, (cuuint64_t)c->cfg.n_kv_heads, (cuuint64_t)c->cfg.n_pages};
    // (a single head or page has no stride of its own)
    const cuuint64_t strides[3] = {(cuuint64_t)token, c->cfg.n_kv_heads > 1 ? (cuuint64_t)head : D, c->cfg.n_pages > 1 ? (cuuint64_t)page : D};
    const cuuint32_t box[4] = {(cuuint32_t)D, (cuuint32_t)(c->cfg.page_size < kAttnTile ? c->cfg.page_size : kAttnTile), 1, 1};
    const cuuint32_t one[4] = {1, 1, 1, 1};
    const CUresult r = c->encode(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(base), dims, strides, box, one,
                                 CU_TENSOR_MAP_INTERLEAVE_NONE, D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                                 CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? WISV_OK : WISV_EINVAL;
}

// Programmatic dependent launch: the block set-up (barriers, TMEM) runs while the kernel before it in the stream ends.
template <typename E, int D>
int launch_attn8(const wisv_cache* c, const CUtensorMap& tmK, const CUtensorMap& tmV, Attn8Params& p, cudaStream_t st)
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
    cfg.dynamicSmemBytes = kAttnSmem;
    const Attn8Params& q = p;
    if (p.rows) {
        cfg.blockDim = dim3(kAttnThreads);
        WISV_TRY_CUDA(cudaLaunchKernelEx(&cfg, attn8_rows_kernel<E, D>, tmK, tmV, q));
        return WISV_OK;
    }
    const int cols = a8_cols(p.tpt * p.group);
    p.q_bytes = (uint32_t)(a8_parts<E>::n * cols * D);
    p.p_bytes = (uint32_t)a8_p_bytes<E>(cols);
    // what is left of shared memory: stages of keys and values in even numbers; a value stage is held longer (behind the exponentials)
    const int left = kAttnSmem - kA8Slack - kA8Small - kA8Scales * kA8ScaleBytes - 2 * (int)(p.q_bytes + p.p_bytes);
    const int stages = left / (int)a8_tile_bytes<D>(), v = (stages + 2) / 4 * 2, k = (stages - (v < kA8Stages ? v : kA8Stages)) / 2 * 2;
    p.v_stages = v < kA8Stages ? v : kA8Stages;
    p.k_stages = k < kA8Stages ? k : kA8Stages;
    cfg.blockDim = dim3(kA8Threads);
    WISV_TRY_CUDA(cols == 16   ? cudaLaunchKernelEx(&cfg, attn8_kernel<E, D, 16>, tmK, tmV, q)
                  : cols == 32 ? cudaLaunchKernelEx(&cfg, attn8_kernel<E, D, 32>, tmK, tmV, q)
                  : cols == 48 ? cudaLaunchKernelEx(&cfg, attn8_kernel<E, D, 48>, tmK, tmV, q)
                               : cudaLaunchKernelEx(&cfg, attn8_kernel<E, D, 64>, tmK, tmV, q));
    return WISV_OK;
}

}  // namespace

extern "C" {

int wisv_cache_append_q8(wisv_cache* c, const wisv_q8_pages* pages, const wisv_q8_append* a, void* cuda_stream)
{
    if (!c || !pages || !a) return WISV_EINVAL;
    if (a->T < 0) return WISV_ESHAPE;
    if (a->T == 0) return WISV_OK;
    if (!a->k || !a->v || !a->slot_map) return WISV_EINVAL;
    if (misaligned(a->k) || misaligned(a->v)) return WISV_EALIGN;
    const int64_t s[] = {a->k_token_stride, a->k_head_stride, a->v_token_stride, a->v_head_stride};
    for (int64_t x : s) if (x % 8) return WISV_EALIGN;
    int r = check_pools(c, pages);
    if (r != WISV_OK) return r;
    Q8AppendParams p;
    p.pg = pools_of(c, pages);
    p.T = a->T;
    p.vecs = c->cfg.n_kv_heads * c->cfg.head_dim / 16;
    p.k = static_cast<const uint4*>(a->k);
    p.v = static_cast<const uint4*>(a->v);
    p.kt = s[0] / 8; p.kh = s[1] / 8; p.vt = s[2] / 8; p.vh = s[3] / 8;
    p.slot_map = a->slot_map;
    const int64_t grid = ((int64_t)a->T * p.vecs + kQ8Threads - 1) / kQ8Threads;
    if (grid > 0x7fffffffLL) return WISV_ESHAPE;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool bf = c->cfg.dtype == WISV_DT_BF16;
    if (c->cfg.head_dim == 128)
        r = bf ? launch(append_q8_kernel<__nv_bfloat16, 128>, (int)grid, kQ8Threads, 0, 1, st, p)
               : launch(append_q8_kernel<__half, 128>, (int)grid, kQ8Threads, 0, 1, st, p);
    else
        r = bf ? launch(append_q8_kernel<__nv_bfloat16, 64>, (int)grid, kQ8Threads, 0, 1, st, p)
               : launch(append_q8_kernel<__half, 64>, (int)grid, kQ8Threads, 0, 1, st, p);
    if (r == WISV_OK) ++c->launches;
    return r;
}

int wisv_cache_read_q8(wisv_cache* c, const wisv_q8_pages* pages, const wisv_q8_read* a, void* cuda_stream)
{
    if (!c || !pages || !a) return WISV_EINVAL;
    if (a->B < 1 || a->T < 0 || a->max_blocks < 1 || a->table_stride < a->max_blocks || (int64_t)a->max_blocks << c->page_shift > 0x7fff0000LL ||
        (!a->off && (a->n_uniform < 0 || (int64_t)a->B * a->n_uniform != a->T)))
        return WISV_ESHAPE;
    if (a->B > c->cfg.max_requests) return WISV_ECAPACITY;
    if (a->T == 0) return WISV_OK;
    if (!a->block_table || !a->k || !a->v) return WISV_EINVAL;
    if (misaligned(a->k) || misaligned(a->v)) return WISV_EALIGN;
    const int64_t s[] = {a->k_token_stride, a->k_head_stride, a->v_token_stride, a->v_head_stride};
    for (int64_t x : s) if (x % 8) return WISV_EALIGN;
    int r = check_pools(c, pages);
    if (r != WISV_OK) return r;
    Q8ReadParams p;
    p.pg = pools_of(c, pages);
    p.B = a->B; p.T = a->T;
    p.vecs = c->cfg.n_kv_heads * c->cfg.head_dim / 16;
    // rows of a block: two pieces of each thread, of as many rows as that makes
    p.tokens = 2 * kQ8Threads / p.vecs;
    p.tokens = p.tokens < 1 ? 1 : p.tokens > kQ8ReadTokens ? kQ8ReadTokens : p.tokens;
    p.uniform = a->n_uniform; p.max_blocks = a->max_blocks; p.n_pages = c->cfg.n_pages; p.clear_rest = a->clear_rest;
    p.off = a->off; p.start = a->start; p.block_table = a->block_table; p.table_stride = a->table_stride;
    p.k = static_cast<uint4*>(a->k); p.v = static_cast<uint4*>(a->v);
    p.kt = s[0] / 8; p.kh = s[1] / 8; p.vt = s[2] / 8; p.vh = s[3] / 8;
    const int grid = (int)(((int64_t)a->T + p.tokens - 1) / p.tokens);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool bf = c->cfg.dtype == WISV_DT_BF16;
    if (c->cfg.head_dim == 128)
        r = bf ? launch(read_q8_kernel<__nv_bfloat16, 128>, grid, kQ8Threads, 0, 1, st, p)
               : launch(read_q8_kernel<__half, 128>, grid, kQ8Threads, 0, 1, st, p);
    else
        r = bf ? launch(read_q8_kernel<__nv_bfloat16, 64>, grid, kQ8Threads, 0, 1, st, p)
               : launch(read_q8_kernel<__half, 64>, grid, kQ8Threads, 0, 1, st, p);
    if (r == WISV_OK) ++c->launches;
    return r;
}

int wisv_cache_attend_q8(wisv_cache* c, const wisv_q8_pages* pages, const wisv_q8_attend* a, void* cuda_stream)
{
    if (!c || !pages || !a) return WISV_EINVAL;
    if (a->B < 1 || a->T < 0 || a->max_new < 1 || a->max_blocks < 1 || a->table_stride < a->max_blocks ||
        (int64_t)a->max_blocks << c->page_shift > 0x7fff0000LL || (!a->q_off && (int64_t)a->B * a->max_new != a->T))
        return WISV_ESHAPE;
    if (a->B > c->cfg.max_requests) return WISV_ECAPACITY;
    if (a->T == 0) return WISV_OK;
    if (!a->q || !a->out || !a->kv_len || !a->block_table || !(a->scale >= 0.0f) || isinf(a->scale)) return WISV_EINVAL;
    if (misaligned(a->q) || misaligned(a->out)) return WISV_EALIGN;
    const int64_t s[] = {a->q_token_stride, a->q_head_stride, a->o_token_stride, a->o_head_stride};
    for (int64_t x : s) if (x % 8) return WISV_EALIGN;
    int r = check_pools(c, pages);
    if (r != WISV_OK) return r;
    const int64_t codes[] = {pages->k_page_stride, pages->k_token_stride, pages->k_head_stride, pages->v_page_stride, pages->v_token_stride, pages->v_head_stride};
    for (int64_t x : codes) if (x < 0) return WISV_EALIGN;
    if (!pages->k_token_stride || !pages->v_token_stride) return WISV_EALIGN;
    CUtensorMap tmK, tmV;
    r = encode_codes(c, &tmK, pages->k, pages->k_page_stride, pages->k_token_stride, pages->k_head_stride);
    if (r == WISV_OK) r = encode_codes(c, &tmV, pages->v, pages->v_page_stride, pages->v_token_stride, pages->v_head_stride);
    if (r != WISV_OK) return r;
    const int group = c->cfg.n_heads / c->cfg.n_kv_heads, D = c->cfg.head_dim;
    Attn8Params p;
    memset(&p, 0, sizeof p);
    // rows of a request as rows of the products where they are more than a tile's columns on the average (wisv_attn8r.cuh has both sides' figures)
    p.rows = (int64_t)a->T * group > (int64_t)kA8Cols * a->B;
    const int tile = (p.rows ? kAttnTile : kA8Cols) / group;
    p.tpt = tile < a->max_new ? tile : a->max_new;
    // every unit of every item has to count in 31 bits, whatever the lengths on the device say
    const int64_t items = (a->T + p.tpt - 1) / p.tpt + a->B, tiles = ((int64_t)a->max_blocks << c->page_shift) / kAttnTile + 2 + kA8ItemCost;
    if (items * tiles > 0x7ffe0000LL / c->cfg.n_kv_heads) return WISV_ESHAPE;
    p.B = a->B; p.T = a->T; p.n_kv = c->cfg.n_kv_heads; p.group = group;
    p.page_shift = c->page_shift; p.n_pages = c->cfg.n_pages; p.max_blocks = a->max_blocks;
    p.uniform = a->max_new; p.clear_rest = a->clear_rest; p.q_off = a->q_off; p.kv_len = a->kv_len; p.block_table = a->block_table;
    p.table_stride = a->table_stride;
    p.q = a->q; p.qt = s[0]; p.qh = s[1];
    p.out = a->out; p.ot = s[2]; p.oh = s[3]; p.lse = a->lse;
    p.ks = pages->k_scale; p.vs = pages->v_scale;
    p.ksp = pages->ks_page_stride; p.ksh = pages->ks_head_stride; p.vsp = pages->vs_page_stride; p.vsh = pages->vs_head_stride;
    p.scale_log2 = (a->scale > 0.0f ? a->scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
    p.inv_group = 1.0f / (float)group;
    p.wait_limit = (uint32_t)((c->wait_clocks + 1023) >> 10); p.stalled = c->stalled;
    p.err = c->err; p.part_o = c->part_o; p.part_ml = c->part_ml; p.count = c->count;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool bf = c->cfg.dtype == WISV_DT_BF16;
    if (D == 128) r = bf ? launch_attn8<__nv_bfloat16, 128>(c, tmK, tmV, p, st) : launch_attn8<__half, 128>(c, tmK, tmV, p, st);
    else r = bf ? launch_attn8<__nv_bfloat16, 64>(c, tmK, tmV, p, st) : launch_attn8<__half, 64>(c, tmK, tmV, p, st);
    if (r == WISV_OK) ++c->launches;
    return r;
}

}  // extern "C"
