// C entry points of the 8-bit cache of uncompressed layers: argument checks and dispatch.
#include "append8.cuh"
#include "sm100_ptx.cuh"
#include "tc_kernels.cuh"

namespace {

int fail8(lorc_ctx* ctx, int code, const char* msg) {
    ctx->err = msg;
    return code;
}

int fail8_cuda(lorc_ctx* ctx, cudaError_t e, const char* where) {
    ctx->err = std::string(where) + ": " + cudaGetErrorString(e);
    return LORC_ERR_CUDA;
}

int check8(lorc_ctx* ctx, int layer, const lorc_cache8* c, int T, const void* in, const void* out, Cache8View* cv) {
    if (layer < 0 || layer >= ctx->desc.n_layers) return fail8(ctx, LORC_ERR_LAYER, "layer index out of range");
    if (!ctx->layers[layer].loaded) return fail8(ctx, LORC_ERR_LAYER, "no factors loaded for this layer");
    if (ctx->layers[layer].mode != LORC_MODE_FULL)
        return fail8(ctx, LORC_ERR_UNSUPPORTED, "cache8: the layer is compressed; the 8-bit cache is for uncompressed layers");
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->seq_lens) return fail8(ctx, LORC_ERR_ARG, "cache8: null pointer");
    if (!in || !out) return fail8(ctx, LORC_ERR_ARG, "cache8: null input or output");
    if (((uintptr_t)in & 15) || ((uintptr_t)out & 15)) return fail8(ctx, LORC_ERR_ARG, "cache8: inputs and outputs must be 16-byte aligned");
    if (((uintptr_t)c->k & 15) || ((uintptr_t)c->v & 15)) return fail8(ctx, LORC_ERR_ARG, "cache8: k and v must be 16-byte aligned");
    if (((uintptr_t)c->k_scale & 3) || ((uintptr_t)c->v_scale & 3) || ((uintptr_t)c->seq_lens & 3) || ((uintptr_t)c->page_table & 3))
        return fail8(ctx, LORC_ERR_ARG, "cache8: scales, lengths and page table must be 4-byte aligned");
    if (c->type != LORC_CACHE8_INT8 && c->type != LORC_CACHE8_E4M3) return fail8(ctx, LORC_ERR_ARG, "cache8: unknown type");
    if (c->batch <= 0) return fail8(ctx, LORC_ERR_ARG, "cache8: batch must be positive");
    if (c->max_seq_len <= 0) return fail8(ctx, LORC_ERR_ARG, "cache8: max_seq_len must be positive");
    if (c->max_seq_len > ctx->desc.max_pos) return fail8(ctx, LORC_ERR_ARG, "cache8: max_seq_len exceeds the context's max_pos");
    long long capacity;
    if (c->page_table) {
        if (c->page_size <= 0 || c->page_size % LORC_CACHE8_BLOCK || c->max_pages_per_seq <= 0 || c->n_pages <= 0)
            return fail8(ctx, LORC_ERR_ARG, "cache8: bad paging parameters (page_size must be a positive multiple of 16)");
        capacity = (long long)c->page_size * c->max_pages_per_seq;
    } else {
        if (c->seq_stride <= 0 || c->seq_stride % LORC_CACHE8_BLOCK || c->seq_stride > 0x7fffffffll)
            return fail8(ctx, LORC_ERR_ARG, "cache8: seq_stride must be a positive multiple of 16");
        capacity = c->seq_stride;
    }
    if (c->max_seq_len > capacity) return fail8(ctx, LORC_ERR_ARG, "cache8: max_seq_len exceeds the cache capacity");
    if (T <= 0 || T > c->max_seq_len) return fail8(ctx, LORC_ERR_ARG, "cache8: T must be positive and not exceed max_seq_len");
    if ((long long)c->batch * T > 0x3fffffffll) return fail8(ctx, LORC_ERR_ARG, "cache8: batch * T is too large");
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return fail8_cuda(ctx, e, "cache8");
    if (dev != ctx->device) return fail8(ctx, LORC_ERR_ARG, "cache8: the context's device is not the current one");
    cv->k = (uint8_t*)c->k;
    cv->v = (uint8_t*)c->v;
    cv->k_scale = c->k_scale;
    cv->v_scale = c->v_scale;
    cv->page_table = c->page_table;
    cv->seq_lens = c->seq_lens;
    cv->batch = c->batch;
    cv->max_seq_len = c->max_seq_len;
    cv->page_size = c->page_table ? c->page_size : 0;
    cv->max_pages_per_seq = c->max_pages_per_seq;
    cv->n_pages = c->n_pages;
    cv->type = c->type;
    cv->n = ctx->n;
    cv->n_kv = ctx->desc.n_kv_heads;
    cv->seq_stride = c->seq_stride;
    cv->capacity = capacity;
    return LORC_OK;
}

int attend8(lorc_ctx* ctx, int layer, const lorc_cache8* cache, const void* q, void* out, int T, void* stream, const char* name) {
    if (!ctx) return LORC_ERR_ARG;
    Cache8View cv;
    const int rc = check8(ctx, layer, cache, T, q, out, &cv);
    if (rc) return rc;
    const bool expand = lorc_prefill8_supported(ctx, cv, T);
    if (!expand && !lorc_decode8_fits(ctx, cv, T)) return fail8(ctx, LORC_ERR_ARG, "cache8: batch * max_seq_len is too large (2^30 units of 64 tokens)");
    if (!lorc_get_tmap_encode()) return fail8(ctx, LORC_ERR_CUDA, "cache8: the driver offers no tensor maps");
    const size_t need = expand ? lorc_prefill8_scratch_bytes(ctx, cv.batch, cv.max_seq_len, T)
                               : lorc_decode8_scratch_bytes(ctx, cv.batch, cv.max_seq_len, T);
    if (!ctx->ws || need > ctx->ws_bytes)
        return fail8(ctx, LORC_ERR_WORKSPACE, "cache8: workspace missing or too small (see lorc_cache8_workspace_bytes)");
    int launches = 0;
    cudaError_t e;
    if (expand) {
        LorcStageTimer timer(ctx, LORC_STAGE_SCORE, (cudaStream_t)stream);
        e = lorc_prefill8_launch(ctx, cv, (const bf16*)q, (bf16*)out, T, ctx->ws, (cudaStream_t)stream, &launches);
    } else {
        e = lorc_decode8_launch(ctx, cv, (const bf16*)q, (bf16*)out, T, ctx->ws, (cudaStream_t)stream, &launches);
    }
    ctx->launches += launches;
    ctx->last_path = expand ? 2 : 3;
    return e == cudaSuccess ? LORC_OK : fail8_cuda(ctx, e, name);
}

}  // namespace

extern "C" {

size_t lorc_cache8_workspace_bytes(const lorc_ctx* ctx, int batch, int max_seq_len, int T) {
    if (!ctx || batch <= 0 || max_seq_len <= 0 || T <= 0) return 0;
    size_t need = lorc_append8_scratch_most(ctx, batch, T);
    const size_t d = lorc_decode8_scratch_bytes(ctx, batch, max_seq_len, T);
    if (d > need) need = d;
    if (T > 1 && !(ctx->desc.flags & LORC_FLAG_DEBUG_FP32)) {
        const size_t f = lorc_prefill8_scratch_most(ctx, batch, max_seq_len, T);
        if (f > need) need = f;
    }
    return need;
}

int lorc_append8(lorc_ctx* ctx, int layer, const lorc_cache8* cache, const void* x, int T, void* stream) {
    if (!ctx) return LORC_ERR_ARG;
    Cache8View cv;
    const int rc = check8(ctx, layer, cache, T, x, cache ? cache->k : nullptr, &cv);
    if (rc) return rc;
    if (!ctx->ws || lorc_append8_scratch_bytes(ctx, cv.batch, T) > ctx->ws_bytes)
        return fail8(ctx, LORC_ERR_WORKSPACE, "append8: workspace missing or too small (see lorc_cache8_workspace_bytes)");
    int launches = 0;
    LorcStageTimer timer(ctx, LORC_STAGE_APPEND, (cudaStream_t)stream);
    const cudaError_t e = lorc_append8_launch(ctx, ctx->layers[layer], cv, (const bf16*)x, T, ctx->ws, (cudaStream_t)stream, &launches);
    ctx->launches += launches;
    ctx->last_path = lorc_append8_way(ctx, cv.batch, T) != APPEND8_MMA ? 2 : ctx->desc.flags & LORC_FLAG_DEBUG_FP32 ? 1 : 3;
    return e == cudaSuccess ? LORC_OK : fail8_cuda(ctx, e, "lorc_append8");
}

int lorc_decode_attn8(lorc_ctx* ctx, int layer, const lorc_cache8* cache, const void* q, void* out, void* stream) {
    return attend8(ctx, layer, cache, q, out, 1, stream, "lorc_decode_attn8");
}

int lorc_prefill_attn8(lorc_ctx* ctx, int layer, const lorc_cache8* cache, const void* q, void* out, int T, void* stream) {
    return attend8(ctx, layer, cache, q, out, T, stream, "lorc_prefill_attn8");
}

}  // extern "C"
