// C ABI of one decoding step over a paged key-value cache: argument checks of the operators whose kernels are in kv_plan.cu,
// qk_rope.cu, attention_paged.cu and linear_w4.cu.
#include <math.h>

#include "nm_common.cuh"

namespace {

nm_status need_table(const nm_ctx* ctx, int slot)
{
    if (slot < 0 || slot >= NM_NUM_SLOTS) return NM_ERR_INVALID_ARG;
    return ctx->h_tables[slot].loaded ? NM_OK : NM_ERR_NO_TABLE;
}

bool float_type(nm_dtype t) { return t == NM_F32 || t == NM_BF16 || t == NM_F16; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
bool rows16(int64_t stride, size_t es) { return (stride * (int64_t)es) % 16 == 0; }

// Counts of requests, tokens and pages, and elements of a token's row: the kernels step through them in 32 bits, some thousands at a time.
constexpr int64_t DECODE_MAX = 1 << 30;

// The distances of a cache's pages, tokens and heads: none negative, 16-byte rows (or a distance that is never used).
nm_status check_cache(int32_t num_pages, int32_t page_size, int64_t sp, int64_t st, int64_t sh, size_t es)
{
    if (num_pages < 1 || page_size < 1 || (int64_t)num_pages * page_size > INT32_MAX) return NM_ERR_SHAPE;
    if (sp < 0 || st < 0 || sh < 0) return NM_ERR_SHAPE;
    return rows16(sp, es) && rows16(st, es) && rows16(sh, es) ? NM_OK : NM_ERR_ALIGNMENT;
}

nm_status check_attn_paged(const nm_attn_paged_desc* d)
{
    if (d->B < 0 || d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads || d->max_len < 0) return NM_ERR_SHAPE;
    if (d->B > DECODE_MAX || d->max_len > DECODE_MAX || (int64_t)d->heads * d->d > DECODE_MAX) return NM_ERR_SHAPE;
    if ((double)d->B * d->heads * d->max_len > 1e15) return NM_ERR_SHAPE;   // the workspace's size fits 64 bits
    if (!float_type(d->dtype)) return NM_ERR_UNSUPPORTED;
    if (d->d < 8 || d->d > 256 || d->d % 8) return NM_ERR_SHAPE;
    if (d->max_pages < 0 || d->page_size < 1 || d->max_len > (int64_t)d->max_pages * d->page_size) return NM_ERR_SHAPE;
    return check_cache(d->num_pages, d->page_size, d->stride_page, d->stride_token, d->stride_head, nm_dtype_size(d->dtype));
}

}  // namespace

extern "C" {

nm_status nm_kv_plan(nm_ctx* ctx, const nm_kv_plan_desc* d, void* stream)
{
    if (!ctx || !d) return NM_ERR_INVALID_ARG;
    if (d->B < 0 || d->page_size < 1 || d->max_pages < 0 || d->max_tokens < 0 || d->free_capacity < 0) return NM_ERR_SHAPE;
    if (d->B > DECODE_MAX || d->max_tokens > DECODE_MAX || d->free_capacity > DECODE_MAX) return NM_ERR_SHAPE;
    if ((int64_t)d->max_pages * d->page_size > INT32_MAX || d->ld_tables < d->max_pages) return NM_ERR_SHAPE;
    if (!d->free_count || !d->free_count_out || !d->token_start) return NM_ERR_INVALID_ARG;
    if (d->B > 0 && (!d->lengths || !d->new_tokens || !d->lengths_out)) return NM_ERR_INVALID_ARG;
    if (d->B > 0 && d->max_pages > 0 && !d->block_tables) return NM_ERR_INVALID_ARG;
    if (d->free_capacity > 0 && !d->free_pages) return NM_ERR_INVALID_ARG;
    if (d->max_tokens > 0 && (!d->slots || !d->positions)) return NM_ERR_INVALID_ARG;
    const void* arrays[] = {d->lengths, d->new_tokens, d->free_count, d->block_tables, d->free_pages, d->lengths_out, d->free_count_out,
                            d->token_start, d->slots, d->positions};
    for (const void* p : arrays)
        if (!aligned4(p)) return NM_ERR_ALIGNMENT;
    NmDeviceScope device(ctx);
    return device.ok ? nm_launch_kv_plan(ctx, d, (cudaStream_t)stream) : NM_ERR_CUDA;
}

nm_status nm_qk_norm_rope_pwl(nm_ctx* ctx, const nm_qk_rope_desc* d, void* stream)
{
    if (!ctx || !d) return NM_ERR_INVALID_ARG;
    if (d->T < 0 || d->T > DECODE_MAX || d->heads < 0 || d->kv_heads < 0 || (int64_t)d->heads + 2 * (int64_t)d->kv_heads > INT32_MAX) return NM_ERR_SHAPE;
    if (!float_type(d->dtype)) return NM_ERR_UNSUPPORTED;
    if (d->d < 8 || d->d > 256 || d->d % 8) return NM_ERR_SHAPE;
    if (d->rot < 0 || d->rot > d->d || d->rot % (d->pairs ? 8 : 16)) return NM_ERR_SHAPE;
    if ((d->gamma_q || d->gamma_k) && (d->rsqrt_slot < 0 || d->rsqrt_slot >= NM_NUM_SLOTS)) return NM_ERR_INVALID_ARG;
    if (nm_qk_rope_norms(d)) {
        const nm_status s = need_table(ctx, d->rsqrt_slot);
        if (s != NM_OK) return s;
    }
    if (d->T == 0 || (d->heads == 0 && d->kv_heads == 0)) return NM_OK;
    const int64_t row = ((int64_t)d->heads + 2 * (int64_t)d->kv_heads) * d->d;
    if (row > DECODE_MAX) return NM_ERR_SHAPE;
    if (!d->qkv || (d->heads > 0 && !d->q_out)) return NM_ERR_INVALID_ARG;
    if (d->ld_qkv < row || (d->heads > 0 && d->ld_q < (int64_t)d->heads * d->d)) return NM_ERR_SHAPE;
    if (d->k_out && d->ld_k < (int64_t)d->kv_heads * d->d) return NM_ERR_SHAPE;
    if (!d->k_cache != !d->v_cache || (d->k_cache && !d->slots)) return NM_ERR_INVALID_ARG;
    if (d->rot > 0 && (!d->positions || !d->cos_sin)) return NM_ERR_INVALID_ARG;
    if (d->rot > 0 && d->max_position < 1) return NM_ERR_SHAPE;
    const size_t es = nm_dtype_size(d->dtype);
    if (d->k_cache) {
        const nm_status s = check_cache(d->num_pages, d->page_size, d->stride_page, d->stride_token, d->stride_head, es);
        if (s != NM_OK) return s;
    }
    if (!nm_aligned16(d->qkv) || !nm_aligned16(d->q_out) || !nm_aligned16(d->k_out) || !nm_aligned16(d->k_cache) ||
        !nm_aligned16(d->v_cache) || !nm_aligned16(d->cos_sin) || !nm_aligned16(d->gamma_q) || !nm_aligned16(d->gamma_k) ||
        !aligned4(d->positions) || !aligned4(d->slots))
        return NM_ERR_ALIGNMENT;
    if (!rows16(d->ld_qkv, es) || (d->heads > 0 && !rows16(d->ld_q, es)) || (d->k_out && !rows16(d->ld_k, es))) return NM_ERR_ALIGNMENT;
    NmDeviceScope device(ctx);
    return device.ok ? nm_launch_qk_rope(ctx, d, (cudaStream_t)stream) : NM_ERR_CUDA;
}

size_t nm_attention_paged_workspace_bytes(const nm_attn_paged_desc* d)
{
    return d && check_attn_paged(d) == NM_OK ? nm_attention_paged_bytes(d) : 0;
}

nm_status nm_attention_pwl_paged(nm_ctx* ctx, const nm_attn_paged_desc* d, void* workspace, size_t ws_bytes, void* stream)
{
    if (!ctx || !d) return NM_ERR_INVALID_ARG;
    nm_status s = check_attn_paged(d);
    if (s != NM_OK) return s;
    s = need_table(ctx, d->exp_slot);
    if (s != NM_OK) return s;
    s = need_table(ctx, d->recip_slot);
    if (s != NM_OK) return s;
    if (!(d->scale > 0.0f) || !isfinite(d->scale)) return NM_ERR_INVALID_ARG;
    if (d->token_start && (d->rows < 0 || d->rows > DECODE_MAX)) return NM_ERR_SHAPE;
    if (d->B == 0 || (d->token_start && d->rows == 0)) return NM_OK;
    if (!d->Q || !d->k_cache || !d->v_cache || !d->lengths || !d->out || (d->max_pages > 0 && !d->block_tables)) return NM_ERR_INVALID_ARG;
    const size_t es = nm_dtype_size(d->dtype);
    const int64_t row = (int64_t)d->heads * d->d;
    if (d->ld_q < row || d->ld_out < row || d->ld_tables < d->max_pages) return NM_ERR_SHAPE;
    if (!nm_aligned16(d->Q) || !nm_aligned16(d->k_cache) || !nm_aligned16(d->v_cache) || !nm_aligned16(d->out) ||
        !aligned4(d->block_tables) || !aligned4(d->lengths) || !aligned4(d->token_start) || !rows16(d->ld_q, es) || !rows16(d->ld_out, es))
        return NM_ERR_ALIGNMENT;
    const size_t need = nm_attention_paged_bytes(d);
    if (need > 0 && (!workspace || ws_bytes < need)) return NM_ERR_WORKSPACE;
    if (need > 0 && ((uintptr_t)workspace & 255u)) return NM_ERR_ALIGNMENT;
    NmDeviceScope device(ctx);
    return device.ok ? nm_launch_attention_paged(ctx, d, workspace, (cudaStream_t)stream) : NM_ERR_CUDA;
}

nm_status nm_linear_pwl_w4(nm_ctx* ctx, const nm_linear_w4_desc* d, void* stream)
{
    if (!ctx || !d) return NM_ERR_INVALID_ARG;
    if (d->M < 0 || d->N < 0 || d->K < 0 || d->M > DECODE_MAX || d->N > DECODE_MAX || d->K > DECODE_MAX) return NM_ERR_SHAPE;
    if (!float_type(d->dtype)) return NM_ERR_UNSUPPORTED;
    if (d->group != 32 && d->group != 64 && d->group != 128) return NM_ERR_UNSUPPORTED;
    if (d->slot != NM_SLOT_NONE) {
        const nm_status s = need_table(ctx, d->slot);
        if (s != NM_OK) return s;
    }
    if (d->M == 0 || d->N == 0) return NM_OK;
    if (d->K == 0 || d->K % d->group) return NM_ERR_SHAPE;
    if (!d->A || !d->codes || !d->scales || !d->out) return NM_ERR_INVALID_ARG;
    if (d->lda < d->K || d->ld_codes < d->K / 2 || d->ld_scales < d->K / d->group || d->ldo < d->N || (d->residual && d->ldr < d->N))
        return NM_ERR_SHAPE;
    const size_t es = nm_dtype_size(d->dtype);
    if (!nm_aligned16(d->A) || !nm_aligned16(d->codes) || !nm_aligned16(d->out) || !nm_aligned16(d->residual) || !aligned4(d->bias) ||
        ((uintptr_t)d->scales & (es - 1)))
        return NM_ERR_ALIGNMENT;
    if (!rows16(d->lda, es) || d->ld_codes % 16 || !rows16(d->ldo, es) || (d->residual && !rows16(d->ldr, es))) return NM_ERR_ALIGNMENT;
    NmDeviceScope device(ctx);
    return device.ok ? nm_launch_linear_w4(ctx, d, (cudaStream_t)stream) : NM_ERR_CUDA;
}

}  // extern "C"
