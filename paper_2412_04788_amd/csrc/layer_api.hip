// C ABI of the layer operators: checks of the specs, stream order, launches.
#include <cmath>

#include "context.hpp"
#include "guide_layer.h"
#include "layer_kernels.hpp"

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
size_t elem_bytes(uint32_t type) { return type == GUIDE_F32 ? 4 : 2; }
bool elem_aligned(const void *p, uint32_t type) { return (uintptr_t)p % elem_bytes(type) == 0; }

// A stride between rows that there is only one of means nothing: it becomes the row's width.
void one_row(uint64_t rows, int64_t &stride, uint64_t width) {
    if (rows == 1) stride = (int64_t)width;
}

// A row-major typed tensor's pointer and row stride.
int check_rows(guide_ctx *ctx, const char *name, const void *p, uint32_t type, int64_t stride, uint64_t width) {
    if (!p) return fail(ctx, GUIDE_E_ARG, "%s is NULL", name);
    if (!elem_aligned(p, type)) return fail(ctx, GUIDE_E_ARG, "%s is not aligned to its type", name);
    if (stride < 0 || (uint64_t)stride < width) return fail(ctx, GUIDE_E_ARG, "%s: row stride below the row's %llu elements", name, (unsigned long long)width);
    if (stride > INT32_MAX) return fail(ctx, GUIDE_E_RANGE, "%s: row stride above 2^31 - 1", name);
    return GUIDE_OK;
}

// Code and scale buffers of rows of `groups` groups.
int check_codes(guide_ctx *ctx, const char *name, const uint8_t *codes, const uint8_t *scales, int64_t codes_stride, int64_t scales_stride,
                uint32_t bits, uint64_t groups) {
    if (!codes || !scales) return fail(ctx, GUIDE_E_ARG, "%s: codes or scales are NULL", name);
    if (!aligned16(codes) || codes_stride % 16 != 0) return fail(ctx, GUIDE_E_ARG, "%s: codes and their stride must be multiples of 16 bytes", name);
    if (codes_stride < 0 || (uint64_t)codes_stride < groups * bits * 4 || scales_stride < 0 || (uint64_t)scales_stride < groups)
        return fail(ctx, GUIDE_E_ARG, "%s: stride below the row's %llu groups", name, (unsigned long long)groups);
    return GUIDE_OK;
}

// q, k, v or out of the attentions: [tokens][heads][d] with two strides.
int check_heads(guide_ctx *ctx, const char *name, const void *p, int64_t stride, int64_t head_stride, uint32_t heads, uint32_t d) {
    if (!p) return fail(ctx, GUIDE_E_ARG, "%s is NULL", name);
    if (!elem_aligned(p, GUIDE_BF16)) return fail(ctx, GUIDE_E_ARG, "%s is not aligned to its type", name);
    if (stride < d || (heads > 1 && head_stride < d)) return fail(ctx, GUIDE_E_ARG, "%s: a stride is below the head's %u channels", name, d);
    if (stride > (1 << 24) || head_stride > INT32_MAX) return fail(ctx, GUIDE_E_RANGE, "%s: token stride above 2^24 or head stride above 2^31 - 1", name);
    return GUIDE_OK;
}

// Ready to launch on `stream` of the context's device.
int begin(guide_ctx *ctx, const DeviceGuard &guard, hipStream_t stream) {
    if (!guard.ok) return fail(ctx, GUIDE_E_DEVICE, "cannot make device %d current", ctx->device);
    return order_after_previous(ctx, stream);
}

int launched(guide_ctx *ctx, hipError_t e, const char *what) { return e == hipSuccess ? GUIDE_OK : hip_fail(ctx, e, what); }

#define GUIDE_TRY(call)                 \
    do {                                \
        const int rc_ = (call);         \
        if (rc_) return rc_;            \
    } while (0)

int check_16bit(guide_ctx *ctx, uint32_t type) {
    return type == GUIDE_BF16 || type == GUIDE_F16 ? GUIDE_OK : fail(ctx, GUIDE_E_ARG, "type %u is neither GUIDE_BF16 nor GUIDE_F16", type);
}

int check_quant(guide_ctx *ctx, uint32_t type, uint32_t bits) {
    if (type > GUIDE_F32) return fail(ctx, GUIDE_E_ARG, "unknown type %u", type);
    if (bits != 4 && bits != 8) return fail(ctx, GUIDE_E_ARG, "codes of %u bits: 4 or 8", bits);
    return GUIDE_OK;
}

int check_groups(guide_ctx *ctx, uint32_t rows, uint64_t groups) {
    if (rows * groups >= (1ull << 30)) return fail(ctx, GUIDE_E_RANGE, "2^30 or more groups");
    return GUIDE_OK;
}

int check_scale(guide_ctx *ctx, float scale) {
    return std::isfinite(scale) && scale > 0.0f ? GUIDE_OK : fail(ctx, GUIDE_E_ARG, "scale must be finite and above zero");
}

int check_group_heads(guide_ctx *ctx, uint32_t n_h, uint32_t n_kv, uint32_t d) {
    if (n_h == 0 || n_kv == 0 || n_h % n_kv != 0) return fail(ctx, GUIDE_E_ARG, "%u query heads over %u KV heads", n_h, n_kv);
    if (n_h > 65535) return fail(ctx, GUIDE_E_RANGE, "more than 65535 heads");
    if (d != 64 && d != 128) return fail(ctx, GUIDE_E_RANGE, "head dimension %u: 64 or 128", d);
    return GUIDE_OK;
}

int check_cache(guide_ctx *ctx, const guide_cache *c) {
    if (!c) return fail(ctx, GUIDE_E_ARG, "cache is NULL");
    if (c->n_kv == 0 || c->n_kv > 65535) return fail(ctx, c->n_kv ? GUIDE_E_RANGE : GUIDE_E_ARG, "%u KV heads", c->n_kv);
    if (c->d != 64 && c->d != 128) return fail(ctx, GUIDE_E_RANGE, "head dimension %u: 64 or 128", c->d);
    if (c->kv_block == 0 || c->kv_block % 16 != 0 || c->kv_block > 1024)
        return fail(ctx, GUIDE_E_RANGE, "pages of %u tokens: a multiple of 16, at most 1024", c->kv_block);
    if (c->n_pages > INT32_MAX) return fail(ctx, GUIDE_E_RANGE, "2^31 or more pages");
    if (c->n_pages && (!c->codes || !c->scales)) return fail(ctx, GUIDE_E_ARG, "the cache's codes or scales are NULL");
    if (!aligned16(c->codes) || !aligned16(c->scales)) return fail(ctx, GUIDE_E_ARG, "the cache's codes and scales must be 16-byte aligned");
    return GUIDE_OK;
}

int cache_tokens(guide_ctx *ctx, const guide_cache *cache, const guide_cache_tokens *asked, void *stream, bool read) {
    if (!ctx) return GUIDE_E_ARG;
    GUIDE_TRY(check_cache(ctx, cache));
    if (!asked) return fail(ctx, GUIDE_E_ARG, "tokens is NULL");
    guide_cache_tokens spec = *asked, *const t = &spec;
    one_row(t->tokens, t->k_stride, cache->d);
    one_row(t->tokens, t->v_stride, cache->d);
    GUIDE_TRY(check_16bit(ctx, t->type));
    if (t->tokens == 0) return GUIDE_OK;
    if (t->tokens > INT32_MAX) return fail(ctx, GUIDE_E_RANGE, "2^31 or more tokens");
    GUIDE_TRY(check_heads(ctx, "k", t->k, t->k_stride, t->k_head_stride, cache->n_kv, cache->d));
    GUIDE_TRY(check_heads(ctx, "v", t->v, t->v_stride, t->v_head_stride, cache->n_kv, cache->d));
    if (!t->slots) return fail(ctx, GUIDE_E_ARG, "slots is NULL");
    DeviceGuard guard(ctx->device);
    GUIDE_TRY(begin(ctx, guard, (hipStream_t)stream));
    return launched(ctx, read ? launch_cache_read(*cache, *t, (hipStream_t)stream) : launch_cache_append(*cache, *t, (hipStream_t)stream),
                    read ? "cache read launch" : "cache append launch");
}

}  // namespace

extern "C" {

int guide_quantise(guide_ctx *ctx, const guide_quantise_spec *asked, void *stream) {
    if (!ctx) return GUIDE_E_ARG;
    if (!asked) return fail(ctx, GUIDE_E_ARG, "spec is NULL");
    guide_quantise_spec spec = *asked, *const s = &spec;
    one_row(s->rows, s->x_stride, s->cols);
    one_row(s->rows, s->codes_stride, ((uint64_t)s->cols + 31) / 32 * s->bits * 4);
    one_row(s->rows, s->scales_stride, ((uint64_t)s->cols + 31) / 32);
    GUIDE_TRY(check_quant(ctx, s->type, s->bits));
    if (s->rows == 0 || s->cols == 0) return GUIDE_OK;
    if (s->cols > INT32_MAX - 64) return fail(ctx, GUIDE_E_RANGE, "2^31 - 64 or more columns");
    const uint64_t groups = ((uint64_t)s->cols + 31) / 32;
    GUIDE_TRY(check_groups(ctx, s->rows, groups));
    GUIDE_TRY(check_rows(ctx, "x", s->x, s->type, s->x_stride, s->cols));
    GUIDE_TRY(check_codes(ctx, "output", s->codes, s->scales, s->codes_stride, s->scales_stride, s->bits, groups));
    DeviceGuard guard(ctx->device);
    GUIDE_TRY(begin(ctx, guard, (hipStream_t)stream));
    return launched(ctx, launch_quantise(*s, (hipStream_t)stream), "quantise launch");
}

int guide_rms_norm(guide_ctx *ctx, const guide_norm_spec *asked, void *stream) {
    if (!ctx) return GUIDE_E_ARG;
    if (!asked) return fail(ctx, GUIDE_E_ARG, "spec is NULL");
    guide_norm_spec spec = *asked, *const s = &spec;
    one_row(s->rows, s->x_stride, s->d);
    one_row(s->rows, s->residual_stride, s->d);
    one_row(s->rows, s->total_stride, s->d);
    one_row(s->rows, s->codes_stride, ((uint64_t)s->d + 31) / 32 * s->bits * 4);
    one_row(s->rows, s->scales_stride, ((uint64_t)s->d + 31) / 32);
    GUIDE_TRY(check_quant(ctx, s->type, s->bits));
    if (!(s->eps >= 0.0f) || !std::isfinite(s->eps)) return fail(ctx, GUIDE_E_ARG, "eps must be finite and not negative");
    if (s->d > GUIDE_NORM_MAX_WIDTH) return fail(ctx, GUIDE_E_RANGE, "width %u above %d", s->d, GUIDE_NORM_MAX_WIDTH);
    if (s->rows == 0 || s->d == 0) return GUIDE_OK;
    const uint64_t groups = (s->d + 31u) / 32u;
    GUIDE_TRY(check_groups(ctx, s->rows, groups));
    GUIDE_TRY(check_rows(ctx, "x", s->x, s->type, s->x_stride, s->d));
    if (s->residual) GUIDE_TRY(check_rows(ctx, "residual", s->residual, s->type, s->residual_stride, s->d));
    if (s->total) GUIDE_TRY(check_rows(ctx, "total", s->total, s->type, s->total_stride, s->d));
    if (!s->weight || !elem_aligned(s->weight, s->type)) return fail(ctx, GUIDE_E_ARG, "weight is NULL or not aligned to its type");
    GUIDE_TRY(check_codes(ctx, "output", s->codes, s->scales, s->codes_stride, s->scales_stride, s->bits, groups));
    DeviceGuard guard(ctx->device);
    GUIDE_TRY(begin(ctx, guard, (hipStream_t)stream));
    return launched(ctx, launch_norm(*s, (hipStream_t)stream), "norm launch");
}

int guide_product(guide_ctx *ctx, const guide_product_spec *asked, void *stream) {
    if (!ctx) return GUIDE_E_ARG;
    if (!asked) return fail(ctx, GUIDE_E_ARG, "spec is NULL");
    guide_product_spec spec = *asked, *const s = &spec;
    one_row(s->m, s->a_codes_stride, (uint64_t)s->k / 32 * s->a_bits * 4);
    one_row(s->m, s->a_scales_stride, s->k / 32);
    one_row(s->n, s->w_codes_stride, s->k / 2);
    one_row(s->n, s->w_scales_stride, s->k / 32);
    one_row(s->m, s->out_stride, s->n);
    GUIDE_TRY(check_quant(ctx, s->type, s->a_bits));
    if (s->type == GUIDE_F32 && s->a_bits == 8)
        return fail(ctx, GUIDE_E_ARG, "8-bit activations into 32 bits: the matrix unit does not hold those sums to 32 bits");
    if (s->k % GUIDE_MX_GROUP != 0) return fail(ctx, GUIDE_E_ARG, "k = %u is no multiple of %d", s->k, GUIDE_MX_GROUP);
    if (s->m > GUIDE_PRODUCT_MAX || s->n > GUIDE_PRODUCT_MAX || s->k > GUIDE_PRODUCT_MAX)
        return fail(ctx, GUIDE_E_RANGE, "m, n or k above %d", GUIDE_PRODUCT_MAX);
    if (s->m == 0 || s->n == 0) return GUIDE_OK;
    GUIDE_TRY(check_rows(ctx, "out", s->out, s->type, s->out_stride, s->n));
    if (s->k) {
        GUIDE_TRY(check_codes(ctx, "a", s->a_codes, s->a_scales, s->a_codes_stride, s->a_scales_stride, s->a_bits, s->k / 32));
        GUIDE_TRY(check_codes(ctx, "w", s->w_codes, s->w_scales, s->w_codes_stride, s->w_scales_stride, 4, s->k / 32));
        if (s->a_codes_stride > INT32_MAX || s->a_scales_stride > INT32_MAX || s->w_codes_stride > INT32_MAX || s->w_scales_stride > INT32_MAX)
            return fail(ctx, GUIDE_E_RANGE, "a stride above 2^31 - 1");
    }
    DeviceGuard guard(ctx->device);
    GUIDE_TRY(begin(ctx, guard, (hipStream_t)stream));
    return launched(ctx, launch_product(*s, ctx->layer_scratch, (hipStream_t)stream), "product launch");
}

int guide_prompt_attention(guide_ctx *ctx, const guide_prompt_spec *asked, void *stream) {
    if (!ctx) return GUIDE_E_ARG;
    if (!asked) return fail(ctx, GUIDE_E_ARG, "spec is NULL");
    guide_prompt_spec spec = *asked, *const s = &spec;
    one_row(s->total_q, s->q_stride, s->d);
    one_row(s->total_q, s->out_stride, s->d);
    one_row(s->total_k, s->k_stride, s->d);
    one_row(s->total_k, s->v_stride, s->d);
    GUIDE_TRY(check_16bit(ctx, s->type));
    GUIDE_TRY(check_group_heads(ctx, s->n_h, s->n_kv, s->d));
    GUIDE_TRY(check_scale(ctx, s->scale));
    if (s->n_seq == 0 || s->total_q == 0) return GUIDE_OK;
    if (s->total_q > (1u << 30) || s->total_k > (1u << 30) || s->n_seq > (1u << 20))
        return fail(ctx, GUIDE_E_RANGE, "more than 2^30 queries or keys, or 2^20 sequences");
    if (!s->q_starts || !s->k_starts) return fail(ctx, GUIDE_E_ARG, "q_starts or k_starts is NULL");
    GUIDE_TRY(check_heads(ctx, "q", s->q, s->q_stride, s->q_head_stride, s->n_h, s->d));
    GUIDE_TRY(check_heads(ctx, "out", s->out, s->out_stride, s->out_head_stride, s->n_h, s->d));
    if (s->total_k) {
        GUIDE_TRY(check_heads(ctx, "k", s->k, s->k_stride, s->k_head_stride, s->n_kv, s->d));
        GUIDE_TRY(check_heads(ctx, "v", s->v, s->v_stride, s->v_head_stride, s->n_kv, s->d));
    }
    DeviceGuard guard(ctx->device);
    GUIDE_TRY(begin(ctx, guard, (hipStream_t)stream));
    return launched(ctx, launch_prompt_attention(*s, ctx->layer_scratch, (hipStream_t)stream), "prompt attention launch");
}

int guide_cache_append(guide_ctx *ctx, const guide_cache *cache, const guide_cache_tokens *tokens, void *stream) {
    return cache_tokens(ctx, cache, tokens, stream, false);
}

int guide_cache_read(guide_ctx *ctx, const guide_cache *cache, const guide_cache_tokens *tokens, void *stream) {
    return cache_tokens(ctx, cache, tokens, stream, true);
}

size_t guide_cache_attention_workspace_bytes(uint32_t n_seq, uint32_t n_h, uint32_t n_kv, uint32_t d, uint64_t max_len) {
    if (n_seq == 0 || n_h == 0 || n_kv == 0 || n_h % n_kv != 0) return 0;
    return cache_attention_workspace(n_seq, n_h, n_kv, d, max_len);
}

int guide_cache_attention(guide_ctx *ctx, const guide_cache *cache, const guide_cache_queries *asked, void *workspace, size_t workspace_bytes,
                          void *stream) {
    if (!ctx) return GUIDE_E_ARG;
    GUIDE_TRY(check_cache(ctx, cache));
    if (!asked) return fail(ctx, GUIDE_E_ARG, "queries is NULL");
    guide_cache_queries spec = *asked, *const s = &spec;
    one_row(s->n_seq, s->q_stride, cache->d);
    one_row(s->n_seq, s->out_stride, cache->d);
    one_row(s->n_seq, s->pages_stride, s->max_pages);
    GUIDE_TRY(check_16bit(ctx, s->type));
    GUIDE_TRY(check_group_heads(ctx, s->n_h, cache->n_kv, cache->d));
    GUIDE_TRY(check_scale(ctx, s->scale));
    if (s->n_seq == 0) return GUIDE_OK;
    const uint64_t max_len = (uint64_t)s->max_pages * cache->kv_block;
    if (s->n_seq > 65535 || max_len > (1u << 30)) return fail(ctx, GUIDE_E_RANGE, "more than 65535 sequences, or tables of more than 2^30 tokens");
    if ((uint64_t)s->n_seq * s->n_h > INT32_MAX / 64) return fail(ctx, GUIDE_E_RANGE, "more than 2^25 rows of queries");
    GUIDE_TRY(check_heads(ctx, "q", s->q, s->q_stride, s->q_head_stride, s->n_h, cache->d));
    GUIDE_TRY(check_heads(ctx, "out", s->out, s->out_stride, s->out_head_stride, s->n_h, cache->d));
    if (!s->lengths || (s->max_pages && !s->pages)) return fail(ctx, GUIDE_E_ARG, "pages or lengths is NULL");
    if (s->pages_stride < s->max_pages) return fail(ctx, GUIDE_E_ARG, "pages: row stride below max_pages");
    const size_t need = cache_attention_workspace(s->n_seq, s->n_h, cache->n_kv, cache->d, max_len);
    if (need && !workspace) return fail(ctx, GUIDE_E_ARG, "workspace is NULL");
    if (workspace_bytes < need) return fail(ctx, GUIDE_E_NOMEM, "workspace has %zu bytes, %zu are needed", workspace_bytes, need);
    if ((uintptr_t)workspace % 4 != 0) return fail(ctx, GUIDE_E_ARG, "the workspace must be 4-byte aligned");
    DeviceGuard guard(ctx->device);
    GUIDE_TRY(begin(ctx, guard, (hipStream_t)stream));
    return launched(ctx, launch_cache_attention(*cache, *s, workspace, (hipStream_t)stream), "cache attention launch");
}

}  // extern "C"
