// Checks of arguments that the entry points of the 8-bit cache share (private, host).
#pragma once
#include "kv8.h"

namespace {

constexpr size_t ALIGN = 256;

#define HIP_TRY(x)                               \
    do {                                         \
        if ((x) != hipSuccess) return SSSD_EHIP; \
    } while (0)

struct Sizes8 {
    int blocks_per_seq, n_pages;
    size_t scales_at, layer_bytes, cache_bytes, ws_bytes;
};

[[maybe_unused]] int sizes8(const sssd_kv8_config *c, Sizes8 &S)
{
    if (!c || (c->format != SSSD_KV8_E4M3 && c->format != SSSD_KV8_INT8)) return SSSD_EINVAL;
    if (c->n_layers <= 0 || c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->max_batch <= 0 || c->max_seq <= 0 || c->n_pages < 0) return SSSD_EINVAL;
    if (c->head_dim != 64 && c->head_dim != 128) return SSSD_EINVAL;
    if (c->n_q_heads % c->n_kv_heads || c->n_q_heads / c->n_kv_heads > 64 || c->max_seq > INT32_MAX - 64) return SSSD_EINVAL;
    S.blocks_per_seq = (c->max_seq + KV8_BLOCK - 1) / KV8_BLOCK;
    const int64_t all = (int64_t)c->max_batch * S.blocks_per_seq;
    if (!c->n_pages && all > INT32_MAX) return SSSD_EINVAL;
    S.n_pages = c->n_pages ? c->n_pages : (int)all;
    // at most 2^31 pages x 2^31 heads: checked before they are multiplied by the bytes of a record
    size_t records = 0;
    if (__builtin_mul_overflow((size_t)S.n_pages, (size_t)c->n_kv_heads, &records) || records > SIZE_MAX / (64 * 128 + 8) - ALIGN) return SSSD_EINVAL;
    S.scales_at = records * 64 * c->head_dim;
    S.layer_bytes = (S.scales_at + records * sizeof(float2) + ALIGN - 1) / ALIGN * ALIGN;
    if (__builtin_mul_overflow(S.layer_bytes, (size_t)c->n_layers, &S.cache_bytes)) return SSSD_EINVAL;
    S.ws_bytes = kv8_attention_ws(c->head_dim);
    return SSSD_OK;
}

[[maybe_unused]] int check_cache(const sssd_kv8 *kv, int layer, Sizes8 &S)
{
    if (!kv) return SSSD_EINVAL;
    const int rc = sizes8(&kv->cfg, S);
    if (rc) return rc;
    if (!kv->cache || (uintptr_t)kv->cache % ALIGN || !kv->status || layer < 0 || layer >= kv->cfg.n_layers) return SSSD_EINVAL;
    if (!kv->block_table && (int64_t)S.n_pages < (int64_t)kv->cfg.max_batch * S.blocks_per_seq) return SSSD_EINVAL;
    if (kv->flags & ~SSSD_NO_WAIT) return SSSD_EINVAL;
    if (kv->cache_bytes < S.cache_bytes) return SSSD_ECAPACITY;
    return SSSD_OK;
}

[[maybe_unused]] Kv8Geom geom(const sssd_kv8 *kv, const Sizes8 &S) { return Kv8Geom{kv->block_table, S.blocks_per_seq, S.n_pages, kv->cfg.n_kv_heads, kv->cfg.max_seq}; }

// Strides of dimensions of one element play no part.
[[maybe_unused]] int make_rows(const sssd_rows *r, int B, int n, int heads, Rows8 &out)
{
    if (!r || !r->data || (r->type != SSSD_F32 && r->type != SSSD_BF16)) return SSSD_EINVAL;
    const int size = r->type == SSSD_BF16 ? 2 : 4;
    if ((uintptr_t)r->data % size) return SSSD_EINVAL;
    out.p = (char *)r->data;
    out.bs = B > 1 ? r->batch_stride : 0;
    out.rs = n > 1 ? r->row_stride : 0;
    out.hs = heads > 1 ? r->head_stride : 0;
    out.bf16 = r->type == SSSD_BF16;
    const int64_t per = 16 / size;
    out.vec = (uintptr_t)r->data % 16 == 0 && out.bs % per == 0 && out.rs % per == 0 && out.hs % per == 0;
    return SSSD_OK;
}

constexpr int64_t MOST_THREADS = ((int64_t)1 << 32) - 1;   // of a launch

}  // namespace
