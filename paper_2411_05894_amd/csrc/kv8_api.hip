// C ABI of the 8-bit KV cache and of rotary positions (include/sssd_kv8.h): checks of arguments, and launches.
#include "kv8_host.h"

#include <cmath>

namespace {

bool make_rope(const sssd_rope *r, int head_dim, Rope8 &out)
{
    if (!r->turns || r->rotary_dims < 2 || r->rotary_dims % 2 || r->rotary_dims > head_dim || r->rotary_dims > 2 * ROPE_TABLE) return false;
    if (r->pairs != SSSD_ROPE_HALVES && r->pairs != SSSD_ROPE_NEIGHBOURS) return false;
    out = Rope8{r->turns, r->rotary_dims, r->pairs == SSSD_ROPE_NEIGHBOURS, r->magnitude, Div(r->rotary_dims / 2)};
    return true;
}

}  // namespace

extern "C" {

int sssd_kv8_sizes(const sssd_kv8_config *cfg, size_t *cache_bytes, size_t *ws_bytes, int32_t *blocks_per_seq, int32_t *n_pages)
{
    Sizes8 S;
    const int rc = sizes8(cfg, S);
    if (rc) return rc;
    if (cache_bytes) *cache_bytes = S.cache_bytes;
    if (ws_bytes) *ws_bytes = S.ws_bytes;
    if (blocks_per_seq) *blocks_per_seq = S.blocks_per_seq;
    if (n_pages) *n_pages = S.n_pages;
    return SSSD_OK;
}

int sssd_rope_frequencies(const sssd_rope_config *c, double *turns)
{
    if (!c || !turns || c->rotary_dims < 2 || c->rotary_dims > 1024 || c->rotary_dims % 2 || !(c->base > 1.f)) return SSSD_EINVAL;
    if (c->scaling != SSSD_ROPE_PLAIN && c->scaling != SSSD_ROPE_LINEAR && c->scaling != SSSD_ROPE_BANDS) return SSSD_EINVAL;
    if (c->scaling != SSSD_ROPE_PLAIN && !(c->factor > 0.f)) return SSSD_EINVAL;
    if (c->scaling == SSSD_ROPE_BANDS && (!(c->low >= 0.f) || !(c->high > c->low) || c->original <= 0)) return SSSD_EINVAL;
    const double two_pi = 6.283185307179586476925286766559;
    for (int i = 0; i < c->rotary_dims / 2; ++i) {
        double f = std::pow((double)c->base, -2.0 * i / c->rotary_dims) / two_pi;
        if (c->scaling == SSSD_ROPE_LINEAR) f /= c->factor;
        if (c->scaling == SSSD_ROPE_BANDS) {
            double w = (c->original * f - c->low) / ((double)c->high - c->low);
            w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
            f *= w + (1.0 - w) / c->factor;
        }
        turns[i] = f;
    }
    return SSSD_OK;
}

int sssd_op_rope(const sssd_rows *x, const sssd_rows *out, int32_t B, int32_t n, int32_t heads, int32_t head_dim, const int32_t *positions,
                 const sssd_rope *rope, void *stream)
{
    if (B <= 0 || n <= 0 || heads <= 0 || heads > 65535 || head_dim <= 0 || head_dim > 8192 || !positions || !rope) return SSSD_EINVAL;
    Rows8 from, to;
    Rope8 rp;
    if (make_rows(x, B, n, heads, from) || make_rows(out, B, n, heads, to) || from.bf16 != to.bf16 || !make_rope(rope, head_dim, rp)) return SSSD_EINVAL;
    if (from.p == to.p && (from.bs != to.bs || from.rs != to.rs || from.hs != to.hs)) return SSSD_EINVAL;
    if ((int64_t)B * n > MOST_THREADS / 256) return SSSD_ECAPACITY;
    const RopeWork w = rope_work(B, n, head_dim, heads, rp.r, rp.neighbours, 256, 1);
    if ((int64_t)((w.total + w.rows - 1) / w.rows) * ((heads + w.per - 1) / w.per) > MOST_THREADS / 256) return SSSD_ECAPACITY;
    HIP_TRY(launch_rope(from, to, positions, rp, w, (hipStream_t)stream));
    return SSSD_OK;
}

// What append and read share: the sequences and rows of a call and the blocks that they touch.
static int store_args(const sssd_kv8 *kv, int32_t layer, int32_t first, int32_t B, int32_t n, const sssd_rows *k, const sssd_rows *v, const int32_t *lens,
                      const int32_t *counts, Kv8StoreArgs &a)
{
    Sizes8 S;
    int rc = check_cache(kv, layer, S);
    if (rc) return rc;
    const sssd_kv8_config &c = kv->cfg;
    if (first < 0 || B <= 0 || n <= 0) return SSSD_EINVAL;
    if ((int64_t)first + B > c.max_batch || (n > c.max_seq && !counts)) return SSSD_ECAPACITY;
    a = Kv8StoreArgs{};
    if ((rc = make_rows(k, B, n, c.n_kv_heads, a.k)) || (rc = make_rows(v, B, n, c.n_kv_heads, a.v))) return rc;
    if (a.k.bf16 != a.v.bf16) return SSSD_EINVAL;
    a.g = geom(kv, S);
    a.codes = (uint8_t *)kv->cache + (size_t)layer * S.layer_bytes;
    a.scales = (float2 *)(a.codes + S.scales_at);
    a.layer_bytes = S.layer_bytes;
    a.first = first; a.B = B; a.n = n;
    a.blocks = S.blocks_per_seq;
    if (n <= c.max_seq && (n + 2 * KV8_BLOCK - 2) / KV8_BLOCK < a.blocks) a.blocks = (n + 2 * KV8_BLOCK - 2) / KV8_BLOCK;   // the first may begin at a block's last row
    a.lens = lens; a.counts = counts; a.status = kv->status;
    if ((int64_t)B * a.blocks > MOST_THREADS / (4 * c.head_dim) / c.n_kv_heads) return SSSD_ECAPACITY;
    return SSSD_OK;
}

int sssd_kv8_append(const sssd_kv8 *kv, int32_t layer, int32_t first, int32_t B, int32_t n, const sssd_rows *k, const sssd_rows *v,
                    const int32_t *lens, const int32_t *counts, const sssd_rope *rope, const int32_t *parents, const sssd_rows *q,
                    const sssd_rows *q_out, void *stream)
{
    if (!lens) return SSSD_EINVAL;
    Kv8StoreArgs a;
    const int rc = store_args(kv, layer, first, B, n, k, v, lens, counts, a);
    if (rc) return rc;
    if ((parents && n > 32) || !q != !q_out || (q && !rope)) return SSSD_EINVAL;
    a.parents = parents;
    const sssd_kv8_config &c = kv->cfg;
    if (rope && !make_rope(rope, c.head_dim, a.rope)) return SSSD_EINVAL;
    if (q) {
        if (make_rows(q, B, n, c.n_q_heads, a.q) || make_rows(q_out, B, n, c.n_q_heads, a.q_out) || a.q.bf16 != a.q_out.bf16) return SSSD_EINVAL;
        if (a.q.p == a.q_out.p && (a.q.bs != a.q_out.bs || a.q.rs != a.q_out.rs || a.q.hs != a.q_out.hs)) return SSSD_EINVAL;
        // with the threads that store: both halves of what a launch may have
        if ((int64_t)B * n > MOST_THREADS / 2 / (2 * c.head_dim) || (int64_t)B * a.blocks > MOST_THREADS / 2 / (4 * c.head_dim) / c.n_kv_heads)
            return SSSD_ECAPACITY;
        a.work = rope_work(B, n, c.head_dim, c.n_q_heads, a.rope.r, a.rope.neighbours, 2 * c.head_dim, 4);
    }
    HIP_TRY(launch_kv8_append(a, c.format, c.head_dim, (hipStream_t)stream));
    return SSSD_OK;
}

int sssd_kv8_read(const sssd_kv8 *kv, int32_t layer, int32_t first, int32_t B, int32_t n, const int32_t *start, const int32_t *counts,
                  const sssd_rows *k, const sssd_rows *v, void *stream)
{
    Kv8StoreArgs a;
    const int rc = store_args(kv, layer, first, B, n, k, v, start, counts, a);
    if (rc) return rc;
    HIP_TRY(launch_kv8_read(a, kv->cfg.format, kv->cfg.head_dim, (hipStream_t)stream));
    return SSSD_OK;
}

int sssd_kv8_attention(const sssd_kv8 *kv, int32_t layer, int32_t B, int32_t n, const sssd_rows *q, const sssd_rows *out, const int32_t *lens,
                       const int32_t *counts, const int32_t *parents, int32_t window, int32_t sinks, void *stream)
{
    Sizes8 S;
    int rc = check_cache(kv, layer, S);
    if (rc) return rc;
    const sssd_kv8_config &c = kv->cfg;
    if (!lens || B <= 0 || n <= 0 || window < 0 || sinks < 0 || !kv->workspace || (uintptr_t)kv->workspace % ALIGN) return SSSD_EINVAL;
    if (B > c.max_batch || n > 32 || n > c.max_seq || kv->ws_bytes < S.ws_bytes) return SSSD_ECAPACITY;
    Kv8AttnArgs a{};
    if ((rc = make_rows(q, B, n, c.n_q_heads, a.q)) || (rc = make_rows(out, B, n, c.n_q_heads, a.out))) return rc;
    if (a.q.bf16 != a.out.bf16) return SSSD_EINVAL;
    a.g = geom(kv, S);
    a.codes = (const uint8_t *)kv->cache + (size_t)layer * S.layer_bytes;
    a.scales = (const float2 *)(a.codes + S.scales_at);
    a.B = B; a.n = n; a.gq = c.n_q_heads / c.n_kv_heads;
    a.lens = lens; a.counts = counts; a.parents = parents; a.status = kv->status;
    a.window = window < c.max_seq ? window : 0;   // nothing is farther back
    a.sinks = sinks < c.max_seq ? sinks : c.max_seq;
    a.hand.polls = kv->flags & SSSD_NO_WAIT ? 0 : HAND_POLLS;
    // a row of queries and a thread each in the merge, at most 32 passes of 256 threads a kv head otherwise
    if ((int64_t)B * c.n_q_heads > MOST_THREADS / (32 * 256)) return SSSD_ECAPACITY;
    HIP_TRY(launch_kv8_attention(a, c.format, c.head_dim, kv->workspace, (hipStream_t)stream));
    return SSSD_OK;
}

int sssd_kv8_commit_tree(const sssd_kv8 *kv, int32_t B, int32_t n, int32_t *lens, const int32_t *accepted_len, const int32_t *accepted_path,
                         void *stream)
{
    Sizes8 S;
    const int rc = check_cache(kv, 0, S);
    if (rc) return rc;
    const sssd_kv8_config &c = kv->cfg;
    if (!lens || !accepted_len || B <= 0 || n <= 0) return SSSD_EINVAL;
    if (B > c.max_batch || n > 32 || n > c.max_seq) return SSSD_ECAPACITY;
    if ((int64_t)B * c.n_layers > MOST_THREADS / (4 * c.head_dim) / c.n_kv_heads) return SSSD_ECAPACITY;
    Kv8StoreArgs a{};
    a.g = geom(kv, S);
    a.codes = (uint8_t *)kv->cache;
    a.scales = (float2 *)(a.codes + S.scales_at);
    a.layer_bytes = S.layer_bytes;
    a.B = B; a.n = n; a.lens = lens; a.status = kv->status;
    HIP_TRY(launch_kv8_commit(a, c.format, c.head_dim, c.n_layers, accepted_len, accepted_path, lens, (hipStream_t)stream));
    return SSSD_OK;
}

int sssd_kv8_sync(const sssd_kv8 *kv, void *stream)
{
    if (!kv || !kv->status) return SSSD_EINVAL;
    hipStream_t s = (hipStream_t)stream;
    int32_t flag = 0;
    HIP_TRY(hipMemcpyAsync(&flag, kv->status, sizeof(flag), hipMemcpyDeviceToHost, s));
    HIP_TRY(hipStreamSynchronize(s));
    if (!flag) return SSSD_OK;
    HIP_TRY(hipMemsetAsync(kv->status, 0, sizeof(flag), s));
    HIP_TRY(hipStreamSynchronize(s));
    return flag & KV8_RANGE ? SSSD_ENOSPACE : SSSD_EINVAL;
}

}  // extern "C"
