// Attention of a step's new rows over an 8-bit KV cache whose sequences share prefixes in groups: the prefix is read once for all rows of a group.
//
// Mathematics.  softmax over prefix and own rows is joined from partial results (m, l, o) as in kv8_attention.h: a prefix has one per row and segment, the rows
// behind it (the sequence's own ones and the new ones) one per segment of theirs; with M the largest m, l = sum 2^(m - M) l, o likewise, out = o / l.
//
// Split.  The rows of all sequences of a group, side by side, are the queries of its prefix, and all see all of it: no masks.  A wave takes up to three tiles of
// 16 of them over its segment's blocks; four waves of a workgroup have different rows and read the same blocks, from the first one's cache lines, or, where a group has few
// rows, different segments.  What lies behind the prefix goes as sequences do alone, and a last launch joins both.
#include "kv8_attention.h"
#include "kv8_host.h"

namespace {

// A wave per row of the batch.
template <int HD> __global__ __launch_bounds__(256) void kv8_shared_merge_kernel(Kv8SharedArgs a)
{
    constexpr int E = HD / 16, U = 4;
    const int R = a.n * a.gq, nkv = a.g.nkv, lane = threadIdx.x & 63;
    const uint32_t task = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const uint32_t head_of = task / (uint32_t)R;
    const int r = (int)(task - head_of * R), b = (int)(head_of / (uint32_t)nkv), kvh = (int)(head_of - (uint32_t)b * nkv);
    if (b >= a.B) return;
    int len, count;
    bool ok = kv8_rows(a.lens, a.counts, b, a.n, a.g.max_seq, len, count), sane;
    const Group g = group_of(a, b, lane, sane);
    ok = ok && len >= g.blocks * KV8_BLOCK;
    const int sg = lane >> 4, cl = lane & 15;
    const RowOut o(r, a.gq, kvh);
    char *to = a.out.at(b, o.j, o.head);
    if (!ok) {
#pragma unroll
        for (int e = 0; e < E; e += 4)
            if (sg == e / 4) store4(a.out, to, cl * E + e, f32x4{0.f, 0.f, 0.f, 0.f});
        return;
    }
    if (r >= count * a.gq) return;
    const int n_pre = g.blocks ? prefix_cut(g.blocks, a.prefix_segments).n : 0;
    const int n_seg = n_pre + cut_of(((len + count + 31) >> 5) - g.blocks, a.plan.share).n;
    const int row = b * R + r;
    auto slot = [&](int s) { return shared_slot(a, s < n_pre ? s : a.prefix_segments + s - n_pre, kvh, row); };
    float m_all = NONE, v_all = NONE, den = 0.f, num[E];
#pragma unroll
    for (int e = 0; e < E; ++e) num[e] = 0.f;
    const bool many = n_seg > 4 * U;
    if (many)
        for (int s = lane; s < n_seg; s += 64) {
            const f32x4 x = a.part_ml[slot(s)];
            m_all = fmaxf(m_all, x[0]);
            v_all = fmaxf(v_all, x[2]);
        }
    for (int base = 0; base < n_seg; base += 4 * U) {
        f32x4 ml[U], pv[U][E / 4];
#pragma unroll
        for (int u = 0; u < U; ++u) {   // past the last segment: that one again, not added
            const size_t at = slot(min(base + 4 * u + sg, n_seg - 1));
            ml[u] = a.part_ml[at];
#pragma unroll
            for (int e = 0; e < E; e += 4) pv[u][e / 4] = *reinterpret_cast<const f32x4 *>(a.part_o + at * HD + cl * E + e);
        }
        if (base == 0) {
            if (!many)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    m_all = fmaxf(m_all, ml[u][0]);
                    v_all = fmaxf(v_all, ml[u][2]);
                }
#pragma unroll
            for (int x = 32; x > 0; x >>= 1) {
                m_all = fmaxf(m_all, __shfl_xor(m_all, x));
                v_all = fmaxf(v_all, __shfl_xor(v_all, x));
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool on = base + 4 * u + sg < n_seg;
            const float w = on ? __builtin_amdgcn_exp2f(ml[u][0] - m_all) : 0.f, wv = __builtin_ldexpf(w, (int)(ml[u][2] - v_all));
            den = on ? __builtin_fmaf(w, ml[u][1], den) : den;
#pragma unroll
            for (int e = 0; e < E; ++e) num[e] = on ? __builtin_fmaf(wv, pv[u][e / 4][e % 4], num[e]) : num[e];
        }
    }
    den = rows_sum(den);
    const float inv = den != 0.f ? 1.f / den : 0.f;
#pragma unroll
    for (int e = 0; e < E; e += 4) {
        f32x4 y;
#pragma unroll
        for (int x = 0; x < 4; ++x) y[x] = __builtin_ldexpf(rows_sum(num[e + x]) * inv, (int)v_all - 127);
        if (sg == e / 4) store4(a.out, to, cl * E + e, y);
    }
}

template <int HD, int FMT, int PARTS> hipError_t launch_shared(const Kv8SharedArgs &a, int rt_prefix, int rt, hipStream_t s)
{
    if (a.groups > 0) {
        const uint32_t pairs = (uint32_t)a.g.nkv * a.prefix_share;
        const dim3 grid((pairs + 7) / 8 * 8 * a.tiles);
#define KV8_PRE(RT) hipLaunchKernelGGL((kv8_attn_kernel<HD, FMT, RT, PARTS, 4, KV8_PREFIX>), grid, dim3(256), 0, s, a)
        switch (rt_prefix) {
        case 1: KV8_PRE(1); break;
        case 2: KV8_PRE(2); break;
        default: KV8_PRE(3); break;
        }
#undef KV8_PRE
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 grid(((uint32_t)a.B * a.g.nkv + 7) / 8 * 8 * a.plan.share * a.plan.passes);
#define KV8_REST(RT) hipLaunchKernelGGL((kv8_attn_kernel<HD, FMT, RT, PARTS, 4, KV8_BEHIND>), grid, dim3(256), 0, s, a)
    switch (rt) {
    case 1: KV8_REST(1); break;
    case 2: KV8_REST(2); break;
    default: KV8_REST(3); break;
    }
#undef KV8_REST
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kv8_shared_merge_kernel<HD>, dim3(((uint32_t)a.rows_all * a.g.nkv + 3) / 4), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <int HD> hipError_t launch_format(const Kv8SharedArgs &a, int fmt, int rt_prefix, int rt, hipStream_t s)
{
    if (fmt == SSSD_KV8_E4M3) return a.q.bf16 ? launch_shared<HD, SSSD_KV8_E4M3, 1>(a, rt_prefix, rt, s) : launch_shared<HD, SSSD_KV8_E4M3, 2>(a, rt_prefix, rt, s);
    return a.q.bf16 ? launch_shared<HD, SSSD_KV8_INT8, 1>(a, rt_prefix, rt, s) : launch_shared<HD, SSSD_KV8_INT8, 2>(a, rt_prefix, rt, s);
}

}  // namespace

Kv8SharedPlan kv8_shared_plan(int B, int n, int gq, int nkv, int groups)
{
    Kv8SharedPlan p{};
    const int64_t rows = (int64_t)B * n * gq, each = groups > 0 ? (rows + groups - 1) / groups : rows;   // rows of a group, if they are all alike
    const int tiles = (int)((each + 15) / 16);
    p.rt = tiles < KV8_MAX_TILES ? tiles : KV8_MAX_TILES;
    p.wave_rows = tiles <= p.rt ? 1 : tiles <= 2 * p.rt ? 2 : 4;
    const int64_t per = p.wave_rows * p.rt * 16;
    p.tiles = (int)(rows / per + groups);
    const int64_t units = (each + per - 1) / per * (groups > 0 ? groups : 1) * nkv;
    const int64_t share = KV8_GROUPS / units;
    p.share = share < 1 ? 1 : share > 64 ? 64 : (int)share;
    p.segments = p.share * 4 / p.wave_rows;
    return p;
}

// For every number of groups: a prefix's results are at most those of KV8_GROUPS workgroups of 4 * KV8_MAX_TILES row tiles or, where there are more workgroups than that, four a
// row; the rest's at most those of KV8_GROUPS workgroups of KV8_MAX_TILES tiles, or one a row.
size_t kv8_shared_ws(int B, int n, int gq, int nkv, int d)
{
    const size_t slots = (size_t)KV8_GROUPS * KV8_MAX_TILES * 16 * 5 + 5 * (size_t)B * n * gq * nkv;
    return slots * (d * sizeof(float) + sizeof(f32x4));
}

extern "C" {

int sssd_kv8_shared_sizes(const sssd_kv8_config *cfg, int32_t B, int32_t n, size_t *ws_bytes)
{
    Sizes8 S;
    const int rc = sizes8(cfg, S);
    if (rc) return rc;
    if (B <= 0 || n <= 0 || !ws_bytes) return SSSD_EINVAL;
    if (B > cfg->max_batch || n > 32 || n > cfg->max_seq || (int64_t)B * n * cfg->n_q_heads > MOST_THREADS / 64) return SSSD_ECAPACITY;
    *ws_bytes = kv8_shared_ws(B, n, cfg->n_q_heads / cfg->n_kv_heads, cfg->n_kv_heads, cfg->head_dim);
    return SSSD_OK;
}

int sssd_kv8_attention_shared(const sssd_kv8 *kv, int32_t layer, int32_t B, int32_t n, const sssd_rows *q, const sssd_rows *out, const int32_t *lens,
                              const int32_t *counts, const int32_t *parents, int32_t groups, const int32_t *starts, const int32_t *shared,
                              void *workspace, size_t ws_bytes, void *stream)
{
    Sizes8 S;
    int rc = check_cache(kv, layer, S);
    if (rc) return rc;
    const sssd_kv8_config &c = kv->cfg;
    if (!lens || B <= 0 || n <= 0 || groups < 0 || (groups > 0 && (!starts || !shared)) || !workspace || (uintptr_t)workspace % ALIGN) return SSSD_EINVAL;
    size_t need = 0;
    if ((rc = sssd_kv8_shared_sizes(&c, B, n, &need))) return rc;
    if (groups > B || ws_bytes < need) return SSSD_ECAPACITY;
    Kv8SharedArgs a{};
    if ((rc = make_rows(q, B, n, c.n_q_heads, a.q)) || (rc = make_rows(out, B, n, c.n_q_heads, a.out))) return rc;
    if (a.q.bf16 != a.out.bf16) return SSSD_EINVAL;
    a.g = geom(kv, S);
    a.codes = (const uint8_t *)kv->cache + (size_t)layer * S.layer_bytes;
    a.scales = (const float2 *)(a.codes + S.scales_at);
    a.B = B; a.n = n; a.gq = c.n_q_heads / c.n_kv_heads;
    a.lens = lens; a.counts = counts; a.parents = parents; a.status = kv->status;
    a.plan = kv8_plan(B, n, a.gq, c.n_kv_heads, S.blocks_per_seq, !a.q.bf16);
    const int tiles = (n * a.gq + 15) / 16;
    a.rows_pad = tiles * 16;
    const Kv8SharedPlan p = kv8_shared_plan(B, n, a.gq, c.n_kv_heads, groups);
    a.groups = groups; a.starts = starts; a.shared = shared;
    a.tiles = p.tiles; a.wave_rows = p.wave_rows; a.prefix_share = p.share; a.prefix_segments = p.segments;
    a.rows_all = B * n * a.gq;
    a.part_o = (float *)workspace;
    a.part_ml = reinterpret_cast<f32x4 *>(a.part_o + (size_t)(p.segments + a.plan.share) * c.n_kv_heads * a.rows_all * c.head_dim);
    // workgroups of 256 threads
    if (((int64_t)c.n_kv_heads * p.share + 7) / 8 * 8 * p.tiles > MOST_THREADS / 256 || ((int64_t)B * c.n_kv_heads + 7) / 8 * 8 * a.plan.share * a.plan.passes > MOST_THREADS / 256)
        return SSSD_ECAPACITY;
    const int rt = (tiles + a.plan.passes - 1) / a.plan.passes;
    hipStream_t s = (hipStream_t)stream;
    HIP_TRY(c.head_dim == 128 ? launch_format<128>(a, c.format, p.rt, rt, s) : launch_format<64>(a, c.format, p.rt, rt, s));
    return SSSD_OK;
}

}  // extern "C"
