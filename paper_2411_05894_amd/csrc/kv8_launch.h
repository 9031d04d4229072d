// Launches of attention of sequences by themselves.
#ifndef SSSD_KV8_LAUNCH_H
#define SSSD_KV8_LAUNCH_H

#include "kv8_attention.h"

#include <algorithm>

namespace {

template <int HD, int FMT, int RT, int PARTS, int NW, int MODE>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void kv8_attn_kernel(Kv8Args<MODE> a)
{
    __shared__ AttnShared<HD, RT, PARTS, NW, MODE> sh;
    attend_group<HD, FMT, RT, PARTS, NW, MODE>(a, sh, blockIdx.x);
}

// The merge as a launch of its own, where a group's segments are not on one die: one wave per query row.
template <int HD, int MODE> __global__ __launch_bounds__(256) void kv8_merge_kernel(Kv8Args<MODE> a, int R)
{
    const uint32_t task = blockIdx.x * 4 + (threadIdx.x >> 6), nkv = a.g.nkv;
    if (task >= (uint32_t)a.B * nkv * R) return;
    const int r = (int)(task % (uint32_t)R), kvh = (int)(task / (uint32_t)R % nkv), b = (int)(task / ((uint32_t)R * nkv));
    int len, count;
    if (!kv8_rows(a.lens, a.counts, b, a.n, a.g.max_seq, len, count) || r >= count * a.gq) return;
    if constexpr (MODE == KV8_APART) {
        bool sane;
        if (len < group_of(a, b, threadIdx.x & 63, sane).blocks * KV8_BLOCK) return;
    }
    const Cut cut = cut_of(span_of(len, count, a.window, a.sinks).n, a.plan.share);
    if (cut.n > 1) merge_rows<HD, 1, 5, true, false>(a, b, kvh, r, 1, r + 1, cut.n, threadIdx.x & 63);
}

template <int MODE, int HD, int FMT, int PARTS> hipError_t launch_parts(const Kv8Args<MODE> &a, int rt, hipStream_t s)
{
    const dim3 grid(((uint32_t)a.B * a.g.nkv + 7) / 8 * 8 * a.plan.share * a.plan.passes);
    // Eight waves to a workgroup where a compute unit has one workgroup, of long segments and more than a wave alone on its SIMD gets done while
    // the cache streams: float32 queries, or several passes over the cache.  us, four / eight: 8B f32 B = 4, n = 9, 32768 70 / 68; 70B B = 16,
    // n = 9, 2048 bf16 27.7 / 26.3, f32 36.3 / 34.7; B = 7, n = 13, 700..1500 f32 24.1 / 21.6; not: bf16 in one pass, 8B B = 4, 32768 57.3 / 59.7,
    // many segments, f32 B = 1, 2048 11.4 / 13.0, two workgroups on a unit, B = 16, n = 32, 500 13.4 / 19.6
    const bool eight = HD == 128 && rt > 1 && a.plan.share <= 8 && (int64_t)a.B * a.g.nkv * a.plan.share * a.plan.passes <= 256 && (PARTS == 2 || a.plan.passes > 1);
#define KV8_ATTN(RT, NW) hipLaunchKernelGGL((kv8_attn_kernel<HD, FMT, RT, PARTS, NW, MODE>), grid, dim3(NW * 64), 0, s, a)
    if constexpr (HD == 128) {
        if (eight) {
            if (rt == 2) KV8_ATTN(2, 8);
            else KV8_ATTN(3, 8);
            return hipGetLastError();
        }
    }
    switch (rt) {
    case 1: KV8_ATTN(1, 4); break;
    case 2: KV8_ATTN(2, 4); break;
    default: KV8_ATTN(3, 4); break;
    }
#undef KV8_ATTN
    return hipGetLastError();
}
template <int MODE, int HD> hipError_t launch_hd(const Kv8Args<MODE> &a, int fmt, int rt, hipStream_t s)
{
    hipError_t e;
    if (fmt == SSSD_KV8_E4M3) e = a.q.bf16 ? launch_parts<MODE, HD, SSSD_KV8_E4M3, 1>(a, rt, s) : launch_parts<MODE, HD, SSSD_KV8_E4M3, 2>(a, rt, s);
    else e = a.q.bf16 ? launch_parts<MODE, HD, SSSD_KV8_INT8, 1>(a, rt, s) : launch_parts<MODE, HD, SSSD_KV8_INT8, 2>(a, rt, s);
    if (e != hipSuccess || a.plan.share == 1 || a.hand.words) return e;
    const int R = a.n * a.gq;
    hipLaunchKernelGGL((kv8_merge_kernel<HD, MODE>), dim3(((uint32_t)a.B * a.g.nkv * R + 3) / 4), dim3(256), 0, s, a, R);
    return hipGetLastError();
}

// ws: zero but for calls of this kind
template <int MODE> hipError_t launch_attention(Kv8Args<MODE> a, int fmt, int d, void *ws, hipStream_t s)
{
    const int tiles = (a.n * a.gq + 15) / 16;
    int64_t blocks = a.g.blocks_per_seq;   // that a sequence can have
    if (a.window > 0) blocks = std::min(blocks, ((int64_t)a.window + a.n + 30) / 32 + 1 + ((int64_t)a.sinks + 31) / 32);
    a.plan = kv8_plan(a.B, a.n, a.gq, a.g.nkv, (int)blocks, !a.q.bf16);
    const int rt = (tiles + a.plan.passes - 1) / a.plan.passes;
    a.rows_pad = tiles * 16;
    a.hand.words = a.plan.share > 1 && a.plan.in_die ? (uint64_t *)ws : nullptr;
    a.part_o = reinterpret_cast<float *>((char *)ws + HAND_WORDS);
    a.part_ml = reinterpret_cast<f32x4 *>(a.part_o + (size_t)KV8_GROUPS * KV8_MAX_TILES * 16 * d);
    return d == 128 ? launch_hd<MODE, 128>(a, fmt, rt, s) : launch_hd<MODE, 64>(a, fmt, rt, s);
}

}  // namespace

#endif
