// What attention over a KV cache in 8 bits is made of on the device (private): the kernel that goes over the blocks, for one batch of sequences each on its own
// and for batches that share prefixes, and the joining of partial results.
#pragma once
#include "kv8.h"

#include <type_traits>

namespace {


__device__ __forceinline__ f32x4 mfma16(const half8_t &a, const half8_t &b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

constexpr float NONE = -3.402823466e38f;   // reference of a row that has seen nothing: below every score
// Probabilities are kept below 2^15 (the largest float16 is 65504): the reference of the exponents is put 2^7 below a row's maximum and
// follows once the maximum has outgrown it by 2^15.  So they lose no bits to float16's small numbers until they are 2^-21 of the largest.
constexpr float REF_BELOW = 7.f, REF_MOST = 15.f;
// From scores of this size on they are rounded before the reference is subtracted: unrounded products of the row's largest could lie above a
// reference made of a rounded one by more than float16 holds.
constexpr float HUGE_SCORE = 0x1p20f;
// V's codes are converted in units of a scale that follows the largest, V_ABOVE octaves late.  A block is taken as it comes while its own scale is at most
// that far above the unit and V_BELOW below it, where float16 holds code * ratio exactly (it would down to 2^-15 for 8-bit floats and 2^-24 for integers), and
// at most both together above the smallest one met: what its probabilities lose (2^-32 of the row's largest) is then worth no more than 2^-20 of that one's
// values.  Other blocks are far: multiplied as they are, with probabilities relative to the block's own maximum (or REF_FAR below the row's reference, where
// that is higher), and added in 32 bits.
constexpr int V_ABOVE = 4, V_BELOW = 8;
constexpr float REF_FAR = 96.f;

// max / sum over the four lanes 16 apart that share a query row
__device__ __forceinline__ float rows_max(float x)
{
    auto h = __builtin_amdgcn_permlane32_swap(f32_bits(x), f32_bits(x), false, false);
    x = fmaxf(bits_f32(h[0]), bits_f32(h[1]));
    h = __builtin_amdgcn_permlane16_swap(f32_bits(x), f32_bits(x), false, false);
    return fmaxf(bits_f32(h[0]), bits_f32(h[1]));
}
__device__ __forceinline__ float rows_sum(float x)
{
    auto h = __builtin_amdgcn_permlane32_swap(f32_bits(x), f32_bits(x), false, false);
    x = bits_f32(h[0]) + bits_f32(h[1]);
    h = __builtin_amdgcn_permlane16_swap(f32_bits(x), f32_bits(x), false, false);
    return bits_f32(h[0]) + bits_f32(h[1]);
}

// A score's distance from the reference, the score rounded on the way as it is where it is huge.
__device__ __forceinline__ float above(float s, float sc, float m)
{
#pragma clang fp contract(off)
    return s * sc - m;
}

// max over 8 or 16 neighbouring lanes
template <int N> __device__ __forceinline__ float row_max(float x)
{
    auto other = [&](auto ctrl) { return bits_f32((uint32_t)__builtin_amdgcn_mov_dpp((int)f32_bits(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    x = fmaxf(x, other(std::integral_constant<int, 0xB1>()));          // lane ^ 1
    x = fmaxf(x, other(std::integral_constant<int, 0x4E>()));          // lane ^ 2
    x = fmaxf(x, other(std::integral_constant<int, 0x141>()));         // mirrored within eight
    if (N == 16) x = fmaxf(x, other(std::integral_constant<int, 0x140>()));   // ... within sixteen
    return x;
}

// v_maximum3_f32; fmaxf costs another instruction per score, because a product of matrices might leave a signalling NaN
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

__device__ __forceinline__ uint32_t half2_bits(half2_t x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ uint32_t pack_half2(float a, float b)   // to nearest even
{
    const f32x2_t v = {a, b};
    return half2_bits(__builtin_convertvector(v, half2_t));
}
__device__ __forceinline__ void split_half2(float a, float b, uint32_t &hi, uint32_t &lo)   // x ~= hi + lo, 22 bits
{
    hi = pack_half2(a, b);
    const half2_t h = __builtin_bit_cast(half2_t, hi);
    lo = pack_half2(a - (float)h[0], b - (float)h[1]);
}

// Eight codes as float16, times `ratio` (a power of two).
template <int FMT> __device__ __forceinline__ half8_t codes_half8(uint32_t w0, uint32_t w1, float ratio)
{
    u32x4 r;
    if (FMT == SSSD_KV8_E4M3) {
        r[0] = half2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, ratio, false));
        r[1] = half2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, ratio, true));
        r[2] = half2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, ratio, false));
        r[3] = half2_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, ratio, true));
    } else {   // 0x64xx is 1024 + xx, and xx the code + 128
        const _Float16 f = (_Float16)ratio, off = (_Float16)(-1152.f * ratio);
        const half2_t m = {f, f}, o = {off, off};
        auto two = [&](uint32_t w, uint32_t sel) {
            return half2_bits(__builtin_elementwise_fma(__builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, sel)), m, o));
        };
        r[0] = two(w0, 0x04010400u);
        r[1] = two(w0, 0x04030402u);
        r[2] = two(w1, 0x04010400u);
        r[3] = two(w1, 0x04030402u);
    }
    return __builtin_bit_cast(half8_t, r);
}

// The blocks of a sequence that some row of the call can see: `sink` at its front, then those from `from` on.
struct Span {
    int sink, from, n;
    __device__ __forceinline__ int block(int i) const { return i < sink ? i : i - sink + from; }
};
__device__ __forceinline__ Span span_of(int len, int count, int window, int sinks)
{
    const int end = (len + count + 31) >> 5;
    Span s{0, 0, end};
    if (window > 0 && len >= window) {
        s.from = (len - window + 1) >> 5;            // the root row sees farthest back
        s.sink = min((int)(((unsigned)sinks + 31u) >> 5), s.from);
        s.n = s.sink + end - s.from;
    }
    return s;
}
struct Cut {
    int each, n;   // blocks per segment (the last may have fewer), segments
};
// By the sequence's own blocks and the call's plan alone: what the others hold changes no bit.  At least four blocks a segment, one for each wave (300
// positions of 8B, float32, with eight at least 8.9 us, so 8.2; 2048 9.7 either way); up to eight are one segment, which need not be joined.  Long segments are
// whole rounds of four waves (4 x 32768 bf16 58 us, else 60; one of 32768 float32 27.5, else 28.3; but 16 sequences of 4000 with 32 rows 56.5, else 54.6).
__device__ __forceinline__ Cut cut_of(int blocks, int share)
{
    auto up = [](int x, int y) { return (int)(((unsigned)x + (unsigned)y - 1u) / (unsigned)y); };
    if (blocks <= 0) return Cut{1, 1};
    const int fair = up(blocks, share), least = blocks <= 8 ? 8 : 4;
    Cut c;
    c.each = up(blocks, up(blocks, max(fair, least)));
    if (c.each >= 16) c.each = (c.each + 3) & ~3;
    c.n = up(blocks, c.each);
    return c;
}

struct RowOut {   // where query row r of (sequence, kv head) goes
    int j, head;
    __device__ __forceinline__ RowOut(int r, int gq, int kvh) : j((int)((unsigned)r / (unsigned)gq)), head(kvh * gq + r - j * gq) {}
};
__device__ __forceinline__ void store4(const Rows8 &o, char *row, int ch, const f32x4 &y)
{
    if (!o.vec) {
#pragma unroll
        for (int i = 0; i < 4; ++i) store1(o, row, ch + i, y[i]);
    } else if (o.bf16) {
        *reinterpret_cast<uint2 *>(row + ch * 2) = uint2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
    } else {
        *reinterpret_cast<f32x4 *>(row + ch * 4) = y;
    }
}

// The segments of ROWS query rows r0, r0 + step, ... (below r_end) of a (sequence, kv head) merged by one wave, in fixed order: lanes
// 16s .. 16s+15 take segments s, s+4, ... with HD/16 channels each, U of them in one round of independent loads.  MANY: in several rounds.
// DIE: workgroups of this launch, on this die, stored them.
template <int HD, int ROWS, int U, bool MANY, bool DIE>
__device__ __forceinline__ void merge_rows(const Kv8AttnArgs &a, int b, int kvh, int r0, int step, int r_end, int n_seg, int lane)
{
    constexpr int E = HD / 16;
    const int sg = lane >> 4, cl = lane & 15;
    const size_t slot0 = ((size_t)b * a.g.nkv + kvh) * a.plan.share * a.rows_pad;
    const float *part_o = a.part_o + slot0 * HD;
    const f32x4 *part_ml = a.part_ml + slot0;
    const DieBuffer die_o(part_o, (size_t)n_seg * a.rows_pad * HD * sizeof(float)), die_ml(part_ml, (size_t)n_seg * a.rows_pad * sizeof(f32x4));
    auto row = [&](int i) { return min(r0 + i * step, r_end - 1); };
    auto stats = [&](int s, int r) { return DIE ? die_ml.load4((s * a.rows_pad + r) * 16) : part_ml[s * a.rows_pad + r]; };
    float num[ROWS][E], den[ROWS], m_all[ROWS], v_all[ROWS];   // v_all: the unit of the sums, that of the segment with the largest
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        m_all[i] = v_all[i] = NONE;
        if (MANY)
            for (int s = lane; s < n_seg; s += 64) {
                const f32x4 x = stats(s, row(i));
                m_all[i] = fmaxf(m_all[i], x[0]);
                v_all[i] = fmaxf(v_all[i], x[2]);
            }
        den[i] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) num[i][e] = 0.f;
    }
    for (int base = 0; base < (MANY ? n_seg : 1); base += 4 * U) {
        f32x4 pv[ROWS][U][E / 4];
        f32x4 ml[ROWS][U];
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
            for (int u = 0; u < U; ++u) {   // past the last segment: that one again, not added
                const int s = min(base + 4 * u + sg, n_seg - 1), at = (s * a.rows_pad + row(i)) * HD + cl * E;
                ml[i][u] = stats(s, row(i));
#pragma unroll
                for (int e = 0; e < E; e += 4) pv[i][u][e / 4] = DIE ? die_o.load4(at * 4, e * 4) : *reinterpret_cast<const f32x4 *>(part_o + at + e);
            }
        if (base == 0) {
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                if (!MANY) {
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        m_all[i] = fmaxf(m_all[i], ml[i][u][0]);
                        v_all[i] = fmaxf(v_all[i], ml[i][u][2]);
                    }
                    m_all[i] = rows_max(m_all[i]);
                    v_all[i] = rows_max(v_all[i]);
                } else {
#pragma unroll
                    for (int x = 32; x > 0; x >>= 1) {
                        m_all[i] = fmaxf(m_all[i], __shfl_xor(m_all[i], x));
                        v_all[i] = fmaxf(v_all[i], __shfl_xor(v_all[i], x));
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool on = base + 4 * u + sg < n_seg;
                const float w = on ? __builtin_amdgcn_exp2f(ml[i][u][0] - m_all[i]) : 0.f, wv = __builtin_ldexpf(w, (int)(ml[i][u][2] - v_all[i]));
                den[i] = on ? __builtin_fmaf(w, ml[i][u][1], den[i]) : den[i];
#pragma unroll
                for (int e = 0; e < E; ++e) num[i][e] = on ? __builtin_fmaf(wv, pv[i][u][e / 4][e % 4], num[i][e]) : num[i][e];
            }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        den[i] = rows_sum(den[i]);
        const float inv = den[i] != 0.f ? 1.f / den[i] : 0.f;   // a row that sees nothing: 0
        const int r = r0 + i * step;
        if (r >= r_end) continue;
        const RowOut o(r, a.gq, kvh);
        char *to = a.out.at(b, o.j, o.head);
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            f32x4 y;
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] = __builtin_ldexpf(rows_sum(num[i][e + x]) * inv, (int)v_all[i] - 127);
            if (sg == e / 4) store4(a.out, to, cl * E + e, y);
        }
    }
}

// Positions t0 .. t0+31 that a row sees, bit by bit: the old ones from `low` on (or among the first), of the new ones those of its word.
__device__ __forceinline__ uint32_t visible(int t0, int len, int low, int sinks, uint32_t word)
{
    auto below = [](int x) { return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1u; };
    const int at = t0 - len;
    const uint32_t old = below(-at) & (~below(low - t0) | below(sinks - t0));
    const uint32_t fresh = at >= 32 ? 0u : at >= 0 ? word >> at : at > -32 ? word << -at : 0u;
    return old | fresh;
}

// Batches that share prefixes.  Groups are sequences next to each other; group g's share the first shared[g] / 32 blocks.
struct Group {
    int first, n, blocks;   // sequences, and whole blocks that they share (0: nothing)
};
// One round of 64 groups, a lane each; false: the arrays make no sense, and nothing is shared in the whole call.
__device__ __forceinline__ bool group_round(const Kv8SharedArgs &a, int round, int lane, Group &g)
{
    const int i = round * 64 + lane, at = min(i, a.groups - 1);
    const int from = a.starts[at], to = a.starts[at + 1], shared = a.shared[at];
    const bool ok = from >= 0 && to >= from && to <= a.B && shared >= 0 && shared <= a.g.max_seq;
    g = Group{from, ok && i < a.groups ? to - from : 0, shared >> 5};
    if (g.n < 2 || g.blocks == 0) g = Group{from, 0, 0};   // a sequence alone shares with nobody
    return !__any(!ok);
}
// What sequence b shares.
__device__ __forceinline__ Group group_of(const Kv8SharedArgs &a, int b, int lane, bool &ok)
{
    Group mine{b, 1, 0};
    ok = true;
    for (int r = 0; r * 64 < a.groups; ++r) {
        Group g;
        ok = group_round(a, r, lane, g) && ok;
        const uint64_t has = __ballot(b >= g.first && b < g.first + g.n);
        if (has) {
            const int l = __ffsll((long long)has) - 1;
            mine = Group{__builtin_amdgcn_readlane(g.first, l), __builtin_amdgcn_readlane(g.n, l), __builtin_amdgcn_readlane(g.blocks, l)};
        }
    }
    return ok ? mine : Group{b, 1, 0};
}
// The segments of a shared prefix of some blocks: as many as cost least of the two numbers that are best with one workgroup to a compute unit and with two, a block taking PREFIX_BLOCK us
// there and half as much again here; at least four blocks each.  The kernels that make and join them have the same answer, with nothing contracted.
constexpr float PREFIX_BLOCK = 0.65f, PREFIX_BLOCK_TWO = 0.975f;
__device__ __forceinline__ Cut prefix_cut(const Kv8SharedArgs &a, int blocks)
{
#pragma clang fp contract(off)
    auto up = [](int x, int y) { return (int)(((unsigned)x + (unsigned)y - 1u) / (unsigned)y); };
    auto each_of = [&](int most, float block) {   // blocks of a segment
        const int best = (int)__builtin_ceilf(__builtin_amdgcn_sqrtf((float)blocks * (a.prefix_cost / block)));
        return max(max(up(blocks, most), best), 4);
    };
    int each = each_of(a.prefix_segments, PREFIX_BLOCK_TWO), n = up(blocks, each);
    if (a.prefix_once > 0) {
        const int one = each_of(a.prefix_once, PREFIX_BLOCK), n_one = up(blocks, one);
        if (n <= a.prefix_once || (float)one * PREFIX_BLOCK + (float)n_one * a.prefix_cost <= (float)each * PREFIX_BLOCK_TWO + (float)n * a.prefix_cost) {
            each = one;
            n = n_one;
        }
    }
    return Cut{each, n};
}

// What a workgroup on a prefix has: tile `tile` of the group's rows, `rows` to a tile, and its number `pair` among the kv heads of the first segments, the second, ...
struct PrefixTask {
    Group g;   // n = 0: nothing
    Cut cut;
    int tile, pair;
};
// The group's workgroups lie next to each other, tile by tile in whole eights, those of one pair on one die: they read the same blocks.  Workgroups that find nothing come last: in between,
// some compute units had three of those that do, and others one.  sub: segments of a workgroup
__device__ __forceinline__ PrefixTask prefix_task(const Kv8SharedArgs &a, uint32_t bid, int rows, int sub, int lane)
{
    PrefixTask mine{{0, 0, 0}, {0, 0}, 0, 0};
    const int slot = (int)(bid >> 3);
    int before = 0;
    bool ok = true;
    for (int r = 0; r * 64 < a.groups; ++r) {
        Group g;
        ok = group_round(a, r, lane, g) && ok;
        const Cut cut = prefix_cut(a, max(g.blocks, 1));
        const int tiles = (int)(((unsigned)g.n * (unsigned)(a.n * a.gq) + (unsigned)rows - 1u) / (unsigned)rows);
        const int eights = ((cut.n + sub - 1) / sub * a.g.nkv + 7) >> 3, slots = tiles * eights;
        int upto = slots;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
            const int y = __shfl_up(upto, x);
            if (lane >= x) upto += y;
        }
        const int end = before + upto;
        const uint64_t has = __ballot(slot < end && slot >= end - slots);
        if (has) {
            const int l = __ffsll((long long)has) - 1;
            const int at = slot - __builtin_amdgcn_readlane(end - slots, l), per = __builtin_amdgcn_readlane(eights, l);
            mine.g = Group{__builtin_amdgcn_readlane(g.first, l), __builtin_amdgcn_readlane(g.n, l), __builtin_amdgcn_readlane(g.blocks, l)};
            mine.cut = Cut{__builtin_amdgcn_readlane(cut.each, l), __builtin_amdgcn_readlane(cut.n, l)};
            mine.tile = at / per;
            mine.pair = (at - mine.tile * per) * 8 + (int)(bid & 7);
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    if (!ok) mine.g.n = 0;
    return mine;
}
// Where the partial result of a row of the batch lies: prefixes' segments first.
__device__ __forceinline__ size_t shared_slot(const Kv8SharedArgs &a, int segment, int kvh, int row) { return ((size_t)segment * a.g.nkv + kvh) * a.rows_all + row; }

// What a workgroup goes over: the blocks of a sequence, the same with those that its group shares read through the table of the first, a sequence's blocks behind what its group shares, or
// blocks that a group shares.
enum Kv8Mode : int { KV8_ALONE, KV8_APART, KV8_BEHIND, KV8_PREFIX };
template <int MODE> using Kv8Args = std::conditional_t<MODE == KV8_ALONE, Kv8AttnArgs, Kv8SharedArgs>;
// How a kernel hands them on: those of sequences alone as a copy, of which the compiler makes loads with fewer round trips (40 calls of all kinds 0.8 % less); of the others, a copy's pointers
// would no longer be known to be to global memory.
template <int MODE> using Kv8Pass = std::conditional_t<MODE == KV8_ALONE, const Kv8AttnArgs, const Kv8SharedArgs &>;

// PARTS: the query operand is float16 (1: bf16 queries) or float16 hi + lo (2: float32 queries), and so are the probabilities.
// grid: workgroups of one (sequence, kv head) have block indexes of one residue modulo 8: its segments, and their passes next to each other.
// KV8_PREFIX: the waves of a workgroup have the same row tiles and are on segments next to each other; a wave's partial results are its own.
template <int HD, int RT, int PARTS, int NW, int MODE> struct AttnShared {   // LDS of a workgroup
    static constexpr int KS = HD / 32, DT = HD / 16, QT = DT / NW, TR = NW == 4 ? RT : RT <= 2 ? RT : 2;
    static constexpr int QREC = RT * KS * PARTS * 64, RRED = NW * (NW - 1) * TR * QT * 64, QSETS = MODE == KV8_PREFIX ? NW : 1;
    u32x4 lds[MODE == KV8_PREFIX ? QREC * NW : QREC > RRED ? QREC : RRED];
    float row_scale_s[RT * 16 * QSETS];
    uint32_t word_s[RT * 16];
    int low_s[RT * 16], way_s;
    float2 ml_s[NW][RT * 16];
    int vref_s[NW];
};
// bid: the workgroup's number among those of this kind
template <int HD, int FMT, int RT, int PARTS, int NW, int MODE>
__device__ __forceinline__ void attend_group(Kv8Pass<MODE> a, AttnShared<HD, RT, PARTS, NW, MODE> &sh, const uint32_t bid)
{
    using Shared = AttnShared<HD, RT, PARTS, NW, MODE>;
    constexpr int KS = Shared::KS, DT = Shared::DT, QT = Shared::QT, TR = Shared::TR, QREC = Shared::QREC;
    constexpr bool PRE = MODE == KV8_PREFIX;
    u32x4 *lds = sh.lds;
    float *row_scale_s = sh.row_scale_s;
    uint32_t *word_s = sh.word_s;
    int *low_s = sh.low_s, &way_s = sh.way_s, *vref_s = sh.vref_s;
    auto &ml_s = sh.ml_s;

    const int passes = a.plan.passes, share = a.plan.share, nkv = a.g.nkv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int q = lane >> 4, c = lane & 15;
    int pass, segment, b, kvh;
    int skip = 0, n_rows = 0;   // blocks that are another workgroup's; rows of a group
    Cut prefix{1, 1};
    if constexpr (PRE) {
        const PrefixTask task = prefix_task(a, bid, RT * 16, NW, lane);
        segment = (int)((uint32_t)task.pair / (uint32_t)nkv);
        kvh = task.pair - segment * nkv;
        segment *= NW;
        if (task.g.n == 0 || segment >= task.cut.n) return;
        segment += wave;
        b = task.g.first;
        skip = task.g.blocks;
        n_rows = task.g.n * a.n * a.gq;
        pass = task.tile;
        prefix = task.cut;
    } else {
        const uint32_t slot = bid >> 3, x = slot / (uint32_t)passes, row = x / (uint32_t)share;
        pass = (int)(slot - x * passes);
        segment = (int)(x - row * share);
        const uint32_t u = row * 8 + ((bid - row) & 7);   // heads rotate over the dies
        b = (int)(u / (uint32_t)nkv);
        kvh = (int)u - b * nkv;
    }
    if (b >= a.B) return;   // groups are in whole eights
    int len = 0, count = 0;
    bool ok = true;
    if constexpr (!PRE) ok = kv8_rows(a.lens, a.counts, b, a.n, a.g.max_seq, len, count);
    const int rt0 = pass * RT;

    // A thread's share of the queries is requested ahead of everything that depends on lens: eight channels of a row at a time.
    constexpr int TPR = HD / 8, RPP = (PRE ? 64 : NW * 64) / TPR, QN = (RT * 16 + RPP - 1) / RPP;   // threads of a row, rows at a time
    const int q_part = threadIdx.x % TPR, q_row = (PRE ? lane : (int)threadIdx.x) / TPR;
    u32x4 *q_lds = lds + (PRE ? wave * QREC : 0);
    float *scale_lds = row_scale_s + (PRE ? wave * RT * 16 : 0);
    float qx[QN][8];
    u32x4 qv[QN][PARTS];
#pragma unroll
    for (int i = 0; i < QN; ++i) {
        const char *row;
        if constexpr (PRE) {
            const int r = min(rt0 * 16 + i * RPP + q_row, n_rows - 1), of = (int)((unsigned)r / (unsigned)(a.n * a.gq));
            const RowOut o(r - of * a.n * a.gq, a.gq, kvh);
            row = a.q.at(b + of, o.j, o.head);
        } else {
            const RowOut o(min(rt0 * 16 + i * RPP + q_row, a.n * a.gq - 1), a.gq, kvh);   // past the last: that one again, used by no row
            row = a.q.at(b, o.j, o.head);
        }
        if (a.q.vec) {
#pragma unroll
            for (int x = 0; x < PARTS; ++x) qv[i][x] = *reinterpret_cast<const u32x4 *>(row + q_part * 16 * PARTS + x * 16);
        } else {
#pragma unroll
            for (int x = 0; x < 8; ++x)
                qx[i][x] = PARTS == 1 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(row)[q_part * 8 + x]) : reinterpret_cast<const float *>(row)[q_part * 8 + x];
        }
    }
    int up = lane - 1;
    if (!PRE && a.parents && lane < a.n) up = a.parents[(size_t)b * a.n + lane];
    int front = b;   // the sequence whose table has the first `skip` blocks
    if constexpr (MODE == KV8_BEHIND || MODE == KV8_APART) {
        bool sane;
        const Group g = group_of(a, b, lane, sane);
        skip = g.blocks;
        front = g.first;
        if (!sane && bid == 0 && threadIdx.x == 0) atomicOr(a.status, KV8_RANGE);
        if (len < skip * KV8_BLOCK) ok = false;   // shorter than what it is said to share
    }

    if (MODE == KV8_BEHIND && !ok) {   // the merge writes zeros
        if (segment == 0 && kvh == 0 && pass == 0 && threadIdx.x == 0) atomicOr(a.status, KV8_RANGE);
        return;
    }
    if (!ok) {   // zeros
        if (segment == 0) {
            if (kvh == 0 && pass == 0 && threadIdx.x == 0) atomicOr(a.status, KV8_RANGE);
            for (int i = threadIdx.x; i < RT * 16 * (HD / 4); i += NW * 64) {
                const int r = rt0 * 16 + i / (HD / 4);
                const RowOut o(r, a.gq, kvh);
                if (o.j < a.n) store4(a.out, a.out.at(b, o.j, o.head), i % (HD / 4) * 4, f32x4{0.f, 0.f, 0.f, 0.f});
            }
        }
        return;
    }
    const int rows = PRE ? n_rows : count * a.gq;
    if (!PRE && rt0 * 16 >= rows) return;
    Span span = span_of(len, count, a.window, a.sinks);
    if constexpr (MODE == KV8_BEHIND) span = Span{0, skip, span.n - skip};
    if constexpr (PRE) span = Span{0, 0, skip};
    Cut cut = cut_of(span.n, share);
    if constexpr (PRE) cut = prefix;
    if (!PRE && segment >= cut.n) return;
    // blocks of a wave: first + off, and every STEP-th behind it
    constexpr int STEP = PRE ? 1 : NW;
    const int off = PRE ? 0 : wave;
    const int first = segment * cut.each, n_blk = PRE && (segment >= cut.n || rt0 * 16 >= rows) ? 0 : min(cut.each, span.n - first);
    const int n_it = n_blk > off ? (n_blk - off + STEP - 1) / STEP : 0;

    // Pages and scales of this wave's blocks: lane l keeps those of its block number 64 * chunk + l, one chunk ahead.
    struct Ahead {
        int record;
        float2 scale;
    };
    auto look = [&](int chunk) {
        const int i = min(first + off + STEP * (64 * chunk + lane), span.n - 1);
        Ahead x;
        const int entry = kv8_entry(a.g, MODE == KV8_APART && span.block(i) < skip ? front : b, span.block(i));
        const int page = min(max(entry, 0), a.g.n_pages - 1);
        if (entry != page && kvh == 0 && pass == 0) atomicOr(a.status, KV8_RANGE);
        x.record = page * nkv + kvh;
        x.scale = a.scales[(uint32_t)x.record];
        return x;
    };
    int chunk = 0;
    Ahead now = look(0), next = now;

    constexpr int KR = HD / 32, VR = HD / 32;   // 16-byte records of a lane
    u32x4 k[KR], v[VR];
    auto block = [&](int i) {
        const int at = i < n_it ? i : 0;
        const uint32_t record = (uint32_t)__builtin_amdgcn_readlane(at >> 6 == chunk ? now.record : next.record, at & 63);
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.codes) + (size_t)record * (64 * HD), 0, i < n_it ? 64 * HD : 0, 0x00027000);
    };
    auto load_k = [&](int i) {
        const auto p = block(i);
#pragma unroll
        for (int x = 0; x < KR; ++x) k[x] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(p, lane * 16, x * 1024, 0));
    };
    auto load_v = [&](int i) {
        const auto p = block(i);
#pragma unroll
        for (int x = 0; x < VR; ++x) v[x] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(p, lane * 16, 32 * HD + x * 1024, 0));
    };
    load_k(0);
    load_v(0);
    if (n_it > 64) next = look(1);

    // Query operands: a row's channels times a power of two that brings its largest below 2^15, as float16.
#pragma unroll
    for (int i = 0; i < QN; ++i) {
        const int r = i * RPP + q_row;
        if (a.q.vec) {
            if (PARTS == 1) {
                unpack_bf16x8(qv[i][0], qx[i]);
            } else {
#pragma unroll
                for (int x = 0; x < 8; ++x) qx[i][x] = bits_f32(qv[i][PARTS == 2 ? x >> 2 : 0][x & 3]);
            }
        }
        float most = 0.f;
#pragma unroll
        for (int x = 0; x < 8; ++x) most = fmaxf(most, fabsf(qx[i][x]));
        most = row_max<TPR>(most);
        const int e = (int)(f32_bits(most) >> 23);   // 2^(e-127) <= most < 2^(e-126)
        const int to = e == 0 || e == 255 ? 127 : min(268 - e, 253);   // biased exponent of the factor, 2^(141-e)
        const float f = bits_f32((uint32_t)to << 23);
        u32x4 hi, lo;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            uint32_t h, l = 0;
            if (PARTS == 2) split_half2(qx[i][2 * x] * f, qx[i][2 * x + 1] * f, h, l);
            else h = pack_half2(qx[i][2 * x] * f, qx[i][2 * x + 1] * f);
            hi[x] = h;
            lo[x] = l;
        }
        if (QN * RPP > RT * 16 && r >= RT * 16) continue;   // an odd tile of 64 channels
        const int rec = (((r >> 4) * KS + (q_part >> 2)) * PARTS) * 64 + (q_part & 3) * 16 + (r & 15);
        q_lds[rec] = hi;
        if (PARTS == 2) q_lds[rec + 64] = lo;
        if (q_part == 0) scale_lds[r] = bits_f32((uint32_t)(254 - to) << 23);
    }
    // What the rows see of the new ones, and where their windows begin.
    if (!PRE && wave == 0) {
        uint32_t word = kv8_chain_word(lane & 31);
        if (a.parents) {
            bool bad;
            word = kv8_tree_word(up, count, lane, bad);
            if (segment == 0 && kvh == 0 && pass == 0 && __any(bad) && lane == 0) atomicOr(a.status, KV8_RANGE);
        }
        const int depth = __popc(word) - 1;
        if (a.window > 0 && a.window < count) {   // ancestors farther than the window go, but for those among the first positions
            uint32_t near = 0;
            for (int i = 0; i < count; ++i) {
                const int d = __builtin_amdgcn_readlane(depth, i);
                if (depth - d < a.window || len + d < a.sinks) near |= 1u << i;
            }
            word &= near;
        }
        const int r = lane, j = min(RowOut(rt0 * 16 + r, a.gq, kvh).j, 31);
        const uint32_t w = (uint32_t)__shfl((int)word, j);
        const int d = __shfl(depth, j);
        if (r < RT * 16) {
            word_s[r] = w;
            low_s[r] = a.window > 0 ? len + d - a.window + 1 : 0;
        }
    }
    __syncthreads();
    float row_scale[RT];
    const float soft = 1.4426950408889634f * rsqrtf((float)HD);   // log2(e) / sqrt(d)
#pragma unroll
    for (int t = 0; t < RT; ++t) row_scale[t] = scale_lds[t * 16 + c] * soft;

    f32x4 o[RT][DT], l_run[RT];   // l_run: sums of probabilities, by a product with ones: the same in every register of a lane's column
    float m_run[RT];
    // Biased exponents of V's scales: the sums' and the smallest of all, beyond all of them while there is none, and those of blocks that are taken as they come,
    // v_from .. v_from + v_span.
    int v_ref = -256, v_low = 256, v_from = 512;
    uint32_t v_span = V_ABOVE + V_BELOW;
    const int v_first = __builtin_amdgcn_readlane((int)f32_bits(now.scale.y), 0) >> 23 & 255;
    if (n_it > 0 && v_first != 127) {   // no block of zeros
        v_ref = v_first;
        v_from = v_ref - V_BELOW;
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[t][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        l_run[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run[t] = NONE;
    }
    const half8_t ones = __builtin_bit_cast(half8_t, u32x4{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u});
    bool huge = false;   // some row's reference has been HUGE_SCORE
    const int all_from = a.window > 0 ? len + count - a.window : 0;   // every row sees the old positions from here on

    // Chunks are a loop of their own: where the loop over blocks changes them, pages and scales move between registers on the way round, and every block begins with a wait for all
    // that is under way, its own V among it (8B, 4 sequences of 32768 bf16 captured 63 us instead of 55).
    for (int i0 = 0; i0 < n_it; i0 += 64) {
        if (i0 > 0) {
            chunk = i0 >> 6;
            now = next;
            next = look(chunk + 1);
        }
        for (int i = i0, end = min(i0 + 64, n_it); i < end; ++i) {
            const int t0 = span.block(first + off + STEP * i) * 32;
            const float k_scale = bits_f32((uint32_t)__builtin_amdgcn_readlane((int)f32_bits(now.scale.x), i & 63));
            int v_e = __builtin_amdgcn_readlane((int)f32_bits(now.scale.y), i & 63) >> 23 & 255;
            int ql = lane;
            if (RT * PARTS > 2) asm volatile("" : "+v"(ql));   // the query operands are read again for every block: hoisted, they would not fit the registers
            f32x4 s[RT][2];   // s[t][u][r]: position t0 + 16u + 4q + r for query row c of tile t
#pragma unroll
            for (int t = 0; t < RT; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
            // The operands of a step (32 channels, hi or lo) are read a step ahead: LDS answers after some hundred cycles, and one wave alone has
            // nothing else to do meanwhile.
            u32x4 qq[2][RT];
            auto fetch = [&](int x) {
#pragma unroll
                for (int t = 0; t < RT; ++t) qq[x & 1][t] = q_lds[(t * KS * PARTS + x) * 64 + ql];
            };
            half8_t kk[2];
            fetch(0);
#pragma unroll
            for (int x = 0; x < KS * PARTS; ++x) {
                if (x + 1 < KS * PARTS) fetch(x + 1);
                if (x % PARTS == 0) {
                    const int ks = x / PARTS;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const u32x4 &w = k[u * (KS / 2) + ks % (KS / 2)];
                        kk[u] = ks < KS / 2 ? codes_half8<FMT>(w[0], w[1], 1.f) : codes_half8<FMT>(w[2], w[3], 1.f);
                    }
                }
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int u = 0; u < 2; ++u) s[t][u] = mfma16(kk[u], __builtin_bit_cast(half8_t, qq[x & 1][t]), s[t][u]);
                if (RT * PARTS > 2) __builtin_amdgcn_sched_barrier(0);
            }
            load_k(i + 1);
            const bool whole = PRE || (t0 + 32 <= len && (t0 >= all_from || t0 + 32 <= a.sinks));   // all rows see all of the block
            float sc[RT], mx[RT];   // mx: of the lane's own eight positions
            bool grow = huge;
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                sc[t] = __builtin_amdgcn_fmed3f(row_scale[t] * k_scale, 0x1p-126f, 0x1p127f);   // neither 0 nor infinite: times -INFINITY or 0
                if (!whole) {
                    const uint32_t mine = visible(t0, len, low_s[t * 16 + c], a.sinks, word_s[t * 16 + c]) >> (4 * q);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[t][u][r] = mine & (1u << (16 * u + r)) ? s[t][u][r] : -INFINITY;
                }
                mx[t] = max3(max3(s[t][0][0], s[t][0][1], s[t][0][2]), max3(s[t][0][3], s[t][1][0], s[t][1][1]), max3(s[t][1][2], s[t][1][3], s[t][1][3]));
                grow = grow || above(mx[t], sc[t], m_run[t]) > REF_MOST;
            }
            if (__any(grow)) {
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const float m = rows_max(mx[t]);
                    const float m_new = above(m, sc[t], m_run[t]) > REF_MOST ? above(m, sc[t], REF_BELOW) : m_run[t], alpha = __builtin_amdgcn_exp2f(m_run[t] - m_new);
                    m_run[t] = m_new;
                    huge = huge || __any(fabsf(m_new) >= HUGE_SCORE && m_new != NONE);
                    l_run[t] *= alpha;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) o[t][dt] *= alpha;
                }
                if (huge)
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        const bool mine = fabsf(m_run[t]) >= HUGE_SCORE;   // by the row alone: the others change none of its bits
#pragma unroll
                        for (int u = 0; u < 2; ++u) s[t][u] = mine ? s[t][u] * sc[t] : s[t][u];
                        sc[t] = mine ? 1.f : sc[t];
                    }
            }
            u32x4 pk[RT][PARTS];
            auto weigh = [&](int t, float ref) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e >> 1][2 * (e & 1)], sc[t], -ref));
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e >> 1][2 * (e & 1) + 1], sc[t], -ref));
                    uint32_t hi, lo;
                    if (PARTS == 2) {
                        split_half2(p0, p1, hi, lo);
                        pk[t][PARTS - 1][e] = lo;
                    } else {
                        hi = pack_half2(p0, p1);
                    }
                    pk[t][0][e] = hi;
                }
            };
            auto codes = [&](int dt, float ratio) {
                const u32x4 &w = v[dt >> 1];
                return dt & 1 ? codes_half8<FMT>(w[2], w[3], ratio) : codes_half8<FMT>(w[0], w[1], ratio);
            };
            auto times = [&](const half8_t &x, int t, f32x4 sum) {
#pragma unroll
                for (int part = 0; part < PARTS; ++part) sum = mfma16(x, __builtin_bit_cast(half8_t, pk[t][part]), sum);
                return sum;
            };
            // The sums are in units of 2^(v_ref - 127), a V scale: they move to a larger one only when a block's outgrows it, and not for a block of zeros, whose
            // scale says nothing.
            const int low_was = v_low;
            v_low = min(v_low, v_e);
            if (__builtin_expect((uint32_t)(v_e - v_from) > v_span, false)) {
                uint32_t any = 0;
#pragma unroll
                for (int x = 0; x < VR; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) any |= FMT == SSSD_KV8_E4M3 ? v[x][e] & 0x7F7F7F7Fu : v[x][e] ^ 0x80808080u;
                const bool some = __any(any != 0), far = some && v_ref >= 0;
                if (some) {
                    const float down = bits_f32((uint32_t)max(v_ref - v_e + 127, 0) << 23);
                    if (v_e > v_ref) {
#pragma unroll
                        for (int t = 0; t < RT; ++t)
#pragma unroll
                            for (int dt = 0; dt < DT; ++dt) o[t][dt] *= down;
                    }
                    v_ref = max(v_ref, v_e);
                    const int top = min(v_ref + V_ABOVE, v_low + V_ABOVE + V_BELOW);
                    v_from = top < v_ref - V_BELOW ? 512 : v_ref - V_BELOW;   // 512: beyond all
                    v_span = (uint32_t)(top - v_from) & 31u;
                }
                if (far) {
                    const f32x4 none = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY}, zero = f32x4{0.f, 0.f, 0.f, 0.f};
                    const float down = bits_f32((uint32_t)max(v_e - v_ref + 127, 0) << 23);
                    float back[RT];   // from the block's reference and scale to the row's reference and the unit
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        const float m = rows_max(max3(max3(s[t][0][0], s[t][0][1], s[t][0][2]), max3(s[t][0][3], s[t][1][0], s[t][1][1]), max3(s[t][1][2], s[t][1][3], s[t][1][3])));
                        const float ref = fmaxf(above(m, sc[t], REF_BELOW), m_run[t] - REF_FAR);
                        weigh(t, ref);
                        s[t][0] = s[t][1] = none;   // then there is nothing left of the block
                        back[t] = __builtin_amdgcn_exp2f(ref - m_run[t]);
                        l_run[t] += times(ones, t, zero) * back[t];
                        back[t] *= down;
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        const half8_t vv = codes(dt, 1.f);
#pragma unroll
                        for (int t = 0; t < RT; ++t) o[t][dt] += times(vv, t, zero) * back[t];
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                if (!some) v_low = low_was;
                v_e = v_ref;
#pragma unroll
                for (int x = 0; x < VR; ++x) asm volatile("" : "+v"(v[x]));   // its codes as halves are not kept for what follows: 32 registers
            }
            const float ratio = bits_f32((uint32_t)(v_e - v_ref + 127) << 23);   // 2^-V_BELOW .. 2^V_ABOVE
#pragma unroll
            for (int t = 0; t < RT; ++t) weigh(t, m_run[t]);
#pragma unroll
            for (int t = 0; t < RT; ++t) l_run[t] = times(ones, t, l_run[t]);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const half8_t vv = codes(dt, ratio);
#pragma unroll
                for (int t = 0; t < RT; ++t) o[t][dt] = times(vv, t, o[t][dt]);
            }
            load_v(i + 1);
        }
    }

    if constexpr (PRE) {
        if (n_it > 0)
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const int row = (rt0 + t) * 16 + c;
                if (row >= rows) continue;
                const size_t at = shared_slot(a, segment, kvh, b * a.n * a.gq + row);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4 *>(a.part_o + at * HD + dt * 16 + 4 * q) = o[t][dt];
                if (q == 0) a.part_ml[at] = f32x4{m_run[t], l_run[t][0], (float)v_ref, 0.f};
            }
        return;
    }

    // The waves' sums on one reference per row, each wave ending with a quarter of the channels.
    f32x4 *red = reinterpret_cast<f32x4 *>(lds);
    const int dt0 = wave * QT;
    f32x4 own[RT][QT];
    __syncthreads();   // the query operands have been read
#pragma unroll
    for (int t = 0; t < RT; ++t)
        if (q == 0) ml_s[wave][t * 16 + c] = float2{m_run[t], l_run[t][0]};
    if (lane == 0) vref_s[wave] = v_ref;
#pragma unroll
    for (int w = 0; w < NW; ++w)
        if (w == wave)
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int x = 0; x < QT; ++x) own[t][x] = o[t][w * QT + x];
    auto part = [&](int quarter, int from, int t, int x) -> f32x4 & {
        return red[(((quarter * (NW - 1) + from - (from > quarter ? 1 : 0)) * TR + t % TR) * QT + x) * 64 + lane];
    };
#pragma unroll
    for (int tt = 0; tt < RT; tt += TR) {
        if (tt > 0) __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w)
            if (w != wave)
#pragma unroll
                for (int t = tt; t < tt + TR && t < RT; ++t)
#pragma unroll
                    for (int x = 0; x < QT; ++x) part(w, wave, t, x) = o[t][w * QT + x];
        __syncthreads();
        int v_all = vref_s[0];
#pragma unroll
        for (int w = 1; w < NW; ++w) v_all = max(v_all, vref_s[w]);
#pragma unroll
        for (int t = tt; t < tt + TR && t < RT; ++t) {
            const int row = (rt0 + t) * 16 + c;
            float2 s4[NW];
            float m_all = NONE;
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                s4[i] = ml_s[(wave + i) & (NW - 1)][t * 16 + c];
                m_all = fmaxf(m_all, s4[i].x);
            }
            float l_all = 0.f;
            f32x4 y[QT];   // in units of the waves' largest
#pragma unroll
            for (int x = 0; x < QT; ++x) y[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const int w = (wave + i) & (NW - 1);
                const float f = __builtin_amdgcn_exp2f(s4[i].x - m_all), fv = __builtin_ldexpf(f, vref_s[w] - v_all);
                l_all += s4[i].y * f;
#pragma unroll
                for (int x = 0; x < QT; ++x) y[x] += (i ? part(wave, w, t, x) : own[t][x]) * fv;
            }
            if (row >= rows) continue;
            if ((MODE == KV8_ALONE || MODE == KV8_APART) && cut.n == 1) {
                const RowOut ro(row, a.gq, kvh);
                const float inv = l_all != 0.f ? 1.f / l_all : 0.f;   // a row that sees nothing: 0
                char *to = a.out.at(b, ro.j, ro.head);
#pragma unroll
                for (int x = 0; x < QT; ++x) {
                    f32x4 z;
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[e] = __builtin_ldexpf(y[x][e] * inv, v_all - 127);
                    store4(a.out, to, (dt0 + x) * 16 + 4 * q, z);
                }
            } else {
                size_t at = (((size_t)b * nkv + kvh) * share + segment) * a.rows_pad + row;
                if constexpr (MODE == KV8_BEHIND) at = shared_slot(a, a.prefix_segments + segment, kvh, b * a.n * a.gq + row);
#pragma unroll
                for (int x = 0; x < QT; ++x) *reinterpret_cast<f32x4 *>(a.part_o + at * HD + (dt0 + x) * 16 + 4 * q) = y[x];
                if (wave == 0 && q == 0) a.part_ml[at] = f32x4{m_all, l_all, (float)v_all, 0.f};
            }
        }
    }
    if (MODE == KV8_BEHIND || cut.n == 1 || !a.hand.words) return;
    const int group = (b * nkv + kvh) * passes + pass;
    HandWay way = hand_wait(a.hand, group, cut.n, hand_arrive(a.hand, group), &way_s);
    if (way == HAND_TURN_IN) way = hand_turn_in(a.hand, group, cut.n, &way_s);
    uint64_t left = way == HAND_SHARE ? hand_leave(a.hand, group) : 0;   // under way while the shares are done
    if (way != HAND_NOTHING) {   // the rows of this pass shared out over the waves of all segments
        const int r_end = min(rows, (rt0 + RT) * 16), step = (way == HAND_ALL ? 1 : cut.n) * NW;
        int r = rt0 * 16 + (way == HAND_ALL ? wave : wave * cut.n + segment);
        // as many rows at once as the wave has, up to four, when they have few segments
#define KV8_MERGE(ROWS, U, MANY) for (; r < r_end; r += ROWS * step) merge_rows<HD, ROWS, U, MANY, true>(a, b, kvh, r, step, r_end, cut.n, lane)
        if (cut.n > 16) KV8_MERGE(1, 8, false);   // 32 at most: eight heads share 256 workgroups
        else if (cut.n > 8) KV8_MERGE(1, 4, false);
        else if (cut.n > 4) {
            if (r + step < r_end) KV8_MERGE(2, 2, false);
            else KV8_MERGE(1, 2, false);
        } else {
            if (r + 2 * step < r_end) KV8_MERGE(4, 1, false);
            else if (r + step < r_end) KV8_MERGE(2, 1, false);
            else KV8_MERGE(1, 1, false);
        }
#undef KV8_MERGE
    }
    if (way != HAND_SHARE) left = hand_leave(a.hand, group);
    hand_clear(a.hand, group, cut.n, left);
}

}  // namespace
