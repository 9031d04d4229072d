// Attention of a step's new rows over a KV cache in 8 bits: softmax(q . k / sqrt(d)) over what a row sees, times v.
//
// Mathematics.  One pass over the cache with, per row, a reference m of the exponents, l = sum of p and o = sum of p v for p = 2^(score * log2(e) - m);
// when m moves, l and o are multiplied by 2^(old - new).  m is not the running maximum but follows it lazily (REF_BELOW, REF_MOST), so that hardly any block
// pays for it.  Sums over waves and segments are brought to one m at the end.
//
// Products are float16 matrix instructions (16 x 16 x 32) with 32-bit sums: an 8-bit code is a float16 exactly, in either format, at one conversion per two
// codes.  The other operand is rounded to 11 bits or, for float32 queries, split into hi + lo with 22: queries after their row's largest has been
// brought below 2^15 by a power of two, probabilities as they are.  K's scales join the factor of the exponent; V's go into the conversion of its codes, relative
// to the largest one so far, where float16 holds that (V_ABOVE, V_BELOW).
//
// Layout and split.  A score product gives a lane four positions of one query row, twice a block: just what the second product takes from it as an operand (V is
// stored for that), so probabilities stay in registers.  Queries lie in LDS as operands.  A workgroup is four or eight waves on the
// blocks of one (sequence, kv head) in turn; a wave requests a block's K and V as soon as it has used those before.  Sequences are cut into segments by the
// plan (kv8_plan, cut_of), joined inside the launch where one die can hold them.
//
// What bounds it: from some thousands of positions a chip's worth of workgroups on the stream of the cache.  us, captured (and called one behind the other, where
// launches overlap): 8B, B = 4, n = 9, 32768 bf16 269 MB in 58 (55), 4.6 TB/s, of which some 45 stream at 6 TB/s, as fast as the blocks are read in the same
// order by a kernel that does nothing else (46 us), around them 5 until K is there and the queries are operands and 3 for the sums of waves and segments;
// float32 queries 68 (twice the products).  B = 32, n = 5, 1024..4096 173 MB in 47 (42): one workgroup per head and sequence, so the longest decides; all
// of 2500 35.8.  Short ones on the chain of round trips: arguments, lens, page, block, sums of waves, partial results, their arrival: B = 1, n = 9, 2048
// float32 9.7 (8.9), of which K is requested after 2.2 and the rows are joined in the last 2.
#include "kv8.h"

#include <algorithm>
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

// PARTS: the query operand is float16 (1: bf16 queries) or float16 hi + lo (2: float32 queries), and so are the probabilities.
// grid: workgroups of one (sequence, kv head) have block indexes of one residue modulo 8: its segments, and their passes next to each other.
template <int HD, int FMT, int RT, int PARTS, int NW>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void kv8_attn_kernel(Kv8AttnArgs a)
{
    constexpr int KS = HD / 32, DT = HD / 16, QT = DT / NW, TR = NW == 4 ? RT : RT <= 2 ? RT : 2;
    constexpr int QREC = RT * KS * PARTS * 64, RRED = NW * (NW - 1) * TR * QT * 64;
    __shared__ u32x4 lds[QREC > RRED ? QREC : RRED];
    __shared__ float row_scale_s[RT * 16];
    __shared__ uint32_t word_s[RT * 16];
    __shared__ int low_s[RT * 16], way_s;
    __shared__ float2 ml_s[NW][RT * 16];
    __shared__ int vref_s[NW];

    const int passes = a.plan.passes, share = a.plan.share, nkv = a.g.nkv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int q = lane >> 4, c = lane & 15;
    int pass, segment, b, kvh;
    {
        const uint32_t slot = blockIdx.x >> 3, x = slot / (uint32_t)passes, row = x / (uint32_t)share;
        pass = (int)(slot - x * passes);
        segment = (int)(x - row * share);
        const uint32_t u = row * 8 + ((blockIdx.x - row) & 7);   // heads rotate over the dies
        b = (int)(u / (uint32_t)nkv);
        kvh = (int)u - b * nkv;
    }
    if (b >= a.B) return;   // groups are in whole eights
    int len, count;
    const bool ok = kv8_rows(a.lens, a.counts, b, a.n, a.g.max_seq, len, count);
    const int rt0 = pass * RT;

    // A thread's share of the queries is requested ahead of everything that depends on lens: eight channels of a row at a time.
    constexpr int TPR = HD / 8, RPP = NW * 64 / TPR, QN = (RT * 16 + RPP - 1) / RPP;   // threads of a row, rows at a time
    const int q_part = threadIdx.x % TPR, q_row = threadIdx.x / TPR;
    float qx[QN][8];
    u32x4 qv[QN][PARTS];
#pragma unroll
    for (int i = 0; i < QN; ++i) {
        const RowOut o(min(rt0 * 16 + i * RPP + q_row, a.n * a.gq - 1), a.gq, kvh);   // past the last: that one again, used by no row
        const char *row = a.q.at(b, o.j, o.head);
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
    if (a.parents && lane < a.n) up = a.parents[(size_t)b * a.n + lane];

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
    const int rows = count * a.gq;
    if (rt0 * 16 >= rows) return;
    const Span span = span_of(len, count, a.window, a.sinks);
    const Cut cut = cut_of(span.n, share);
    if (segment >= cut.n) return;
    const int first = segment * cut.each, n_blk = min(cut.each, span.n - first);
    const int n_it = n_blk > wave ? (n_blk - wave + NW - 1) / NW : 0;

    // Pages and scales of this wave's blocks: lane l keeps those of its block number 64 * chunk + l, one chunk ahead.
    struct Ahead {
        int record;
        float2 scale;
    };
    auto look = [&](int chunk) {
        const int i = min(first + wave + NW * (64 * chunk + lane), span.n - 1);
        Ahead x;
        const int entry = kv8_entry(a.g, b, span.block(i));
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
        lds[rec] = hi;
        if (PARTS == 2) lds[rec + 64] = lo;
        if (q_part == 0) row_scale_s[r] = bits_f32((uint32_t)(254 - to) << 23);
    }
    // What the rows see of the new ones, and where their windows begin.
    if (wave == 0) {
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
    for (int t = 0; t < RT; ++t) row_scale[t] = row_scale_s[t * 16 + c] * soft;

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

    for (int i = 0; i < n_it; ++i) {
        if (i >> 6 != chunk) {
            chunk = i >> 6;
            now = next;
            next = look(chunk + 1);
        }
        const int t0 = span.block(first + wave + NW * i) * 32;
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
            for (int t = 0; t < RT; ++t) qq[x & 1][t] = lds[(t * KS * PARTS + x) * 64 + ql];
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
        const bool whole = t0 + 32 <= len && (t0 >= all_from || t0 + 32 <= a.sinks);   // all rows see all of the block
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
            if (cut.n == 1) {
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
                const size_t at = (((size_t)b * nkv + kvh) * share + segment) * a.rows_pad + row;
#pragma unroll
                for (int x = 0; x < QT; ++x) *reinterpret_cast<f32x4 *>(a.part_o + at * HD + (dt0 + x) * 16 + 4 * q) = y[x];
                if (wave == 0 && q == 0) a.part_ml[at] = f32x4{m_all, l_all, (float)v_all, 0.f};
            }
        }
    }
    if (cut.n == 1 || !a.hand.words) return;
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

// The merge as a launch of its own, where a group's segments are not on one die: one wave per query row.
template <int HD> __global__ __launch_bounds__(256) void kv8_merge_kernel(Kv8AttnArgs a, int R)
{
    const uint32_t task = blockIdx.x * 4 + (threadIdx.x >> 6), nkv = a.g.nkv;
    if (task >= (uint32_t)a.B * nkv * R) return;
    const int r = (int)(task % (uint32_t)R), kvh = (int)(task / (uint32_t)R % nkv), b = (int)(task / ((uint32_t)R * nkv));
    int len, count;
    if (!kv8_rows(a.lens, a.counts, b, a.n, a.g.max_seq, len, count) || r >= count * a.gq) return;
    const Cut cut = cut_of(span_of(len, count, a.window, a.sinks).n, a.plan.share);
    if (cut.n > 1) merge_rows<HD, 1, 5, true, false>(a, b, kvh, r, 1, r + 1, cut.n, threadIdx.x & 63);
}

template <int HD, int FMT, int PARTS> hipError_t launch_parts(const Kv8AttnArgs &a, int rt, hipStream_t s)
{
    const dim3 grid(((uint32_t)a.B * a.g.nkv + 7) / 8 * 8 * a.plan.share * a.plan.passes);
    // Eight waves to a workgroup where a compute unit has one workgroup, of long segments and more than a wave alone on its SIMD gets done while
    // the cache streams: float32 queries, or several passes over the cache.  us, four / eight: 8B f32 B = 4, n = 9, 32768 70 / 68; 70B B = 16,
    // n = 9, 2048 bf16 27.7 / 26.3, f32 36.3 / 34.7; B = 7, n = 13, 700..1500 f32 24.1 / 21.6; not: bf16 in one pass, 8B B = 4, 32768 57.3 / 59.7,
    // many segments, f32 B = 1, 2048 11.4 / 13.0, two workgroups on a unit, B = 16, n = 32, 500 13.4 / 19.6
    const bool eight = HD == 128 && rt > 1 && a.plan.share <= 8 && (int64_t)a.B * a.g.nkv * a.plan.share * a.plan.passes <= 256 && (PARTS == 2 || a.plan.passes > 1);
#define KV8_ATTN(RT, NW) hipLaunchKernelGGL((kv8_attn_kernel<HD, FMT, RT, PARTS, NW>), grid, dim3(NW * 64), 0, s, a)
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
template <int HD> hipError_t launch_hd(const Kv8AttnArgs &a, int fmt, int rt, hipStream_t s)
{
    hipError_t e;
    if (fmt == SSSD_KV8_E4M3) e = a.q.bf16 ? launch_parts<HD, SSSD_KV8_E4M3, 1>(a, rt, s) : launch_parts<HD, SSSD_KV8_E4M3, 2>(a, rt, s);
    else e = a.q.bf16 ? launch_parts<HD, SSSD_KV8_INT8, 1>(a, rt, s) : launch_parts<HD, SSSD_KV8_INT8, 2>(a, rt, s);
    if (e != hipSuccess || a.plan.share == 1 || a.hand.words) return e;
    const int R = a.n * a.gq;
    hipLaunchKernelGGL(kv8_merge_kernel<HD>, dim3(((uint32_t)a.B * a.g.nkv * R + 3) / 4), dim3(256), 0, s, a, R);
    return hipGetLastError();
}

}  // namespace

// How a call is cut, by what the host knows of it.  A pass over the cache takes one to three row tiles of queries; more tiles read the cache less often, but
// their workgroups have more to set up, to add over their waves and to join.
//  - Short sequences (as long as they can be: `blocks`): a tile a pass, while its workgroups fit on the chip together.  us, one tile / as few passes as
//    can be, of 9 rows of 8B: float32 B = 1, 300 8.2 / 11.4, 2048 9.2 / 11.5, 8192 13.9 / 16.2, 16384 18.8 / 19.3, 32768 29.0 / 26.6; B = 8, 2048
//    19.5 / 20.0, 4096 30.6 / 26.9; bf16 B = 1, 8192 13.5 / 14.8, 16384 18.2 / 17.2; two
//    tiles, n = 5, bf16 B = 5, 1000 10.1 / 10.4, 2048 13.3 / 12.1; 70B float32 B = 5, 300 7.4 / 13.5; B = 6, 1500 15.5 / 22.3; sixteen tiles, n = 32,
//    B = 3, 1000 16.6 / 21.6, B = 1, 4000 21.0 / 17.6, bf16 B = 2, 4000 25.9 / 20.9; more workgroups than fit, 8B B = 16, n = 32, 500 18.5 / 13.8.
//  - Else by rounds of 256 workgroups and what a block costs a pass of one, two and three tiles.  us, by that / fewest passes / one tile: 70B float32
//    B = 7, n = 13, 700..1500 21.4 / 26.8 / 21.0; B = 2, n = 32, 4000 bf16 20.9 / 24.9 / 25.8; 8B B = 16, n = 32, 500 13.8 / 16.9 / 18.5;
//    B = 4, n = 9, 32768 57.4 / 57.7 / 76.8.
//  - Segments of a sequence so that 256 workgroups have work; twice that where 256 in whole segments leave a quarter of the chip idle (8B B = 12, 3000
//    24.6, without 27.8; for all calls: B = 32, 2500 41, now 36).
// The limits were found with 8 kv heads of 128 channels; others go by the same ones, unmeasured.
Kv8Plan kv8_plan(int B, int n, int gq, int nkv, int blocks, bool f32)
{
    const int tiles = (n * gq + 15) / 16;
    const int64_t heads = (int64_t)B * nkv;
    Kv8Plan p;
    const bool brief = heads * blocks <= (f32 ? 3500 : tiles > 2 ? 2750 : 2000) && heads * blocks * tiles <= 15000 && heads * tiles <= 512;
    if (brief) p.passes = tiles;
    double best = 0;
    for (int rt = KV8_MAX_TILES; rt >= 1 && !brief; --rt) {
        const int passes = (tiles + rt - 1) / rt;
        const int64_t units = heads * passes;
        static const double block[4] = {0, 0.75, 1.0, 1.4};
        const double cost = units <= 256 ? block[rt] / (256 / units) : block[rt] * ((units + 255) / 256);
        if (rt == KV8_MAX_TILES || cost < best) {
            best = cost;
            p.passes = passes;
        }
    }
    const int64_t units = heads * p.passes;
    int64_t share = 256 / units;
    if (share * units <= 192) share = 512 / units;
    p.share = share < 1 ? 1 : share > 64 ? 64 : (int)share;
    p.in_die = heads % 8 == 0 && units <= HAND_GROUPS;
    return p;
}

size_t kv8_attention_ws(int d) { return HAND_WORDS + (size_t)KV8_GROUPS * KV8_MAX_TILES * 16 * (d * sizeof(float) + sizeof(f32x4)); }

hipError_t launch_kv8_attention(Kv8AttnArgs a, int fmt, int d, void *ws, hipStream_t s)
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
    return d == 128 ? launch_hd<128>(a, fmt, rt, s) : launch_hd<64>(a, fmt, rt, s);
}
