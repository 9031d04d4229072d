// Attention of a step's new rows over an 8-bit KV cache whose sequences share prefixes in groups: the prefix is read once for all rows of a group.
//
// Mathematics.  softmax over prefix and own rows is joined from partial results (m, l, o) as in kv8_attention.h: a prefix has one per row and segment, the rows
// behind it (the sequence's own ones and the new ones) one per segment of theirs; with M the largest m, l = sum 2^(m - M) l, o likewise, out = o / l.
//
// Split.  The rows of all sequences of a group, side by side, are the queries of its prefix, and all see all of it: no masks.  A wave takes one or two tiles of
// 16 of them over its segment's blocks; four waves of a workgroup have different rows and share the blocks' operands in LDS or, where a group has few rows, are on different segments,
// as a sequence's alone.  What lies behind the prefix goes as sequences do alone, in the same launch, and a last one joins both.  Where that would take longer than every sequence by itself
// (apart_us), they go by themselves, the shared blocks read through the first one's table (kv8_apart.hip).
//
// What bounds it.  us, kernels of this / of the call for sequences alone: 64 sequences of one row on 32768 positions (8B, bf16) 61 + 10 / 232, 35 GFLOP, for which a
// large product takes 26; 20 sequences of one row of 8B on 4096 16.3 + 5.0 / 20.3; 4 on 2048 9.9 + 4.7 / 9.0; eight of 9 rows, float32, on 2048 20.8 + 5.3 / 20.6; 32 of one on 512 13.4 + 4.1 / 8.4; eight of one
// on 32768 21 + 9.3 / 84.  With many rows, matrix instructions are under way for 55 % of the loop's time (30 % of the
// kernel's), exponentials, conversions and what is read of LDS for the rest; around it 5 to 6 us until the first operands are there, and the partial results, 35 MB out and in for the 64 sequences.  Few rows and short
// prefixes: that start and the second launch, 4 us at least, and partial results of every wave.
#include "kv8_attention.h"
#include "kv8_host.h"

#include <algorithm>
#include <cmath>

namespace {

// Many rows: four waves of a workgroup with one or two row tiles each on the same blocks.  Codes are requested two pairs of blocks ahead, a quarter by each wave,
// turned into float16 operands once for all four and handed round in LDS (two pairs of room, one barrier a pair); queries stay in registers.  Three tiles do not fit the registers
// of two waves on a SIMD (92 us instead of 62 for the 64 sequences), nor do two of float32 queries, which are twice the operands.
//
// V's scales: the unit of the sums is the largest of the segment, known before the first block.  Where all of them lie within V_SPAN octaves, codes are converted in that unit, which
// float16 holds exactly (down to 2^-21 for 8-bit floats, 2^-12 for integers); else blocks are multiplied as they are, with probabilities relative to the
// block's own maximum (or REF_FAR below the row's reference, where that is higher), and added in 32 bits.
constexpr int V_SPAN = V_ABOVE + V_BELOW;

template <int HD> struct PrefixShared {   // LDS of a workgroup: operands of two pairs of blocks
    u32x4 ring[2][2 * (HD / 8) * 64];
};
template <int HD, int FMT, int RT, int PARTS> __device__ __forceinline__ void prefix_group(const Kv8SharedArgs &a, PrefixShared<HD> &sh, const uint32_t bid)
{
    constexpr int KS = HD / 32, DT = HD / 16, REC = HD / 16, MINE = REC / 4;   // 16-byte records of a lane: of a block (K's, V's), of a wave
    constexpr int BLOCK_OPS = 2 * REC * 64;   // operands of a block
    auto &ring = sh.ring;
    const int nkv = a.g.nkv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, q = lane >> 4, c = lane & 15;
    const PrefixTask task = prefix_task(a, bid, 4 * RT * 16, 1, lane);
    const Group g = task.g;
    const Cut cut = task.cut;
    const int tile = task.tile, segment = (int)((uint32_t)task.pair / (uint32_t)nkv), kvh = task.pair - segment * nkv;
    if (g.n == 0 || segment >= cut.n) return;
    const int each = a.n * a.gq, rows = g.n * each, row0 = (tile * 4 + wave) * RT * 16;
    const int first = segment * cut.each, n_it = min(cut.each, g.blocks - first);
    const bool mine = row0 < rows;

    struct Ahead {
        int record;
        float2 scale;
    };
    auto look = [&](int chunk) {   // lane l: block 64 * chunk + l of the segment
        const int i = first + min(64 * chunk + lane, n_it - 1);
        Ahead x;
        const int entry = kv8_entry(a.g, g.first, i);
        const int page = min(max(entry, 0), a.g.n_pages - 1);
        if (entry != page && kvh == 0 && tile == 0) atomicOr(a.status, KV8_RANGE);
        x.record = page * nkv + kvh;
        x.scale = a.scales[(uint32_t)x.record];
        return x;
    };
    int chunk = 0;
    Ahead now = look(0), next = now;

    // Query operands: row c of tile t, channels 32 ks + 8 q .. + 7, times a power of two that brings the row's largest below 2^15.
    u32x4 qq[RT][KS][PARTS];
    float row_scale[RT];
    const float soft = 1.4426950408889634f * rsqrtf((float)HD);   // log2(e) / sqrt(d)
    {
        u32x4 lo[RT][KS], hi[RT][KS];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int r = min(row0 + t * 16 + c, rows - 1), of = (int)((unsigned)r / (unsigned)each);   // past the last: that one again, used by no row
            const RowOut o(r - of * each, a.gq, kvh);
            const char *row = a.q.at(g.first + of, o.j, o.head);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) fetch8(a.q, row, 32 * ks + 8 * q, lo[t][ks], hi[t][ks]);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            float most = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                float v[8];
                decode8(a.q, lo[t][ks], hi[t][ks], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[i]));
            }
            most = rows_max(most);
            const int e = (int)(f32_bits(most) >> 23);   // 2^(e-127) <= most < 2^(e-126)
            const int to = e == 0 || e == 255 ? 127 : min(268 - e, 253);   // biased exponent of the factor, 2^(141-e)
            const float f = bits_f32((uint32_t)to << 23);
            row_scale[t] = bits_f32((uint32_t)(254 - to) << 23) * soft;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                float v[8];
                decode8(a.q, lo[t][ks], hi[t][ks], v);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t h, l = 0;
                    if (PARTS == 2) split_half2(v[2 * i] * f, v[2 * i + 1] * f, h, l);
                    else h = pack_half2(v[2 * i] * f, v[2 * i + 1] * f);
                    qq[t][ks][0][i] = h;
                    if (PARTS == 2) qq[t][ks][PARTS - 1][i] = l;
                }
            }
        }
    }

    // A wave's records of a block: K's are those below REC / 2, then V's.  Blocks go in pairs; where block i is multiplied, scores are made of block i + 1 already, so K's
    // pairs are one block ahead of V's.
    u32x4 raw[2][MINE];
    auto is_v = [&](int x) { return wave + 4 * x >= REC / 2; };
    auto request = [&](int i) {   // V's records of blocks i and i + 1, K's of i + 1 and i + 2 (behind the last: that one again)
#pragma unroll
        for (int two = 0; two < 2; ++two)
#pragma unroll
            for (int x = 0; x < MINE; ++x) {
                const int at = min(i + two + (is_v(x) ? 0 : 1), n_it - 1);
                const uint32_t record = (uint32_t)__builtin_amdgcn_readlane(at >> 6 == chunk ? now.record : next.record, at & 63);
                const auto p = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.codes) + (size_t)record * (64 * HD), 0, 64 * HD, 0x00027000);
                raw[two][x] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(p, lane * 16, (wave + 4 * x) * 1024, 0));
            }
    };
    request(-1);   // K of block 0 (and what is not used)

    // The segment's largest and smallest scale of V (biased exponents).
    int v_ref = (int)(f32_bits(now.scale.y) >> 23 & 255), v_low = v_ref;
    for (int i = 1; i * 64 < n_it; ++i) {
        const int e = (int)(f32_bits(look(i).scale.y) >> 23 & 255);
        v_ref = max(v_ref, e);
        v_low = min(v_low, e);
    }
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) {
        v_ref = max(v_ref, __shfl_xor(v_ref, i));
        v_low = min(v_low, __shfl_xor(v_low, i));
    }
    v_ref = __builtin_amdgcn_readfirstlane(v_ref);
    const bool wide = __builtin_amdgcn_readfirstlane(v_ref - v_low) > V_SPAN;
    if (n_it > 64) next = look(1);

    // Operand tiles in LDS: of a pair, K's [u][ks] and then V's [dt].
    auto hand = [&](int i, u32x4 *to) {
#pragma unroll
        for (int two = 0; two < 2; ++two) {
            const int at = min(i + two, n_it - 1);
            const int e = __builtin_amdgcn_readlane((int)f32_bits(at >> 6 == chunk ? now.scale.y : next.scale.y), at & 63) >> 23 & 255;
            const float v_ratio = wide ? 1.f : bits_f32((uint32_t)(e - v_ref + 127) << 23);
#pragma unroll
            for (int x = 0; x < MINE; ++x) {
                const int rec = wave + 4 * x, p = is_v(x) ? rec - REC / 2 : rec % (KS / 2);
                const float ratio = is_v(x) ? v_ratio : 1.f;
                const u32x4 &w = raw[two][x];
                u32x4 *tile_at = to + two * BLOCK_OPS + (is_v(x) ? REC + 2 * p : rec / (KS / 2) * KS + p) * 64 + lane;
                tile_at[0] = __builtin_bit_cast(u32x4, codes_half8<FMT>(w[0], w[1], ratio));
                tile_at[(is_v(x) ? 1 : KS / 2) * 64] = __builtin_bit_cast(u32x4, codes_half8<FMT>(w[2], w[3], ratio));
            }
        }
    };

    f32x4 o[RT][DT], l_run[RT];   // l_run: sums of probabilities, by a product with ones: the same in every register of a lane's column
    float m_run[RT], sc[RT];
    f32x4 s[RT][2];   // s[t][u][r]: position 16u + 4q + r of the block for query row c of tile t
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[t][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        l_run[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run[t] = NONE;
    }
    const half8_t ones = __builtin_bit_cast(half8_t, u32x4{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u});
    bool huge = false;   // some row's reference has been HUGE_SCORE

    auto scores = [&](const u32x4 *at, f32x4 (&to)[RT][2]) {
#pragma unroll
        for (int t = 0; t < RT; ++t) to[t][0] = to[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const half8_t kk = __builtin_bit_cast(half8_t, at[(u * KS + ks) * 64 + lane]);
#pragma unroll
                for (int part = 0; part < PARTS; ++part)
#pragma unroll
                    for (int t = 0; t < RT; ++t) to[t][u] = mfma16(kk, __builtin_bit_cast(half8_t, qq[t][ks][part]), to[t][u]);
            }
    };
    auto lane_most = [&](int t) { return max3(max3(s[t][0][0], s[t][0][1], s[t][0][2]), max3(s[t][0][3], s[t][1][0], s[t][1][1]), max3(s[t][1][2], s[t][1][3], s[t][1][3])); };
    // The references of the rows, for the block whose scores are in s.
    auto refer = [&](int i) {
        const float k_scale = bits_f32((uint32_t)__builtin_amdgcn_readlane((int)f32_bits(i >> 6 == chunk ? now.scale.x : next.scale.x), i & 63));
        float mx[RT];   // of the lane's own eight positions
        bool grow = huge;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            sc[t] = __builtin_amdgcn_fmed3f(row_scale[t] * k_scale, 0x1p-126f, 0x1p127f);   // neither 0 nor infinite: times -INFINITY or 0
            mx[t] = lane_most(t);
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
                    const bool own = fabsf(m_run[t]) >= HUGE_SCORE;   // by the row alone: the others change none of its bits
#pragma unroll
                    for (int u = 0; u < 2; ++u) s[t][u] = own ? s[t][u] * sc[t] : s[t][u];
                    sc[t] = own ? 1.f : sc[t];
                }
        }
    };
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
    auto times = [&](const half8_t &x, int t, f32x4 sum) {
#pragma unroll
        for (int part = 0; part < PARTS; ++part) sum = mfma16(x, __builtin_bit_cast(half8_t, pk[t][part]), sum);
        return sum;
    };
    auto value = [&](const u32x4 *at, int dt) { return __builtin_bit_cast(half8_t, at[(REC + dt) * 64 + lane]); };
    // Block i, whose scores are in s, times its values; the scores of block i + 1 instead.  at: the operands.  One tile's probabilities are made while
    // another's are multiplied.
    auto attend = [&](int i, const u32x4 *at) {
        f32x4 ahead[RT][2];
        half8_t vv[DT];
        weigh(0, m_run[0]);
        scores(at, ahead);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) vv[dt] = value(at, dt);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (t + 1 < RT) weigh(t + 1, m_run[t + 1]);
            l_run[t] = times(ones, t, l_run[t]);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[t][dt] = times(vv[dt], t, o[t][dt]);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) s[t][0] = ahead[t][0], s[t][1] = ahead[t][1];
        if (i + 1 < n_it) refer(i + 1);
    };
    auto attend_wide = [&](int i, const u32x4 *at) {
        const f32x4 zero = f32x4{0.f, 0.f, 0.f, 0.f};
        const int e = __builtin_amdgcn_readlane((int)f32_bits(now.scale.y), i & 63) >> 23 & 255;
        const float down = bits_f32((uint32_t)max(e - v_ref + 127, 0) << 23);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const float ref = fmaxf(above(rows_max(lane_most(t)), sc[t], REF_BELOW), m_run[t] - REF_FAR);
            weigh(t, ref);
            float back = __builtin_amdgcn_exp2f(ref - m_run[t]);   // from the block's reference and scale to the row's reference and the unit
            l_run[t] += times(ones, t, zero) * back;
            back *= down;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                o[t][dt] += times(value(at, dt), t, zero) * back;
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        scores(at, s);
        if (i + 1 < n_it) refer(i + 1);
    };

    hand(-1, ring[1]);
    request(0);
    __syncthreads();
    if (mine) {
        scores(ring[1], s);
        refer(0);
    }
    hand(0, ring[0]);
    request(2);
    auto all = [&](auto step) {
        for (int i = 0; i < n_it; i += 2) {
            if (i >> 6 != chunk) {
                chunk = i >> 6;
                now = next;
                next = look(chunk + 1);
            }
            const int half = i >> 1 & 1;
            __syncthreads();   // the operands of this turn are there, those of the one before have been read
            __builtin_amdgcn_sched_barrier(0);
            hand(i + 2, ring[half ^ 1]);
            request(i + 4);
            if (!mine) continue;
            step(i, ring[half]);
            if (i + 1 < n_it) step(i + 1, ring[half] + BLOCK_OPS);
        }
    };
    if (__builtin_expect(wide, false)) all(attend_wide);
    else all(attend);

#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int row = row0 + t * 16 + c;
        if (row >= rows) continue;
        const size_t at = shared_slot(a, segment, kvh, g.first * each + row);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4 *>(a.part_o + at * HD + dt * 16 + 4 * q) = o[t][dt];
        if (q == 0) a.part_ml[at] = f32x4{m_run[t], l_run[t][0], (float)v_ref, 0.f};
    }
}

// The partial results of ROWS rows r0 .. (below r_end) of a (sequence, kv head), by one wave: lanes 16s .. 16s+15 take segments s, s+4, ... with HD/16 channels each, U of them in one
// round of independent loads.  MANY: in several rounds.
template <int HD, int ROWS, int U, bool MANY> __device__ __forceinline__ void join_rows(const Kv8SharedArgs &a, int b, int kvh, int r0, int r_end, int n_pre, int n_seg, int lane)
{
    constexpr int E = HD / 16;
    const int sg = lane >> 4, cl = lane & 15, each = a.n * a.gq;
    auto slot = [&](int s, int i) { return shared_slot(a, s < n_pre ? s : a.prefix_segments + s - n_pre, kvh, b * each + min(r0 + i, r_end - 1)); };
    float m_all[ROWS], v_all[ROWS], den[ROWS], num[ROWS][E];   // v_all: the unit of the sums, that of the segment with the largest
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        m_all[i] = v_all[i] = NONE;
        den[i] = 0.f;
        if (MANY)
            for (int s = lane; s < n_seg; s += 64) {
                const f32x4 x = a.part_ml[slot(s, i)];
                m_all[i] = fmaxf(m_all[i], x[0]);
                v_all[i] = fmaxf(v_all[i], x[2]);
            }
#pragma unroll
        for (int e = 0; e < E; ++e) num[i][e] = 0.f;
    }
    for (int base = 0; base < (MANY ? n_seg : 1); base += 4 * U) {
        f32x4 ml[ROWS][U], pv[ROWS][U][E / 4];
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
            for (int u = 0; u < U; ++u) {   // past the last segment: that one again, not added
                const size_t at = slot(min(base + 4 * u + sg, n_seg - 1), i);
                ml[i][u] = a.part_ml[at];
#pragma unroll
                for (int e = 0; e < E; e += 4) pv[i][u][e / 4] = *reinterpret_cast<const f32x4 *>(a.part_o + at * HD + cl * E + e);
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
        const float inv = den[i] != 0.f ? 1.f / den[i] : 0.f;
        if (r0 + i >= r_end) continue;
        const RowOut o(r0 + i, a.gq, kvh);
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

// ROWS rows of a (sequence, kv head) to a wave: four where there are rows enough to fill the chip all the same.  us, four / one: 32 sequences of
// 4 rows of 70B, five segments, 8.9 / 10.3.
template <int HD, int ROWS> __global__ __launch_bounds__(256) void kv8_shared_merge_kernel(Kv8SharedArgs a)
{
    const int each = a.n * a.gq, chunks = (each + ROWS - 1) / ROWS, nkv = a.g.nkv, lane = threadIdx.x & 63;
    const uint32_t task = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const uint32_t head_of = task / (uint32_t)chunks;
    const int r0 = (int)(task - head_of * chunks) * ROWS, b = (int)(head_of / (uint32_t)nkv), kvh = (int)(head_of - (uint32_t)b * nkv);
    if (b >= a.B) return;
    int len, count;
    bool ok = kv8_rows(a.lens, a.counts, b, a.n, a.g.max_seq, len, count), sane;
    const Group g = group_of(a, b, lane, sane);
    ok = ok && len >= g.blocks * KV8_BLOCK;
    if (!ok) {
        for (int i = lane; i < ROWS * (HD / 4); i += 64) {
            const int r = r0 + i / (HD / 4);
            const RowOut o(r, a.gq, kvh);
            if (r < each) store4(a.out, a.out.at(b, o.j, o.head), i % (HD / 4) * 4, f32x4{0.f, 0.f, 0.f, 0.f});
        }
        return;
    }
    const int r_end = count * a.gq;
    if (r0 >= r_end) return;
    const int n_pre = g.blocks ? prefix_cut(a, g.blocks).n : 0;
    const int n_seg = n_pre + cut_of(((len + count + 31) >> 5) - g.blocks, a.plan.share).n;
    if (n_seg <= 4) join_rows<HD, ROWS, 1, false>(a, b, kvh, r0, r_end, n_pre, n_seg, lane);
    else if (n_seg <= 8) join_rows<HD, ROWS, 2, false>(a, b, kvh, r0, r_end, n_pre, n_seg, lane);
    else
        for (int r = r0; r < min(r0 + ROWS, r_end); ++r) {
            if (n_seg <= 16) join_rows<HD, 1, 4, false>(a, b, kvh, r, r + 1, n_pre, n_seg, lane);
            else if (n_seg <= 32) join_rows<HD, 1, 8, false>(a, b, kvh, r, r + 1, n_pre, n_seg, lane);
            else join_rows<HD, 1, 8, true>(a, b, kvh, r, r + 1, n_pre, n_seg, lane);
        }
}

// Both kinds of workgroups in one launch, those of prefixes first: they take longest, and the others fill in behind them.  RTP: row tiles of a wave of a prefix; FEW: its waves
// are on different segments.
template <int HD, int FMT, int PARTS, int RTP, bool FEW, int RT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void kv8_shared_kernel(Kv8SharedArgs a)
{
    union Shared {
        PrefixShared<HD> many;
        AttnShared<HD, RTP, PARTS, 4, KV8_PREFIX> few;
        AttnShared<HD, RT, PARTS, 4, KV8_BEHIND> rest;
    };
    constexpr size_t BYTES = std::max(FEW ? sizeof(Shared::few) : sizeof(Shared::many), sizeof(Shared::rest));
    __shared__ __align__(16) char lds[BYTES];
    if (blockIdx.x >= (uint32_t)a.prefix_groups) attend_group<HD, FMT, RT, PARTS, 4, KV8_BEHIND>(a, *reinterpret_cast<AttnShared<HD, RT, PARTS, 4, KV8_BEHIND> *>(lds), blockIdx.x - a.prefix_groups);
    else if constexpr (FEW) attend_group<HD, FMT, RTP, PARTS, 4, KV8_PREFIX>(a, *reinterpret_cast<AttnShared<HD, RTP, PARTS, 4, KV8_PREFIX> *>(lds), blockIdx.x);
    else prefix_group<HD, FMT, RTP, PARTS>(a, *reinterpret_cast<PrefixShared<HD> *>(lds), blockIdx.x);
}

template <int HD, int FMT, int PARTS> hipError_t launch_shared(Kv8SharedArgs a, int rt_prefix, int rt, hipStream_t s)
{
    a.prefix_groups = a.groups > 0 ? ((uint32_t)a.g.nkv * a.prefix_share + 7) / 8 * 8 * a.tiles : 0;
    const dim3 grid(a.prefix_groups + ((uint32_t)a.B * a.g.nkv + 7) / 8 * 8 * a.plan.share * a.plan.passes);
#define KV8_SHARED(RTP, FEW, RT) hipLaunchKernelGGL((kv8_shared_kernel<HD, FMT, PARTS, RTP, FEW, RT>), grid, dim3(256), 0, s, a)
#define KV8_REST(RTP, FEW)                        \
    do {                                          \
        if (rt == 1) KV8_SHARED(RTP, FEW, 1);     \
        else if (rt == 2) KV8_SHARED(RTP, FEW, 2); \
        else KV8_SHARED(RTP, FEW, 3);             \
    } while (0)
    if (a.wave_rows == 1) {
        if (rt_prefix == 1) KV8_REST(1, true);
        else KV8_REST(2, true);
    } else if (PARTS == 2 || rt_prefix == 1) {
        KV8_REST(1, false);
    } else {
        KV8_REST(3 - PARTS, false);
    }
#undef KV8_REST
#undef KV8_SHARED
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const uint32_t each = a.n * a.gq, heads = (uint32_t)a.B * a.g.nkv;
    if ((uint64_t)heads * each >= 8192) hipLaunchKernelGGL((kv8_shared_merge_kernel<HD, 4>), dim3((heads * ((each + 3) / 4) + 3) / 4), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((kv8_shared_merge_kernel<HD, 1>), dim3((heads * each + 3) / 4), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <int HD> hipError_t launch_format(const Kv8SharedArgs &a, int fmt, int rt_prefix, int rt, hipStream_t s)
{
    if (fmt == SSSD_KV8_E4M3) return a.q.bf16 ? launch_shared<HD, SSSD_KV8_E4M3, 1>(a, rt_prefix, rt, s) : launch_shared<HD, SSSD_KV8_E4M3, 2>(a, rt_prefix, rt, s);
    return a.q.bf16 ? launch_shared<HD, SSSD_KV8_INT8, 1>(a, rt_prefix, rt, s) : launch_shared<HD, SSSD_KV8_INT8, 2>(a, rt_prefix, rt, s);
}

}  // namespace

// Row tiles of a wave, and how many workgroups go over a prefix at most, for groups that are all alike and prefixes as long as they can be; shorter ones take fewer (prefix_cut).  Few rows: a workgroup's waves are on different segments.  Else, with s workgroups to
// a row tile and prefix, about
//     blocks / s * (0.65 us, or half as much again where compute units have two of them, in as many rounds as they come in) + s * rows * nkv * 264 ps, for 528 bytes of partial results a row, out and in, at 4 TB/s
// and 0.04 us a segment for what the joining of it takes.  us, by that / as many as the chip holds: best of eight with 9 rows on 2048 positions 31 / 37, 32 sequences of 4 rows on 2000
// of 70B 41 / 49, two prompts of 70B 64 / 64, 64 of one on 32768 and 16 of 9 on 4096 the same.  More workgroups than find something to do hold those that lie behind them up by some 3 us.
Kv8SharedPlan kv8_shared_plan(int B, int n, int gq, int nkv, int blocks, int groups, bool f32)
{
    Kv8SharedPlan p{};
    const int64_t rows = (int64_t)B * n * gq, each = groups > 0 ? (rows + groups - 1) / groups : rows;
    const int64_t tiles = (each + 15) / 16;
    if (tiles <= 2) {
        p.rt = (int)tiles;
        p.wave_rows = 1;
    } else {
        p.rt = f32 || tiles <= 4 ? 1 : 2;
        p.wave_rows = 4;
    }
    const int64_t per = p.wave_rows * p.rt * 16;
    p.tiles = (int)((rows + per - 1) / per + std::max(groups, 1) - 1);
    const int64_t tiles_all = (each + per - 1) / per * (groups > 0 ? groups : 1), units = tiles_all * nkv;
    const int sub = 4 / p.wave_rows;   // segments of a workgroup
    const double segment_cost = (double)rows * nkv * 2.64e-4 + 0.04;
    auto on_die = [&](int64_t s) { return tiles_all * ((s * nkv + 7) / 8); };   // workgroups on a die at most, of 32 compute units
    double best = 0;
    p.share = 1;
    for (int64_t s = 1; s == 1 || (s <= 64 && s * units <= KV8_GROUPS && (s - 1) * sub * 4 < blocks); ++s) {
        const double cost = std::ceil((double)blocks / (s * sub)) * (on_die(s) <= 32 ? 0.65 : 0.975 * ((on_die(s) + 63) / 64)) + s * sub * segment_cost;
        if (s == 1 || cost < best) {
            best = cost;
            p.share = (int)s;
        }
    }
    p.us = 18 + best;
    p.segments = p.share * sub;
    p.once = 0;
    for (int s = p.share; s > 0 && !p.once; --s)
        if (on_die(s) <= 32) p.once = s * sub;
    p.cost = (float)segment_cost;
    return p;
}

// The same of a call whose sequences go by themselves: a block takes a workgroup so much by row tiles, and more where compute units have several workgroups; or what it takes to get it there, the less
// the more of a group's sequences, and passes of theirs, read the same one at the same time.  Of 384 batches of 4 to 64 sequences in up to eight groups, with 1 to 32 rows, of 8B, 70B and other numbers of heads, on
// 512 to 32768 positions, and of 152 others in up to 128 groups, whichever is said to be the lesser took 0.3 and 0.8 % longer than whichever was, all going by themselves 14 and 20 %, none 30 and 21 %; it takes one
// kv head with many rows to be joined faster than it is (24 of 9 rows of 32 heads, bf16, 16384: by themselves 88, joined 160).  us, by themselves / joined, five in a row in a graph: 32 of 9 rows of 8B bf16
// 512 15.1 / 29.8, 2048 28.6 / 41.7, 8192 80.4 / 70.5, 32768 264 / 192, f32 18.0 / 31.8, 34.9 / 47.8, 97.8 / 108, 351 / 365; 8 of one row bf16 9.4 / 14.9, 12.4 / 15.7, 27.1 / 19.3, 84.0 / 28.7.  Like the plans it
// goes by how long sequences can be.
static double apart_us(int B, int groups, int nkv, int tiles, int blocks, bool f32, const Kv8Plan &p)
{
    static const double block[2][KV8_MAX_TILES + 1] = {{0, 0.142, 0.20, 0.29}, {0, 0.178, 0.243, 0.326}};
    const int rt = (tiles + p.passes - 1) / p.passes;
    const double rounds = (double)B * nkv * p.passes * p.share / 256, same = (double)B / std::max(groups, 1) * p.passes;
    const double longer = rounds <= 1 ? 1 : std::ceil(rounds) * (!f32 ? 0.77 : rt == 1 ? 0.83 : 1);
    return 13 + blocks * std::max(block[f32][rt] * longer, 0.30 * std::min(1.0, 8 / same) * std::max(1.0, rounds)) / p.share;
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
    if (!lens || B <= 0 || n <= 0 || groups < 0 || (groups > 0 && (!starts || !shared)) || !workspace || (uintptr_t)workspace % ALIGN || !kv->workspace ||
        (uintptr_t)kv->workspace % ALIGN)
        return SSSD_EINVAL;
    size_t need = 0;
    if ((rc = sssd_kv8_shared_sizes(&c, B, n, &need))) return rc;
    if (groups > B || ws_bytes < need || kv->ws_bytes < S.ws_bytes) return SSSD_ECAPACITY;
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
    const Kv8SharedPlan p = kv8_shared_plan(B, n, a.gq, c.n_kv_heads, S.blocks_per_seq, groups, !a.q.bf16);
    a.groups = groups; a.starts = starts; a.shared = shared;
    hipStream_t s = (hipStream_t)stream;
    if ((groups == 0 || apart_us(B, groups, c.n_kv_heads, tiles, S.blocks_per_seq, !a.q.bf16, a.plan) <= p.us) && (int64_t)B * c.n_q_heads <= MOST_THREADS / (32 * 256)) {
        a.hand.polls = kv->flags & SSSD_NO_WAIT ? 0 : HAND_POLLS;
        HIP_TRY(launch_kv8_apart(a, c.format, c.head_dim, kv->workspace, s));
        return SSSD_OK;
    }
    a.tiles = p.tiles; a.wave_rows = p.wave_rows; a.prefix_share = p.share; a.prefix_segments = p.segments;
    a.prefix_once = p.once;
    a.prefix_cost = p.cost;
    a.rows_all = B * n * a.gq;
    a.part_o = (float *)workspace;
    a.part_ml = reinterpret_cast<f32x4 *>(a.part_o + (size_t)(p.segments + a.plan.share) * c.n_kv_heads * a.rows_all * c.head_dim);
    // workgroups of 256 threads
    if (((int64_t)c.n_kv_heads * p.share + 7) / 8 * 8 * p.tiles + ((int64_t)B * c.n_kv_heads + 7) / 8 * 8 * a.plan.share * a.plan.passes > MOST_THREADS / 256)
        return SSSD_ECAPACITY;
    const int rt = (tiles + a.plan.passes - 1) / a.plan.passes;
    HIP_TRY(c.head_dim == 128 ? launch_format<128>(a, c.format, p.rt, rt, s) : launch_format<64>(a, c.format, p.rt, rt, s));
    return SSSD_OK;
}

}  // extern "C"
