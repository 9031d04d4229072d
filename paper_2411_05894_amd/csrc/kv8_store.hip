// Rotary positions, and writing, reading back and committing rows of a KV cache in 8 bits.
//
// All of it is bound by memory for prompts and by a launch and two or three dependent round trips for a step's few rows.  Captured, inputs in memory: a
// rotation of 9 rows 3.2 us (the launch alone 3), of 8191 rows of 40 heads of 128 in bf16 38.5 (168 MB, 4.4 TB/s); an append of 9 rows in 8 heads 4.9, with
// 32 heads of queries the same, of 100001 rows 132 (614 MB, 4.7 TB/s; a copy of 1 GiB 5.2), with the queries 455 (5.0 TB/s); reading 9 rows back 3.7, 32768 48
// (4.2 TB/s); committing trees of 9 rows of 16 sequences in 32 layers 46, of which writing each touched block anew needs 13 (67 MB) and the two launches 6.
//
// A block's scale needs all of its live rows, so a workgroup takes whole blocks: 32 rows of a head, sixteen values a thread, in the order of K's records.
// Rows that were there before are taken out of their codes and go through the new scale like new ones.
#include "kv8.h"

namespace {

// ------------------------------------------------------------------------------------------------ codes ----
// The scale of a block of largest finite magnitude `most`: the smallest power of two with most <= 448 s or 127 s, at least 2^-126; 1 for
// none.  From the bits: most = 1.m * 2^(E-127), and 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6.
template <int FMT> __device__ __forceinline__ float block_scale(float most)
{
    const int bits = (int)f32_bits(most), e = bits >> 23, m = bits & 0x7FFFFF;
    const int x = FMT == SSSD_KV8_E4M3 ? e - 8 + (m > 0x600000) : e - 6 + (m > 0x7E0000);   // biased exponent of the scale
    return bits == 0 ? 1.f : bits_f32((uint32_t)max(x, 1) << 23);
}

// Magnitudes of new rows above LARGEST are taken as infinite: rounded up, they would stand for 2^128.  What the cache holds is finite; the largest code, in place of
// an infinite value beside one of 2^127, stands for more.
constexpr float LARGEST = 0x1p127f, LARGEST_HELD = 0x1.fffffep127f;

// Four codes of values already divided by the scale.
template <int FMT> __device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d)
{
    if (FMT == SSSD_KV8_E4M3) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
    auto code = [](float x) { return (uint32_t)((int)__builtin_rintf(x) + 128); };
    return code(a) | code(b) << 8 | code(c) << 16 | code(d) << 24;
}
template <int FMT> __device__ __forceinline__ void from_codes(uint32_t w, float s, float *x)
{
    if (FMT == SSSD_KV8_E4M3) {
        const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo[0] * s;
        x[1] = lo[1] * s;
        x[2] = hi[0] * s;
        x[3] = hi[1] * s;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)((int)(w >> (8 * i) & 0xFFu) - 128) * s;
    }
}
// Both runs of a thread (Place) over the scale, as codes.
template <int FMT> __device__ __forceinline__ u32x4 row_codes(const float (&x)[8], const float (&y)[8], float inv)
{
    return u32x4{to_codes<FMT>(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), to_codes<FMT>(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv),
                 to_codes<FMT>(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv), to_codes<FMT>(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)};
}
template <int FMT> constexpr float largest_code() { return FMT == SSSD_KV8_E4M3 ? 448.f : 127.f; }

// What a workgroup of an append or a read is there for (the same for all lanes, which a quotient hides from the compiler: it would load lens and pages
// lane by lane).
struct StorePlace {
    int b, step, h0, h1;
    __device__ __forceinline__ StorePlace(const Kv8StoreArgs &a, int id)
    {
        const int x = __builtin_amdgcn_readfirstlane((uint32_t)id / (uint32_t)a.chunks);
        h0 = (id - x * a.chunks) * a.per;
        h1 = min(h0 + a.per, a.g.nkv);
        b = __builtin_amdgcn_readfirstlane((uint32_t)x / (uint32_t)a.blocks);
        step = x - b * a.blocks;
    }
};

// Largest magnitude over a workgroup of 2 * HD threads.
template <int HD> __device__ __forceinline__ float group_max(float x, float *most_s)
{
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) x = fmaxf(x, __shfl_xor(x, i));
    if ((threadIdx.x & 63) == 0) most_s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = most_s[0];
#pragma unroll
    for (int w = 1; w < HD / 32; ++w) x = fmaxf(x, most_s[w]);
    return x;
}

// A thread of a workgroup on a block: two runs of eight channels of one row, `c` and `c + HD/2`; for K that is record threadIdx.x.
template <int HD> struct Place {
    int row, c;
    __device__ __forceinline__ Place()
    {
        const int rec = threadIdx.x, l = rec & 63, p = (rec >> 6) % (HD / 64), u = (rec >> 6) / (HD / 64);
        row = 16 * u + (l & 15);
        c = 32 * p + 8 * (l >> 4);
    }
};

// V records pass through LDS, [row][channel] with rows HD + 4 bytes apart (a wave's byte accesses then spread over the banks).
template <int HD> struct Turn {
    static constexpr int PITCH = HD + 4;
    static __device__ __forceinline__ void place(int e, int &row, int &ch)   // byte e of record threadIdx.x
    {
        const int l = threadIdx.x & 63, p = threadIdx.x >> 6, q = l >> 4, i = e & 7;
        row = (i < 4 ? 0 : 12) + 4 * q + i;
        ch = 32 * p + 16 * (e >> 3) + (l & 15);
    }
    // record -> the thread's row
    static __device__ __forceinline__ u32x4 rows(const u32x4 &rec, uint8_t *lds, const Place<HD> &at)
    {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            int row, ch;
            place(e, row, ch);
            lds[row * PITCH + ch] = (uint8_t)(rec[e >> 2] >> (8 * (e & 3)));
        }
        __syncthreads();
        const uint8_t *a = lds + at.row * PITCH + at.c;
        auto word = [](const uint8_t *x) { return *reinterpret_cast<const uint32_t *>(x); };
        return u32x4{word(a), word(a + 4), word(a + HD / 2), word(a + HD / 2 + 4)};
    }
    // the thread's row -> record
    static __device__ __forceinline__ u32x4 record(const u32x4 &mine, uint8_t *lds, const Place<HD> &at)
    {
        uint8_t *a = lds + at.row * PITCH + at.c;
        auto put = [](uint8_t *x, uint32_t w) { *reinterpret_cast<uint32_t *>(x) = w; };
        put(a, mine[0]);
        put(a + 4, mine[1]);
        put(a + HD / 2, mine[2]);
        put(a + HD / 2 + 4, mine[3]);
        __syncthreads();
        u32x4 rec = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            int row, ch;
            place(e, row, ch);
            rec[e >> 2] |= (uint32_t)lds[row * PITCH + ch] << (8 * (e & 3));
        }
        return rec;
    }
};

template <int HD> __device__ __forceinline__ u32x4 *block_record(uint8_t *codes, int page, int nkv, int h, int is_v)
{
    return reinterpret_cast<u32x4 *>(codes + ((size_t)page * nkv + h) * (64 * HD) + is_v * (32 * HD)) + threadIdx.x;
}

// ------------------------------------------------------------------------------------------------- rope ----
// Both runs of a Place rotated, of a head that is rotated as a whole: by halves they are each other's partners, and neighbours lie in a run.  angle(i): cos
// and sin of the thread's i-th of eight.
template <typename Angle> __device__ __forceinline__ void rotate_whole(bool neighbours, Angle angle, float (&x)[8], float (&y)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float &a = neighbours ? (i < 4 ? x[2 * i & 7] : y[2 * i & 7]) : x[i];
        float &b = neighbours ? (i < 4 ? x[(2 * i & 7) + 1] : y[(2 * i & 7) + 1]) : y[i];
        const float2 t = angle(i);
        const float u = a;
        a = u * t.x - b * t.y;
        b = b * t.x + u * t.y;
    }
}
// ... of a head whose first channels are.  cs: the angles of the row's pairs.  By halves the partners are fetched again (they are in a cache: another
// thread of the workgroup has just read them).
template <int HD>
__device__ __forceinline__ void rotate_part(const Rope8 &rp, const Rows8 &r, const char *row, int c0, const float2 *cs, float (&x)[8], float (&y)[8])
{
    const int half = rp.r >> 1;
    auto run = [&](int ch, float (&v)[8]) {
        if (ch >= rp.r) return;
        if (rp.neighbours) {
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                if (ch + i < rp.r) {
                    const float2 t = cs[(ch + i) >> 1];
                    const float u = v[i];
                    v[i] = u * t.x - v[i + 1] * t.y;
                    v[i + 1] = v[i + 1] * t.x + u * t.y;
                }
        } else if (half % 8 == 0) {
            const bool low = ch < half;
            float other[8];
            load8(r, row, low ? ch + half : ch - half, other);
            cs += low ? ch : ch - half;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = low ? v[i] * cs[i].x - other[i] * cs[i].y : v[i] * cs[i].x + other[i] * cs[i].y;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (ch + i < rp.r) {
                    const bool low = ch + i < half;
                    const float2 t = cs[low ? ch + i : ch + i - half];
                    const float other = load1(r, row, low ? ch + i + half : ch + i - half);
                    v[i] = low ? v[i] * t.x - other * t.y : v[i] * t.x + other * t.y;
                }
        }
    };
    asm volatile("" : "+v"(c0));   // addresses and angles anew for every head: kept over the loop, they would take a hundred registers
    run(c0, x);
    run(c0 + HD / 2, y);
}

// Rows of heads rotated by a workgroup of T threads: R rows, heads h0 .. h1-1 of each.  The angles of the rows' pairs are worked out once, in LDS
// (some thirty instructions each); then the threads pass over the rows in the order of memory, a unit each: by halves U pairs (i .. i+U-1 with
// their partners), as neighbours U/2 pairs that lie in a row, or U channels that pass.
// Measured against a thread with the angles of eight pairs in registers that takes them through several heads (32 places of 256 bytes at a time, a
// row's stride apart): 8191 rows of 40 heads of 128, bf16, 49.6 -> 43.5 us cold, now 38.5 (168 MB, 4.4 TB/s; a copy of 1 GiB 5.2).
struct RopeRow {
    int b, j, position, on;   // on: 0 where the row is left as it is
};
template <int T, int U, typename Row>
__device__ __forceinline__ void rope_units(const Rope8 &rp, const Rows8 &x, const Rows8 &out, const RopeWork &w, int rows, int h0, int h1, const float2 *table, Row row)
{
    const int half = rp.r >> 1, units = w.units;
    const bool halves = !rp.neighbours;
    const int turning = halves ? half / U : rp.r / U;      // U divides them
    const uint32_t per_row = (uint32_t)(h1 - h0) * units, all = per_row * rows;
    for (uint32_t i = threadIdx.x; i < all; i += T) {
        uint32_t r = 0, z = i;   // a workgroup's rows are ROPE_ROWS at most
#pragma unroll
        for (int y = 1; y < ROPE_ROWS; ++y)
            if (z >= per_row) {
                z -= per_row;
                ++r;
            }
        const uint32_t h = (uint32_t)w.by_units((int)z);
        const int unit = (int)(z - h * units);
        const RopeRow at = row((int)r);
        if (!at.on) continue;
        const char *src = x.at(at.b, at.j, h0 + (int)h);
        char *dst = out.at(at.b, at.j, h0 + (int)h);
        const bool pass = unit >= turning;
        const int ch = pass ? rp.r + (unit - turning) * U : unit * U;
        const float2 *cs = table + r * half;
        if constexpr (U == 8) {
            float v[8];
            if (pass) {
                if (x.p == out.p) continue;
                load8(x, src, ch, v);
            } else if (halves) {
                float u[8], y[8];
                load8(x, src, ch, u);
                load8(x, src, ch + half, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 t = cs[ch + e];
                    v[e] = u[e] * t.x - y[e] * t.y;
                    y[e] = y[e] * t.x + u[e] * t.y;
                }
                store8(out, dst, ch + half, y);
            } else {
                load8(x, src, ch, v);
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float2 t = cs[(ch + e) >> 1];
                    const float u = v[e];
                    v[e] = u * t.x - v[e + 1] * t.y;
                    v[e + 1] = v[e + 1] * t.x + u * t.y;
                }
            }
            store8(out, dst, ch, v);
        } else if (pass) {
            if (x.p == out.p) continue;
            for (int e = 0; e < U && ch + e < w.d; ++e) store1(out, dst, ch + e, load1(x, src, ch + e));
        } else {   // a pair
            const int other = halves ? ch + half : ch + 1;
            const float2 t = cs[halves ? ch : ch >> 1];
            float u, y;
            load_pair(x, src, ch, other, u, y);
            const float v = u * t.x - y * t.y, w = y * t.x + u * t.y;
            if (out.bf16) {
                reinterpret_cast<uint16_t *>(dst)[ch] = (uint16_t)pack_bf16x2(v, 0.f);
                reinterpret_cast<uint16_t *>(dst)[other] = (uint16_t)pack_bf16x2(w, 0.f);
            } else {
                reinterpret_cast<float *>(dst)[ch] = v;
                reinterpret_cast<float *>(dst)[other] = w;
            }
        }
    }
}
template <int T, typename Row>
__device__ __forceinline__ void rope_rows(const Rope8 &rp, const Rows8 &x, const Rows8 &out, const RopeWork &w, int group, int chunk, float2 *table, RopeRow *rows_s, Row row)
{
    const uint32_t row0 = (uint32_t)group * w.rows;
    const int rows = (int)min((uint32_t)w.rows, w.total - row0), half = rp.r >> 1;
    if ((int)threadIdx.x < rows) rows_s[threadIdx.x] = row(row0 + threadIdx.x);
    __syncthreads();
    for (int i = threadIdx.x; i < rows * half; i += T) {
        const int r = rp.by_half(i);
        rope_cos_sin(rp, rows_s[r].position, rp.turns[i - r * half], table[i].x, table[i].y);
    }
    __syncthreads();
    const int h0 = chunk * w.per, h1 = min(h0 + w.per, w.heads);
    auto of = [&](int r) { return rows_s[r]; };
    if (w.unit == 8) rope_units<T, 8>(rp, x, out, w, rows, h0, h1, table, of);
    else if (w.unit == 2) rope_units<T, 2>(rp, x, out, w, rows, h0, h1, table, of);
    else rope_units<T, 1>(rp, x, out, w, rows, h0, h1, table, of);
}

struct RopeArgs {
    Rows8 x, out;
    const int32_t *positions;
    Rope8 rope;
    RopeWork w;
};

__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a)
{
    __shared__ float2 table[ROPE_TABLE];
    __shared__ RopeRow rows_s[ROPE_ROWS];
    rope_rows<256>(a.rope, a.x, a.out, a.w, blockIdx.x, blockIdx.y, table, rows_s, [&](uint32_t row) {
        const uint32_t b = row / a.w.n;
        return RopeRow{(int)b, (int)(row - b * a.w.n), a.positions[row], 1};
    });
}

// The page of block `step` of the rows that a call moves for sequence b, or -1: a block past them, or the sequence is rejected, which one of
// its workgroups (`tell`) reports.  Every workgroup looks at all pages of the sequence, so that its blocks agree.
template <int T> __device__ __forceinline__ int touched_page(const Kv8StoreArgs &a, int b, int step, bool tell, int &len, int &count)
{
    const bool fits = kv8_rows(a.lens, a.counts, b, a.n, a.g.max_seq, len, count);
    if (!fits) {
        if (tell && step == 0 && threadIdx.x == 0) atomicOr(a.status, KV8_RANGE);
        return -1;
    }
    const int blk0 = len >> 5, last = (len + count - 1) >> 5;
    if (count == 0 || blk0 + step > last) return -1;
    if (a.g.table) {
        bool bad = false;
        const int32_t *entries = a.g.table + (size_t)(a.first + b) * a.g.blocks_per_seq + blk0;
        const int n = last - blk0 + 1;
        for (int i = (int)threadIdx.x * 4; i < n; i += T * 4) {   // four at a time, the last four once more
            int32_t four[4];
            if (n >= 4) {
                __builtin_memcpy(four, entries + min(i, n - 4), sizeof(four));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) four[e] = entries[min(e, n - 1)];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) bad |= (uint32_t)four[e] >= (uint32_t)a.g.n_pages;
        }
        if (__syncthreads_or(bad)) {
            if (tell && step == 0 && threadIdx.x == 0) atomicOr(a.status, KV8_RANGE);
            return -1;
        }
    }
    return kv8_entry(a.g, a.first + b, blk0 + step);
}

// ----------------------------------------------------------------------------------------------- append ----
// Workgroup = (sequence, touched block, `per` kv heads, K or V), MANY: more than one; behind them the workgroups that rotate queries.
template <int HD, int FMT, bool MANY> __global__ __launch_bounds__(2 * HD) void append_kernel(Kv8StoreArgs a, int storing)
{
    constexpr int T = 2 * HD, PITCH = HD / 2 + 2;
    __shared__ float most_s[2][HD / 32];
    __shared__ __align__(16) uint8_t turn_s[32 * Turn<HD>::PITCH];
    __shared__ __align__(16) float2 table[32 * PITCH];   // angles of the block's rows, or of a workgroup's rows of queries
    __shared__ RopeRow rows_s[ROPE_ROWS];
    warm(a);
    const int lane = threadIdx.x & 63;
    int id = blockIdx.x;
    int len, count;
    if (id >= storing) {
        id -= storing;
        const int groups = (int)((a.work.total + a.work.rows - 1) / a.work.rows), chunk = id / groups;
        rope_rows<T>(a.rope, a.q, a.q_out, a.work, id - chunk * groups, chunk, table, rows_s, [&](uint32_t row) {
            RopeRow r;
            r.b = (int)(row / a.work.n);
            r.j = (int)row - r.b * a.n;
            int len, count;
            r.on = kv8_rows(a.lens, a.counts, r.b, a.n, a.g.max_seq, len, count) && r.j < count;
            r.position = len + r.j;
            if (a.parents && r.on) {   // a thread walks up; a workgroup has few rows
                const int32_t *up = a.parents + (size_t)r.b * a.n;
                int depth = 0;
                for (int x = r.j; x > 0; ++depth) {
                    const int y = up[x];
                    x = y < 0 || y >= x ? x - 1 : y;
                }
                r.position = len + depth;
            }
            return r;
        });
        return;
    }
    const int is_v = id & 1;
    id >>= 1;
    const StorePlace w(a, id);
    const int b = w.b, step = w.step, h0 = w.h0, h1 = w.h1;
    const Place<HD> at;
    const bool turns = !is_v && a.rope.turns, whole = a.rope.r == HD;
    double mine[8];   // the frequencies of the thread's angles, requested ahead of what depends on lens
    if (turns && whole) {
#pragma unroll
        for (int i = 0; i < 8; ++i) mine[i] = a.rope.turns[a.rope.neighbours ? (at.c >> 1) + (i & 3) + (i >> 2) * (HD / 4) : at.c + i];
    }
    const int page = touched_page<T>(a, b, step, h0 == 0 && !is_v, len, count);
    if (page < 0) return;
    const int blk = (len >> 5) + step;
    const int j = blk * 32 + at.row - len;
    const Rows8 &in = is_v ? a.v : a.k;
    const bool is_new = j >= 0 && j < count;
    const char *row = in.at(b, is_new ? j : 0, h0);
    const int64_t next = in.hs * (in.bf16 ? 2 : 4);
    // A head's rows, and what the block holds of it, are requested while the one before it is stored.
    const bool holds = blk * 32 < len;   // older rows
    u32x4 raw[4], old{};
    float s_old = 0.f;
    auto scale_of = [&](int h) { return reinterpret_cast<float *>(a.scales + (size_t)page * a.g.nkv + h) + is_v; };
    auto fetch = [&](int h, const char *from) {
        if (holds) {
            old = *block_record<HD>(a.codes, page, a.g.nkv, h, is_v);
            s_old = *scale_of(h);
        }
        if (is_new) {
            fetch8(in, from, at.c, raw[0], raw[1]);
            fetch8(in, from, at.c + HD / 2, raw[2], raw[3]);
        }
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = u32x4{0, 0, 0, 0};
    fetch(h0, row);
    // Angles once for all heads, in LDS (in registers they would leave fewer waves): a thread its own eight, or, of a head that is rotated in part, all
    // threads those of the block's rows between them.  us of a prompt of 32768 in 8 heads of 128: angles for every head anew 67, once 50.
    f32x4 *own = reinterpret_cast<f32x4 *>(table) + threadIdx.x;   // cos and sin of two angles at own[T * i]
    float2 here[8];                                                // ... of one head alone
    auto angle = [&](int i) {
        if (!MANY) return here[i];
        const f32x4 t = own[T * (i >> 1)];
        return float2{t[2 * (i & 1)], t[2 * (i & 1) + 1]};
    };
    if (turns) {
        uint32_t word = 0;
        if (a.parents) {
            bool bad;
            word = kv8_tree_word(lane < count ? a.parents[(size_t)b * a.n + lane] : 0, count, lane, bad);
            if (step == 0 && h0 == 0 && threadIdx.x < 64 && __any(bad) && lane == 0) atomicOr(a.status, KV8_RANGE);
        }
        auto position = [&](int j) { return len + (a.parents ? __popc((uint32_t)__shfl((int)word, j & 31)) - 1 : j); };
        if (whole) {
            const int p = position(j);
            if (!MANY) {
#pragma unroll
                for (int i = 0; i < 8; ++i) rope_cos_sin(a.rope, p, mine[i], here[i].x, here[i].y);
            } else if (is_new) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float c0, s0, c1, s1;
                    rope_cos_sin(a.rope, p, mine[2 * i], c0, s0);
                    rope_cos_sin(a.rope, p, mine[2 * i + 1], c1, s1);
                    own[T * i] = f32x4{c0, s0, c1, s1};
                }
            }
        } else {
            const int first = max(len - blk * 32, 0), half = a.rope.r >> 1, all = (min(len + count - blk * 32, 32) - first) * half;
#pragma unroll 1
            for (int base = 0; base < all; base += T) {
                const int e = min(base + (int)threadIdx.x, all - 1), r = a.rope.by_half(e), i = e - r * half;
                float2 t;
                rope_cos_sin(a.rope, position(blk * 32 + first + r - len), a.rope.turns[i], t.x, t.y);
                table[(first + r) * PITCH + i] = t;
            }
            __syncthreads();
        }
    }
    int h = h0;
    do {
        float x[8], y[8];
        decode8(in, raw[0], raw[1], x);
        decode8(in, raw[2], raw[3], y);
        if (holds) {
            if (is_v) {
                if (MANY && h > h0) __syncthreads();   // turn_s has been read
                old = Turn<HD>::rows(old, turn_s, at);
                __syncthreads();   // ... again
            }
            if (j < 0) {
                from_codes<FMT>(old[0], s_old, x);
                from_codes<FMT>(old[1], s_old, x + 4);
                from_codes<FMT>(old[2], s_old, y);
                from_codes<FMT>(old[3], s_old, y + 4);
            }
        }
        if (turns && is_new) {
            if (!whole) rotate_part<HD>(a.rope, in, row, at.c, table + at.row * PITCH, x, y);
            else if (a.rope.neighbours) rotate_whole(true, angle, x, y);
            else rotate_whole(false, angle, x, y);
        }
        if (MANY && h + 1 < h1) fetch(h + 1, row + next);
        float most = 0.f;
        bool odd = false;
        const float largest = j < 0 ? LARGEST_HELD : LARGEST;
        auto finite = [&](float x) { return fabsf(x) <= largest; };
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            most = fmaxf(most, fmaxf(finite(x[i]) ? fabsf(x[i]) : 0.f, finite(y[i]) ? fabsf(y[i]) : 0.f));
            odd |= !finite(x[i]) || !finite(y[i]);
        }
        const float s = block_scale<FMT>(group_max<HD>(most, most_s[h & 1])), inv = bits_f32((254u << 23) - f32_bits(s));
        if (__any(odd)) {
            if (lane == 0) atomicOr(a.status, KV8_NOT_FINITE);
            const float top = largest_code<FMT>() * s;
            auto mend = [&](float z) { return finite(z) ? z : z != z ? 0.f : copysignf(top, z); };
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = mend(x[i]);
                y[i] = mend(y[i]);
            }
        }
        const u32x4 mine = row_codes<FMT>(x, y, inv);
        *block_record<HD>(a.codes, page, a.g.nkv, h, is_v) = is_v ? Turn<HD>::record(mine, turn_s, at) : mine;   // the next head's codes come behind the barrier of its maximum
        if (threadIdx.x == 0) *scale_of(h) = s;
        row += next;
    } while (MANY && ++h < h1);
}

// ------------------------------------------------------------------------------------------------- read ----
template <int HD, int FMT> __global__ __launch_bounds__(2 * HD) void read_kernel(Kv8StoreArgs a)
{
    __shared__ __align__(16) uint8_t turn_s[32 * Turn<HD>::PITCH];
    int id = blockIdx.x;
    const int is_v = id & 1;
    id >>= 1;
    const StorePlace w(a, id);
    const int b = w.b, step = w.step, h0 = w.h0, h1 = w.h1;
    int start, count;
    const int page = touched_page<2 * HD>(a, b, step, h0 == 0 && !is_v, start, count);
    if (page < 0) return;
    const int blk = (start >> 5) + step;
    const Place<HD> at;
    const int j = blk * 32 + at.row - start;
    const bool wanted = j >= 0 && j < count;
    const Rows8 &out = is_v ? a.v : a.k;
    char *row = out.at(b, wanted ? j : 0, h0);
    const float *scale = reinterpret_cast<const float *>(a.scales + (size_t)page * a.g.nkv) + is_v;
    u32x4 rec = *block_record<HD>(a.codes, page, a.g.nkv, h0, is_v);
    float s = scale[2 * h0];
    for (int h = h0; h < h1; ++h, row += out.hs * (out.bf16 ? 2 : 4)) {
        const int ahead = min(h + 1, h1 - 1);
        const u32x4 rec_next = *block_record<HD>(a.codes, page, a.g.nkv, ahead, is_v);
        const float s_next = scale[2 * ahead];
        if (is_v) {
            if (h > h0) __syncthreads();   // turn_s has been read
            rec = Turn<HD>::rows(rec, turn_s, at);
        }
        if (wanted) {
            float x[8], y[8];
            from_codes<FMT>(rec[0], s, x);
            from_codes<FMT>(rec[1], s, x + 4);
            from_codes<FMT>(rec[2], s, y);
            from_codes<FMT>(rec[3], s, y + 4);
            store8(out, row, at.c, x);
            store8(out, row, at.c + HD / 2, y);
        }
        rec = rec_next;
        s = s_next;
    }
}

// ----------------------------------------------------------------------------------------------- commit ----
// Whether a sequence's step is committed; acc: accepted drafts, node: in lanes 1..acc of every wave, what lies there.
__device__ __forceinline__ bool commit_ok(const Kv8StoreArgs &g, const int32_t *accepted, const int32_t *path, int b, int &len, int &acc, int &node)
{
    const int lane = threadIdx.x & 63;
    len = g.lens[b];
    acc = accepted[b];
    node = lane;
    if (len < 0 || acc < 0 || acc >= g.n) return false;
    if (path) {
        if (lane > 0 && lane <= acc) node = path[(size_t)b * g.n + lane];
        const int before = __shfl_up(node, 1);
        if (!__all(lane == 0 || lane > acc || (node > before && node < g.n))) return false;
    }
    const int farthest = __shfl(node, acc);   // the path's last row
    if ((int64_t)len + farthest >= g.g.max_seq) return false;
    const int blk = (len >> 5) + lane;
    bool ok = true;
    if (blk <= (len + farthest) >> 5) {
        const int page = kv8_entry(g.g, b, blk);
        ok = page >= 0 && page < g.g.n_pages;
    }
    return __all(ok);
}

// Workgroup = (layer, sequence, kv head, K or V): the one or two blocks that a step's rows lie in are taken apart, their live rows put in
// place and both blocks written anew, each with the scale of what it holds then.  Paths that move nothing are left alone.
template <int HD, int FMT>
__global__ __launch_bounds__(2 * HD) void commit_kernel(Kv8StoreArgs a, const int32_t *accepted, const int32_t *path)
{
    __shared__ float most_s[HD / 32];
    __shared__ __align__(16) uint8_t rows_s[2][32 * HD], turn_s[32 * Turn<HD>::PITCH];
    int id = blockIdx.x;
    const int is_v = id & 1;
    id >>= 1;
    const int x0 = (uint32_t)id / (uint32_t)a.g.nkv, h = id - x0 * a.g.nkv, layer = (uint32_t)x0 / (uint32_t)a.B, b = x0 - layer * a.B;
    int len, acc, node;
    if (!commit_ok(a, accepted, path, b, len, acc, node)) return;   // the launch that advances lens reports it
    const int farthest = __shfl(node, acc);
    if (farthest == acc) return;                                    // strictly increasing from 1: nothing moves
    const Place<HD> at;
    uint8_t *codes = a.codes + layer * a.layer_bytes;
    float2 *scales = reinterpret_cast<float2 *>(reinterpret_cast<char *>(a.scales) + layer * a.layer_bytes);
    const int blk0 = len >> 5, from_last = (len + farthest) >> 5, to_last = (len + acc) >> 5;
    float s_old[2] = {1.f, 1.f};
    for (int x = 0; x <= from_last - blk0; ++x) {   // at most two
        const int page = kv8_entry(a.g, b, blk0 + x);
        u32x4 rec = *block_record<HD>(codes, page, a.g.nkv, h, is_v);
        const float2 both = scales[(size_t)page * a.g.nkv + h];
        s_old[x] = is_v ? both.y : both.x;
        if (is_v) {
            rec = Turn<HD>::rows(rec, turn_s, at);
            __syncthreads();
        }
        uint32_t *to = reinterpret_cast<uint32_t *>(rows_s[x] + at.row * HD + at.c);
        to[0] = rec[0];
        to[1] = rec[1];
        to[HD / 8] = rec[2];
        to[HD / 8 + 1] = rec[3];
    }
    __syncthreads();
    for (int x = 0; x <= to_last - blk0; ++x) {
        const int page = kv8_entry(a.g, b, blk0 + x), t = (blk0 + x) * 32 + at.row, i = t - len;
        float v[8], w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = w[e] = 0.f;
        const int from_node = __shfl(node, max(min(i, acc), 0));
        if (i <= acc) {
            const int src = (i <= 0 ? t : len + from_node) - blk0 * 32;
            const uint32_t *from = reinterpret_cast<const uint32_t *>(rows_s[src >> 5] + (src & 31) * HD + at.c);
            const float s = src < 32 ? s_old[0] : s_old[1];
            from_codes<FMT>(from[0], s, v);
            from_codes<FMT>(from[1], s, v + 4);
            from_codes<FMT>(from[HD / 8], s, w);
            from_codes<FMT>(from[HD / 8 + 1], s, w + 4);
        }
        float most = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, fmaxf(fabsf(v[e]), fabsf(w[e])));
        const float s = block_scale<FMT>(group_max<HD>(most, most_s)), inv = bits_f32((254u << 23) - f32_bits(s));
        u32x4 mine = row_codes<FMT>(v, w, inv);
        if (is_v) mine = Turn<HD>::record(mine, turn_s, at);
        *block_record<HD>(codes, page, a.g.nkv, h, is_v) = mine;
        if (threadIdx.x == 0) (is_v ? scales[(size_t)page * a.g.nkv + h].y : scales[(size_t)page * a.g.nkv + h].x) = s;
        __syncthreads();   // most_s and turn_s are used again
    }
}

__global__ __launch_bounds__(64) void advance_kernel(Kv8StoreArgs a, const int32_t *accepted, const int32_t *path, int32_t *lens)
{
    const int b = blockIdx.x;
    int len, acc, node;
    const bool ok = commit_ok(a, accepted, path, b, len, acc, node);
    if (threadIdx.x != 0) return;
    if (ok) lens[b] = len + acc + 1;
    else atomicOr(a.status, KV8_RANGE);
}

}  // namespace

// Units of eight channels where pairs and the channels that pass divide into them, else single pairs.  A workgroup takes as many rows, with all their
// heads, as have `each` units for a thread, while eight workgroups are left for every compute unit: one in a rotation alone (8191 rows of 40 heads of 128
// in bf16 38.5 us, three rows a workgroup 43.8; 12000 of 16 of 64 14.8, one row a workgroup 17.2), four beside rows that are stored, where a workgroup
// has more to look up first and fewer fit (prompts of 32768 with 32 heads of queries 157, one 175).  Few rows are cut by heads, too.
RopeWork rope_work(int B, int n, int d, int heads, int r, bool neighbours, int threads, int each)
{
    RopeWork w;
    const int turning = neighbours ? r : r / 2;
    w.unit = turning % 8 == 0 && (d - r) % 8 == 0 ? 8 : (neighbours ? 2 : 1);
    w.units = turning / w.unit + (d - r + w.unit - 1) / w.unit;
    w.n = n; w.d = d; w.heads = heads;
    w.total = (uint32_t)B * n;
    const uint32_t fit = ROPE_TABLE * 2 / r, left = w.total / 2048;
    const int64_t fill = (int64_t)threads * each / ((int64_t)heads * w.units);
    w.rows = fill < 1 ? 1 : fill > ROPE_ROWS ? ROPE_ROWS : (uint32_t)fill;
    if (w.rows > left) w.rows = left < 1 ? 1 : left;
    if (w.rows > fit) w.rows = fit;
    const uint32_t groups = (w.total + w.rows - 1) / w.rows;
    const int64_t most = ((int64_t)heads * w.units + threads - 1) / threads;   // a unit for every thread
    int64_t chunks = groups < 512 ? 512 / groups : 1;
    if (chunks > most) chunks = most;
    w.per = (int)((heads + chunks - 1) / chunks);
    const uint32_t exact = UINT32_MAX / w.units / w.units;   // of by_units
    if ((uint32_t)w.per > exact) w.per = exact;
    w.by_units = Div((int)w.units);
    return w;
}

hipError_t launch_rope(const Rows8 &x, const Rows8 &out, const int32_t *positions, const Rope8 &rope, const RopeWork &w, hipStream_t s)
{
    const RopeArgs a{x, out, positions, rope, w};
    hipLaunchKernelGGL(rope_kernel, dim3((w.total + w.rows - 1) / w.rows, (w.heads + w.per - 1) / w.per), dim3(256), 0, s, a);
    return hipGetLastError();
}

#define KV8_LAUNCH(kernel, grid, ...)                                                                          \
    do {                                                                                                       \
        if (d == 128 && fmt == SSSD_KV8_E4M3) KV8_LAUNCH_AS((kernel(128, SSSD_KV8_E4M3)), 256, grid, __VA_ARGS__); \
        else if (d == 128) KV8_LAUNCH_AS((kernel(128, SSSD_KV8_INT8)), 256, grid, __VA_ARGS__);                \
        else if (fmt == SSSD_KV8_E4M3) KV8_LAUNCH_AS((kernel(64, SSSD_KV8_E4M3)), 128, grid, __VA_ARGS__);     \
        else KV8_LAUNCH_AS((kernel(64, SSSD_KV8_INT8)), 128, grid, __VA_ARGS__);                               \
    } while (0)
#define KV8_LAUNCH_AS(kernel, threads, grid, ...) hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), 0, s, __VA_ARGS__)
#define APPEND_ONE(HD, FMT) append_kernel<HD, FMT, false>
#define APPEND_MANY(HD, FMT) append_kernel<HD, FMT, true>
#define READ(HD, FMT) read_kernel<HD, FMT>
#define COMMIT(HD, FMT) commit_kernel<HD, FMT>

// Workgroups of an append or a read, each of `per` kv heads while 800 are left: what is the same for all heads, the angles and the look at every page of
// the sequence, is then done once.  us, one head / several: prompts in 8 heads of 128 with a rotation, 4001 11.8 / 10.8 (two), 8192 20.5 / 16.1 (four),
// 32768 67 / 50 (eight, and with a block table 83 / 54); 16 prompts of 512 20.0 / 16.0; 500 workgroups instead of 800, 4001 11.7 (four), 8192 19.9 (eight).
// Reads have the pages alone: with a table, 100001 221 / 157 (four), 32768 60 / 54.5; without one 48 / 50.
static int store_groups(Kv8StoreArgs &a, int most)
{
    const int64_t all = (int64_t)a.B * a.blocks * 2 * a.g.nkv, per = all / 800;
    if (most > a.g.nkv) most = a.g.nkv;
    a.per = per < 1 ? 1 : per > most ? most : (int)per;
    a.chunks = (a.g.nkv + a.per - 1) / a.per;
    a.per = (a.g.nkv + a.chunks - 1) / a.chunks;
    return a.B * a.blocks * 2 * a.chunks;
}

hipError_t launch_kv8_append(Kv8StoreArgs a, int fmt, int d, hipStream_t s)
{
    const int store = store_groups(a, 8);
    const int turn = a.q.p ? (int)((a.work.total + a.work.rows - 1) / a.work.rows) * ((a.work.heads + a.work.per - 1) / a.work.per) : 0;
    if (a.per > 1) KV8_LAUNCH(APPEND_MANY, store + turn, a, store);
    else KV8_LAUNCH(APPEND_ONE, store + turn, a, store);
    return hipGetLastError();
}

hipError_t launch_kv8_read(Kv8StoreArgs a, int fmt, int d, hipStream_t s)
{
    KV8_LAUNCH(READ, store_groups(a, a.g.table ? 4 : 1), a);
    return hipGetLastError();
}

hipError_t launch_kv8_commit(const Kv8StoreArgs &a, int fmt, int d, int layers, const int32_t *accepted, const int32_t *path, int32_t *lens, hipStream_t s)
{
    if (path) KV8_LAUNCH(COMMIT, layers * a.B * a.g.nkv * 2, a, accepted, path);
    hipLaunchKernelGGL(advance_kernel, dim3(a.B), dim3(64), 0, s, a, accepted, path, lens);
    return hipGetLastError();
}
