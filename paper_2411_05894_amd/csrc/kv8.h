// 8-bit KV cache: layout, codes and what its kernels share (private).
//
// A layer is [page][kv head] records of 64 * head_dim bytes -- the codes of a block of 32 positions, K and then V -- followed by the
// scales, float2 {K, V} per [page][kv head].  Within a record both are in the order in which the matrix instructions take their operands
// (16x16x32: lane l holds row l % 16, 8 k-slots from 8 * (l / 16)), two operand tiles side by side so that a lane's share of both is one
// 16-byte load and a wave's 1 KiB in a row:
//   K: for u (16 positions), p < head_dim/64: lane l's 16 bytes are position 16u + l%16, channels 32p + 8(l/16) .. +7, then the same ones
//      plus head_dim/2 (pairs of a rotation by halves lie in one record: the writer needs no neighbour for them)
//   V: for p < head_dim/32: lane l's 16 bytes are channel 32p + l%16 at positions 4(l/16) .. +3 and 16 + 4(l/16) .. +3, then channel
//      32p + 16 + l%16: the positions whose scores that lane owns after the two score products, so probabilities are operands as they are
// Integer codes are stored plus 128: a byte behind 0x64 is then the float16 1024 + code + 128.
#pragma once
#include "../../include/sssd_kv8.h"
#include "common.h"
#include "handover.h"

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));

constexpr int KV8_BLOCK = 32;   // positions of a page

// Bits of the status word
constexpr int KV8_RANGE = 1, KV8_NOT_FINITE = 2;

// All cache lines of a kernel's arguments requested at once: read where they are used they cost a round trip to memory each, one behind the other.
template <typename T> __device__ __forceinline__ void warm(const T &args)
{
    const uint32_t *p = reinterpret_cast<const uint32_t *>(&args);
#pragma unroll
    for (size_t i = 0; i < sizeof(T) / 4; i += 16) asm volatile("" ::"s"(p[i]));
    asm volatile("" ::"s"(p[sizeof(T) / 4 - 1]));
}

struct Kv8Geom {
    const int32_t *table;   // device [max_batch][blocks_per_seq], or nullptr: contiguous runs
    int blocks_per_seq, n_pages, nkv, max_seq;
};
__device__ __forceinline__ int kv8_entry(const Kv8Geom &g, int b, int blk)
{
    const size_t at = (size_t)b * g.blocks_per_seq + blk;
    return g.table ? g.table[at] : (int)at;
}

// Rows of heads as a kernel takes them (sssd_rows); `vec`: 16 bytes at a time.
struct Rows8 {
    char *p;
    int64_t bs, rs, hs;   // elements
    int bf16, vec;
    __device__ __forceinline__ char *at(int b, int j, int h) const { return p + (b * bs + j * rs + h * hs) * (bf16 ? 2 : 4); }
};
__device__ __forceinline__ void unpack_bf16x8(const u32x4 &u, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bits_f32(u[i] << 16);
        x[2 * i + 1] = bits_f32(u[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ float load1(const Rows8 &r, const char *row, int ch)
{
    return r.bf16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(row)[ch]) : reinterpret_cast<const float *>(row)[ch];
}
__device__ __forceinline__ void load_pair(const Rows8 &r, const char *row, int i, int j, float &x, float &y)   // neither waits for the other
{
    if (r.bf16) {
        const uint16_t u = reinterpret_cast<const uint16_t *>(row)[i], v = reinterpret_cast<const uint16_t *>(row)[j];
        x = bf16_to_f32(u);
        y = bf16_to_f32(v);
    } else {
        x = reinterpret_cast<const float *>(row)[i];
        y = reinterpret_cast<const float *>(row)[j];
    }
}
__device__ __forceinline__ void load8(const Rows8 &r, const char *row, int ch, float (&x)[8])
{
    if (!r.vec) {   // one branch on the type for all eight: none of the loads waits for another
        if (r.bf16) {
            uint16_t u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = reinterpret_cast<const uint16_t *>(row)[ch + i];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = bf16_to_f32(u[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = reinterpret_cast<const float *>(row)[ch + i];
        }
    } else if (r.bf16) {
        unpack_bf16x8(*reinterpret_cast<const u32x4 *>(row + ch * 2), x);
    } else {
        const f32x4 lo = *reinterpret_cast<const f32x4 *>(row + ch * 4), hi = *reinterpret_cast<const f32x4 *>(row + ch * 4 + 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = lo[i];
            x[4 + i] = hi[i];
        }
    }
}
// Eight channels as they were loaded, in one or two registers of 16 bytes: turned into numbers only when they are used, so that nothing waits for them
// before.
__device__ __forceinline__ void fetch8(const Rows8 &r, const char *row, int ch, u32x4 &lo, u32x4 &hi)
{
    if (!r.vec) {
        float x[8];
        load8(r, row, ch, x);
        lo = u32x4{f32_bits(x[0]), f32_bits(x[1]), f32_bits(x[2]), f32_bits(x[3])};
        hi = u32x4{f32_bits(x[4]), f32_bits(x[5]), f32_bits(x[6]), f32_bits(x[7])};
    } else if (r.bf16) {
        lo = *reinterpret_cast<const u32x4 *>(row + ch * 2);
    } else {
        lo = *reinterpret_cast<const u32x4 *>(row + ch * 4);
        hi = *reinterpret_cast<const u32x4 *>(row + ch * 4 + 16);
    }
}
__device__ __forceinline__ void decode8(const Rows8 &r, const u32x4 &lo, const u32x4 &hi, float (&x)[8])
{
    if (r.vec && r.bf16) {
        unpack_bf16x8(lo, x);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = bits_f32(lo[i]);
            x[4 + i] = bits_f32(hi[i]);
        }
    }
}
// bf16: rounded once, to nearest even (what is no number stays none)
__device__ __forceinline__ void store1(const Rows8 &r, char *row, int ch, float x)
{
    if (r.bf16) reinterpret_cast<uint16_t *>(row)[ch] = (uint16_t)pack_bf16x2(x, 0.f);
    else reinterpret_cast<float *>(row)[ch] = x;
}
__device__ __forceinline__ void store8(const Rows8 &r, char *row, int ch, const float (&x)[8])
{
    if (!r.vec) {
        if (r.bf16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) reinterpret_cast<uint16_t *>(row)[ch + i] = (uint16_t)pack_bf16x2(x[i], 0.f);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) reinterpret_cast<float *>(row)[ch + i] = x[i];
        }
    } else if (r.bf16) {
        *reinterpret_cast<u32x4 *>(row + ch * 2) = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
    } else {
        *reinterpret_cast<f32x4 *>(row + ch * 4) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4 *>(row + ch * 4 + 16) = f32x4{x[4], x[5], x[6], x[7]};
    }
}

// Rows of sequence b in a call of n; false: rejected.
__device__ __forceinline__ bool kv8_rows(const int32_t *lens, const int32_t *counts, int b, int n, int max_seq, int &len, int &count)
{
    len = lens ? lens[b] : 0;
    count = counts ? counts[b] : n;
    return len >= 0 && count >= 0 && count <= n && (int64_t)len + count <= max_seq;
}

// The draft tree of one sequence, in lanes 0 .. n-1 of a wave (n <= 32), each with its row's parent: every lane's word of visible new rows,
// itself and its ancestors.  Five rounds of doubling: a lane adds what the row sees that it points to and points to where that one pointed.  bad: a parent
// outside [0, lane), taken as lane - 1.
__device__ __forceinline__ uint32_t kv8_tree_word(int up, int n, int lane, bool &bad)
{
    bad = lane > 0 && lane < n && (up < 0 || up >= lane);
    if (bad) up = lane - 1;
    if (lane == 0 || lane >= n) up = 0;
    uint32_t word = 1u << (lane & 31);
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        word |= (uint32_t)__shfl((int)word, up);
        up = __shfl(up, up);
    }
    return word;
}
__device__ __forceinline__ uint32_t kv8_chain_word(int j) { return (2u << j) - 1u; }

struct Rope8 {
    const double *turns;
    int r, neighbours;
    float magnitude;
    Div by_half;   // quotients by r / 2
};
// cos and sin of 2 pi frac(position * turns), times the magnitude.  The product in 64 bits: at position 10^6 a 32-bit angle is off by 0.06.  Its quarter
// turn and the rest r, |r| <= 1/8, are told apart in 64 bits too, so that what is rounded to 32 is small; then with z = r^2, sin = r (2 pi + z P(z)) and
// cos = 1 + z Q(z), the polynomials through (sin(2 pi r) / r - 2 pi) / z and (cos(2 pi r) - 1) / z at the Chebyshev nodes of 0 .. 1/64.  Both are off by
// at most 2.5 * 2^-25, and by 0.65 * 2^-25 in the root mean square, where rounding alone makes 0.58.
__device__ __forceinline__ void rope_cos_sin(const Rope8 &rp, int position, double turns, float &c, float &s)
{
    const double t = __builtin_amdgcn_fract((double)position * turns), quarters = __builtin_rint(4.0 * t);
    const float r = (float)__builtin_fma(-0.25, quarters, t), z = r * r;
    const int n = (int)quarters;
    const float two_pi = 0x1.921fb6p+2f, rest = -0x1.777a5cp-23f;   // 2 pi = two_pi + rest
    const float p = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(0x1.4cb74ap+5f, z, -0x1.32ce1ep+6f), z, 0x1.466bc2p+6f), z, -0x1.4abbcep+5f), z, rest);
    const float q = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(0x1.db6466p+5f, z, -0x1.55cb98p+6f), z, 0x1.03c1eap+6f), z, -0x1.3bd3ccp+4f);
    const float sine = __builtin_fmaf(r, two_pi, r * p), cosine = __builtin_fmaf(z, q, 1.f);
    c = bits_f32(f32_bits(n & 1 ? sine : cosine) ^ ((uint32_t)(n + 1) & 2u) << 30) * rp.magnitude;
    s = bits_f32(f32_bits(n & 1 ? cosine : sine) ^ ((uint32_t)n & 2u) << 30) * rp.magnitude;
}

// A rotation shared out over workgroups: `rows` rows and `per` heads each, a unit at a time.
constexpr int ROPE_TABLE = 512, ROPE_ROWS = 4;   // pairs of a workgroup's rows in LDS (sssd_rope_config allows 512 a row); rows of a workgroup
struct RopeWork {
    int d, heads, per, unit;      // unit: 8 channels, 2 or 1
    uint32_t n, units, rows, total;   // units of a row and head; rows of the whole call
    Div by_units;
};
RopeWork rope_work(int B, int n, int d, int heads, int r, bool neighbours, int threads, int each);

struct Kv8StoreArgs {
    Kv8Geom g;
    uint8_t *codes;      // the layer (commit: layer 0)
    float2 *scales;
    size_t layer_bytes;
    int first, B, n, blocks;   // blocks: of a sequence that a call may touch at most
    int per, chunks;           // append, read: kv heads of a workgroup, workgroups for all of them
    Rows8 k, v, q, q_out;      // q.p null: no queries
    const int32_t *lens, *counts, *parents;
    Rope8 rope;                // turns null: none
    RopeWork work;             // of the queries
    int32_t *status;
};
hipError_t launch_rope(const Rows8 &x, const Rows8 &out, const int32_t *positions, const Rope8 &rope, const RopeWork &w, hipStream_t s);
hipError_t launch_kv8_append(Kv8StoreArgs a, int fmt, int d, hipStream_t s);
hipError_t launch_kv8_read(Kv8StoreArgs a, int fmt, int d, hipStream_t s);
hipError_t launch_kv8_commit(const Kv8StoreArgs &a, int fmt, int d, int layers, const int32_t *accepted, const int32_t *path, int32_t *lens, hipStream_t s);

// How the attention's work is cut: `share` segments of a sequence at most, `passes` over the cache for the 16-row tiles of queries.
struct Kv8Plan {
    int passes, share;
    int in_die;   // a (sequence, kv head)'s workgroups run on one die, where its segments can be merged inside the launch
};
constexpr int KV8_GROUPS = 512, KV8_MAX_TILES = 3;   // workgroups of a launch whose segments are merged, row tiles of a pass
struct Kv8AttnArgs {
    Kv8Geom g;
    const uint8_t *codes;    // the layer
    const float2 *scales;
    int B, n, gq;            // gq: query heads of a kv head
    Rows8 q, out;
    const int32_t *lens, *counts, *parents;
    int window, sinks;       // window 0: all positions
    float *part_o;           // [sequence][kv head][segment][rows_pad][d] sums
    f32x4 *part_ml;          // ... reference of the exponents (log2), sum of probabilities, biased exponent of the sums' unit
    int rows_pad;            // rows of a (sequence, kv head) in whole tiles
    Kv8Plan plan;
    Hand hand;               // words for segments merged inside the launch, or none
    int32_t *status;
};
struct Kv8SharedArgs : Kv8AttnArgs {   // of a batch whose sequences share prefixes in groups
    int groups;
    const int32_t *starts, *shared;
    int tiles;             // workgroups' row tiles of all groups at most
    int wave_rows;         // waves of a workgroup on row tiles of their own: 4, or 1 with the others on other segments
    int prefix_share;      // workgroups on a prefix at most
    int prefix_groups;     // workgroups of a launch that are on prefixes
    int prefix_segments;   // segments of a prefix at most: prefix_share * 4 / wave_rows
    int prefix_once;       // as many while compute units have one workgroup each; 0: they have more
    float prefix_cost;     // us that a segment more takes, blocks apart
    int rows_all;          // B * n * gq
};
Kv8Plan kv8_plan(int B, int n, int gq, int nkv, int blocks, bool f32);   // blocks: of a sequence at most
struct Kv8SharedPlan {
    int rt, wave_rows, tiles, share, segments, once;   // row tiles of a wave; the others as in Kv8SharedArgs
    float cost;
    double us;             // what a call takes, about, for prefixes as long as they can be
};
Kv8SharedPlan kv8_shared_plan(int B, int n, int gq, int nkv, int blocks, int groups, bool f32);   // blocks: of a sequence at most
size_t kv8_shared_ws(int B, int n, int gq, int nkv, int d);
size_t kv8_attention_ws(int d);   // bytes behind the workspace that any call's partial results take
hipError_t launch_kv8_apart(Kv8SharedArgs a, int fmt, int d, void *ws, hipStream_t s);
hipError_t launch_kv8_attention(Kv8AttnArgs a, int fmt, int d, void *ws, hipStream_t s);
