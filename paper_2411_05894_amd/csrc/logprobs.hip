// Log-probabilities of given tokens, their ranks, the entropy and the most probable tokens of rows of logits.
//
// Mathematics.  With x_i = (z_i - M) / T for the largest logit M, S = 1 + s, s the sum of exp(x_i) over all tokens but one of the largest, and t = sum exp(x_i) x_i:
//   log p_i = x_i - log(1 + s),   H = log(1 + s) - t / (1 + s)
// so that what is nearly certain keeps its digits: log p of the likeliest token is -log1p(s), however small s is.
//
// Split.  A row is cut into tiles that a workgroup holds in registers: every logit is loaded once, all loads of a thread at once, and the maximum is known before
// anything is summed.  A tile leaves (M, s, t), how many of its logits come before each given token, and its own most probable tokens in order; a wave per row joins
// the tiles.  Sums are taken over tiles in a fixed order.
//
// The most probable tokens of a tile: the n-th largest of the threads' own largest logits, or less (the smallest over waves of the ceil(n / waves)-th largest of a wave's),
// bounds them from below: what is at or above it is listed, and its place counted against the rest of the list.  Where the list would overflow (equal logits), they are
// taken out one by one.
#include "../../include/sssd_ops.h"
#include "common.h"

#include <algorithm>

namespace {

constexpr int LT = 512, LWAVES = LT / 64;   // threads of a tile's workgroup
constexpr int LIST = 1024;                  // tokens listed at most
constexpr int MOST_TOKENS = SSSD_LOGPROBS_MAX_TOKENS, MOST_TOP = SSSD_LOGPROBS_MAX_TOP;

// Order of tokens: larger logit first, then the lower id; what is no number counts as -infinity.  As one word, larger first: keys of logits ascend with
// them (-0 is 0), ids are inverted.
__device__ __forceinline__ uint32_t logit_key(float z)
{
    const uint32_t u = f32_bits(z + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) { return bits_f32(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
__device__ __forceinline__ float ordered(float z) { return fmaxf(z, -INFINITY); }
__device__ __forceinline__ uint64_t token_key(float z, int id) { return (uint64_t)logit_key(ordered(z)) << 32 | (uint32_t)~id; }

struct LogArgs {
    const char *logits;
    int64_t stride;      // elements
    int rows, vocab, tile, tiles, n_tokens, n_top;
    float k, inv_t;      // log2(e) / T, 1 / T
    const int32_t *tokens;
    float *logprobs, *entropy, *top_logprobs;
    int32_t *ranks, *top_ids;
    f32x4 *stats;        // [row][tile] M, s, t, -
    int32_t *before;     // [row][tile][token]
    uint64_t *best;      // [row][tile][top]
};

// Sum, largest of a workgroup; red: LWAVES words.
__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) x = fmaxf(x, __shfl_xor(x, i));
    return x;
}
__device__ __forceinline__ float wave_add(float x)
{
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) x += __shfl_xor(x, i);
    return x;
}
__device__ __forceinline__ uint64_t wave_max64(uint64_t x)
{
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) {
        const uint64_t y = (uint64_t)__shfl_xor((unsigned long long)x, i);
        x = y > x ? y : x;
    }
    return x;
}

// V: 16-byte loads of a thread; a tile is at most LT * V * 16 bytes of logits.  grid: tiles of a row next to each other
template <int V, bool BF16> __global__ __launch_bounds__(LT) void logprob_tile_kernel(LogArgs a)
{
    constexpr int PER = BF16 ? 8 : 4, SIZE = BF16 ? 2 : 4, N = V * PER + 1;   // logits of a load; of a thread: one of the ends besides
    __shared__ float red_s[LWAVES], sum_s[LWAVES], turn_s[LWAVES];
    __shared__ uint32_t bound_s[LWAVES], listed_s;
    __shared__ uint64_t list_s[LIST];
    __shared__ int count_s[LWAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t row_of = blockIdx.x / (uint32_t)a.tiles;
    const int tile = (int)(blockIdx.x - row_of * a.tiles);
    const int64_t row = row_of;
    const int lo = tile * a.tile, hi = min(a.vocab, lo + a.tile);
    const char *base = a.logits + row * a.stride * SIZE;
    // ids lo .. lo+head-1 and those behind the last whole 16 bytes: one a thread
    const int head = min((int)((16 - (uintptr_t)(base + (int64_t)lo * SIZE) % 16) % 16 / SIZE), hi - lo);
    const int vecs = (hi - lo - head) / PER, rest = lo + head + vecs * PER, ends = head + hi - rest;
    const u32x4 *at = reinterpret_cast<const u32x4 *>(base + (int64_t)(lo + head) * SIZE);
    u32x4 raw[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i * LT + (int)threadIdx.x < vecs) raw[i] = at[i * LT + threadIdx.x];
    auto load = [&](int id) { return BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(base)[id]) : reinterpret_cast<const float *>(base)[id]; };
    const int end_id = (int)threadIdx.x < head ? lo + (int)threadIdx.x : rest + (int)threadIdx.x - head;
    float z[N];
    z[N - 1] = (int)threadIdx.x < ends ? load(end_id) : -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const bool on = i * LT + (int)threadIdx.x < vecs;
#pragma unroll
        for (int e = 0; e < PER; ++e)
            z[i * PER + e] = !on ? -INFINITY : BF16 ? bits_f32(e & 1 ? raw[i][e / 2] & 0xFFFF0000u : raw[i][e / 2] << 16) : bits_f32(raw[i][e % 4]);
    }
    auto id_of = [&](int i) { return i == N - 1 ? end_id : lo + head + ((i / PER) * LT + (int)threadIdx.x) * PER + i % PER; };
    auto live = [&](int i) { return i == N - 1 ? (int)threadIdx.x < ends : (i / PER) * LT + (int)threadIdx.x < vecs; };

    float top = -INFINITY;   // not counting what is no number
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, z[i]);
    const float wave_top = wave_max(top);
    if (lane == 0) red_s[wave] = wave_top;
    if (threadIdx.x == 0) listed_s = 0;
    __syncthreads();
    float most = red_s[0];
#pragma unroll
    for (int w = 1; w < LWAVES; ++w) most = fmaxf(most, red_s[w]);

    // The thread that holds the first of the largest leaves it out of its sum.
    uint64_t holders = __ballot(top == most);
    int first_wave = 0;
#pragma unroll
    for (int w = LWAVES - 1; w >= 0; --w) first_wave = red_s[w] == most ? w : first_wave;
    bool skip = wave == first_wave && lane == __ffsll((long long)holders) - 1;
    const float ref = most == -INFINITY ? 0.f : most;   // a tile of nothing: sums of 0
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = (z[i] - ref) * a.k, e = __builtin_amdgcn_exp2f(x);
        t = __builtin_fmaf(e, fmaxf(x, -16384.f), t);   // 0 * -infinity is 0 here
        const bool out = skip && z[i] == most;
        s += out ? 0.f : e;
        skip = skip && !out;
    }
    s = wave_add(s);
    t = wave_add(t);
    if (lane == 0) {
        sum_s[wave] = s;
        turn_s[wave] = t;
    }
    const int64_t slot = row * a.tiles + tile;
    // ranks
    for (int j = 0; j < a.n_tokens; ++j) {
        const int token = a.tokens[row * a.n_tokens + j];
        int n = 0;
        if (token >= 0 && token < a.vocab) {
            const float v = ordered(load(token));
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float o = ordered(z[i]);
                n += live(i) && (o > v || (o == v && id_of(i) < token)) ? 1 : 0;
            }
        }
#pragma unroll
        for (int i = 32; i > 0; i >>= 1) n += __shfl_xor(n, i);
        __syncthreads();   // the counts before have been read
        if (lane == 0) count_s[wave] = n;
        __syncthreads();
        if (threadIdx.x == 0) {
            n = 0;
#pragma unroll
            for (int w = 0; w < LWAVES; ++w) n += count_s[w];
            a.before[slot * a.n_tokens + j] = n;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        s = t = 0.f;
#pragma unroll
        for (int w = 0; w < LWAVES; ++w) {
            s += sum_s[w];
            t += turn_s[w];
        }
        a.stats[slot] = f32x4{most, s, t, 0.f};
    }
    const int n_top = min(a.n_top, hi - lo);
    if (a.n_top == 0) return;
    uint64_t *best = a.best + slot * a.n_top;
    if ((int)threadIdx.x >= n_top && (int)threadIdx.x < a.n_top) best[threadIdx.x] = 0;   // behind every token's

    // a bound: the nth-largest of a wave's lanes, the smallest of the waves all of whose lanes have logits
    const int whole = max(min(vecs >> 6, LWAVES), 1), nth = (n_top + whole - 1) / whole;
    {
        float left = top, bound = top;
        for (int i = 0; i < nth; ++i) {
            bound = wave_max(left);
            const uint64_t has = __ballot(left == bound);
            if (lane == __ffsll((long long)has) - 1) left = -INFINITY;
        }
        if (lane == 0) bound_s[wave] = logit_key(bound);
    }
    __syncthreads();
    uint32_t bound_k = bound_s[0];
#pragma unroll
    for (int w = 1; w < LWAVES; ++w) bound_k = w < whole ? min(bound_k, bound_s[w]) : bound_k;
    const float bound = key_logit(bound_k);
    if (top >= bound)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float o = ordered(z[i]);
            if (live(i) && o >= bound) {
                const uint32_t k = atomicAdd(&listed_s, 1u);
                if (k < LIST) list_s[k] = token_key(o, id_of(i));
            }
        }
    __syncthreads();
    const int listed = (int)listed_s;
    if (listed <= LIST) {
        for (int i = threadIdx.x; i < listed; i += LT) {
            const uint64_t mine = list_s[i];
            int place = 0;
            for (int j = 0; j < listed; ++j) place += list_s[j] > mine;
            if (place < n_top) best[place] = mine;
        }
        return;
    }
    uint64_t below = ~0ull;   // taken so far
    for (int k = 0; k < n_top; ++k) {
        uint64_t mine = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t key = live(i) ? token_key(z[i], id_of(i)) : 0;
            mine = key < below && key > mine ? key : mine;
        }
        mine = wave_max64(mine);
        __syncthreads();
        if (lane == 0) list_s[wave] = mine;
        __syncthreads();
        below = list_s[0];
#pragma unroll
        for (int w = 1; w < LWAVES; ++w) below = list_s[w] > below ? list_s[w] : below;
        if (threadIdx.x == 0) best[k] = below;
    }
}

// (M, s, t) of two parts; k: log2(e) / T.  t is in units of log2.
struct Part {
    float m, s, t;
};
__device__ __forceinline__ Part join(const Part &a, const Part &b, float k)
{
    const bool first = a.m >= b.m;
    const Part &x = first ? a : b, &y = first ? b : a;
    if (y.m == -INFINITY) return Part{x.m, x.s + y.s, x.t + y.t};   // nothing, or what is no number
    const float d = (y.m - x.m) * k, w = __builtin_amdgcn_exp2f(d), n = 1.f + y.s;
    return Part{x.m, __builtin_fmaf(w, n, x.s), x.t + w * __builtin_fmaf(n, fmaxf(d, -16384.f), y.t)};
}

constexpr int JT = 256, JLIST = 1024;   // threads of a row's workgroup, tokens listed at most

template <bool BF16> __global__ __launch_bounds__(JT) void logprob_join_kernel(LogArgs a)
{
    __shared__ float all_s[2];   // M, log(1 + s)
    __shared__ uint64_t list_s[JLIST], bound_s;
    __shared__ uint32_t listed_s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x, slot = row * a.tiles;
    const char *base = a.logits + row * a.stride * (BF16 ? 2 : 4);
    auto load = [&](int id) { return BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(base)[id]) : reinterpret_cast<const float *>(base)[id]; };
    const uint64_t *best = a.best + slot * a.n_top;
    if (wave == 0) {
        Part p{-INFINITY, 0.f, 0.f};
        for (int i = lane; i < a.tiles; i += 64) {
            const f32x4 x = a.stats[slot + i];
            p = join(p, Part{x[0], x[1], x[2]}, a.k);
        }
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {   // both of a pair in the same order
            const Part o{__shfl_xor(p.m, i), __shfl_xor(p.s, i), __shfl_xor(p.t, i)};
            p = lane & i ? join(o, p, a.k) : join(p, o, a.k);
        }
        const bool none = !(fabsf(p.m) < INFINITY);   // no finite logit, or an infinite one: no distribution
        const float log_s = none ? NAN : log1pf(p.s);
        if (lane == 0) {
            all_s[0] = p.m;
            all_s[1] = log_s;
            if (a.entropy) a.entropy[row] = log_s - p.t * 0.69314718056f / (1.f + p.s);
        }
    } else if (wave == 1 && a.n_top > 0) {
        // The n_top-th largest of the row is no smaller than the last of any tile's list, nor than the smallest of the tiles' nth ones.
        const int nth = (a.n_top + a.tiles - 1) / a.tiles;
        uint64_t last = 0, least = 0;   // least: inverted
        for (int i = lane; i < a.tiles; i += 64) {
            const uint64_t x = best[(int64_t)i * a.n_top + a.n_top - 1], y = ~best[(int64_t)i * a.n_top + nth - 1];
            last = x > last ? x : last;
            least = y > least ? y : least;
        }
        last = wave_max64(last);
        least = ~wave_max64(least);
        if (lane == 0) {
            bound_s = last > least ? last : least;
            listed_s = 0;
        }
    }
    __syncthreads();
    const float m = all_s[0], log_s = all_s[1];
    auto logprob = [&](float z) { return (z - m) * a.inv_t - log_s; };
    for (int j = wave; j < a.n_tokens; j += JT / 64) {
        const int token = a.tokens[row * a.n_tokens + j];
        const bool there = token >= 0 && token < a.vocab;
        int n = 0;
        for (int i = lane; i < a.tiles; i += 64) n += a.before[(slot + i) * a.n_tokens + j];
#pragma unroll
        for (int i = 32; i > 0; i >>= 1) n += __shfl_xor(n, i);
        if (lane == 0) {
            a.logprobs[row * a.n_tokens + j] = there ? logprob(load(token)) : -INFINITY;
            if (a.ranks) a.ranks[row * a.n_tokens + j] = there ? n : -1;
        }
    }
    if (a.n_top == 0) return;
    auto put = [&](int k, uint64_t key) {
        const int id = (int)~(uint32_t)key;
        a.top_ids[row * a.n_top + k] = id;
        a.top_logprobs[row * a.n_top + k] = logprob(load(id));
    };
    const int64_t all = (int64_t)a.tiles * a.n_top;
    const uint64_t bound = bound_s;
    for (int64_t i = threadIdx.x; i < all; i += JT) {
        const uint64_t key = best[i];
        if (key && key >= bound) {
            const uint32_t k = atomicAdd(&listed_s, 1u);
            if (k < JLIST) list_s[k] = key;
        }
    }
    __syncthreads();
    const int listed = (int)listed_s;
    if (listed <= JLIST) {
        for (int i = threadIdx.x; i < listed; i += JT) {
            const uint64_t mine = list_s[i];
            int place = 0;
            for (int j = 0; j < listed; ++j) place += list_s[j] > mine;
            if (place < a.n_top) put(place, mine);
        }
        return;
    }
    uint64_t below = ~0ull;   // one by one, those taken so far left out
    for (int k = 0; k < a.n_top; ++k) {
        uint64_t mine = 0;
        for (int64_t i = threadIdx.x; i < all; i += JT) {
            const uint64_t key = best[i];
            mine = key < below && key > mine ? key : mine;
        }
        mine = wave_max64(mine);
        __syncthreads();
        if (lane == 0) list_s[wave] = mine;
        __syncthreads();
        below = list_s[0];
#pragma unroll
        for (int w = 1; w < JT / 64; ++w) below = list_s[w] > below ? list_s[w] : below;
        if (threadIdx.x == 0) put(k, below);
    }
}

// Tiles: small while there are few rows, so that they spread over the chip.
struct LogPlan {
    int v, tile, tiles;
};
LogPlan log_plan(int64_t rows, int vocab, bool bf16)
{
    LogPlan p;
    const int per = bf16 ? 8 : 4;
    p.v = 8;
    while (p.v > 2 && rows * (((int64_t)vocab + LT * p.v * per - 1) / (LT * p.v * per)) < 512) p.v /= 2;
    const int64_t most = (int64_t)LT * p.v * per;
    p.tiles = (int)((vocab + most - 1) / most);
    p.tile = (int)((((int64_t)vocab + p.tiles - 1) / p.tiles + per - 1) / per * per);
    p.tiles = (vocab + p.tile - 1) / p.tile;
    return p;
}
struct LogScratch {
    size_t before, best, bytes;
};
LogScratch log_scratch(int64_t rows, const LogPlan &p, int n_tokens, int n_top)
{
    LogScratch s;
    const size_t slots = (size_t)rows * p.tiles;
    s.best = slots * sizeof(f32x4);
    s.before = s.best + slots * n_top * sizeof(uint64_t);
    s.bytes = (s.before + slots * n_tokens * sizeof(int32_t) + 255) / 256 * 256;
    return s;
}

}  // namespace

extern "C" {

size_t sssd_op_logprobs_scratch_bytes(int32_t type, int32_t rows, int32_t vocab, int32_t n_tokens, int32_t n_top)
{
    if ((type != SSSD_F32 && type != SSSD_BF16) || rows <= 0 || vocab <= 0 || n_tokens < 0 || n_tokens > MOST_TOKENS || n_top < 0 || n_top > MOST_TOP || n_top > vocab) return 0;
    return log_scratch(rows, log_plan(rows, vocab, type == SSSD_BF16), n_tokens, n_top).bytes;
}

int sssd_op_logprobs(const void *logits, int32_t type, int32_t rows, int32_t vocab, int64_t row_stride, float temperature, const int32_t *tokens,
                     int32_t n_tokens, float *logprobs, int32_t *ranks, float *entropy, int32_t n_top, int32_t *top_ids, float *top_logprobs, void *scratch,
                     size_t scratch_bytes, void *stream)
{
    if (!logits || (type != SSSD_F32 && type != SSSD_BF16) || rows <= 0 || vocab <= 0 || n_tokens < 0 || n_top < 0 || n_top > vocab) return SSSD_EINVAL;
    if (n_tokens > MOST_TOKENS || n_top > MOST_TOP) return SSSD_ECAPACITY;
    if ((n_tokens > 0 && (!tokens || !logprobs)) || (n_top > 0 && (!top_ids || !top_logprobs))) return SSSD_EINVAL;
    const bool bf16 = type == SSSD_BF16;
    if ((uintptr_t)logits % (bf16 ? 2 : 4) || (rows > 1 && row_stride < 0)) return SSSD_EINVAL;
    const float k = 1.4426950408889634f / temperature;
    if (!(temperature > 0.f) || !(k > 0.f) || !(k <= 3.0e38f)) return SSSD_EINVAL;
    const LogPlan p = log_plan(rows, vocab, bf16);
    const LogScratch z = log_scratch(rows, p, n_tokens, n_top);
    if (!scratch || (uintptr_t)scratch % 16) return SSSD_EINVAL;
    if (scratch_bytes < z.bytes || (int64_t)rows * p.tiles > UINT32_MAX / LT) return SSSD_ECAPACITY;
    LogArgs a{};
    a.logits = (const char *)logits;
    a.stride = rows > 1 ? row_stride : 0;
    a.rows = rows; a.vocab = vocab; a.tile = p.tile; a.tiles = p.tiles;
    a.n_tokens = n_tokens; a.n_top = n_top;
    a.k = k;
    a.inv_t = 1.f / temperature;
    a.tokens = tokens; a.logprobs = logprobs; a.ranks = ranks; a.entropy = entropy; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
    a.stats = (f32x4 *)scratch;
    a.best = (uint64_t *)((char *)scratch + z.best);
    a.before = (int32_t *)((char *)scratch + z.before);
    hipStream_t s = (hipStream_t)stream;
    const dim3 grid((uint32_t)rows * p.tiles);
#define TILE(V)                                                                                          \
    do {                                                                                                 \
        if (bf16) hipLaunchKernelGGL((logprob_tile_kernel<V, true>), grid, dim3(LT), 0, s, a);           \
        else hipLaunchKernelGGL((logprob_tile_kernel<V, false>), grid, dim3(LT), 0, s, a);               \
    } while (0)
    switch (p.v) {
    case 2: TILE(2); break;
    case 4: TILE(4); break;
    default: TILE(8); break;
    }
#undef TILE
    if (hipGetLastError() != hipSuccess) return SSSD_EHIP;
    if (bf16) hipLaunchKernelGGL(logprob_join_kernel<true>, dim3(rows), dim3(JT), 0, s, a);
    else hipLaunchKernelGGL(logprob_join_kernel<false>, dim3(rows), dim3(JT), 0, s, a);
    return hipGetLastError() == hipSuccess ? SSSD_OK : SSSD_EHIP;
}

}  // extern "C"
