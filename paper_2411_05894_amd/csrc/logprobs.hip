// Log-probabilities of given tokens, their ranks, the entropy and the most probable tokens of rows of logits.
//
// Mathematics.  With x_i = (z_i - M) / T for the largest logit M, S = 1 + s, s the sum of exp(x_i) over all tokens but one of the largest, and t = sum exp(x_i) x_i:
//   log p_i = x_i - log(1 + s),   H = log(1 + s) - t / (1 + s)
// so that what is nearly certain keeps its digits: log p of the likeliest token is -log1p(s), however small s is.
//
// Split.  A workgroup goes over a row, or a part of one where there are few rows, a chunk of 1024 16-byte loads at a time, the next one under way; its waves know nothing of each other until
// the end.  A wave keeps the largest logit M so far and how many there were of it, per lane s and t of the others relative to a logit r near M (so that hardly any chunk
// changes it), how many come before each given token, and a list of its most probable tokens: what is above the last of n in a list that was full, at first above the n-th largest of its lanes'
// largest logits.  Parts leave all that in memory, and a second launch joins them.  The order of sums is fixed.
//
// What bounds it: thirteen instructions a logit, an exponential among them, and in their shadow the reading.  us, four in a row in a graph: 1501 rows of 128256, one token with its rank and one alternative,
// bf16 96 (4.0 TB/s; 90 where inputs change), float32 164 (4.7 TB/s; a kernel that only reads takes 54 and 108); without the alternative 89 and 152, 20 alternatives 137 and 179.  9 rows: 8.6 and 6.3 for the
// joining, both round trips behind one another.
#include "../../include/sssd_ops.h"
#include "common.h"

#include <algorithm>
#include <type_traits>

namespace {

constexpr int LT = 256, LWAVES = LT / 64;   // threads of a workgroup
constexpr int LIST = 192;                   // a wave's list of tokens: two rounds of its lanes behind a list that has been cut
constexpr int MOST_TOKENS = SSSD_LOGPROBS_MAX_TOKENS, MOST_TOP = SSSD_LOGPROBS_MAX_TOP;
static_assert(LIST >= MOST_TOP + 64);
constexpr int MOST_VOCAB = 1 << 30;         // places behind the last token are numbers, too
constexpr float FAR = 4.f;                  // octaves of probability that M may be away from r
constexpr float MOST_OFF = 0x1p20f;         // r k beyond that is rounded by more than a sixteenth of an octave

// Order of tokens: larger logit first, then the lower id; what is no number counts as -infinity.  As one word, larger first: keys of logits ascend with
// them (-0 is 0), ids are inverted.
__device__ __forceinline__ uint32_t logit_key(float z)
{
    const uint32_t u = f32_bits(z + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) { return bits_f32(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
__device__ __forceinline__ float next_below(float z)   // a finite or infinite one above the lowest; the same for both zeros
{
    const int u = (int)f32_bits(z + 0.f);
    return bits_f32((uint32_t)(u == 0 ? (int)0x80000001u : u > 0 ? u - 1 : u + 1));
}
__device__ __forceinline__ float ordered(float z) { return fmaxf(z, -INFINITY); }
__device__ __forceinline__ uint64_t token_key(float z, int id) { return (uint64_t)logit_key(ordered(z)) << 32 | (uint32_t)~id; }

struct LogArgs {
    const char *logits;
    int64_t stride;      // elements
    int rows, vocab, part, parts, n_tokens, n_top;   // part: logits of a part
    float k, inv_t;      // log2(e) / T, 1 / T
    const int32_t *tokens;
    float *logprobs, *entropy, *top_logprobs;
    int32_t *ranks, *top_ids;
    f32x4 *stats;        // [row][part] M, s, t, -
    int32_t *before;     // [row][part][token]
    uint64_t *best;      // [row][part][top]
};

// Over a wave, the same in every lane: neighbours, then eights, sixteens and halves of the wave.
template <typename F> __device__ __forceinline__ float wave_all(float x, F f)
{
    auto dpp = [&](auto ctrl) { return bits_f32((uint32_t)__builtin_amdgcn_mov_dpp((int)f32_bits(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    x = f(x, dpp(std::integral_constant<int, 0xB1>()));    // lane ^ 1
    x = f(x, dpp(std::integral_constant<int, 0x4E>()));    // lane ^ 2
    x = f(x, dpp(std::integral_constant<int, 0x141>()));   // mirrored within eight
    x = f(x, dpp(std::integral_constant<int, 0x140>()));   // ... within sixteen
    auto h = __builtin_amdgcn_permlane16_swap(f32_bits(x), f32_bits(x), false, false);
    x = f(bits_f32(h[0]), bits_f32(h[1]));
    h = __builtin_amdgcn_permlane32_swap(f32_bits(x), f32_bits(x), false, false);
    return f(bits_f32(h[0]), bits_f32(h[1]));
}
__device__ __forceinline__ float wave_max(float x)
{
    return wave_all(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_add(float x)
{
    return wave_all(x, [](float a, float b) { return a + b; });
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

// How many lanes.
__device__ __forceinline__ int lanes_of(bool x) { return (int)__popcll(__ballot(x)); }

// What lanes of a wave stored in LDS is there for the others.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// (M, s, t): the largest logit, and the sums of the others relative to it, t in units of log2.
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

struct Row {   // what comes out of one
    const LogArgs &a;
    int64_t row;
    float m, log_s;
    __device__ __forceinline__ Row(const LogArgs &a, int64_t row, const Part &p, bool writes) : a(a), row(row), m(p.m)
    {
        const bool none = !(fabsf(p.m) < INFINITY);   // no finite logit, or an infinite one: no distribution
        log_s = none ? NAN : log1pf(p.s);
        if (writes && a.entropy) a.entropy[row] = log_s - p.t * 0.69314718056f / (1.f + p.s);
    }
    // the difference may be beyond float32's range, the quotient not
    __device__ __forceinline__ float logprob(float z) const { return __builtin_fmaf(z, 0.5f, -0.5f * m) * (2.f * a.inv_t) - log_s; }
    __device__ __forceinline__ void token(int j, bool there, float z, int before) const
    {
        a.logprobs[row * a.n_tokens + j] = there ? logprob(z) : -INFINITY;
        if (a.ranks) a.ranks[row * a.n_tokens + j] = there ? before : -1;
    }
    __device__ __forceinline__ void top(int k, uint64_t key) const
    {
        a.top_ids[row * a.n_top + k] = (int)~(uint32_t)key;
        a.top_logprobs[row * a.n_top + k] = logprob(key_logit((uint32_t)(key >> 32)));
    }
};

// WHOLE: a workgroup has a whole row.  grid: parts of a row next to each other
template <bool BF16, bool WHOLE> __global__ __launch_bounds__(LT) __attribute__((amdgpu_waves_per_eu(6))) void logprob_kernel(LogArgs a)
{
    constexpr int PER = BF16 ? 8 : 4, SIZE = BF16 ? 2 : 4, V = (WHOLE ? 16 : 8) / PER;   // logits of a 16-byte load, loads of a thread and chunk
    __shared__ float token_z_s[MOST_TOKENS];
    __shared__ int token_s[MOST_TOKENS], before_s[LWAVES][MOST_TOKENS], listed_s[LWAVES];
    __shared__ Part part_s[LWAVES];
    __shared__ uint64_t list_s[LWAVES][LIST];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t row_of = WHOLE ? blockIdx.x : blockIdx.x / (uint32_t)a.parts;
    const int part = WHOLE ? 0 : (int)(blockIdx.x - row_of * a.parts);
    const int64_t row = row_of;
    const int lo = part * a.part, hi = min(a.vocab, lo + a.part);
    const char *base = a.logits + row * a.stride * SIZE;
    auto load = [&](int id) { return BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(base)[id]) : reinterpret_cast<const float *>(base)[id]; };
    // ids lo .. lo+head-1 and those behind the last whole 16 bytes: one a thread
    const int head = min((int)((16 - (uintptr_t)(base + (int64_t)lo * SIZE) % 16) % 16 / SIZE), hi - lo);
    const int vecs = (hi - lo - head) / PER, rest = lo + head + vecs * PER, ends = head + hi - rest;
    const u32x4 *from = reinterpret_cast<const u32x4 *>(base + (int64_t)(lo + head) * SIZE);
    const uint32_t empty = BF16 ? 0xFF80FF80u : 0xFF800000u;   // -infinity
    u32x4 raw[V];
    auto request = [&](int first) {   // vectors from there on
        if (first + V * LT <= vecs) {
#pragma unroll
            for (int i = 0; i < V; ++i) raw[i] = from[first + i * LT + (int)threadIdx.x];
            return;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            raw[i] = u32x4{empty, empty, empty, empty};
            if (first + i * LT + (int)threadIdx.x < vecs) raw[i] = from[first + i * LT + (int)threadIdx.x];
        }
    };
    request(0);
    const int end_id = (int)threadIdx.x < head ? lo + (int)threadIdx.x : rest + (int)threadIdx.x - head;
    const float z_end = (int)threadIdx.x < ends ? load(end_id) : -INFINITY;
    if ((int)threadIdx.x < a.n_tokens) {
        const int token = a.tokens[row * a.n_tokens + threadIdx.x];
        const bool there = token >= 0 && token < a.vocab;
        token_s[threadIdx.x] = there ? token : -1;
        token_z_s[threadIdx.x] = there ? load(token) : INFINITY;
    }
    for (int j = lane; j < a.n_tokens; j += 64) before_s[wave][j] = 0;
    __syncthreads();
    const int n_tokens = a.ranks ? a.n_tokens : 0, n_top = min(a.n_top, hi - lo);
    const int token0 = n_tokens > 0 ? token_s[0] : 0;
    const float v0 = n_tokens > 0 ? ordered(token_z_s[0]) : INFINITY, below0 = next_below(v0);

    // most: the wave's largest so far; s, t: the lane's.  Exponents are (z - ref) k; for bf16, which instructions bound and not the reading, z k + off in one of them, with off = -ref k as
    // that is rounded, which moves r by as much for all.
    float most = -INFINITY, ref = 0.f, off = 0.f, s = 0.f, t = 0.f;
    auto near = [](float off) { return BF16 && fabsf(off) <= MOST_OFF; };
    auto exponent = [&](float z) { return near(off) ? __builtin_fmaf(z, a.k, off) : (z - ref) * a.k; };
    int equal = 0, before0 = 0, listed = 0;
    float least = -INFINITY;    // what is below it is not among the wave's n_top
    uint64_t least_key = 0;
    uint64_t *list = list_s[wave];

    // The list's n_top first, in order.
    auto cut = [&]() {
        wave_sync();
        uint64_t mine[LIST / 64];
        int place[LIST / 64];
        auto places = [&](auto rounds) {
            constexpr int E = decltype(rounds)::value;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                mine[e] = lane + 64 * e < listed ? list[lane + 64 * e] : 0;
                place[e] = 0;
            }
            for (int j = 0; j < listed; ++j) {
                const uint64_t other = list[j];
#pragma unroll
                for (int e = 0; e < E; ++e) place[e] += other > mine[e];
            }
            wave_sync();
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (mine[e] && place[e] < n_top) list[place[e]] = mine[e];
        };
        if (listed <= 64) places(std::integral_constant<int, 1>());
        else places(std::integral_constant<int, LIST / 64>());
        wave_sync();
        if (listed >= n_top) {
            listed = n_top;
            least_key = list[n_top - 1];
            least = key_logit((uint32_t)(least_key >> 32));
        }
    };
    // N logits a lane, z[i] of token first + i / PER * LT * PER + i % PER while that is below `end`: the others are -infinity.
    auto chunk = [&](auto n_of, const auto &z, int first, int end) {
        constexpr int N = decltype(n_of)::value, G = N == 1 ? 1 : PER;
        float top = z[0];
#pragma unroll
        for (int i = 1; i + 1 < N; i += 2) top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(z[i], z[i + 1]), top);
        if (N % 2 == 0) top = __builtin_elementwise_maximum(top, z[N - 1]);
        if (__any(top != top)) {   // not counting what is no number
            top = -INFINITY;
#pragma unroll
            for (int i = 0; i < N; ++i) top = fmaxf(top, z[i]);
        }
        const bool holds = __any(top >= most);   // hardly any chunk but the first
        const float here = holds ? bits_f32((uint32_t)__builtin_amdgcn_readfirstlane((int)f32_bits(wave_max(top)))) : most;
        if (here > most) {
            if (equal) {   // those that were the largest join the others
                const float x = exponent(most), e = __builtin_amdgcn_exp2f(x) * (float)equal;
                s += lane == 0 ? e : 0.f;
                t += lane == 0 ? e * x : 0.f;
            }
            const float next = -here * a.k, d = near(off) && near(next) ? next - off : (ref - here) * a.k;
            if (!equal || !(d >= -FAR)) {
                const float f = __builtin_amdgcn_exp2f(d);
                if (equal) {
                    t = __builtin_fmaf(fmaxf(d, -16384.f), s, t) * f;
                    s *= f;
                }
                ref = here;
                off = next;
            }
            most = here;
            equal = 0;
        }
        auto sums = [&](auto holding, auto counting, auto one) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float x = decltype(one)::value ? __builtin_fmaf(z[i], a.k, off) : (z[i] - ref) * a.k;
                float e = __builtin_amdgcn_exp2f(x);
                if (decltype(holding)::value) {
                    const bool is = z[i] == most;
                    e = is ? 0.f : e;
                    equal += lanes_of(is);
                }
                t = __builtin_fmaf(e, fmaxf(x, -16384.f), t);   // 0 * -infinity is 0 here
                s += e;
                if (decltype(counting)::value) before0 += lanes_of(z[i] > (first + i / PER * LT * PER + G <= token0 ? below0 : v0));
            }
        };
        const bool counts = v0 > -INFINITY && __any(top >= v0);
        auto both = [&](auto holding, auto one) {
            if (counts) sums(holding, std::true_type(), one);
            else sums(holding, std::false_type(), one);
        };
        if (BF16 && !near(off)) both(std::true_type(), std::false_type());
        else if (holds && most > -INFINITY) both(std::true_type(), std::integral_constant<bool, BF16>());
        else both(std::false_type(), std::integral_constant<bool, BF16>());
        // Tokens that come before the given ones: larger logits, and of equal ones those of lower ids -- what is larger than the next number below.
        auto id_of = [&](int i) { return first + i / PER * LT * PER + i % PER; };
        for (int j = 0; j < n_tokens; ++j) {
            const int token = token_s[j];
            const float v = ordered(token_z_s[j]);
            int n = 0;
            if (v == -INFINITY) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float o = ordered(z[i]);
                    n += lanes_of(id_of(i) < end && (o > v || id_of(i) < token));
                }
            } else if (__any(top >= v)) {
                if (j > 0) {
                    const float below = next_below(v);
#pragma unroll
                    for (int i = 0; i < N; ++i) n += lanes_of(z[i] > (first + i / PER * LT * PER + G <= token ? below : v));
                }
                const int off = token - first;
                bool has = false;   // the token is one of those of a load of the lane's, and not the first of them
#pragma unroll
                for (int l = 0; l < N / PER; ++l) has = has || (off > l * LT * PER && off < l * LT * PER + PER);
                if (__any(has))
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int within = off - i / PER * LT * PER;
                        n += lanes_of(within > i % PER && within < PER && z[i] == v);
                    }
            }
            if (n && lane == 0) before_s[wave][j] += n;
        }
        if (n_top == 0) return;
        if (least == -INFINITY) {   // the wave's first logits
            const int lanes = lanes_of(top > -INFINITY);
            if (lanes >= n_top) {
                float left = top;
                for (int i = 0; i < n_top; ++i) {
                    least = wave_max(left);
                    const uint64_t has = __ballot(left == least);
                    if (lane == __ffsll((long long)has) - 1) left = -INFINITY;
                }
            }
        }
        if (__any(top >= least))
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!__any(z[i] >= least || least == -INFINITY)) continue;
                const uint64_t key = token_key(z[i], id_of(i));
                bool take = ordered(z[i]) >= least && id_of(i) < end && key > least_key;
                uint64_t who = __ballot(take);
                if (listed + (int)__popcll(who) > LIST) {
                    cut();
                    take = take && key > least_key;
                    who = __ballot(take);
                }
                if (take) list[listed + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = key;
                listed += (int)__popcll(who);
            }
        if (listed > n_top + n_top / 4) cut();   // so that the next chunks have fewer to list
    };
    {
        // the ends are chunks of one logit a lane: before and behind the others
        const float z[1] = {z_end};
        if (ends > 0 && wave == 0) chunk(std::integral_constant<int, 1>(), z, end_id, (int)threadIdx.x < ends ? end_id + 1 : end_id);
    }
    for (int at = 0; at < vecs; at += V * LT) {
        float z[V * PER];
#pragma unroll
        for (int i = 0; i < V * PER; ++i) {
            const uint32_t w = BF16 ? raw[i / PER][i % PER / 2] : raw[i / PER][i % PER];
            z[i] = bits_f32(!BF16 ? w : i & 1 ? w & 0xFFFF0000u : w << 16);
        }
        request(at + V * LT);
        chunk(std::integral_constant<int, V * PER>(), z, lo + head + (at + (int)threadIdx.x) * PER, rest);
    }
    if (n_top > 0) cut();
    // relative to the wave's largest
    const float x = exponent(most), f = equal ? __builtin_amdgcn_exp2f(-x) : 1.f;
    t = wave_add(t);
    s = wave_add(s);
    if (equal) {
        t = __builtin_fmaf(-x, s, t) * f;
        s = __builtin_fmaf(s, f, (float)(equal - 1));
    }
    if (lane == 0) {
        part_s[wave] = Part{most, s, t};
        listed_s[wave] = listed;
        if (n_tokens > 0) before_s[wave][0] += before0;
    }
    __syncthreads();
    Part p = part_s[0];
#pragma unroll
    for (int w = 1; w < LWAVES; ++w) p = join(p, part_s[w], a.k);
    const int64_t slot = row * a.parts + part;
    const Row r(a, row, WHOLE ? p : Part{0.f, 0.f, 0.f}, WHOLE && threadIdx.x == 0);
    if (!WHOLE && threadIdx.x == 0) a.stats[slot] = f32x4{p.m, p.s, p.t, 0.f};
    if ((int)threadIdx.x < a.n_tokens) {
        int n = 0;
#pragma unroll
        for (int w = 0; w < LWAVES; ++w) n += before_s[w][threadIdx.x];
        if (WHOLE) r.token(threadIdx.x, token_s[threadIdx.x] >= 0, token_z_s[threadIdx.x], n);
        else a.before[slot * a.n_tokens + threadIdx.x] = n;
    }
    // a token's place among the waves' lists, which are in order
    uint64_t *best = a.best + slot * a.n_top;
    int all = 0;
#pragma unroll
    for (int w = 0; w < LWAVES; ++w) all += listed_s[w];
    for (int i = lane; i < listed; i += 64) {
        const uint64_t mine = list[i];
        int place = i;
#pragma unroll
        for (int w = 0; w < LWAVES; ++w)
            if (w != wave)
                for (int j = 0; j < listed_s[w] && place < n_top; ++j) place += list_s[w][j] > mine;
        if (place >= n_top) continue;
        if (WHOLE) r.top(place, mine);
        else best[place] = mine;
    }
    if (!WHOLE)
        for (int i = threadIdx.x; i < a.n_top; i += LT)
            if (i >= all) best[i] = 0;   // behind every token's
}

constexpr int JT = 256, JLIST = 1024;   // threads of a row's workgroup, tokens listed at most

// The parts of a row.
template <bool BF16> __global__ __launch_bounds__(JT) void logprob_join_kernel(LogArgs a)
{
    __shared__ Part part_s;
    __shared__ uint64_t list_s[JLIST], bound_s;
    __shared__ uint32_t listed_s;
    __shared__ int before_s[MOST_TOKENS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x, slot = row * a.parts;
    const char *base = a.logits + row * a.stride * (BF16 ? 2 : 4);
    auto load = [&](int id) { return BF16 ? bf16_to_f32(reinterpret_cast<const uint16_t *>(base)[id]) : reinterpret_cast<const float *>(base)[id]; };
    const uint64_t *best = a.best + slot * a.n_top;
    // a given token's logit, requested ahead of everything
    const int token = (int)threadIdx.x < a.n_tokens ? a.tokens[row * a.n_tokens + threadIdx.x] : -1;
    const bool there = token >= 0 && token < a.vocab;
    const float token_z = there ? load(token) : 0.f;
    constexpr int EARLY = 4;   // tokens of a thread that are requested before it is known which of them count
    const int64_t all = (int64_t)a.parts * a.n_top;
    uint64_t keys[EARLY];
#pragma unroll
    for (int e = 0; e < EARLY; ++e) keys[e] = (int)threadIdx.x + e * JT < all ? best[threadIdx.x + e * JT] : 0;
    if (wave == 0) {
        Part p{-INFINITY, 0.f, 0.f};
        for (int i = lane; i < a.parts; i += 64) {
            const f32x4 x = a.stats[slot + i];
            p = join(p, Part{x[0], x[1], x[2]}, a.k);
        }
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {   // both of a pair in the same order
            const Part o{__shfl_xor(p.m, i), __shfl_xor(p.s, i), __shfl_xor(p.t, i)};
            p = lane & i ? join(o, p, a.k) : join(p, o, a.k);
        }
        if (lane == 0) part_s = p;
    } else if (wave == 1 && a.n_top > 0) {
        // The n_top-th largest of the row is no smaller than the last of any part's list, nor than the smallest of the parts' nth ones.
        const int nth = (a.n_top + a.parts - 1) / a.parts;
        uint64_t last = 0, least = 0;   // least: inverted
        for (int i = lane; i < a.parts; i += 64) {
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
    if (wave >= 2 && a.ranks)
        for (int j = wave - 2; j < a.n_tokens; j += JT / 64 - 2) {
            int n = 0;
            for (int i = lane; i < a.parts; i += 64) n += a.before[(slot + i) * a.n_tokens + j];
#pragma unroll
            for (int i = 32; i > 0; i >>= 1) n += __shfl_xor(n, i);
            if (lane == 0) before_s[j] = n;
        }
    __syncthreads();
    const Row r(a, row, part_s, threadIdx.x == 0);
    if ((int)threadIdx.x < a.n_tokens) r.token(threadIdx.x, there, token_z, before_s[threadIdx.x]);
    if (a.n_top == 0) return;
    const uint64_t bound = bound_s;
    auto list = [&](uint64_t key) {
        if (key && key >= bound) {
            const uint32_t k = atomicAdd(&listed_s, 1u);
            if (k < JLIST) list_s[k] = key;
        }
    };
#pragma unroll
    for (int e = 0; e < EARLY; ++e) list(keys[e]);
    for (int64_t i = threadIdx.x + EARLY * JT; i < all; i += JT) list(best[i]);
    __syncthreads();
    const int listed = (int)listed_s;
    if (listed <= JLIST) {
        for (int i = threadIdx.x; i < listed; i += JT) {
            const uint64_t mine = list_s[i];
            int place = 0;
            for (int j = 0; j < listed; ++j) place += list_s[j] > mine;
            if (place < a.n_top) r.top(place, mine);
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
        if (threadIdx.x == 0) r.top(k, below);
    }
}

// Whole rows while there are enough of them to fill the chip, else parts.  us, one token, its rank and one alternative of 128256 logits, bf16 / float32: 400 rows in three parts 45 / 46, 768 in two 61 / 86,
// 900 in two, which are more workgroups than the chip holds at once (six on a compute unit), 85 / 121, whole they would take 70 / 101; 1024 whole 71 / 105, 1536 97 / 165, 1600, a second round, 130 / 206,
// 4001 235 / 402.
struct LogPlan {
    int part, parts;
};
LogPlan log_plan(int64_t rows, int vocab)
{
    const int64_t want = (1024 + rows - 1) / rows, most = ((int64_t)vocab + 2047) / 2048;   // parts of 2048 logits at least
    LogPlan p;
    p.parts = (int)std::max<int64_t>(1, std::min(want, most));
    p.part = (int)((((int64_t)vocab + p.parts - 1) / p.parts + 7) / 8 * 8);
    p.parts = (int)(((int64_t)vocab + p.part - 1) / p.part);
    return p;
}
struct LogScratch {
    size_t before, best, bytes;
};
LogScratch log_scratch(int64_t rows, const LogPlan &p, int n_tokens, int n_top)
{
    LogScratch s;
    const size_t slots = p.parts > 1 ? (size_t)rows * p.parts : 0;
    s.best = slots * sizeof(f32x4);
    s.before = s.best + slots * n_top * sizeof(uint64_t);
    s.bytes = (s.before + slots * n_tokens * sizeof(int32_t) + 255) / 256 * 256;
    return s;
}

}  // namespace

extern "C" {

size_t sssd_op_logprobs_scratch_bytes(int32_t type, int32_t rows, int32_t vocab, int32_t n_tokens, int32_t n_top)
{
    if ((type != SSSD_F32 && type != SSSD_BF16) || rows <= 0 || vocab <= 0 || n_tokens < 0 || n_tokens > MOST_TOKENS || n_top < 0 || n_top > MOST_TOP || n_top > vocab || vocab > MOST_VOCAB) return 0;
    return log_scratch(rows, log_plan(rows, vocab), n_tokens, n_top).bytes;
}

int sssd_op_logprobs(const void *logits, int32_t type, int32_t rows, int32_t vocab, int64_t row_stride, float temperature, const int32_t *tokens,
                     int32_t n_tokens, float *logprobs, int32_t *ranks, float *entropy, int32_t n_top, int32_t *top_ids, float *top_logprobs, void *scratch,
                     size_t scratch_bytes, void *stream)
{
    if (!logits || (type != SSSD_F32 && type != SSSD_BF16) || rows <= 0 || vocab <= 0 || n_tokens < 0 || n_top < 0 || n_top > vocab) return SSSD_EINVAL;
    if (n_tokens > MOST_TOKENS || n_top > MOST_TOP || vocab > MOST_VOCAB) return SSSD_ECAPACITY;
    if ((n_tokens > 0 && (!tokens || !logprobs)) || (n_top > 0 && (!top_ids || !top_logprobs))) return SSSD_EINVAL;
    const bool bf16 = type == SSSD_BF16;
    if ((uintptr_t)logits % (bf16 ? 2 : 4) || (rows > 1 && row_stride < 0)) return SSSD_EINVAL;
    const float k = 1.4426950408889634f / temperature;
    // where a difference of logits is beyond float32's range, times k it is beyond that of exponents
    if (!(temperature > 0.f) || !(k >= 1e-36f) || !(k <= 1.5e38f)) return SSSD_EINVAL;
    const LogPlan p = log_plan(rows, vocab);
    const LogScratch z = log_scratch(rows, p, n_tokens, n_top);
    if (z.bytes && (!scratch || (uintptr_t)scratch % 16)) return SSSD_EINVAL;
    if (scratch_bytes < z.bytes || (int64_t)rows * p.parts > UINT32_MAX / LT) return SSSD_ECAPACITY;
    LogArgs a{};
    a.logits = (const char *)logits;
    a.stride = rows > 1 ? row_stride : 0;
    a.rows = rows; a.vocab = vocab; a.part = p.part; a.parts = p.parts;
    a.n_tokens = n_tokens; a.n_top = n_top;
    a.k = k;
    a.inv_t = 1.f / temperature;
    a.tokens = tokens; a.logprobs = logprobs; a.ranks = ranks; a.entropy = entropy; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
    a.stats = (f32x4 *)scratch;
    a.best = (uint64_t *)((char *)scratch + z.best);
    a.before = (int32_t *)((char *)scratch + z.before);
    hipStream_t s = (hipStream_t)stream;
    const dim3 grid((uint32_t)rows * p.parts);
    if (p.parts == 1) {
        if (bf16) hipLaunchKernelGGL((logprob_kernel<true, true>), grid, dim3(LT), 0, s, a);
        else hipLaunchKernelGGL((logprob_kernel<false, true>), grid, dim3(LT), 0, s, a);
        return hipGetLastError() == hipSuccess ? SSSD_OK : SSSD_EHIP;
    }
    if (bf16) hipLaunchKernelGGL((logprob_kernel<true, false>), grid, dim3(LT), 0, s, a);
    else hipLaunchKernelGGL((logprob_kernel<false, false>), grid, dim3(LT), 0, s, a);
    if (hipGetLastError() != hipSuccess) return SSSD_EHIP;
    if (bf16) hipLaunchKernelGGL(logprob_join_kernel<true>, dim3(rows), dim3(JT), 0, s, a);
    else hipLaunchKernelGGL(logprob_join_kernel<false>, dim3(rows), dim3(JT), 0, s, a);
    return hipGetLastError() == hipSuccess ? SSSD_OK : SSSD_EHIP;
}

}  // extern "C"
