// Pages of an 8-bit KV cache: slots that become continuations of others, room for the next rows, a pool without holes.
//
// Nothing is computed but integers: a page's references after a call are those before, less the table entries that let go of it, plus those that take it; pages
// without references are free, and the lowest free ones are taken first, in the order of slots and blocks, by counting over the pool.  So results do not depend
// on the order in which workgroups run: additions and minima of integers are all that is done atomically.
//
// A call is all or nothing.  It is planned first (fork_plan_kernel adds the differences up beside the references, reserve_kernel and compact_kernel look
// everything over), one workgroup decides, and only then are table, references and pages written.
//
// What bounds it: the pages that are copied, in all layers, at the rate of a copy (1001 pages of 64 KiB in 8 layers, 1.05 GB out and in, 201 us of a kernel, 5.2 TB/s); without many, the
// launches and the one workgroup's round trips.  us of kernels: 64 slots forked from four prompts, 3.5 + 4.5 for the plan and the decision, 9.6 for table and 31 pages in 16 layers; room for 9 rows
// of 16 sequences 7.9, for prompts of up to 4001 12, and 3.4 to 5.1 for the copies behind it.  One workgroup decides since the others would wait for each other's counts: a launch
// apiece is what that would cost, and a pool's references are read by one in rounds of 4096.
#include "kv8_host.h"

#include <algorithm>

namespace {

constexpr int PT = 1024;   // threads of the workgroup that decides
constexpr int PER = 4;     // neighbouring pages of a thread in a pass over the pool
constexpr int MOST_PAGES = 1 << 30;   // places behind the last one are numbers, too

// One per workspace.  `fault` and `delta` (behind it, a word per page) are zero before and after every call.
struct PagesHead {
    int32_t fault;       // raised while a call is planned
    int32_t go;          // the decision: 1, or 0 for nothing
    int32_t copies;      // pages to copy
    int32_t used;        // pages in use
};
constexpr size_t HEAD_BYTES = 256;

struct PagesArgs {
    Kv8Geom g;                 // of the pool
    int slots;                 // max_batch
    int32_t *table, *refs;
    const int32_t *origins;    // fork
    int32_t *lens;             // fork; reserve: read only
    const int32_t *counts;     // reserve
    int first, B, n;           // reserve
    int32_t *moved, *in_use;   // compact; may be null
    int32_t *to_table, *to_refs;   // compact to another pool, or null
    int to_pages;
    PagesHead *head;
    int32_t *delta;            // [n_pages]
    int32_t *map;              // [n_pages]: reserve: how many ask for a page; compact: where it goes
    unsigned long long *low;   // [n_pages]: reserve: the first place that asks for a page
    int32_t *was;              // [slots][blocks_per_seq]: fork: the table as it was
    int32_t *want, *got, *len; // [slots]: fork: page to copy or -1, its copy, the new length
    int2 *copy;                // [n_pages]: from, to
    int3 *need;                // [n_pages]: reserve: slot, block, the page there before or -1
    int32_t *status;
};
struct CopyArgs {              // pages as bytes: a layer is all pages' codes and then all pages' scales
    const PagesHead *head;
    const int2 *copy;
    const uint8_t *from;
    uint8_t *to;
    size_t from_layer, to_layer, from_scales, to_scales;   // bytes of a layer, and of its codes
    int layers, code_bytes, scale_bytes, chunks;           // of a page; chunks of COPY bytes
};
constexpr int COPY = 256 * 16 * 4;   // bytes a workgroup copies at a time

__device__ __forceinline__ int agent_load(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Sum over the threads in front, of a whole workgroup of PT; total: of all.
__device__ __forceinline__ int scan_group(int x, int &total, int *lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = x;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const int y = __shfl_up(upto, i);
        if (lane >= i) upto += y;
    }
    __syncthreads();   // lds has been read
    if (lane == 63) lds[wave] = upto;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < PT / 64; ++w) {
        const int y = lds[w];
        before += w < wave ? y : 0;
        total += y;
    }
    return before + upto - x;
}

// The lowest `n` pages for which free(page, which of its thread's): take(i, page) for the i-th of them.  Whole workgroup; returns how many there are, at most n.
template <typename Free, typename Take> __device__ __forceinline__ int find_pages(int pages, int n, int *lds, Free free, Take take)
{
    int found = 0;
    for (int base = 0; base < pages && found < n; base += PT * PER) {
        bool is[PER];
        int mine = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int p = base + (int)threadIdx.x * PER + e;
            is[e] = p < pages && free(p, e);
            mine += is[e];
        }
        int total, at = found + scan_group(mine, total, lds);
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (is[e]) {
                if (at < n) take(at, base + (int)threadIdx.x * PER + e);
                ++at;
            }
        found += total;
    }
    return min(found, n);
}

__device__ __forceinline__ int blocks_of(int len) { return (int)(((unsigned)len + 31u) >> 5); }

// ------------------------------------------------------------------------------------------------------------ fork ----
// Slot b's row after the call, as far as it comes from the table: blocks of its origin's rows but the last one, partly filled, where that is to be copied.
struct Fork {
    int origin, len, part;   // part: that block, or -1: stays where it is
};

// grid (runs of blocks, slots)
__global__ __launch_bounds__(256) void fork_plan_kernel(PagesArgs a)
{
    __shared__ int low_s[4];
    const int b = blockIdx.y, per = a.g.blocks_per_seq;
    const int origin = a.origins[b];
    bool bad = origin < -1 || origin >= a.slots;
    const int len = bad || origin < 0 ? 0 : a.lens[origin];
    bad = bad || len < 0 || len > a.g.max_seq;
    const int live = bad ? 0 : blocks_of(len);
    int heir = b;
    if (!bad && (len & 31) && origin != b) {   // the origin itself where it stays, else the lowest slot
        if (a.origins[origin] == origin) {
            heir = origin;
        } else {
            int low = a.slots;
            for (int s = threadIdx.x; s < b; s += 256) low = a.origins[s] == origin ? min(low, s) : low;
#pragma unroll
            for (int i = 32; i > 0; i >>= 1) low = min(low, __shfl_xor(low, i));
            if ((threadIdx.x & 63) == 0) low_s[threadIdx.x >> 6] = low;
            __syncthreads();
            heir = min(b, min(min(low_s[0], low_s[1]), min(low_s[2], low_s[3])));
        }
    }
    const int part = heir != b ? len >> 5 : -1;
    const int run = 256 * 8;
    for (int i = blockIdx.x * run + threadIdx.x; i < min(per, (int)(blockIdx.x + 1) * run); i += 256) {
        const size_t at = (size_t)b * per + i;
        const int old = a.table[at];
        int now = -1;
        if (i < live) {
            now = a.table[(size_t)origin * per + i];
            bad = bad || now < 0 || now >= a.g.n_pages || a.refs[now] <= 0;
        }
        bad = bad || old < -1 || old >= a.g.n_pages || (old >= 0 && a.refs[old] <= 0);
        a.was[at] = old;
        if (i == part) {
            a.want[b] = now;
            now = -1;
        }
        if (!bad && old != now) {
            if (old >= 0) atomicAdd(&a.delta[old], -1);
            if (now >= 0) atomicAdd(&a.delta[now], 1);
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.len[b] = len;
        if (part < 0) a.want[b] = -1;
    }
    if (__any(bad) && (threadIdx.x & 63) == 0) atomicOr(&a.head->fault, 1);
}

__global__ __launch_bounds__(PT) void fork_decide_kernel(PagesArgs a)
{
    __shared__ int lds[PT / 64];
    int n = 0;
    const bool fault = a.head->fault != 0;
    for (int base = 0; base < a.slots && !fault; base += PT) {   // pages to copy, in the order of slots
        const int b = base + threadIdx.x, page = b < a.slots ? a.want[b] : -1;
        int total;
        const int at = n + scan_group(page >= 0, total, lds);
        if (page >= 0 && at < a.g.n_pages) {
            a.copy[at].x = page;
            a.map[at] = b;
        }
        n += total;
    }
    __syncthreads();
    bool go = !fault && n <= a.g.n_pages;
    if (go && n > 0) {
        const int found = find_pages(a.g.n_pages, n, lds, [&](int p, int) { return a.refs[p] + a.delta[p] == 0; }, [&](int i, int p) { a.copy[i].y = p; });
        go = found == n;
        __syncthreads();
        if (go)
            for (int i = threadIdx.x; i < n; i += PT) {
                const int p = a.copy[i].y;
                a.got[a.map[i]] = p;
                a.delta[p] = 1 - a.refs[p];   // whatever the call's differences are: the page had none left
            }
    }
    if (threadIdx.x == 0) {
        a.head->go = go;
        a.head->copies = go ? n : 0;
        a.head->fault = 0;
        if (!go) atomicOr(a.status, KV8_RANGE);
    }
}

// ----------------------------------------------------------------------------------------------------------- copying ----
__device__ __forceinline__ void copy_pages(const CopyArgs &c, int first, int step)
{
    const int copies = c.head->copies;
    const uint64_t total = (uint64_t)copies * c.layers * c.chunks;
    for (uint64_t i = first; i < total; i += step) {
        const uint32_t which = (uint32_t)(i / c.chunks), chunk = (uint32_t)(i - (uint64_t)which * c.chunks);
        const uint32_t layer = which / (uint32_t)copies, k = which - layer * (uint32_t)copies;
        const int2 move = c.copy[k];
        const uint8_t *from = c.from + layer * c.from_layer;
        uint8_t *to = c.to + layer * c.to_layer;
        const u32x4 *src = reinterpret_cast<const u32x4 *>(from + (size_t)move.x * c.code_bytes);
        u32x4 *dst = reinterpret_cast<u32x4 *>(to + (size_t)move.y * c.code_bytes);
        const int at = (int)chunk * (COPY / 16) + (int)threadIdx.x, end = c.code_bytes / 16;
        u32x4 x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + 256 * e < end) x[e] = src[at + 256 * e];
        if (chunk == 0)
            for (int s = threadIdx.x * 8; s < c.scale_bytes; s += 256 * 8)
                *reinterpret_cast<float2 *>(to + c.to_scales + (size_t)move.y * c.scale_bytes + s) =
                    *reinterpret_cast<const float2 *>(from + c.from_scales + (size_t)move.x * c.scale_bytes + s);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + 256 * e < end) dst[at + 256 * e] = x[e];
    }
}

// Workgroups: `rows` for the table's runs, `pool` for the references, the others copy.
__global__ __launch_bounds__(256) void fork_write_kernel(PagesArgs a, CopyArgs c, int runs, int rows, int pool)
{
    const bool go = a.head->go != 0;
    int id = blockIdx.x;
    if (id < rows) {
        if (!go) return;
        const int b = id / runs, run = 256 * 8, per = a.g.blocks_per_seq, first = (id - b * runs) * run;
        const int origin = a.origins[b], len = a.len[b], live = blocks_of(len), copied = a.want[b];
        const int32_t *row = a.was + (size_t)(origin < 0 ? 0 : origin) * per;
        for (int i = first + threadIdx.x; i < min(per, first + run); i += 256) {
            int page = i < live ? row[i] : -1;
            if (copied >= 0 && i == len >> 5) page = a.got[b];
            a.table[(size_t)b * per + i] = page;
        }
        if (first == 0 && threadIdx.x == 0) a.lens[b] = len;
        return;
    }
    id -= rows;
    if (id < pool) {
        for (int e = 0; e < 4; ++e) {
            const int p = id * 1024 + e * 256 + threadIdx.x;
            if (p >= a.g.n_pages) return;
            const int d = a.delta[p];
            if (d) {
                if (go) a.refs[p] += d;
                a.delta[p] = 0;
            }
        }
        return;
    }
    copy_pages(c, id - pool, gridDim.x - rows - pool);
}

// ---------------------------------------------------------------------------------------------------------- reserve ----
// One workgroup: the blocks that the call's rows touch, slot by slot, a thread each, in as many rounds as they take.  What a thread has read stays with it for up to KEEP rounds
// (1885 blocks of prompts 12 us of kernel, 17 when only one round is kept).
constexpr int KEEP = 4;
struct Asked {
    bool on, bad, live;   // live: rows that live are in the block
    int slot, blk, page, refs;
};
__global__ __launch_bounds__(PT) void reserve_kernel(PagesArgs a)
{
    __shared__ int off_s[PT], len_s[PT], lds[PT / 64], fault_s, shared_s;
    const int per = a.g.blocks_per_seq;
    int early[PER];   // the front of the pool, in case pages are wanted
#pragma unroll
    for (int e = 0; e < PER; ++e) early[e] = (int)threadIdx.x * PER + e < a.g.n_pages ? a.refs[threadIdx.x * PER + e] : 1;
    if (threadIdx.x == 0) fault_s = shared_s = 0;
    __syncthreads();
    auto place = [&](int slot, int blk) { return (size_t)slot * per + blk; };
    // Sequences base .. base + PT - 1: where their blocks begin among those of the round; how many there are.
    auto sequences = [&](int base) {
        const int i = base + (int)threadIdx.x;
        int len = 0, n = 0, total;
        if (i < a.B) {
            const int count = a.counts ? a.counts[i] : a.n;
            len = a.lens[i];
            const bool ok = len >= 0 && count >= 0 && count <= a.n && (int64_t)len + count <= a.g.max_seq;
            if (!ok) fault_s = 1;
            n = ok && count > 0 ? blocks_of(len + count) - (len >> 5) : 0;
            len = ok ? len : 0;
        }
        const int at = scan_group(n, total, lds);
        off_s[threadIdx.x] = at;
        len_s[threadIdx.x] = len;
        __syncthreads();
        return total;
    };
    auto entry = [&](int base, int k, int total) {
        Asked x{k < total, false, false, 0, 0, -1, 0};
        if (!x.on) return x;
        int lo = 0, hi = PT - 1;   // the last sequence that begins at or before k: it has blocks
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (off_s[mid] <= k) lo = mid;
            else hi = mid - 1;
        }
        x.slot = a.first + base + lo;
        x.blk = (len_s[lo] >> 5) + k - off_s[lo];
        x.live = (int64_t)x.blk * 32 < len_s[lo];
        x.page = a.table[place(x.slot, x.blk)];
        return x;
    };
    auto counted = [&](Asked &x) {
        x.bad = x.page < -1 || x.page >= a.g.n_pages;
        x.refs = x.bad || x.page < 0 ? 0 : a.refs[x.page];
        x.bad = x.bad || (x.page >= 0 && x.refs <= 0);
    };
    int total = a.B <= PT ? sequences(0) : 0;
    const bool kept = a.B <= PT && total <= KEEP * PT;
    Asked mine[KEEP];
#pragma unroll
    for (int r = 0; r < KEEP; ++r) {
        mine[r] = Asked{false, false, false, 0, 0, -1, 0};
        if (kept && r * PT < total) mine[r] = entry(0, r * PT + (int)threadIdx.x, total);
    }
#pragma unroll
    for (int r = 0; r < KEEP; ++r)
        if (kept && r * PT < total) counted(mine[r]);
    // f(what is asked) for all blocks in order, the same number of times in every thread
    auto all = [&](auto f) {
        if (kept) {
#pragma unroll
            for (int r = 0; r < KEEP; ++r)
                if (r * PT < total) f(mine[r]);
            return;
        }
        for (int base = 0; base < a.B; base += PT) {
            if (a.B > PT) total = sequences(base);
            for (int r = 0; r < total; r += PT) {
                Asked x = entry(base, r + threadIdx.x, total);
                counted(x);
                f(x);
            }
            __syncthreads();
        }
    };
    // pages that several entries name: their counters
    all([&](const Asked &x) {
        if (x.bad) {
            fault_s = 1;
        } else if (x.refs > 1) {
            shared_s = 1;
            __hip_atomic_store(&a.map[x.page], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(&a.low[x.page], ~0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    });
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const bool fault = fault_s != 0;
    int n = 0;
    if (!fault && shared_s) {
        all([&](const Asked &x) {
            if (x.refs <= 1) return;
            atomicAdd(&a.map[x.page], 1);
            atomicMin(&a.low[x.page], (unsigned long long)place(x.slot, x.blk));
        });
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    if (!fault)
        all([&](const Asked &x) {
            bool wants = x.on && x.page < 0;
            if (x.refs > 1) {   // where all who share a page ask for it, the first one keeps it
                const unsigned long long low = __hip_atomic_load(&a.low[x.page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                wants = !(agent_load(&a.map[x.page]) == x.refs && low == place(x.slot, x.blk));
            }
            int sum;
            const int at = n + scan_group(wants, sum, lds);
            if (wants && at < a.g.n_pages) {
                a.need[at] = int3{x.slot, x.blk, x.page};
                a.copy[at].x = x.page >= 0 && x.live ? x.page : -1;
            }
            n += sum;
        });
    __syncthreads();
    bool go = !fault && n <= a.g.n_pages;
    if (go && n > 0) {
        const int found = find_pages(a.g.n_pages, n, lds, [&](int p, int e) { return (p < PT * PER ? early[e] : a.refs[p]) == 0; }, [&](int i, int p) { a.copy[i].y = p; });
        go = found == n;
    }
    __syncthreads();
    int copies = 0;
    if (go)
        for (int base = 0; base < n; base += PT) {
            const int i = base + threadIdx.x;
            int2 move{-1, 0};
            if (i < n) {
                move = a.copy[i];
                const int3 need = a.need[i];
                a.table[place(need.x, need.y)] = move.y;
                a.refs[move.y] = 1;
                if (need.z >= 0) atomicAdd(&a.refs[need.z], -1);
            }
            int total;   // those with live rows to the front: at or before their own places
            const int at = copies + scan_group(move.x >= 0, total, lds);
            if (move.x >= 0) a.copy[at] = move;
            copies += total;
        }
    if (threadIdx.x == 0) {
        a.head->copies = copies;
        if (!go) atomicOr(a.status, KV8_RANGE);
    }
}

__global__ __launch_bounds__(256) void copy_kernel(CopyArgs c) { copy_pages(c, blockIdx.x, gridDim.x); }

// ---------------------------------------------------------------------------------------------------------- compact ----
// Some entry of the table is none of a page in use.  first, step: of a thread
__device__ __forceinline__ bool unsound(const PagesArgs &a, size_t first, size_t step)
{
    const size_t n = (size_t)a.slots * a.g.blocks_per_seq;
    bool bad = false;
    for (size_t i = first; i < n; i += step) {
        const int p = a.table[i];
        bad = bad || p < -1 || p >= a.g.n_pages || (p >= 0 && a.refs[p] <= 0);
    }
    return bad;
}
__global__ __launch_bounds__(256) void compact_check_kernel(PagesArgs a)
{
    if (__any(unsound(a, (size_t)blockIdx.x * 256 + threadIdx.x, (size_t)gridDim.x * 256)) && (threadIdx.x & 63) == 0) atomicOr(&a.head->fault, 1);
}
// Up to so many entries the workgroup that plans looks them over itself, four a thread, instead of a launch in front of it (call with
// 300 pages 19.8 -> 16.2 us).
constexpr size_t FEW_ENTRIES = 4 * PT;

__global__ __launch_bounds__(PT) void compact_plan_kernel(PagesArgs a)
{
    __shared__ int lds[PT / 64];
    const int pages = a.g.n_pages;
    bool fault = a.head->fault != 0;
    if ((size_t)a.slots * a.g.blocks_per_seq <= FEW_ENTRIES) fault = __syncthreads_or(unsound(a, threadIdx.x, PT));
    int used = 0;
    for (int base = 0; base < pages; base += PT * PER) {
        int mine = 0, total;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int p = base + (int)threadIdx.x * PER + e;
            mine += p < pages && a.refs[p] > 0;
        }
        scan_group(mine, total, lds);
        used += total;
    }
    const bool go = !fault && (!a.to_table || used <= a.to_pages);
    int copies = 0;
    if (go) {
        if (a.to_table) {   // all of them, in order
            copies = used;
            find_pages(pages, used, lds, [&](int p, int) { return a.refs[p] > 0; }, [&](int i, int p) {
                a.map[p] = i;
                a.copy[i] = int2{p, i};
            });
            for (int p = threadIdx.x; p < pages; p += PT)
                if (a.refs[p] <= 0) a.map[p] = -1;
        } else {   // the i-th in use behind the first `used` pages into the i-th hole among them
            for (int p = threadIdx.x; p < pages; p += PT) a.map[p] = a.refs[p] > 0 ? p : -1;
            copies = find_pages(used, used, lds, [&](int p, int) { return a.refs[p] <= 0; }, [&](int i, int p) { a.copy[i].y = p; });
            __syncthreads();
            find_pages(pages - used, copies, lds, [&](int p, int) { return a.refs[used + p] > 0; }, [&](int i, int p) { a.copy[i].x = used + p; });
            __syncthreads();
            for (int i = threadIdx.x; i < copies; i += PT) {
                const int2 move = a.copy[i];
                a.map[move.x] = move.y;
                a.refs[move.y] = a.refs[move.x];
                a.refs[move.x] = 0;
            }
        }
        __syncthreads();
        if (a.moved)
            for (int p = threadIdx.x; p < pages; p += PT) a.moved[p] = a.map[p];
    }
    if (threadIdx.x == 0) {
        a.head->go = go;
        a.head->copies = copies;
        a.head->used = used;
        a.head->fault = 0;
        if (a.in_use) *a.in_use = used;
        if (!go) atomicOr(a.status, KV8_RANGE);
    }
}

__global__ __launch_bounds__(256) void compact_write_kernel(PagesArgs a, CopyArgs c, int rows, int pool)
{
    int id = blockIdx.x;
    if (id < rows + pool && !a.head->go) return;
    if (id < rows) {
        const size_t n = (size_t)a.slots * a.g.blocks_per_seq;
        int32_t *to = a.to_table ? a.to_table : a.table;
        for (size_t i = (size_t)id * 256 + threadIdx.x; i < n; i += (size_t)rows * 256) {
            const int p = a.table[i];
            to[i] = p >= 0 ? a.map[p] : -1;
        }
        return;
    }
    id -= rows;
    if (id < pool) {
        const int used = a.head->used;
        for (int p = id * 256 + threadIdx.x; p < a.to_pages; p += pool * 256) a.to_refs[p] = p < used ? a.refs[a.copy[p].x] : 0;
        return;
    }
    copy_pages(c, id - pool, gridDim.x - rows - pool);
}

// ------------------------------------------------------------------------------------------------------------- host ----
struct PagesSizes {
    size_t delta, map, low, was, want, got, len, copy, need, bytes;
};
bool pages_sizes(const sssd_kv8_config &c, const Sizes8 &S, PagesSizes &z)
{
    size_t entries, at = HEAD_BYTES;
    if (__builtin_mul_overflow((size_t)c.max_batch, (size_t)S.blocks_per_seq, &entries) || entries > SIZE_MAX / 64) return false;
    auto take = [&](size_t n, size_t size) {
        const size_t here = at;
        at = (at + n * size + 255) / 256 * 256;
        return here;
    };
    const size_t pages = S.n_pages, slots = c.max_batch;
    z.delta = take(pages, 4);
    z.map = take(pages, 4);
    z.low = take(pages, 8);
    z.was = take(entries, 4);
    z.want = take(slots, 4);
    z.got = take(slots, 4);
    z.len = take(slots, 4);
    z.copy = take(pages, sizeof(int2));
    z.need = take(pages, sizeof(int3));
    z.bytes = at;
    return true;
}

int check_pages(const sssd_kv8 *kv, const sssd_kv8_pages *p, Sizes8 &S, PagesArgs &a)
{
    if (!kv || !p || !p->table || !p->refs || kv->block_table != p->table) return SSSD_EINVAL;
    const int rc = check_cache(kv, 0, S);
    if (rc) return rc;
    PagesSizes z;
    if (!pages_sizes(kv->cfg, S, z) || !p->workspace || (uintptr_t)p->workspace % ALIGN) return SSSD_EINVAL;
    if (p->ws_bytes < z.bytes || S.n_pages > MOST_PAGES) return SSSD_ECAPACITY;
    a = PagesArgs{};
    a.g = geom(kv, S);
    a.slots = kv->cfg.max_batch;
    a.table = p->table;
    a.refs = p->refs;
    char *ws = (char *)p->workspace;
    a.head = (PagesHead *)ws;
    a.delta = (int32_t *)(ws + z.delta);
    a.map = (int32_t *)(ws + z.map);
    a.low = (unsigned long long *)(ws + z.low);
    a.was = (int32_t *)(ws + z.was);
    a.want = (int32_t *)(ws + z.want);
    a.got = (int32_t *)(ws + z.got);
    a.len = (int32_t *)(ws + z.len);
    a.copy = (int2 *)(ws + z.copy);
    a.need = (int3 *)(ws + z.need);
    a.status = kv->status;
    return SSSD_OK;
}

CopyArgs copy_args(const PagesArgs &a, const sssd_kv8 *from, const Sizes8 &F, const sssd_kv8 *to, const Sizes8 &T)
{
    CopyArgs c{};
    c.head = a.head;
    c.copy = a.copy;
    c.from = (const uint8_t *)from->cache;
    c.to = (uint8_t *)to->cache;
    c.from_layer = F.layer_bytes;
    c.to_layer = T.layer_bytes;
    c.from_scales = F.scales_at;
    c.to_scales = T.scales_at;
    c.layers = from->cfg.n_layers;
    c.code_bytes = from->cfg.n_kv_heads * 64 * from->cfg.head_dim;
    c.scale_bytes = from->cfg.n_kv_heads * (int)sizeof(float2);
    c.chunks = (c.code_bytes + COPY - 1) / COPY;
    return c;
}
// Workgroups that copy `most` pages at most: eight to a compute unit go round.
uint32_t copy_groups(const CopyArgs &c, int64_t most)
{
    const int64_t chunks = (int64_t)c.layers * c.chunks;
    return (uint32_t)(most >= 2048 / chunks + 1 ? 2048 : std::max<int64_t>(1, most * chunks));
}

constexpr int64_t MOST_GROUPS = MOST_THREADS / 256 - 4096;

}  // namespace

extern "C" {

int sssd_kv8_pages_sizes(const sssd_kv8_config *cfg, size_t *ws_bytes)
{
    Sizes8 S;
    const int rc = sizes8(cfg, S);
    if (rc) return rc;
    PagesSizes z;
    if (!ws_bytes || !pages_sizes(*cfg, S, z)) return SSSD_EINVAL;
    *ws_bytes = z.bytes;
    return SSSD_OK;
}

int sssd_kv8_fork(const sssd_kv8 *kv, const sssd_kv8_pages *pages, const int32_t *origins, int32_t *lens, void *stream)
{
    Sizes8 S;
    PagesArgs a;
    const int rc = check_pages(kv, pages, S, a);
    if (rc) return rc;
    if (!origins || !lens) return SSSD_EINVAL;
    a.origins = origins;
    a.lens = lens;
    const int64_t runs = (S.blocks_per_seq + 256 * 8 - 1) / (256 * 8), rows = runs * a.slots, pool = ((int64_t)S.n_pages + 1023) / 1024;
    if (a.slots > 65535 || rows + pool > MOST_GROUPS) return SSSD_ECAPACITY;
    const CopyArgs c = copy_args(a, kv, S, kv, S);
    hipStream_t s = (hipStream_t)stream;
    hipLaunchKernelGGL(fork_plan_kernel, dim3((uint32_t)runs, a.slots), dim3(256), 0, s, a);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(fork_decide_kernel, dim3(1), dim3(PT), 0, s, a);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(fork_write_kernel, dim3((uint32_t)(rows + pool) + copy_groups(c, a.slots)), dim3(256), 0, s, a, c, (int)runs, (int)rows, (int)pool);
    HIP_TRY(hipGetLastError());
    return SSSD_OK;
}

int sssd_kv8_reserve(const sssd_kv8 *kv, const sssd_kv8_pages *pages, int32_t first, int32_t B, int32_t n, const int32_t *lens, const int32_t *counts,
                     void *stream)
{
    Sizes8 S;
    PagesArgs a;
    const int rc = check_pages(kv, pages, S, a);
    if (rc) return rc;
    if (!lens || first < 0 || B <= 0 || n <= 0) return SSSD_EINVAL;
    if ((int64_t)first + B > a.slots || (n > kv->cfg.max_seq && !counts)) return SSSD_ECAPACITY;
    const int64_t blocks = std::min<int64_t>(S.blocks_per_seq, ((int64_t)n + 62) / 32);   // that a sequence's rows touch
    if (B * blocks > INT32_MAX) return SSSD_ECAPACITY;
    a.lens = const_cast<int32_t *>(lens);
    a.counts = counts;
    a.first = first;
    a.B = B;
    a.n = n;
    const CopyArgs c = copy_args(a, kv, S, kv, S);
    hipStream_t s = (hipStream_t)stream;
    hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(PT), 0, s, a);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(copy_kernel, dim3(copy_groups(c, B)), dim3(256), 0, s, c);
    HIP_TRY(hipGetLastError());
    return SSSD_OK;
}

int sssd_kv8_compact(const sssd_kv8 *kv, const sssd_kv8_pages *pages, const sssd_kv8 *to, const sssd_kv8_pages *to_pages, int32_t *moved, int32_t *in_use,
                     void *stream)
{
    Sizes8 S, T;
    PagesArgs a;
    int rc = check_pages(kv, pages, S, a);
    if (rc) return rc;
    if (!to != !to_pages) return SSSD_EINVAL;
    a.moved = moved;
    a.in_use = in_use;
    CopyArgs c = copy_args(a, kv, S, kv, S);
    if (to) {
        PagesArgs other;
        if ((rc = check_pages(to, to_pages, T, other))) return rc;
        const sssd_kv8_config &x = kv->cfg, &y = to->cfg;
        if (x.format != y.format || x.n_layers != y.n_layers || x.n_kv_heads != y.n_kv_heads || x.head_dim != y.head_dim || x.max_batch != y.max_batch ||
            S.blocks_per_seq != T.blocks_per_seq)
            return SSSD_EINVAL;
        if (to->cache == kv->cache || to_pages->table == pages->table || to_pages->refs == pages->refs) return SSSD_EINVAL;
        a.to_table = to_pages->table;
        a.to_refs = to_pages->refs;
        a.to_pages = T.n_pages;
        c = copy_args(a, kv, S, to, T);
    }
    const size_t entries = (size_t)a.slots * S.blocks_per_seq;
    const int rows = (int)std::min<size_t>((entries + 255) / 256, 1024), pool = to ? std::min((T.n_pages + 255) / 256, 256) : 0;
    hipStream_t s = (hipStream_t)stream;
    if (entries > FEW_ENTRIES) {
        hipLaunchKernelGGL(compact_check_kernel, dim3(rows), dim3(256), 0, s, a);
        HIP_TRY(hipGetLastError());
    }
    hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(PT), 0, s, a);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(compact_write_kernel, dim3((uint32_t)(rows + pool) + copy_groups(c, S.n_pages)), dim3(256), 0, s, a, c, rows, pool);
    HIP_TRY(hipGetLastError());
    return SSSD_OK;
}

}  // extern "C"
