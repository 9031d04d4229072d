"""What several continuations of one prompt need, one dict of plain values per case.

A case has a "kind":
  fork      the slots of a paged 8-bit cache become continuations of other slots, all at once: whole blocks are shared, the last one, where it is partly
            filled, is copied for all but one of them, in every layer; slots are emptied, pages that nobody names are free again.
  reserve   the blocks that a step's (or a prompt's) rows will be written to become pages of their sequences' own: missing ones are taken from the pool,
            shared ones replaced, with their rows where some of them live.
  compact   the pages in use move to the front of the pool, or to another pool.
  shared    attention of a step's new rows over an 8-bit cache whose sequences share a long prefix in groups.
  logprobs  log-probabilities and ranks of given tokens, the entropy and the most probable tokens of rows of logits.

Pages are bytes here: a layer of a pool is all pages' codes and then all pages' scales.  What attention reads is code * scale: the code an 8-bit float (4
bits of exponent, 3 of mantissa) or an 8-bit integer, the scale the smallest power of two that keeps every row of a block of 32 in range.  Inputs come from
the seed alone; `exact` restates every kind, numbers in 64 bits and tables on the host.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
BLOCK = 32
SHAPES = {
    "tiny": dict(nq=4, nkv=2, d=64),
    "8b": dict(nq=32, nkv=8, d=128),
    "70b": dict(nq=64, nkv=8, d=128),
}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _fork(name, shape, layers, slots, prompts, ctx, ctx_max, prune):
    """prune: all slots hold continuations, some end, others go on in their place; else the prompts' first continuations."""
    c = dict(kind="fork", shape=shape, layers=layers, slots=slots, prompts=prompts, ctx=ctx, ctx_max=ctx_max, prune=prune)
    return dict(c, name=name) if name else c


def _reserve(name, shape, layers, slots, n, ctx, ctx_max, shared, padded):
    """shared: how many slots still share the block that they would write to with another one."""
    c = dict(kind="reserve", shape=shape, layers=layers, slots=slots, n=n, ctx=ctx, ctx_max=ctx_max, shared=shared, padded=padded)
    return dict(c, name=name) if name else c


def _compact(name, shape, layers, slots, pages, used, to_pages):
    """used: pages in use, by slots' rows; to_pages: of another pool that takes them, 0: in place."""
    c = dict(kind="compact", shape=shape, layers=layers, slots=slots, pages=pages, used=used, to_pages=to_pages)
    return dict(c, name=name) if name else c


def _shared(name, shape, fmt, dtype, groups, prefix, alone, n, rows, rows_max=0, tree=False, padded=False):
    """groups: sizes; prefix: whole blocks' positions that the first group shares (the next ones share half of the one before); alone: sequences
    behind the groups that share nothing; each sequence has rows .. rows_max rows of its own before the n new ones."""
    c = dict(kind="shared", shape=shape, fmt=fmt, dtype=dtype, groups=groups, prefix=prefix, alone=alone, n=n, rows=rows, rows_max=rows_max or rows,
             tree=tree, padded=padded)
    return dict(c, name=name) if name else c


def _logprobs(name, rows, vocab, dtype, tokens, top, temperature=1.0, banned=0):
    """banned: every so-manyth token is masked, 0: none."""
    c = dict(kind="logprobs", rows=rows, vocab=vocab, dtype=dtype, tokens=tokens, top=top, temperature=temperature, banned=banned)
    return dict(c, name=name) if name else c


def listed():
    return [
        # eight answers to one prompt
        _fork("fork_8b_best_of_8", "8b", 32, 8, 1, 2001, 2001, False),
        # 64 slots of four prompts: half of the continuations end and the better ones take their places
        _fork("fork_70b_64_slots", "70b", 16, 64, 4, 300, 1500, True),
        # a step of nine rows for a small batch
        _reserve("reserve_step_9rows", "8b", 4, 16, 9, 300, 2000, 2, False),
        # prompts of up to 4001 tokens admitted beside forked sequences that were rolled back into shared blocks
        _reserve("reserve_prompts_4001", "8b", 8, 24, 4001, 0, 900, 11, True),
        # a small pool after many sequences have ended
        _compact("compact_300_pages", "tiny", 2, 12, 300, 131, 0),
        # half of a large pool is holes: its pages go to a smaller one
        _compact("compact_to_1100_pages", "8b", 8, 40, 1900, 1001, 1100),
        # four answers of a small model to a short prompt, plain decoding
        _shared("shared_tiny_4", "tiny", "e4m3", "f32", "4", 512, 0, 1, 5, 60),
        # best of eight with eight drafts each
        _shared("shared_8b_best_of_8_k8", "8b", "e4m3", "f32", "8", 2048, 0, 9, 1, 300),
        # a serving batch behind two system prompts, ragged, padded trees of drafts
        _shared("shared_70b_two_prompts", "70b", "int8", "bf16", "17,9", 4000, 3, 5, 100, 1500, tree=True, padded=True),
        # many short questions about one long document
        _shared("shared_8b_64_long", "8b", "e4m3", "bf16", "64", 32768, 0, 1, 33, 400),
        # the tokens of a step of nine rows, five alternatives each
        _logprobs("logprobs_9rows", 9, 128256, "f32", 1, 5),
        # scoring a prompt of 1501 tokens
        _logprobs("logprobs_prompt_1501", 1501, 128256, "bf16", 1, 1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["fork", "reserve", "compact", "shared", "shared", "shared", "logprobs", "logprobs"])
    shape = rng.choice(["tiny", "8b", "8b", "70b"])
    if kind == "fork":
        layers, slots = rng.randint(1, 7), _log(rng, 2, 64)
        ctx = _log(rng, 1, 1500)
        return _fork("", shape, layers, slots, rng.randint(1, max(1, min(slots // 2, 6))), rng.choice([ctx, max(1, ctx // 4)]), ctx, rng.random() < 0.5)
    if kind == "reserve":
        slots = _log(rng, 2, 48)
        ctx = _log(rng, 1, 1500)
        n = rng.randint(1, 32) if rng.random() < 0.6 else _log(rng, 33, 80000 // slots if slots > 20 else 4001)
        return _reserve("", shape, rng.randint(1, 8), slots, n, rng.choice([ctx, ctx // 3]), ctx, rng.randint(0, slots - 1), rng.random() < 0.5)
    if kind == "compact":
        pages = _log(rng, 8, 1900)
        used = rng.randint(1, max(1, min(pages, 1000)))
        return _compact("", shape, rng.randint(1, 8), _log(rng, 1, 48), pages, used, rng.choice([0, 0, used, used + rng.randint(1, 200)]))
    if kind == "shared":
        s = SHAPES[shape]
        n = rng.choice([1, rng.randint(1, 9), rng.randint(1, 32)])
        sizes = [_log(rng, 1, 40) for _ in range(rng.choice([1, 1, 2, 4]))]
        B = sum(sizes)
        most = 64 * 32 * 32768 // (B * n * s["nq"])
        prefix = _log(rng, BLOCK, max(BLOCK, min(32768, most * 3 // 4))) // BLOCK * BLOCK
        own_rows = _log(rng, 1, max(2, min(2000, most // 4, 60000 // B)))
        return _shared("", shape, rng.choice(["e4m3", "int8"]), rng.choice(["f32", "bf16"]), ",".join(str(x) for x in sizes), prefix, rng.choice([0, 0, 1, 5]), n,
                       rng.choice([own_rows, max(1, own_rows // 5)]), own_rows, tree=rng.random() < 0.3, padded=rng.random() < 0.3)
    vocab = rng.choice([1024, 32001, 128256, _log(rng, 100, 200000)])
    rows = _log(rng, 1, max(2, min(1501, 1501 * 128256 // vocab // 2)))
    return _logprobs("", rows, vocab, rng.choice(["f32", "bf16"]), rng.choice([1, 1, 2, 7]), rng.choice([0, 1, 5, 20]), rng.choice([1.0, 1.0, 0.6, 1.5]), rng.choice([0, 0, 3]))


# ---------------------------------------------------------------- inputs ----
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 6271 + 41)
    return g


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _spread(lo, hi, count):
    """Lengths spread evenly over [lo, hi]: part of the case, so that its work is fixed."""
    return [hi - (hi - lo) * (b * 11 % 31) // 30 for b in range(count)]


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _page_bytes(case):
    """(codes, scales) of a page of one layer."""
    s = SHAPES[case["shape"]]
    return s["nkv"] * 64 * s["d"], s["nkv"] * 8


def _layer_bytes(case, pages):
    codes, scales = _page_bytes(case)
    return (pages * (codes + scales) + 255) // 256 * 256


def _tables(case, seed):
    """What the host knows of a paging case before the call: a table and lens as lists, the pool's size, and what the call takes beside them."""
    rng = random.Random(int(seed) * 13 + 5)
    slots = case["slots"]
    extra = {}
    if case["kind"] == "fork":
        per = _blocks(case["ctx_max"])
        pages = case["prompts"] * per + slots * 2 + 7
        free = rng.sample(range(pages), pages)
        of = [b % case["prompts"] for b in range(slots)]
        lens_of = _spread(case["ctx"], case["ctx_max"], case["prompts"])
        table, lens = [[-1] * (per + 1) for _ in range(slots)], [0] * slots
        for b in range(slots):
            if b < case["prompts"]:
                n = lens_of[b]
                for i in range(_blocks(n)):
                    table[b][i] = free.pop()
                lens[b] = n
            elif case["prune"]:
                n = lens_of[of[b]]
                for i in range(_blocks(n)):
                    table[b][i] = table[of[b]][i] if i < n // BLOCK else free.pop()
                lens[b] = n
        origins = list(of)
        if case["prune"]:     # the later half of every prompt's continuations ends; an earlier one takes the place, or nobody
            origins = []
            for b in range(slots):
                rank, all_of = b // case["prompts"], len(range(of[b], slots, case["prompts"]))
                keep = (all_of + 1) // 2
                origins.append(b if rank < keep else of[b] + case["prompts"] * rng.randrange(keep))
            if slots >= 8:
                origins[-1] = -1
        extra["origins"] = origins
    elif case["kind"] == "reserve":
        lens = _spread(case["ctx"], case["ctx_max"], slots)
        counts = [case["n"] - (b * 7 % 5) * case["n"] // 6 for b in range(slots)] if case["padded"] else [case["n"]] * slots
        per = max(_blocks(n + c) for n, c in zip(lens, counts))
        pages = sum(_blocks(n + c) for n, c in zip(lens, counts)) + 2 * slots + 5
        free = rng.sample(range(pages), pages)
        table = [[-1] * per for _ in range(slots)]
        for b in range(slots):
            for i in range(_blocks(lens[b])):
                table[b][i] = free.pop()
        last = min(case["shared"], slots - 1)
        for b in range(last):     # slots that were forked from one and rolled back to its length
            lens[b], counts[b], table[b] = lens[last], min(counts[b], counts[last]), list(table[last])
        extra["counts"] = counts
    else:
        each = [case["used"] // slots + (1 if b < case["used"] % slots else 0) for b in range(slots)]
        pages, per = case["pages"], max(each) + 1
        free = rng.sample(range(pages), pages)
        table = [[free.pop() if i < n else -1 for i in range(per)] for n in each]
        lens = [n * BLOCK for n in each]
    refs = [0] * pages
    for row in table:
        for p in row:
            if p >= 0:
                refs[p] += 1
    return dict(extra, table=table, lens=lens, refs=refs, pages=pages, per=per)


def _bytes(case, seed, pages, salt=0):
    g = _gen(seed + 1000003 * salt)
    return torch.randint(0, 256, (case["layers"], _layer_bytes(case, pages)), generator=g, device=DEV, dtype=torch.uint8)


def _sizes(case):
    return [int(x) for x in case["groups"].split(",")]


def _batch(case):
    """Group of every sequence (-1: none), positions that each group shares (whole blocks), rows of its own and new ones of every sequence."""
    sizes = _sizes(case)
    group = [i for i, m in enumerate(sizes) for _ in range(m)] + [-1] * case["alone"]
    prefix = [max(BLOCK, (case["prefix"] >> i) // BLOCK * BLOCK) for i in range(len(sizes))]
    rows = _spread(case["rows"], case["rows_max"], len(group))
    counts = [max(1, case["n"] - b % 3) if case["padded"] else case["n"] for b in range(len(group))]
    return group, prefix, rows, counts


def _heads(g, shape, dtype):
    """Rows of keys: a few channels of every head are several times as large as the others."""
    x = torch.randn(shape, generator=g, device=DEV)
    gain = torch.exp2((torch.rand(shape[-2:], generator=g, device=DEV) - 0.5) * 2)
    gain[..., ::29] *= 6.0
    return (x * gain).to(dtype)


def _shared_inputs(case, seed):
    """(prefixes' K and V, own rows' K and V with the new ones behind them, q, parents)."""
    g = _gen(seed)
    s, n = SHAPES[case["shape"]], case["n"]
    group, prefix, rows, counts = _batch(case)
    B, own_rows = len(group), _blocks(max(rows) + n) * BLOCK
    pre = [(_heads(g, (p, s["nkv"], s["d"]), torch.bfloat16), torch.randn(p, s["nkv"], s["d"], generator=g, device=DEV).to(torch.bfloat16)) for p in prefix]
    K, V = _heads(g, (B, own_rows, s["nkv"], s["d"]), torch.bfloat16), torch.randn(B, own_rows, s["nkv"], s["d"], generator=g, device=DEV).to(torch.bfloat16)
    q = torch.randn(B, n, s["nq"], s["d"], generator=g, device=DEV).to(TYPES[case["dtype"]])
    parents = (torch.rand((B, n), generator=g, device=DEV) * torch.arange(n, device=DEV)).to(torch.int32) if case["tree"] else None
    return pre, K, V, q, parents


def _logits(case, seed):
    g = _gen(seed)
    rows, vocab = case["rows"], case["vocab"]
    z = torch.empty(rows, vocab, dtype=TYPES[case["dtype"]], device=DEV)
    sharp = torch.rand(rows, 1, generator=g, device=DEV) * 3 + 0.5         # from nearly flat rows to nearly certain ones
    for a in range(0, rows, 64):
        z[a:a + 64] = (torch.randn(min(64, rows - a), vocab, generator=g, device=DEV) * sharp[a:a + 64]).to(z.dtype)
    best = torch.randint(0, vocab, (rows, 1), generator=g, device=DEV)
    z.scatter_add_(1, best, (4 * sharp * torch.rand(rows, 1, generator=g, device=DEV)).to(z.dtype))
    if case["banned"]:
        z[:, 1::case["banned"]] = -math.inf
    tokens = torch.randint(0, vocab, (rows, case["tokens"]), generator=g, device=DEV)
    tokens[:, 0] = torch.where(torch.rand(rows, generator=g, device=DEV) < 0.7, best[:, 0], tokens[:, 0])
    return z, tokens.to(torch.int32)


def prepare(case, seed):
    kind = case["kind"]
    state = dict(case=case)
    if kind in ("fork", "reserve", "compact"):
        h = _tables(case, seed)
        table, refs, lens = _int(h["table"]), _int(h["refs"]), _int(h["lens"])
        state.update(table0=table, refs0=refs, table=table.clone(), refs=refs.clone(), lens=lens, pages=h["pages"])
        if kind == "fork":
            state["origins"] = _int(h["origins"])
        if kind == "reserve":
            state["counts"] = _int(h["counts"])
        if kind == "compact":
            state["moved"], state["in_use"] = torch.zeros_like(refs), torch.zeros(1, dtype=torch.int32, device=DEV)
        pool = _bytes(case, seed, h["pages"])
        second = _bytes(case, seed, case["to_pages"], 1) if kind == "compact" and case["to_pages"] else None
        if own:
            from paper_2411_05894_amd import kv8
            s = SHAPES[case["shape"]]

            def paged(pages, data):
                cache = kv8.Kv8Cache(case["layers"], s["nq"], s["nkv"], s["d"], case["slots"], table.shape[1] * BLOCK, "e4m3", n_pages=pages, device=DEV)
                cache.cache.copy_(data.view(-1))
                return kv8.Kv8Pages(cache)
            state["book"] = paged(h["pages"], pool)
            state["book"].table.copy_(table)
            state["book"].refs.copy_(refs)
            if second is not None:
                state["to"] = paged(case["to_pages"], second)
        else:
            state["pool"] = pool
            if second is not None:
                state.update(to_pool=second, to_table=torch.full_like(table, -1), to_refs=torch.zeros(case["to_pages"], dtype=torch.int32, device=DEV))
        return state
    if kind == "logprobs":
        state["logits"], state["tokens"] = _logits(case, seed)
        return state
    s, n = SHAPES[case["shape"]], case["n"]
    group, prefix, rows, counts = _batch(case)
    B, sizes = len(group), _sizes(case)
    pre, K, V, q, parents = _shared_inputs(case, seed)
    front = [prefix[i] if i >= 0 else 0 for i in group]
    state.update(q=q, parents=parents, out=torch.zeros(q.shape, dtype=q.dtype, device=DEV), lens=_int([a + b for a, b in zip(front, rows)]),
                 counts=_int(counts) if case["padded"] else None)
    if own:
        from paper_2411_05894_amd import kv8
        per = _blocks(max(a + b for a, b in zip(front, rows)) + n)
        total = sum(prefix) // BLOCK + B * (_blocks(max(rows) + n) + 1)
        cache = kv8.Kv8Cache(1, s["nq"], s["nkv"], s["d"], B, per * BLOCK, case["fmt"], n_pages=total, device=DEV)
        book = kv8.Kv8Pages(cache)
        starts, at = [], 0
        origins, lens = list(range(B)), torch.zeros(B, dtype=torch.int32, device=DEV)
        for i, m in enumerate(sizes):      # the first sequence of a group holds its prefix, the others are forked from it
            starts.append(at)
            here = torch.zeros(B, dtype=torch.int32, device=DEV)
            here[at] = prefix[i]
            book.sssd_kv8_reserve(prefix[i], lens, here)
            cache.sssd_kv8_append(0, pre[i][0][None], pre[i][1][None], lens[at:at + 1] * 0, counts=here[at:at + 1], first=at)
            lens[at] = prefix[i]
            origins[at:at + m] = [at] * m
            at += m
        book.sssd_kv8_fork(_int(origins), lens)
        fill = _int([a + c for a, c in zip(rows, counts)])
        book.sssd_kv8_reserve(K.shape[1], lens, fill)
        cache.sssd_kv8_append(0, K, V, lens, counts=fill)
        state.update(cache=cache, book=book, starts=_int(starts + [at]), shared=_int(prefix),
                     workspace=cache.sssd_kv8_shared_workspace(B, n))
    else:
        live = _below(_int([a + c for a, c in zip(rows, counts)]), K.shape[1])
        state.update(rows=_int(rows), held=[_quantised(x, live, case["fmt"]) for x in (K, V)],
                     pre=[[_quantised(x[None], torch.ones(1, len(x), dtype=torch.bool, device=DEV), case["fmt"]) for x in pair] for pair in pre])
    return state


# ------------------------------------------------------------ plain forms ----
def _below(n, rows):
    return torch.arange(rows, device=DEV)[None, :] < n[:, None]


def _quantised(x, live, fmt):
    """(codes [B, rows, heads, d], scales [B, blocks, heads]) of x, whose rows are whole blocks."""
    B, rows, heads, d = x.shape
    x = torch.where(live[..., None, None], x.float(), 0.0).view(B, rows // BLOCK, BLOCK, heads, d)
    m, e = torch.frexp(x.abs().amax((2, 4)))
    top, mant = (9, 0.875) if fmt == "e4m3" else (7, 127.0 / 128.0)
    e = torch.where(m > 0, e - top + (m > mant), 0).clamp(-126, 127)
    scale = ((e + 127) << 23).to(torch.int32).view(torch.float32)
    codes = x / scale[:, :, None, :, None]
    codes = codes.to(torch.float8_e4m3fn) if fmt == "e4m3" else codes.round().to(torch.int8)
    return codes.view(B, rows, heads, d), scale


def _values(codes, scale):
    B, rows, heads, d = codes.shape
    return (codes.float().view(B, rows // BLOCK, BLOCK, heads, d) * scale[:, :, None, :, None]).view(B, rows, heads, d)


def _parts(case, pool, pages):
    """Views of a pool: codes [layers, pages, bytes], scales likewise."""
    codes, scales = _page_bytes(case)
    return (pool[:, :pages * codes].view(case["layers"], pages, codes), pool[:, pages * codes:pages * (codes + scales)].view(case["layers"], pages, scales))


def _counted(table, pages):
    seen = torch.where(table >= 0, table, pages).flatten().long()
    return torch.zeros(pages + 1, dtype=torch.int32, device=DEV).scatter_add_(0, seen, torch.ones_like(seen, dtype=torch.int32))[:pages]


def _lowest_free(refs, wanted):
    """For every place that `wanted` marks a free page, the lowest first; pages behind the last one otherwise."""
    order = torch.cumsum((refs == 0).int(), 0)
    need = torch.cumsum(wanted.flatten().int(), 0)
    return torch.searchsorted(order, need.to(order.dtype)).view(wanted.shape).to(torch.int32)


def _copy_pages(case, pool, pages, src, dst, to=None, to_pages=0):
    for a, b in zip(_parts(case, pool, pages), _parts(case, pool if to is None else to, to_pages or pages)):
        b[:, dst.long()] = a[:, src.long()]


def _plain_fork(state):
    case, table, lens = state["case"], state["table"], state["lens"]
    origins = state["origins"].long()
    slots, per = table.shape
    slot = torch.arange(slots, device=DEV)
    safe = origins.clamp(min=0)
    length = torch.where(origins >= 0, lens[safe], 0)
    blk = torch.arange(per, device=DEV)
    new = torch.where(blk < ((length + BLOCK - 1) // BLOCK)[:, None], table[safe], -1)
    # the last, partly filled block stays with the origin where that goes on itself, else with the lowest slot
    same = (origins[None, :] == origins[:, None]) & (origins >= 0)[:, None]
    lowest = torch.where(same, slot[None, :], slots).amin(1)
    heir = torch.where(origins[safe] == safe, slot == origins, slot == lowest)
    copied = (length % BLOCK > 0) & ~heir & (origins >= 0)
    part = (length // BLOCK).clamp(max=per - 1).long()[:, None]
    kept = torch.where(copied[:, None] & (blk == part), -1, new)
    refs = _counted(kept, state["pages"])
    page = _lowest_free(refs, copied)
    old = torch.gather(new, 1, part)[:, 0]
    new = torch.where(copied[:, None] & (blk == part), page[:, None], new)
    which = torch.nonzero(copied)[:, 0]
    _copy_pages(case, state["pool"], state["pages"], old[which], page[which])
    table.copy_(new)
    state["refs"].copy_(_counted(new, state["pages"]))
    lens.copy_(length)
    return [state["pool"], table, state["refs"], lens]


def _plain_reserve(state):
    case, table, refs, pages = state["case"], state["table"], state["refs"], state["pages"]
    table.copy_(state["table0"])
    refs.copy_(state["refs0"])
    lens, counts = state["lens"], state["counts"]
    slots, per = table.shape
    blk = torch.arange(per, device=DEV)
    touched = (blk >= (lens // BLOCK)[:, None]) & (blk < ((lens + counts + BLOCK - 1) // BLOCK)[:, None]) & (counts > 0)[:, None]
    place = torch.arange(slots * per, device=DEV).view(slots, per)
    many = touched & (table >= 0)
    page = torch.where(many, table, pages).long()
    asked = torch.zeros(pages + 1, dtype=torch.int32, device=DEV).scatter_add_(0, page.flatten(), torch.ones_like(page.flatten(), dtype=torch.int32))
    first = torch.full((pages + 1,), slots * per, dtype=torch.int64, device=DEV).scatter_reduce_(0, page.flatten(), place.flatten(), "amin")
    held = torch.cat([refs, refs.new_ones(1)])
    others = many & (held[page] > 1) & ~((asked[page] == held[page]) & (first[page] == place))     # where all who share it ask, the first keeps it
    wanted = touched & (table < 0) | others
    fresh = _lowest_free(refs, wanted)
    live = others & (blk * BLOCK < lens[:, None])
    at = torch.nonzero(live)
    _copy_pages(case, state["pool"], pages, table[at[:, 0], at[:, 1]], fresh[at[:, 0], at[:, 1]])
    table.copy_(torch.where(wanted, fresh, table))
    refs.copy_(_counted(table, pages))
    return [state["pool"], table, refs]


def _plain_compact(state):
    case, table, refs, pages = state["case"], state["table"], state["refs"], state["pages"]
    table.copy_(state["table0"])
    refs.copy_(state["refs0"])
    used = refs > 0
    count = used.int().sum()
    page = torch.arange(pages, device=DEV)
    rank = torch.cumsum(used.int(), 0) - 1
    if case["to_pages"]:
        moved = torch.where(used, rank, -1)
        src = torch.nonzero(used)[:, 0]
        _copy_pages(case, state["pool"], pages, src, moved[src], state["to_pool"], case["to_pages"])
        table_out, refs_out = state["to_table"], state["to_refs"]
        refs_out.zero_()
        refs_out[moved[src]] = refs[src]
    else:
        movers, holes = torch.nonzero(used & (page >= count))[:, 0], torch.nonzero(~used & (page < count))[:, 0]
        moved = torch.where(used, page, -1)
        moved[movers] = holes
        _copy_pages(case, state["pool"], pages, movers, holes)
        table_out, refs_out = table, refs
        refs[holes] = refs[movers]
        refs[movers] = 0
    moved = moved.to(torch.int32)
    table_out.copy_(torch.where(table >= 0, moved[table.clamp(min=0).long()], -1))
    state["moved"].copy_(moved)
    state["in_use"].copy_(count)
    return [state["to_pool"] if case["to_pages"] else state["pool"], table_out, refs_out, state["moved"], state["in_use"]]


def _plain_shared(state):
    case = state["case"]
    s, n = SHAPES[case["shape"]], case["n"]
    nq, nkv, d = s["nq"], s["nkv"], s["d"]
    g = nq // nkv
    group, prefix, _, _ = _batch(case)
    B, q = len(group), state["q"]
    rows = state["rows"].long()[:, None]
    k, v = (_values(*x) for x in state["held"])
    at = torch.arange(k.shape[1], device=DEV)
    row = torch.arange(n, device=DEV)
    parents = (row - 1).expand(B, n) if state["parents"] is None else state["parents"]
    steps = (parents[..., None] == row) & (row > 0)[:, None] | (row[:, None] == row)     # a row leads to its parent or to itself
    bits = (torch.linalg.matrix_power(steps.double(), n) > 0).long()                     # [B, row, new row]: itself or an ancestor
    new = (at - rows).clamp(0, n - 1)
    seen = torch.gather(bits, 2, new[:, None, :].expand(B, n, -1)) > 0
    visible = (at < rows)[:, None] | (seen & ((at >= rows) & (at < rows + n))[:, None])
    qh = q.float().view(B, n, nkv, g, d).permute(2, 0, 1, 3, 4).reshape(nkv, B, n * g, d)
    mine = torch.matmul(qh, k.permute(2, 0, 3, 1).contiguous()) / math.sqrt(d)           # [nkv, B, n * g, own rows]
    mine = mine.view(nkv, B, n, g, -1).masked_fill(~visible[None, :, :, None, :], -math.inf).view(nkv, B, n * g, -1)
    v = v.permute(2, 0, 1, 3).contiguous()
    out = torch.empty(nkv, B, n * g, d, device=DEV)
    first = 0
    for size, pre in zip(_sizes(case) + [1] * case["alone"], state["pre"] + [None] * case["alone"]):
        b = slice(first, first + size)
        first += size
        most = mine[:, b].amax(-1, keepdim=True)
        if pre is not None:      # the prefix once, for the rows of all sequences of the group
            pk, pv = (_values(*x)[0].permute(1, 0, 2).contiguous() for x in pre)
            far = torch.matmul(qh[:, b].reshape(nkv, size * n * g, d), pk.transpose(1, 2).contiguous()) / math.sqrt(d)
            most = torch.maximum(most, far.amax(-1, keepdim=True).view(most.shape))
            far = torch.exp(far - most.view(nkv, -1, 1))
        p = torch.exp(mine[:, b] - most)
        total, o = p.sum(-1, keepdim=True), torch.matmul(p, v[:, b])
        if pre is not None:
            total = total + far.sum(-1).view(total.shape)
            o = o + torch.matmul(far, pv).view(o.shape)
        out[:, b] = o / total
    out = out.view(nkv, B, n, g, d).permute(1, 2, 0, 3, 4).reshape(B, n, nq, d).to(q.dtype)
    if case["padded"]:           # rows that a sequence does not have stay as they were
        out = torch.where(_below(state["counts"], n)[..., None, None], out, state["out"])
    return out


def _plain_logprobs(state):
    case, z, tokens = state["case"], state["logits"].float(), state["tokens"].long()
    ids = torch.arange(case["vocab"], device=DEV)
    x = (z - z.amax(1, keepdim=True)) / case["temperature"]
    p = torch.exp(x)
    total = p.sum(1, keepdim=True)
    log_total = torch.log(total)
    own_logit = torch.gather(z, 1, tokens)
    ranks = torch.stack([((z > t[:, None]) | (z == t[:, None]) & (ids < i[:, None])).sum(1, dtype=torch.int32) for t, i in zip(own_logit.T, tokens.T)], 1)
    entropy = log_total[:, 0] - torch.where(p > 0, p * x, 0.0).sum(1) / total[:, 0]
    outs = [torch.gather(x, 1, tokens) - log_total, ranks, entropy]
    if case["top"]:
        top_ids = []
        left = z.clone()
        for _ in range(case["top"]):
            best = torch.where(left == left.amax(1, keepdim=True), ids, case["vocab"]).amin(1, keepdim=True)
            top_ids.append(best)
            left.scatter_(1, best, -math.inf)
        top_ids = torch.cat(top_ids, 1)
        outs += [top_ids.to(torch.int32), torch.gather(x, 1, top_ids) - log_total]
    return outs


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return {"fork": _plain_fork, "reserve": _plain_reserve, "compact": _plain_compact, "shared": _plain_shared, "logprobs": _plain_logprobs}[kind](state)
    if kind == "logprobs":
        from paper_2411_05894_amd import binding as sv
        got = sv.sssd_op_logprobs(state["logits"], state["tokens"], n_top=case["top"], temperature=case["temperature"])
        return list(got) if case["top"] else list(got[:3])
    if kind == "shared":
        state["cache"].sssd_kv8_attention_shared(0, state["q"], state["lens"], state["out"], state["starts"], state["shared"], state["workspace"],
                                                 counts=state["counts"], parents=state["parents"])
        return state["out"]
    book = state["book"]
    if kind == "fork":
        book.sssd_kv8_fork(state["origins"], state["lens"])
        return [_pool(book), book.table, book.refs, state["lens"]]
    book.table.copy_(state["table0"])
    book.refs.copy_(state["refs0"])
    if kind == "reserve":
        book.sssd_kv8_reserve(case["n"], state["lens"], state["counts"])
        return [_pool(book), book.table, book.refs]
    to = state.get("to", book)
    book.sssd_kv8_compact(to=state.get("to"), moved=state["moved"], in_use=state["in_use"])
    return [_pool(to), to.table, to.refs, state["moved"], state["in_use"]]


def _pool(book):
    return book.cache.cache.view(book.cache.cfg.n_layers, -1)


# ------------------------------------------------------------------ work ----
def work(case):
    kind = case["kind"]
    if kind in ("fork", "reserve", "compact"):
        h = _tables(case, 0)
        _, _, _, copies = _moves(case, h)
        entries, pages = len(h["table"]) * h["per"], len(h["refs"]) + (case["to_pages"] if kind == "compact" else 0)
        return dict(bytes=2.0 * len(copies) * case["layers"] * sum(_page_bytes(case)) + 8.0 * (entries + pages), flops=float(entries + pages))
    if kind == "logprobs":
        n = case["rows"] * case["vocab"]
        return dict(bytes=n * (4.0 if case["dtype"] == "f32" else 2.0) + case["rows"] * (12.0 * case["tokens"] + 4 + 8.0 * case["top"]), flops=5.0 * n)
    s = SHAPES[case["shape"]]
    group, prefix, rows, counts = _batch(case)
    nq, nkv, d = s["nq"], s["nkv"], s["d"]
    size = 4 if case["dtype"] == "f32" else 2
    front = [prefix[i] if i >= 0 else 0 for i in group]
    pairs = sum(c * (a + r + (c + 1) / 2) for a, r, c in zip(front, rows, counts))
    held = sum(prefix) + sum(r + c for r, c in zip(rows, counts))
    return dict(bytes=2.0 * nkv * held * (d + 4 / BLOCK) + 2.0 * size * nq * d * sum(counts), flops=4.0 * pairs * nq * d)


# ----------------------------------------------------------------- exact ----
def _moves(case, h):
    """What a paging call leaves: (table, lens, refs or None, copied pages), one slot after the other on the host."""
    table, lens = [list(r) for r in h["table"]], list(h["lens"])
    slots, copies = len(table), []
    if case["kind"] == "fork":
        origins = h["origins"]
        heirs = {}
        for b in list(range(slots)):
            if origins[b] == b:
                heirs[b] = b
        for b in range(slots):
            if origins[b] >= 0:
                heirs.setdefault(origins[b], b)
        out, wanting = [], []
        for b in range(slots):
            o = origins[b]
            n = lens[o] if o >= 0 else 0
            row = [table[o][i] if i * BLOCK < n else -1 for i in range(h["per"])]
            if n % BLOCK and heirs[o] != b:
                wanting.append((b, n // BLOCK, row[n // BLOCK]))
                row[n // BLOCK] = -1
            out.append(row)
        named = {p for row in out for p in row}
        spare = (p for p in range(h["pages"]) if p not in named)
        for b, i, page in wanting:
            out[b][i] = next(spare)
            copies.append((page, out[b][i]))
        return out, [lens[o] if o >= 0 else 0 for o in origins], None, copies
    if case["kind"] == "reserve":
        refs = list(h["refs"])
        spare = iter([p for p in range(h["pages"]) if not refs[p]])
        asks = [(b, i) for b in range(slots) if h["counts"][b] for i in range(lens[b] // BLOCK, _blocks(lens[b] + h["counts"][b]))]
        by_page = {}
        for b, i in asks:
            if table[b][i] >= 0:
                by_page.setdefault(table[b][i], []).append((b, i))
        for b, i in asks:
            p = table[b][i]
            if p >= 0 and (refs[p] == 1 or (len(by_page[p]) == refs[p] and by_page[p][0] == (b, i))):
                continue
            table[b][i] = next(spare)
            if p >= 0 and i * BLOCK < lens[b]:
                copies.append((p, table[b][i]))
        return table, lens, None, copies
    refs = h["refs"]
    used = [p for p in range(h["pages"]) if refs[p]]
    if case["to_pages"]:
        to = {p: i for i, p in enumerate(used)}
        copies = list(to.items())
    else:
        holes = [p for p in range(len(used)) if not refs[p]]
        copies = list(zip([p for p in used if p >= len(used)], holes))
        to = {p: p for p in used}
        to.update(copies)
    return [[to[p] if p >= 0 else -1 for p in row] for row in table], lens, [to.get(p, -1) for p in range(h["pages"])], copies


def _round_code(y, fmt):
    """The nearest code of each value, ties to the even one."""
    if fmt == "int8":
        low = torch.floor(y)
        up = (y - low > 0.5) | ((y - low == 0.5) & (low % 2 != 0))
        return low + up.double()
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -20))), -6, 8) - 3)
    low = torch.floor(y.abs() / step)
    rest = y.abs() / step - low
    return torch.sign(y) * (low + ((rest > 0.5) | ((rest == 0.5) & (low % 2 == 1))).double()) * step


def _stored(x, fmt):
    """x [rows, heads, d] from the start of a block: the values that the cache holds."""
    rows, heads, d = x.shape
    whole = torch.zeros(_blocks(rows) * BLOCK, heads, d, dtype=torch.float64, device=DEV)
    whole[:rows] = x
    limit = 448.0 if fmt == "e4m3" else 127.0
    blocks = whole.view(-1, BLOCK, heads, d)
    most = blocks.abs().amax((1, 3), keepdim=True)
    s = torch.exp2(torch.ceil(torch.log2(torch.clamp(most, min=1e-300) / limit)))
    s = torch.where(most <= limit * s / 2, s / 2, s)
    s = torch.where(most > limit * s, s * 2, s)
    s = torch.where(most > 0, s, torch.ones_like(s))
    return (_round_code(blocks / s, fmt) * s).view(-1, heads, d)[:rows]


def exact(case, seed):
    kind = case["kind"]
    if kind in ("fork", "reserve", "compact"):
        h = _tables(case, seed)
        table, lens, moved, copies = _moves(case, h)
        there = kind == "compact" and case["to_pages"]
        pages = case["to_pages"] if there else h["pages"]
        pool = _bytes(case, seed, h["pages"])
        to = _bytes(case, seed, pages, 1) if there else pool
        codes, scales = _page_bytes(case)
        for layer in range(case["layers"]):
            was = pool[layer].clone()
            for a, b in copies:
                to[layer, b * codes:(b + 1) * codes] = was[a * codes:(a + 1) * codes]
                at, was_at = pages * codes + b * scales, h["pages"] * codes + a * scales
                to[layer, at:at + scales] = was[was_at:was_at + scales]
        refs = [0] * pages
        for row in table:
            for p in row:
                if p >= 0:
                    refs[p] += 1
        outs = [to, _int(table), _int(refs)]
        if kind == "fork":
            return outs + [_int(lens)]
        return outs if kind == "reserve" else outs + [_int(moved), _int([sum(r > 0 for r in h["refs"])])]
    if kind == "logprobs":
        logits, tokens = _logits(case, seed)
        rows, top = case["rows"], case["top"]
        outs = [torch.zeros(rows, case["tokens"], dtype=torch.float64, device=DEV), torch.zeros(rows, case["tokens"], dtype=torch.int32, device=DEV),
                torch.zeros(rows, dtype=torch.float64, device=DEV), torch.zeros(rows, top, dtype=torch.int32, device=DEV),
                torch.zeros(rows, top, dtype=torch.float64, device=DEV)]
        for a in range(0, rows, 128):
            z = logits[a:a + 128].double()
            order = torch.sort(z, dim=1, descending=True, stable=True)[1]
            lp = torch.log_softmax(z / case["temperature"], 1)
            t = tokens[a:a + 128].long()
            outs[0][a:a + 128] = torch.gather(lp, 1, t)
            place = torch.empty_like(order).scatter_(1, order, torch.arange(case["vocab"], device=DEV).expand(len(z), -1))
            outs[1][a:a + 128] = torch.gather(place, 1, t).int()
            outs[2][a:a + 128] = -torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(1)
            outs[3][a:a + 128] = order[:, :top].int()
            outs[4][a:a + 128] = torch.gather(lp, 1, order[:, :top])
        return outs if top else outs[:3]
    s, n, fmt = SHAPES[case["shape"]], case["n"], case["fmt"]
    nq, nkv, d = s["nq"], s["nkv"], s["d"]
    pre, K, V, q, parents = _shared_inputs(case, seed)
    group, prefix, rows, counts = _batch(case)
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    tree = parents.cpu().tolist() if parents is not None else [[j - 1 for j in range(n)]] * len(group)
    fronts = [[_stored(x.double(), fmt) for x in pair] for pair in pre]
    for b, (i, held, c) in enumerate(zip(group, rows, counts)):
        kb, vb = _stored(K[b, :held + c].double(), fmt), _stored(V[b, :held + c].double(), fmt)
        if i >= 0:
            kb, vb = torch.cat([fronts[i][0], kb]), torch.cat([fronts[i][1], vb])
        base = len(kb) - c
        kk, vv = kb.permute(1, 2, 0).contiguous(), vb.permute(1, 0, 2).contiguous()
        score = torch.matmul(q[b, :c].double().view(c, nkv, nq // nkv, d).permute(1, 0, 2, 3).reshape(nkv, -1, d), kk).view(nkv, c, nq // nkv, -1) / math.sqrt(d)
        for j in range(c):
            line = {j}
            up = j
            while up:
                up = tree[b][up]
                line.add(up)
            hidden = [base + x for x in range(c) if x not in line]
            if hidden:
                score[:, j][..., hidden] = -math.inf
        o = torch.matmul(torch.softmax(score, -1).view(nkv, -1, base + c), vv).view(nkv, c, nq // nkv, d)
        out[b, :c] = o.permute(1, 0, 2, 3).reshape(c, nq, d)
    return out
