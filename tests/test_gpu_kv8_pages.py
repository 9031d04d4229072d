"""sssd_kv8_fork / reserve / compact against plain statements on lists (tests/pages_reference.py), pages as bytes: tables, counts, lengths and every byte of
the pool have to be equal, and nothing may change where a call is refused on the device."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

import pages_reference as ref
from paper_2411_05894_amd import kv8
from paper_2411_05894_amd.binding import SSSD_ENOSPACE, SSSD_OK

DEV = "cuda:0"


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Pool:
    """A cache of random bytes and who has its pages, here and on lists."""

    def __init__(self, slots, max_seq, pages, layers=2, nkv=2, d=64, fmt="e4m3", seed=1):
        self.cache = kv8.Kv8Cache(layers, nkv, nkv, d, slots, max_seq, fmt, n_pages=pages, device=DEV)
        self.book = kv8.Kv8Pages(self.cache)
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.cache.cache.copy_(torch.randint(0, 256, self.cache.cache.shape, generator=g, device=DEV, dtype=torch.uint8))
        self.layers, self.codes, self.scales, self.pages, self.max_seq = layers, nkv * 64 * d, nkv * 8, pages, max_seq
        self.slots, self.per = slots, self.cache.blocks_per_seq
        self.set([[-1] * self.per for _ in range(slots)], [0] * pages, [0] * slots)

    def set(self, table, refs, lens):
        self.table, self.refs, self.lens = table, refs, list(lens)
        self.book.table.copy_(ints(table))
        self.book.refs.copy_(ints(refs))
        self.d_lens = ints(lens)

    def bytes(self):
        return self.cache.cache.view(self.layers, -1).clone()

    def moved(self, copies, was, out=None, pages=None):
        """The pool's bytes once `copies` are made."""
        out = was.clone() if out is None else out
        pages = pages or self.pages
        for a, b in copies:
            out[:, b * self.codes:(b + 1) * self.codes] = was[:, a * self.codes:(a + 1) * self.codes]
            x, y = self.pages * self.codes + a * self.scales, pages * self.codes + b * self.scales
            out[:, y:y + self.scales] = was[:, x:x + self.scales]
        return out

    def check(self, want, bytes_):
        table, refs = want[:2]
        assert self.book.table.tolist() == table
        assert self.book.refs.tolist() == refs
        assert torch.equal(self.bytes(), bytes_)

    def fork(self, origins):
        want, was = ref.fork(self.table, self.refs, self.lens, origins, self.max_seq), self.bytes()
        self.book.sssd_kv8_fork(ints(origins), self.d_lens)
        if want is None:
            assert self.cache.sssd_kv8_sync() == SSSD_ENOSPACE
            self.check((self.table, self.refs), was)
        else:
            assert self.cache.sssd_kv8_sync() == SSSD_OK
            self.check(want, self.moved(want[3], was))
            self.table, self.refs, self.lens = want[:3]
        assert self.d_lens.tolist() == self.lens
        return want

    def reserve(self, n, lens, counts=None, first=0):
        want, was = ref.reserve(self.table, self.refs, lens, counts or [n] * len(lens), first, n, self.max_seq), self.bytes()
        self.book.sssd_kv8_reserve(n, ints(lens), None if counts is None else ints(counts), first=first)
        if want is None:
            assert self.cache.sssd_kv8_sync() == SSSD_ENOSPACE
            self.check((self.table, self.refs), was)
        else:
            assert self.cache.sssd_kv8_sync() == SSSD_OK
            self.check(want, self.moved(want[2], was))
            self.table, self.refs = want[:2]
        return want

    def compact(self, to=None):
        want, was = ref.compact(self.table, self.refs, None if to is None else to.pages), self.bytes()
        moved, in_use = torch.full_like(self.book.refs, -7), ints([-7])
        there = to or self
        before = there.bytes(), there.table, there.refs
        self.book.sssd_kv8_compact(to=None if to is None else to.book, moved=moved, in_use=in_use)
        assert in_use.item() == sum(n > 0 for n in self.refs)
        if want is None:
            assert self.cache.sssd_kv8_sync() == SSSD_ENOSPACE
            there.check(before[1:], before[0])
            assert (moved == -7).all()
        else:
            assert self.cache.sssd_kv8_sync() == SSSD_OK
            if to is not None:
                self.check((self.table, self.refs), was)
            there.check(want, self.moved(want[3], was, before[0].clone(), there.pages))
            assert moved.tolist() == want[2]
            there.table, there.refs = want[:2]
        return want


SHAPES = [dict(layers=1, nkv=1, d=64), dict(layers=3, nkv=8, d=128, fmt="int8"), dict(layers=2, nkv=3, d=64), dict(layers=2, nkv=5, d=128)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("seed", range(4))
def test_a_life_of_a_pool(shape, seed):
    """Sequences admitted, grown, forked, reordered, rolled back, ended and compacted at random, every call against the statement; some of them are
    refused for want of pages."""
    rng = random.Random(seed)
    slots, max_seq = rng.choice([1, 3, 8, 20]), rng.choice([32, 100, 333])
    pool = Pool(slots, max_seq, rng.randint(slots, slots * ref.blocks(max_seq)), seed=seed, **shape)
    refused = done = 0
    for turn in range(40):
        what = rng.random()
        if what < 0.45:
            n = rng.randint(1, rng.choice([9, 40, max_seq]))
            first = rng.randrange(slots)
            B = rng.randint(1, slots - first)
            lens = [pool.lens[first + k] for k in range(B)]
            counts = [rng.randint(0, min(n, max_seq - a)) for a in lens]
            print(f"pool {shape} {seed} turn {turn}: reserve {n} {lens} {counts} {first}", flush=True)
            want = pool.reserve(n, lens, counts, first)
            if want is not None:
                for k in range(B):
                    pool.lens[first + k] += rng.randint(0, counts[k])
                pool.d_lens.copy_(ints(pool.lens))
        elif what < 0.85:
            kind = rng.choice(["any", "permute", "expand", "trim", "end"])
            origins = {"any": [rng.randint(-1, slots - 1) for _ in range(slots)], "permute": rng.sample(range(slots), slots),
                       "expand": [rng.randrange(slots)] * slots, "trim": list(range(slots)),
                       "end": [b if rng.random() < 0.6 else -1 for b in range(slots)]}[kind]
            if rng.random() < 0.3:       # rolled back first, maybe into shared blocks
                pool.lens = [rng.randint(0, n) for n in pool.lens]
                pool.d_lens.copy_(ints(pool.lens))
            print(f"pool {shape} {seed} turn {turn}: fork {origins} {pool.lens}", flush=True)
            want = pool.fork(origins)
        else:
            print(f"pool {shape} {seed} turn {turn}: compact", flush=True)
            want = pool.compact()
        refused, done = refused + (want is None), done + (want is not None)
    assert done > 5


@pytest.mark.parametrize("slots,max_seq,pages", [(1, 1, 1), (2, 31, 2), (5, 64, 11), (65, 70, 400), (300, 33, 700), (1030, 40, 3000), (3, 70000, 5000)])
def test_sizes(slots, max_seq, pages):
    """One slot and one page to more slots than threads and rows of more blocks than a workgroup's run."""
    rng = random.Random(slots)
    pool = Pool(slots, max_seq, pages, layers=1, nkv=1)
    lens = [rng.randint(0, max_seq) for _ in range(slots)]
    for b in rng.sample(range(slots), slots):      # as many as the pool holds
        if sum(ref.blocks(lens[c]) for c in range(slots)) > pages:
            lens[b] = min(lens[b], 20 if b % 3 else 0)
    pool.reserve(max_seq, [0] * slots, lens)
    pool.lens = lens if pool.refs.count(0) < pages or not any(lens) else [0] * slots
    pool.d_lens.copy_(ints(pool.lens))
    pool.fork([rng.randrange(slots) for _ in range(slots)])
    pool.fork([b if b % 2 else -1 for b in range(slots)])
    pool.compact()
    pool.reserve(5, [min(n, max_seq - min(5, max_seq)) for n in pool.lens], [min(5, max_seq)] * slots if max_seq < 5 else None)


def filled(pages=40, slots=4, max_seq=200, lens=(70, 64, 0, 100)):
    pool = Pool(slots, max_seq, pages)
    pool.reserve(max_seq, [0] * slots, list(lens))
    pool.lens = list(lens)
    pool.d_lens.copy_(ints(pool.lens))
    return pool


def test_forks_that_copy_and_forks_that_need_not():
    pool = filled()
    assert len(pool.fork([0, 0, 0, 0])[3]) == 3          # one of the four goes on with the part-filled block
    assert pool.fork([0, -1, -1, -1])[3] == []
    pool = filled()
    assert pool.fork([3, 0, 1, 2])[3] == []              # a permutation copies nothing
    assert pool.fork([1, 1, 1, 0])[3] != []              # the lowest of those who continue slot 1 has its page: it is gone itself
    pool = filled()
    assert pool.fork([1, 1, 1, 1])[3] == []              # 64 rows: whole blocks
    assert pool.refs.count(4) == 2
    assert pool.fork([-1] * 4)[1] == [0] * 40


def test_pages_that_a_caller_holds():
    """A count above the table's entries keeps a page: it is not free when all slots let go of it, and who writes to it gets a copy."""
    pool = filled()
    held = pool.table[3][3]
    pool.refs[held] += 1
    pool.book.refs.copy_(ints(pool.refs))
    want = pool.reserve(3, [100], first=3)
    assert want[2] and want[2][0][0] == held
    pool.lens[3] = 103
    pool.d_lens.copy_(ints(pool.lens))
    assert pool.fork([-1] * 4)[1][held] == 1
    pool.compact()


def test_who_shares_a_block_and_writes_to_it():
    pool = filled()
    pool.fork([0, 0, 0, 0])
    pool.lens = [40] * 4                                  # back into a shared block
    pool.d_lens.copy_(ints(pool.lens))
    before = [list(r) for r in pool.table]
    want = pool.reserve(9, [40] * 4)
    assert [r[1] == b[1] for r, b in zip(pool.table, before)] == [True, False, False, False] and len(want[2]) == 3
    pool = filled()
    pool.fork([0, 0, 0, 0])
    want = pool.reserve(9, [40, 40], first=1)             # others go on sharing it: both get their own
    assert len(want[2]) == 2
    pool = filled()
    pool.fork([0, 0, 0, 0])
    want = pool.reserve(9, [32] * 4)                      # nothing in it is live: replaced without a copy
    assert want[2] == []
    assert pool.reserve(4, [0, 3, 5, 7], [0, 0, 0, 0])[2] == []


def test_calls_that_cannot_be_done_do_nothing():
    for change in (dict(origins=[0, 4, 1, 2]), dict(origins=[-2, 0, 1, 2]), dict(lens=[70, 201, 0, 100], origins=[0, 1, 2, 3]), dict(lens=[-1, 64, 0, 100]),
                   dict(lens=[70, 64, 33, 100], origins=[2, 2, 2, 2])):
        pool = filled()
        if "lens" in change:
            pool.lens = change["lens"]
            pool.d_lens.copy_(ints(pool.lens))
        assert pool.fork(change.get("origins", [0, 1, 2, 3])) is None, change
    for lens, counts, n in (([70, -1], None, 5), ([70, 198], None, 5), ([70, 64], [6, 0], 5), ([70, 64], [5, -1], 5)):
        assert filled().reserve(n, lens, counts) is None
    pool = filled(pages=9)                                # 3 + 2 + 4 pages: none left
    assert pool.fork([0, 0, 2, 3]) is not None            # slot 1's two pages are free by then
    pool = filled(pages=9)
    assert pool.fork([0, 1, 0, 3]) is None
    assert pool.reserve(33, [70, 64, 0, 100]) is None
    assert pool.reserve(26, [70, 64, 0, 100], [26, 0, 0, 0]) is not None
    for spoil in (40, -2, 100000):
        pool = filled()
        pool.table[1][0] = spoil
        pool.book.table.copy_(ints(pool.table))
        assert pool.fork([0, 0, 2, 3]) is None
        assert pool.compact() is None
        assert pool.reserve(3, [0], first=1) is None
        assert pool.reserve(3, [70]) is not None          # nothing of the spoiled row is looked at
    pool = filled()
    pool.table[0][5] = pool.refs.index(0)                 # names a page that counts nothing
    pool.book.table.copy_(ints(pool.table))
    assert pool.fork([0, 1, 2, 3]) is None and pool.compact() is None
    small = Pool(4, 200, 8)
    assert filled().compact(small) is None
    # and what comes after a refused call is as if it had not been
    pool = filled(pages=10)
    assert pool.fork([0, 0, 0, 0]) is not None and pool.fork([0, 1, 9, 9]) is None and pool.reserve(90, [70] * 4) is None
    assert pool.fork([2, 2, -1, -1]) is not None


@pytest.mark.parametrize("to", [9, 10, 40, 4100])
def test_to_another_pool(to):
    pool = filled(pages=60)
    pool.fork([0, 1, 3, 3])
    pool.fork([1, 0, 2, 3])
    other = Pool(4, 200, to, seed=5)
    other.reserve(20, [0, 0], [20, 20])                   # what it held is gone
    pool.compact(other)
    large = Pool(4, 200, 333, seed=6)
    if other.refs.count(0) < to:
        other.compact(large)
        large.lens = list(pool.lens)
        large.d_lens.copy_(ints(large.lens))
        large.fork([1, 1, 2, 2])


def test_large_pools():
    """More pages than one pass of a workgroup over the pool looks at, the free ones at its far end."""
    pool = Pool(6, 32 * 3000, 12289, layers=1, nkv=1)
    n = 32 * 2040
    assert pool.reserve(32 * 3000, [0] * 6, [n + 5, n, n + 31, 0, n, n + 1]) is not None
    pool.lens = [n + 5, n, n + 31, 0, n, n + 1]
    pool.d_lens.copy_(ints(pool.lens))
    assert pool.fork([0, 0, 0, 2, 2, 5]) is not None
    pool.fork([5, -1, 3, -1, -1, 5])
    assert pool.compact() is not None


def test_captured_calls_replay():
    """A step's fork and reserve in a graph, replayed with other origins, eager work between; every replay as the statement."""
    pool = filled(pages=60)
    origins, lens, counts = ints([0, 0, 2, 3]), pool.d_lens, ints([9] * 4)
    stream = torch.cuda.Stream()
    keep = [t.clone() for t in (pool.book.table, pool.book.refs, lens, pool.cache.cache)]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        pool.book.sssd_kv8_fork(origins, lens)
        pool.book.sssd_kv8_reserve(9, lens, counts)
        pool.book.sssd_kv8_compact()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pool.book.sssd_kv8_fork(origins, lens)
        pool.book.sssd_kv8_reserve(9, lens, counts)
        pool.book.sssd_kv8_compact()
    for t, k in zip((pool.book.table, pool.book.refs, lens, pool.cache.cache), keep):
        t.copy_(k)
    for who in ([0, 0, 2, 3], [1, 1, 1, 0], [3, 2, -1, 0], [0, 0, 0, 0]):
        origins.copy_(ints(who))
        was = pool.bytes()
        graph.replay()
        other = filled(pages=45)
        other.fork([0, 0, 0, 1])
        torch.cuda.synchronize()
        table, refs, pool.lens, copies = ref.fork(pool.table, pool.refs, pool.lens, who, 200)
        was = pool.moved(copies, was)
        table, refs, copies = ref.reserve(table, refs, pool.lens, [9] * 4, 0, 9, 200)
        was = pool.moved(copies, was)
        table, refs, _, copies, _ = ref.compact(table, refs)
        pool.check((table, refs), pool.moved(copies, was))
        pool.table, pool.refs = table, refs
        assert lens.tolist() == pool.lens
    assert pool.cache.sssd_kv8_sync() == SSSD_OK


def test_no_call_allocates():
    pool = filled()
    torch.cuda.synchronize()
    free, origins = torch.cuda.mem_get_info()[0], ints([0, 0, 0, 3])
    for _ in range(10):
        pool.book.sssd_kv8_fork(origins, pool.d_lens)
        pool.book.sssd_kv8_reserve(3, pool.d_lens)
        pool.book.sssd_kv8_compact()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free


@pytest.mark.parametrize("slots,max_seq", [(4, 200), (4, 40000), (1024, 128), (1024, 129), (1025, 96)])
def test_forks_of_few_and_many_entries(slots, max_seq):
    """Few slots and as many as the deciding workgroup has threads, or more, rows of one block and of more than a workgroup's run; and what is refused."""
    rng = random.Random(slots + max_seq)
    pool = Pool(slots, max_seq, 3 * slots + 40, layers=1, nkv=1)
    lens = [rng.randint(0, min(max_seq, 70)) for _ in range(slots)]
    lens[0], lens[1] = 70, 33
    pool.reserve(70, [0] * slots, lens)
    pool.lens = list(lens)
    pool.d_lens.copy_(ints(lens))
    origins = [rng.choice([-1, b, rng.randrange(slots)]) for b in range(slots)]
    origins[-1] = origins[2] = 1
    assert pool.fork(origins) is not None
    assert pool.fork([b if rng.random() < 0.8 else rng.randrange(slots) for b in range(slots)]) is not None
    state = pool.table, pool.refs, pool.lens
    live = next(b for b in range(slots) if pool.lens[b] > 32)
    for row, block, value in ((live, 0, -2 ** 31), (live, 1, -1), (live, 0, 2 ** 31 - 1), (slots - 1, pool.per - 1, -2 ** 31), (0, pool.per - 1, -2)):
        spoiled = [list(r) for r in state[0]]
        spoiled[row][block] = value
        pool.set(spoiled, state[1], state[2])
        assert pool.fork([live if b == 0 else b for b in range(slots)]) is None, (row, block, value)
    for row, origin in ((0, slots), (slots - 1, -2), (1, 2 ** 31 - 1), (2, -2 ** 31)):
        pool.set(*state)
        assert pool.fork([origin if b == row else b for b in range(slots)]) is None, (row, origin)
    for length in (-1, -2 ** 31, max_seq + 1, 2 ** 31 - 1):
        pool.set(state[0], state[1], [length if b == live else n for b, n in enumerate(state[2])])
        assert pool.fork(list(range(slots))) is None, length
    pool.set(*state)
    assert pool.fork(list(range(slots))[::-1]) is not None


@pytest.mark.parametrize("blocks", [1, 1023, 1024, 1025, 2048, 2049, 3500, 4095, 4096, 4097, 5300])
def test_reserves_of_many_blocks(blocks):
    """As many blocks as a round of the workgroup has threads, as it keeps, and more; some of them shared, some in place already."""
    slots = 5
    each = (blocks + slots - 1) // slots
    pool = Pool(slots, 32 * each + 64, blocks + 40, layers=1, nkv=1)
    counts = [32 * min(each, max(0, blocks - b * each)) for b in range(slots)]
    pool.reserve(9, [0], [9])
    pool.lens[0] = 9
    pool.d_lens.copy_(ints(pool.lens))
    assert pool.fork([0] * slots) is not None                     # slots 1 .. 4 have a block of their own for 9 rows
    pool.lens = [min(n, c) // 2 for n, c in zip(pool.lens, counts)]
    assert sum(ref.blocks(a + c) - a // 32 for a, c in zip(pool.lens, counts)) >= blocks
    assert pool.reserve(32 * each, pool.lens, counts) is not None
    pool.lens = [a + c for a, c in zip(pool.lens, counts)]
    pool.d_lens.copy_(ints(pool.lens))
    assert pool.fork([0, 0] + list(range(2, slots))) is not None
    pool.lens[:2] = [0, 0]
    assert pool.reserve(32 * each, [0] * slots, [min(counts[0], 64), counts[0], 0, 5, 0]) is not None
