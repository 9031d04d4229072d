"""sssd_kv8_attention_shared, each of its ways by name: joined with few rows to a prefix, joined with many, and sequences by themselves.  Which one a call takes shows in its
workspace, which only joined calls write.  Bounds and batches are those of tests/test_gpu_kv8_shared.py."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import test_gpu_kv8_shared as shared
from kv8_reference import attend
from paper_2411_05894_amd import kv8
from paper_2411_05894_amd import binding as sv
from paper_2411_05894_amd.binding import SSSD_ENOSPACE, SSSD_OK

DEV = "cuda:0"
Batch, ints, random_parents = shared.Batch, shared.ints, shared.random_parents
MARK = 0x5A
LONG = 200000


@pytest.fixture
def long_room(monkeypatch):
    """Sequences that could be so long that prefixes are joined."""
    monkeypatch.setattr(shared, "LONGER", LONG)


@pytest.fixture
def no_room(monkeypatch):
    monkeypatch.setattr(shared, "LONGER", 0)


def way(batch, call):
    """What `call` returns, and how it went: "apart", or "few" or "many" rows of a prefix to a workgroup, by the rows that a group has on average (two tiles of 16 are few)."""
    batch.workspace.fill_(MARK)
    got = call()
    torch.cuda.synchronize()
    groups = max(len(batch.shared), 1)
    rows = -(-batch.B * batch.n * (batch.nq // batch.cache.n_kv_heads) // groups)
    return got, "apart" if bool((batch.workspace == MARK).all()) else "few" if rows <= 32 else "many"


# heads, groups, own rows, n, sequences in no group, the way
FEW = [((4, 2, 64), [(3, 320), (5, 1500)], [5, 70], 2), ((32, 8, 128), [(2, 700)] * 12, [3, 100, 31], 1), ((8, 8, 64), [(12, 900), (20, 64)], [40, 1], 1), ((64, 8, 128), [(2, 2048)], [60], 1),
       ((8, 1, 64), [(2, 64), (2, 3000), (2, 32), (2, 65)] * 3, [33, 0], 1)]
MANY = [((8, 2, 128), [(40, 1200)], [200, 5], 5), ((32, 8, 128), [(17, 2048), (8, 320)], [60, 64, 1], 3), ((4, 2, 64), [(40, 640)], [3, 1], 9), ((64, 8, 128), [(9, 4001), (3, 333)], [7, 100], 9),
        ((8, 2, 64), [(30, 20000)], [5, 44], 3), ((6, 6, 128), [(65, 512)], [9], 1),
        ((64, 8, 128), [(4, 2048)], [60], 1), ((8, 1, 64), [(2, 64), (2, 3000), (2, 32), (2, 65)] * 3, [33, 0], 2)]

EITHER = [((8, 1, 128), [(20, 1200)], [200, 5], 5)]      # bfloat16 joined, float32 by themselves


def as_said(went, kind):
    return went in kind.split(" or ")


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind,case", [("few", c) for c in FEW] + [("many", c) for c in MANY] + [("many or apart", c) for c in EITHER])
def test_joined(long_room, kind, case, dtype, fmt):
    (nq, nkv, d), groups, own, n = case
    batch = Batch(fmt, nq, nkv, d, groups, own, n, alone=2)
    a, went = way(batch, lambda: batch.check(dtype))
    assert as_said(went, kind)
    assert torch.equal(a, batch.check(dtype))
    parents = [random_parents(n, 7 + b) for b in range(batch.B)]
    batch.check(dtype, parents)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind,heads,groups,n", [("few", (4, 2, 64), [(4, 1200)] * 4, 3), ("few", (16, 2, 128), [(3, 2100)] * 6, 1), ("many or apart", (8, 1, 128), [(20, 1200)], 5), ("many", (8, 2, 128), [(40, 1200)], 5),
                                                 ("many", (4, 2, 64), [(33, 1200), (20, 300)], 4), ("many", (64, 8, 128), [(12, 2000)], 2)])
@pytest.mark.parametrize("scales", [(12, -12), (-12, -6, 0, 6, 12), (-30, 20, -3), (0, -4, -8)])
def test_values_of_many_sizes(long_room, kind, heads, groups, n, dtype, fmt, scales):
    """V's blocks within and beyond what a prefix's operands hold in one unit."""
    batch = Batch(fmt, *heads, groups, [200, 5], n, scales=list(scales), seed=6)
    assert as_said(way(batch, lambda: batch.check(dtype))[1], kind)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind,heads,groups,n", [("few", (4, 2, 64), [(4, 640)] * 4, 2), ("many or apart", (8, 1, 128), [(20, 640)], 5), ("many", (8, 2, 128), [(40, 640)], 5)])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -20, 2.0 ** 25])
def test_blocks_of_zeros(long_room, kind, heads, groups, n, dtype, size):
    """Blocks whose V is 0, and others whose K is: their scale is 1, whatever that of the others."""
    batch = Batch("e4m3", *heads, groups, [5, 70], n, spread=1.0)
    cache, book = batch.cache, batch.book
    at = 0
    for m, p in groups:
        k, v = batch.held[0][at:at + 1, :p].clone(), batch.held[1][at:at + 1, :p].clone() * size
        v[:, 64:96] = 0
        v[:, 160:352] = 0
        k[:, 32:64] = 0
        cache.sssd_kv8_append(batch.layer, k.contiguous(), v.contiguous(), ints([0]), first=at)
        at += m
    assert cache.sssd_kv8_sync() == SSSD_OK
    cache.sssd_kv8_read(batch.layer, None, ints([a + c for a, c in zip(batch.lens, batch.counts)]), *batch.held)
    assert (batch.held[1][0, 64:96] == 0).all() and (batch.held[1][0, 128:160] != 0).any()
    assert as_said(way(batch, lambda: batch.check(dtype))[1], kind)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind,groups,n", [("few", [(4, 900)] * 4, 2), ("few", [(3, 300), (9, 64)] * 2, 1), ("many", [(20, 900)], 3), ("many", [(12, 300), (2, 2000)], 4)])
def test_a_row_that_is_no_number_spoils_itself_alone(long_room, kind, groups, n, dtype):
    batch = Batch("e4m3", 8, 2, 64, groups, [7, 90], n)
    good, went = way(batch, lambda: batch.check(dtype))
    assert went == kind
    q = batch.q.to(dtype)
    q[1, n - 1, 3, 5], q[batch.B - 1, 0, 0, 0], q[2, 0, 7] = float("nan"), float("inf"), float("-inf")
    out = torch.full_like(q, 5.5)
    assert way(batch, lambda: batch.run(q, out))[1] == kind
    spoilt = torch.zeros(q.shape[:3], dtype=torch.bool, device=DEV)
    spoilt[1, n - 1, 3] = spoilt[batch.B - 1, 0, 0] = spoilt[2, 0, 7] = True
    assert torch.equal(out[~spoilt], good[~spoilt])


@pytest.mark.parametrize("kind,groups,n", [("few", [(4, 500), (3, 100), (4, 640), (2, 64)], 2), ("many", [(14, 500), (13, 100)], 3)])
def test_what_is_out_of_range(long_room, kind, groups, n):
    """A sequence shorter than what it is said to share, or of a bad length or count, is set to 0; nobody else's bits change.  Rows from counts[b] on stay."""
    batch = Batch("e4m3", 8, 2, 64, groups, [7, 90], n)
    q = batch.q
    good, went = way(batch, lambda: batch.check(torch.float32))
    assert went == kind
    for who, length in ((0, -5), (2, 479), (1, 10 ** 6), (0, 0), (3, 2 ** 31 - 1), (batch.B - 1, 63)):
        out, lens = torch.full_like(q, 5.5), list(batch.lens)
        lens[who] = length
        assert way(batch, lambda: batch.run(q, out, lens=lens))[1] == kind
        assert batch.cache.sssd_kv8_sync() == SSSD_ENOSPACE
        assert (out[who] == 0).all()
        assert all(torch.equal(out[b], good[b]) for b in range(batch.B) if b != who)
    out = torch.full_like(q, 5.5)
    starts = list(batch.starts)
    starts[1] = batch.B + 1
    batch.run(q, out, starts=starts)
    assert batch.cache.sssd_kv8_sync() == SSSD_ENOSPACE
    for b in range(batch.B):
        batch.compare(b, q, out)
    counts = [(b * 3) % (n + 1) for b in range(batch.B)]
    batch.counts = counts
    batch.check(torch.float32)
    batch.counts = [n + 1 if b == 2 else c for b, c in enumerate(counts)]
    out = torch.full_like(q, 5.5)
    batch.run(q, out)
    assert batch.cache.sssd_kv8_sync() == SSSD_ENOSPACE and (out[2] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind,n", [("few", 1), ("many", 3)])
def test_a_step_replays_while_sequences_come_and_go(dtype, kind, n):
    """Room, store and attention of a step in one graph; between replays slots are forked and emptied, the groups' arrays changed, other work done eagerly."""
    B, nq, nkv, d, max_seq = 24, 8, 2, 64, 200000
    cache = kv8.Kv8Cache(1, nq, nkv, d, B, max_seq, "e4m3", n_pages=300, device=DEV)
    book = kv8.Kv8Pages(cache)
    g = torch.Generator(device=DEV).manual_seed(9)
    lens, counts = ints([0] * B), ints([n] * B)
    first = torch.randn(1, 330, nkv, d, generator=g, device=DEV)
    book.sssd_kv8_reserve(330, lens[:1].contiguous())
    cache.sssd_kv8_append(0, first, first, lens[:1].contiguous())
    lens[0] = 330
    who = [0] * (B - 3) + [-1] * 3
    book.sssd_kv8_fork(ints(who), lens)
    counts[B - 3:] = 0
    groups = 4
    starts, said, workspace = ints([0, 8, 16, B - 3, B]), ints([330, 330, 330, 0]), cache.sssd_kv8_shared_workspace(B, n)
    q = torch.zeros(B, n, nq, d, device=DEV, dtype=dtype)
    k, v = (torch.zeros(B, n, nkv, d, device=DEV) for _ in range(2))
    out = torch.zeros_like(q)

    def step():
        book.sssd_kv8_reserve(n, lens, counts)
        cache.sssd_kv8_append(0, k, v, lens, counts=counts)
        cache.sssd_kv8_attention_shared(0, q, lens, out, starts, said, workspace, counts=counts)
    keep = [t.clone() for t in (book.table, book.refs, cache.cache)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t, x in zip((book.table, book.refs, cache.cache), keep):
        t.copy_(x)
    turns = [(None, None), ([b // 2 for b in range(B)], [0, 2, 4, 12, B]), ([0] * B, [0, B, B, B, B]), ([b if b % 5 else -1 for b in range(B)], [0, 0, 0, 0, 0]), (None, None)]
    assert kind == ("few" if B * n * (nq // nkv) <= 32 * groups else "many")
    for turn, (who, at) in enumerate(turns):
        if who is not None:
            book.sssd_kv8_fork(ints(who), lens)
            counts.copy_(ints([0 if o < 0 else n for o in who]))
            starts.copy_(ints(at))
            said.copy_(ints([330] * groups))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        out.fill_(5.5)
        workspace.fill_(MARK)
        graph.replay()
        was, c = lens.tolist(), counts.tolist()
        other = torch.randn(500, 500, device=DEV) @ torch.randn(500, 500, device=DEV)
        assert other.isfinite().all() and cache.sssd_kv8_sync() == sv.SSSD_OK, turn
        assert not bool((workspace == MARK).all())
        total = max(a + m for a, m in zip(was, c))
        kk, vv = (torch.zeros(B, total, nkv, d, device=DEV) for _ in range(2))
        cache.sssd_kv8_read(0, None, ints([a + m for a, m in zip(was, c)]), kk, vv)
        for b in range(B):
            assert (out[b, c[b]:] == 5.5).all()
            if c[b]:
                want, mass, most = attend(q[b], kk[b, :was[b] + n].double(), vv[b, :was[b] + n].double(), was[b])
                bound = mass * (2 * most * (2.0 ** -22 + 256 * 2.0 ** -24) + 2.0 ** -20)
                if dtype == torch.bfloat16:
                    bound = bound + mass * 2.0 ** -11 + (want.abs() + bound) * torch.finfo(torch.bfloat16).eps / 2
                assert ((out[b].double() - want).abs() <= bound).all(), (turn, b)
        lens += counts


def test_sequences_by_themselves(no_room):
    """Short prefixes, and batches whose rows fill the chip as they are: nothing to join, the workspace is left alone.  The last has more workgroups than the chip holds at once."""
    for heads, groups, own, n in (((8, 2, 64), [(6, 500)], [7, 90], 3), ((4, 2, 64), [(4, 512)], [33], 1), ((64, 8, 128), [(64, 320)], [3], 9)):
        batch = Batch("e4m3", *heads, groups, own, n)
        out, went = way(batch, lambda: batch.check(torch.float32))
        assert went == "apart", (heads, groups, n)
