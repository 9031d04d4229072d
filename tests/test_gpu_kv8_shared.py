"""sssd_kv8_attention_shared against 64 bits on the values that the cache holds (tests/kv8_reference.py), sequence by sequence.

Bounds: those of sssd_kv8_attention (tests/test_gpu_kv8_attention.py says where they come from): with S the largest sum |q_i k_i| / sqrt(d) of a row, its scores
are off by at most e = S (2^-22 + 256 * 2^-24), and each output by sum(p |v|) * (2 e + 2^-20); the joining of prefix and rest is that of segments.  bf16: probabilities to 11
bits (half a step, 2^-11, of sum(p |v|)) and one rounding of the output."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from kv8_reference import attend
from paper_2411_05894_amd import kv8
from paper_2411_05894_amd.binding import SSSD_ENOSPACE, SSSD_NO_WAIT, SSSD_OK, SssdError

DEV = "cuda:0"
LONGER = 0      # positions that a sequence could have beyond what the batch needs


@pytest.fixture(autouse=True, params=["as long as they are", "room for more"])
def room(request):
    """How long sequences can be decides whether short prefixes are read for all rows of a group at once or by each sequence: both have to be right."""
    global LONGER
    LONGER = 0 if request.param == "as long as they are" else 200000


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def random_parents(n, seed):
    g = torch.Generator().manual_seed(seed)
    return [0] + [int(torch.randint(0, j, (1,), generator=g)) for j in range(1, n)]


class Batch:
    """Groups of sequences forked from one that holds their prefix, each with rows of its own; `alone`: sequences behind them in no group."""

    def __init__(self, fmt, nq, nkv, d, groups, own, n, alone=0, counts=None, seed=1, extra=0, spread=1.0, scales=None, layers=1):
        """groups: [(sequences, positions of the prefix)]; own: rows before the new ones, of sequence b own[b % len]."""
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.B = B = sum(m for m, _ in groups) + alone
        self.n, self.nq = n, nq
        front = [p for m, p in groups for _ in range(m)] + [0] * alone
        self.own = [own[b % len(own)] for b in range(B)]
        self.lens = [a + b for a, b in zip(front, self.own)]
        self.counts = counts or [n] * B
        longest = max(self.lens) + n + extra
        max_seq = longest + LONGER
        pages = sum((p + 31) // 32 for _, p in groups) + sum((a + n + 31) // 32 + 1 for a in self.own) + 3
        self.cache = kv8.Kv8Cache(layers, nq, nkv, d, B, max_seq, fmt, n_pages=pages, device=DEV)
        self.book = kv8.Kv8Pages(self.cache)
        starts, origins, lens = [0], list(range(B)), [0] * B
        self.layer = layers - 1

        def rows(count, length):
            k, v = (torch.randn(count, length, nkv, d, generator=g, device=DEV) * spread for _ in range(2))
            k[..., ::29] *= 5
            if scales is not None:      # V of very different sizes along the sequence
                v *= torch.exp2(torch.tensor([float(scales[(i // 100) % len(scales)]) for i in range(length)], device=DEV))[:, None, None]
            return k, v
        for m, p in groups:
            at = starts[-1]
            if p:
                k, v = rows(1, p)
                self.book.sssd_kv8_reserve(p, ints([0]), first=at)
                self.cache.sssd_kv8_append(self.layer, k, v, ints([0]), first=at)
            lens[at] = p
            origins[at:at + m] = [at] * m
            starts.append(at + m)
        self.d_lens = ints(lens)
        self.book.sssd_kv8_fork(ints(origins), self.d_lens)
        total = max(a + c for a, c in zip(self.own, self.counts))
        fill = ints([a + c for a, c in zip(self.own, self.counts)])
        k, v = rows(B, max(total, 1))
        self.book.sssd_kv8_reserve(max(total, 1), self.d_lens, fill)
        self.cache.sssd_kv8_append(self.layer, k, v, self.d_lens, counts=fill)
        assert self.cache.sssd_kv8_sync() == SSSD_OK
        self.starts, self.shared = starts, [p for _, p in groups]
        self.q = torch.randn(B, n, nq, d, generator=g, device=DEV)
        held = [torch.zeros(B, longest, nkv, d, device=DEV) for _ in range(2)]
        self.cache.sssd_kv8_read(self.layer, None, ints([a + c for a, c in zip(self.lens, self.counts)]), *held)
        self.held = held
        self.workspace = self.cache.sssd_kv8_shared_workspace(B, n)

    def run(self, q, out, parents=None, starts=None, shared=None, lens=None):
        self.cache.sssd_kv8_attention_shared(self.layer, q, ints(lens or self.lens), out, ints(starts or self.starts), ints(self.shared if shared is None else shared),
                                             self.workspace, counts=None if self.counts == [self.n] * self.B else ints(self.counts),
                                             parents=ints(parents) if parents else None)

    def compare(self, b, q, out, parents=None):
        """(squared error, squared size) of sequence b, within its bounds."""
        c = self.counts[b]
        assert (out[b, c:] == 5.5).all()
        if not c:
            return 0.0, 0.0
        total = self.lens[b] + c
        want, mass, most = attend(q[b, :c], self.held[0][b, :total].double(), self.held[1][b, :total].double(), self.lens[b], parents[b] if parents else None)
        bound = mass * (2 * most * (2.0 ** -22 + 256 * 2.0 ** -24) + 2.0 ** -20)
        if q.dtype == torch.bfloat16:
            bound = bound + mass * 2.0 ** -11 + (want.abs() + bound) * torch.finfo(torch.bfloat16).eps / 2
        err = (out[b, :c].double() - want).abs()
        assert (err <= bound).all(), (b, float((err / bound).max()))
        return float((err ** 2).sum()), float((want ** 2).sum())

    def check(self, dtype, parents=None, q=None, **how):
        q = (self.q if q is None else q).to(dtype)
        out = torch.full(q.shape, 5.5, dtype=dtype, device=DEV)
        self.run(q, out, parents, **how)
        assert self.cache.sssd_kv8_sync() == SSSD_OK
        sums = [self.compare(b, q, out, parents) for b in range(self.B)]
        if dtype == torch.float32:
            assert sum(x for x, _ in sums) <= (4e-6) ** 2 * sum(y for _, y in sums)
        return out


SHAPES = [(4, 2, 64), (32, 8, 128), (8, 1, 64), (6, 6, 128), (64, 8, 128), (64, 1, 128)]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("nq,nkv,d", SHAPES)
def test_groups(fmt, dtype, nq, nkv, d):
    """Prefixes from less than a block to several segments, ends inside and at blocks, groups of one to many, sequences in none, padded rows."""
    for groups, own, n, alone, counts in (([(2, 32)], [0], 1, 0, None), ([(3, 31)], [1, 0, 33], 2, 0, [2, 1, 0]), ([(4, 100), (1, 70), (2, 64)], [5, 40, 0], 5, 2, None),
                                          ([(9, 700)], [3, 100, 31, 32], 9, 1, [9, 8, 7, 9, 9, 1, 0, 9, 9, 4]), ([(2, 33), (5, 1500)], [300, 2], 3, 0, None),
                                          ([(17, 2048), (8, 320)], [60, 64, 1], 1, 3, None)):
        print(f"kv8 shared {fmt} {dtype} {nq}/{nkv}x{d} {groups} {own} {n}", flush=True)
        Batch(fmt, nq, nkv, d, groups, own, n, alone, counts).check(dtype)


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (32, 8, 128)])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_every_number_of_rows(fmt, nq, nkv, d):
    """1 .. 32 new rows of groups of several sizes: waves' row tiles and segments of every kind, chains and trees."""
    for n in range(1, 33):
        for groups in ([(1 + n % 4, 96 + 32 * n), (2 + n // 3, 257)], [(3, 320)]):
            batch = Batch(fmt, nq, nkv, d, groups, [n, 37], n, seed=n)
            batch.check(torch.float32 if n % 2 else torch.bfloat16, [random_parents(n, 10 * n + b) for b in range(batch.B)] if n % 3 == 0 else None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_sequences_and_groups(dtype):
    Batch("int8", 4, 2, 64, [(2, 64 + 32 * (i % 3)) for i in range(70)], [3, 1, 40], 2, 5).check(dtype)      # more groups than a wave has lanes
    Batch("e4m3", 32, 8, 128, [(150, 320)], [3, 1], 1).check(dtype)
    Batch("e4m3", 8, 8, 128, [(40, 4096), (23, 64)], [20, 3], 4).check(dtype)
    Batch("int8", 8, 2, 64, [(6, 20000)], [5], 3).check(dtype)                                               # segments that a chunk of pages does not cover


def test_what_is_shared_may_be_said_in_less():
    """Fewer positions than are the same, other groups of the same sequences, none: the same results but for the order of sums."""
    batch = Batch("e4m3", 8, 2, 64, [(6, 500)], [7, 90], 3)
    outs = [batch.check(torch.float32), batch.check(torch.float32, shared=[499]), batch.check(torch.float32, shared=[40]), batch.check(torch.float32, shared=[31]),
            batch.check(torch.float32, starts=[0, 2, 6], shared=[500, 256]), batch.check(torch.float32, starts=[1, 5], shared=[480]),
            batch.check(torch.float32, starts=[2, 3, 3, 6], shared=[500, 500, 64]), batch.check(torch.float32, starts=[6], shared=[])]
    plain = torch.full_like(outs[0], 5.5)
    batch.cache.sssd_kv8_attention(0, batch.q, ints(batch.lens), plain)
    for o in outs:
        assert (o - plain).abs().max() <= 1e-5 * plain.abs().max()


def test_a_call_repeats_its_bits():
    batch = Batch("int8", 32, 8, 128, [(5, 1000), (12, 300)], [7, 90], 3)
    a, b = batch.check(torch.float32), batch.check(torch.float32)
    assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_of_many_sizes(fmt, dtype):
    """V blocks up to 2^24 apart, in prefix and rest; prefix and rest far apart; tiny and huge queries."""
    Batch(fmt, 4, 2, 64, [(4, 1200)], [300, 5], 3, scales=[-12, -6, 0, 6, 12], seed=5).check(dtype)
    Batch(fmt, 8, 1, 128, [(7, 1200)], [200, 5], 5, scales=[12, -12], seed=6).check(dtype)
    Batch(fmt, 4, 2, 64, [(3, 300)], [5], 3, spread=1e-6, seed=7).check(dtype)
    wide = Batch(fmt, 4, 2, 64, [(3, 300)], [50], 4, seed=8)
    q = wide.q.clone()
    q[0, 0], q[0, 1], q[1, 2, 0], q[2, 3] = 0, q[0, 1] * 1e-30, q[1, 2, 0] * 1e-41, q[2, 3] * 3.0
    wide.check(dtype, q=q)


def test_a_row_that_is_no_number_spoils_itself_alone():
    batch = Batch("e4m3", 8, 2, 64, [(5, 300)], [7, 90], 3)
    good = batch.check(torch.float32)
    q = batch.q.clone()
    q[1, 1, 3, 5], q[4, 0, 0, 0] = float("nan"), float("inf")
    out = torch.full_like(q, 5.5)
    batch.run(q, out)
    spoilt = torch.zeros(q.shape[:3], dtype=torch.bool, device=DEV)
    spoilt[1, 1, 3] = spoilt[4, 0, 0] = True
    assert torch.equal(out[~spoilt], good[~spoilt])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sequences", [1, 2, 9, 40])
def test_scores_of_every_magnitude(dtype, sequences):
    """Neighbouring keys are a sixteenth of the largest apart, so with scores of 2^11 and more only the largest count, and these are equal: the mean of their values, wherever they
    lie -- in the prefix, behind it, in both."""
    d, prefix, own, n = 64, 160, 33, 2
    for where in ("prefix", "own", "both"):
        batch = Batch("e4m3", 4, 2, d, [(max(sequences, 2), prefix)], [own], n, alone=1 if sequences == 1 else 0, seed=11)
        cache, B = batch.cache, batch.B
        g = torch.Generator(device=DEV).manual_seed(12)
        k = torch.zeros(B, prefix + own + n, 2, d, device=DEV)
        steps = torch.randint(0, 8, (prefix + own + n,), generator=g, device=DEV).float()
        top = {"prefix": [3, 77], "own": [prefix + 2, prefix + 30], "both": [5, prefix + 4]}[where]
        steps[::32] = 8.0                                     # every block has the same scale
        steps[top] = 9.0
        k[..., 0] = (steps / 16.0 + 0.375)[None, :, None]
        v = torch.randn(B, prefix + own + n, 2, d, generator=g, device=DEV)
        v[:, :prefix] = v[:1, :prefix]
        for first, end, lens in ((0, prefix, [0] * B), (prefix, prefix + own + n, batch.lens)):
            at = [0] if first == 0 else list(range(B))
            for b in at:
                if first and batch.lens[b] < prefix:          # the one that shares nothing
                    continue
                cache.sssd_kv8_append(0, k[b:b + 1, first:end].contiguous(), v[b:b + 1, first:end].contiguous(), ints([first]), first=b)
        kk, vv = (torch.zeros_like(k) for _ in range(2))
        cache.sssd_kv8_read(0, None, ints([a + n for a in batch.lens]), kk, vv)
        for size in (1e3, 1e6, 1e20, 1e34):
            q = torch.zeros(B, n, 4, d, device=DEV)
            q[..., 0] = torch.tensor([size, -size * 0.5, size * 3, size * 0.25], device=DEV)
            q = q.to(dtype)
            out = torch.full_like(q, 5.5)
            batch.run(q, out)
            for b in range(B):
                if batch.lens[b] < prefix:
                    continue
                total = batch.lens[b] + n
                want, mass, _ = attend(q[b], kk[b, :total].double(), vv[b, :total].double(), batch.lens[b])
                bound = mass * 2.0 ** -20 + (want.abs() * 2.0 ** -8 + mass * 2.0 ** -10 if dtype == torch.bfloat16 else 0)
                bad = (out[b].double() - want).abs() > bound
                assert not bad.any(), (where, size, b, float(((out[b].double() - want).abs() / bound).max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layouts(dtype):
    """Queries in the middle of a QKV product, outputs heads first, unaligned ones."""
    batch = Batch("int8", 8, 2, 64, [(6, 500), (2, 40)], [7, 90], 3, 1, layers=3)
    want = batch.check(dtype)
    B, n, nq, d = batch.q.shape
    qkv = torch.randn(B, n, nq + 4, d, device=DEV).to(dtype)
    qkv[:, :, :nq] = batch.q.to(dtype)
    heads_first = torch.full((B, nq, n, d), 5.5, dtype=dtype, device=DEV).transpose(1, 2)
    off = torch.full((B, n, nq, d + 1), 5.5, dtype=dtype, device=DEV)[..., 1:]
    for q, out in ((qkv[:, :, :nq], heads_first), (batch.q.to(dtype), off)):
        batch.run(q, out)
        assert torch.equal(out, want)
    wide = torch.zeros(B, n, nq, d + 3, dtype=dtype, device=DEV)[..., 2:d + 2]
    wide.copy_(batch.q.to(dtype))
    out = torch.full_like(want, 5.5)
    batch.run(wide, out)
    assert torch.equal(out, want)


def test_what_is_out_of_range():
    """Arrays that make no sense: nothing is shared, the status raised.  A sequence shorter than what it is said to share, or of a bad length, is set to 0,
    the others of its group are not touched; the first one's length plays no part for them."""
    batch = Batch("e4m3", 8, 2, 64, [(4, 500), (3, 100)], [7, 90], 3)
    q = batch.q
    for starts, shared in (([0, 4, 8], [500, 100]), ([-1, 4, 7], [500, 100]), ([0, 5, 4], [500, 100]), ([0, 4, 7], [-1, 100]), ([0, 4, 7], [500, 10 ** 9]), ([4, 0, 7], [500, 100]),
                           ([0, 4, 2 ** 31 - 1], [500, 100]), ([0, -2 ** 31, 7], [500, 100])):
        out = torch.full_like(q, 5.5)
        batch.run(q, out, starts=starts, shared=shared)
        assert batch.cache.sssd_kv8_sync() == SSSD_ENOSPACE
        for b in range(batch.B):
            batch.compare(b, q, out)
    good = batch.check(torch.float32)
    for who, length in ((0, -5), (2, 479), (1, 10 ** 6), (0, 0), (3, 2 ** 31 - 1)):
        out = torch.full_like(q, 5.5)
        lens = list(batch.lens)
        lens[who] = length
        batch.run(q, out, lens=lens)
        assert batch.cache.sssd_kv8_sync() == SSSD_ENOSPACE
        assert (out[who] == 0).all()
        assert all(torch.equal(out[b], good[b]) for b in range(batch.B) if b != who)
    batch.counts = [3, 0, 3, 2, 1, 3, 3]
    out = torch.full_like(q, 5.5)
    batch.run(q, out)
    assert (out[1] == 5.5).all() and (out[3, 2:] == 5.5).all() and (out[4, 1:] == 5.5).all()
    batch.counts[2] = 4
    batch.run(q, out)
    assert batch.cache.sssd_kv8_sync() == SSSD_ENOSPACE and (out[2] == 0).all()


def test_pages_outside_the_pool():
    """Reported, and made safe; other groups are as they were."""
    batch = Batch("e4m3", 8, 2, 64, [(4, 500), (3, 100)], [7, 90], 3)
    good = batch.check(torch.float32)
    batch.book.table[0, 3] = 10 ** 6
    out = torch.full_like(batch.q, 5.5)
    batch.run(batch.q, out)
    assert batch.cache.sssd_kv8_sync() == SSSD_ENOSPACE and torch.equal(out[4:], good[4:])


def test_workspaces():
    batch = Batch("e4m3", 8, 2, 64, [(4, 500)], [7], 3)
    batch.workspace = torch.empty(batch.workspace.numel() - 256, dtype=torch.uint8, device=DEV)
    with pytest.raises(SssdError):
        batch.run(batch.q, torch.empty_like(batch.q))
    batch.workspace = torch.full((batch.cache.sssd_kv8_shared_workspace(4, 3).numel() // 4,), float("nan"), device=DEV)      # any contents
    batch.check(torch.float32)


@pytest.mark.parametrize("n", [1, 9])
def test_segments_joined_without_waiting(n):
    """The same bits, whoever joins a sequence's segments; and what the call leaves behind in the cache's own workspace serves plain attention."""
    batch = Batch("e4m3", 32, 8, 128, [(4, 2000), (3, 640)], [30, 200], n, 1)
    a = batch.check(torch.float32)
    batch.cache.args.flags = SSSD_NO_WAIT
    b = batch.check(torch.float32)
    batch.cache.args.flags = 0
    assert torch.equal(a, b) and torch.equal(a, batch.check(torch.float32))
    plain = torch.full_like(a, 5.5)
    batch.cache.sssd_kv8_attention(0, batch.q, ints(batch.lens), plain)
    for i in range(batch.B):
        batch.compare(i, batch.q, plain)


def test_replays_and_streams():
    """Two batches captured, replayed on two streams at once with other queries, eager work between."""
    batches = [Batch("e4m3", 32, 8, 128, [(6, 900)], [30, 200], 5, seed=1), Batch("int8", 8, 2, 64, [(3, 64), (9, 300)], [3], 2, seed=2)]
    graphs, keeps = [], []
    for b in batches:
        q, out, args = b.q.clone(), torch.full_like(b.q, 5.5), (ints(b.lens), ints(b.starts), ints(b.shared))

        def call(cache=b.cache, q=q, out=out, args=args, ws=b.workspace):
            cache.sssd_kv8_attention_shared(0, q, args[0], out, args[1], args[2], ws)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            call()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append((graph, stream))
        keeps.append((q, out, args))
    for turn in range(4):
        for b, (q, _, _) in zip(batches, keeps):
            q.copy_(torch.randn(q.shape, generator=torch.Generator(device=DEV).manual_seed(turn), device=DEV))
        torch.cuda.synchronize()
        for graph, stream in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
        Batch("int8", 4, 2, 64, [(2, 64)], [3], 2).check(torch.float32)
        torch.cuda.synchronize()
        for b, (q, out, _) in zip(batches, keeps):
            eager = torch.full_like(out, 5.5)
            b.run(q, eager)
            assert torch.equal(out, eager)
            for i in range(b.B):
                b.compare(i, q, out)
