"""sssd_kv8_attention against 64 bits on the values that the cache holds (tests/kv8_reference.py).

Bounds.  float32: q and the probabilities are held to 22 bits, codes exactly; products are summed in 32 bits, 2 * 128 terms a score.  With
S the largest sum |q_i k_i| / sqrt(d) of a row, its scores are off by at most e = S (2^-22 + 256 * 2^-24), its probabilities by a factor
exp(2e), each output by sum(p |v|) * (2 e + 2^-20) (exp2, probabilities, sums and the joining of segments: 16 roundings).  That is the worst
case for every element; roundings are independent, so the 2-norm of all errors is held to 4e-6 of the result's (three sources of 2^-23 each of
scores of up to ten).  bf16: probabilities to 11 bits (half a step, 2^-11, of sum(p |v|)) and one rounding of the output."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from kv8_reference import Cache, attend
from paper_2411_05894_amd import kv8
from paper_2411_05894_amd.binding import SSSD_ENOSPACE, SSSD_OK

DEV = "cuda:0"


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def random_parents(n, seed):
    g = torch.Generator().manual_seed(seed)
    return [0] + [int(torch.randint(0, j, (1,), generator=g)) for j in range(1, n)]


class Batch:
    """A filled cache and what it holds."""

    def __init__(self, fmt, nq, nkv, d, lens, n, counts=None, paged=False, seed=1, spread=1.0, extra=0, cut=None, long=False):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.B, self.n, self.lens, self.counts = len(lens), n, lens, counts or [n] * len(lens)
        max_seq = max(lens) + n + extra
        if long:                       # room for sequences so long that the queries go through the cache several tiles at a time
            max_seq += 32 * (3500 // (self.B * nkv) + 1)
        self.cache = kv8.Kv8Cache(2, nq, nkv, d, self.B, max_seq, fmt, device=DEV)
        if paged:
            t = torch.randperm(self.cache.n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
            self.cache.sssd_kv8_set_block_table(t.view(self.B, -1).to(DEV))
        rows = max(lens) + n
        k, v = (torch.randn(self.B, rows, nkv, d, generator=g, device=DEV) * spread for _ in range(2))
        k[..., ::29] *= 5
        if cut is not None:            # values of very different sizes along the sequence
            v *= torch.exp2(((torch.arange(rows, device=DEV) // cut) % 5 - 2).float() * 6)[:, None, None]
        total = [a + c for a, c in zip(lens, self.counts)]
        self.cache.sssd_kv8_append(1, k, v, torch.zeros(self.B, dtype=torch.int32, device=DEV), counts=ints(total))
        assert self.cache.sssd_kv8_sync() == SSSD_OK
        self.held = []
        for b in range(self.B):
            pair = []
            for x in (k, v):
                c = Cache(nkv, d, fmt, DEV)
                c.append(0, x[b, :total[b]])
                pair.append(c.x)
            self.held.append(pair)
        self.q = torch.randn(self.B, n, nq, d, generator=g, device=DEV)

    def check(self, dtype, parents=None, window=0, sinks=0, q=None):
        q = (self.q if q is None else q).to(dtype)
        out = torch.full(q.shape, 5.5, dtype=dtype, device=DEV)
        self.cache.sssd_kv8_attention(1, q, ints(self.lens), out, counts=None if self.counts == [self.n] * self.B else ints(self.counts),
                                      parents=ints(parents) if parents else None, window=window, sinks=sinks)
        assert self.cache.sssd_kv8_sync() == SSSD_OK
        off = size = 0.0
        for b in range(self.B):
            c = self.counts[b]
            assert (out[b, c:] == 5.5).all()
            if not c:
                continue
            want, mass, most = attend(q[b, :c], *self.held[b], self.lens[b], parents[b] if parents else None, window, sinks)
            e = most * (2.0 ** -22 + 256 * 2.0 ** -24)
            bound = mass * (2 * e + 2.0 ** -20)
            if dtype == torch.bfloat16:
                bound = bound + mass * 2.0 ** -11 + (want.abs() + bound) * torch.finfo(torch.bfloat16).eps / 2
            err = (out[b, :c].double() - want).abs()
            assert (err <= bound).all(), (b, float((err / bound).max()))
            off, size = off + float((err ** 2).sum()), size + float((want ** 2).sum())
        if dtype == torch.float32:
            assert off <= (4e-6) ** 2 * size, (off / size) ** 0.5
        return out


SHAPES = [(4, 2, 64), (32, 8, 128), (8, 1, 64), (6, 6, 128), (64, 8, 128), (64, 1, 128)]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("nq,nkv,d", SHAPES)
@pytest.mark.parametrize("long", [False, True])
def test_lengths(fmt, dtype, nq, nkv, d, long):
    """From an empty context to several segments, ends inside and at blocks, ragged and padded."""
    for lens, n, counts, paged in (([0], 1, None, False), ([0, 1, 31, 32, 33], 2, [2, 1, 2, 0, 2], True), ([255, 256, 257, 7], 5, None, False),
                                   ([1000, 3, 4100], 9, [9, 7, 9], True), ([2047], 9, None, False), ([70, 600], 32, [32, 17], False)):
        print(f"kv8 attention {fmt} {dtype} {nq}/{nkv}x{d} {lens} {n} {long}", flush=True)
        Batch(fmt, nq, nkv, d, lens, n, counts, paged, long=long).check(dtype)


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (32, 8, 128)])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("long", [False, True])
def test_every_number_of_rows(fmt, nq, nkv, d, long):
    """1 .. 32 new rows: row tiles and passes of every size, chains and trees."""
    batch = Batch(fmt, nq, nkv, d, [37, 300], 32, seed=2, long=long)
    full, held = batch.q, batch.held
    for n in range(1, 33):
        batch.n, batch.counts, batch.q = n, [n] * 2, full[:, :n].contiguous()
        batch.held = [[x[:a + n] for x in pair] for a, pair in zip(batch.lens, held)]
        batch.check(torch.float32 if n % 2 else torch.bfloat16, [random_parents(n, 10 * n + b) for b in range(2)] if n % 3 == 0 else None)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 3), (7, 0), (31, 40), (32, 4), (33, 33), (64, 5), (300, 0), (1000, 64), (5000, 4), (17, 5000), (2**31 - 1, 2**31 - 1)])
@pytest.mark.parametrize("tree", [False, True])
def test_windows(window, sinks, tree):
    """Windows shorter than the step, ending inside blocks, longer than the context; first positions that overlap the window."""
    for fmt, nq, nkv, d, dtype in (("e4m3", 8, 2, 64, torch.float32), ("int8", 8, 1, 128, torch.bfloat16), ("int8", 4, 4, 128, torch.float32)):
        lens, n = [0, 5, 63, 500, 2300], 13
        batch = Batch(fmt, nq, nkv, d, lens, n, [13, 13, 12, 13, 5], paged=True, seed=3)
        print(f"kv8 window {window} {sinks} {fmt} {dtype}", flush=True)
        batch.check(dtype, [random_parents(n, b) for b in range(5)] if tree else None, window, sinks)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_wide_windows(dtype):
    """Windows of many blocks over several sequences, whose queries go through the cache several tiles at a time."""
    for nq, n, window, sinks in ((32, 9, 6000, 4), (64, 13, 5999, 100)):
        Batch("int8", nq, 8, 128, [9000, 6003, 7777], n, [n, n, 3], seed=18).check(dtype, [random_parents(n, b) for b in range(3)], window, sinks)


def test_rows_outside_the_window_are_not_read():
    """Pages that no row can see may be anything: here they are not in the pool's live part at all."""
    batch = Batch("e4m3", 4, 2, 64, [1500], 4, seed=4)
    a = batch.check(torch.float32, window=100, sinks=3)
    t = torch.arange(batch.cache.n_pages, dtype=torch.int32).view(1, -1)
    t[0, 1:40] = 10 ** 6
    batch.cache.sssd_kv8_set_block_table(t.to(DEV))
    b = batch.check(torch.float32, window=100, sinks=3)
    assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_values_of_many_sizes(fmt):
    """V blocks whose scales differ by up to 2^24 in either order, and tiny and huge keys and queries."""
    Batch(fmt, 4, 2, 64, [1200, 33], 5, seed=5, cut=100).check(torch.float32)
    Batch(fmt, 4, 2, 64, [700], 5, seed=6, spread=1e-6).check(torch.float32)
    big = Batch(fmt, 4, 2, 64, [700], 5, seed=6, spread=1e3)
    big.check(torch.float32, q=big.q * 1e-3)
    wide = Batch(fmt, 4, 2, 64, [700], 5, seed=7)
    q = wide.q.clone()
    q[0, 0], q[0, 1], q[0, 2, 0], q[0, 3] = 0, q[0, 1] * 1e-30, q[0, 2, 0] * 1e-41, q[0, 3] * 3.0
    wide.check(torch.float32, q=q)


def test_a_sharp_and_a_flat_softmax():
    """Maxima that grow along the context by far more than the reference's slack, and all scores the same."""
    batch = Batch("int8", 2, 1, 64, [2000], 1, seed=8)
    cache, d = batch.cache, 64
    rows = 2001
    k = torch.zeros(1, rows, 1, d, device=DEV)
    k[0, :, 0, 0] = torch.linspace(-100, 100, rows, device=DEV)
    v = torch.randn(1, rows, 1, d, device=DEV)
    for kk in (k, k.flip(1), torch.zeros_like(k)):
        kk = kk.contiguous()
        cache.sssd_kv8_append(1, kk, v, ints([0]))
        held = []
        for x in (kk, v):
            c = Cache(1, d, "int8", DEV)
            c.append(0, x[0])
            held.append(c.x)
        batch.held = [held]
        q = torch.zeros(1, 1, 2, d, device=DEV)
        q[..., 0] = 16.0
        batch.check(torch.float32, q=q)


def extreme(keys, channel, q, dtype):
    """One head whose keys are `keys` in one channel; -> (out, want, sum of p |v|)."""
    d, n = 64, 4
    rows = len(keys)
    cache = kv8.Kv8Cache(1, 2, 1, d, 1, rows, "e4m3", device=DEV)
    k, v = torch.zeros(1, rows, 1, d, device=DEV), torch.randn(1, rows, 1, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(17))
    k[0, :, 0, channel] = torch.tensor(keys, device=DEV)
    cache.sssd_kv8_append(0, k, v, ints([0]))
    kk, vv = torch.empty_like(k), torch.empty_like(v)
    cache.sssd_kv8_read(0, None, None, kk, vv)
    assert torch.equal(kk, k)                      # the keys are codes
    qq = torch.zeros(1, n, 2, d, device=DEV)
    qq[..., 0] = torch.tensor(q, device=DEV)
    qq = qq.to(dtype)
    out = torch.zeros_like(qq)
    cache.sssd_kv8_attention(0, qq, ints([rows - n]), out)
    assert cache.sssd_kv8_sync() == SSSD_OK
    want, mass, _ = attend(qq[0], kk[0].double(), vv[0].double(), rows - n)
    return out[0].double(), want, mass


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_scores_of_every_magnitude(dtype):
    """Neighbouring keys are a sixteenth of the largest apart, so with scores of 2^11 and more only the largest count, and these are equal: the result is
    their values' mean, off by the 16 roundings of 2^-24 of the bound above and by those of bf16.  With scores of 0, from whatever scales, it is the
    mean of all that is seen."""
    bound = 2.0 ** -20 if dtype == torch.float32 else 2.0 ** -20 + 2.0 ** -11 + torch.finfo(dtype).eps / 2 * (1 + 2.0 ** -10)
    for sign in (1.0, -1.0):
        for size in (2.0 ** 10, 2.0 ** 50, 2.0 ** -60):
            keys = [sign * size * (1 + (7 * i) % 16) for i in range(300)]
            for score in (2.0 ** 11, 2.0 ** 20, 2.0 ** 24, 2.0 ** 27, 2.0 ** 28, 2.0 ** 29, 2.0 ** 32, 2.0 ** 50, 1.0e30, 1.0e34):
                q = score / size * 1.2345678
                if not 1e-37 < q < 1e37:
                    continue
                out, want, mass = extreme(keys, 0, q, dtype)
                assert ((out - want).abs() <= bound * mass).all(), (sign, size, score)
    for q, size in ((1e-30, 2.0 ** -120), (2e-38, 2.0 ** -126), (1e38, 2.0 ** 126), (1e38, 2.0 ** -126), (1e-37, 2.0 ** 126), (1e-41, 1.0)):
        out, want, mass = extreme([size * (1 + i % 2) for i in range(75)], 1, q, dtype)
        assert ((out - want).abs() <= bound * mass).all(), (q, size)
    for q, size in ((1e-30, 2.0 ** -120), (2e-38, 2.0 ** -126)):
        out, want, mass = extreme([size * (1 + i % 2) for i in range(75)], 0, q, dtype)
        assert ((out - want).abs() <= bound * mass).all(), (q, size)


def test_numbers_that_are_none():
    """A row of q that is no number spoils its own output alone; the rows that follow a sequence in its last block, and whole pages that nobody
    owns, may hold anything."""
    batch = Batch("e4m3", 4, 2, 64, [90, 41], 3, seed=9, extra=64)
    clean = batch.check(torch.float32)
    q = batch.q.clone()
    q[0, 1, 2, 5] = float("nan")
    q[1, 0, 0, 0] = float("inf")
    out = torch.zeros_like(q)
    batch.cache.sssd_kv8_attention(1, q, ints(batch.lens), out)
    assert not out[0, 1, 2].isfinite().any() and not out[1, 0, 0].isfinite().any()
    out[0, 1, 2], out[1, 0, 0] = clean[0, 1, 2], clean[1, 0, 0]
    assert torch.equal(out, clean)
    page = 2 * 64 * 64
    codes = batch.cache.cache[batch.cache.cache.numel() // 2:]       # layer 1
    per_seq = batch.cache.blocks_per_seq
    for b, last in ((0, 92 // 32), (1, 43 // 32)):
        codes[(b * per_seq + last + 1) * page:(b + 1) * per_seq * page] = 0x7F      # e4m3: no number
    out = torch.zeros_like(clean)
    batch.cache.sssd_kv8_attention(1, batch.q, ints(batch.lens), out)
    assert torch.equal(out, clean)


def test_strides_and_neighbours():
    """Queries and outputs in the middle of wider rows, at odd addresses, heads before rows; what lies beside them stays."""
    batch = Batch("int8", 8, 2, 64, [200, 77], 6, [6, 4], seed=10)
    for dtype in (torch.float32, torch.bfloat16):
        want = batch.check(dtype)
        q = batch.q.to(dtype)
        wide = torch.full((2, 6, 11, 64), 2.25, dtype=dtype, device=DEV)
        wide[:, :, 1:9] = q
        into = torch.full((2, 6, 11, 64), 5.5, dtype=dtype, device=DEV)
        batch.cache.sssd_kv8_attention(1, wide[:, :, 1:9], ints(batch.lens), into[:, :, 2:10], counts=ints(batch.counts))
        assert torch.equal(into[:, :, 2:10], want) and (into[:, :, :2] == 5.5).all() and (into[:, :, 10:] == 5.5).all()
        odd_q, odd_out = (torch.full((2 * 6 * 8 * 64 + 1,), 5.5, dtype=dtype, device=DEV)[1:].view(2, 6, 8, 64) for _ in range(2))
        odd_q.copy_(q)
        batch.cache.sssd_kv8_attention(1, odd_q, ints(batch.lens), odd_out, counts=ints(batch.counts))
        assert torch.equal(odd_out, want)
        by_head = q.transpose(1, 2).contiguous().transpose(1, 2)
        out = torch.full((2, 8, 6, 64), 5.5, dtype=dtype, device=DEV).transpose(1, 2)
        batch.cache.sssd_kv8_attention(1, by_head, ints(batch.lens), out, counts=ints(batch.counts))
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("long", [False, True])
def test_the_other_sequences_change_no_bit(dtype, long):
    a = Batch("e4m3", 32, 8, 128, [1500, 90, 3000], 5, seed=11, long=long)
    first = a.check(dtype)
    k = torch.randn(1, 60, 8, 128, device=DEV)
    for b in (1, 2):
        a.cache.sssd_kv8_append(1, k, k, ints([0]), first=b)
    out = torch.zeros_like(first)
    a.cache.sssd_kv8_attention(1, a.q.to(dtype), ints([1500, 40, 55]), out, counts=ints([5, 2, 5]))
    assert torch.equal(out[0], first[0]) and not torch.equal(out[2], first[2])
    for _ in range(20):
        again = torch.zeros_like(first)
        a.cache.sssd_kv8_attention(1, a.q.to(dtype), ints([1500, 40, 55]), again, counts=ints([5, 2, 5]))
        assert torch.equal(again, out)


@pytest.mark.parametrize("what", ["negative", "long", "count", "negative_count"])
def test_rejected_sequences_give_zeros(what):
    batch = Batch("int8", 8, 2, 64, [200, 77, 150], 6, seed=12)
    want = batch.check(torch.float32)
    lens, counts = list(batch.lens), [6, 6, 6]
    if what == "negative":
        lens[1] = -5
    if what == "long":
        lens[1] = 201
    if what == "count":
        counts[1] = 7
    if what == "negative_count":
        counts[1] = -1
    out = torch.full_like(want, 5.5)
    batch.cache.sssd_kv8_attention(1, batch.q, ints(lens), out, counts=ints(counts))
    assert batch.cache.sssd_kv8_sync() == SSSD_ENOSPACE and batch.cache.sssd_kv8_sync() == SSSD_OK
    assert torch.equal(out[[0, 2]], want[[0, 2]]) and (out[1] == 0).all()


def test_a_page_outside_the_pool_is_reported():
    batch = Batch("int8", 8, 2, 64, [200, 77], 6, seed=13, paged=True)
    want = batch.check(torch.float32)
    t = batch.cache._block_table.clone()
    for wrong in (batch.cache.n_pages, -1, 2**31 - 1, -2**31):
        t[1, 1] = wrong
        batch.cache.sssd_kv8_set_block_table(t)
        out = torch.zeros_like(want)
        batch.cache.sssd_kv8_attention(1, batch.q, ints(batch.lens), out)
        assert batch.cache.sssd_kv8_sync() == SSSD_ENOSPACE
        assert torch.equal(out[0], want[0])


def test_bad_parents_are_taken_as_the_row_before():
    batch = Batch("e4m3", 8, 2, 64, [40], 6, seed=14)
    good = batch.check(torch.float32, [[0, 0, 1, 2, 3, 3]])
    out = torch.zeros_like(good)
    batch.cache.sssd_kv8_attention(1, batch.q, ints([40]), out, parents=ints([[0, 0, 7, -1, 4, 3]]))
    assert batch.cache.sssd_kv8_sync() == SSSD_ENOSPACE
    assert torch.equal(out, good)


def test_many_sequences_and_a_long_one():
    """More sequences than compute units, and one of 70001 positions."""
    Batch("int8", 8, 2, 64, [(37 * b) % 200 for b in range(300)], 2, seed=15).check(torch.bfloat16)
    Batch("e4m3", 16, 2, 128, [70001], 3, seed=16).check(torch.float32)


def test_pages_behind_four_gib():
    pages = 5 * (1 << 30) // (8 * 64 * 128)
    cache = kv8.Kv8Cache(1, 8, 8, 128, 1, 96, "e4m3", n_pages=pages, device=DEV)
    small = kv8.Kv8Cache(1, 8, 8, 128, 1, 96, "e4m3", device=DEV)
    cache.sssd_kv8_set_block_table(ints([[pages - 1, 0, pages - 2]]))
    x, q = torch.randn(1, 80, 8, 128, device=DEV), torch.randn(1, 4, 8, 128, device=DEV)
    outs = []
    for c in (cache, small):
        c.sssd_kv8_append(0, x, x, ints([0]))
        outs.append(torch.zeros_like(q))
        c.sssd_kv8_attention(0, q, ints([76]), outs[-1])
    assert torch.equal(*outs)


@pytest.mark.parametrize("nq,nkv,d,B,n", [
    (32, 8, 128, 4, 9), (32, 8, 128, 2, 32), (64, 8, 128, 2, 9), (64, 8, 128, 7, 13), (64, 8, 128, 1, 1), (32, 8, 128, 33, 5),   # one pass and several, four and eight waves
    (64, 8, 64, 3, 9), (16, 2, 64, 1, 7), (16, 2, 128, 3, 7), (24, 8, 128, 5, 5), (48, 8, 64, 20, 6)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("long", [False, True])
def test_plans(nq, nkv, d, B, n, dtype, long):
    """Passes, row tiles, waves and segments of every kind, segments joined inside the launch and by a second one; those joined without waiting give
    the same bits."""
    lens = [(1700 * (b + 1)) % 2300 + (b == 0) * 1500 for b in range(B)]
    batch = Batch("int8" if n % 2 else "e4m3", nq, nkv, d, lens, n, paged=True, seed=n, long=long)
    print(f"kv8 plan {nq}/{nkv}x{d} B {B} n {n} {dtype} {long}", flush=True)
    want = batch.check(dtype)
    batch.cache.args.flags = 2       # SSSD_NO_WAIT
    for _ in range(3):
        assert torch.equal(batch.check(dtype), want)
    batch.cache.args.flags = 0
    assert torch.equal(batch.check(dtype), want)
