"""sssd_kv8_attention over blocks of V whose scales lie far apart, against 64 bits on the values that the cache holds.

Keys are +1 or -1 in one channel and 0 in the others, so that a score is one product: of an exact code, and of a query of eight bits.  It is off by the roundings of
its factor, of the product and of the reference, four of 2^-24 of it, so probabilities by a factor exp(2 * 4 * 2^-24 * most) with `most` the largest score; outputs by sum(p |v|) times
that and 2^-20 (exp2, probabilities of 22 bits, sums and the joining of waves and segments: 16 roundings).  Probabilities of blocks whose scales
are within 2^12 of each other are multiples of 2^-32 of the row's largest or less.  bf16: half a step of 11 bits of the probabilities, and of the output."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from kv8_reference import attend
from paper_2411_05894_amd import kv8
from paper_2411_05894_amd.binding import SSSD_OK

DEV = "cuda:0"
ORDERS = ["first", "last", "mixed"]


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def check(fmt, dtype, nq, nkv, d, lens, n, sign, size, q0, room=0, parents=None, window=0, sinks=0, close=False, seed=1, uniform=False, least=0.0):
    """sign, size [B][positions]: of each position's key, and of its V (uniform: up to that size); least: half a step of the smallest results."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, rows = size.shape
    cache = kv8.Kv8Cache(1, nq, nkv, d, B, rows + room, fmt, device=DEV)
    k, v = torch.zeros(B, rows, nkv, d, device=DEV), torch.randn(B, rows, nkv, d, generator=g, device=DEV)
    k[..., 0] = sign.float().to(DEV)[..., None]
    if uniform:
        v = torch.rand(v.shape, generator=g, device=DEV) * 2 - 1
    v = (v.double() * size.to(DEV)[..., None, None]).float()
    cache.sssd_kv8_append(0, k, v, ints([0] * B), counts=ints([a + n for a in lens]))
    kk, vv = torch.empty_like(k), torch.empty_like(v)
    cache.sssd_kv8_read(0, None, ints([a + n for a in lens]), kk, vv)
    q = torch.randn(B, n, nq, d, generator=g, device=DEV).to(torch.bfloat16)     # of what no key has
    q[..., 0] = q0
    q = q.to(dtype)
    out = torch.full(q.shape, 5.5, dtype=dtype, device=DEV)
    cache.sssd_kv8_attention(0, q, ints(lens), out, parents=ints(parents) if parents else None, window=window, sinks=sinks)
    assert cache.sssd_kv8_sync() == SSSD_OK
    for b in range(B):
        total = lens[b] + n
        assert torch.equal(kk[b, :total], k[b, :total])
        want, mass, most = attend(q[b], kk[b, :total].double(), vv[b, :total].double(), lens[b], parents[b] if parents else None, window, sinks)
        bound = mass * (8 * most * 2.0 ** -24 + 2.0 ** -20) + least
        if close:
            bound = bound + 2.0 ** -32 * vv[b, :total].double().abs().sum(0).repeat_interleave(nq // nkv, 0)
        if dtype == torch.bfloat16:
            bound = bound + mass * 2.0 ** -11 + (want.abs() + bound) * torch.finfo(torch.bfloat16).eps / 2
        err = (out[b].double() - want).abs()
        assert (err <= bound).all(), (b, float((err / bound.clamp(min=1e-300)).max()))


def large_blocks(order, B, blocks, seed):
    """Which blocks have the large values: those that waves meet first, or last, or any."""
    if order == "mixed":
        return torch.rand(B, blocks, generator=torch.Generator().manual_seed(seed)) < 0.5
    first = torch.arange(blocks) < blocks // 2
    return (first if order == "first" else ~first).expand(B, blocks).clone()


# a segment of two blocks a wave; whole sequences of one workgroup; passes of one, two and three tiles, four waves and eight
PLANS = [(4, 2, 64, 1, 3, 8, 0), (32, 8, 128, 1, 1, 8, 0), (32, 8, 128, 33, 1, 21, 0), (16, 8, 64, 33, 2, 21, 0), (32, 8, 128, 4, 9, 90, 40000), (64, 8, 128, 4, 5, 40, 40000),
         (64, 8, 128, 2, 13, 40, 40000)]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("nq,nkv,d,B,n,blocks,room", PLANS)
def test_the_weight_lies_on_small_values(fmt, dtype, order, nq, nkv, d, B, n, blocks, room):
    """Large blocks with the same weight, with 2^-14 to 2^-40 of it and with next to none."""
    large = large_blocks(order, B, blocks, blocks).repeat_interleave(32, 1)
    n_last = [blocks * 32 - n] * B
    for gap in ((4, 5, 8, 9, 16, 25, 30, 60) if B * n < 20 else (9, 25, 60)):
        for q0 in (0.0, 40.0, 80.0, 112.0, 640.0) if B * n < 20 else (112.0,):
            print(f"kv8 scales {fmt} {dtype} {nq}/{nkv}x{d} B {B} n {n} {order} 2^{gap} q {q0}", flush=True)
            check(fmt, dtype, nq, nkv, d, n_last, n, torch.where(large, -1.0, 1.0), torch.where(large, 2.0 ** gap, 1.0).double(), q0, room, close=gap <= 12)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("nq,nkv,d,B,n,blocks,room", PLANS[:5])
def test_blocks_of_zeros(fmt, dtype, order, nq, nkv, d, B, n, blocks, room):
    """Their scale is 1, whatever the others' values are."""
    zero = large_blocks(order, B, blocks, blocks + 1).repeat_interleave(32, 1)
    for size in (1e-3, 1e-6, 1e-30, 1e30):
        for q0 in (0.0, 40.0):
            print(f"kv8 zeros {fmt} {dtype} {nq}/{nkv}x{d} B {B} n {n} {order} {size} q {q0}", flush=True)
            check(fmt, dtype, nq, nkv, d, [blocks * 32 - n] * B, n, torch.where(zero, -1.0, 1.0), torch.where(zero, 0.0, size).double(), q0, room, close=True)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_values_that_a_row_does_not_see(fmt, dtype):
    """Siblings in a block behind the old ones; positions before a window that other rows still see."""
    n, lens = 5, [127, 255, 31]
    size = torch.ones(3, 260, dtype=torch.float64)
    for b, a in enumerate(lens):
        size[b, a + 1:a + n] = 2.0 ** 40
    sign = torch.ones(3, 260)
    for parents in ([[0, 0, 0, 0, 0]] * 3, [[0, 0, 1, 0, 3]] * 3):
        check(fmt, dtype, 8, 2, 64, lens, n, sign, size, 3.0, parents=parents)
    size = torch.ones(1, 300, dtype=torch.float64)
    size[0, :96] = 2.0 ** 50
    for window in (200, 202, 203):
        check(fmt, dtype, 8, 2, 128, [295], n, torch.ones(1, 300), size, 1.0, window=window)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_a_sequence_of_ever_larger_blocks(fmt):
    """The unit moves with every block that a wave meets, up and down; probabilities fall as values grow."""
    for step in (3, 5, 9, 12):
        blocks = 40
        at = torch.arange(blocks).repeat_interleave(32) // 4
        for e in (at, 9 - at, (at * 7) % 10):
            size = torch.exp2(e.double() * step)[None]
            check(fmt, torch.float32, 4, 2, 64, [blocks * 32 - 1], 1, torch.where(at[None] % 2 == 0, 1.0, -1.0), size, 24.0, room=8000)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("nq,nkv,d,B,n,blocks,room", PLANS + [(4, 2, 64, 1, 3, 40, 0), (6, 3, 128, 2, 2, 90, 0)])
def test_values_at_the_ends_of_the_range(fmt, dtype, nq, nkv, d, B, n, blocks, room):
    """Up to 2^127, the largest that the cache takes as finite, with every other block 2^30 smaller or not, and down to subnormal numbers, where results are
    rounded to multiples of 2^-149, or in bf16 of 2^-133.  Segments of one sequence, joined inside the launch or by a second one, among them."""
    for q0 in (0.0, 3.0):
        for top in (127, 124, 120, -100, -118, -126):
            for gap in (0, 30):
                if top - gap < -126:
                    continue
                print(f"kv8 ends {fmt} {dtype} {nq}/{nkv}x{d} B {B} n {n} 2^{top} - {gap} q {q0}", flush=True)
                large = large_blocks("mixed", B, blocks, blocks + 7).repeat_interleave(32, 1)
                size = torch.where(large, 2.0 ** top, 2.0 ** (top - gap)).double()
                check(fmt, dtype, nq, nkv, d, [blocks * 32 - n] * B, n, torch.where(large, -1.0, 1.0), size, q0, room, uniform=True,
                      least=2.0 ** -149 if dtype == torch.float32 else 2.0 ** -149 + 2.0 ** -134)
