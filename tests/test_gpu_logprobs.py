"""sssd_op_logprobs against 64 bits.  Ranks and ids have to be equal.  Bounds of the numbers, u = 2^-24: x = (z - M) / T goes through three roundings, exp2 of
x log2(e) (one more, and its own of 2u), so a term of S is off by (4 |x| + 2) u of itself; a chain of sums has at most 65 terms of a thread, 6 + 8 of its
workgroup and tiles / 64 + 6 of the row.  With E the mean over the distribution: log S by (4 E|x| + c) u and its own rounding, a log-probability by 3 |x| u and two roundings more,
the entropy by (4 E x^2 + (2 + 2 c) E|x| + 4 (E|x|)^2 + 4 E|x| + c) u and three roundings of its two parts."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2411_05894_amd import binding as sv

DEV = "cuda:0"
U = 2.0 ** -24


def want(z, tokens, n_top, temperature):
    z = z.double()
    order_z = torch.where(z.isnan(), -math.inf, z)
    order = torch.sort(order_z, dim=1, descending=True, stable=True)[1]
    place = torch.empty_like(order).scatter_(1, order, torch.arange(z.shape[1], device=DEV).expand(len(z), -1))
    x = (z - z.amax(1, keepdim=True)) / temperature
    p = torch.exp(x)
    s = p.sum(1, keepdim=True)
    p, rest = p / s, torch.where(x == x.amax(1, keepdim=True), 0.0, p).sum(1, keepdim=True)
    ties = (x == x.amax(1, keepdim=True)).sum(1, keepdim=True) - 1
    log_s = torch.log1p(rest + ties)                     # nearly certain rows keep their digits
    lp = x - log_s
    xx = torch.where(p > 0, x, 0.0)
    return dict(lp=lp, order=order, place=place, e1=(p * xx.abs()).sum(1), e2=(p * xx * xx).sum(1), log_s=log_s[:, 0],
                entropy=log_s[:, 0] - (p * xx).sum(1), x=x)


def check(z, tokens, n_top, temperature=1.0):
    rows, vocab = z.shape
    t = None if tokens is None else tokens.to(torch.int32)
    lp, ranks, entropy, ids, top = sv.sssd_op_logprobs(z, t, n_top, temperature)
    w = want(z, tokens, n_top, temperature)
    c = 65 + 6 + 8 + 6 + vocab // (2048 * 64) + 4

    def near(got, lp_want, x):
        bound = (4 * w["e1"][:, None] + c) * U + 3 * x.abs() * U + (lp_want.abs() + w["log_s"][:, None]) * 4 * U
        same = (got.double() == lp_want) | (got.isnan() & lp_want.isnan()) | ((got.double() - lp_want).abs() <= bound)
        # log-probabilities below float32's range are -infinity
        assert (same | (got == -math.inf) & (lp_want < -3.4e38)).all(), float(((got.double() - lp_want).abs() / bound).nan_to_num(0).max())
    if tokens is not None:
        there = (tokens >= 0) & (tokens < vocab)
        safe = tokens.clamp(0, vocab - 1).long()
        place = torch.gather(w["place"], 1, safe)
        assert torch.equal(ranks.long(), torch.where(there, place, -1))
        lw, xw = torch.gather(w["lp"], 1, safe), torch.gather(w["x"], 1, safe)
        near(torch.where(there, lp, 0.0), torch.where(there, lw, 0.0), torch.where(there, xw, 0.0).nan_to_num(0, 0, 0))
        assert (lp[~there] == -math.inf).all()
    if n_top:
        assert torch.equal(ids.long(), w["order"][:, :n_top])
        near(top, torch.gather(w["lp"], 1, w["order"][:, :n_top]), torch.gather(w["x"], 1, w["order"][:, :n_top]).nan_to_num(0, 0, 0))
    e1, e2 = w["e1"], w["e2"]
    bound = (4 * e2 + (2 + 2 * c) * e1 + 4 * e1 ** 2 + 4 * e1 + c) * U + 3 * (e1 + w["log_s"]) * U
    assert ((entropy.isnan() & w["entropy"].isnan()) | ((entropy.double() - w["entropy"]).abs() <= bound)).all()
    return lp, ranks, entropy, ids, top


def random_rows(rows, vocab, seed, dtype=torch.float32, spread=3.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g, device=DEV) * spread).to(dtype), torch.randint(0, vocab, (rows, 32), generator=g, device=DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 2), (3, 7), (2, 63), (5, 100), (4, 1000), (1, 1024), (7, 4097), (33, 2049), (2, 32001), (9, 128256), (3, 128257), (150, 16385),
                                        (600, 16391), (1, 300007), (2000, 5)])
def test_sizes(dtype, rows, vocab):
    z, tokens = random_rows(rows, vocab, rows + vocab, dtype)
    for m, n_top, temperature in ((1, 0, 1.0), (0, min(5, vocab), 1.0), (3, min(20, vocab), 0.7), (32, min(64, vocab), 1.9)):
        print(f"logprobs {dtype} {rows} {vocab} {m} {n_top}", flush=True)
        check(z, tokens[:, :m].contiguous() if m else None, n_top, temperature)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks_and_equal_logits(dtype):
    """Rows with most tokens masked, by -infinity or the type's lowest value; all equal; two values; ascending, descending; a row of nothing but the lowest value."""
    vocab = 20011
    z, tokens = random_rows(12, vocab, 5, dtype)
    low = torch.finfo(dtype).min
    z[0, 1:] = -math.inf
    z[1, :-1] = -math.inf
    z[2, ::2] = -math.inf
    z[3, 7:] = low
    z[4] = 1.25
    z[5] = low
    z[6] = torch.where(torch.arange(vocab, device=DEV) % 3 == 0, 2.0, 1.0).to(dtype)
    z[7] = torch.linspace(-30, 30, vocab, device=DEV).to(dtype)
    z[8] = torch.linspace(30, -30, vocab, device=DEV).to(dtype)
    z[9] = torch.where(torch.arange(vocab, device=DEV) % 2 == 0, 0.0, -0.0).to(dtype)      # equal, whatever their sign
    z[10] = -math.inf
    z[10, 500:503] = 3.0
    z[11, 100:] = z[11, :1]
    tokens[:, 0], tokens[:, 1], tokens[:, 2] = 0, vocab - 1, 501
    for n_top in (1, 5, 64):
        check(z, tokens, n_top)
        check(z[:, 1:], tokens.clamp(max=vocab - 2), n_top)       # rows begin elsewhere


def test_rows_without_a_distribution():
    """No finite logit, an infinite one, one that is no number: no numbers in that row, the others as alone; order and ranks all the same."""
    z, tokens = random_rows(7, 9000, 6)
    clean = sv.sssd_op_logprobs(z, tokens.to(torch.int32), 5)
    z[1] = -math.inf
    z[2, 77] = math.inf
    z[3, 4000] = math.nan
    z[4] = math.nan
    z[5, 5] = z[5, 8000] = math.inf
    tokens[3, 0], tokens[2, 0], tokens[5, 0] = 4000, 77, 8000
    lp, ranks, entropy, ids, top = got = sv.sssd_op_logprobs(z, tokens.to(torch.int32), 5)
    w = want(z, tokens, 5, 1.0)
    for r in range(1, 6):
        assert lp[r].isnan().all() and entropy[r].isnan() and top[r].isnan().all()
        assert torch.equal(ids[r].long(), w["order"][r, :5]) and torch.equal(ranks[r].long(), w["place"][r][tokens[r]])
    for r in (0, 6):
        assert all(torch.equal(a[r], b[r]) for a, b in zip(got, clean))
    lp = sv.sssd_op_logprobs(z, torch.tensor([[-1, 9000, 2 ** 31 - 1, -2 ** 31]] * 7, dtype=torch.int32, device=DEV))
    assert (lp[0] == -math.inf).all() and (lp[1] == -1).all()


def test_nearly_certain_rows_keep_their_digits():
    """log p = -log1p(s) of the likeliest token for s down to 1e-30, to a few units of its own last place."""
    vocab = 5000
    z = torch.full((30, vocab), -200.0, device=DEV)
    z[:, 123] = 0.0
    gap = torch.linspace(0.1, 69.0, 30, device=DEV)
    z[:, 4000] = -gap
    lp, ranks, entropy, ids, top = sv.sssd_op_logprobs(z, torch.full((30, 1), 123, dtype=torch.int32, device=DEV), 2)
    s = torch.exp(-gap.double())
    assert ((lp[:, 0].double() + torch.log1p(s)).abs() <= torch.log1p(s) * (4 * gap + 8) * U).all()
    exact = torch.log1p(s) + s / (1 + s) * gap.double()
    assert ((entropy.double() - exact).abs() <= exact * (8 * gap + 20) * U).all()
    assert (ids == torch.tensor([123, 4000], device=DEV)).all()


@pytest.mark.parametrize("temperature", [1e-30, 1e-3, 50.0, 1e30])
def test_temperatures(temperature):
    z, tokens = random_rows(5, 3001, 8)
    check(z, tokens, 7, temperature)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_apart_and_unaligned(dtype):
    """Rows with others between them, that begin off 16 bytes, all the same one."""
    z, tokens = random_rows(6, 5003, 9, dtype)
    for view in (z[::2], z[:, 1:], z[:, 3:4000], z[1::3, 5:70], z[:1].expand(6, -1), z.flatten()[2:2 + 4 * 6001].view(4, 6001)):
        t = tokens[:len(view)].clamp(max=view.shape[1] - 1)
        a, b = sv.sssd_op_logprobs(view, t.to(torch.int32), 9), check(view.contiguous(), t, 9)
        check(view, t, 9)
        assert torch.equal(a[1], b[1]) and torch.equal(a[3], b[3])


def test_far_rows():
    """Rows beyond 2^31 bytes."""
    vocab, rows = 128256, 9000
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device=DEV)
    part, tokens = random_rows(3, vocab, 10, torch.bfloat16)
    z[-3:] = part
    all_tokens = torch.zeros(rows, 1, dtype=torch.int32, device=DEV)
    all_tokens[-3:] = tokens[:, :1].int()
    lp, ranks, entropy, ids, top = sv.sssd_op_logprobs(z, all_tokens, 3)
    assert torch.equal(ids[:2].cpu(), torch.tensor([[0, 1, 2]] * 2, dtype=torch.int32))
    w = want(part, tokens[:, :1], 3, 1.0)
    assert torch.equal(ids[-3:].long(), w["order"][:, :3]) and torch.equal(ranks[-3:].long(), torch.gather(w["place"], 1, tokens[:, :1]))


def test_replays_and_another_stream():
    z, tokens = random_rows(9, 32000, 11)
    t = tokens[:, :2].to(torch.int32).contiguous()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        sv.sssd_op_logprobs(z, t, 5)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = sv.sssd_op_logprobs(z, t, 5)
    for turn in range(4):
        z.copy_(random_rows(9, 32000, 20 + turn)[0])
        graph.replay()
        eager = sv.sssd_op_logprobs(z, t, 5)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(7, 9001), (1100, 9001)])
def test_logits_far_from_zero(dtype, rows, vocab):
    """Rows about one large number, and rows that climb or fall from one to another, so that exponents are taken in either way within a row."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    tokens = torch.randint(0, vocab, (rows, 3), generator=g, device=DEV)
    up = torch.arange(vocab, device=DEV) / vocab
    starts = torch.tensor([-1e6, 1e6, 100.0, -7e5, 7.3e5, -3e7, -2e38], device=DEV).repeat(rows // 7 + 1)[:rows, None]
    ends = torch.tensor([1e6, -1e6, -1e4, -7e5, 7.2e5, 1e3, 2e38], device=DEV).repeat(rows // 7 + 1)[:rows, None]
    z = (starts * (1 - up) + ends * up + torch.randn(rows, vocab, generator=g, device=DEV) * 3).to(dtype)
    for temperature in (1.0, 1e-3, 1e4, 1e-20):
        check(z, tokens, 5, temperature)
